// Sums of the table's gradient over the workgroups that formed parts of it.
#include "kernels.h"
#include "score_attn.h"

namespace pb {
namespace {

// dtable[bucket][head] from the workgroups' parts, a wave each, in fp64.
__global__ __launch_bounds__(64) void score_dtable_sum(ScoreArgs a, int parts) {
  const int h = blockIdx.x % a.heads, n = blockIdx.x / a.heads;
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += 64)
    s += (double)a.bias_part[((size_t)i * a.heads + h) * a.buckets + n];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x == 0) a.dtable[n * a.heads + h] = (float)s * (a.dscale == 0.f ? 0.f : 1.f);
}

}  // namespace

void launch_score_dtable_sum(const ScoreArgs& a, int parts, hipStream_t s) {
  score_dtable_sum<<<(unsigned)(a.heads * a.buckets), 64, 0, s>>>(a, parts);
}
}  // namespace pb

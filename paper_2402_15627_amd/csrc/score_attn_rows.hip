// Attention with terms in its scores, row by row from the definition, and the learned
// table's gradient.
#include "kernels.h"
#include "score_attn.h"

namespace pb {
namespace {

using namespace score;

// One row a wave; rows r of (batch, head, position).
template <typename T, int D, int WHAT>
__global__ __launch_bounds__(256) void score_rows(ScoreArgs a, long long rows) {
  const long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (r >= rows) return;
  const int S = WHAT == 2 ? a.seq_k : a.seq_q, H = WHAT == 2 ? a.kv_heads : a.heads;
  const int i = (int)(r % S), h = (int)(r / S % H), b = (int)(r / S / H);
  if constexpr (WHAT == 0) fwd_row<T, D>(a, b, h, i, lane);
  else if constexpr (WHAT == 1) dq_row<T, D>(a, b, h, i, lane);
  else dkdv_row<T, D>(a, b, h, i, lane);
}

// The table's gradient: sums of P (dP - delta) by bucket.  A workgroup has
// kScoreBiasRows queries of a head, a row a wave at a time, and walks its keys twice:
// for delta = sum of P dP, from unrounded values, and for the sums.  Each lane adds to
// its own place of each bucket, so no order of additions is left to chance.
template <typename T, int D>
__global__ __launch_bounds__(256) void score_dtable(ScoreArgs a, int blocks) {
  extern __shared__ float acc[];  // [wave][bucket][lane]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int blk = blockIdx.x % blocks, h = blockIdx.x / blocks % a.heads;
  const int b = blockIdx.x / blocks / a.heads, kvh = h / a.group;
  float* mine = acc + wave * a.buckets * 64 + lane;
  for (int n = 0; n < a.buckets; ++n) mine[n * 64] = 0.f;
  const int i_end = min(a.seq_q, (blk + 1) * kScoreBiasRows);
  for (int i = blk * kScoreBiasRows + wave; i < i_end; i += 4) {
    const int p = i + a.seq_k - a.seq_q;
    const Bounds d = bounds_of(a, b, p);
    const int first = window_first(a, d, p), last = window_last(a, d, p);
    const T *qr = q_row<T, D>(a, b, i, h), *gr = do_row<T, D>(a, b, i, h);
    const float L = a.lse[lse_at(a, b, h, i)];
    const int begin = d.pe > d.ds ? d.ds : first, end = L == kNegInf ? 0 : max(last + 1, d.pe);
    float delta = 0.f, sum = 0.f;
    for (int pass = 0; pass < 2; ++pass) {
      for (int j = begin + lane; j < end; j += 64) {
        if (!(j < d.pe || (j >= first && j <= last))) continue;
        const Pair x = pair_of<T, D>(a, qr, gr, kv_row<T, D>(a, a.k, b, j, kvh),
                                     kv_row<T, D>(a, a.v, b, j, kvh), h, p - j, L, delta);
        if (pass) mine[bucket_of(a, p - j) * 64] += x.dz;
        else sum += x.dz;
      }
      if (!pass) delta = wave_sum(sum);
    }
  }
  __syncthreads();
  float* out = a.bias_part + (((size_t)b * blocks + blk) * a.heads + h) * a.buckets;
  for (int n = wave; n < a.buckets; n += 4) {
    float s = 0.f;
    for (int w = 0; w < 4; ++w) s += acc[(w * a.buckets + n) * 64 + lane];
    s = wave_sum(s);
    if (lane == 0) out[n] = s;
  }
}
// dtable[bucket][head] from the workgroups' parts, a wave each, in fp64.
__global__ __launch_bounds__(64) void score_dtable_sum(ScoreArgs a, int parts) {
  const int h = blockIdx.x % a.heads, n = blockIdx.x / a.heads;
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += 64)
    s += (double)a.bias_part[((size_t)i * a.heads + h) * a.buckets + n];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
  if (threadIdx.x == 0) a.dtable[n * a.heads + h] = (float)s;
}

template <typename T, int D, int WHAT>
void rows_td(const ScoreArgs& a, hipStream_t s) {
  const long long rows = WHAT == 2 ? (long long)a.batch * a.seq_k * a.kv_heads
                                   : (long long)a.batch * a.seq_q * a.heads;
  score_rows<T, D, WHAT><<<(unsigned)((rows + 3) / 4), 256, 0, s>>>(a, rows);
}
template <typename T, int D>
void bwd_td(const ScoreArgs& a, hipStream_t s) {
  rows_td<T, D, 1>(a, s);
  rows_td<T, D, 2>(a, s);
  if (!a.dtable) return;
  const int blocks = (a.seq_q + kScoreBiasRows - 1) / kScoreBiasRows;
  score_dtable<T, D><<<(unsigned)(blocks * a.heads * a.batch), 256,
                       (size_t)4 * a.buckets * 64 * 4, s>>>(a, blocks);
  launch_score_dtable_sum(a, blocks * a.batch, s);
}
#define PB_BY_TYPE(fn, ...)                                   \
  do {                                                        \
    if (dt == Dt::BF16) {                                     \
      if (head_dim == 64) fn<bf16, 64>(__VA_ARGS__);          \
      else if (head_dim == 96) fn<bf16, 96>(__VA_ARGS__);     \
      else fn<bf16, 128>(__VA_ARGS__);                        \
    } else {                                                  \
      if (head_dim == 64) fn<float, 64>(__VA_ARGS__);         \
      else if (head_dim == 96) fn<float, 96>(__VA_ARGS__);    \
      else fn<float, 128>(__VA_ARGS__);                       \
    }                                                         \
  } while (0)
template <typename T, int D>
void fwd_td(const ScoreArgs& a, hipStream_t s) {
  rows_td<T, D, 0>(a, s);
}

}  // namespace

void launch_score_dtable_sum(const ScoreArgs& a, int parts, hipStream_t s) {
  score_dtable_sum<<<(unsigned)(a.heads * a.buckets), 64, 0, s>>>(a, parts);
}
void launch_score_forward(Dt dt, int head_dim, const ScoreArgs& a, hipStream_t s) {
  PB_BY_TYPE(fwd_td, a, s);
}
void launch_score_backward(Dt dt, int head_dim, const ScoreArgs& a, hipStream_t s) {
  PB_BY_TYPE(bwd_td, a, s);
}

}  // namespace pb

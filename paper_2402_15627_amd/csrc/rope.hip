// Rotary positions over the heads of up to kRopeMaxTensors tensors (Q and K of
// the packed in-projection output, or their gradients).
//
//   (y_a, y_b) = m (x_a cos t - x_b sin t, x_b cos t + x_a sin t)
//
// for the pair i of a head, (a, b) = (i, i + r/2) or (2 i, 2 i + 1), with t the
// token's position times the pair's frequency and m the magnitude.  The gradient
// is the transposed map: t negated, the same m.
//
// A position may be far out (millions), where t in fp32 would be off by whole
// radians: the angle is formed in turns, position times f_i / 2 pi in fp64, and
// reduced to [-1/2, 1/2] there (error of the fp64 product 2^-53 of all turns, 1e-10 at a
// million).  Sine and cosine are fp32's of its leading 24 bits, turned on by the bits
// behind them to first order (without, they are off by up to 1.12e-7, 3.2e-8 rms).
//
// HBM-bound: every element is read and written once (2 e bytes) for 3 operations: 8192
// tokens x 80 heads x 128 in bf16 61.5 us, 5.5 TB/s; below a megabyte or two a launch's
// latency (four tokens x 80 heads 4 us, 8 a call back to back).
// A workgroup takes some tokens by some heads of one tensor, up to kItems 16-byte
// pieces a thread (a pair of pieces r/2 apart in the half layout).  It first
// issues all its loads, then forms the cosines and sines of its tokens into LDS
// once for all heads, so the loads cover the trigonometry, then rotates.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace pb {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kItems = 4;         // items a thread holds
constexpr int kTrigPairs = 2048;  // (token, pair) cosines and sines in LDS: 16 KB

// V consecutive elements as fp32, elementwise (VEC = false) or as one 16-byte access.
// The stores bypass the caches' retention (nothing here reads them again: 74 -> 66 us for
// 8192 tokens x 80 heads x 128), and with STREAM the loads too.
template <typename T, int V, bool VEC, bool STREAM>
PB_DEV void load_v(const T* p, float* v) {
  if constexpr (VEC) {
    static_assert(V * sizeof(T) == 16, "one access");
    u32x4 w;
    if constexpr (STREAM) w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < V; ++e)
      v[e] = V == 4 ? __uint_as_float(w[e & 3]) : e & 1 ? hi_bf(w[e >> 1 & 3]) : lo_bf(w[e >> 1 & 3]);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = load1<T>(p + e);
  }
}
template <typename T, int V, bool VEC>
PB_DEV void store_v(T* p, const float* v) {
  if constexpr (VEC) {
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = V == 4 ? __float_as_uint(v[e]) : pack_bf2(v[2 * e % V], v[(2 * e + 1) % V]);
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(p));
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) p[e] = (T)v[e];
  }
}

// V: elements of a piece.  Half layout: an item is the pieces at i and i + r/2, V
// pairs; adjacent pairs: an item is one piece, V / 2 pairs.  Items past the
// rotated part (only where the output is another buffer) copy a piece.
template <typename T, int V, bool VEC, bool ADJ, bool STREAM>
__global__ __launch_bounds__(kRopeThreads) void rope_kernel(RopeArgs a, int tile_tokens,
                                                            int tile_heads, int slices) {
  __shared__ float2 trig[kTrigPairs];
  int part = 0, slice = blockIdx.y;
  while (slice >= slices) slice -= slices, ++part;
  const int heads = min(tile_heads, a.heads[part] - slice * tile_heads);
  if (heads <= 0) return;  // the whole workgroup: a tensor of fewer heads
  const long long t0 = (long long)blockIdx.x * tile_tokens;
  const int tokens = (int)min((long long)tile_tokens, a.tokens - t0);
  const T* in = (const T*)a.in[part];  // may be out: an item is read before it is written
  T* out = (T*)a.out[part];
  const long long ld_in = a.ld_in[part], ld_out = a.ld_out[part];
  const int d = a.head_dim, half = a.rot_dim / 2;
  const int rot_items = ADJ ? a.rot_dim / V : half / V;
  const int items = rot_items + (a.copy_rest[part] ? (d - a.rot_dim) / V : 0);
  const int total = tokens * heads * items;

  float x[kItems][2 * V];
  long long at_out[kItems];
  int pair[kItems];  // first pair of the item in trig, -1: copied, -2: none
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const int i = threadIdx.x + k * kRopeThreads;
    pair[k] = -2;
    if (i >= total) continue;
    const int th = i / items, it = i - th * items;
    const int t = th / heads, h = slice * tile_heads + th - t * heads;
    const bool rot = it < rot_items;
    const int e = rot ? it * V : a.rot_dim + (it - rot_items) * V;
    const T* p = in + (t0 + t) * ld_in + (long long)h * d + e;
    load_v<T, V, VEC, STREAM>(p, x[k]);
    if (!ADJ && rot) load_v<T, V, VEC, STREAM>(p + half, x[k] + V);
    at_out[k] = (t0 + t) * ld_out + (long long)h * d + e;
    pair[k] = rot ? t * half + (ADJ ? e / 2 : e) : -1;
  }

  for (int i = threadIdx.x; i < tokens * half; i += kRopeThreads) {
    const int t = i / half, f = i - t * half;
    const long long pos = a.pos ? a.pos[t0 + t] : (long long)((unsigned)(t0 + t) % (unsigned)a.seq);
    const double turns = (double)pos * a.turns[f], half_turns = 2.0 * (turns - rint(turns));
    const float lead = (float)half_turns;
    const float rest = (float)(half_turns - (double)lead) * 3.14159265f;
    float s0, c0;
    sincospif(lead, &s0, &c0);
    const float s = __builtin_fmaf(c0, rest, s0), c = __builtin_fmaf(-s0, rest, c0);
    trig[i] = make_float2(c * a.magnitude, (a.backward ? -s : s) * a.magnitude);
  }
  __syncthreads();

#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    if (pair[k] == -2) continue;
    T* p = out + at_out[k];
    if (pair[k] == -1) {
      store_v<T, V, VEC>(p, x[k]);
      continue;
    }
    float y[2 * V];
    if constexpr (ADJ) {
#pragma unroll
      for (int e = 0; e < V; e += 2) {
        const float2 cs = trig[pair[k] + e / 2];
        y[e] = x[k][e] * cs.x - x[k][e + 1] * cs.y;
        y[e + 1] = x[k][e + 1] * cs.x + x[k][e] * cs.y;
      }
      store_v<T, V, VEC>(p, y);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 cs = trig[pair[k] + e];
        y[e] = x[k][e] * cs.x - x[k][V + e] * cs.y;
        y[V + e] = x[k][V + e] * cs.x + x[k][e] * cs.y;
      }
      store_v<T, V, VEC>(p, y);
      store_v<T, V, VEC>(p + half, y + V);
    }
  }
}

template <typename T, int V, bool VEC, bool ADJ, bool STREAM>
void run(const RopeArgs& a, hipStream_t s) {
  const int half = a.rot_dim / 2;
  const int items = (ADJ ? a.rot_dim / V : half / V) + (a.head_dim - a.rot_dim) / V;
  int most_heads = 0;
  long long all = 0;
  for (int i = 0; i < a.n; ++i) {
    most_heads = std::max(most_heads, a.heads[i]);
    all += a.tokens * a.heads[i] * items;
  }
  // items of a workgroup: all that its threads can hold, fewer while that leaves
  // CUs without any
  const int most = kItems * kRopeThreads;
  const int want = (int)std::min<long long>(most, std::max<long long>(kRopeThreads, all / 512));
  const int tile_heads = std::min(most_heads, std::max(1, want / items));
  const int tile_tokens =
      std::max(1, std::min(want / (tile_heads * items), kTrigPairs / half));
  const int slices = (most_heads + tile_heads - 1) / tile_heads;
  const dim3 grid((unsigned)((a.tokens + tile_tokens - 1) / tile_tokens), slices * a.n);
  rope_kernel<T, V, VEC, ADJ, STREAM><<<grid, kRopeThreads, 0, s>>>(a, tile_tokens, tile_heads, slices);
}

template <typename T>
void run_type(const RopeArgs& a, bool interleaved, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  // 16-byte pieces: every piece of every head starts at a multiple of 16 bytes
  bool vec = a.head_dim % V == 0 && (interleaved ? a.rot_dim : a.rot_dim / 2) % V == 0;
  for (int i = 0; i < a.n; ++i)
    vec = vec && (uintptr_t)a.in[i] % 16 == 0 && (uintptr_t)a.out[i] % 16 == 0 &&
          a.ld_in[i] % V == 0 && a.ld_out[i] % V == 0;
  // Streaming loads where a wave's accesses cover whole 128-byte lines: adjacent pairs, or
  // half heads that are whole lines (8192 tokens x 80 heads of 128, all rotated: 66 -> 63
  // us and 69 -> 66; half heads of 64 bytes, 8192 x 40 with half of 128 rotated, 35 -> 37,
  // since a line's other half is then fetched again).
  const bool lines = a.rot_dim / 2 * sizeof(T) % 128 == 0;
  if (interleaved) {
    if (vec) run<T, V, true, true, true>(a, s);
    else run<T, 2, false, true, false>(a, s);
  } else {
    if (vec && lines) run<T, V, true, false, true>(a, s);
    else if (vec) run<T, V, true, false, false>(a, s);
    else run<T, 1, false, false, false>(a, s);
  }
}

}  // namespace

void launch_rope(Dt dt, const RopeArgs& a, bool interleaved, hipStream_t s) {
  if (dt == Dt::BF16) run_type<bf16>(a, interleaved, s);
  else run_type<float>(a, interleaved, s);
}

}  // namespace pb

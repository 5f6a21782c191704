// What the bf16 kernels of attention with terms in its scores share beside
// score_attn.h: rows of several heads in a tile, the key tiles that a block of rows
// visits, the cap on scores in base 2, the biases of a tile.
#pragma once

#include "attn_tiles.h"
#include "score_attn.h"

namespace pb {
namespace {

using score::Bounds;
using score::bounds_of;
using score::window_first;
using score::window_last;

// A block's rows are (position, head) pairs of the `pack` heads that share a key head
// (a part of them where there are more than eight): row r is query r / pack of head
// r mod pack.  Keys and values are then read once for all of them, and the gradients of
// shared heads are sums within a workgroup.
struct Packed {
  int pack;       // heads of a block
  uint32_t magic; // ceil(2^32 / pack): rows below 2^29 divide by a high product
  PB_DEV explicit Packed(int n) : pack(n), magic((uint32_t)((0x100000000ull + n - 1) / n)) {}
  PB_DEV int pos(int r) const { return pack == 1 ? r : (int)__umulhi((uint32_t)r, magic); }
};

// What the bf16 values x of pair leave of u and v, in bf16: 16 bits of each in both.  (A dot
// product with (-1, 0) or (0, -1): the difference is exact, in one instruction.  The
// constants come in registers: as an immediate, (-1, 0) is read as fp32's -1, which is (0, -1).)
PB_DEV bf16x2 rest_of(bf16x2 pair, float u, float v) {
  uint32_t first = 0xbf80u, second = 0xbf800000u;
  asm("" : "+s"(first), "+s"(second));
  return bf16x2{
      (bf16)__builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, first), u, false),
      (bf16)__builtin_amdgcn_fdot2_f32_bf16(pair, __builtin_bit_cast(bf16x2, second), v, false)};
}

// A row of D features in the merges: kLanes lanes with kChunks times 8 features each, chunk
// c of lane l from 8 (l + c kLanes) on.  The lanes divide a wave's, so a row lies in one
// wave, which alone writes it: merged, or where any of it is not finite, by the definition.
template <int D>
struct MergeLanes {
  static constexpr int kLanes = D == 96 ? 4 : D / 8, kChunks = D / 8 / kLanes;
  static PB_DEV int at(int l, int c) { return 8 * (l + c * kLanes); }
  static PB_DEV bool any(bool x) {  // of the row's lanes
    const unsigned long long all = __builtin_amdgcn_ballot_w64(x);
    const int first = (int)(threadIdx.x & 63) / kLanes * kLanes;
    return (all >> first) & ((1ull << kLanes) - 1);
  }
};

PB_DEV int wave_imin(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}
PB_DEV int wave_imax(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = max(v, __shfl_xor(v, o, 64));
  return __builtin_amdgcn_readfirstlane(v);
}

// Keys of one row: first .. first + len - 1 by the window, pfirst .. pfirst + plen - 1 by
// the prefix.
struct RowKeys {
  int first, len, pfirst, plen;
  // bit k: whether key k0 + k is seen
  static PB_DEV uint64_t below(int n) { return n >= 64 ? ~0ull : n <= 0 ? 0 : (1ull << n) - 1; }
  PB_DEV uint64_t bits(int k0) const {
    return (below(first - k0 + len) & ~below(first - k0)) |
           (below(pfirst - k0 + plen) & ~below(pfirst - k0));
  }
};
PB_DEV RowKeys row_keys(const ScoreArgs& a, int b, int p) {
  const Bounds d = bounds_of(a, b, p);
  const int first = window_first(a, d, p);
  return RowKeys{first, d.de > d.ds ? window_last(a, d, p) - first + 1 : 0, d.ds, d.pe - d.ds};
}

// A block's n tiles shared out over at most `most` chunks of `least` tiles or more.
struct Share {
  int size, used;  // tiles of a chunk, chunks
  PB_DEV Share(int n, int most, int least)
      : size(max((n + most - 1) / most, most > 1 ? least : 1)), used((n + size - 1) / size) {}
};

// The key tiles (of TL) that positions p0 .. p1 of a batch row visit: up to two runs,
// the prefixes' and the windows', in ascending order.  lo .. hi: the keys that any of
// them sees, and all between.
struct KeyTiles {
  int t0, n0, t1, n;  // tile i is t0 + i below n0, then t1 + i - n0; n in all
  int lo, hi;
  PB_DEV int tile(int i) const { return i < n0 ? t0 + i : t1 + i - n0; }
};
template <int TL>
PB_DEV KeyTiles key_tiles(const ScoreArgs& a, int b, int p0, int p1, int lane) {
  int w0 = 0x7fffffff, w1 = -1, x0 = 0x7fffffff, x1 = -1;
  if (!a.docs && !a.prefix) {
    const Bounds d{0, a.seq_k, 0};
    w0 = window_first(a, d, p0), w1 = window_last(a, d, p1);
  } else {
    for (int p = p0 + lane; p <= p1; p += 64) {
      const RowKeys k = row_keys(a, b, p);
      if (k.len > 0) w0 = min(w0, k.first), w1 = max(w1, k.first + k.len - 1);
      if (k.plen > 0) x0 = min(x0, k.pfirst), x1 = max(x1, k.pfirst + k.plen - 1);
    }
    w0 = wave_imin(w0), w1 = wave_imax(w1), x0 = wave_imin(x0), x1 = wave_imax(x1);
  }
  KeyTiles k{0, 0, 0, 0, min(w0, x0), max(w1, x1)};
  int wa = w0 / TL, wb = w1 < 0 ? -1 : w1 / TL, xa = x0 / TL, xb = x1 < 0 ? -1 : x1 / TL;
  if (wb < 0 || (xb >= 0 && xa < wa)) {  // the run that begins first comes first
    const int ta = wa, tb = wb;
    wa = xa, wb = xb, xa = ta, xb = tb;
  }
  if (wb < 0) return k;
  k.t0 = wa;
  if (xb < 0 || xa <= wb + 1) {
    k.n0 = max(wb, xb) - wa + 1;
    k.n = k.n0;
  } else {
    k.n0 = wb - wa + 1;
    k.t1 = xa;
    k.n = k.n0 + xb - xa + 1;
  }
  return k;
}

// t = tanh(scale u / cap); the score is cap t, what the cap leaves of its gradient 1 - t^2, or
// 4 w (1 - w) with w = 1 / (1 + e^(2|x|)) beyond 1/2, where 1 - t^2 would lose what t is
// rounded to (a tenth of itself at |x| = 7.5).
// Tiles differ in how far their scores go, so a wave looks at its largest |x| = |scale u /
// cap| first: to 1/8 three terms in x^2 are good to 2^-24, to 1/2 five, beyond 1 - 2 / (1 +
// e^(2|x|)) takes over from 1/2 on.  (An exponential and a reciprocal take eight
// instructions' time each.)  What follows takes t: the product with cap is part of the
// exponential's or of the bias's fused multiply.
struct Cap {
  float k, small;  // scale / cap, and |u| of x = 1/8
  float a1, a2, b1, b2, b3, b4;  // (k: the first coefficient of either)
  float top;       // cap times a unit (log2 e for base 2)
  PB_DEV Cap(float scale, float cap, float unit = kLog2e) {
    k = scale / cap, small = 0.125f / k;
    a1 = kA1 * k * (k * k), a2 = kA2 * k * (k * k) * (k * k);
    top = cap * unit;
    const float k3 = k * (k * k), k5 = k3 * (k * k), k7 = k5 * (k * k), k9 = k7 * (k * k);
    b1 = kB1 * k3, b2 = kB2 * k5, b3 = kB3 * k7, b4 = kB4 * k9;
    for (float* x : {&k, &small, &a1, &a2, &b1, &b2, &b3, &b4, &top})  // scalar registers
      *x = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(*x)));
  }
  // tanh(x) / x in x^2 of least largest relative error (by Remez exchange): 7e-9 to 1/8,
  // 1.4e-8 to 1/2; in fp32 4.3e-8 and 6.5e-8
  static constexpr float kA1 = -0.33332599f, kA2 = 0.13207752f;  // (1 + ..)
  static constexpr float kB1 = -0.33333069f, kB2 = 0.13324779f, kB3 = -0.052986075f,
                         kB4 = 0.017135007f;
  PB_DEV float near(float u) const {
    const float w = u * u;
    return u * fmaf(fmaf(a2, w, a1), w, k);
  }
  PB_DEV float half(float u) const {
    const float w = u * u;
    return u * fmaf(fmaf(fmaf(fmaf(b4, w, b3), w, b2), w, b1), w, k);
  }
  static PB_DEV float slope(float t) { return fmaf(-t, t, 1.f); }
  // d: the slope
  PB_DEV float any(float u, float& d) const {
    const float x = u * k;
    const float e = __builtin_amdgcn_exp2f(2.f * kLog2e * fabsf(x));
    const float w = __builtin_amdgcn_rcpf(1.f + e), t = fmaf(-2.f, w, 1.f), y = half(u);
    const bool in = fabsf(x) <= 0.5f;
    d = in ? slope(y) : 4.f * fmaf(-w, w, w);
    return in ? y : __builtin_copysignf(t, x);
  }
  // of some of a wave's products, by the largest of them in any lane; slopes: f(i, e, slope
  // of s[i][e])
  template <typename V, int N>
  PB_DEV void apply(V (&s)[N]) const {
    apply(s, [](int, int, float) {});
  }
  template <typename V, int N, typename F>
  PB_DEV void apply(V (&s)[N], F f) const {
    constexpr int W = sizeof(V) / 4;
    float largest = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int e = 0; e < W; ++e) largest = fmaxf(largest, fabsf(s[i][e]));
    if (!__builtin_amdgcn_ballot_w64(largest > small)) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) s[i][e] = near(s[i][e]), f(i, e, slope(s[i][e]));
    } else if (!__builtin_amdgcn_ballot_w64(largest > 4.f * small)) {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) s[i][e] = half(s[i][e]), f(i, e, slope(s[i][e]));
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < W; ++e) {
          float d;
          s[i][e] = any(s[i][e], d);
          f(i, e, d);
        }
    }
  }
};

// Biases of learned buckets.  A tile of NP positions and NK keys has NP + NK -
// 1 distances: where they span buckets, the workgroup writes the bias of each (for each
// of the block's heads) into LDS a tile ahead, key after key in ascending order, so that
// a lane reads runs of neighbours; beyond the last bucket's first distance one value
// does for a tile.  Bytes: the table of the block's heads, the first distances, the
// buckets of distances below kMap, two tiles' biases.
struct BiasLds {
  static constexpr int kMap = kScoreMap;
  int stride;  // floats of a head's biases in a tile
  int tab, first, map, tile0, bytes;
  __host__ __device__ BiasLds(int at, int buckets, int pack, int positions, int keys) {
    stride = positions + keys;  // (one spare: an odd stride for even sizes)
    tab = at;
    first = tab + 4 * buckets * pack;
    map = first + 4 * kScoreMaxBuckets;
    tile0 = map + kMap;
    bytes = tile0 + 8 * stride * pack;
  }
  PB_DEV int tile(int buf, int pack) const { return tile0 + buf * 4 * stride * pack; }
};
// Tables of a workgroup (its first barrier comes after): heads h0 .. h0 + pack - 1, times a
// unit.
PB_DEV void bias_prologue(const ScoreArgs& a, const BiasLds& l, unsigned char* smem, int h0,
                          int pack, int tid, int threads, float unit = kLog2e) {
  float* tab = (float*)(smem + l.tab);
  for (int x = tid; x < a.buckets * pack; x += threads) {
    tab[x] = score::bias_value(a.table[(size_t)(x / pack) * a.heads + h0 + x % pack]) * unit;
  }
  int* first = (int*)(smem + l.first);
  if (tid < a.side) first[tid] = a.first[tid];
  for (int x = tid; x < kScoreMap / 4; x += threads) ((uint32_t*)(smem + l.map))[x] = a.map[x];
}
PB_DEV int bias_search(const int* first, int side, int d) {
  int lo = 0, hi = side - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= d) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
PB_DEV int bias_bucket(const ScoreArgs& a, const BiasLds& l, const unsigned char* smem, int n) {
  const int d = a.causal ? max(n, 0) : abs(n);
  const int k = d < BiasLds::kMap ? smem[l.map + d]
                                  : bias_search((const int*)(smem + l.first), a.side, d);
  return k + (!a.causal && n < 0 ? a.side : 0);
}
// The bucket of every distance n0 .. n1, or -1 where it is not known to be one.
PB_DEV int bias_uniform(const ScoreArgs& a, int last, int n0, int n1) {
  if (n0 >= last) return a.side - 1;
  if (a.causal) return n1 <= 0 ? 0 : -1;
  return n1 <= -last ? 2 * a.side - 1 : -1;
}
// Biases of a tile: entry x of a head is of distance top - x.
PB_DEV void bias_tile(const ScoreArgs& a, const BiasLds& l, unsigned char* smem, int buf, int pack,
                      int top, int tid, int threads) {
  float* out = (float*)(smem + l.tile(buf, pack));
  const float* tab = (const float*)(smem + l.tab);
  for (int x = tid; x < l.stride; x += threads) {
    const int k = bias_bucket(a, l, smem, top - x);
    for (int h = 0; h < pack; ++h) out[h * l.stride + x] = tab[k * pack + h];
  }
}

}  // namespace
}  // namespace pb

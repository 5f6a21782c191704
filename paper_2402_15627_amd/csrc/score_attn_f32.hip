// Attention with terms in its scores in fp32, forward and backward, on
// v_mfma_f32_16x16x4_f32.  The layout is that of attn_f32.hip: a workgroup of four waves
// (eight in a backward of long rows and few workgroups) has 16 rows (queries of the heads
// that share a key head, see Packed; or keys) and walks tiles of 16 of the other side, its
// waves in turn; everything is computed transposed, so that a lane owns one row and the
// probabilities leave the score accumulators in the order in which the next product
// contracts them; fragments go from global memory to registers, and the waves' parts are
// merged through LDS.
//
// Scores, with their terms, are natural logarithms here and turn to base 2 in the
// exponential, with the roundings of the products with log2 e added back.  The row term is
// delta = sum of dO O.  The table's gradient comes out of the dQ role: each lane adds dz to a
// place of its own for each bucket.  Its terms cancel (a row's sum to zero), so with a table
// that role goes over its tiles twice, first for the sums of P and of P dP: P is over its own
// sum then and delta what the same products give, and what lse and o are rounded to drops
// out (the table's gradient at 1447 tokens, 12 heads over 3 x 64, window 2 and a prefix: 2e-6
// off -> 4e-7; 128 tokens, 4 x 64: 19.2 us -> 20.2).
//
// A workgroup with a non-finite result computes its rows again by the definition, which
// reads visible rows alone.  Bound by the chain of loads, products and exponentials in each
// wave: 2 x 333 tokens, 16 heads over 4 x 96, forward 22.5 us with the matrix cores busy
// 18% (30 TFLOP/s), backward 89.
#include "kernels.h"
#include "score_attn_tiles.h"

namespace pb {
namespace {

constexpr int kNoBias = 0, kSlopes = 1, kTable = 2;
constexpr int kR = 16;   // rows of a block and of a tile
constexpr int kFwd = 4;  // waves of a workgroup of the forward

// 2^(s log2 e - ref), and e^(s - L), each with what the products with log2 e lose.
constexpr float kLog2eRest = 1.9259630e-8f;  // log2 e - kLog2e
PB_DEV float exp_ref(float s, float ref) {
  return exp2_hw(fmaf(s, kLog2eRest, fmaf(s, kLog2e, -ref)));
}
PB_DEV float exp_less(float s, float L) {
  const float L2 = L * kLog2e, left = fmaf(L, kLog2eRest, fmaf(L, kLog2e, -L2));
  return exp2_hw(fmaf(s, kLog2eRest, fmaf(s, kLog2e, -L2) - left));
}
PB_DEV float sum_groups(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
PB_DEV float max_groups(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
PB_DEV bool finite4(const f32x4& v) {
  return (v[0] - v[0]) + (v[1] - v[1]) + (v[2] - v[2]) + (v[3] - v[3]) == 0.f;
}

// Features 16 s + 4 g .. + 3 of a row.
template <int D>
PB_DEV void row_frag(const float* __restrict__ row, int g, f32x4 (&v)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; ++s) v[s] = *reinterpret_cast<const f32x4*>(row + 16 * s + 4 * g);
}
// Products of rows a (tile) and b (block), two chains.
template <int D>
PB_DEV f32x4 dot_rows(const f32x4 (&a)[D / 16], const f32x4 (&b)[D / 16]) {
  f32x4 acc[2] = {zero4(), zero4()};
#pragma unroll
  for (int s = 0; s < D / 16; ++s)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc[s & 1] = __builtin_amdgcn_mfma_f32_16x16x4f32(a[s][j], b[s][j], acc[s & 1], 0, 0, 0);
  return acc[0] + acc[1];
}
// out[db](feature 16 db + 4 g + e, block's row) += sum over the tile's rows of X p; x[j]
// points to feature l & 15 of row 4 g + j.
template <int D>
PB_DEV void add_rows(const float* const (&x)[4], const f32x4& p, f32x4 (&out)[D / 16]) {
#pragma unroll
  for (int db = 0; db < D / 16; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      out[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j][16 * db], p[j], out[db], 0, 0, 0);
}

// Sum of the waves' [16][D] parts; each thread's float4 number n is row(n), col(n).
template <int D, int W>
struct Merge {
  static constexpr int kVec = (kR * D / 4 + 64 * W - 1) / (64 * W);
  static constexpr int kFloats = W * kR * (D + 4);
  static PB_DEV bool has(int n) { return (int)threadIdx.x + 64 * W * n < kR * D / 4; }
  static PB_DEV int row(int n) { return ((int)threadIdx.x + 64 * W * n) / (D / 4); }
  static PB_DEV int col(int n) { return 4 * (((int)threadIdx.x + 64 * W * n) % (D / 4)); }
  static PB_DEV void run(float* __restrict__ buf, const f32x4 (&part)[D / 16], float f, int wave,
                         int i, int g, f32x4 (&sum)[kVec]) {
#pragma unroll
    for (int db = 0; db < D / 16; ++db)
      *reinterpret_cast<f32x4*>(buf + (wave * kR + i) * (D + 4) + 16 * db + 4 * g) = part[db] * f;
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kVec; ++n) {
      sum[n] = zero4();
      if (!has(n)) continue;
#pragma unroll
      for (int w = 0; w < W; ++w)
        sum[n] += *reinterpret_cast<const f32x4*>(buf + (w * kR + row(n)) * (D + 4) + col(n));
    }
  }
};
template <int D, int W>
__host__ __device__ BiasLds bias_of(const ScoreArgs& a) {
  return BiasLds(Merge<D, W>::kFloats * 4, a.buckets, a.pack, 0, 0);
}

// Scores of a tile with their terms, natural; z0: the capped ones before their bias.
template <bool CAP, int BIAS>
struct Terms {
  const ScoreArgs& a;
  const BiasLds& bl;
  const unsigned char* smem;
  Cap cap;
  PB_DEV Terms(const ScoreArgs& a_, const BiasLds& b_, const unsigned char* s)
      : a(a_), bl(b_), smem(s), cap(a_.scale, CAP ? a_.cap : 1.f, 1.f) {}
  PB_DEV f32x4 base(f32x4 s) const {
    f32x4 slope;
    return base(s, slope);
  }
  // slope: what the cap leaves of their gradients
  PB_DEV f32x4 base(f32x4 s, f32x4& slope) const {
    if constexpr (CAP) {
      f32x4 x[1] = {s};
      cap.apply(x, [&](int, int e, float d) { slope[e] = d; });
      return x[0] * a.cap;
    }
    return s * a.scale;
  }
  // of head h0 + hh at distance n
  PB_DEV float bias(int h0, int hh, int n) const {
    if constexpr (BIAS == kSlopes) return -a.slopes[h0 + hh] * (float)abs(n);
    if constexpr (BIAS == kTable)
      return ((const float*)(smem + bl.tab))[bias_bucket(a, bl, smem, n) * a.pack + hh];
    return 0.f;
  }
};
PB_DEV void bias_tables(const ScoreArgs& a, const BiasLds& bl, unsigned char* smem, int h0,
                        int threads) {
  bias_prologue(a, bl, smem, h0, a.pack, threadIdx.x, threads, 1.f);
  __syncthreads();
}

// A block of 16 packed rows: what forward and dQ share.
struct RowBlock {
  int b, h0, kvh, r0, rows, off, r, i, hh, p;
  Packed pk;
  RowKeys keys;
  KeyTiles kt;
  PB_DEV RowBlock(const ScoreArgs& a, int blk, int hb, int lane) : pk(a.pack) {
    const int sets = a.heads / a.pack;
    b = hb / sets, h0 = hb % sets * a.pack, kvh = h0 / a.group;
    rows = a.seq_q * a.pack, off = a.seq_k - a.seq_q, r0 = blk * kR;
    r = r0 + (lane & 15);
    const int rc = min(r, rows - 1);
    i = pk.pos(rc), hh = rc - i * a.pack, p = i + off;
    keys = row_keys(a, b, p);
    if (r >= rows) keys = RowKeys{0, 0, 0, 0};
    kt = key_tiles<kR>(a, b, off + pk.pos(r0), off + pk.pos(min(r0 + kR, rows) - 1), lane);
  }
  PB_DEV int head_of(int row, int& pos) const {
    pos = pk.pos(row);
    return h0 + row - pos * pk.pack;
  }
};

// ---------------------------------------------------------------- forward
// EARLY: V is requested ahead of the scores' products and the next K right behind them.
// That takes 20 to 60 registers more, which pay where a CU has one workgroup (us, without
// and with; the last with 512 workgroups):
//   1 token over 4096, 32 heads over 8 x 128   150  99
//   4 x 7 over 2048, 16 over 4 x 96             89  54
//   256, 8 x 128                              13.5 12.2
//   1000, 4 x 96                              28.4 25.8
//   1024, 8 x 128                             49.5 55.6
template <int D, bool CAP, int BIAS, bool EARLY>
__global__ __launch_bounds__(64 * kFwd) void score_fwd_f32(ScoreArgs a) {
  constexpr int W = kFwd;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float ml[2][W][kR];
  float* buf = (float*)smem;
  const BiasLds bl = bias_of<D, W>(a);
  const int hb_n = a.batch * (a.heads / a.pack), nblk = gridDim.x / hb_n;
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RowBlock t(a, nblk - 1 - blockIdx.x / hb_n, blockIdx.x % hb_n, lane);
  if constexpr (BIAS == kTable) bias_tables(a, bl, smem, t.h0, 64 * W);
  const Terms<CAP, BIAS> terms(a, bl, smem);
  f32x4 qf[D / 16], acc[D / 16];
  row_frag<D>(score::q_row<float, D>(a, t.b, t.i, t.h0 + t.hh), g, qf);
#pragma unroll
  for (int db = 0; db < D / 16; ++db) acc[db] = zero4();
  float m = kNegInf, l = 0.f;
  auto key_row = [&](int k) { return max(t.kt.lo, min(k, t.kt.hi)); };
  f32x4 kf[D / 16];
  auto load_k = [&](int n) {
    row_frag<D>(score::kv_row<float, D>(a, a.k, t.b, key_row(t.kt.tile(n) * kR + i), t.kvh), g, kf);
  };
  if (EARLY && wave < t.kt.n) load_k(wave);
  for (int n = wave; n < t.kt.n; n += W) {
    const int k0 = t.kt.tile(n) * kR;
    if constexpr (!EARLY) load_k(n);
    const float* vr[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      vr[j] = score::kv_row<float, D>(a, a.v, t.b, key_row(k0 + 4 * g + j), t.kvh) + i;
    f32x4 vf[D / 16];
    if constexpr (EARLY) {
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) vf[db][j] = vr[j][16 * db];
      __builtin_amdgcn_sched_barrier(0);
    }
    f32x4 s = terms.base(dot_rows<D>(kf, qf));
    if constexpr (EARLY) {
      __builtin_amdgcn_sched_barrier(0);
      if (n + W < t.kt.n) load_k(n + W);
      __builtin_amdgcn_sched_barrier(0);
    }
    const uint32_t see = (uint32_t)(t.keys.bits(k0) >> (4 * g));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[e] += terms.bias(t.h0, t.hh, t.p - (k0 + 4 * g + e));
      s[e] = see & (1u << e) ? s[e] : kNegInf;
    }
    const float mt = max_groups(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))) * kLog2e;
    const float mn = fmaxf(m, mt), mu = mn == kNegInf ? 0.f : mn, f = exp2_hw(m - mu);
#pragma unroll
    for (int e = 0; e < 4; ++e)
      s[e] = s[e] == kNegInf ? 0.f : exp_ref(s[e], mu);
    l = l * f + ((s[0] + s[1]) + (s[2] + s[3]));
    m = mn;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) acc[db] *= f;
    if constexpr (EARLY) {
#pragma unroll
      for (int db = 0; db < D / 16; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[db] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[db][j], s[j], acc[db], 0, 0, 0);
    } else {
      add_rows<D>(vr, s, acc);
    }
  }
  l = sum_groups(l);
  if (g == 0) ml[0][wave][i] = m, ml[1][wave][i] = l;
  __syncthreads();
  float M = kNegInf, L = 0.f;
#pragma unroll
  for (int w = 0; w < W; ++w) M = fmaxf(M, ml[0][w][i]);
  const float mu = M == kNegInf ? 0.f : M;
#pragma unroll
  for (int w = 0; w < W; ++w) L += ml[1][w][i] * exp2_hw(ml[0][w][i] - mu);
  f32x4 o[Merge<D, W>::kVec];
  Merge<D, W>::run(buf, acc, L == 0.f ? 0.f : exp2_hw(m - mu) / L, wave, i, g, o);
  const float ls = L == 0.f ? kNegInf : fmaf(M, kLn2, logf(L));
  bool bad = wave == 0 && g == 0 && t.r < t.rows && !(L - L == 0.f);
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n)
    bad |= Merge<D, W>::has(n) && t.r0 + Merge<D, W>::row(n) < t.rows && !finite4(o[n]);
  if (__syncthreads_or(bad)) {
    for (int r = t.r0 + wave; r < min(t.r0 + kR, t.rows); r += W) {
      int pos;
      const int h = t.head_of(r, pos);
      score::fwd_row<float, D>(a, t.b, h, pos, lane);
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n) {
    const int r = t.r0 + Merge<D, W>::row(n);
    if (!Merge<D, W>::has(n) || r >= t.rows) continue;
    int pos;
    const int h = t.head_of(r, pos);
    *reinterpret_cast<f32x4*>(score::o_row<float, D>(a, t.b, pos, h) + Merge<D, W>::col(n)) = o[n];
  }
  if (wave == 0 && g == 0 && t.r < t.rows) a.lse[score::lse_at(a, t.b, t.h0 + t.hh, t.i)] = ls;
}

// --------------------------------------------------------------- backward
template <int D, bool CAP, int BIAS, int W>
PB_DEV void dq_block(const ScoreArgs& a, int blk, int nblk, int hb) {
  constexpr int kPad = 65;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* buf = (float*)smem;
  const BiasLds bl = bias_of<D, W>(a);
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RowBlock t(a, blk, hb, lane);
  float* slots = (float*)(smem + bl.bytes);
  float* mine = slots + wave * a.buckets * kPad + lane;
  if constexpr (BIAS == kTable) {
    bias_tables(a, bl, smem, t.h0, 64 * W);
    if (a.dtable)
      for (int n = 0; n < a.buckets; ++n) mine[n * kPad] = 0.f;
  }
  const Terms<CAP, BIAS> terms(a, bl, smem);
  const int h = t.h0 + t.hh;
  const float L = a.lse[score::lse_at(a, t.b, h, t.i)];
  // (a row that sees nothing may hold anything; e^(s - inf) is 0)
  const bool live = (t.keys.len > 0 || t.keys.plen > 0) && L != kNegInf;
  f32x4 qf[D / 16], gf[D / 16], dq[D / 16], x = zero4();
  row_frag<D>(score::q_row<float, D>(a, t.b, t.i, h), g, qf);
  row_frag<D>(score::do_row<float, D>(a, t.b, t.i, h), g, gf);
  row_frag<D>(score::o_row<float, D>(a, t.b, t.i, h), g, dq);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    x += dq[s] * gf[s];
    dq[s] = zero4();
    if (!live) qf[s] = gf[s] = zero4();
  }
  float dl = sum_groups((x[0] + x[1]) + (x[2] + x[3])), inv = 1.f;
  if (!live) dl = 0.f;
  auto key_row = [&](int k) { return max(t.kt.lo, min(k, t.kt.hi)); };
  if constexpr (BIAS == kTable) {
    __shared__ float part[2][W][kR];
    float sp = 0.f, sd = 0.f;
    for (int n = wave; n < t.kt.n; n += W) {
      const int k0 = t.kt.tile(n) * kR;
      f32x4 kf[D / 16], vf[D / 16];
      row_frag<D>(score::kv_row<float, D>(a, a.k, t.b, key_row(k0 + i), t.kvh), g, kf);
      row_frag<D>(score::kv_row<float, D>(a, a.v, t.b, key_row(k0 + i), t.kvh), g, vf);
      const f32x4 z = terms.base(dot_rows<D>(kf, qf)), dp = dot_rows<D>(vf, gf);
      const uint32_t see = live ? (uint32_t)(t.keys.bits(k0) >> (4 * g)) : 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float s = z[e] + terms.bias(t.h0, t.hh, t.p - (k0 + 4 * g + e));
        const float p = see & (1u << e) && s != kNegInf ? exp_less(s, L) : 0.f;
        sp += p;
        sd = p == 0.f ? sd : fmaf(p, dp[e], sd);  // (dP behind the mask may be anything)
      }
    }
    sp = sum_groups(sp), sd = sum_groups(sd);
    if (g == 0) part[0][wave][i] = sp, part[1][wave][i] = sd;
    __syncthreads();
    sp = sd = 0.f;
#pragma unroll
    for (int w = 0; w < W; ++w) sp += part[0][w][i], sd += part[1][w][i];
    if (sp != 0.f) inv = 1.f / sp, dl = sd / sp;
  }
  for (int n = wave; n < t.kt.n; n += W) {
    const int k0 = t.kt.tile(n) * kR;
    f32x4 kf[D / 16], vf[D / 16];
    row_frag<D>(score::kv_row<float, D>(a, a.k, t.b, key_row(k0 + i), t.kvh), g, kf);
    row_frag<D>(score::kv_row<float, D>(a, a.v, t.b, key_row(k0 + i), t.kvh), g, vf);
    const float* kr[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      kr[j] = score::kv_row<float, D>(a, a.k, t.b, key_row(k0 + 4 * g + j), t.kvh) + i;
    f32x4 slope;
    const f32x4 z = terms.base(dot_rows<D>(kf, qf), slope);
    f32x4 ds = dot_rows<D>(vf, gf);
    const uint32_t see = live ? (uint32_t)(t.keys.bits(k0) >> (4 * g)) : 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n_ = t.p - (k0 + 4 * g + e);
      const float s = z[e] + terms.bias(t.h0, t.hh, n_);
      ds[e] = see & (1u << e) && s != kNegInf ? exp_less(s, L) * inv * (ds[e] - dl) : 0.f;
      if constexpr (BIAS == kTable)
        if (a.dtable && (see & (1u << e)))
          unsafeAtomicAdd(&mine[bias_bucket(a, bl, smem, n_) * kPad], ds[e]);
      if constexpr (CAP) ds[e] *= slope[e];
    }
    add_rows<D>(kr, ds, dq);
  }
  f32x4 o[Merge<D, W>::kVec];
  Merge<D, W>::run(buf, dq, a.dscale, wave, i, g, o);  // (its barrier: every wave's sums are there)
  if constexpr (BIAS == kTable) {
    if (a.dtable)
      for (int y = threadIdx.x; y < a.buckets * a.pack; y += 64 * W) {
        const int n = y % a.buckets, hh = y / a.buckets;
        float s = 0.f;
        for (int q = 0; q < kR; ++q) {
          int pos;
          if (t.head_of(t.r0 + q, pos) != t.h0 + hh) continue;
          for (int w = 0; w < W; ++w)
#pragma unroll
            for (int k = 0; k < 4; ++k) s += slots[(w * a.buckets + n) * kPad + q + 16 * k];
        }
        a.bias_part[(((size_t)t.b * nblk + blk) * a.heads + t.h0 + hh) * a.buckets + n] = s;
      }
  }
  bool bad = false;
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n)
    bad |= Merge<D, W>::has(n) && t.r0 + Merge<D, W>::row(n) < t.rows && !finite4(o[n]);
  if (__syncthreads_or(bad)) {
    for (int r = t.r0 + wave; r < min(t.r0 + kR, t.rows); r += W) {
      int pos;
      const int hr = t.head_of(r, pos);
      score::dq_row<float, D>(a, t.b, hr, pos, lane);
    }
    return;
  }
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n) {
    const int r = t.r0 + Merge<D, W>::row(n);
    if (!Merge<D, W>::has(n) || r >= t.rows) continue;
    int pos;
    const int hr = t.head_of(r, pos);
    *reinterpret_cast<f32x4*>((float*)a.dq + ((size_t)t.b * a.seq_q + pos) * a.ld_dq + hr * D +
                              Merge<D, W>::col(n)) = o[n];
  }
}

template <int D, bool CAP, int BIAS, int W>
PB_DEV void dkdv_block(const ScoreArgs& a, int blk, int hb) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* buf = (float*)smem;
  const BiasLds bl = bias_of<D, W>(a);
  const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = hb / a.kv_heads, kvh = hb % a.kv_heads, j0 = blk * kR, key = j0 + i;
  const int off = a.seq_k - a.seq_q, kc = min(key, a.seq_k - 1);
  const Packed pk(a.pack);
  const Terms<CAP, BIAS> terms(a, bl, smem);
  int sf = 0, sn = 0;
  if (key < a.seq_k) {
    const Bounds d = bounds_of(a, b, key);
    if (d.de > d.ds) {
      sf = max(score::seen_first(a, d, key), off);
      sn = max(score::seen_last(a, d, key) - sf + 1, 0);
    }
  }
  const int lo = wave_imin(sn > 0 ? sf : 0x7fffffff), hi = wave_imax(sn > 0 ? sf + sn - 1 : -1);
  f32x4 kf[D / 16], vf[D / 16], dk[D / 16], dv[D / 16];
  row_frag<D>(score::kv_row<float, D>(a, a.k, b, kc, kvh), g, kf);
  row_frag<D>(score::kv_row<float, D>(a, a.v, b, kc, kvh), g, vf);
#pragma unroll
  for (int db = 0; db < D / 16; ++db) dk[db] = dv[db] = zero4();
  const int r_lo = hi < 0 ? 0 : (lo - off) * a.pack, r_hi = hi < 0 ? -1 : (hi - off + 1) * a.pack - 1;
  for (int h0 = kvh * a.group; h0 < (kvh + 1) * a.group; h0 += a.pack) {
    if constexpr (BIAS == kTable) {
      __syncthreads();  // (every wave is done with the last heads' table)
      bias_tables(a, bl, smem, h0, 64 * W);
    }
    for (int r0 = r_lo / kR * kR + kR * wave; r0 <= r_hi; r0 += kR * W) {
      auto row_of = [&](int r, int& h) {
        const int x = max(r_lo, min(r, r_hi)), pos = pk.pos(x);
        h = h0 + x - pos * a.pack;
        return pos;
      };
      int h;
      const int qi = row_of(r0 + i, h);
      f32x4 qf[D / 16], gf[D / 16], x = zero4();
      row_frag<D>(score::do_row<float, D>(a, b, qi, h), g, gf);
      row_frag<D>(score::o_row<float, D>(a, b, qi, h), g, qf);
#pragma unroll
      for (int s = 0; s < D / 16; ++s) x += qf[s] * gf[s];
      // row i's terms in every lane with l & 15 = i; a lane needs rows 4 g + e
      const float dli = sum_groups((x[0] + x[1]) + (x[2] + x[3]));
      const float Li = a.lse[score::lse_at(a, b, h, qi)];
      row_frag<D>(score::q_row<float, D>(a, b, qi, h), g, qf);
      const float *qr[4], *gr[4];
      int pos[4], hh[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int y = row_of(r0 + 4 * g + j, hh[j]);
        qr[j] = score::q_row<float, D>(a, b, y, hh[j]) + i;
        gr[j] = score::do_row<float, D>(a, b, y, hh[j]) + i;
        hh[j] -= h0;
        const int r = r0 + 4 * g + j;
        pos[j] = r >= r_lo && r <= r_hi ? y + off : -1;
      }
      f32x4 slope;
      const f32x4 z = terms.base(dot_rows<D>(qf, kf), slope);
      f32x4 pr, ds = dot_rows<D>(gf, vf);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float L = __shfl(Li, 4 * g + e, 64), dl = __shfl(dli, 4 * g + e, 64);
        const bool see = pos[e] >= 0 && (unsigned)(pos[e] - sf) < (unsigned)sn && L != kNegInf;
        const float s = z[e] + terms.bias(h0, hh[e], pos[e] - key);
        pr[e] = see && s != kNegInf ? exp_less(s, L) : 0.f;
        ds[e] = pr[e] == 0.f ? 0.f : pr[e] * (ds[e] - dl);
        if constexpr (CAP) ds[e] *= slope[e];
      }
      add_rows<D>(gr, pr, dv);
      add_rows<D>(qr, ds, dk);
    }
  }
  f32x4 ov[Merge<D, W>::kVec], ok[Merge<D, W>::kVec];
  Merge<D, W>::run(buf, dv, 1.f, wave, i, g, ov);
  __syncthreads();
  Merge<D, W>::run(buf, dk, a.dscale, wave, i, g, ok);
  bool bad = false;
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n)
    bad |= Merge<D, W>::has(n) && j0 + Merge<D, W>::row(n) < a.seq_k &&
           !(finite4(ov[n]) && finite4(ok[n]));
  if (__syncthreads_or(bad)) {
    for (int r = j0 + wave; r < min(j0 + kR, a.seq_k); r += W)
      score::dkdv_row<float, D>(a, b, kvh, r, lane);
    return;
  }
#pragma unroll
  for (int n = 0; n < Merge<D, W>::kVec; ++n)
    if (Merge<D, W>::has(n) && j0 + Merge<D, W>::row(n) < a.seq_k) {
      const size_t at = ((size_t)b * a.seq_k + j0 + Merge<D, W>::row(n)) * a.ld_dkv + kvh * D +
                        Merge<D, W>::col(n);
      *reinterpret_cast<f32x4*>((float*)a.dk + at) = ok[n];
      *reinterpret_cast<f32x4*>((float*)a.dv + at) = ov[n];
    }
}

// Both roles in one launch, in turn, each longest first.
template <int D, bool CAP, int BIAS, int W>
__global__ __launch_bounds__(64 * W) void score_bwd_f32(ScoreArgs a, int nk, int nq) {
  const int id = blockIdx.x, mn = min(nk, nq);
  const bool kv = id < 2 * mn ? !(id & 1) : nk > nq;
  const int x = id < 2 * mn ? id >> 1 : id - mn;
  if (kv) {
    const int n = a.batch * a.kv_heads;
    dkdv_block<D, CAP, BIAS, W>(a, x / n, x % n);
  } else {
    const int n = a.batch * (a.heads / a.pack), nblk = nq / n;
    dq_block<D, CAP, BIAS, W>(a, nblk - 1 - x / n, nblk, x % n);
  }
}

unsigned row_blocks(const ScoreArgs& a) {
  return (unsigned)((a.seq_q * a.pack + kR - 1) / kR * a.batch * (a.heads / a.pack));
}
#define PB_BY_TERMS(KERNEL, ...)                                            \
  do {                                                                      \
    if (a.cap > 0.f) {                                                      \
      if (a.table) KERNEL(true, kTable);                                    \
      else if (a.slopes) KERNEL(true, kSlopes);                             \
      else KERNEL(true, kNoBias);                                           \
    } else {                                                                \
      if (a.table) KERNEL(false, kTable);                                   \
      else if (a.slopes) KERNEL(false, kSlopes);                            \
      else KERNEL(false, kNoBias);                                          \
    }                                                                       \
  } while (0)

template <int D>
void fwd_d(const ScoreArgs& a, hipStream_t s) {
  const size_t lds = a.table ? bias_of<D, kFwd>(a).bytes : Merge<D, kFwd>::kFloats * 4;
  const unsigned grid = row_blocks(a);
#define PB_FWD(C, B)                                                                   \
  do {                                                                                 \
    if (grid <= 256) score_fwd_f32<D, C, B, true><<<grid, 64 * kFwd, lds, s>>>(a);     \
    else score_fwd_f32<D, C, B, false><<<grid, 64 * kFwd, lds, s>>>(a);                \
  } while (0)
  PB_BY_TERMS(PB_FWD);
#undef PB_FWD
}

// Waves of a backward workgroup: eight where the longest row of tiles, shared by four,
// would take half as long again as all tiles over the card's waves (two a SIMD), and has
// 32 tiles; else four.  Timed (us, four and eight waves):
//   333 x 2, 16 over 4 x 96          99.6  88.6     1024, 8 x 128                173 179
//   1000, 4 x 96                       84    69     900 x 2, 8 over 4 x 64       130 152
//   2048, 2 x 128                     213   164     4096, 4 x 64                 541 575
//   700 x 2, 8 over 2 x 64, a table   156   127     2048, 16 x 96, window 256    239 316
//   1 over 4096, 32 over 8 x 128      253   186     256, 4 x 128                25.8 26.8
int bwd_waves(const ScoreArgs& a, int nk, int nq) {
  const long long rows = ((long long)a.seq_q * a.pack + kR - 1) / kR, sets = a.group / a.pack;
  const long long reach = (long long)(a.causal ? 1 : 2) * a.window + kR;
  const double kv = (double)sets * (a.prefix ? rows : std::min(rows, reach * a.pack / kR + 2));
  const double q = score_most_tiles(a, kR, kR);
  const double half = a.causal && a.window >= a.seq_k ? 0.5 : 1.0;
  const double all = half * (nk * kv + nq * q) / 2048, longest = std::max(kv, q);
  return longest >= 32 && longest / 4 >= 1.5 * all ? 8 : 4;
}
template <int D, int W>
size_t bwd_lds(const ScoreArgs& a) {
  return (a.table ? bias_of<D, W>(a).bytes : Merge<D, W>::kFloats * 4) +
         (a.dtable ? (size_t)W * a.buckets * 65 * 4 : 0);
}
template <int D, int W>
void bwd_w(const ScoreArgs& a, int nk, int nq, hipStream_t s) {
  const size_t lds = bwd_lds<D, W>(a);
#define PB_BWD(C, B) score_bwd_f32<D, C, B, W><<<nk + nq, 64 * W, lds, s>>>(a, nk, nq)
  PB_BY_TERMS(PB_BWD);
#undef PB_BWD
}
template <int D>
void bwd_d(const ScoreArgs& a, hipStream_t s) {
  const int nq = (int)row_blocks(a), nk = (a.seq_k + kR - 1) / kR * a.batch * a.kv_heads;
  // (a table of many buckets leaves room for four waves' sums)
  if (bwd_waves(a, nk, nq) == 8 && bwd_lds<D, 8>(a) <= 152 * 1024) bwd_w<D, 8>(a, nk, nq, s);
  else bwd_w<D, 4>(a, nk, nq, s);
  if (a.dtable)
    launch_score_dtable_sum(a, (a.seq_q * a.pack + kR - 1) / kR * a.batch, s);
}

}  // namespace

size_t score_bias_part_floats_f32(const ScoreArgs& a) {
  return (size_t)a.batch * ((a.seq_q * a.pack + kR - 1) / kR) * a.heads * a.buckets;
}

void launch_score_forward_f32(int head_dim, const ScoreArgs& a, hipStream_t s) {
  if (head_dim == 64) fwd_d<64>(a, s);
  else if (head_dim == 96) fwd_d<96>(a, s);
  else fwd_d<128>(a, s);
}
void launch_score_backward_f32(int head_dim, const ScoreArgs& a, hipStream_t s) {
  if (head_dim == 64) bwd_d<64>(a, s);
  else if (head_dim == 96) bwd_d<96>(a, s);
  else bwd_d<128>(a, s);
}

}  // namespace pb

// Forward of attention with terms in its scores, bf16, on v_mfma_f32_16x16x32_bf16.
//
// A workgroup of four waves has 128 rows (of several heads that share a key head, see
// Packed), wave w rows 32 w .. + 31 as two 16-row column blocks, and walks 64-key tiles
// of the keys that its rows see: S^T = K Q^T (4 x 2 blocks of 16 x 16; a lane holds 16
// scores of each of two rows), the terms and the mask on those registers, the online
// softmax, O^T += V^T P^T.  As in attn.hip the running maximum moves only when a score
// passes it by more than 8 (base 2), and iteration t runs tile t + 1's score products
// beside tile t's exponentials.  The row sums are of unrounded probabilities (lse is
// kept in fp32 and the gradient's probabilities follow from it).
//
// Probabilities enter O as bf16.  WIDE adds the products with what that rounding leaves
// (16 bits of each in all), so that o is off by its own rounding alone (1.66e-3 in norm,
// without 1.7e-3 to 2.1e-3): half as many matrix products again and one and a half vector
// instructions a score.
//
// LDS: K and V in two slots each; iteration t loads K of tile t + 2 and V of tile t + 1.
// That leaves 16 KB of a CU's half for the rows' keys (read back in partial tiles only)
// and the biases, so that two workgroups share a CU.
//
// Measured (WIDE, and without): 8192 tokens of packed documents, 16 heads over 4 x 128,
// window 4096, bias by distance 204 us (156), 508 TFLOP/s of 4 d operations a pair, matrix
// cores busy 28% and vector instructions 43% under the profiler; 4096 x 16 heads of
// 64 without terms 78 (62; attn.hip 62); a token over 4 x 8192 keys, 40 heads over 8, 39.7
// (34), of which K and V at 4.1 TB/s 32.8 (28).
//
// At head_dim 128 registers are full: 4 to 18 spill with WIDE (7 to 17 without, none without
// terms), nearly all of them around the loop and in partial tiles.
//
// A non-finite value behind the mask makes a product non-finite (0 x Inf).  A wave with a
// non-finite output computes its rows again by the definition, which reads visible keys
// alone.
#include "kernels.h"
#include "score_attn_tiles.h"

namespace pb {
namespace {

template <typename T>
struct Type {
  using type = T;
};
constexpr int kRows = 128;  // rows of a workgroup
constexpr int kTL = 64;     // keys of a tile
constexpr int kMinTiles = 4;  // of a chunk
constexpr int kNoBias = 0, kSlopes = 1, kTable = 2;

template <int D>
constexpr int tiles_bytes() {
  return 4 * kTL * 2 * D;
}
template <int D>
BiasLds bias_lds(const ScoreArgs& a) {
  return BiasLds(tiles_bytes<D>() + kRows * (int)sizeof(RowKeys), a.buckets, a.pack,
                 (kRows + a.pack - 1) / a.pack + 1, kTL);
}

template <int D, bool CAP, int BIAS, bool WIDE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void score_fwd_bf16(
    ScoreArgs a, int nc, float* __restrict__ po, float* __restrict__ plse,
    int* __restrict__ used) {
  constexpr int TL = kTL, TB = TL * 2 * D, KS = D / 32, DB = D / 16;
  constexpr bool LEAN = WIDE && D == 128;  // registers
  constexpr bool kZ = BIAS != kNoBias;  // scores are turned to base 2 with their bias
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  auto k_off = [](int s) { return (uint32_t)(s * TB); };
  auto v_off = [](int s) { return (uint32_t)((2 + s) * TB); };
  RowKeys* keys_of = (RowKeys*)(smem + 4 * TB);

  // workgroups of all heads' last blocks first (under a causal mask the longest)
  const Packed pk(a.pack);
  const int hb_n = a.batch * (a.heads / a.pack), rows = a.seq_q * a.pack;
  const int nblk = (rows + kRows - 1) / kRows;
  const int hb = (int)(blockIdx.x % hb_n), bx = (int)(blockIdx.x / hb_n);
  const int b = hb / (a.heads / a.pack), h0 = hb % (a.heads / a.pack) * a.pack;
  const int kvh = h0 / a.group;
  const int chunk = bx % nc, r0 = (nblk - 1 - bx / nc) * kRows;
  const int off = a.seq_k - a.seq_q;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, col = lane & 15;
  const int p_first = off + pk.pos(r0), p_last = off + pk.pos(min(r0 + kRows, rows) - 1);

  const KeyTiles kt = key_tiles<TL>(a, b, p_first, p_last, lane);
  const Share share(kt.n, nc, kMinTiles);
  const int t_begin = chunk * share.size, n = min(kt.n - t_begin, share.size);
  const int qw0 = r0 + 32 * wave;
  const bool split = share.used > 1;
  if (chunk >= max(share.used, 1)) return;
  if (nc > 1 && chunk == 0 && tid == 0) used[(size_t)hb * nblk + r0 / kRows] = share.used;
  const size_t part0 = (size_t)chunk * a.batch * a.heads * a.seq_q;
  auto row_at = [&](int r) {  // of lse, and of the partial results
    const int i = pk.pos(r);
    return score::lse_at(a, b, h0 + r - i * a.pack, i);
  };
  if (n <= 0) {  // nothing is seen
    for (int x = tid; x < kRows * (D / 8); x += 256) {
      const int r = r0 + x / (D / 8);
      if (r >= rows) break;
      const int i = pk.pos(r);
      *reinterpret_cast<u32x4*>(score::o_row<bf16, D>(a, b, i, h0 + r - i * a.pack) +
                                8 * (x % (D / 8))) = u32x4{0, 0, 0, 0};
    }
    if (tid < kRows && r0 + tid < rows) a.lse[row_at(r0 + tid)] = kNegInf;
    return;
  }

  const bf16* kb = score::kv_row<bf16, D>(a, a.k, b, 0, kvh);
  const bf16* vb = score::kv_row<bf16, D>(a, a.v, b, 0, kvh);
  const BiasLds bl(4 * TB + kRows * (int)sizeof(RowKeys), a.buckets, a.pack,
                   (kRows + a.pack - 1) / a.pack + 1, TL);

  using DmaK = DmaRows<D, TL, 4>;
  using DmaV = DmaRows<D, TL, 4, true>;
  constexpr int PK = DmaK::NPW;
  const FwdLds<D> la(lane);
  // The lane's pieces of a tile; kept for tiles of which every row is a key between lo
  // and hi, formed anew where rows beyond are read from the nearest of those.
  // (LEAN: formed anew each tile from the first piece's, with the lane's places in LDS)
  uint32_t at_k[PK], at_v[PK];
  auto pieces = [&](const auto& dma, int lo, int hi, uint32_t (&at)[PK]) {
#pragma unroll
    for (int x = 0; x < PK; ++x)
      at[x] = (uint32_t)max(lo, min(dma.row[x], hi)) * (uint32_t)(2 * a.ld_kv) + dma.cof[x];
  };
  uint32_t lean_r = 0, lean_c = 0;
  if constexpr (LEAN) {
    const DmaK first(wave, lane);
    lean_r = (uint32_t)first.row[0] * (uint32_t)(2 * a.ld_kv), lean_c = first.cof[0];
  } else {
    pieces(DmaK(wave, lane), 0, TL - 1, at_k);
    pieces(DmaV(wave, lane), 0, TL - 1, at_v);
  }
  auto issue = [&](const bf16* base, auto type, const uint32_t (&whole)[PK], int i, uint32_t slot) {
    using Dma = typename decltype(type)::type;
    const int kv0 = kt.tile(t_begin + i) * TL;
    const bf16* tile = base + (size_t)kv0 * a.ld_kv;
    if (LEAN && kv0 >= kt.lo && kv0 + TL - 1 <= kt.hi) {
      // piece x begins 4 x rows on, its chunks are those of the first with bit 1 of x / 2
      // turned (in V, whose swizzle leaves bit 4 of the row out, with bit 0 of the wave's)
      uint32_t c = lean_c ^ (Dma::kV ? 16u * (wave & 1) : 0u);
      asm volatile("" : "+v"(c));
#pragma unroll
      for (int x = 0; x < PK; ++x)
        dma16s(tile + (size_t)(4 * x) * a.ld_kv, lean_r + (c ^ (32u * (x >> 1))),
               lds0 + slot + (uint32_t)((wave * PK + x) * 1024));
    } else if (kv0 >= kt.lo && kv0 + TL - 1 <= kt.hi) {
#pragma unroll
      for (int x = 0; x < PK; ++x)
        dma16s(tile, whole[x], lds0 + slot + (uint32_t)((wave * PK + x) * 1024));
    } else {
      uint32_t at[PK];
      int l = lane;
      asm("" : "+v"(l));  // (or its rows and columns would be kept over the loop)
      pieces(Dma(wave, l), max(kt.lo - kv0, 0), min(kt.hi - kv0, TL - 1), at);
#pragma unroll
      for (int x = 0; x < PK; ++x)
        dma16s(tile, at[x], lds0 + slot + (uint32_t)((wave * PK + x) * 1024));
    }
  };
  auto issue_k = [&](int i) { issue(kb, Type<DmaK>{}, at_k, i, k_off(i & 1)); };
  auto issue_v = [&](int i) { issue(vb, Type<DmaV>{}, at_v, i, v_off(i & 1)); };
  issue_k(0);
  if (n > 1) issue_k(1);
  issue_v(0);

  bf16x8 qf[2][KS];
  float slope2[2] = {0.f, 0.f};  // of the lane's rows
  int pos[2];
  int bias_at[2];                        // their heads' biases and positions in them
  int first_hi = 0, last_lo = 0x7fffffff, pre_hi = 0, pre_lo = 0;
  {
    first_hi = -1;
    int pf_hi = -1, pl_lo = 0x7fffffff;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = qw0 + 16 * j + col, rc = min(r, rows - 1);
      const int i = pk.pos(rc), h = h0 + rc - i * a.pack, p = i + off;
      const bf16* qr = score::q_row<bf16, D>(a, b, i, h);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) qf[j][ks] = load_row_frag(qr + 32 * ks + 8 * g, r < rows);
      RowKeys k = row_keys(a, b, p);
      if (r >= rows) k = RowKeys{0, 0, 0, 0};
      if (g == 0) keys_of[32 * wave + 16 * j + col] = k;
      first_hi = max(first_hi, k.len > 0 ? k.first : 0x7fffffff);
      last_lo = min(last_lo, k.first + k.len - 1);
      pf_hi = max(pf_hi, k.plen > 0 ? k.pfirst : 0x7fffffff);
      pl_lo = min(pl_lo, k.pfirst + k.plen - 1);
      pos[j] = p;
      if constexpr (BIAS == kSlopes) slope2[j] = -a.slopes[h] * kLog2e;
      if constexpr (BIAS == kTable)
        bias_at[j] = (h - h0) * bl.stride + (p_last - p) + 8 * g;
    }
    // (lane groups hold the same rows)
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) {
      first_hi = max(first_hi, __shfl_xor(first_hi, o, 64));
      last_lo = min(last_lo, __shfl_xor(last_lo, o, 64));
      pf_hi = max(pf_hi, __shfl_xor(pf_hi, o, 64));
      pl_lo = min(pl_lo, __shfl_xor(pl_lo, o, 64));
    }
    // keys that all rows of the wave see, by their windows or by their prefixes
    first_hi = __builtin_amdgcn_readfirstlane(first_hi);
    last_lo = __builtin_amdgcn_readfirstlane(last_lo);
    pre_hi = __builtin_amdgcn_readfirstlane(pf_hi);
    pre_lo = __builtin_amdgcn_readfirstlane(pl_lo);
  }
  int bias_last = 0;
  float far[2][2];  // bias of the last bucket of either side (causal: of bucket 0)
  auto near_tile = [&](int i) {  // whether the tile's distances span buckets
    const int kv0 = kt.tile(t_begin + i) * TL;
    return bias_uniform(a, bias_last, p_first - kv0 - TL + 1, p_last - kv0) < 0;
  };
  auto build = [&](int i) {  // biases of tile i, where it needs any
    if (near_tile(i))
      bias_tile(a, bl, smem, i & 1, a.pack, p_last - kt.tile(t_begin + i) * TL, tid, 256);
  };
  if constexpr (BIAS == kTable) {
    bias_last = a.first[a.side - 1];
    bias_prologue(a, bl, smem, h0, a.pack, tid, 256);
    __syncthreads();
    build(0);
    if (n > 1) build(1);
    const float* tab = (const float*)(smem + bl.tab);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int h = bias_at[j] / bl.stride;
      far[j][0] = tab[(a.side - 1) * a.pack + h];
      far[j][1] = tab[(a.causal ? 0 : 2 * a.side - 1) * a.pack + h];
    }
  }
  const Cap cap(a.scale, CAP ? a.cap : 1.f);

  const float c2 = CAP ? cap.top : a.scale * kLog2e;  // (of tanh, with a cap)
  float m_run[2] = {kNegInf, kNegInf}, l_run[2] = {0.f, 0.f};
  f32x4 o[DB][2];
#pragma unroll
  for (int db = 0; db < DB; ++db) o[db][0] = o[db][1] = zero4();

  f32x4 sa[4][2], sb[4][2];
  bf16x8 pf[2][2], pl[2][2], kf[2][4], vf[3][2];  // (pl: what pf leaves, with WIDE)
  float m_use[2];

  auto place = [&](uint32_t base, const auto& of, int n, uint32_t bits) {
    if constexpr (!LEAN) return base + of[n];
    uint32_t x = base + of[0];  // (rows begin at multiples of 256 bytes)
    asm volatile("" : "+v"(x));
    return x ^ (bits * n);
  };
  auto read_k = [&](uint32_t base, int ks) {
    const uint32_t at = place(base, la.k, ks, 64);
#pragma unroll
    for (int k4 = 0; k4 < 4; ++k4)
      kf[ks & 1][k4] = lds_b128(at + 2 * D * score_row_off(k4));
  };
  auto read_v = [&](uint32_t base, int db) {
    const uint32_t at = place(base, la.v, db, 32);
#pragma unroll
    for (int sp = 0; sp < 2; ++sp)
      vf[db % 3][sp] = lds_tr2(at + 2 * D * 32 * sp, 2 * D * 4);
  };
  auto exp_unit = [&](const f32x4 (&sc)[4][2], int u) {
    const int j = u >> 2, sp = (u >> 1) & 1, h = u & 1;
    float p[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      p[e] = exp2_hw(kZ ? sc[2 * sp + h][j][e] - m_use[j]
                        : fmaf(sc[2 * sp + h][j][e], c2, -m_use[j]));
#pragma unroll
    for (int e = 0; e < 4; ++e) pf[sp][j][4 * h + e] = (bf16)p[e];
    if constexpr (WIDE) {
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        const int at = 4 * h + e;
        const bf16x2 x = rest_of(bf16x2{pf[sp][j][at], pf[sp][j][at + 1]}, p[e], p[e + 1]);
        pl[sp][j][at] = x[0], pl[sp][j][at + 1] = x[1];
      }
    }
    l_run[j] += (p[0] + p[1]) + (p[2] + p[3]);
  };
  auto score_phase = [&](uint32_t kbase, int ks, f32x4 (&sn)[4][2]) {
    if (ks + 1 < KS) read_k(kbase, ks + 1);
#pragma unroll
    for (int k4 = 0; k4 < 4; ++k4) {
      sn[k4][0] = mfma16(kf[ks & 1][k4], qf[0][ks], ks ? sn[k4][0] : zero4());
      sn[k4][1] = mfma16(kf[ks & 1][k4], qf[1][ks], ks ? sn[k4][1] : zero4());
    }
  };
  auto score_sched = [&](int ks, bool valu) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      __builtin_amdgcn_sched_group_barrier(kSgMfma, 1, 0);
      if (ks + 1 < KS) __builtin_amdgcn_sched_group_barrier(kSgDsRead, 1, 0);
      if (valu) __builtin_amdgcn_sched_group_barrier(kSgValu, 3, 0);
      __builtin_amdgcn_sched_group_barrier(kSgMfma, 1, 0);
      if (valu) __builtin_amdgcn_sched_group_barrier(kSgValu, 3, 0);
    }
  };
  auto exp_phase = [&](const f32x4 (&sc)[4][2], int ks) {
#pragma unroll
    for (int u = ks * 8 / KS; u < (ks + 1) * 8 / KS; ++u) exp_unit(sc, u);
  };
  auto keep_exps = [&](int ks) {
#pragma unroll
    for (int u = ks * 8 / KS; u < (ks + 1) * 8 / KS; ++u)
      if (u % 2 == 1 || u == (ks + 1) * 8 / KS - 1) {
        keep(pf[(u >> 1) & 1][u >> 2]);
        if constexpr (WIDE) keep(pl[(u >> 1) & 1][u >> 2]);
      }
    keep(l_run[0]);
    keep(l_run[1]);
  };
  // the terms of tile i's scores, and its mask where the wave does not see all of it
  auto terms = [&](f32x4 (&sc)[4][2], int i) {
    const int kv0 = kt.tile(t_begin + i) * TL;
    if constexpr (CAP) cap.apply(reinterpret_cast<f32x4(&)[8]>(sc));
    if constexpr (BIAS == kSlopes) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float d0 = (float)(pos[j] - kv0 - 8 * g);
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[k4][j][e] =
                fmaf(slope2[j], fabsf(d0 - (float)(score_row_off(k4) + e)), sc[k4][j][e] * c2);
      }
    }
    if constexpr (BIAS == kTable) {
      const int u = bias_uniform(a, bias_last, p_first - kv0 - TL + 1, p_last - kv0);
      const float* bt = (const float*)(smem + bl.tile(i & 1, a.pack));
      if (u < 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              sc[k4][j][e] = fmaf(sc[k4][j][e], c2, bt[bias_at[j] + score_row_off(k4) + e]);
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float f = u == a.side - 1 ? far[j][0] : far[j][1];
#pragma unroll
          for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
            for (int e = 0; e < 4; ++e) sc[k4][j][e] = fmaf(sc[k4][j][e], c2, f);
        }
      }
    }
    const bool full = (kv0 >= first_hi && kv0 + TL - 1 <= last_lo) ||
                      (kv0 >= pre_hi && kv0 + TL - 1 <= pre_lo);
    if (!full) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // (a bit a key: window and prefix cost one test)
        const uint64_t see = keys_of[32 * wave + 16 * j + col].bits(kv0) >> (8 * g);
        const uint32_t half[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
        for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            sc[k4][j][e] = half[k4 >> 1] & (1u << (4 * (k4 & 1) + e)) ? sc[k4][j][e] : kNegInf;
      }
    }
  };
  auto lane_max = [&](const f32x4 (&sc)[4][2], float (&mx)[2]) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float m = sc[0][j][0];
#pragma unroll
      for (int k4 = 0; k4 < 4; ++k4)
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, sc[k4][j][e]);
      mx[j] = kZ ? m : m * c2;
    }
  };
  auto pv_phase = [&](uint32_t vbase, int db) {
    if (db + 2 < DB) read_v(vbase, db + 2);
#pragma unroll
    for (int sp = 0; sp < 2; ++sp) {
      o[db][0] = mfma16(vf[db % 3][sp], pf[sp][0], o[db][0]);
      o[db][1] = mfma16(vf[db % 3][sp], pf[sp][1], o[db][1]);
      if constexpr (WIDE) {
        o[db][0] = mfma16(vf[db % 3][sp], pl[sp][0], o[db][0]);
        o[db][1] = mfma16(vf[db % 3][sp], pl[sp][1], o[db][1]);
      }
    }
  };
  auto pv_sched = [&](int db, bool valu) {
#pragma unroll
    for (int r = 0; r < (WIDE ? 8 : 4); ++r) {
      __builtin_amdgcn_sched_group_barrier(kSgMfma, 1, 0);
      if (r < 4 && db + 2 < DB) __builtin_amdgcn_sched_group_barrier(kSgDsRead, 1, 0);
      if (valu) __builtin_amdgcn_sched_group_barrier(kSgValu, 4, 0);
    }
  };
  auto update_max = [&](const float (&mx)[2], float (&alpha)[2]) {
    alpha[0] = alpha[1] = 1.f;
    const bool any = __builtin_amdgcn_ballot_w64(mx[0] > m_run[0] + 8.f || mx[1] > m_run[1] + 8.f);
    if (any) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float m_new = fmaxf(m_run[j], max4groups(mx[j]));
        alpha[j] = m_new == kNegInf ? 1.f : exp2_hw(m_run[j] - m_new);
        m_run[j] = m_new;
      }
    }
    return any;
  };

  auto iteration = [&](int i, f32x4 (&cur)[4][2], f32x4 (&nxt)[4][2], auto NEXT) {
    constexpr bool has_next = decltype(NEXT)::value;
#pragma unroll
    for (int j = 0; j < 2; ++j) m_use[j] = m_run[j] == kNegInf ? 0.f : m_run[j];
    wait_dma_all();   // V of tile i and K of tile i + 1, requested an iteration ago
    block_barrier();  // ... for every wave; the slots of tile i - 1 are free
    if (i + 2 < n) {
      issue_k(i + 2);
      if constexpr (BIAS == kTable) build(i + 2);
    }
    if (has_next) issue_v(i + 1);
    const uint32_t kbase = lds0 + k_off((i + 1) & 1), vbase = lds0 + v_off(i & 1);
    if (has_next) read_k(kbase, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (has_next) score_phase(kbase, ks, nxt);
      exp_phase(cur, ks);
      score_sched(ks, true);
      keep_exps(ks);
      __builtin_amdgcn_sched_barrier(0);
    }
    float mx[2] = {kNegInf, kNegInf};
    // (the first V fragments take the registers that the last K fragments leave)
    read_v(vbase, 0);
    read_v(vbase, 1);
    __builtin_amdgcn_sched_barrier(0);
    if (has_next) {
      terms(nxt, i + 1);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      pv_phase(vbase, db);
      if (has_next && db == 0) lane_max(nxt, mx);
      pv_sched(db, has_next && db == 0);
      if (has_next && db == 0) keep(mx[0]), keep(mx[1]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (has_next) {
      float alpha[2];
      if (update_max(mx, alpha)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          l_run[j] *= alpha[j];
#pragma unroll
          for (int db = 0; db < DB; ++db)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[db][j][e] *= alpha[j];
        }
      }
    }
  };

  // prologue: tile 0's scores, terms and maximum
  wait_dma_all();
  block_barrier();
  if (qw0 >= rows) {  // a wave without rows only loads for the others
    for (int i = 0; i < n; ++i) {
      wait_dma_all();
      block_barrier();
      if (i + 2 < n) {
        issue_k(i + 2);
        if constexpr (BIAS == kTable) build(i + 2);
      }
      if (i + 1 < n) issue_v(i + 1);
    }
    return;
  }
  read_k(lds0 + k_off(0), 0);
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) {
    score_phase(lds0 + k_off(0), ks, sa);
    score_sched(ks, false);
    __builtin_amdgcn_sched_barrier(0);
  }
  {
    terms(sa, 0);
    float mx[2], alpha[2];
    lane_max(sa, mx);
    update_max(mx, alpha);  // o and l are zero: nothing to rescale
  }
  using T_ = std::true_type;
  using F_ = std::false_type;
  int i = 0;
  for (; i + 2 < n; i += 2) {
    iteration(i, sa, sb, T_{});
    iteration(i + 1, sb, sa, T_{});
  }
  if (n - i == 2) {
    iteration(i, sa, sb, T_{});
    iteration(i + 1, sb, sa, F_{});
  } else {
    iteration(i, sa, sb, F_{});
  }

  float inv[2], bad = 0.f;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    l_run[j] = sum4groups(l_run[j]);
    inv[j] = l_run[j] == 0.f ? 0.f : 1.0f / l_run[j];
    m_use[j] = m_run[j] == kNegInf ? 0.f : m_run[j];
    if (qw0 + 16 * j + col < rows) {
      bad = fmaf(l_run[j], 0.f, bad);
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e) bad = fmaf(o[db][j][e], 0.f, bad);
    }
  }
  if (!split && __builtin_amdgcn_ballot_w64(bad != 0.f)) {
    for (int r = qw0; r < min(qw0 + 32, rows); ++r) {
      const int i2 = pk.pos(r);
      score::fwd_row<bf16, D>(a, b, h0 + r - i2 * a.pack, i2, lane);
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int r = qw0 + 16 * j + col;
    if (r >= rows) continue;
    const int i2 = pk.pos(r), h = h0 + r - i2 * a.pack;
    const size_t row = score::lse_at(a, b, h, i2);
    const float l2 = m_use[j] + log2f(l_run[j]);  // (-inf where nothing is seen)
    if (!split) {
      bf16* orow = score::o_row<bf16, D>(a, b, i2, h) + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const float v[4] = {o[db][j][0] * inv[j], o[db][j][1] * inv[j], o[db][j][2] * inv[j],
                            o[db][j][3] * inv[j]};
        store4(orow + 16 * db, v);
      }
      if (g == 0) a.lse[row] = l2 * kLn2;
    } else {
      float* prow = po + (part0 + row) * D + 4 * g;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<f32x4*>(prow + 16 * db) =
            f32x4{o[db][j][0] * inv[j], o[db][j][1] * inv[j], o[db][j][2] * inv[j],
                  o[db][j][3] * inv[j]};
      if (g == 0) plse[part0 + row] = l2;
    }
  }
}

// Merge of a split forward, in chunk order: the chunks' outputs weighted by 2^(lse_c -
// lse).
template <int D>
__global__ __launch_bounds__(256) void score_fwd_merge(ScoreArgs a, const float* __restrict__ po,
                                                       const float* __restrict__ plse,
                                                       const int* __restrict__ used) {
  const size_t all = (size_t)a.batch * a.heads * a.seq_q;
  using ML = MergeLanes<D>;
  const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) / ML::kLanes;
  const int g = threadIdx.x % ML::kLanes, lane = threadIdx.x & 63;
  const size_t row = min(at, all - 1);
  const int i = (int)(row % a.seq_q), bh = (int)(row / a.seq_q);
  const int sets = a.heads / a.pack, b = bh / a.heads, h = bh % a.heads;
  const int blocks = (a.seq_q * a.pack + kRows - 1) / kRows;
  const int nc = used[((size_t)b * sets + h / a.pack) * blocks + (i * a.pack + h % a.pack) / kRows];
  const bool mine = at < all && nc > 1;  // (else its workgroup wrote it)
  float m = kNegInf, l = 0.f, acc[ML::kChunks][8] = {}, bad = 0.f;
  if (mine) {
#pragma unroll 4
    for (int c = 0; c < nc; ++c) m = fmaxf(m, plse[c * all + row]);
    for (int c0 = 0; c0 < nc; c0 += 4) {
      float v[4][ML::kChunks][8], w[4];  // (four loads in flight)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const size_t from = min(c0 + c, nc - 1) * all + row;
#pragma unroll
        for (int x = 0; x < ML::kChunks; ++x) load8(po + from * D + ML::at(g, x), v[c][x]);
        w[c] = plse[from];
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (c0 + c >= nc || w[c] == kNegInf) continue;
        w[c] = exp2_hw(w[c] - m);
        l += w[c];
#pragma unroll
        for (int x = 0; x < ML::kChunks; ++x)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            acc[x][e] = fmaf(w[c], v[c][x][e], acc[x][e]);
            bad = fmaf(v[c][x][e], 0.f, bad);
          }
      }
    }
    bad = fmaf(l, 0.f, bad);
  }
  const bool again = ML::any(bad != 0.f);
  unsigned long long rows = __builtin_amdgcn_ballot_w64(again);
  if (mine && !again) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
    for (int x = 0; x < ML::kChunks; ++x) {
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[x][e] *= inv;
      store8(score::o_row<bf16, D>(a, bh / a.heads, i, bh % a.heads) + ML::at(g, x), acc[x]);
    }
    if (g == 0) a.lse[row] = l == 0.f ? kNegInf : (m + log2f(l)) * kLn2;
  }
  while (rows) {  // rows with a non-finite part, again by the definition
    const int first = __builtin_ctzll(rows);
    const int i2 = __builtin_amdgcn_readlane(i, first), bh2 = __builtin_amdgcn_readlane(bh, first);
    rows &= ~__builtin_amdgcn_ballot_w64(i == i2 && bh == bh2);
    score::fwd_row<bf16, D>(a, bh2 / a.heads, bh2 % a.heads, i2, lane);
  }
}

template <int D>
void fwd_d(const ScoreArgs& a, const ScorePlan& p, void* part, hipStream_t s) {
  float* po = (float*)part;
  const size_t all = (size_t)a.batch * a.heads * a.seq_q;
  float* plse = po ? po + (size_t)p.chunks * all * D : nullptr;
  int* used = po ? (int*)(plse + (size_t)p.chunks * all) : nullptr;
  const unsigned grid = (unsigned)((size_t)a.batch * (a.heads / a.pack) * p.chunks *
                                   ((a.seq_q * a.pack + kRows - 1) / kRows));
  const bool cap = a.cap > 0.f;
  const int bias = a.slopes ? kSlopes : a.table ? kTable : kNoBias;
  const size_t lds = a.table ? bias_lds<D>(a).bytes
                             : tiles_bytes<D>() + kRows * sizeof(RowKeys);
#define PB_FWD(C, B)                                                                          \
  do {                                                                                        \
    if (a.wide) score_fwd_bf16<D, C, B, true><<<grid, 256, lds, s>>>(a, p.chunks, po, plse, used); \
    else score_fwd_bf16<D, C, B, false><<<grid, 256, lds, s>>>(a, p.chunks, po, plse, used);  \
  } while (0)
  if (cap) {
    if (bias == kTable) PB_FWD(true, kTable);
    else if (bias == kSlopes) PB_FWD(true, kSlopes);
    else PB_FWD(true, kNoBias);
  } else {
    if (bias == kTable) PB_FWD(false, kTable);
    else if (bias == kSlopes) PB_FWD(false, kSlopes);
    else PB_FWD(false, kNoBias);
  }
#undef PB_FWD
  if (p.chunks > 1)
    score_fwd_merge<D><<<(unsigned)((all * MergeLanes<D>::kLanes + 255) / 256), 256, 0, s>>>(a, po, plse,
                                                                                      used);
}

}  // namespace

size_t score_fwd_part_bytes(int head_dim, const ScoreArgs& a, const ScorePlan& p) {
  if (p.chunks < 2) return 0;
  const size_t blocks = (size_t)(a.seq_q * a.pack + kRows - 1) / kRows;
  return ((size_t)p.chunks * a.batch * a.heads * a.seq_q * (head_dim + 1) +
          (size_t)a.batch * (a.heads / a.pack) * blocks) * 4;
}

// Split as in attn.hip: where the grid has fewer than 2048 waves, into as many chunks as
// bring it to 1536, of four tiles at least; a tile takes about 1.4 us, the merge 3.5 us
// and its traffic.  Timed without WIDE (us, 1, 2, 4, 8, 12, 16 chunks):
//   4 x 1 token over 8192, 40 heads over 8 x 128   232 123  68  42  35  36
//   1 token over 1000, 8 x 64                       24  18  14  14  14  14
//   2048, 12 x 128, capped                          60  49  50  64  72  81
//   4096, 4 x 128, capped                          105  70  51  56  68  78
//   128 over 4096, 16 over 4 x 128                  77  47  31  25  26  27
//   1024, 8 x 128                                   26  24  23  26  27  27
ScorePlan score_fwd_plan(int head_dim, const ScoreArgs& a) {
  const long long blocks = (long long)a.batch * (a.heads / a.pack) *
                           ((a.seq_q * a.pack + kRows - 1) / kRows);
  const int most = score_most_tiles(a, kRows, kTL);
  if (blocks * 4 >= 2048) return ScorePlan{1};
  const int want = (int)((1536 + blocks * 4 - 1) / (blocks * 4));
  const int m = std::min(want, most / kMinTiles);
  if (m < 2) return ScorePlan{1};
  const ScorePlan q{m};
  const double merge_us = 3.5 + 2.0 * (double)score_fwd_part_bytes(head_dim, a, q) / 8e6;
  return 1.4 * (most - (most + m - 1) / m) < merge_us ? ScorePlan{1} : q;
}

void launch_score_forward_bf16(int head_dim, const ScoreArgs& a, const ScorePlan& p, void* part,
                               hipStream_t s) {
  if (head_dim == 64) fwd_d<64>(a, p, part, s);
  else if (head_dim == 96) fwd_d<96>(a, p, part, s);
  else fwd_d<128>(a, p, part, s);
}

}  // namespace pb

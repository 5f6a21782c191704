// Gradients of attention with terms in its scores, bf16, on v_mfma_f32_32x32x16_bf16.
//
// Row terms (lse in base 2, delta) come from a launch of their own, laid out in the order of
// the blocks' rows.  Then one launch has two roles, as in attn.hip:
//   dK, dV: 128 keys over 32-row tiles of the heads that share the key head, so that the
//     gradients of shared heads are one sum (of more than eight heads several, merged in
//     order);
//   dQ: 128 rows over 64-key tiles.
// P = 2^(s - lse) with the scores' terms as in the forward, dS = P (dP - delta), times
// 1 - tanh^2 with a cap for dQ and dK.  How many tiles a block has depends on documents
// that only the device knows, so a block that the plan cuts shares its own tiles out.
//
// P and dS enter the products as bf16.  WIDE adds those with what that rounding leaves (16
// bits of each in all), and its delta = sum of P dP is summed over the tiles in a launch
// before (scores and dP once more); without, delta = sum of dO O, whose O is rounded.  In
// norm dq, dk and dv are off by 1.66e-3 with, their own rounding; without, dv 2.1e-3 to
// 2.4e-3, dq and dk 2.6e-3 to 2.8e-3 over rows of 500 keys and more, 5.2e-3 over rows of two.
//
// The table's gradient sums dz = P (dP - delta) by bucket, and there delta has to be
// better than a sum of dO O: dQ's rows also give e = the sum of their dz, by which delta is
// off (the exact ones sum to zero), and the sums of dz and of P over the tiles beyond the
// last bucket's first distance.  A last launch goes over the other tiles again, with the
// row terms put right.
//
// Bound by the vector instructions of the terms beside the products, at two waves a SIMD
// (registers).  Measured (WIDE, and without): 4096 tokens of packed documents, 16 heads over
// 4 x 128, capped 346 us (229), 287 TFLOP/s of 10 d operations a pair, where 24 d (14 d) are
// done; matrix cores busy 32% and vector instructions 42% of the two roles' launch, 21% and
// 53% of the row terms'.  4096 x 16 heads of 64: without terms 265 (169; attn.hip 240), capped
// 322 (217), with a table 301 (202) and its gradient 331 (232).
//
// Non-finite values behind the mask are met as in the forward.
#include "kernels.h"
#include "score_attn_tiles.h"

namespace pb {
namespace {

#define PB_INLINE __attribute__((always_inline))

constexpr int kNoBias = 0, kSlopes = 1, kTable = 2;
constexpr int kBlockK = 128, kTileQ = 32;  // dK, dV: keys of a workgroup, rows of a tile
constexpr int kBlockQ = 128, kTileK = 64;  // dQ: rows of a workgroup, keys of a tile
constexpr int kSums = 5;  // of a row: e; dz and P beyond the last bucket, of either side

// (By value: a choice of two members would be one of their addresses, and keep the whole
// of the kernel's arguments in memory.)
template <typename T>
PB_DEV T pick(bool first, T x, T y) {
  return first ? x : y;
}

// Rows of all blocks: [batch][head / pack][position][head mod pack].
PB_DEV size_t packed_row(const ScoreArgs& a, int hb, int r) {
  return (size_t)hb * a.seq_q * a.pack + r;
}

// A row's lse in base 2; of one that sees nothing infinity, for probabilities of 2^-inf.
PB_DEV float base2(float L) { return L == kNegInf ? -kNegInf : L * kLog2e; }

// ------------------------------------------------------------- row terms
// Both operands read once, D / 8 lanes a row (four for head_dim 96).
template <int D>
__global__ __launch_bounds__(256) void score_terms(ScoreArgs a, float* __restrict__ L2,
                                                   float* __restrict__ minus_delta) {
  constexpr int kLanes = D == 96 ? 4 : D / 8, kChunks = D / 8 / kLanes;
  const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const size_t all = (size_t)a.batch * a.seq_q * a.heads;
  const int l = threadIdx.x % kLanes;
  // heads fastest: neighbouring rows of memory
  const size_t x = min(at, all - 1);
  const int h = (int)(x % a.heads), i = (int)(x / a.heads % a.seq_q);
  const int b = (int)(x / a.heads / a.seq_q);
  const bf16 *o = score::o_row<bf16, D>(a, b, i, h), *g = score::do_row<bf16, D>(a, b, i, h);
  float acc = 0.f;
#pragma unroll
  for (int c = 0; c < kChunks; ++c) {
    float u[8], v[8];
    load8(o + 8 * (l + c * kLanes), u);
    load8(g + 8 * (l + c * kLanes), v);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc = fmaf(u[e], v[e], acc);
  }
#pragma unroll
  for (int s = 1; s < kLanes; s <<= 1) acc += __shfl_xor(acc, s, 64);
  if (l != 0 || at >= all) return;
  const float L = a.lse[score::lse_at(a, b, h, i)];
  const size_t to = packed_row(a, b * (a.heads / a.pack) + h / a.pack, i * a.pack + h % a.pack);
  L2[to] = base2(L);
  minus_delta[to] = L == kNegInf ? 0.f : -acc;
}

// A TL-row tile in the layout of dma_tile (attn_tiles.h): offset(0 .. TL - 1) is that of a
// row from base, in bytes.
template <int D, int TL, int NW, typename Offset>
PB_DEV void dma_rows(const bf16* base, Offset offset, uint32_t lds_tile, int wave, int lane) {
  constexpr int RB = 2 * D, NP = TL * RB / 1024;
  asm("" : "+v"(lane));  // (nothing derived from it is kept over a loop)
#pragma unroll
  for (int i = 0; i < (NP + NW - 1) / NW; ++i) {
    const int pc = NP % NW == 0 ? wave * (NP / NW) + i : i * NW + wave;
    if (NP % NW != 0 && pc >= NP) break;  // wave-uniform
    const int p = pc * 1024 + 16 * lane;
    const int r = p / RB, slot = (p / 16) % (RB / 16);
    dma16s(base, offset(r) + 16 * chunk_at<D>(r, slot),
           __builtin_amdgcn_readfirstlane(lds_tile + pc * 1024));
  }
}

// A lane's places in a tile of dma_rows: its reads' addresses follow from three of them by
// an exclusive or or an addition each (frag_row and frag_tr would keep one for each step
// over the loop, some fifty registers).  Tiles begin at multiples of 256 bytes.
template <int D>
struct LaneReads {
  uint32_t row[D == 96 ? 2 : 1];  // features 8 fh .. + 7 of row fr
  uint32_t tr[2];                 // rows 4 fh + j and 8 more, features (fr & 16) + 4 q
  PB_DEV explicit LaneReads(int lane) {
    const int fr = lane & 31, fh = lane >> 5, i = lane & 15, j = i >> 2, q = i & 3;
    row[0] = fr * 2 * D + 16 * chunk_at<D>(fr, fh);
    if constexpr (D == 96) row[1] = fr * 2 * D + 16 * (chunk_at<D>(fr, fh) ^ 2);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int t = 4 * fh + j + 8 * k;
      tr[k] = t * 2 * D + 16 * chunk_at<D>(t, 2 * (fr >> 4) + (q >> 1)) + 8 * (q & 1);
    }
  }
  // the places in the tile at lds (a fresh copy: nothing derived is kept over a loop)
  PB_DEV LaneReads at(uint32_t lds) const {
    LaneReads x = *this;
    x.row[0] += lds;
    asm volatile("" : "+v"(x.row[0]));
    if constexpr (D == 96) {
      x.row[1] += lds;
      asm volatile("" : "+v"(x.row[1]));
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x.tr[k] += lds;
      asm volatile("" : "+v"(x.tr[k]));
    }
    return x;
  }
  // 8 features of step ks, `bytes` further on
  PB_DEV bf16x8 rows(int ks, int bytes) const {
    if constexpr (D == 96) return lds_b128(row[ks & 1] + 64 * (ks >> 1) + bytes);
    else return lds_b128((row[0] ^ (32 * ks)) + bytes);
  }
  // 8 rows (as frag_tr) of features 32 db + fr, k-step s
  PB_DEV bf16x8 cols(int db, int s, int bytes) const {
    const int more = s * 16 * 2 * D + bytes;
    if constexpr (D == 96) return lds_tr_pair(tr[0] + 64 * db + more, tr[1] + 64 * db + more);
    else return lds_tr_pair((tr[0] ^ (64 * db)) + more, (tr[1] ^ (64 * db)) + more);
  }
  static PB_DEV bf16x8 lds_tr_pair(uint32_t x, uint32_t y) {
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PB_LDS s16x4*)x);
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PB_LDS s16x4*)y);
    const bf16x4 a4 = __builtin_bit_cast(bf16x4, a), b4 = __builtin_bit_cast(bf16x4, b);
    return bf16x8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
  }
};

// A wave's 32 rows of results, f x, from accumulators (a lane has row l & 31, features 32 db
// + 8 j + 4 (l >> 5) + e) to memory by way of `lds` (the wave's own, 64 D bytes), so that
// lanes store neighbouring pieces: a lane's own four features at a time make 32 pieces of
// lines a store (dK and dV of 2048 tokens, 40 heads, window 512: 155 us against 146 for all
// gradients; dQ's stores cost nothing measurable).
PB_DEV void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int D>
PB_DEV void store_rows(unsigned char* lds, const f32x16 (&x)[D / 32], float f, bf16* out, size_t ld,
                       int rows, int lane) {
  asm("" : "+v"(lane));  // (nothing derived from it is kept over the loop before)
  const int fr = lane & 31, fh = lane >> 5;
  lds_done();
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = x[db][4 * j + e] * f;
      store4((bf16*)(lds + fr * 2 * D + 16 * chunk_at<D>(fr, 4 * db + j) + 8 * fh), v);
    }
  lds_done();
#pragma unroll
  for (int n = 0; n < D / 16; ++n) {
    const int r = (64 * n + lane) / (D / 8), c = (64 * n + lane) % (D / 8);
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + r * 2 * D + 16 * chunk_at<D>(r, c));
    if (r < rows) *reinterpret_cast<u32x4*>(out + r * ld + 8 * c) = v;
  }
}
// The same in fp32, rows of D.
template <int D>
PB_DEV void store_rows(unsigned char* lds, const f32x16 (&x)[D / 32], float f, float* out, int rows,
                       int lane) {
  asm("" : "+v"(lane));
  const int fr = lane & 31, fh = lane >> 5;
#pragma unroll
  for (int db = 0; db < D / 32; ++db) {
    lds_done();
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4*>(lds + fr * 128 + 16 * ((2 * j + fh) ^ (fr & 7))) =
          f32x4{x[db][4 * j] * f, x[db][4 * j + 1] * f, x[db][4 * j + 2] * f, x[db][4 * j + 3] * f};
    lds_done();
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const int r = 8 * n + (lane >> 3), c = lane & 7;
      const f32x4 v = *reinterpret_cast<const f32x4*>(lds + r * 128 + 16 * (c ^ (r & 7)));
      if (r < rows) *reinterpret_cast<f32x4*>(out + (size_t)r * D + 32 * db + 4 * c) = v;
    }
  }
}

// What k-step s of p (as probs_frag) leaves.
PB_DEV bf16x8 rest_frag(const f32x16* p, int s, const bf16x8& rounded) {
  const f32x16& a = p[s >> 1];
  const int o = 8 * (s & 1);
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; e += 2) {
    const bf16x2 x = rest_of(bf16x2{rounded[e], rounded[e + 1]}, a[o + e], a[o + e + 1]);
    r[e] = x[0], r[e + 1] = x[1];
  }
  return r;
}

struct BwdWork {
  float *L2, *minus_delta;  // row terms, in the blocks' order
  float *pdk, *pdv, *pdq;   // partial results of split blocks, [chunk][row][D]
  float* sums;              // [chunk][kSums][rows] (with dtable)
  float* pdelta;            // parts of delta, [chunk][rows] (of blocks in chunks)
  int *kv_used, *q_used, *d_used;  // chunks of each block, [set][batch, head][block]
  int kv_nc, q_nc, d_nc;           // at most
};
constexpr int kMinTilesKv = 12, kMinTilesQ = 4, kMinTilesD = 4;  // of a chunk
__host__ __device__ inline int row_blocks(const ScoreArgs& a) {
  return (a.seq_q * a.pack + kBlockQ - 1) / kBlockQ;
}
__host__ __device__ inline int key_blocks(const ScoreArgs& a) {
  return (a.seq_k + kBlockK - 1) / kBlockK;
}

// ------------------------------------------------------------------ dK, dV
// A wave has 32 keys: K and both accumulators in registers, V in LDS beside the row
// tiles (each with its row terms, positions and biases), which all four waves share.
// S = Q K^T and dP = dO V^T come out with a key a lane and four rows an element group;
// P and dS go from there into dV^T += dO^T P and dK^T += Q^T dS.
// (A "P" and a "dS" wave for each 32 keys, as in attn.hip, take 24 registers less but
// hand P over through LDS: the wave with the scores' terms has twice the other's work,
// and each waits for the other once a tile.)
template <int D>
struct KvLds {
  static constexpr int kV = kBlockK * 2 * D;
  static constexpr int kTile = kTileQ * 2 * D;
  // Q, dO, then of each row: lse, -delta, position, and its bias (slope, place or value)
  static constexpr int kStage = 2 * kTile + 4 * kTileQ * 4;
  static constexpr int kBytes = kV + 2 * kStage;
  static __host__ __device__ BiasLds bias(const ScoreArgs& a) {
    return BiasLds(kBytes, a.buckets, a.pack, (kTileQ + a.pack - 1) / a.pack + 1, kBlockK);
  }
};

template <int D, bool CAP, int BIAS, bool WIDE>
PB_DEV void dkdv_block(const ScoreArgs& a, const BwdWork& w, int bx, int hb) {
  constexpr int TL = kTileQ, NB = kBlockK, TB = TL * 2 * D;
  using L = KvLds<D>;
  constexpr int STAGE = L::kStage;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  const int b = hb / a.kv_heads, kvh = hb % a.kv_heads;
  // chunk: a set of heads, and a run of its row tiles
  const int parts = a.group / a.pack, subs = w.kv_nc / parts;
  const int chunk = bx % w.kv_nc, kblk = bx / w.kv_nc, k0 = kblk * NB;
  const int set = chunk / subs, h0 = kvh * a.group + set * a.pack;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int fr = lane & 31, fh = lane >> 5;
  const int off = a.seq_k - a.seq_q;
  const Packed pk(a.pack);
  const int key = k0 + 32 * wave + fr, key_c = min(key, a.seq_k - 1);

  // queries that see the lane's key: positions sf .. sf + sn - 1; all keys' together, and
  // the wave's: any of them, and all
  int sf = 0, sn = 0, lo = 0x7fffffff, hi = -1;
  for (int x = 0; x < NB / 64; ++x) {
    const int j = k0 + 64 * x + lane;
    int f = 0, n = 0;
    if (j < a.seq_k) {
      const Bounds d = bounds_of(a, b, j);
      if (d.de > d.ds) {
        f = max(score::seen_first(a, d, j), off);
        n = max(score::seen_last(a, d, j) - f + 1, 0);
      }
    }
    if (n > 0) lo = min(lo, f), hi = max(hi, f + n - 1);
    if (wave / 2 == x) {
      sf = __shfl(f, 32 * (wave & 1) + fr, 64);
      sn = __shfl(n, 32 * (wave & 1) + fr, 64);
    }
  }
  lo = wave_imin(lo), hi = wave_imax(hi);
  const int any_lo = wave_imin(sn > 0 ? sf : 0x7fffffff), any_hi = wave_imax(sf + sn - 1);
  const int all_lo = wave_imax(sn > 0 ? sf : 0x7fffffff), all_hi = wave_imin(sf + sn - 1);
  const int r_lo = hi < 0 ? 0 : (lo - off) * a.pack, r_hi = hi < 0 ? -1 : (hi - off + 1) * a.pack - 1;
  const int t_lo = r_lo / TL, tiles = hi < 0 ? 0 : r_hi / TL - t_lo + 1;
  const Share share(tiles, subs, kMinTilesKv);
  const int t_begin = chunk % subs * share.size, nt = min(tiles - t_begin, share.size);
  const bool split = parts > 1 || share.used > 1;
  if (w.kv_nc > 1 && tid == 0 && chunk % subs == 0)
    w.kv_used[((size_t)set * a.batch * a.kv_heads + hb) * key_blocks(a) + kblk] = share.used;
  if (nt <= 0) {
    if (chunk % subs || split) return;  // fewer chunks than there may be
    for (int x = tid; x < NB * (D / 8); x += 256) {  // nobody sees these keys
      const int j = k0 + x / (D / 8);
      if (j >= a.seq_k) break;
      const size_t at = ((size_t)b * a.seq_k + j) * a.ld_dkv + kvh * D + 8 * (x % (D / 8));
      *reinterpret_cast<u32x4*>((bf16*)a.dk + at) = u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>((bf16*)a.dv + at) = u32x4{0, 0, 0, 0};
    }
    return;
  }

  auto tile_row = [&](int i) PB_INLINE { return (t_lo + t_begin + i) * TL; };
  auto tile_span = [&](int i, int& p0, int& p1) PB_INLINE {  // positions of tile i
    const int r = tile_row(i);
    p0 = off + pk.pos(r);
    p1 = off + pk.pos(r + TL - 1);
  };
  const BiasLds bl = L::bias(a);
  const int bias_last = BIAS == kTable ? a.first[a.side - 1] : 0;
  auto uniform = [&](int i) PB_INLINE {
    int p0, p1;
    tile_span(i, p0, p1);
    return bias_uniform(a, bias_last, p0 - k0 - NB + 1, p1 - k0);
  };
  const bf16* q0 = score::q_row<bf16, D>(a, b, 0, h0);
  const bf16* g0 = score::do_row<bf16, D>(a, b, 0, h0);
  const size_t row0 = packed_row(a, b * (a.heads / a.pack) + h0 / a.pack, 0);
  auto issue_stage = [&](int i) PB_INLINE {
    const int r0 = tile_row(i);
    const uint32_t at = lds0 + L::kV + (i & 1) * STAGE;
    // rows beyond those that see any of the keys are read from the nearest that do
    auto row_of = [&](int r) PB_INLINE { return max(r_lo, min(r0 + r, r_hi)); };
    const int y0 = pk.pos(max(r_lo, r0));  // (of the tile's first row that is read)
    auto offset = [&](int r, int ld) PB_INLINE {
      const int x = row_of(r), y = pk.pos(x);
      return (uint32_t)(y - y0) * (uint32_t)(2 * ld) + (uint32_t)(x - y * a.pack) * (2 * D);
    };
    dma_rows<D, TL, 4>(q0 + (size_t)y0 * a.ld_q,
                       [&](int r) PB_INLINE { return offset(r, a.ld_q); }, at, wave, lane);
    dma_rows<D, TL, 4>(g0 + (size_t)y0 * a.ld_do,
                       [&](int r) PB_INLINE { return offset(r, a.ld_do); }, at + TB, wave, lane);
    if (wave == 0)
      dma4(pick(lane < 32, w.L2, w.minus_delta) + row0 + row_of(lane & 31),
           __builtin_amdgcn_readfirstlane(at + 2 * TB));
    if (wave == 1 && lane < TL) {
      const int r = r0 + lane, y = pk.pos(r), hh = r - y * a.pack;
      int* rows_of = (int*)(smem + L::kV + (i & 1) * STAGE + 2 * TB + 2 * TL * 4);
      rows_of[lane] = y + off;
      if constexpr (BIAS == kSlopes) ((float*)rows_of)[TL + lane] = -a.slopes[h0 + hh] * kLog2e;
      if constexpr (BIAS == kTable) {
        const int u = uniform(i);
        if (u < 0) rows_of[TL + lane] = hh * bl.stride + off + pk.pos(r0 + TL - 1) - (y + off);
        else ((float*)rows_of)[TL + lane] = ((const float*)(smem + bl.tab))[u * a.pack + hh];
      }
    }
  };
  auto build = [&](int i) PB_INLINE {
    int p0, p1;
    tile_span(i, p0, p1);
    if (uniform(i) < 0) bias_tile(a, bl, smem, i & 1, a.pack, p1 - k0, tid, 256);
  };
  dma_rows<D, NB, 4>(score::kv_row<bf16, D>(a, a.v, b, k0, kvh), [&](int r) PB_INLINE {
    return (uint32_t)min(r, a.seq_k - 1 - k0) * (uint32_t)(2 * a.ld_kv);
  }, lds0, wave, lane);
  if constexpr (BIAS == kTable) {
    bias_prologue(a, bl, smem, h0, a.pack, tid, 256);
    __syncthreads();
    build(0);
  }
  issue_stage(0);
  const bf16* kr = score::kv_row<bf16, D>(a, a.k, b, key_c, kvh);
  bf16x8 kf[D / 16];
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) kf[ks] = load_row_frag(kr + 16 * ks + 8 * fh, key < a.seq_k);
  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) dk[i] = dv[i] = zero16();
  const Cap cap(a.scale, CAP ? a.cap : 1.f);
  const float c2 = CAP ? cap.top : a.scale * kLog2e;  // (of tanh, with a cap)
  const LaneReads<D> places(lane);

  for (int i = 0; i < nt; ++i) {
    __builtin_amdgcn_s_setprio(0);
    wait_dma_all();   // tile i, requested an iteration ago
    block_barrier();  // ... for every wave; and every wave is done with tile i - 1
    if (i + 1 < nt) {
      issue_stage(i + 1);
      if constexpr (BIAS == kTable) build(i + 1);
    }
    int p0, p1;
    tile_span(i, p0, p1);
    if (p1 < any_lo || p0 > any_hi) continue;
    const uint32_t stage = L::kV + (i & 1) * STAGE;
    const LaneReads<D> qr = places.at(lds0 + stage), vr = places.at(lds0 + 32 * wave * 2 * D);
    const float* ls = (const float*)(smem + stage + 2 * TB);
    const int* row_pos = (const int*)(ls + 2 * TL);
    // Lane holds key `key` and rows r0 + 8 j + 4 fh + e of element 4 j + e.
    f32x16 sc[1] = {zero16()}, dp;
#pragma unroll
    for (int j = 0; j < 4; ++j) {  // dP - delta
      const f32x4 D4 = *reinterpret_cast<const f32x4*>(ls + TL + 8 * j + 4 * fh);
#pragma unroll
      for (int e = 0; e < 4; ++e) dp[4 * j + e] = D4[e];
    }
    // (fragments one step ahead of their products, and no further: registers; a wave at
    // its products goes before the SIMD's other one: capped scores 3%)
    bf16x8 fq[2], fg[2], fv[2];
    auto read = [&](int ks) PB_INLINE {
      fq[ks & 1] = qr.rows(ks, 0);
      fg[ks & 1] = qr.rows(ks, TB);
      fv[ks & 1] = vr.rows(ks, 0);
    };
    __builtin_amdgcn_s_setprio(1);
    read(0);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      if (ks + 1 < D / 16) read(ks + 1);
      sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fq[ks & 1], kf[ks], sc[0], 0, 0, 0);
      dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fg[ks & 1], fv[ks & 1], dp, 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    if constexpr (CAP) {
      cap.apply(sc, [&](int, int e, float d) PB_INLINE { dp[e] *= d; });
    }
    if constexpr (BIAS == kSlopes) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 P4 = *reinterpret_cast<const u32x4*>(row_pos + 8 * j + 4 * fh);
        const f32x4 X4 = *reinterpret_cast<const f32x4*>(row_pos + TL + 8 * j + 4 * fh);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sc[0][4 * j + e] = fmaf(X4[e], fabsf((float)((int)P4[e] - key)), sc[0][4 * j + e] * c2);
      }
    }
    if constexpr (BIAS == kTable) {
      const bool near = uniform(i) < 0;
      const float* bt = (const float*)(smem + bl.tile(i & 1, a.pack)) + (key - k0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        u32x4 X4 = *reinterpret_cast<const u32x4*>(row_pos + TL + 8 * j + 4 * fh);
        if (near)
#pragma unroll
          for (int e = 0; e < 4; ++e) X4[e] = __float_as_uint(bt[(int)X4[e]]);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sc[0][4 * j + e] = fmaf(sc[0][4 * j + e], c2, __uint_as_float(X4[e]));
      }
    }
    if (!(p0 >= all_lo && p1 <= all_hi)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const u32x4 P4 = *reinterpret_cast<const u32x4*>(row_pos + 8 * j + 4 * fh);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          sc[0][4 * j + e] =
              (unsigned)((int)P4[e] - sf) < (unsigned)sn ? sc[0][4 * j + e] : kNegInf;
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 L4 = *reinterpret_cast<const f32x4*>(ls + 8 * j + 4 * fh);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float z = sc[0][4 * j + e];
        sc[0][4 * j + e] = exp2_hw(BIAS != kNoBias ? z - L4[e] : fmaf(z, c2, -L4[e]));
        dp[4 * j + e] *= sc[0][4 * j + e];
      }
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int s2 = 0; s2 < TL / 16; ++s2) {
      const bf16x8 pf = probs_frag(sc, s2), df = probs_frag(&dp, s2);
      bf16x8 pl, dl;
      if constexpr (WIDE) pl = rest_frag(sc, s2, pf), dl = rest_frag(&dp, s2, df);
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const bf16x8 gc = qr.cols(db, s2, TB), qc = qr.cols(db, s2, 0);
        dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gc, pf, dv[db], 0, 0, 0);
        dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qc, df, dk[db], 0, 0, 0);
        if constexpr (WIDE) {
          dv[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(gc, pl, dv[db], 0, 0, 0);
          dk[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(qc, dl, dk[db], 0, 0, 0);
        }
      }
    }
  }

  const int j0 = k0 + 32 * wave;
  unsigned char* mine = smem + 32 * wave * 2 * D;  // the wave's V, of which it is done
  if (split) {
    const size_t keys = (size_t)a.batch * a.kv_heads * a.seq_k;
    const size_t at = ((size_t)chunk * keys + (size_t)hb * a.seq_k + j0) * D;
    store_rows<D>(mine, dk, a.dscale, w.pdk + at, a.seq_k - j0, lane);
    store_rows<D>(mine, dv, 1.f, w.pdv + at, a.seq_k - j0, lane);
    return;
  }
  float bad = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) bad = fmaf(dk[db][e], 0.f, fmaf(dv[db][e], 0.f, bad));
  if (__builtin_amdgcn_ballot_w64(key < a.seq_k && bad != 0.f)) {
    for (int j = j0; j < min(j0 + 32, a.seq_k); ++j)
      score::dkdv_row<bf16, D>(a, b, kvh, j, lane);
    return;
  }
  const size_t at = ((size_t)b * a.seq_k + j0) * a.ld_dkv + kvh * D;
  store_rows<D>(mine, dk, a.dscale, (bf16*)a.dk + at, a.ld_dkv, a.seq_k - j0, lane);
  store_rows<D>(mine, dv, 1.f, (bf16*)a.dv + at, a.ld_dkv, a.seq_k - j0, lane);
}

// --------------------------------------------------------- rows over key tiles
// What dQ and the table's gradient share: 128 rows, a lane's row and its P and dz of a
// 64-key tile.
template <int D, bool CAP, int BIAS>
struct RowTiles {
  const ScoreArgs& a;
  const BwdWork& w;
  unsigned char* smem;
  int b, h0, kvh, r0, rows, off, lane, wave, fr, fh, r, i, h, p;
  int p_first, p_last, w_first, w_last;  // positions of the block, and of the wave
  float L2, dl, slope2;
  int bias_at, bias_last;
  RowKeys keys;
  bf16x8 qf[D / 16], gf[D / 16];
  Cap cap;
  BiasLds bl;
  Packed pk;

  // terms: whether the row terms are there
  PB_DEV RowTiles(const ScoreArgs& a_, const BwdWork& w_, unsigned char* s, int lds_at, int blk,
                  int hb, bool terms = true)
      : a(a_), w(w_), smem(s), cap(a_.scale, CAP ? a_.cap : 1.f),
        bl(lds_at, a_.buckets, a_.pack, (kBlockQ + a_.pack - 1) / a_.pack + 1, kTileK),
        pk(a_.pack) {
    const int sets = a.heads / a.pack;
    b = hb / sets, h0 = hb % sets * a.pack, kvh = h0 / a.group;
    rows = a.seq_q * a.pack, off = a.seq_k - a.seq_q, r0 = blk * kBlockQ;
    lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    fr = lane & 31, fh = lane >> 5;
    r = r0 + 32 * wave + fr;
    const int rc = min(r, rows - 1);
    i = pk.pos(rc), h = h0 + rc - i * a.pack, p = i + off;
    p_first = off + pk.pos(r0), p_last = off + pk.pos(min(r0 + kBlockQ, rows) - 1);
    w_first = off + pk.pos(min(r0 + 32 * wave, rows - 1));
    w_last = off + pk.pos(min(r0 + 32 * wave + 31, rows - 1));
    const bf16 *q = score::q_row<bf16, D>(a, b, i, h), *g = score::do_row<bf16, D>(a, b, i, h);
    keys = row_keys(a, b, p);
    if (r >= rows) keys = RowKeys{0, 0, 0, 0};
    // (a row that sees nothing may hold anything)
    const bool any = keys.len > 0 || keys.plen > 0;
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      qf[ks] = load_row_frag(q + 16 * ks + 8 * fh, any);
      gf[ks] = load_row_frag(g + 16 * ks + 8 * fh, any);
    }
    const size_t at = packed_row(a, hb, rc);
    L2 = terms ? w.L2[at] : base2(a.lse[score::lse_at(a, b, h, i)]);
    dl = terms ? -w.minus_delta[at] : 0.f;
    slope2 = BIAS == kSlopes ? -a.slopes[h] * kLog2e : 0.f;
    bias_last = BIAS == kTable ? a.first[a.side - 1] : 0;
    bias_at = BIAS == kTable ? (h - h0) * bl.stride + (p_last - p) + 4 * fh : 0;
  }
  PB_DEV void tables() {
    bias_prologue(a, bl, smem, h0, a.pack, threadIdx.x, 256);
    __syncthreads();
  }
  PB_DEV int uniform(int kv0) const {
    return bias_uniform(a, bias_last, p_first - kv0 - kTileK + 1, p_last - kv0);
  }
  PB_DEV int wave_uniform(int kv0) const {
    return bias_uniform(a, bias_last, w_first - kv0 - kTileK + 1, w_last - kv0);
  }
  PB_DEV void build(int kv0, int buf) {
    if (uniform(kv0) < 0) bias_tile(a, bl, smem, buf, a.pack, p_last - kv0, threadIdx.x, 256);
  }
  PB_DEV void request(const KeyTiles& kt, int kv0, uint32_t lds_k, uint32_t lds_v) const {
    const int lo = max(kt.lo - kv0, 0), hi = min(kt.hi - kv0, kTileK - 1);
    const bf16 *k = score::kv_row<bf16, D>(a, a.k, b, kv0, kvh),
               *v = score::kv_row<bf16, D>(a, a.v, b, kv0, kvh);
    auto offset = [&](int x) PB_INLINE {
      return (uint32_t)max(lo, min(x, hi)) * (uint32_t)(2 * a.ld_kv);
    };
    dma_rows<D, kTileK, 4>(k, offset, lds_k, wave, lane);
    dma_rows<D, kTileK, 4>(v, offset, lds_v, wave, lane);
  }
  // P and dz of the lane's row and keys kv0 + 32 h2 + 8 j + 4 fh + e (element 4 j + e).
  // see: the row's keys of the tile.  SLOPE: 0, dz as it is; 1, times what the cap leaves;
  // 2, that apart, in slope.
  // kr: the lane's places in the K tile; V's is kTileK rows further on.
  template <int SLOPE>
  PB_DEV void pair(int kv0, int h2, int buf, const LaneReads<D>& kr, uint64_t see,
                    f32x16 (&pr)[1], f32x16 (&dz)[1], f32x16& slope) {
    const float c2 = CAP ? cap.top : a.scale * kLog2e;  // (of tanh, with a cap)
    pr[0] = zero16();
    dz[0] = zero16();
    bf16x8 fk[2], fv[2];
    auto read = [&](int ks) PB_INLINE {
      fk[ks & 1] = kr.rows(ks, 32 * h2 * 2 * D);
      fv[ks & 1] = kr.rows(ks, (kTileK + 32 * h2) * 2 * D);
    };
    read(0);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
      if (ks + 1 < D / 16) read(ks + 1);
      pr[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fk[ks & 1], qf[ks], pr[0], 0, 0, 0);
      dz[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fv[ks & 1], gf[ks], dz[0], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) dz[0][x] -= dl;
    if constexpr (CAP)
      cap.apply(pr, [&](int, int x, float d) PB_INLINE {
        if constexpr (SLOPE == 1) dz[0][x] *= d;
        if constexpr (SLOPE == 2) slope[x] = d;
      });
    if constexpr (BIAS == kSlopes) {
      const float d0 = (float)(p - kv0 - 32 * h2 - 4 * fh);
#pragma unroll
      for (int x = 0; x < 16; ++x)
        pr[0][x] = fmaf(slope2, fabsf(d0 - (float)(8 * (x >> 2) + (x & 3))), pr[0][x] * c2);
    }
    if constexpr (BIAS == kTable) {
      const int u = uniform(kv0);
      if (u < 0) {
        const float* bt = (const float*)(smem + bl.tile(buf, a.pack)) + bias_at + 32 * h2;
#pragma unroll
        for (int x = 0; x < 16; ++x) pr[0][x] = fmaf(pr[0][x], c2, bt[8 * (x >> 2) + (x & 3)]);
      } else {
        const float f = ((const float*)(smem + bl.tab))[u * a.pack + h - h0];
#pragma unroll
        for (int x = 0; x < 16; ++x) pr[0][x] = fmaf(pr[0][x], c2, f);
      }
    }
    const uint32_t mine = (uint32_t)(see >> (32 * h2));
    if (__builtin_amdgcn_ballot_w64(mine != ~0u)) {
      const uint32_t bits = mine >> (4 * fh);
#pragma unroll
      for (int x = 0; x < 16; ++x)
        pr[0][x] = bits & (1u << (8 * (x >> 2) + (x & 3))) ? pr[0][x] : kNegInf;
    }
#pragma unroll
    for (int x = 0; x < 16; ++x) {
      pr[0][x] = exp2_hw(BIAS != kNoBias ? pr[0][x] - L2 : fmaf(pr[0][x], c2, -L2));
      dz[0][x] *= pr[0][x];
      // (behind the mask dP may be anything: sums over a row take none of it)
      if constexpr (BIAS == kTable || SLOPE == 0) dz[0][x] = pr[0][x] == 0.f ? 0.f : dz[0][x];
    }
  }
};

// n key tiles of a block from t_begin on, by way of two slots of K and V: f(first key, the
// row's keys of the tile, slot, places of K) for those that the wave sees any of.
template <int D, bool CAP, int BIAS, typename F>
PB_DEV void each_tile(RowTiles<D, CAP, BIAS>& t, const KeyTiles& kt, int t_begin, int n,
                      uint32_t lds0, F f) {
  constexpr int TB = kTileK * 2 * D;
  auto kv_of = [&](int i) PB_INLINE { return kt.tile(t_begin + i) * kTileK; };
  auto k_off = [&](int s) PB_INLINE { return lds0 + (2 * s) * TB; };
  auto v_off = [&](int s) PB_INLINE { return lds0 + (2 * s + 1) * TB; };
  if constexpr (BIAS == kTable) {
    t.tables();
    t.build(kv_of(0), 0);
  }
  t.request(kt, kv_of(0), k_off(0), v_off(0));
  const LaneReads<D> places(t.lane);
  for (int i = 0; i < n; ++i) {
    const int cur = i & 1, kv0 = kv_of(i);
    wait_dma_all();
    block_barrier();
    if (i + 1 < n) {
      t.request(kt, kv_of(i + 1), k_off(cur ^ 1), v_off(cur ^ 1));
      if constexpr (BIAS == kTable) t.build(kv_of(i + 1), cur ^ 1);
    }
    const uint64_t see = t.keys.bits(kv0);
    if (!__builtin_amdgcn_ballot_w64(see != 0)) continue;
    f(kv0, see, cur, places.at(lds0 + (2 * cur) * TB));
  }
}

template <int D, bool CAP, int BIAS, bool WIDE>
PB_DEV void dq_block(const ScoreArgs& a, const BwdWork& w, int bx, int hb) {
  constexpr int TB = kTileK * 2 * D;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  const int nblk = (a.seq_q * a.pack + kBlockQ - 1) / kBlockQ;
  const int chunk = bx % w.q_nc;
  RowTiles<D, CAP, BIAS> t(a, w, smem, 4 * TB, nblk - 1 - bx / w.q_nc, hb);
  const KeyTiles kt = key_tiles<kTileK>(a, t.b, t.p_first, t.p_last, t.lane);
  const Share share(kt.n, w.q_nc, kMinTilesQ);
  const int t_begin = chunk * share.size, n = min(kt.n - t_begin, share.size);
  const bool split = share.used > 1;
  if (chunk >= max(share.used, 1)) return;
  if (w.q_nc > 1 && threadIdx.x == 0 && chunk == 0)
    w.q_used[(size_t)hb * nblk + nblk - 1 - bx / w.q_nc] = share.used;
  const size_t all = (size_t)a.batch * a.heads * a.seq_q;
  const size_t row = (size_t)chunk * all + packed_row(a, hb, min(t.r, t.rows - 1));

  f32x16 dq[D / 32];
#pragma unroll
  for (int x = 0; x < D / 32; ++x) dq[x] = zero16();
  float sums[kSums] = {0.f, 0.f, 0.f, 0.f, 0.f};
  if (n > 0)
    each_tile(t, kt, t_begin, n, lds0,
              [&](int kv0, uint64_t see, int cur, const LaneReads<D>& kr) PB_INLINE {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        f32x16 pr[1], dz[1], slope;
        t.template pair<BIAS == kTable ? 2 : 1>(kv0, h2, cur, kr, see, pr, dz, slope);
        if constexpr (BIAS == kTable) {
          if (a.dtable) {
            float s = 0.f, sp = 0.f;
#pragma unroll
            for (int x = 0; x < 16; ++x) s += dz[0][x];
            sums[0] += s;
            const int u = t.wave_uniform(kv0);
            if (u >= 0) {
#pragma unroll
              for (int x = 0; x < 16; ++x) sp += pr[0][x];
              if (u == a.side - 1) sums[1] += s, sums[2] += sp;
              else sums[3] += s, sums[4] += sp;
            }
          }
          if constexpr (CAP)
#pragma unroll
            for (int x = 0; x < 16; ++x) dz[0][x] *= slope[x];
        }
        bf16x8 df[2], dl[2];
#pragma unroll
        for (int s2 = 0; s2 < 2; ++s2) {
          df[s2] = probs_frag(dz, s2);
          if constexpr (WIDE) dl[s2] = rest_frag(dz, s2, df[s2]);
        }
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int s2 = 0; s2 < 2; ++s2) {
            const bf16x8 kc = kr.cols(db, 2 * h2 + s2, 0);
            dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kc, df[s2], dq[db], 0, 0, 0);
            if constexpr (WIDE)
              dq[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kc, dl[s2], dq[db], 0, 0, 0);
          }
      }
    });
  if constexpr (BIAS == kTable) {
    if (a.dtable) {
#pragma unroll
      for (int x = 0; x < kSums; ++x) {
        const float s = sums[x] + __shfl_xor(sums[x], 32, 64);
        if (t.r < t.rows && t.fh == 0)
          w.sums[((size_t)chunk * kSums + x) * all + packed_row(a, hb, t.r)] = s;
      }
    }
  }
  if (split) {
    if (t.r >= t.rows) return;
    float* prow = w.pdq + row * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(prow + 32 * db + 8 * j + 4 * t.fh) =
            f32x4{dq[db][4 * j] * a.dscale, dq[db][4 * j + 1] * a.dscale,
                  dq[db][4 * j + 2] * a.dscale, dq[db][4 * j + 3] * a.dscale};
    return;
  }
  float bad = 0.f;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) bad = fmaf(dq[db][e], 0.f, bad);
  if (__builtin_amdgcn_ballot_w64(t.r < t.rows && bad != 0.f)) {
    const int w0 = t.r0 + 32 * t.wave;
    for (int r = w0; r < min(w0 + 32, t.rows); ++r) {
      const int i = t.pk.pos(r);
      score::dq_row<bf16, D>(a, t.b, t.h0 + r - i * a.pack, i, t.lane);
    }
    return;
  }
  if (t.r >= t.rows) return;
  bf16* out = (bf16*)a.dq + ((size_t)t.b * a.seq_q + t.i) * a.ld_dq + t.h * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = dq[db][4 * j + e] * a.dscale;
      store4(out + 32 * db + 8 * j + 4 * t.fh, v);
    }
}

// The row terms from unrounded values, of a block's rows or of a chunk's part of their
// tiles.
template <int D, bool CAP, int BIAS>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void score_delta_bf16(
    ScoreArgs a, BwdWork w) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  const int hb_n = a.batch * (a.heads / a.pack), hb = blockIdx.x % hb_n;
  const int bx = blockIdx.x / hb_n, nblk = row_blocks(a), blk = nblk - 1 - bx / w.d_nc;
  const int chunk = bx % w.d_nc;
  RowTiles<D, CAP, BIAS> t(a, w, smem, 4 * kTileK * 2 * D, blk, hb, false);
  const KeyTiles kt = key_tiles<kTileK>(a, t.b, t.p_first, t.p_last, t.lane);
  const Share share(kt.n, w.d_nc, kMinTilesD);
  const int t_begin = chunk * share.size, n = min(kt.n - t_begin, share.size);
  if (chunk >= max(share.used, 1)) return;
  if (w.d_nc > 1 && threadIdx.x == 0 && chunk == 0) w.d_used[(size_t)hb * nblk + blk] = share.used;
  float delta = 0.f;
  if (n > 0)
    each_tile(t, kt, t_begin, n, lds0,
              [&](int kv0, uint64_t see, int cur, const LaneReads<D>& kr) PB_INLINE {
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        f32x16 pr[1], dz[1], slope;
        t.template pair<0>(kv0, h2, cur, kr, see, pr, dz, slope);
        float s = 0.f;
#pragma unroll
        for (int x = 0; x < 16; ++x) s += dz[0][x];
        delta += s;
      }
    });
  delta += __shfl_xor(delta, 32, 64);
  if (t.r >= t.rows || t.fh != 0) return;
  const size_t row = packed_row(a, hb, t.r);
  if (chunk == 0) w.L2[row] = t.L2;
  if (share.used > 1) w.pdelta[(size_t)chunk * a.batch * a.heads * a.seq_q + row] = delta;
  else w.minus_delta[row] = -delta;
}
// ... from the parts of blocks in chunks, in their order.
__global__ __launch_bounds__(256) void score_delta_merge(ScoreArgs a, BwdWork w) {
  const size_t all = (size_t)a.batch * a.heads * a.seq_q, set = (size_t)a.seq_q * a.pack;
  const size_t row = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (row >= all) return;
  const int n = w.d_used[row / set * row_blocks(a) + row % set / kBlockQ];
  if (n < 2) return;
  float delta = 0.f;
  for (int c = 0; c < n; ++c) delta += w.pdelta[c * all + row];
  w.minus_delta[row] = -delta;
}

// Both roles in one launch, in turn, each with its (under a causal mask) longest blocks
// first, all heads' before the next.
template <int D, bool CAP, int BIAS, bool WIDE>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void score_bwd_bf16(
    ScoreArgs a, BwdWork w, int nk, int nq) {
  const int id = blockIdx.x, mn = min(nk, nq);
  const bool kv = id < 2 * mn ? !(id & 1) : nk > nq;
  const int x = id < 2 * mn ? id >> 1 : id - mn;
  if (kv) {
    const int n = a.batch * a.kv_heads;
    dkdv_block<D, CAP, BIAS, WIDE>(a, w, x / n, x % n);
  } else {
    const int n = a.batch * (a.heads / a.pack);
    dq_block<D, CAP, BIAS, WIDE>(a, w, x / n, x % n);
  }
}

// ----------------------------------------------------- the table's gradient
// Sums by bucket of 128 rows' dz over the tiles whose distances span buckets, with delta
// put right by e; those beyond come from dQ's sums: dz less e P.
//
// Keys of one distance from their rows lie on a diagonal of a wave's 32 x 64 tile: the
// wave writes its dz to LDS (over K and V, once all waves are done with them) and reads
// diagonals back, 32 values a lane in all, each lane those of one head, and adds the sum
// of each to its own place for the distance's bucket.  (An LDS atomic for each dz, the
// direct way, takes about 130 cycles a wave and CU: 8192 tokens, 40 heads, window 1024
// 470 us against 72.)
template <int D>
struct DtableLds {
  static constexpr int kRow = kTileK + 4;  // floats of a row of dz
  static constexpr int kTiles = 2 * kTileK * 2 * D;
  static constexpr int kStaged = 4 * 32 * kRow * 4;
  static constexpr int kBytes = kTiles > kStaged ? kTiles : kStaged;
  static __host__ __device__ BiasLds bias(const ScoreArgs& a) {
    return BiasLds(kBytes, a.buckets, a.pack, (kBlockQ + a.pack - 1) / a.pack + 1, kTileK);
  }
};
template <int D, bool CAP>
__global__ __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2))) void score_dtable_bf16(
    ScoreArgs a, BwdWork w, int nblk) {
  constexpr int TB = kTileK * 2 * D, kRow = DtableLds<D>::kRow;
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  const int hb_n = a.batch * (a.heads / a.pack);
  const int hb = blockIdx.x % hb_n, blk = nblk - 1 - blockIdx.x / hb_n;
  RowTiles<D, CAP, kTable> t(a, w, smem, DtableLds<D>::kBytes, blk, hb);
  // a place for each bucket and lane, then the bucket of each distance of a tile
  float* acc = (float*)(smem + t.bl.bytes);
  unsigned char* ids = smem + t.bl.bytes + 4 * a.buckets * 64 * 4;
  float* mine = acc + (size_t)t.wave * a.buckets * 64 + t.lane;
  for (int n = 0; n < a.buckets; ++n) mine[n * 64] = 0.f;
  t.tables();
  const size_t all = (size_t)a.batch * a.heads * a.seq_q;
  float sums[kSums] = {0.f, 0.f, 0.f, 0.f, 0.f};
  if (t.r < t.rows)
    for (int c = 0; c < (w.q_nc > 1 ? max(w.q_used[(size_t)hb * nblk + blk], 1) : 1); ++c)
#pragma unroll
      for (int x = 0; x < kSums; ++x)
        sums[x] += w.sums[((size_t)c * kSums + x) * all + packed_row(a, hb, t.r)];
  t.dl += sums[0];
  // (pack is a power of two here: lane and row have one head, and blocks begin with head 0)
  const int span = 32 / a.pack, hh = t.lane % a.pack, y = t.lane / a.pack, step = 64 / a.pack;
  if (t.fh == 0) {
    mine[(a.side - 1) * 64] += fmaf(-sums[0], sums[2], sums[1]);
    mine[(a.causal ? 0 : 2 * a.side - 1) * 64] += fmaf(-sums[0], sums[4], sums[3]);
  }
  const KeyTiles kt = key_tiles<kTileK>(a, t.b, t.p_first, t.p_last, t.lane);
  const LaneReads<D> places(t.lane);
  float* staged = (float*)smem + t.wave * 32 * kRow;
  // from the block's last position to the wave's
  const int after = t.p_last - (t.off + t.pk.pos(t.r0 + 32 * t.wave + 31));
  for (int i = 0; i < kt.n; ++i) {
    const int kv0 = kt.tile(i) * kTileK;
    if (t.uniform(kv0) >= 0) continue;
    block_barrier();  // the tile before has been read by all
    t.request(kt, kv0, lds0, lds0 + TB);
    t.build(kv0, 0);
    for (int x = threadIdx.x; x < t.bl.stride; x += 256)
      ids[x] = (unsigned char)bias_bucket(a, t.bl, smem, t.p_last - kv0 - x);
    wait_dma_all();
    block_barrier();
    const uint64_t see = t.keys.bits(kv0);
    // (where the wave's rows are all beyond, dQ has summed)
    const bool any = t.wave_uniform(kv0) < 0 && __builtin_amdgcn_ballot_w64(see != 0);
    f32x16 dz[2][1];
    if (any) {
      const LaneReads<D> kr = places.at(lds0);
#pragma unroll
      for (int h2 = 0; h2 < 2; ++h2) {
        f32x16 pr[1], slope;
        t.template pair<0>(kv0, h2, 0, kr, see, pr, dz[h2], slope);
      }
    }
    block_barrier();  // every wave is done with K and V
    if (!any) continue;
#pragma unroll
    for (int h2 = 0; h2 < 2; ++h2)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<f32x4*>(staged + t.fr * kRow + 32 * h2 + 8 * j + 4 * t.fh) =
            f32x4{dz[h2][0][4 * j], dz[h2][0][4 * j + 1], dz[h2][0][4 * j + 2], dz[h2][0][4 * j + 3]};
    // Entry x (as in bias_tile, from the wave's last position on) of position q is key x -
    // (span - 1) + q; where that is below 0, key + 64 is on diagonal x + 64.
    for (int m = 0; m < a.pack; ++m) {
      const int x = y + step * m;
      float lo = 0.f, hi = 0.f;
#pragma unroll 8
      for (int q = 0; q < span; ++q) {
        const int key = x - (span - 1) + q;
        const float v = staged[(q * a.pack + hh) * kRow + (key & 63)];
        lo += key >= 0 ? v : 0.f;
        hi += key >= 0 ? 0.f : v;
      }
      const int at = x + after;  // (rows past the end lie beyond the block's last position)
      if (at >= 0) mine[ids[at] * 64] += lo;
      if (x < span - 1 && at + 64 >= 0) mine[ids[at + 64] * 64] += hi;
    }
  }
  __syncthreads();
  // a wave a bucket: sums over the waves, then over the lanes of a head
  for (int n = t.wave; n < a.buckets; n += 4) {
    float s = 0.f;
#pragma unroll
    for (int wv = 0; wv < 4; ++wv) s += acc[(wv * a.buckets + n) * 64 + t.lane];
    for (int o = 32; o >= a.pack; o >>= 1) s += __shfl_xor(s, o, 64);
    if (t.lane < a.pack)
      a.bias_part[(((size_t)t.b * nblk + blk) * a.heads + t.h0 + t.lane) * a.buckets + n] = s;
  }
}

// ----------------------------------------------------------------- merges
// Sums of a split block's parts, in chunk order.  A row with a non-finite part is computed
// again by the definition.
template <int D, bool KEYS>
__global__ __launch_bounds__(256) void score_bwd_merge(ScoreArgs a, BwdWork w) {
  const int H = KEYS ? a.kv_heads : a.heads, S = KEYS ? a.seq_k : a.seq_q;
  const size_t all = (size_t)a.batch * H * S;
  using ML = MergeLanes<D>;
  const size_t at = ((size_t)blockIdx.x * 256 + threadIdx.x) / ML::kLanes;
  const int g = threadIdx.x % ML::kLanes, lane = threadIdx.x & 63;
  const size_t row = min(at, all - 1);
  int b, h, i;
  const int* used;  // of set 0
  if (KEYS) {
    i = (int)(row % S), h = (int)(row / S % H), b = (int)(row / S / H);
    used = w.kv_used + ((size_t)b * H + h) * key_blocks(a) + i / kBlockK;
  } else {
    const int r = (int)(row % ((size_t)S * a.pack)), hb = (int)(row / ((size_t)S * a.pack));
    i = r / a.pack, h = hb % (H / a.pack) * a.pack + r % a.pack, b = hb / (H / a.pack);
    used = w.q_used + (size_t)hb * row_blocks(a) + r / kBlockQ;
  }
  const int sets = KEYS ? a.group / a.pack : 1, subs = (KEYS ? w.kv_nc : w.q_nc) / sets;
  const bool whole = sets == 1 && *used <= 1;  // written by its workgroup
  float acc[2][ML::kChunks][8] = {}, bad = 0.f;
  if (!whole) {
#pragma unroll
    for (int k = 0; k < (KEYS ? 2 : 1); ++k) {
      const float* from = pick(KEYS, pick(k != 0, w.pdv, w.pdk), w.pdq) + row * D;
      for (int s = 0; s < sets; ++s)
        for (int c0 = 0, n = used[(size_t)s * a.batch * H * key_blocks(a)]; c0 < n; c0 += 4) {
          float v[4][ML::kChunks][8];  // (four loads in flight)
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int x = 0; x < ML::kChunks; ++x)
              load8(from + (size_t)(s * subs + min(c0 + c, n - 1)) * all * D + ML::at(g, x), v[c][x]);
#pragma unroll
          for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int x = 0; x < ML::kChunks; ++x)
#pragma unroll
              for (int e = 0; e < 8; ++e) acc[k][x][e] += c0 + c < n ? v[c][x][e] : 0.f;
        }
#pragma unroll
      for (int x = 0; x < ML::kChunks; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) bad = fmaf(acc[k][x][e], 0.f, bad);
    }
  }
  const bool again = ML::any(at < all && bad != 0.f);
  unsigned long long rows = __builtin_amdgcn_ballot_w64(again);
  if (at < all && !again && !whole) {
#pragma unroll
    for (int x = 0; x < ML::kChunks; ++x) {
      if (KEYS) {
        const size_t to = ((size_t)b * S + i) * a.ld_dkv + h * D + ML::at(g, x);
        store8((bf16*)a.dk + to, acc[0][x]);
        store8((bf16*)a.dv + to, acc[1][x]);
      } else {
        store8((bf16*)a.dq + ((size_t)b * S + i) * a.ld_dq + h * D + ML::at(g, x), acc[0][x]);
      }
    }
  }
  while (rows) {
    const int first = __builtin_ctzll(rows);
    const int i2 = __builtin_amdgcn_readlane(i, first), h2 = __builtin_amdgcn_readlane(h, first);
    const int b2 = __builtin_amdgcn_readlane(b, first);
    rows &= ~__builtin_amdgcn_ballot_w64(i == i2 && h == h2 && b == b2);
    if (KEYS) score::dkdv_row<bf16, D>(a, b2, h2, i2, lane);
    else score::dq_row<bf16, D>(a, b2, h2, i2, lane);
  }
}

size_t round64(size_t floats) { return (floats + 63) & ~(size_t)63; }

// The workspace's parts, in floats from its start.
struct BwdLayout {
  size_t L2, delta, bias, sums, pdelta, pdk, pdv, pdq, kv_used, q_used, d_used, total;
};
BwdLayout bwd_layout(int D, const ScoreArgs& a, const ScoreBwdPlan& p) {
  const size_t rows = (size_t)a.batch * a.heads * a.seq_q;
  const size_t keys = (size_t)a.batch * a.kv_heads * a.seq_k;
  BwdLayout l{};
  size_t at = 0;
  auto take = [&](size_t n) {
    const size_t from = at;
    at += round64(n);
    return from;
  };
  l.L2 = take(rows), l.delta = take(rows);
  l.bias = take(a.buckets ? (size_t)a.batch * row_blocks(a) * a.heads * a.buckets : 0);
  l.sums = take(a.buckets ? (size_t)p.q.chunks * kSums * rows : 0);
  l.pdelta = take(p.d.chunks > 1 ? (size_t)p.d.chunks * rows : 0);
  l.pdk = take(p.kv.chunks > 1 ? (size_t)p.kv.chunks * keys * D : 0);
  l.pdv = take(p.kv.chunks > 1 ? (size_t)p.kv.chunks * keys * D : 0);
  l.pdq = take(p.q.chunks > 1 ? (size_t)p.q.chunks * rows * D : 0);
  l.kv_used = take(p.kv.chunks > 1 ? (size_t)a.batch * a.heads / a.pack * key_blocks(a) : 0);
  l.q_used = take(p.q.chunks > 1 ? (size_t)a.batch * a.heads / a.pack * row_blocks(a) : 0);
  l.d_used = take(p.d.chunks > 1 ? (size_t)a.batch * a.heads / a.pack * row_blocks(a) : 0);
  l.total = at;
  return l;
}

template <int D>
void bwd_d(const ScoreArgs& a, const ScoreBwdPlan& p, float* ws, hipStream_t s) {
  const BwdLayout l = bwd_layout(D, a, p);
  BwdWork w{ws + l.L2, ws + l.delta, ws + l.pdk, ws + l.pdv, ws + l.pdq, ws + l.sums, ws + l.pdelta,
            (int*)(ws + l.kv_used), (int*)(ws + l.q_used), (int*)(ws + l.d_used),
            p.kv.chunks, p.q.chunks, p.d.chunks};
  ScoreArgs x = a;
  x.bias_part = ws + l.bias;
  x.minus_delta = a.wide ? w.minus_delta : nullptr;
  const size_t rows = (size_t)a.batch * a.heads * a.seq_q;
  const size_t keys = (size_t)a.batch * a.kv_heads * a.seq_k;
  constexpr int kLanes = D == 96 ? 4 : D / 8;
  if (!a.wide)
    score_terms<D><<<(unsigned)((rows * kLanes + 255) / 256), 256, 0, s>>>(x, w.L2, w.minus_delta);
  const int nk = key_blocks(a) * a.batch * a.kv_heads * p.kv.chunks;
  const int nq = row_blocks(a) * a.batch * (a.heads / a.pack) * p.q.chunks;
  const int nd = row_blocks(a) * a.batch * (a.heads / a.pack) * p.d.chunks;
  const size_t q_tiles = 4 * (size_t)kTileK * 2 * D;
  const bool cap = a.cap > 0.f;
#define PB_BWD(C, B)                                                                              \
  do {                                                                                            \
    size_t lds_q = q_tiles, lds = KvLds<D>::kBytes;                                               \
    if (B == kTable) {                                                                            \
      lds_q = BiasLds((int)q_tiles, a.buckets, a.pack, (kBlockQ + a.pack - 1) / a.pack + 1,       \
                      kTileK).bytes;                                                              \
      lds = KvLds<D>::bias(a).bytes;                                                              \
    }                                                                                             \
    lds = std::max(lds, lds_q);                                                                   \
    if (a.wide) {                                                                                 \
      score_delta_bf16<D, C, B><<<(unsigned)nd, 256, lds_q, s>>>(x, w);                           \
      if (p.d.chunks > 1)                                                                         \
        score_delta_merge<<<(unsigned)((rows + 255) / 256), 256, 0, s>>>(x, w);                   \
      score_bwd_bf16<D, C, B, true><<<(unsigned)(nk + nq), 256, lds, s>>>(x, w, nk, nq);          \
    } else {                                                                                      \
      score_bwd_bf16<D, C, B, false><<<(unsigned)(nk + nq), 256, lds, s>>>(x, w, nk, nq);         \
    }                                                                                             \
  } while (0)
  const int bias = a.slopes ? kSlopes : a.table ? kTable : kNoBias;
  if (cap) {
    if (bias == kTable) PB_BWD(true, kTable);
    else if (bias == kSlopes) PB_BWD(true, kSlopes);
    else PB_BWD(true, kNoBias);
  } else {
    if (bias == kTable) PB_BWD(false, kTable);
    else if (bias == kSlopes) PB_BWD(false, kSlopes);
    else PB_BWD(false, kNoBias);
  }
#undef PB_BWD
  if (p.kv.chunks > 1)
    score_bwd_merge<D, true><<<(unsigned)((keys * MergeLanes<D>::kLanes + 255) / 256), 256, 0, s>>>(x, w);
  if (p.q.chunks > 1)
    score_bwd_merge<D, false><<<(unsigned)((rows * MergeLanes<D>::kLanes + 255) / 256), 256, 0, s>>>(x, w);
  if (!a.dtable) return;
  const int nblk = row_blocks(a);
  const unsigned grid = (unsigned)(nblk * a.batch * (a.heads / a.pack));
  const BiasLds bl = DtableLds<D>::bias(a);
  const size_t lds = bl.bytes + (size_t)4 * a.buckets * 64 * 4 + bl.stride;
  if (cap) score_dtable_bf16<D, true><<<grid, 256, lds, s>>>(x, w, nblk);
  else score_dtable_bf16<D, false><<<grid, 256, lds, s>>>(x, w, nblk);
  launch_score_dtable_sum(x, nblk * a.batch, s);
}

}  // namespace

size_t score_bwd_bytes(int head_dim, const ScoreArgs& a, const ScoreBwdPlan& p) {
  return bwd_layout(head_dim, a, p).total * sizeof(float);
}

// Row tiles of a key block and a set of heads.
static int most_row_tiles(const ScoreArgs& a) {
  const long long all = ((long long)a.seq_q * a.pack + kTileQ - 1) / kTileQ;
  const long long reach = (long long)(a.causal ? 1 : 2) * a.window + kBlockK;
  return (int)(a.prefix ? all : std::min(all, reach * a.pack / kTileQ + 2));
}

ScoreBwdPlan score_bwd_whole(const ScoreArgs& a) { return ScoreBwdPlan{{a.group / a.pack}, {1}, {1}}; }

// A key block has as many row tiles as all heads that share it bring, a row block few key
// tiles, and splitting costs a merge and its traffic (fp32 parts, written and read).  So
// keys are cut down to what the launch takes as a whole (over 512 workgroups at a time;
// half the longest block's tiles on average under a causal mask) or the longest row block
// takes, whichever is more; rows only where few of them see many keys.  Found by timing
// 21 plans each for 12 shapes without WIDE (us; keys' chunks 1, 2, 4, 8):
//   4096 tokens, 16 heads over 4, 128        687 412 295 295
//   the same, capped, three documents        632 361 278 266
//   2048, 12 x 128                           113  88  95 115
//   8192, 4 over 1 x 128                    1297 685 401 302
//   4 x 2048, 16 over 2 x 96                 632 357 270 277
//   2048, 40 x 128, window 512               136 158 184 203
//   4096, 8 x 128, window 1024                91 111 126 131
// The row terms' parts are four bytes a row, so their chunks cost a workgroup's beginning
// (its rows, the first tile) and a launch: one and a half times what runs at a time.  All
// gradients (us, for 1, 512, 1024 workgroups at least):
//   2048, 12 x 128                           148 126 131
//   4096 tokens, 16 heads over 4 x 128       480 479 462
//   4096, 16 x 64                            284 284 268
//   2048, 40 x 128, window 512, with a table 277 277 275
constexpr long long kDeltaBlocks = 768;
ScoreBwdPlan score_bwd_plan(int head_dim, const ScoreArgs& a) {
  ScoreBwdPlan p = score_bwd_whole(a);
  const int sets = p.kv.chunks;
  const long long nk = (long long)key_blocks(a) * a.batch * a.kv_heads * sets;
  const long long nq = (long long)row_blocks(a) * a.batch * (a.heads / a.pack);
  const int kv = most_row_tiles(a), q = score_most_tiles(a, kBlockQ, kTileK);
  const double kv_us = 1.5 * kv, q_us = 2.4 * q;
  const double half = a.causal && a.window >= a.seq_k ? 0.5 : 1.0;
  const double all = half * (nk * kv_us + nq * q_us) / 512;
  auto cut = [&](ScorePlan& s, double us, double target, int most) {
    const int m = std::min((int)std::ceil(us / target - 0.25), most);
    if (m > 1) s.chunks *= m;
  };
  cut(p.kv, kv_us, std::max(all, 0.8 * q_us), kv / kMinTilesKv);
  cut(p.q, q_us, std::max(all, 100.0), q / kMinTilesQ);
  if (a.wide)
    p.d.chunks = (int)std::max(1LL, std::min((kDeltaBlocks + nq - 1) / nq, (long long)q / kMinTilesD));
  return p;
}

void launch_score_backward_bf16(int head_dim, const ScoreArgs& a, const ScoreBwdPlan& p, void* ws,
                                hipStream_t s) {
  if (head_dim == 64) bwd_d<64>(a, p, (float*)ws, s);
  else if (head_dim == 96) bwd_d<96>(a, p, (float*)ws, s);
  else bwd_d<128>(a, p, (float*)ws, s);
}

}  // namespace pb

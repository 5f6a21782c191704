// Tiles of bf16 rows in LDS and their MFMA fragments, shared by the bf16 attention
// kernels: layouts without bank conflicts, LDS-DMA, reductions over lane groups.
#pragma once

#include "common.h"

namespace pb {
namespace {

constexpr float kNegInf = -__builtin_huge_valf();

PB_DEV float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }  // exp2(-inf) = 0

typedef short s16x4 __attribute__((ext_vector_type(4)));
#define PB_LDS __attribute__((address_space(3)))

// ------------------------------------------------------------ LDS tiles
// Every tile is natural: kTL token rows x D features, 2 D bytes per row, the
// 16-byte chunk c of row r stored at chunk c ^ f(r).  For D = 128 (16 chunks
// per row, one 256-byte bank period) f is a 4-bit rotation of r that makes
// both access patterns conflict-free: a 16-byte read by 16 consecutive rows
// at one chunk, and a transposing read of 8 consecutive rows x 4 aligned
// chunks.  D = 64 uses an injective 3-bit variant.  D = 96 (12 chunks, rows
// 192 bytes apart): row r starts at bank group 12 r mod 16 = 4 (3 r mod 4),
// so r mod 4 already spreads rows over the four quarters of the bank period;
// f(r) = (r / 4) mod 4 on the low two chunk bits (which keeps c below 12)
// spreads them within a quarter.  16 rows at one chunk then hit 16 distinct
// bank groups, and so do 4 consecutive rows x 4 aligned chunks.
template <int D>
PB_DEV int rowswz(int r) {
  static_assert(D == 64 || D == 96 || D == 128, "head_dim");
  if constexpr (D == 128) return ((r & 3) << 2) | ((r >> 2) & 3);
  else if constexpr (D == 96) return (r >> 2) & 3;
  else return ((r & 1) << 2) | ((r >> 1) & 3);
}
template <int D>
PB_DEV int chunk_at(int r, int c) { return c ^ rowswz<D>(r); }

PB_DEV void dma16(const void* g, uint32_t lds_byte_addr) {
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "s"(lds_byte_addr)
               : "memory", "m0");
}
PB_DEV void dma4(const void* g, uint32_t lds_byte_addr) {  // lane l's 4 bytes -> base + 4 l
  asm volatile("s_mov_b32 m0, %1\n\tglobal_load_lds_dword %0, off" ::"v"(g), "s"(lds_byte_addr)
               : "memory", "m0");
}
PB_DEV void wait_dma_all() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// Wait until at most n DMA instructions of this wave are still in flight
// (n uniform; values above 15 wait for all).
PB_DEV void wait_dma_upto(int n) {
#define PB_VMCNT_CASE(k) \
  case k: asm volatile("s_waitcnt vmcnt(" #k ")" ::: "memory"); break;
  switch (n) {
    PB_VMCNT_CASE(1) PB_VMCNT_CASE(2) PB_VMCNT_CASE(3) PB_VMCNT_CASE(4) PB_VMCNT_CASE(5)
    PB_VMCNT_CASE(6) PB_VMCNT_CASE(7) PB_VMCNT_CASE(8) PB_VMCNT_CASE(9) PB_VMCNT_CASE(10)
    PB_VMCNT_CASE(11) PB_VMCNT_CASE(12) PB_VMCNT_CASE(13) PB_VMCNT_CASE(14) PB_VMCNT_CASE(15)
    default: asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); break;
  }
#undef PB_VMCNT_CASE
}
PB_DEV void block_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// This wave's share of a natural tile, rows row0 .. row0 + kTL - 1 of a
// [rows_valid, ld] token-major matrix, by LDS-DMA (each lane's 16 bytes land
// at the piece's LDS base + 16 * lane).  Rows past rows_valid are read from
// the last valid row: finite values that the window mask always zeroes.
// The tile is cut into 1 KB pieces (one DMA instruction each); with NW
// dividing their number each wave moves a contiguous run, else piece i goes
// to wave i mod NW.  dma_pieces is the number a wave issues.
template <int D, int TL, int NW>
__host__ __device__ constexpr int dma_pieces(int wave) {
  constexpr int NP = TL * 2 * D / 1024;
  return NP % NW == 0 ? NP / NW : (NP - wave + NW - 1) / NW;
}
template <int D, int TL, int NW>
PB_DEV void dma_tile(const bf16* __restrict__ base, int ld, int row0, int rows_valid,
                     uint32_t lds_tile, int wave, int lane) {
  constexpr int RB = 2 * D;
  constexpr int BYTES = TL * RB;
  constexpr int NP = BYTES / 1024;
  static_assert(BYTES % 1024 == 0, "tiles are whole 1 KB pieces");
#pragma unroll
  for (int i = 0; i < (NP + NW - 1) / NW; ++i) {
    const int pc = NP % NW == 0 ? wave * (NP / NW) + i : i * NW + wave;
    if (NP % NW != 0 && pc >= NP) break;  // wave-uniform
    const int piece = pc * 1024;
    const int p = piece + 16 * lane;
    const int row = p / RB, slot = (p / 16) % (RB / 16);
    const int c = chunk_at<D>(row, slot);
    const int t = min(row0 + row, rows_valid - 1);
    dma16(base + (size_t)t * ld + 8 * c, __builtin_amdgcn_readfirstlane(lds_tile + piece));
  }
}

// MFMA operand with 8 consecutive features of token row `row` (k-step ks of
// the feature contraction, lane half h).
template <int D>
PB_DEV bf16x8 frag_row(const unsigned char* tile, int row, int ks, int h) {
  return *reinterpret_cast<const bf16x8*>(tile + row * (2 * D) + chunk_at<D>(row, 2 * ks + h) * 16);
}
// MFMA operand with 8 tokens of feature row `e` of the transposed tile, in
// the order the probabilities sit in a 32 x 32 accumulator: tokens
// 16 s + 4 h + {0..3} then 16 s + 8 + 4 h + {0..3}.  Two transposing reads:
// lane 4 j + q of a 16-lane group addresses token kb + j, features
// (e & ~15) + 4 q .. +3; lane i receives tokens kb .. kb + 3 of feature
// (e & ~15) + i.
template <int D>
PB_DEV bf16x8 frag_tr(const unsigned char* tile, int e, int s, int h, int lane) {
  const int i = lane & 15, j = i >> 2, q = i & 3;
  const int d0 = (e & ~15) + 4 * q;
  const int c = d0 >> 3, off = (d0 & 7) * 2;
  const int t1 = 16 * s + 4 * h + j, t2 = t1 + 8;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (PB_LDS s16x4*)(tile + t1 * (2 * D) + chunk_at<D>(t1, c) * 16 + off));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (PB_LDS s16x4*)(tile + t2 * (2 * D) + chunk_at<D>(t2, c) * 16 + off));
  const bf16x4 a4 = __builtin_bit_cast(bf16x4, a), b4 = __builtin_bit_cast(bf16x4, b);
  return bf16x8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
}

// Probabilities for MFMA k-step s (16 tokens) from 32-token accumulators.
PB_DEV bf16x8 probs_frag(const f32x16* p, int s) {
  const f32x16& a = p[s >> 1];
  const int o = 8 * (s & 1);
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (bf16)a[o + e];
  return r;
}

PB_DEV f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int e = 0; e < 16; ++e) z[e] = 0.f;
  return z;
}

// 8 consecutive features of one token row from global memory (zero if !ok).
PB_DEV bf16x8 load_row_frag(const bf16* p, bool ok) {
  const u32x4 v = *reinterpret_cast<const u32x4*>(p);
  return ok ? __builtin_bit_cast(bf16x8, v) : bf16x8{};
}

// ====================================================== 16x16x32 tiles
// Tiles for the v_mfma_f32_16x16x32_bf16 kernels, natural token-major like
// the ones above, with their own chunk swizzle: chunk c of row r is stored
// at slot c ^ swz16(r).  The maps are linear in the row bits and were found
// by exhaustive search under a model of the LDS (64 banks of 4 bytes) that
// reproduces the measured behaviour of earlier layouts: a 16-byte read is
// free of conflicts when each 16 lanes hit distinct banks; a transposing
// 8-byte read when each 32 lanes hit distinct banks and, in addition, the
// four rows a 16-lane group reads lie in four distinct 64-byte quarters of
// the bank space (a layout with two of them in one quarter ran the
// forward's O update about six times slower).  Both of the forward's reads
// (K rows in the permuted key order below, one chunk per 16 lanes; the
// transposing reads of V, rows 8 g + j of lane group g) satisfy these for
// head dims 64, 96 and 128; for 96 only the low two chunk bits move, which
// keeps the slot below 12.  Only row bits 0, 1, 3 and 4 enter.
template <int D>
PB_DEV int swz16(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | (((r >> 3) & 1) << 1) | ((r >> 4) & 1);
  else if constexpr (D == 96) return (((r >> 3) & 1) << 1) | ((r >> 4) & 1);
  else return (((r >> 1) & 1) << 2) | (((r >> 3) & 1) << 1) | ((r >> 4) & 1);
}
// The swizzle of tiles read only by transposing reads (V in the forward).
// Same rules, and in addition the two 16-byte halves of a 32-byte row
// segment are never swapped (bit 0 stays), as in the GEMM's transposed
// layout.
template <int D>
PB_DEV int swz16v(int r) {
  if constexpr (D == 128) return ((r & 3) << 2) | (((r >> 3) & 1) << 1);
  else if constexpr (D == 96) return ((r >> 3) & 1) << 1;
  else return (((r >> 1) & 1) << 2) | (((r >> 3) & 1) << 1);
}

// Key order inside a 64-key tile for the score MFMAs.  Score block kb (16
// keys; kb = 2 s + h) uses, as its MFMA row i, key 32 s + 8 (i / 4) + 4 h +
// (i mod 4).  The result row i lands in lane group i / 4 as element i mod 4,
// so lane group g holds keys 32 s + 8 g + 0..3 (block 2 s) and + 4..7 (block
// 2 s + 1): exactly the eight consecutive keys that the probability operand
// of the next MFMA (k-step s of 32 keys) wants from that lane group.
PB_DEV int score_key(int kb, int i) { return 32 * (kb >> 1) + 8 * (i >> 2) + 4 * (kb & 1) + (i & 3); }
constexpr int score_row_off(int kb) { return 32 * (kb >> 1) + 4 * (kb & 1); }

// This lane's LDS byte offsets for the forward's fragment reads inside one
// tile.  swz16 depends only on row bits 0, 1, 3 and 4, which are fixed per
// lane for both reads, so each block's row offset (bits 2 and 5) is a
// constant added to one per-lane base: D/32 bases for K and D/16 for V.
//   k[ks]: A operand of K for score block kb, k-step ks (features 32 ks ..
//          + 31) at k[ks] + 2 D score_row_off(kb): lane l supplies row
//          score_key(kb, l & 15), features 32 ks + 8 (l >> 4) .. + 7.
//   v[db]: A operand of V^T for features 16 db .. + 15 and keys 32 s ..
//          + 31, by two transposing reads at v[db] + 2 D (32 s) and
//          + 2 D (32 s + 4): lane 4 j + q of a 16-lane group addresses key
//          base + j, features 16 db + 4 q .. + 3, and receives keys base ..
//          base + 3 of its own feature 16 db + (l & 15); lane group g takes
//          keys 32 s + 8 g .. + 7.
template <int D>
struct FwdLds {
  uint32_t k[D / 32];
  uint32_t v[D / 16];
  PB_DEV explicit FwdLds(int lane) {
    const int i = lane & 15, g = lane >> 4;
    const int rk = score_key(0, i);
#pragma unroll
    for (int ks = 0; ks < D / 32; ++ks)
      k[ks] = (uint32_t)(rk * 2 * D + (((4 * ks + g) ^ swz16<D>(rk)) * 16));
    const int j = i >> 2, q = i & 3;
    const int tv = 8 * g + j;
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const int d0 = 16 * db + 4 * q;
      v[db] = (uint32_t)(tv * 2 * D + (((d0 >> 3) ^ swz16v<D>(tv)) * 16) + (d0 & 7) * 2);
    }
  }
};
PB_DEV bf16x8 lds_b128(uint32_t addr) { return *(const PB_LDS bf16x8*)addr; }
// Two transposing reads at addr and addr + gap bytes (four keys each).
PB_DEV bf16x8 lds_tr2(uint32_t addr, uint32_t gap) {
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PB_LDS s16x4*)addr);
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((PB_LDS s16x4*)(addr + gap));
  const bf16x4 a4 = __builtin_bit_cast(bf16x4, a), b4 = __builtin_bit_cast(bf16x4, b);
  return bf16x8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
}
// Values consumed by an empty asm: computed by this point (IR passes would
// otherwise sink them to their first use, out of the phase that interleaves
// them with MFMAs).
PB_DEV void keep(const bf16x8& x) { asm volatile("" ::"v"(__builtin_bit_cast(u32x4, x))); }
PB_DEV void keep(float x) { asm volatile("" ::"v"(x)); }
// Scheduling-group masks (sched_group_barrier): matrix, vector ALU, LDS read.
constexpr int kSgMfma = 0x008, kSgValu = 0x002, kSgDsRead = 0x100;

// LDS-DMA of a TL-row tile in the swz16 layout: this wave's NP / NW 1 KB
// pieces (NP = TL 2 D / 1024, a multiple of NW).  Row r of the tile is token
// row0 + r of a [rows_valid, ld] matrix (rows past the end read the last
// one: finite values the window mask always zeroes).  The lane's 16 bytes
// of piece i are global chunk slot ^ swz(row) of its row (swz16, or swz16v
// with VSWZ); row[i] and cof[i] (that chunk's byte offset) are fixed per
// lane.
template <int D, int TL, int NW, bool VSWZ = false>
struct DmaRows {
  static constexpr int NP = TL * 2 * D / 1024;
  static constexpr int NPW = NP / NW;
  static constexpr bool kV = VSWZ;
  static_assert(NP % NW == 0, "whole pieces per wave");
  int row[NPW];
  uint32_t cof[NPW];
  PB_DEV DmaRows(int wave, int lane) {
    constexpr int RB = 2 * D;
#pragma unroll
    for (int i = 0; i < NPW; ++i) {
      const int p = (wave * NPW + i) * 1024 + 16 * lane;
      row[i] = p / RB;
      const int sw = VSWZ ? swz16v<D>(row[i]) : swz16<D>(row[i]);
      cof[i] = (uint32_t)(((p / 16) % (RB / 16)) ^ sw) * 16u;
    }
  }
  // offsets of this wave's pieces for the tile starting at token row0
  PB_DEV void offsets(int row0, int rows_valid, int ld, uint32_t (&off)[NPW]) const {
#pragma unroll
    for (int i = 0; i < NPW; ++i)
      off[i] = (uint32_t)min(row0 + row[i], rows_valid - 1) * (uint32_t)(2 * ld) + cof[i];
  }
  PB_DEV void issue(const bf16* base, const uint32_t (&off)[NPW], uint32_t lds_tile,
                    int wave) const {
#pragma unroll
    for (int i = 0; i < NPW; ++i)
      dma16s(base, off[i], lds_tile + (uint32_t)((wave * NPW + i) * 1024));
  }
};

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
PB_DEV f32x4 zero4() { return f32x4{0.f, 0.f, 0.f, 0.f}; }
PB_DEV f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// Reductions over the four lane groups (lanes l, l ^ 16, l ^ 32, l ^ 48),
// by the two lane-swap instructions.
PB_DEV float max4groups(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  const float y = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false,
                                                  false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
PB_DEV float sum4groups(float x) {
  const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  const float y = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(y), __float_as_uint(y), false,
                                                  false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}
// Sum of the eight bf16 values of an operand, added to acc (two-element dot
// products with (1, 1): the row sums use exactly the rounded probabilities
// that the output MFMA multiplies).
PB_DEV float add_bf16x8(const bf16x8& p, float acc) {
  const bf16x2 one = {(bf16)1.0f, (bf16)1.0f};
  acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[0], p[1]}, one, acc, false);
  acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[2], p[3]}, one, acc, false);
  acc = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[4], p[5]}, one, acc, false);
  return __builtin_amdgcn_fdot2_f32_bf16(bf16x2{p[6], p[7]}, one, acc, false);
}

}  // namespace
}  // namespace pb

// The products of a Newton-Schulz step, all matrices of a call in one launch each:
//
//   gram    A = X X^T          symmetric: tiles on and above the diagonal, each
//                              written to its mirror image too
//   square  B = b A + c A A    symmetric likewise
//   apply   X' = a X + B X
//
// MFMA v_mfma_f32_16x16x32_f16 on the planes of ns_gemm.h, fp32 accumulation.  One
// plane: one product of fp16 values (rounded by 2^-11 at most).  Two planes
// (value h and remainder l): h l + l h + h h, in this order, as one sum over three
// times the length (what is left out, l l, is at most 2^-22 of the product).
//
// 128 x 128 tile per workgroup of four waves, K-tiles of 64 through two LDS stages
// filled by LDS-DMA.
#include <algorithm>

#include "common.h"
#include "gemm_common.h"
#include "ns_gemm.h"

namespace pb {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
#define PB_LDS __attribute__((address_space(3)))

enum class Op { Gram, Square, Apply };

constexpr int kT = 128;           // tile rows and columns
constexpr int kK = 64;            // K-tile
constexpr int kWaves = 4;         // 2 x 2, each 64 x 64
constexpr int kThreads = 64 * kWaves;
constexpr int kOpBytes = kT * kK * 2;                 // one operand's K-tile: 16 KB
constexpr int kPieces = kOpBytes / (1024 * kWaves);   // 1 KB DMA pieces per wave
constexpr int kRowF = kT + 4;     // floats per row of the staged output
static_assert(kNsPad == kK, "X's dimensions are whole K-tiles");

PB_DEV int swz(int row, int c) { return c ^ ((row ^ (row >> 3)) & 7); }
PB_DEV int swz_mn(int k, int c) { return c ^ (4 * (k & 3)) ^ (2 * ((k >> 3) & 1)); }

// Byte offset from the operand tile's first element of this lane's 16 bytes of a
// piece.  KC: rows of the operand are K-contiguous, `rows` of them left; else the
// operand is K rows of which `rows` columns are left.  Past them, the last is read
// (its products are not stored).
template <bool KC>
PB_DEV uint32_t lane_off(int ld, int rows, int p) {
  if constexpr (KC) {
    const int row = p >> 7, c = swz(row, (p >> 4) & 7);
    return (uint32_t)(min(row, rows - 1) * ld + 8 * c) * 2u;
  } else {
    const int k = p >> 8, c = swz_mn(k, (p >> 4) & 15);
    return (uint32_t)(k * ld + min(8 * c, rows - 8)) * 2u;
  }
}
// Fragment of 16 rows (columns) from `base`, k 32 s + 8 (lane >> 4) .. + 7.
template <bool KC>
PB_DEV f16x8 frag(const unsigned char* tile, int base, int s, int lane) {
  if constexpr (KC) {
    const int row = base + (lane & 15);
    return *reinterpret_cast<const f16x8*>(tile + row * 128 + swz(row, 4 * s + (lane >> 4)) * 16);
  } else {
    const int i = lane & 15, mn = base + 4 * (i & 3);
    const int k1 = 32 * s + 8 * (lane >> 4) + (i >> 2), k2 = k1 + 4;
    const int c = mn >> 3, off = (mn & 7) * 2;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (PB_LDS s16x4*)(tile + k1 * 256 + swz_mn(k1, c) * 16 + off));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (PB_LDS s16x4*)(tile + k2 * 256 + swz_mn(k2, c) * 16 + off));
    const f16x4 a4 = __builtin_bit_cast(f16x4, a), b4 = __builtin_bit_cast(f16x4, b);
    return f16x8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
  }
}

int tiles_of(int v) { return (v + kT - 1) / kT; }

struct NsTiles {
  int first[kNsMaxTensors + 1];
};

template <Op OP, int PLANES>
__global__ __launch_bounds__(kThreads, 2) void ns_gemm_kernel(NsTable t, NsTiles tiles, int cur) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kT * kRowF * 4];
  static_assert(4 * kOpBytes <= kT * kRowF * 4, "two stages of two operands");
  constexpr bool BK = OP != Op::Apply;  // B operand K-contiguous
  const int lid = xcd_remap(blockIdx.x, gridDim.x);
  int mi = 0;
#pragma unroll 1
  for (int k = 1; k < t.count; ++k)
    if (lid >= tiles.first[k]) mi = k;
  const NsMat& x = t.mat[mi];
  const int m = x.m, n = x.n, id = lid - tiles.first[mi];
  int tm, tn;
  if constexpr (OP == Op::Apply) {
    tile_of<8>(id, (m + kT - 1) / kT, (n + kT - 1) / kT, tm, tn);
  } else {  // tile id of the triangle tm <= tn, column by column
    tn = (int)((__builtin_sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
    while (tn * (tn + 1) / 2 > id) --tn;
    while ((tn + 1) * (tn + 2) / 2 <= id) ++tn;
    tm = id - tn * (tn + 1) / 2;
  }
  const int m0 = tm * kT, n0 = tn * kT;
  // operands: gram X, X; square A, A; apply B, X
  const _Float16* A = OP == Op::Gram ? x.x[cur] : OP == Op::Square ? x.a : x.b;
  const _Float16* B = OP == Op::Square ? x.a : x.x[cur];
  const int lda = OP == Op::Gram ? n : m, ldb = OP == Op::Square ? m : n;
  const int K = OP == Op::Gram ? n : m;
  const size_t plane_a = (size_t)m * lda, plane_b = (size_t)m * ldb;

  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave & 1) * 64, wn = (wave >> 1) * 64;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  uint32_t aoff[kPieces], boff[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int p = (wave * kPieces + i) * 1024 + 16 * lane;
    aoff[i] = lane_off<true>(lda, m - m0, p);
    boff[i] = lane_off<BK>(ldb, (BK ? m : n) - n0, p);
  }
  const _Float16* abase = A + (size_t)m0 * lda;
  const _Float16* bbase = BK ? B + (size_t)n0 * ldb : B + n0;
  const size_t bstep = BK ? kK : (size_t)kK * ldb;
  const int nk = K / kK, nt = PLANES == 2 ? 3 * nk : nk;
  auto issue = [&](int tt) {
    const int seg = PLANES == 2 ? tt / nk : 2, kt = PLANES == 2 ? tt - seg * nk : tt;
    const _Float16* a = abase + (size_t)kt * kK + (seg == 0 ? plane_a : 0);
    const _Float16* b = bbase + kt * bstep + (seg == 1 ? plane_b : 0);
    const uint32_t at = lds0 + (tt & 1) * 2 * kOpBytes + wave * kPieces * 1024;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      dma16s(a, aoff[i], __builtin_amdgcn_readfirstlane(at + i * 1024));
      dma16s(b, boff[i], __builtin_amdgcn_readfirstlane(at + kOpBytes + i * 1024));
    }
  };

  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  issue(0);
  for (int tt = 0; tt < nt; ++tt) {
    // tile tt has landed for every wave, and every wave is done with tile tt - 1
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tt + 1 < nt) issue(tt + 1);
    const unsigned char* pa = smem + (tt & 1) * 2 * kOpBytes;
    const unsigned char* pb = pa + kOpBytes;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      f16x8 fa[4], fb[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) fa[i] = frag<true>(pa, wm + 16 * i, s, lane);
#pragma unroll
      for (int j = 0; j < 4; ++j) fb[j] = frag<BK>(pb, wn + 16 * j, s, lane);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();

  // Through LDS, so that rows (and the mirror image's rows) go out whole.
  // acc[i][j][e] is row wm + 16 i + (lane & 15), column wn + 16 j + 4 (lane >> 4) + e.
  float* stage = (float*)smem;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4*>(stage + (wm + 16 * i + (lane & 15)) * kRowF + wn + 16 * j +
                                4 * (lane >> 4)) = acc[i][j];
  __syncthreads();
  const int c = 4 * (threadIdx.x & 31);
  const bool cok = n0 + c < (BK ? m : n);
  constexpr float kOut = OP == Op::Gram     ? kNsScaleA / (kNsScaleX * kNsScaleX)
                         : OP == Op::Square ? kNsC * kNsScaleB / (kNsScaleA * kNsScaleA)
                                            : 1.0f / kNsScaleB;
#pragma unroll 4
  for (int r = threadIdx.x >> 5; r < kT; r += kThreads / 32) {
    const int row = m0 + r;
    if (row >= m || !cok) continue;
    float v[4], add[4];
    const f32x4 s4 = *reinterpret_cast<const f32x4*>(stage + r * kRowF + c);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = s4[e] * kOut;
    if constexpr (OP == Op::Gram) {
      ns_store4<PLANES>(x.a + (size_t)row * m + n0 + c, (size_t)m * m, v, 1.0f);
    } else if constexpr (OP == Op::Square) {
      ns_load4<PLANES>(x.a + (size_t)row * m + n0 + c, (size_t)m * m, add,
                       kNsB * kNsScaleB / kNsScaleA);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += add[e];
      ns_store4<PLANES>(x.b + (size_t)row * m + n0 + c, (size_t)m * m, v, 1.0f);
      if (tm != tn) *reinterpret_cast<f32x4*>(stage + r * kRowF + c) = f32x4{v[0], v[1], v[2], v[3]};
    } else {
      ns_load4<PLANES>(x.x[cur] + (size_t)row * n + n0 + c, (size_t)m * n, add, kNsA);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += add[e];
      ns_store4<PLANES>(x.x[cur ^ 1] + (size_t)row * n + n0 + c, (size_t)m * n, v, 1.0f);
    }
  }
  if constexpr (OP != Op::Apply) {
    if (tm == tn) return;
    __syncthreads();
    _Float16* out = OP == Op::Gram ? x.a : x.b;
    const int r4 = 4 * (threadIdx.x & 31);  // four rows of the tile: columns of its image
    if (m0 + r4 >= m) return;
#pragma unroll 4
    for (int cc = threadIdx.x >> 5; cc < kT; cc += kThreads / 32) {
      const int row = n0 + cc;
      if (row >= m) continue;
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = stage[(r4 + e) * kRowF + cc] * (OP == Op::Gram ? kOut : 1.0f);
      ns_store4<PLANES>(out + (size_t)row * m + m0 + r4, (size_t)m * m, v, 1.0f);
    }
  }
}

template <Op OP, int PLANES>
void launch(const NsTable& t, int cur, hipStream_t s) {
  NsTiles tiles{};
  for (int i = 0; i < t.count; ++i) {
    const int tm = tiles_of(t.mat[i].m), tn = tiles_of(t.mat[i].n);
    tiles.first[i + 1] = tiles.first[i] + (OP == Op::Apply ? tm * tn : tm * (tm + 1) / 2);
  }
  ns_gemm_kernel<OP, PLANES><<<tiles.first[t.count], kThreads, 0, s>>>(t, tiles, cur);
}

template <int PLANES>
void step(const NsTable& t, int cur, hipStream_t s) {
  launch<Op::Gram, PLANES>(t, cur, s);
  launch<Op::Square, PLANES>(t, cur, s);
  launch<Op::Apply, PLANES>(t, cur, s);
}

}  // namespace

void launch_ns_step(const NsTable& t, int planes, int cur, hipStream_t s) {
  if (planes == 2) step<2>(t, cur, s);
  else step<1>(t, cur, s);
}

}  // namespace pb

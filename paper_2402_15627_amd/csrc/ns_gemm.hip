// The products of the Newton-Schulz steps, all matrices of a chain in one launch each.
// A step is
//
//   A = X X^T,  B = a I + b A + c A A,  X' = B X
//
// and two steps need X but twice, since A' = X' X'^T = B A B and everything m x m
// commutes:
//
//   A = X X^T,  B = f(A),  A' = (B A) B,  B' = f(A'),  X'' = (B' B) X
//
// Three m x m products for two with X: with half of each symmetric product computed,
// 8 m^3 + 3 (n - m) m^2 operations for 8 m^3 + 6 (n - m) m^2.  (Over more steps the
// spread of A's eigenvalues, the square of X's, costs accuracy: five steps from one A
// lose two digits, pairs between nothing and a factor of 2.5.  256 x 1024: noise alone
// 2.0e-6 off either way; 16 directions beside noise of their elements' size 4.2e-6 in
// pairs and 2.1e-6 step by step, of a hundredth of it 2.7e-5 and 4.5e-5; one plane 3.5e-3
// and 1.7e-3, 3.0e-2 and 3.9e-2.  fp32 is 1.9e-6 and 2.2e-5 off.)
//
//   Sym     L R, L and R symmetric, or X X^T: tiles on and above the diagonal, each
//           written to its mirror image too
//   Square  f(L) likewise
//   Apply   L X
//   Last    the last Apply in 64 x 64 tiles: its result goes to the weights (or to the
//           caller's matrix) from the fp32 sums, which saves a launch.  (In the 256 x 256
//           tiles, where all CUs then write at once, it took 0.9 ms of a 4.3 ms launch
//           over the 175B share, and the pass of its own takes 0.7.)
//
// MFMA v_mfma_f32_16x16x32_f16 on the planes of ns_gemm.h, fp32 accumulation.  One
// plane: one product of fp16 values (rounded by 2^-11 at most).  Two planes (value h
// and remainder l): l h + h h + h l (what is left out, l l, is at most 2^-22 of the
// product).  A K-tile of 128-byte rows is 64 k of one plane or 32 k of both: two planes
// move the same bytes for one and a half times the products.  a goes into B, not into
// Apply's sum: near the end B is about 0.7 to 1.4 instead of -2.7 to -2.0, so its
// rounding moves X' by less (one plane, one row of 777: 3.4e-3 off, 8e-4 so; 512 x 512
// 1.34e-3, 1.24e-3), and apply reads no X beside its operand.
//
// MFMA-bound: the 175B share's products in two planes (44e12 operations a step of five)
// run at 1.38 PFLOP/s, matrix cores busy 72 to 83% at the 1.7 to 1.8 GHz that their power
// allows; in one plane, which the Muon step's bf16 products alone have (5120 x 5120 twice,
// 20480 x 5120), at 1.2, busy 49 to 69%, the operands' way through LDS being longer than
// the products.
//
// Two kernels:
//   - 256 x 256 tiles, eight waves, as the projection GEMMs' LDS-DMA kernel has them
//     (gemm.hip: fragments read two phases ahead, one barrier a K-tile);
//   - 64 x 64 tiles with K split over the waves of a workgroup, for small grids.
// X, A and B are padded to multiples of 64 with zeros, so a K-tile is never partial;
// rows and columns past the end of a tile read the last ones and are not stored.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"
#include "gemm_common.h"
#include "ns_gemm.h"

namespace pb {
namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
#define PB_LDS __attribute__((address_space(3)))

enum class Op { Sym, Square, Apply, Last };
constexpr bool symmetric(Op op) { return op == Op::Sym || op == Op::Square; }

// A product's matrices: of s, or kX for X; and the factor from the sum of its plane
// products to its result's plane values (Last: to its values).
constexpr int kX = -1;
struct Product {
  int left, right, dst;
  float scale;
};
constexpr Product kGram{kX, kX, 0, kNsScaleA / (kNsScaleX * kNsScaleX)};

constexpr int kRow = 64;  // fp16 values of a K-contiguous row of a K-tile: 128 bytes
template <int PLANES>
constexpr int kK = kRow / PLANES;  // k of a K-tile
static_assert(kNsPad == kRow, "X's dimensions are whole K-tiles");

PB_DEV int swz(int row, int c) { return c ^ ((row ^ (row >> 3)) & 7); }
// Rows of W bytes: the four rows of a transposing read, and row groups 8 apart, lie in
// distinct parts of the 256-byte bank period.
template <int W>
PB_DEV int swz_mn(int k, int c) {
  return W >= 256 ? c ^ (4 * (k & 3)) ^ (2 * ((k >> 3) & 1))
                  : c ^ (4 * ((k >> 1) & 1)) ^ (2 * ((k >> 3) & 1));
}

// Byte offset from the operand tile's first element of this lane's 16 bytes of the LDS
// position p, for rows of ld values (both planes counted).  KC: rows of the operand are
// K-contiguous, `rows` of them left; else the operand is K rows of which `rows` columns
// are left.
template <bool KC, int T, int PLANES>
PB_DEV uint32_t lane_off(int ld, int rows, int p) {
  if constexpr (KC) {
    const int row = p >> 7, c = swz(row, (p >> 4) & 7);
    return ((uint32_t)min(row, rows - 1) * (uint32_t)ld + 8 * c) * 2u;
  } else {
    constexpr int kChunks = T * PLANES / 8;  // 16-byte chunks of a k-row
    const int k = p / (16 * kChunks), c = swz_mn<16 * kChunks>(k, (p >> 4) & (kChunks - 1));
    return ((uint32_t)k * (uint32_t)ld + min(8 * c, PLANES * rows - 8)) * 2u;
  }
}
// Fragment f of 16 rows (columns) from `base`: one plane, k 32 f + 8 (lane >> 4) .. + 7;
// two planes, plane f (0 the values, 1 the remainders) of k 8 (lane >> 4) .. + 7.
template <bool KC, int T, int PLANES>
PB_DEV f16x8 frag(const unsigned char* tile, int base, int f, int lane) {
  if constexpr (KC) {
    const int row = base + (lane & 15);
    return *reinterpret_cast<const f16x8*>(tile + row * 128 + swz(row, 4 * f + (lane >> 4)) * 16);
  } else {
    const int i = lane & 15, mn = base + 4 * (i & 3);
    const int k1 = (PLANES == 1 ? 32 * f : 0) + 8 * (lane >> 4) + (i >> 2), k2 = k1 + 4;
    const int c = PLANES == 1 ? mn >> 3 : 8 * (mn >> 5) + 4 * f + ((mn & 31) >> 3);
    constexpr int W = 2 * T * PLANES;  // bytes of a k-row
    const int off = (mn & 7) * 2;
    const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (PB_LDS s16x4*)(tile + k1 * W + swz_mn<W>(k1, c) * 16 + off));
    const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (PB_LDS s16x4*)(tile + k2 * W + swz_mn<W>(k2, c) * 16 + off));
    const f16x4 a4 = __builtin_bit_cast(f16x4, a), b4 = __builtin_bit_cast(f16x4, b);
    return f16x8{a4[0], a4[1], a4[2], a4[3], b4[0], b4[1], b4[2], b4[3]};
  }
}

// ------------------------------------------------------------ work items
// Tile of the triangle tm <= tn of t x t tiles, in bands of four rows walked column by
// column (tiles that run together then share operand strips in an XCD's L2, as in the
// walk of tile_of).
PB_DEV void triangle_tile(int id, int t, int& tm, int& tn) {
  int r0 = 0, g = min(4, t);
  for (;;) {
    const int n = g * (t - r0) - g * (g - 1) / 2;
    if (id < n) break;
    id -= n;
    r0 += g;
    g = min(4, t - r0);
  }
  const int corner = g * (g + 1) / 2;  // column j of the band's first g has j + 1 tiles
  if (id < corner) {
    int j = 0;
    while (id > j) id -= ++j;
    tm = r0 + id;
    tn = r0 + j;
  } else {
    id -= corner;
    tm = r0 + id % g;
    tn = r0 + g + id / g;
  }
}

template <Op OP, int T>
PB_DEV void tile_at(const NsMat& x, int id, int& tm, int& tn) {
  const int t = (x.m + T - 1) / T;
  if constexpr (symmetric(OP)) triangle_tile(id, t, tm, tn);
  else tile_of<4>(id, t, (x.n + T - 1) / T, tm, tn);
}

PB_DEV int place_of(const NsPlan& p, int count, int tile) {
  int i = 0;  // (unrolled: one batch of scalar loads, not a chain of them)
#pragma unroll
  for (int k = 1; k < kNsMaxTensors; ++k)
    if (k < count && tile >= p.first[k]) i = k;
  return i;
}

// Workgroup b's item: tile (counted through the plan) and slice (-1: whole), and the
// tile's place in mat[].  Workgroup b runs on XCD b % 8: the tiles of a matrix (and the
// slices) are dealt out so that each XCD takes a contiguous run of each matrix.
struct Item {
  int tile, slice, place;
};
PB_DEV Item item_of(const NsPlan& p, int count, int b) {
  const int slices = p.tail * p.splits, j = b - p.n_full;
  Item it{b, -1, 0};
  if (j >= 0 && j < slices) {
    const int k = xcd_remap(j, slices);
    it.tile = p.n_full + k / p.splits;
    it.slice = k % p.splits;
    it.place = place_of(p, count, it.tile);
  } else {
    int lo = 0, hi = p.n_full;  // the whole tiles before the cut ones, or those after
    if (j >= 0) lo = hi + p.tail, hi = 0x7fffffff, b -= slices - p.tail;
    it.place = place_of(p, count, b);
    const int f = max(p.first[it.place], lo);
    it.tile = f + xcd_remap(b - f, min(p.first[it.place + 1], hi) - f);
  }
  return it;
}

// Operands of a product: A K-contiguous, B K-contiguous too but for apply's; leading
// dimensions with both planes counted.
struct Operands {
  const _Float16 *A, *B;
  int lda, ldb, K;
};
template <Op OP, int PLANES>
PB_DEV Operands operands(const NsMat& x, const Product& p, int cur) {
  const int m = PLANES * x.ldm, n = PLANES * x.ldn;
  if constexpr (symmetric(OP)) {
    if (p.left == kX) return {x.x[cur], x.x[cur], n, n, x.n};
    return {x.s[p.left], x.s[p.right], m, m, x.m};
  } else {
    return {x.s[p.left], x.x[cur], m, n, x.m};
  }
}

// Matrices of fewer than 16 rows or columns, whose few elements' roundings do not average:
// their steps are not paired (pair_chains), and in 64 x 64 tiles (a call of large matrices
// takes 256 x 256 for all) two planes' products are whole, l l too, and Square's sum is
// fp64.  Off in the median over 30 inputs, so, without either and in fp32: 1 x 777 2.1e-7,
// 8.1e-7 and 5.4e-7; 1 x 64 2.1e-7, 5.4e-7 and 4.0e-7; from 16 rows on fp32 is the
// farthest without.  (For all matrices they would take 4% of a step of small ones.)
__host__ __device__ inline bool few_rows(const NsMat& x) {
  return (x.rows < x.cols ? x.rows : x.cols) < 16;
}

// A's plane values at N consecutive columns n.. of row m, for what Square adds to its
// sums there: a I + b A.
template <Op OP, int PLANES, int N>
PB_DEV void addend(const NsMat& x, const Product& p, int m, int n, float* u) {
  if constexpr (OP == Op::Square)
    ns_load<PLANES, N>(x.s[p.left] + ns_at<PLANES>(x.ldm, m, n), u, 1.0f);
}
// N consecutive columns n.. of row m of a product.  v: the sums (scaled in place), u: those
// of addend().  wide: Square's sum in fp64, rounded once.
template <Op OP, int PLANES, int N>
PB_DEV void store_result(const NsMat& x, const Product& p, int cur, int m, int n, float* v,
                         const float* u, bool wide = false) {
  auto sum = [&](auto zero) {
    using R = decltype(zero);
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const R add = (R)u[e] * (R)(kNsB * kNsScaleB / kNsScaleA) + (m == n + e ? kNsA * kNsScaleB : 0.f);
      v[e] = (float)((R)v[e] * (R)p.scale + add);
    }
  };
  if constexpr (OP == Op::Square) {
    if (wide) sum(0.0);
    else sum(0.f);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] *= p.scale;
  }
  if constexpr (symmetric(OP))
    ns_store<PLANES, N>(x.s[p.dst] + ns_at<PLANES>(x.ldm, m, n), v, 1.0f);
  else ns_store<PLANES, N>(x.x[cur ^ 1] + ns_at<PLANES>(x.ldn, m, n), v, 1.0f);
}
// Eight consecutive rows m.. of column n, v: scaled results.  Symmetric products: the
// mirror image.
template <int PLANES>
PB_DEV void store_mirror8(const NsMat& x, const Product& p, int m, int n, const float* v) {
  ns_store<PLANES, 8>(x.s[p.dst] + ns_at<PLANES>(x.ldm, n, m), v, 1.0f);
}

// ------------------------------------------------------ 256 x 256 tiles
constexpr int kBT = 256;
constexpr int kBThreads = 512;                       // 4 (m) x 2 (n) waves, each 64 x 128
constexpr int kBTile = kBT * kRow * 2;                 // one operand's K-tile: 32 KB
constexpr int kBPieces = kBTile / kBThreads / 16;    // 1 KB pieces per operand per wave: 4
constexpr int kWTM = 64, kWTN = 128;
constexpr int kTM = kWTM / 16, kTN = kWTN / 16;
constexpr int kEpiLds = 32 * kWTN * 4;               // a wave's 32 rows of sums: 16 KB
constexpr size_t kBLds = 4 * (size_t)kBTile;         // two stages of two operands
static_assert(8 * kEpiLds <= (int)kBLds, "staged output fits");

template <int N>
PB_DEV void wait_dma() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// (the wait for LDS is the compiler's own instruction, so that it knows of it)
PB_DEV void block_barrier() {
  __builtin_amdgcn_s_waitcnt(0xc07f);
  asm volatile("s_barrier" ::: "memory");
}

template <Op OP, int PLANES>
__global__ __launch_bounds__(kBThreads, 1) void ns_gemm_big(NsTable t, NsPlan plan, Product prod,
                                                            int cur, float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  constexpr bool BK = symmetric(OP);  // the B operand is K-contiguous
  const Item it = item_of(plan, t.count, blockIdx.x);
  const NsMat& x = t.mat[plan.mat[it.place]];
  int tm, tn;
  tile_at<OP, kBT>(x, it.tile - plan.first[it.place], tm, tn);
  const int m0 = tm * kBT, n0 = tn * kBT, M = x.m, N = BK ? x.m : x.n;
  const Operands o = operands<OP, PLANES>(x, prod, cur);
  const int nk = o.K / kK<PLANES>;
  int kt0 = 0, kt1 = nk;
  if (it.slice >= 0) {
    const int chunk = (nk + plan.splits - 1) / plan.splits;
    kt0 = min(nk, it.slice * chunk);
    kt1 = min(nk, kt0 + chunk);
  }
  const int nt = kt1 - kt0;

  const uint32_t lds0 = (uint32_t)(uintptr_t)(PB_LDS unsigned char*)smem;
  auto a_off = [&](int s) { return (2 * s) * kBTile; };
  auto b_off = [&](int s) { return (2 * s + 1) * kBTile; };
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave & 3) * kWTM, wn = (wave >> 2) * kWTN;

  // Who moves what: every wave its own 4 KB of each operand; but Apply with two planes
  // the first wave of each SIMD both 4 KB regions of its SIMD (two 6144 x 12288: 29.2 ms
  // and 29.3; one plane, 5120 x 5120 twice and 20480 x 5120: 10.56 and 10.51).
  constexpr bool kOwn = BK || PLANES == 1;
  constexpr int kReg = kOwn ? 1 : 2;
  constexpr int kDmaPerTile = 2 * kReg * kBPieces;
  const bool dma_wave = kOwn || wave < 4;
  auto region = [&](int r) { return kOwn ? wave : (wave & 3) + 4 * r; };
  uint32_t aoff[kReg * kBPieces], boff[kReg * kBPieces];
#pragma unroll
  for (int r = 0; r < kReg; ++r)
#pragma unroll
    for (int i = 0; i < kBPieces; ++i) {
      const int p = (region(r) * kBPieces + i) * 1024 + 16 * lane;
      aoff[r * kBPieces + i] = lane_off<true, kBT, PLANES>(o.lda, M - m0, p);
      boff[r * kBPieces + i] = lane_off<BK, kBT, PLANES>(o.ldb, N - n0, p);
    }
  const _Float16* abase = o.A + (size_t)m0 * o.lda;
  const _Float16* bbase = BK ? o.B + (size_t)n0 * o.ldb : o.B + (size_t)PLANES * n0;
  const size_t bstep = BK ? kRow : (size_t)kK<PLANES> * o.ldb;  // values per K-tile
  // this wave's pieces of one operand of the item's K-tile t (half 0: A, half 1: B)
  auto issue_half = [&](int tt, int half) {
    if (!dma_wave) return;
    const int s = tt & 1;
    const _Float16* src = half == 0 ? abase + (size_t)(kt0 + tt) * kRow
                                    : bbase + (size_t)(kt0 + tt) * bstep;
    const uint32_t dst0 = lds0 + (half == 0 ? a_off(s) : b_off(s));
#pragma unroll
    for (int r = 0; r < kReg; ++r)
#pragma unroll
      for (int i = 0; i < kBPieces; ++i)
        dma16s(src, half == 0 ? aoff[r * kBPieces + i] : boff[r * kBPieces + i],
               __builtin_amdgcn_readfirstlane(dst0 + (region(r) * kBPieces + i) * 1024));
  };

  f32x4 acc[kTM][kTN];
#pragma unroll
  for (int i = 0; i < kTM; ++i)
#pragma unroll
    for (int j = 0; j < kTN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  // A K-tile is 8 (one plane) or 12 phases of eight MFMAs, a pair of N blocks times all
  // M blocks of one fragment each; fragments are read kLook phases before the phase that
  // first uses them (gemm.hip has the reasons).
  //   one plane:  phase p takes k-step p / 4 and pair p % 4;
  //   two planes: l h of pairs 0 and 1, h h of both, h l of both, then the same of
  //               pairs 2 and 3: the values of A are first used in phase 2, so they
  //               are read in phase 0, when the last K-tile's are dead.
  constexpr int kPh = PLANES == 2 ? 12 : 8, kLook = 2;
  f16x8 fa[2][kTM], fb[2][kTN];
  auto use = [](int p, int& af, int& bf, int& pair) {
    if (PLANES == 1) {
      af = bf = p >> 2;
      pair = p & 3;
    } else {
      const int q = p % 6;
      af = q < 2;
      bf = q >= 4;
      pair = 2 * (p / 6) + (p & 1);
    }
  };
  // the reads for phase p, of the item's K-tile tt: what no earlier phase has read
  auto reads_a = [](int p) { return PLANES == 1 ? (p & 3) == 0 : p == 0 || p == 2; };
  auto reads_b = [](int p) { return PLANES == 1 || p % 6 < 2 || p % 6 >= 4; };
  auto read_frags = [&](int tt, int p) {
    const int st = tt & 1;
    const unsigned char* pa = smem + a_off(st);
    const unsigned char* pb = smem + b_off(st);
    int af, bf, pair;
    use(p, af, bf, pair);
    if (reads_a(p)) {
#pragma unroll
      for (int i = 0; i < kTM; ++i) fa[af][i] = frag<true, kBT, PLANES>(pa, wm + 16 * i, af, lane);
    }
    if (reads_b(p)) {
#pragma unroll
      for (int j = 2 * pair; j < 2 * pair + 2; ++j)
        fb[bf][j] = frag<BK, kBT, PLANES>(pb, wn + 16 * j, bf, lane);
    }
  };
  auto mma = [&](auto P) {
    constexpr int p = decltype(P)::value;
    int af, bf, pair;
    use(p, af, bf, pair);
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 2 * pair; j < 2 * pair + 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[bf][j], fa[af][i], acc[i][j], 0, 0, 0);
    // one MFMA and one LDS read (a transposed fragment takes two) in turn
    constexpr int pn = (p + kLook) % kPh;
    constexpr int kReads = (reads_a(pn) ? kTM : 0) + (reads_b(pn) ? (BK ? 1 : 2) * 2 : 0);
    constexpr int kMfma = kTM * 2;
    constexpr int pairs = kReads < kMfma ? kReads : kMfma;
#pragma unroll
    for (int u = 0; u < pairs; ++u) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if constexpr (kMfma > pairs) __builtin_amdgcn_sched_group_barrier(0x008, kMfma - pairs, 0);
    if constexpr (kReads > pairs) __builtin_amdgcn_sched_group_barrier(0x100, kReads - pairs, 0);
  };
  auto phase = [&](int tt, auto P) {
    constexpr int p = decltype(P)::value;
    if constexpr (p == kPh - kLook) {
      // every wave has read K-tile tt, and tt + 1 has landed
      wait_dma<0>();
      block_barrier();
      if (tt + 2 < nt) issue_half(tt + 2, 0);
    }
    if constexpr (p == 0)
      if (tt + 1 < nt) issue_half(tt + 1, 1);
    if constexpr (p + kLook < kPh) read_frags(tt, p + kLook);
    else read_frags(tt + 1, p + kLook - kPh);
    mma(P);
    __builtin_amdgcn_sched_barrier(0);
  };
  if (nt > 0) issue_half(0, 0), issue_half(0, 1);
  // (its other half in phase 0, as in every K-tile: with a first K-tile of its own Square
  // in one plane spilled a fragment, and every K-tile waited for the reload and with it for
  // the DMA: 5120 x 5120 twice 293 us, 255 so)
  if (nt > 1) issue_half(1, 0);
  if (nt > 1) wait_dma<kDmaPerTile / 2>();  // tile 0 landed; tile 1 may be in flight
  else wait_dma<0>();
  block_barrier();
#pragma unroll
  for (int p = 0; p < kLook; ++p) {
    read_frags(0, p);
    __builtin_amdgcn_sched_barrier(0);
  }
  for (int tt = 0; tt < nt; ++tt) {
    phase(tt, std::integral_constant<int, 0>{});
    phase(tt, std::integral_constant<int, 1>{});
    phase(tt, std::integral_constant<int, 2>{});
    phase(tt, std::integral_constant<int, 3>{});
    phase(tt, std::integral_constant<int, 4>{});
    phase(tt, std::integral_constant<int, 5>{});
    phase(tt, std::integral_constant<int, 6>{});
    phase(tt, std::integral_constant<int, 7>{});
    if constexpr (PLANES == 2) {
      phase(tt, std::integral_constant<int, 8>{});
      phase(tt, std::integral_constant<int, 9>{});
      phase(tt, std::integral_constant<int, 10>{});
      phase(tt, std::integral_constant<int, 11>{});
    }
  }
  block_barrier();  // every wave is done with the main loop's LDS

  // Through the wave's own 16 KB of LDS, 32 rows at a time (16-byte chunks XOR-ed by the
  // row), so that rows go out in whole lines.  acc[i][j][e] is row wm + 16 i + (lane &
  // 15), column wn + 16 j + 4 (lane >> 4) + e.
  unsigned char* buf = smem + wave * kEpiLds;
  // (opaque, or what is formed from it here would be formed before the main loop and cost
  // it registers)
  int el = lane;
  asm volatile("" : "+v"(el));
  const int c = el & 31, hi = el >> 5;
  const int n = n0 + wn + 4 * c;
  float* pt = it.slice < 0 ? nullptr
                           : part + ((size_t)(it.tile - plan.n_full) * plan.splits + it.slice) *
                                        (kBT * kBT);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int ii = 0; ii < 2; ++ii)
#pragma unroll
      for (int j = 0; j < kTN; ++j) {
        const int rr = 16 * ii + (el & 15), cw = 4 * j + (el >> 4);
        *reinterpret_cast<f32x4*>(buf + rr * (kWTN * 4) + ((cw ^ rr) & 31) * 16) = acc[2 * i + ii][j];
      }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int r = 2 * k + hi;
      f32x4* at = reinterpret_cast<f32x4*>(buf + r * (kWTN * 4) + ((c ^ r) & 31) * 16);
      const int m = m0 + wm + 32 * i + r;
      if (pt) {
        *reinterpret_cast<f32x4*>(pt + (m - m0) * kBT + n - n0) = *at;
        continue;
      }
      const f32x4 s4 = *at;
      float v[4] = {s4[0], s4[1], s4[2], s4[3]};
      if (m < M && n < N) {
        float u[4];
        addend<OP, PLANES, 4>(x, prod, m, n, u);
        store_result<OP, PLANES, 4>(x, prod, cur, m, n, v, u);
        if (symmetric(OP) && tm != tn) *at = f32x4{v[0], v[1], v[2], v[3]};
      }
    }
    if constexpr (symmetric(OP)) {
      // the mirror image: 4 lanes hold the 32 rows of a column, 8 each
      if (pt || tm == tn) continue;
      const int r8 = 8 * (el & 3), mm = m0 + wm + 32 * i + r8;
#pragma unroll
      for (int k = 0; k < kWTN / 16; ++k) {
        const int cc = 16 * k + (el >> 2), nn = n0 + wn + cc;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          v[e] = *reinterpret_cast<const float*>(buf + (r8 + e) * (kWTN * 4) +
                                                 (((cc >> 2) ^ (r8 + e)) & 31) * 16 + (cc & 3) * 4);
        if (nn < N && mm < M) store_mirror8<PLANES>(x, prod, mm, nn, v);
      }
    }
  }
}

// Sum of a split T x T tile's slices, in slice order, and its result: 64 x 64 of the tile
// per workgroup.
template <Op OP, int PLANES, int T>
__global__ __launch_bounds__(256) void ns_reduce_kernel(NsTable t, NsPlan plan, Product prod,
                                                        int cur, const float* __restrict__ part) {
  __shared__ float lds[64][65];
  constexpr int kSub = T / 64;  // blocks across a tile
  const int tail = blockIdx.x / (kSub * kSub), sub = blockIdx.x % (kSub * kSub);
  const int tile = plan.n_full + tail, place = place_of(plan, t.count, tile);
  const NsMat& x = t.mat[plan.mat[place]];
  int tm, tn;
  tile_at<OP, T>(x, tile - plan.first[place], tm, tn);
  const int r0 = sub / kSub * 64, c0 = sub % kSub * 64, cl = 4 * (threadIdx.x & 15);
  const int m0 = tm * T + r0, n0 = tn * T + c0, N = symmetric(OP) ? x.m : x.n;
  // (M and N are multiples of 64: the 64 x 64 block is inside or outside whole)
  if (m0 >= x.m || n0 >= N) return;
  const float* p = part + (size_t)tail * plan.splits * (T * T) + c0 + cl;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int rl = (threadIdx.x >> 4) + 16 * k;
    const float* q = p + (r0 + rl) * T;
    f32x4 s = *reinterpret_cast<const f32x4*>(q);
#pragma unroll 4
    for (int i = 1; i < plan.splits; ++i)
      s += *reinterpret_cast<const f32x4*>(q + (size_t)i * T * T);
    float v[4] = {s[0], s[1], s[2], s[3]}, u[4];
    addend<OP, PLANES, 4>(x, prod, m0 + rl, n0 + cl, u);
    store_result<OP, PLANES, 4>(x, prod, cur, m0 + rl, n0 + cl, v, u);
#pragma unroll
    for (int e = 0; e < 4; ++e) lds[rl][cl + e] = v[e];
  }
  if constexpr (symmetric(OP)) {
    if (tm == tn) return;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int cc = (threadIdx.x >> 3) + 32 * k, r8 = 8 * (threadIdx.x & 7);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = lds[r8 + e][cc];
      store_mirror8<PLANES>(x, prod, m0 + r8, n0 + cc, v);
    }
  }
}

// -------------------------------------------------------- 64 x 64 tiles
// Eight waves; wave w takes K-tiles w, w + 8, ... of the 64 x 64 tile, so the waves
// share no operand values and the loop has no barrier.  Operands go through registers
// and 16 KB of LDS of the wave's own: a fragment's quarter-wave lies in 16 rows, so
// loading it straight from global memory takes 64 cache lookups an instruction (3.4 us
// a K-tile of all waves), where eight lanes that share a row's 128 bytes take 8.  The
// next K-tile's loads are in flight while one is multiplied.  The sums are added
// through LDS in wave order.
constexpr int kST = 64;
constexpr int kSWaves = 8;
constexpr int kSThreads = 64 * kSWaves;
constexpr int kSWaveLds = kST * kST * 4;  // a wave's sums: 16 KB
constexpr size_t kSLds = (size_t)kSWaves * kSWaveLds;

// One operand of a wave.  (M, N and K are multiples of 64: a tile is whole.)
template <bool KC, int PLANES>
struct SmallSide {
  const _Float16* p;  // wave-uniform
  size_t step;
  uint32_t off[8];    // bytes
  PB_DEV void init(const _Float16* X, int ld, int R0, int kt, int lane) {
    p = KC ? X + (size_t)R0 * ld + (size_t)kt * kRow
           : X + (size_t)kt * kK<PLANES> * ld + (size_t)PLANES * R0;
    step = (size_t)kSWaves * (KC ? kRow : kK<PLANES> * (size_t)ld);
#pragma unroll
    for (int q = 0; q < 8; ++q) off[q] = lane_off<KC, kST, PLANES>(ld, kST, 1024 * q + 16 * lane);
  }
  // The next K-tile's 16 bytes of 1 KB piece q.
  PB_DEV void load(u32x4 (&r)[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q)
      r[q] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const char*>(p) + off[q]);
    p += step;
  }
  static PB_DEV void put(const u32x4 (&r)[8], unsigned char* lds, int lane) {
#pragma unroll
    for (int q = 0; q < 8; ++q) *reinterpret_cast<u32x4*>(lds + 1024 * q + 16 * lane) = r[q];
  }
  static PB_DEV void frags(const unsigned char* lds, int lane, f16x8 (&f)[4][2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k) f[i][k] = frag<KC, kST, PLANES>(lds, 16 * i, k, lane);
  }
};

template <Op OP, int PLANES>
__global__ __launch_bounds__(kSThreads, 1) void ns_gemm_small(NsTable t, NsPlan plan, Product prod,
                                                              NsFinish fin, int cur,
                                                              float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
  constexpr bool BK = symmetric(OP);
  const Item it = item_of(plan, t.count, blockIdx.x);
  const NsMat& x = t.mat[plan.mat[it.place]];
  int tm, tn;
  tile_at<OP, kST>(x, it.tile - plan.first[it.place], tm, tn);
  const int m0 = tm * kST, n0 = tn * kST;
  const Operands o = operands<OP, PLANES>(x, prod, cur);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // K-tiles kt0 .. kt0 + nk - 1: the slice's
  int kt0 = 0, nk = o.K / kK<PLANES>;
  if (it.slice >= 0) {
    const int chunk = (nk + plan.splits - 1) / plan.splits;
    kt0 = min(nk, it.slice * chunk);
    nk = min(nk, kt0 + chunk) - kt0;
  }
  unsigned char* own = smem + wave * kSWaveLds;
  const bool few = PLANES == 2 && few_rows(x);

  f32x4 acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  SmallSide<true, PLANES> sa;
  SmallSide<BK, PLANES> sb;
  sa.init(o.A, o.lda, m0, kt0 + wave, lane);
  sb.init(o.B, o.ldb, n0, kt0 + wave, lane);
  u32x4 ra[8], rb[8];
  if (wave < nk) sa.load(ra), sb.load(rb);
  // this thread's part of the result, a row's eight columns (a column's eight rows for a
  // tall matrix's tensor), and what it needs from memory for it, ahead of the products
  const int r = threadIdx.x >> 3, c8 = 8 * (threadIdx.x & 7);
  const bool tall = x.rows > x.cols;
  float u[8];
  if constexpr (OP == Op::Last) weights<8>(x, fin, tall ? n0 + r : m0 + r, (tall ? m0 : n0) + c8, u);
  else if (it.slice < 0) addend<OP, PLANES, 8>(x, prod, m0 + r, n0 + c8, u);
  for (int kt = wave; kt < nk; kt += kSWaves) {
    unsigned char* own_b = own + kSWaveLds / 2;
    sa.put(ra, own, lane);
    sb.put(rb, own_b, lane);
    if (kt + kSWaves < nk) sa.load(ra), sb.load(rb);  // in flight while this one multiplies
    f16x8 fa[4][2], fb[4][2];
    sa.frags(own, lane, fa);
    sb.frags(own_b, lane, fb);
    auto mma = [&](int af, int bf) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j][bf], fa[i][af], acc[i][j], 0, 0, 0);
    };
    if constexpr (PLANES == 2) {
      if (few) mma(1, 1);
      mma(1, 0), mma(0, 1), mma(0, 0);
    }
    else mma(0, 0), mma(1, 1);
  }

  // acc[i][j][e] is row 16 i + (lane & 15), column 16 j + 4 (lane >> 4) + e; 16-byte
  // chunks XOR-ed by the row
  const int waves = max(1, min(kSWaves, nk));
  if (wave < waves) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 16 * i + (lane & 15), c = 4 * j + (lane >> 4);
        *reinterpret_cast<f32x4*>(own + r * (kST * 4) + ((c ^ r) & 15) * 16) = acc[i][j];
      }
  }
  __syncthreads();
  float v[8];
  auto sum_at = [&](int w, int h) {
    return *reinterpret_cast<const f32x4*>(smem + w * kSWaveLds + r * (kST * 4) +
                                           ((((c8 >> 2) + h) ^ r) & 15) * 16);
  };
  f32x4 sum[2];
  if (waves == kSWaves) {
    // all the reads at once: five steps of 256 x 256 in fp32 112.3 us one after the other,
    // 108.1 so (for fewer waves so many reads take longer: 64 x 256 78.4 and 82.1)
    f32x4 q[2][kSWaves];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int w = 0; w < kSWaves; ++w) q[h][w] = sum_at(w, h);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] = q[h][0];
#pragma unroll
      for (int w = 1; w < kSWaves; ++w) sum[h] += q[h][w];
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      sum[h] = sum_at(0, h);
      for (int w = 1; w < waves; ++w) sum[h] += sum_at(w, h);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = sum[e >> 2][e & 3];
  if (it.slice >= 0) {
    float* p = part + ((size_t)(it.tile - plan.n_full) * plan.splits + it.slice) * (kST * kST) +
               r * kST + c8;
    store8<float>(p, v);
    return;
  }
  if constexpr (OP == Op::Last) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= prod.scale;
    if (!tall) finish<8>(x, fin, m0 + r, n0 + c8, v, u);
  } else {
    store_result<OP, PLANES, 8>(x, prod, cur, m0 + r, n0 + c8, v, u, few);
  }
  if (OP == Op::Apply || (OP == Op::Last ? !tall : tm == tn)) return;
  __syncthreads();
  float* turned = (float*)smem;  // [64][65]
#pragma unroll
  for (int e = 0; e < 8; ++e) turned[(c8 + e) * 65 + r] = v[e];
  __syncthreads();
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = turned[r * 65 + c8 + e];  // column r, eight rows
  if constexpr (OP == Op::Last) finish<8>(x, fin, n0 + r, m0 + c8, v, u);
  else store_mirror8<PLANES>(x, prod, m0 + c8, n0 + r, v);
}

// ---------------------------------------------------------------- plans
int tiles_of(Op op, const NsMat& x, int t) {
  const int tm = (x.m + t - 1) / t, tn = (x.n + t - 1) / t;
  return symmetric(op) ? tm * (tm + 1) / 2 : tm * tn;
}

// Time of a K-tile of a 256 x 256 tile with the chip full, and around a tile (launch,
// prologue, epilogue), in us.
template <int PLANES>
constexpr double kStepUs = PLANES == 2 ? 1.9 : 1.65;
constexpr double kTileUs = 14.0, kSplitUs = 9.0;
// The same for the 64 x 64 tiles, a step being a K-tile of each of the eight waves.
template <int PLANES>
constexpr double kSmallStepUs = PLANES == 2 ? 2.05 : 1.9;
constexpr double kSmallTileUs = 2.5, kSmallUs = 5.0, kSmallSplitUs = 7.0;

// When the last of kCUs CUs is done that take groups of equal items one after the other,
// each CU the next item as it ends one.
class Makespan {
 public:
  void take(int n, double us) {
    if (n <= 0) return;
    if (n > 4 * kCUs) {  // (whole rounds in one step)
      const int r = n / kCUs - 2;
      for (int i = 0; i < n_; ++i) c_[i].at += r * us;
      n -= r * kCUs;
    }
    while (n > 0) {
      int first = 0;
      for (int i = 1; i < n_; ++i)
        if (c_[i].at < c_[first].at) first = i;
      const double at = c_[first].at + us;
      int k = std::min(n, c_[first].cus), to = 0;
      n -= k;
      while (to < n_ && c_[to].at != at) ++to;
      if (to == n_ && n_ == kMost) to = first;  // (never seen: an estimate all the same)
      if (to == n_) c_[n_++] = {at, 0};
      c_[to].cus += k;
      if ((c_[first].cus -= k) == 0) c_[first] = c_[--n_];
    }
  }
  double last() const {
    double at = 0.0;
    for (int i = 0; i < n_; ++i) at = std::max(at, c_[i].at);
    return at;
  }

 private:
  static constexpr int kMost = 64;
  struct {
    double at;
    int cus;
  } c_[kMost + 1] = {{0.0, kCUs}};
  int n_ = 1;
};

// The tiles that are estimated to end sooner: 256 x 256, whole rounds of them and tiles
// after those cut along K, all or the ones of the longest K among them; or 64 x 64, all of
// them cut where they are few and K is long.  (The symmetric products of the 175B share,
// 600 tiles of K = 6144 and 84 of 1536: 88 of the long ones cut in two 1.11 ms, those and
// the short ones cut in five 1.26.)
template <int PLANES>
NsLaunch choose(Op op, bool gram, const NsTable& t) {
  NsPlan plan{};
  auto len = [&](int i) { return (gram ? t.mat[i].n : t.mat[i].m) / kK<PLANES>; };
  for (int i = 0; i < t.count; ++i) {  // the longest K first
    int k = i;
    for (; k > 0 && len(plan.mat[k - 1]) < len(i); --k) plan.mat[k] = plan.mat[k - 1];
    plan.mat[k] = i;
  }
  auto count = [&](int size) {
    for (int i = 0; i < t.count; ++i)
      plan.first[i + 1] = plan.first[i] + tiles_of(op, t.mat[plan.mat[i]], size);
    return plan.first[t.count];
  };
  // The items' time, tiles n_full .. n_full + tail - 1 in `splits` slices; us(nk): of an
  // item of nk K-tiles
  auto items = [&](auto us, int n_full, int tail, int splits) {
    Makespan m;
    for (int part = 0; part < 3; ++part) {
      const int lo = part == 0 ? 0 : part == 1 ? n_full : n_full + tail;
      const int hi = part == 0 ? n_full : part == 1 ? n_full + tail : plan.first[t.count];
      for (int i = 0; i < t.count; ++i) {
        const int n = std::min(plan.first[i + 1], hi) - std::max(plan.first[i], lo);
        const int nk = len(plan.mat[i]);
        if (part == 1) m.take(n * splits, us((nk + splits - 1) / splits));
        else m.take(n, us(nk));
      }
    }
    return m.last();
  };
  NsLaunch c{};
  double best = INFINITY;
  auto offer = [&](bool big, int n_full, int tail, int splits, double us) {
    if (us >= best) return;
    best = us;
    c.big = big;
    c.plan = plan;
    c.plan.n_full = n_full;
    c.plan.tail = tail;
    c.plan.splits = splits;
    c.us = us;
  };
  auto big_us = [](int nk) { return kStepUs<PLANES> * nk; };
  int tiles = count(kBT);
  offer(true, tiles, 0, 1, kTileUs + items(big_us, tiles, 0, 1));
  for (int keep = tiles / kCUs; keep >= std::max(0, tiles / kCUs - 1); --keep) {
    const int full = keep * kCUs;
    int end = 0;  // of the matrices with the K of tile `full`
    for (int i = 0; i < t.count && end <= full; ++i)
      if (i + 1 == t.count || len(plan.mat[i]) != len(plan.mat[i + 1])) end = plan.first[i + 1];
    for (int whole = 0; whole < (end < tiles ? 2 : 1); ++whole) {
      const int tail = (whole ? tiles : end) - full;
      for (int s = 2; tail > 0 && s <= 16 && tail * s <= 4 * kCUs; ++s)
        offer(true, full, tail, s,
              kTileUs + items(big_us, full, tail, s) + kSplitUs + 0.05 * tail * s);
    }
  }
  auto small_us = [](int nk) {
    return kSmallTileUs + kSmallStepUs<PLANES> * ((nk + kSWaves - 1) / kSWaves);
  };
  tiles = count(kST);
  for (int s = 1; s <= 16 && (s == 1 || (gram && tiles <= 2 * kCUs / s)); ++s) {
    const int full = s == 1 ? tiles : 0;
    offer(false, full, tiles - full, s,
          kSmallUs + items(small_us, full, tiles - full, s) +
              (s > 1 ? kSmallSplitUs + 0.01 * tiles * s : 0.0));
  }
  return c;
}

template <Op OP, int PLANES>
void launch(const NsTable& t, const NsLaunch& c, const Product& p, const NsFinish& fin, int cur,
            float* part, hipStream_t s) {
  const int tail = c.plan.tail, items = c.plan.first[t.count] + tail * (c.plan.splits - 1);
  if (!c.big) {
    ns_gemm_small<OP, PLANES><<<items, kSThreads, kSLds, s>>>(t, c.plan, p, fin, cur, part);
    if constexpr (OP == Op::Sym)
      if (tail)
        ns_reduce_kernel<OP, PLANES, kST><<<tail, 256, 0, s>>>(t, c.plan, p, cur, part);
  } else if constexpr (OP != Op::Last) {
    ns_gemm_big<OP, PLANES><<<items, kBThreads, kBLds, s>>>(t, c.plan, p, cur, part);
    if (tail)
      ns_reduce_kernel<OP, PLANES, kBT><<<tail * 16, 256, 0, s>>>(t, c.plan, p, cur, part);
  }
}

template <int PLANES>
void iterate(const NsTable& matrices, const NsFinish& fin, int steps, const NsProducts& p,
             float* part, hipStream_t s) {
  constexpr float kSquare = kNsC * kNsScaleB / (kNsScaleA * kNsScaleA);
  NsTable t = matrices;
  int cur = 0;
  auto sym = [&](const NsLaunch& c, const Product& q) {
    launch<Op::Sym, PLANES>(t, c, q, fin, cur, part, s);
  };
  auto square = [&](int from, int to) {
    launch<Op::Square, PLANES>(t, p.square, Product{from, from, to, kSquare}, fin, cur, part, s);
  };
  for (int left = steps; left > 0; cur ^= 1) {
    const int lent = ns_lent(p);  // (A; in pairs B A and B')
    for (int i = 0; i < t.count; ++i)
      if (!matrices.mat[i].s[lent]) t.mat[i].s[lent] = t.mat[i].x[cur ^ 1];
    sym(p.gram, kGram);  // A
    square(0, 1);        // B
    int by = 1;
    float scale = kNsScaleB;  // of what X is multiplied by
    if (p.paired && left > 1) {
      sym(p.square, Product{1, 0, 2, 1.0f / kNsScaleB});  // B A
      sym(p.square, Product{2, 1, 0, 1.0f / kNsScaleB});  // A' = B A B
      square(0, 2);                                       // B'
      sym(p.square, Product{2, 1, 0, kNsScaleQ / (kNsScaleB * kNsScaleB)});  // B' B
      by = 0;
      scale = kNsScaleQ;
      --left;
    }
    --left;
    if (left == 0 && !p.apply.big)
      launch<Op::Last, PLANES>(t, p.apply, Product{by, kX, kX, 1.0f / (scale * kNsScaleX)}, fin,
                               cur, part, s);
    else
      launch<Op::Apply, PLANES>(t, p.apply, Product{by, kX, kX, 1.0f / scale}, fin, cur, part, s);
  }
}

}  // namespace

namespace {

// Estimate of two steps; a launch in a chain costs about kLaunchUs less than by itself.
constexpr double kLaunchUs = 5.0;
double two_steps(const NsProducts& p) {
  return p.paired ? p.gram.us + 5 * p.square.us + p.apply.us - 7 * kLaunchUs
                  : 2 * (p.gram.us + p.square.us + p.apply.us) - 6 * kLaunchUs;
}
double two_steps(const NsChains& c) {
  double us = 0.0;
  for (int k = 0; k < c.count; ++k) us += two_steps(c.p[k]);
  return us;
}

// The table with the matrices for which f holds first; n: their number.
template <typename F>
NsTable ordered(const NsTable& t, F f, int& n) {
  NsTable u{};
  for (int k = 0; k < 2; ++k) {
    for (int i = 0; i < t.count; ++i)
      if (f(t.mat[i]) == (k == 0)) u.mat[u.count++] = t.mat[i];
    if (k == 0) n = u.count;
  }
  auto tiles = [](int v) { return (v + kNsPad - 1) / kNsPad; };
  for (int i = 0; i < u.count; ++i)
    u.tile0[i + 1] = u.tile0[i] + tiles(u.mat[i].rows) * tiles(u.mat[i].cols);
  return u;
}

// One chain, or one of the wide matrices in pairs of steps and one of the others.
NsChains pair_chains(NsTable& t, int planes) {
  auto plan = [&](const NsTable& u, bool paired) {
    auto of = [&](Op op, bool gram) {
      return planes == 2 ? choose<2>(op, gram, u) : choose<1>(op, gram, u);
    };
    return NsProducts{of(Op::Sym, true), of(Op::Square, false), of(Op::Apply, false), paired};
  };
  // Pairs of steps only where X is at least twice as wide as tall: in a square one the
  // roundings of A' show (300 x 300, fp32 2.7e-6 off in pairs, 1.8e-6 step by step; one
  // plane 1.8e-3 and 1.3e-3; 128 x 256 1.3e-6 and 1.4e-6; 1.1e-3 either way).  And not
  // under 16 rows (1 x 777 in pairs 1.6 times as far off; 16 x 777 5.7e-7 step by step and
  // 7.7e-7, where fp32 products are off by 1.3e-6).
  int n = 0;
  const NsTable order = ordered(t, [](const NsMat& x) {
    return !few_rows(x) && std::max(x.rows, x.cols) >= 2 * std::min(x.rows, x.cols);
  }, n);
  NsChains c{1, {t.count}, {planes}, {plan(t, false)}, 0};
  // Five steps, in pairs and step by step: fp32 64 x 1024 99 and 106 us, 256 x 1024 145
  // and 144, 2048 x 4096 1037 and 1085, 4096 x 8192 5670 and 6260; one plane 64 x 4096 98
  // and 111, 1024 x 4096 261 and 291 (chosen); 1024 x 2048, chosen too, 206 and 201.
  if (n == t.count) {
    NsProducts p = c.p[0];
    p.paired = true;
    if (two_steps(p) < two_steps(c) - 0.05 * (p.gram.us + p.apply.us)) c.p[0] = p;
  } else if (n > 0 && two_steps(c) > 3 * 7 * kLaunchUs) {
    // two chains, where the seven launches more are repaid (pairs save a third at most)
    const NsChains d{2, {n, t.count}, {planes, planes},
                     {plan(ns_slice(order, 0, n), true), plan(ns_slice(order, n, t.count), false)}, 0};
    if (two_steps(d) < 0.95 * two_steps(c)) {
      t = order;
      return d;
    }
  }
  return c;
}

}  // namespace

// One plane serves the Muon step's bf16 products from 64 rows and columns on.  Under that
// the roundings of few elements show (16 x 16 off by up to 2.6e-3, 64 x 64 by 1.5e-3) and a
// step is latency:
// five steps of 64 x 256 take 70 us in one plane, of 60 x 256 82 in two.  Beside larger
// matrices the small ones have a chain of their own, or all of a call take two planes,
// whichever is estimated to end sooner.
void ns_plan(NsTable& t, bool f32_products, NsChains* c) {
  int n = 0;
  NsTable order = ordered(t, [](const NsMat& x) { return std::min(x.rows, x.cols) < 64; }, n);
  if (f32_products || n == 0 || n == t.count) {
    *c = pair_chains(t, f32_products || n ? 2 : 1);
  } else {
    NsTable small = ns_slice(order, 0, n), rest = ns_slice(order, n, t.count);
    const NsChains a = pair_chains(small, 2), b = pair_chains(rest, 1);
    *c = pair_chains(t, 2);
    if (two_steps(a) + two_steps(b) < two_steps(*c)) {
      *c = a;
      for (int k = 0; k < b.count; ++k) {
        c->end[c->count] = n + b.end[k];
        c->planes[c->count] = b.planes[k];
        c->p[c->count++] = b.p[k];
      }
      for (int i = 0; i < t.count; ++i) order.mat[i] = i < n ? small.mat[i] : rest.mat[i - n];
      t = ordered(order, [](const NsMat&) { return true; }, n);
    }
  }
  c->partial_floats = 0;
  for (int k = 0; k < c->count; ++k)
    for (const NsLaunch* l : {&c->p[k].gram, &c->p[k].square, &c->p[k].apply})
      c->partial_floats =
          std::max(c->partial_floats, (size_t)l->plan.tail * l->plan.splits *
                                          (l->big ? kBT * kBT : kST * kST));
}

void launch_ns_products(const NsTable& t, const NsFinish& fin, int planes, int steps,
                        const NsProducts& p, float* part, hipStream_t s) {
  if (planes == 2) iterate<2>(t, fin, steps, p, part, s);
  else iterate<1>(t, fin, steps, p, part, s);
}

}  // namespace pb

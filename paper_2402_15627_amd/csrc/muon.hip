// The Muon step's passes over its tensors, and the orthogonalisation of matrices
// by Newton-Schulz steps (Muon: Jordan et al. 2024):
//
//   M = mu M + g,  U = g + mu M (Nesterov) or M;  X = U / (||U||_F + eps)
//   `steps` times:  A = X X^T,  B = a I + b A + c A A,  X = B X
//   w = w (1 - lr decay) - lr scale X
//
// with X of m <= n (U, or its transpose).  The odd polynomial a s + b s^3 + c s^5
// moves every singular value of X in [0, 1] towards 1 and stays in [0, 1.203].
//
//   1. update: M in place, the sum of U^2 per 64 x 64 tile, in fp64
//   2. norm:   1 / (||U||_F + eps) of each matrix (few tiles: part of 3)
//   3. init:   X's fp16 planes, padded to multiples of 64 with zeros
//   4. the products (ns_gemm.hip), each one launch for all matrices of a chain
//   5. finish: w and its copy, or the orthogonalised matrix itself; part of the last
//      product where that runs in small tiles
//
// 1, 3 and 5 are HBM-bound: a 64 x 64 tile per workgroup, 256 contiguous bytes of
// a row per 16 lanes; a tall matrix's tile is transposed through LDS (226 M elements of
// the 175B share: 0.54, 0.53 and 0.61 ms, 5.0, 5.1 and 5.2 TB/s).  A step of those takes
// 33.5 ms, 32 of them products at the matrix cores' power limit; one of six matrices of
// 256 x 256 and 1024 x 256 0.15 ms, 17 launches of about 8 us each in a row.
#include "common.h"
#include "kernels.h"
#include "ns_gemm.h"

namespace pb {
namespace {

constexpr int kTile = 64;
constexpr int kThreads = 256;

PB_DEV int mat_of(const NsTable& t, int tile) {
  int i = 0;
#pragma unroll
  for (int k = 1; k < kNsMaxTensors; ++k)
    if (k < t.count && tile >= t.tile0[k]) i = k;
  return i;
}

// Four columns c..c+3 of a row, of which `left` exist; p: the row's start.
template <typename T>
PB_DEV void load4_cols(const T* p, int c, int left, bool vec, float* v) {
  if (vec && left >= 4) {
    load4<T>(p + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < left ? load1<T>(p + c + e) : 0.f;
  }
}
template <typename T>
PB_DEV void store4_cols(T* p, int c, int left, bool vec, const float* v) {
  if (vec && left >= 4) {
    store4<T>(p + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < left) p[c + e] = (T)v[e];
  }
}

// Whether four columns from a multiple of four on are one aligned access in every row.
template <typename T>
PB_DEV bool rows_vec(const void* p, long long ld) {
  return ld % 4 == 0 && (uintptr_t)p % (4 * sizeof(T)) == 0;
}

// The tile of the tensor that this workgroup takes.
struct TileAt {
  int i, r0, c0;
};
PB_DEV TileAt tile_at(const NsTable& t) {
  const int tile = blockIdx.x, i = mat_of(t, tile), k = tile - t.tile0[i];
  const int across = (t.mat[i].cols + kTile - 1) / kTile;
  return {i, k / across * kTile, k % across * kTile};
}

template <NsMode MODE>
__global__ __launch_bounds__(kThreads) void ns_update_kernel(NsTable t, NsScalars sc,
                                                             double* __restrict__ partial) {
  using T = typename std::conditional<MODE == NsMode::Bf16, bf16, float>::type;
  __shared__ double red[kThreads / 64];
  const TileAt at = tile_at(t);
  const NsMat& x = t.mat[at.i];
  const bool vec = rows_vec<T>(x.src, x.ld_src) &&
                   (MODE != NsMode::Muon || rows_vec<float>(x.mom, x.ld_src));
  const int c = at.c0 + 4 * (threadIdx.x & 15), left = x.cols - c;
  double ss = 0.0;
  float g[4][4], m[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = at.r0 + (threadIdx.x >> 4) + 16 * k;
    const bool in = r < x.rows && left > 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) g[k][e] = m[k][e] = 0.f;
    if (in) load4_cols((const T*)x.src + r * x.ld_src, c, left, vec, g[k]);
    if (MODE == NsMode::Muon && in) load4_cols(x.mom + r * x.ld_src, c, left, vec, m[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = at.r0 + (threadIdx.x >> 4) + 16 * k;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float u = g[k][e];
      if constexpr (MODE == NsMode::Muon) {
        u *= sc.grad_scale;
        m[k][e] = __builtin_fmaf(sc.momentum, m[k][e], u);
        u = sc.nesterov ? __builtin_fmaf(sc.momentum, m[k][e], u) : m[k][e];
      }
      ss += (double)u * u;
    }
    if (MODE == NsMode::Muon && r < x.rows && left > 0)
      store4_cols(x.mom + r * x.ld_src, c, left, vec, m[k]);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// norm[i] = 1 / (||U|| + eps) of matrix i.
constexpr int kNormThreads = 1024;
__global__ __launch_bounds__(kNormThreads) void ns_norm_kernel(NsTable t, float eps,
                                                               const double* __restrict__ partial,
                                                               double* __restrict__ norm) {
  __shared__ double red[kNormThreads / 64];
  const int i = blockIdx.x, end = t.tile0[i + 1];
  double s[4] = {0.0, 0.0, 0.0, 0.0};  // (four loads in flight)
  for (int k = t.tile0[i] + threadIdx.x; k < end; k += 4 * kNormThreads)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const double v = partial[min(k + e * kNormThreads, end - 1)];
      s[e] += k + e * kNormThreads < end ? v : 0.0;
    }
  double ss = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kNormThreads / 64; ++w) ss += red[w];
    norm[i] = 1.0 / (sqrt(ss) + (double)eps);
  }
}

// X's tile of 64 x 64 at (i0, j0) of its padded m x n from U's tile of the tensor.  sums:
// ns_norm_kernel's factors; or (FOLD) the tiles' sums, kThreads to a matrix at most, that
// every workgroup then adds up itself, in the order of that kernel: a launch less for a
// longer start here (five steps of 256 x 256 in fp32 113.7 us with the launch, 112.1
// without; 64 x 256 80.9 and 79.4).
template <NsMode MODE, int PLANES, bool FOLD>
__global__ __launch_bounds__(kThreads) void ns_init_kernel(NsTable t, NsScalars sc,
                                                           const double* __restrict__ sums) {
  using T = typename std::conditional<MODE == NsMode::Bf16, bf16, float>::type;
  __shared__ float lds[kTile][kTile + 1];
  const TileAt at = tile_at(t);
  const NsMat& x = t.mat[at.i];
  const bool tall = x.rows > x.cols;
  const bool vec = rows_vec<T>(x.src, x.ld_src) &&
                   (MODE != NsMode::Muon || rows_vec<float>(x.mom, x.ld_src));
  double f;  // (in fp32 that of a norm past 1e38 has lost its bits)
  if constexpr (FOLD) {
    __shared__ double red[kThreads / 64];
    const int k0 = t.tile0[at.i], n = t.tile0[at.i + 1] - k0;
    double ss = (int)threadIdx.x < n ? sums[k0 + threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
    __syncthreads();
    f = 1.0 / (sqrt(((red[0] + red[1]) + red[2]) + red[3]) + (double)sc.eps);
  } else {
    f = sums[at.i];
  }
  const int cl = 4 * (threadIdx.x & 15), c = at.c0 + cl, left = x.cols - c;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int rl = (threadIdx.x >> 4) + 16 * k, r = at.r0 + rl;
    float u[4] = {0.f, 0.f, 0.f, 0.f}, g[4];
    if (r < x.rows && left > 0) {
      if constexpr (MODE == NsMode::Muon) {
        load4_cols(x.mom + r * x.ld_src, c, left, vec, u);
        if (sc.nesterov) {
          load4_cols((const float*)x.src + r * x.ld_src, c, left, vec, g);
#pragma unroll
          for (int e = 0; e < 4; ++e) u[e] = __builtin_fmaf(sc.momentum, u[e], g[e] * sc.grad_scale);
        }
      } else {
        load4_cols((const T*)x.src + r * x.ld_src, c, left, vec, u);
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float v = (float)(u[e] * f);
      if (tall) lds[cl + e][rl] = v;
      else lds[rl][cl + e] = v;
    }
  }
  __syncthreads();
  const int i0 = tall ? at.c0 : at.r0, j0 = tall ? at.r0 : at.c0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = (threadIdx.x >> 3) + 32 * k, j = 8 * (threadIdx.x & 7);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = lds[i][j + e];
    ns_store<PLANES, 8>(x.x[0] + ns_at<PLANES>(x.ldn, i0 + i, j0 + j), v, kNsScaleX);
  }
}

// The tensors from the last iterate, in x[last], where the last product has not
// written them.
template <int PLANES>
__global__ __launch_bounds__(kThreads) void ns_finish_kernel(NsTable t, NsFinish fin, int last) {
  __shared__ float lds[kTile][kTile + 1];
  const TileAt at = tile_at(t);
  const NsMat& x = t.mat[at.i];
  const bool tall = x.rows > x.cols;
  const int i0 = tall ? at.c0 : at.r0, j0 = tall ? at.r0 : at.c0;
  const int rl = threadIdx.x >> 4, cl = 4 * (threadIdx.x & 15);
  float u[4][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) weights<4>(x, fin, at.r0 + rl + 16 * k, at.c0 + cl, u[k]);
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = (threadIdx.x >> 3) + 32 * k, j = 8 * (threadIdx.x & 7);
    float v[8];
    ns_load<PLANES, 8>(x.x[last] + ns_at<PLANES>(x.ldn, i0 + i, j0 + j), v, 1.0f / kNsScaleX);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (tall) lds[j + e][i] = v[e];
      else lds[i][j + e] = v[e];
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = lds[rl + 16 * k][cl + e];
    finish<4>(x, fin, at.r0 + rl + 16 * k, at.c0 + cl, v, u[k]);
  }
}

// A chain: X's planes, products, the tensors.
template <NsMode MODE, int PLANES>
void run_chain(const NsTable& t, const NsScalars& sc, const NsFinish& fin, const NsProducts& p,
               const double* sums, bool fold, float* part, hipStream_t s) {
  const int tiles = t.tile0[t.count];
  if (fold) ns_init_kernel<MODE, PLANES, true><<<tiles, kThreads, 0, s>>>(t, sc, sums);
  else ns_init_kernel<MODE, PLANES, false><<<tiles, kThreads, 0, s>>>(t, sc, sums);
  launch_ns_products(t, fin, PLANES, sc.steps, p, part, s);
  if (p.apply.big)
    ns_finish_kernel<PLANES><<<tiles, kThreads, 0, s>>>(t, fin, ns_groups(p, sc.steps) & 1);
}

template <NsMode MODE>
void run(const NsTable& t, const NsScalars& sc, Dt copy_dt, const NsChains& c, double* partial,
         double* norm, float* part, hipStream_t s) {
  ns_update_kernel<MODE><<<t.tile0[t.count], kThreads, 0, s>>>(t, sc, partial);
  bool fold = true;
  for (int i = 0; i < t.count; ++i) fold = fold && t.tile0[i + 1] - t.tile0[i] <= kThreads;
  if (!fold) ns_norm_kernel<<<t.count, kNormThreads, 0, s>>>(t, sc.eps, partial, norm);
  const bool bf16_out = MODE == NsMode::Bf16 || (MODE == NsMode::Muon && copy_dt == Dt::BF16);
  const NsFinish fin{MODE, bf16_out, sc.lr};
  for (int k = 0, lo = 0; k < c.count; lo = c.end[k++]) {
    const NsTable u = ns_slice(t, lo, c.end[k]);
    const double* sums = fold ? partial + t.tile0[lo] : norm + lo;
    if (c.planes[k] == 2) run_chain<MODE, 2>(u, sc, fin, c.p[k], sums, fold, part, s);
    else if constexpr (MODE == NsMode::Muon)
      run_chain<MODE, 1>(u, sc, fin, c.p[k], sums, fold, part, s);
  }
}

}  // namespace

void launch_newton_schulz(const NsTable& t, const NsScalars& sc, NsMode mode, Dt copy_dt,
                          const NsChains& c, double* partial, double* norm, float* part,
                          hipStream_t s) {
  switch (mode) {
    case NsMode::Muon: run<NsMode::Muon>(t, sc, copy_dt, c, partial, norm, part, s); break;
    case NsMode::Bf16: run<NsMode::Bf16>(t, sc, copy_dt, c, partial, norm, part, s); break;
    case NsMode::F32: run<NsMode::F32>(t, sc, copy_dt, c, partial, norm, part, s); break;
  }
}

}  // namespace pb

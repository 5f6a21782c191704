// fp16 planes of the Newton-Schulz iterates, shared by the passes (muon.hip) and
// the products (ns_gemm.hip).
#pragma once

#include "common.h"
#include "kernels.h"

namespace pb {

// A plane value is the number times a power of two, rounded to fp16; with two planes the
// second one holds the remainder, rounded again (2^-22 of the number).  The powers keep
// the values high in fp16's range, so that what the remainder loses to subnormals is
// below 2^-36 of the largest spectral norm: no element of a matrix exceeds its norm, and
// with s the singular values of X, in [0, 1.203],
//   X (1.203) and A = X X^T (1.446) times 2^15 stay below 39.4e3 and 47.4e3,
//   B = a + b s^2 + c s^4, in [0.638, 3.445], times 2^14 below 56.4e3,
//   B A (p(s) s: 1.446) times 2^15 below 47.4e3,
//   Q = B' B, of two steps (11.87), times 2^12 below 48.6e3
// of fp16's 65.5e3.
constexpr float kNsScaleX = 32768.0f, kNsScaleA = 32768.0f, kNsScaleB = 16384.0f,
                kNsScaleQ = 4096.0f;
// Coefficients of the step (Jordan et al. 2024).
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Address of element (row, col) of a matrix with rows of ld: one plane is row-major;
// with two, 32 values and their 32 remainders alternate along a row, so that 128 bytes
// of a row hold both of 32 elements.  The remainder lies kNsRest after the value.
constexpr int kNsRest = 32;
template <int PLANES>
PB_DEV size_t ns_at(int ld, int row, int col) {
  if constexpr (PLANES == 1) return (size_t)row * ld + col;
  else return (size_t)row * (2 * ld) + (col >> 5) * 64 + (col & 31);
}
// N (4 or 8) consecutive values from p on, times scale.
template <int PLANES, int N>
PB_DEV void ns_store(_Float16* p, const float* v, float scale) {
  typedef _Float16 vec __attribute__((ext_vector_type(N)));
  vec hi, lo;
#pragma unroll
  for (int e = 0; e < N; ++e) {
    const float x = v[e] * scale;
    hi[e] = (_Float16)x;
    lo[e] = (_Float16)(x - (float)hi[e]);
  }
  *reinterpret_cast<vec*>(p) = hi;
  if constexpr (PLANES == 2) *reinterpret_cast<vec*>(p + kNsRest) = lo;
}
template <int PLANES, int N>
PB_DEV void ns_load(const _Float16* p, float* v, float scale) {
  typedef _Float16 vec __attribute__((ext_vector_type(N)));
  const vec hi = *reinterpret_cast<const vec*>(p);
  vec lo = {};
  if constexpr (PLANES == 2) lo = *reinterpret_cast<const vec*>(p + kNsRest);
#pragma unroll
  for (int e = 0; e < N; ++e) v[e] = ((float)hi[e] + (float)lo[e]) * scale;
}

// What becomes of the last X: the weights' step (Muon; bf16_out: the type of the
// copies), or the matrix itself in its type.
struct NsFinish {
  NsMode mode;
  bool bf16_out;
  float lr;
};
// N elements of row r of a tensor from column c on, X's values there: the weights'
// step and their copy, or the orthogonalised matrix.  Past the row's end, nothing.
template <int N, typename T>
PB_DEV void put(T* p, int left, const float* v) {
  if (left >= N && (uintptr_t)p % (N * sizeof(T) < 16 ? N * sizeof(T) : 16) == 0) {
#pragma unroll
    for (int e = 0; e < N; e += 4) store4<T>(p + e, v + e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (e < left) p[e] = (T)v[e];
  }
}
// The weights there before the step (Muon; else nothing).
template <int N>
PB_DEV void weights(const NsMat& x, const NsFinish& f, int r, int c, float* u) {
  const int left = x.cols - c;
  if (f.mode != NsMode::Muon || r >= x.rows || left <= 0) return;
  const float* w = x.w + r * x.ld_src + c;
  if (left >= N && (uintptr_t)w % 16 == 0) {
#pragma unroll
    for (int e = 0; e < N; e += 4) load4<float>(w + e, u + e);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = e < left ? w[e] : 0.f;
  }
}
// u: those weights, stepped in place.
template <int N>
PB_DEV void finish(const NsMat& x, const NsFinish& f, int r, int c, const float* v, float* u) {
  const int left = x.cols - c;
  if (r >= x.rows || left <= 0) return;
  if (f.mode == NsMode::Muon) {
    const float keep = 1.0f - f.lr * x.decay, step = f.lr * x.scale;
#pragma unroll
    for (int e = 0; e < N; ++e) u[e] = __builtin_fmaf(-step, v[e], u[e] * keep);
    put<N>(x.w + r * x.ld_src + c, left, u);
    if (x.copy) {
      if (f.bf16_out) put<N>((bf16*)x.copy + r * x.ld_src + c, left, u);
      else put<N>((float*)x.copy + r * x.ld_src + c, left, u);
    }
  } else if (f.bf16_out) {
    put<N>((bf16*)x.out + r * x.ld_out + c, left, v);
  } else {
    put<N>((float*)x.out + r * x.ld_out + c, left, v);
  }
}
// `steps` Newton-Schulz steps of every matrix from x[0] on.  Where apply runs in small
// tiles the last product finishes the tensors; else X is in x[ns_groups() & 1].
void launch_ns_products(const NsTable& t, const NsFinish& fin, int planes, int steps,
                        const NsProducts& p, float* part, hipStream_t s);

}  // namespace pb

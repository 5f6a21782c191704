// fp16 planes of the Newton-Schulz iterates, shared by the passes (muon.hip) and
// the products (ns_gemm.hip).
#pragma once

#include "common.h"
#include "kernels.h"

namespace pb {

// A plane value is the number times a power of two, rounded to fp16; with two
// planes the second one holds the remainder, rounded again (2^-22 of the number).
// The powers keep the values high in fp16's range, so that what the remainder
// loses to subnormals is below 2^-39 of the spectral norm: X has a spectral norm
// of at most 1.203, A = X X^T of 1.446 and B of 3.445 (a + b s + c s^2 over s in
// [0, 1.446] lies in [0.638, 3.445]), and no element of a matrix exceeds its norm:
// 39.4e3, 47.4e3 and 56.4e3 of fp16's 65.5e3.
constexpr float kNsScaleX = 32768.0f, kNsScaleA = 32768.0f, kNsScaleB = 16384.0f;
// Coefficients of the step (Jordan et al. 2024).
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));

// Eight consecutive values to the planes `plane` elements apart, times scale.
template <int PLANES>
PB_DEV void ns_store8(_Float16* p, size_t plane, const float* v, float scale) {
  f16x8 hi, lo;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = v[e] * scale;
    hi[e] = (_Float16)x;
    lo[e] = (_Float16)(x - (float)hi[e]);
  }
  *reinterpret_cast<f16x8*>(p) = hi;
  if constexpr (PLANES == 2) *reinterpret_cast<f16x8*>(p + plane) = lo;
}
template <int PLANES>
PB_DEV void ns_store4(_Float16* p, size_t plane, const float* v, float scale) {
  f16x4 hi, lo;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float x = v[e] * scale;
    hi[e] = (_Float16)x;
    lo[e] = (_Float16)(x - (float)hi[e]);
  }
  *reinterpret_cast<f16x4*>(p) = hi;
  if constexpr (PLANES == 2) *reinterpret_cast<f16x4*>(p + plane) = lo;
}
template <int PLANES>
PB_DEV void ns_load8(const _Float16* p, size_t plane, float* v, float scale) {
  const f16x8 hi = *reinterpret_cast<const f16x8*>(p);
  f16x8 lo = {};
  if constexpr (PLANES == 2) lo = *reinterpret_cast<const f16x8*>(p + plane);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = ((float)hi[e] + (float)lo[e]) * scale;
}
template <int PLANES>
PB_DEV void ns_load4(const _Float16* p, size_t plane, float* v, float scale) {
  const f16x4 hi = *reinterpret_cast<const f16x4*>(p);
  f16x4 lo = {};
  if constexpr (PLANES == 2) lo = *reinterpret_cast<const f16x4*>(p + plane);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = ((float)hi[e] + (float)lo[e]) * scale;
}

// One Newton-Schulz step of every matrix: x[cur] -> x[cur ^ 1].
void launch_ns_step(const NsTable& t, int planes, int cur, hipStream_t s);

}  // namespace pb

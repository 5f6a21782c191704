// Root-mean-square norm with the residual's addition, and its gradient.
//
//   forward:  s = x + resid,  r = 1 / sqrt(mean(s^2) + eps),  y = s r gamma
//             and, for an output in 8 bits, c = max |y| / 448 over each group of
//             columns and q = e4m3(y / c)
//   backward: g = dy gamma,  k = mean(g s) r^2,  dx = dsum + r (g - s k),
//             dgamma = sum over rows of dy s r
//
// HBM-bound, one pass each: a row stays in the registers of the TPR threads that
// share it (NC pieces of 8 columns a thread), so it is read once.  Narrow rows
// share a workgroup.  s is stored rounded to the activation type, while y is
// formed from the unrounded sum; the backward takes the stored s and the
// forward's r.
//
// The 8-bit output is computed in fp64 up to its codes: a value next to the
// border between two codes then falls on the side that its definition says,
// whatever the order of the row's sum (in fp32 about one code in 10^6 goes to the
// neighbour, 6 to 12% off).  The arithmetic stays below the memory time.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace pb {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr double kScaleMin = 0x1p-126;  // smallest scale: a group of zeros has this one

// Eight columns from column c of a row of H, elementwise past 16-byte alignment or
// the row's end (those columns read as zero).
template <typename T, bool AL>
PB_DEV void load_cols(const T* row, int c, int H, float* v) {
  if constexpr (AL) {
    load8<T>(row + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < H ? load1<T>(row + c + e) : 0.f;
  }
}
template <typename T, bool AL>
PB_DEV void store_cols(T* row, int c, int H, const float* v) {
  if constexpr (AL) {
    store8<T>(row + c, v);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < H) row[c + e] = (T)v[e];
  }
}

// Sum (or maximum) over the TPR threads that share a row; every one receives it.
// red: one value per wave, used where a row spans waves.
template <int TPR, typename R, typename Op>
PB_DEV R row_reduce(R v, R* red, Op op) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o >= 1; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
  if constexpr (TPR > 64) {
    const int wave = threadIdx.x >> 6;
    __syncthreads();  // red may still be read from an earlier reduction
    if ((threadIdx.x & 63) == 0) red[wave] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int i = 1; i < TPR / 64; ++i) v = op(v, red[i]);
  }
  return v;
}

template <typename T, int TPR, int NC, bool AL, bool Q8>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_fwd_kernel(RmsForward a) {
  using R = typename std::conditional<Q8, double, float>::type;
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
  __shared__ R red[kThreads / 64];
  const int H = a.cols, l = threadIdx.x % TPR;
  for (long long r0 = (long long)blockIdx.x * kRows; r0 < a.rows;
       r0 += (long long)gridDim.x * kRows) {
    // (a row past the end, where rows share a workgroup, is zeros and stores nothing:
    // the lanes of a wave stay together)
    const long long row = r0 + threadIdx.x / TPR;
    const bool live = row < a.rows;
    const long long rc = live ? row : a.rows - 1;
    const T* x = (const T*)a.x + rc * H;
    const T* res = a.resid ? (const T*)a.resid + rc * H : nullptr;
    const T* gamma = (const T*)a.gamma;
    R s[NC][8];
    float xv[NC][8], rv[NC][8];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
#pragma unroll
      for (int e = 0; e < 8; ++e) xv[j][e] = rv[j][e] = 0.f;
      if (c < H && live) {
        load_cols<T, AL>(x, c, H, xv[j]);
        if (res) load_cols<T, AL>(res, c, H, rv[j]);
      }
    }
    R ss = 0;
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[j][e] = (R)xv[j][e] + (R)rv[j][e];
        ss += s[j][e] * s[j][e];
      }
    if (a.sum && live)
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = 8 * (l + j * TPR);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (float)s[j][e];
        if (c < H) store_cols<T, AL>((T*)a.sum + rc * H, c, H, o);
      }
    ss = row_reduce<TPR>(ss, red, [](R p, R q) { return p + q; });
    R r;
    if constexpr (Q8) r = 1.0 / sqrt(ss / H + (double)a.eps);
    else r = 1.0f / sqrtf(ss / H + a.eps);
    if (a.rstd && live && l == 0) a.rstd[row] = (float)r;

    R most = 0;  // max |y| of the row
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
      float g[8], o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) g[e] = 0.f;
      if (c < H) load_cols<T, AL>(gamma, c, H, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        s[j][e] = s[j][e] * r * (R)g[e];
        o[e] = (float)s[j][e];
      }
      if (a.y && live && c < H) store_cols<T, AL>((T*)a.y + rc * H, c, H, o);
      if constexpr (Q8)
#pragma unroll
        for (int e = 0; e < 8; ++e) most = fmax(most, fabs(s[j][e]));
    }
    if constexpr (Q8) {
      const int G = a.group;
      const int groups = G ? (H + G - 1) / G : 1;
      if (!G) most = row_reduce<TPR>(most, red, [](R p, R q) { return fmax(p, q); });
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = 8 * (l + j * TPR);
        R m = most;
        if (G) {  // the G / 8 neighbouring lanes of a group
          m = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) m = fmax(m, fabs(s[j][e]));
          for (int o = G / 16; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
        }
        // the scale as it is kept, in fp32
        const float scale = (float)fmax(m * (1.0 / kE4m3Max), kScaleMin);
        const double inv = 1.0 / (double)scale;
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int p = __builtin_amdgcn_cvt_pk_fp8_f32((float)(s[j][4 * h] * inv),
                                                  (float)(s[j][4 * h + 1] * inv), 0, false);
          p = __builtin_amdgcn_cvt_pk_fp8_f32((float)(s[j][4 * h + 2] * inv),
                                              (float)(s[j][4 * h + 3] * inv), p, true);
          w[h] = (uint32_t)p;
        }
        if (live && c < H) {
          uint8_t* q = a.q8 + rc * H + c;
          if constexpr (AL) {
            *reinterpret_cast<u32x2*>(q) = u32x2{w[0], w[1]};
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (c + e < H) q[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
          }
          if (G ? c % G == 0 : c == 0) a.scales[rc * groups + (G ? c / G : 0)] = scale;
        }
      }
    }
  }
}

// A workgroup takes every gridDim.x-th set of kRows rows and keeps its part of
// dgamma in registers; the rows that share the workgroup add theirs up in LDS, in
// turn, and the workgroup's sums go to part[workgroup][H].
template <typename T, int TPR, int NC, bool AL>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_bwd_kernel(RmsBackward a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
  __shared__ float red[kThreads / 64];
  __shared__ float fold[kRows > 1 ? TPR * NC * 8 : 1];
  const int H = a.cols, l = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  const T* gamma = (const T*)a.gamma;
  float acc[NC][8];
#pragma unroll
  for (int j = 0; j < NC; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[j][e] = 0.f;
  for (long long r0 = (long long)blockIdx.x * kRows; r0 < a.rows;
       r0 += (long long)gridDim.x * kRows) {
    const long long row = r0 + sub;
    const bool live = row < a.rows;
    const long long at = (live ? row : a.rows - 1) * H;
    float s[NC][8], dy[NC][8], g[NC][8];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[j][e] = dy[j][e] = g[j][e] = 0.f;
      if (c < H && live) {
        load_cols<T, AL>((const T*)a.s + at, c, H, s[j]);
        load_cols<T, AL>((const T*)a.dy + at, c, H, dy[j]);
        load_cols<T, AL>(gamma, c, H, g[j]);
      }
    }
    const float r = a.rstd[live ? row : a.rows - 1];
    float k = 0.f;
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        g[j][e] *= dy[j][e];
        s[j][e] *= r;
        k += g[j][e] * s[j][e];
        if (live) acc[j][e] += dy[j][e] * s[j][e];
      }
    k = row_reduce<TPR>(k, red, [](float p, float q) { return p + q; }) / H;
    if (live)
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = 8 * (l + j * TPR);
        if (c < H) {
          float o[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = 0.f;
          if (a.dsum) load_cols<T, AL>((const T*)a.dsum + at, c, H, o);
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] += r * (g[j][e] - s[j][e] * k);
          store_cols<T, AL>((T*)a.dx + at, c, H, o);
        }
      }
  }
  if constexpr (kRows > 1) {
    for (int t = 0; t < kRows; ++t) {
      if (sub == t)
#pragma unroll
        for (int j = 0; j < NC; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float* f = fold + 8 * (l + j * TPR) + e;
            *f = t ? *f + acc[j][e] : acc[j][e];
          }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < H; c += kThreads) a.part[(size_t)blockIdx.x * H + c] = fold[c];
  } else {
#pragma unroll
    for (int j = 0; j < NC; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int c = 8 * (l + j * TPR) + e;
        if (c < H) a.part[(size_t)blockIdx.x * H + c] = acc[j][e];
      }
  }
}

// dgamma[c] = sum over n rows of part, 16 threads a column (n = 0: zeros).
__global__ __launch_bounds__(256) void rms_fold_kernel(const float* __restrict__ part, int n, int H,
                                                       float* __restrict__ dgamma) {
  __shared__ float red[16][17];
  const int cl = threadIdx.x & 15, rl = threadIdx.x >> 4, c = blockIdx.x * 16 + cl;
  float v = 0.f;
  if (c < H)
    for (int i = rl; i < n; i += 16) v += part[(size_t)i * H + c];
  red[rl][cl] = v;
  __syncthreads();
  if (rl == 0 && c < H) {
#pragma unroll
    for (int i = 1; i < 16; ++i) v += red[i][cl];
    dgamma[c] = v;
  }
}

// Threads a row and pieces of 8 columns a thread: rows of up to 128 columns take
// 16 threads, up to 1024 a wave, then the fewest of 256, 512 and 1024 that hold the
// row in four pieces.
template <typename F>
void by_width(int H, F f) {
  const int pieces = (H + 7) / 8;
  auto c = [](auto v) { return v; };
  using std::integral_constant;
  if (pieces <= 16) f(integral_constant<int, 16>{}, integral_constant<int, 1>{});
  else if (pieces <= 64) f(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  else if (pieces <= 128) f(integral_constant<int, 64>{}, integral_constant<int, 2>{});
  else if (pieces <= 256) f(integral_constant<int, 256>{}, integral_constant<int, 1>{});
  else if (pieces <= 512) f(integral_constant<int, 256>{}, integral_constant<int, 2>{});
  else if (pieces <= 768) f(integral_constant<int, 256>{}, integral_constant<int, 3>{});
  else if (pieces <= 1024) f(integral_constant<int, 256>{}, integral_constant<int, 4>{});
  else if (pieces <= 1536) f(integral_constant<int, 512>{}, integral_constant<int, 3>{});
  else if (pieces <= 2048) f(integral_constant<int, 512>{}, integral_constant<int, 4>{});
  else if (pieces <= 3072) f(integral_constant<int, 1024>{}, integral_constant<int, 3>{});
  else f(integral_constant<int, 1024>{}, integral_constant<int, 4>{});
}

bool aligned16(const void* p) { return (uintptr_t)p % 16 == 0; }

template <typename T>
void forward(const RmsForward& a, hipStream_t s) {
  const bool al = a.cols % 8 == 0 && aligned16(a.x) && aligned16(a.resid) && aligned16(a.gamma) &&
                  aligned16(a.sum) && aligned16(a.y) && (uintptr_t)a.q8 % 8 == 0;
  by_width(a.cols, [&](auto tpr, auto nc) {
    constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
    constexpr int threads = TPR < 256 ? 256 : TPR, rows = threads / TPR;
    // (a launch has fewer than 2^32 threads)
    const unsigned grid = (unsigned)std::min<long long>((a.rows + rows - 1) / rows, 1 << 20);
    if (a.q8) {
      if (al) rms_fwd_kernel<T, TPR, NC, true, true><<<grid, threads, 0, s>>>(a);
      else rms_fwd_kernel<T, TPR, NC, false, true><<<grid, threads, 0, s>>>(a);
    } else {
      if (al) rms_fwd_kernel<T, TPR, NC, true, false><<<grid, threads, 0, s>>>(a);
      else rms_fwd_kernel<T, TPR, NC, false, false><<<grid, threads, 0, s>>>(a);
    }
  });
}

template <typename T>
void backward(const RmsBackward& a, hipStream_t s) {
  const bool al = a.cols % 8 == 0 && aligned16(a.s) && aligned16(a.gamma) && aligned16(a.dy) &&
                  aligned16(a.dsum) && aligned16(a.dx);
  const int n = rms_backward_parts(a.rows, a.cols);
  if (n > 0)
    by_width(a.cols, [&](auto tpr, auto nc) {
      constexpr int TPR = decltype(tpr)::value, NC = decltype(nc)::value;
      constexpr int threads = TPR < 256 ? 256 : TPR;
      if (al) rms_bwd_kernel<T, TPR, NC, true><<<n, threads, 0, s>>>(a);
      else rms_bwd_kernel<T, TPR, NC, false><<<n, threads, 0, s>>>(a);
    });
  rms_fold_kernel<<<(a.cols + 15) / 16, 256, 0, s>>>(a.part, n, a.cols, a.dgamma);
}

}  // namespace

int rms_backward_parts(long long rows, int cols) {
  long long n = 0;
  by_width(cols, [&](auto tpr, auto) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int per = TPR < 256 ? 256 / TPR : 1;
    n = std::min<long long>((rows + per - 1) / per, 512);
  });
  return (int)n;
}

void launch_rms_forward(Dt dt, const RmsForward& a, hipStream_t s) {
  if (dt == Dt::BF16) forward<bf16>(a, s);
  else forward<float>(a, s);
}

void launch_rms_backward(Dt dt, const RmsBackward& a, hipStream_t s) {
  if (dt == Dt::BF16) backward<bf16>(a, s);
  else backward<float>(a, s);
}

}  // namespace pb

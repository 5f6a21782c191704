// Root-mean-square norm with the residual's addition, and its gradient.
//
//   forward:  s = x + resid,  r = 1 / sqrt(mean(s^2) + eps),  y = s r gamma
//             and, for an output in 8 bits, c = max |y| / 448 over each group of
//             columns and q = e4m3(y / c)
//   backward: g = dy gamma,  k = mean(g s) r^2,  dx = dsum + r (g - s k),
//             dgamma = sum over rows of dy s r
//
// HBM-bound, one pass each (bf16, 8192 x 5120: forward 60 us and 5.6 TB/s, backward 61 and
// 5.5 with 5 more for dgamma; 2048 x 12288 in 8 bits 42 us): a row stays in the registers
// of the TPR threads that share it (NC pieces of 8 columns a thread), so it is read once.
// Narrow rows share a workgroup.  s is stored rounded to the activation type, while y is
// formed from the unrounded sum; the backward takes the stored s and the forward's r.
//
// The sum of squares is formed in fp64: in fp32 it overflows from elements of 1e19 on and
// vanishes below 1e-23 (8192 x 5120: 60.1 us in fp32, 60.6 so).
//
// The 8-bit output is computed in fp64 up to the quotient y / c, which is rounded to fp32
// and that to e4m3, as a cast of it is: a value next to the border between two codes then
// falls on the side that this definition says, whatever the order of the row's sum (in
// fp32 about one code in 10^6 goes to the neighbour, 6 to 12% off).  2048 x 12288 take 42
// us so and 35 in fp32.  (Rounded once, fp64 to e4m3, some 10 of those 25 million codes,
// within half an fp32 step of the middle of two, would be others.)
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace pb {
namespace {

constexpr float kE4m3Max = 448.0f;
constexpr double kScaleMin = 0x1p-126;  // smallest scale: a group of zeros has this one

// Eight elements as they lie in memory, 16 bytes to a load.  AL: 16-byte aligned; the
// hardware takes any alignment of the element, which rows of an odd width have.
template <typename T>
struct Piece {
  static constexpr int kWords = sizeof(T) / 2;  // 16-byte words
  u32x4 w[kWords];
  PB_DEV float at(int e) const {
    if constexpr (sizeof(T) == 2) return e & 1 ? hi_bf(w[0][e >> 1]) : lo_bf(w[0][e >> 1]);
    else return __uint_as_float(w[e >> 2][e & 3]);
  }
};
// Columns c .. c + 7 of a row of H (past the row's end zeros, where not AL).
template <typename T, bool AL>
PB_DEV Piece<T> load_piece(const T* row, int c, int H) {
  Piece<T> p;
  if (AL || c + 8 <= H) {
#pragma unroll
    for (int k = 0; k < Piece<T>::kWords; ++k) {
      const T* at = row + c + 8 / Piece<T>::kWords * k;
      if constexpr (AL) p.w[k] = *reinterpret_cast<const u32x4*>(at);
      else __builtin_memcpy(&p.w[k], at, 16);
    }
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = c + e < H ? load1<T>(row + c + e) : 0.f;
#pragma unroll
    for (int k = 0; k < 4 * Piece<T>::kWords; ++k)
      p.w[k >> 2][k & 3] = sizeof(T) == 2 ? pack_bf2(v[2 * k], v[2 * k + 1]) : __float_as_uint(v[k]);
  }
  return p;
}
template <typename T>
PB_DEV Piece<T> zero_piece() {
  Piece<T> p;
#pragma unroll
  for (int k = 0; k < Piece<T>::kWords; ++k) p.w[k] = u32x4{0, 0, 0, 0};
  return p;
}
// (Past the caches' retention, where aligned: 62 -> 60 us for the forward of 8192 x 5120,
// 41 -> 36 of 2048 x 12288.)
template <typename T, bool AL>
PB_DEV void store_cols(T* row, int c, int H, const float* v) {
  if (AL || c + 8 <= H) {
#pragma unroll
    for (int k = 0; k < Piece<T>::kWords; ++k) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] = sizeof(T) == 2 ? pack_bf2(v[2 * e], v[2 * e + 1]) : __float_as_uint(v[4 * k + e]);
      T* at = row + c + 8 / Piece<T>::kWords * k;
      if constexpr (AL) __builtin_nontemporal_store(w, reinterpret_cast<u32x4*>(at));
      else __builtin_memcpy(at, &w, 16);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (c + e < H) row[c + e] = (T)v[e];
  }
}

// Sum (or maximum) over the TPR threads that share a row; every one receives it.
// red: a value per wave, where a row spans waves: its two halves are used in turn
// (`turn`), so that one barrier a reduction is enough.
template <int TPR, typename R, typename Op>
PB_DEV R row_reduce(R v, R* red, int& turn, Op op) {
#pragma unroll
  for (int o = (TPR < 64 ? TPR : 64) / 2; o >= 1; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
  if constexpr (TPR > 64) {
    constexpr int kWaves = TPR / 64;
    R* at = red + turn * kWaves;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
    __syncthreads();
    v = at[0];
#pragma unroll
    for (int i = 1; i < kWaves; ++i) v = op(v, at[i]);
  }
  return v;
}

template <typename T, int TPR, int NC, bool AL, bool Q8>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_fwd_kernel(RmsForward a) {
  using R = typename std::conditional<Q8, double, float>::type;
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
  __shared__ double red[2 * (kThreads / 64)];
  const int H = a.cols, l = threadIdx.x % TPR;
  int turn = 0;
  for (long long r0 = (long long)blockIdx.x * kRows; r0 < a.rows;
       r0 += (long long)gridDim.x * kRows) {
    // (a row past the end, where rows share a workgroup, is zeros and stores nothing:
    // the lanes of a wave stay together)
    const long long row = r0 + threadIdx.x / TPR;
    const bool live = row < a.rows;
    const long long at = (live ? row : a.rows - 1) * H;
    // the row as it lies in memory: in fp64 its sums would take four times the registers
    Piece<T> xp[NC], rp[NC];
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
      xp[j] = rp[j] = zero_piece<T>();
      if (c < H && live) {
        xp[j] = load_piece<T, AL>((const T*)a.x + at, c, H);
        if (a.resid) rp[j] = load_piece<T, AL>((const T*)a.resid + at, c, H);
      }
    }
    auto sum = [&](int j, int e) { return (R)xp[j].at(e) + (R)rp[j].at(e); };
    double ss = 0;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
      float o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const R s = sum(j, e);
        o[e] = (float)s;
        ss += (double)s * (double)s;
      }
      if (a.sum && live && c < H) store_cols<T, AL>((T*)a.sum + at, c, H, o);
    }
    ss = row_reduce<TPR>(ss, red, turn, [](double p, double q) { return p + q; });
    const R r = (R)(1.0 / sqrt(ss / H + (double)a.eps));
    if (a.rstd && live && l == 0) a.rstd[row] = (float)r;

    // columns c .. of y
    auto values = [&](int j, int c, R (&y)[8]) {
      Piece<T> g = zero_piece<T>();
      if (c < H) g = load_piece<T, AL>((const T*)a.gamma, c, H);
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = sum(j, e) * r * (R)g.at(e);
    };
    auto largest = [](const R (&y)[8]) {
      R m = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) m = fmax(m, fabs(y[e]));
      return m;
    };
    R most = 0;  // max |y| of the row, where it has one scale
    if constexpr (Q8) {
      if (!a.group) {
#pragma unroll
        for (int j = 0; j < NC; ++j) {
          R y[8];
          values(j, 8 * (l + j * TPR), y);
          most = fmax(most, largest(y));
        }
        most = row_reduce<TPR>(most, red, turn, [](R p, R q) { return fmax(p, q); });
      }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);
      R y[8];
      values(j, c, y);
      if (a.y && live && c < H) {
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = (float)y[e];
        store_cols<T, AL>((T*)a.y + at, c, H, o);
      }
      if constexpr (Q8) {
        const int G = a.group, groups = G ? (H + G - 1) / G : 1;
        R m = most;
        if (G) {  // the G / 8 neighbouring lanes of a group
          m = largest(y);
          for (int o = G / 16; o >= 1; o >>= 1) m = fmax(m, __shfl_xor(m, o, 64));
        }
        // the scale as it is kept, in fp32
        const float scale = (float)fmax(m * (1.0 / kE4m3Max), kScaleMin);
        const double inv = 1.0 / (double)scale;
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          int p = __builtin_amdgcn_cvt_pk_fp8_f32((float)(y[4 * h] * inv),
                                                  (float)(y[4 * h + 1] * inv), 0, false);
          p = __builtin_amdgcn_cvt_pk_fp8_f32((float)(y[4 * h + 2] * inv),
                                              (float)(y[4 * h + 3] * inv), p, true);
          w[h] = (uint32_t)p;
        }
        if (live && c < H) {
          uint8_t* q = a.q8 + at + c;
          if (AL || c + 8 <= H) {
            if constexpr (AL) __builtin_nontemporal_store(u32x2{w[0], w[1]}, reinterpret_cast<u32x2*>(q));
            else __builtin_memcpy(q, w, 8);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (c + e < H) q[e] = (uint8_t)(w[e >> 2] >> (8 * (e & 3)));
          }
          if (G ? c % G == 0 : c == 0)
            a.scales[(live ? row : 0) * groups + (G ? c / G : 0)] = scale;
        }
      }
    }
  }
}

// A workgroup takes every gridDim.x-th set of kRows rows and keeps its part of dgamma
// (and gamma) in registers.
// The rows that share a workgroup add theirs up in LDS, in turn; the workgroup's sums
// go to part[workgroup][rms_part_ld(H)].
template <typename T, int TPR, int NC, bool AL>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void rms_bwd_kernel(RmsBackward a) {
  constexpr int kThreads = TPR < 256 ? 256 : TPR, kRows = kThreads / TPR;
  // The widest rows do not fit into registers beside their sums: their second pass over
  // the row reads it again, from the caches.
  constexpr bool kKeep = TPR <= 512;
  __shared__ float red[2 * (kThreads / 64)];
  __shared__ float fold[kRows > 1 ? TPR * NC * 8 : 1];
  const int H = a.cols, l = threadIdx.x % TPR, sub = threadIdx.x / TPR;
  int turn = 0;
  float acc[NC][8];
  constexpr int kN = kKeep ? NC : 1;
  Piece<T> gp[kN];
#pragma unroll
  for (int j = 0; j < NC; ++j) {
    const int c = 8 * (l + j * TPR);
    if constexpr (kKeep) {
      gp[j] = zero_piece<T>();
      if (c < H) gp[j] = load_piece<T, AL>((const T*)a.gamma, c, H);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[j][e] = 0.f;
  }
  float* part = a.part + (size_t)blockIdx.x * rms_part_ld(H);
  if constexpr (!kKeep) {  // (a row a workgroup)
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
      const float r = a.rstd[row];
      const T* sp = (const T*)a.s + row * H;
      const T* dyp = (const T*)a.dy + row * H;
      float k = 0.f;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = 8 * (l + j * TPR);
        if (c >= H) continue;
        const Piece<T> s = load_piece<T, AL>(sp, c, H), dy = load_piece<T, AL>(dyp, c, H),
                       g = load_piece<T, AL>((const T*)a.gamma, c, H);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float u = dy.at(e) * (s.at(e) * r);
          k += g.at(e) * u;
          acc[j][e] += u;
        }
      }
      k = row_reduce<TPR>(k, red, turn, [](float p, float q) { return p + q; }) / H;
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        const int c = 8 * (l + j * TPR);
        if (c >= H) continue;
        const Piece<T> s = load_piece<T, AL>(sp, c, H), dy = load_piece<T, AL>(dyp, c, H),
                       g = load_piece<T, AL>((const T*)a.gamma, c, H);
        Piece<T> ds = zero_piece<T>();
        if (a.dsum) ds = load_piece<T, AL>((const T*)a.dsum + row * H, c, H);
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = ds.at(e) + r * (dy.at(e) * g.at(e) - s.at(e) * r * k);
        store_cols<T, AL>((T*)a.dx + row * H, c, H, o);
      }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int c = 8 * (l + j * TPR);  // (part's rows are padded to whole pieces)
      if (c < H) store8<float>(part + c, acc[j]);
    }
    return;
  }
  for (long long r0 = (long long)blockIdx.x * kRows; r0 < a.rows;
       r0 += (long long)gridDim.x * kRows) {
    const bool live = r0 + sub < a.rows;
    const long long row = live ? r0 + sub : a.rows - 1, at = row * H;
    Piece<T> s[kN], dy[kN], ds[kN];
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int c = 8 * (l + j * TPR);
      s[j] = dy[j] = ds[j] = zero_piece<T>();
      if (c < H && live) {
        s[j] = load_piece<T, AL>((const T*)a.s + at, c, H);
        dy[j] = load_piece<T, AL>((const T*)a.dy + at, c, H);
        if (a.dsum) ds[j] = load_piece<T, AL>((const T*)a.dsum + at, c, H);
      }
    }
    const float r = a.rstd[row];
    float k = 0.f;
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float u = dy[j].at(e) * (live ? s[j].at(e) * r : 0.f);
        k += gp[j].at(e) * u;
        acc[j][e] += u;
      }
    k = row_reduce<TPR>(k, red, turn, [](float p, float q) { return p + q; }) / H;
    if (live)
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        const int c = 8 * (l + j * TPR);
        if (c >= H) continue;
        float o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = ds[j].at(e) + r * (dy[j].at(e) * gp[j].at(e) - s[j].at(e) * r * k);
        store_cols<T, AL>((T*)a.dx + at, c, H, o);
      }
  }
  if constexpr (kRows > 1) {
    for (int t = 0; t < kRows; ++t) {
      if (sub == t)
#pragma unroll
        for (int j = 0; j < kN; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float* f = fold + 8 * (l + j * TPR) + e;
            *f = t ? *f + acc[j][e] : acc[j][e];
          }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < H; c += kThreads) part[c] = fold[c];
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      const int c = 8 * (l + j * TPR);  // (part's rows are padded to whole pieces)
      if (c < H) store8<float>(part + c, acc[j]);
    }
  }
}

// dgamma[c] = sum over n rows of part: a thread four columns of every 64th row, then the
// 64 threads of a column in LDS (n = 0: zeros).
constexpr int kFoldThreads = 1024;
__global__ __launch_bounds__(kFoldThreads) void rms_fold_kernel(const float* __restrict__ part,
                                                                int n, int H,
                                                                float* __restrict__ dgamma) {
  __shared__ float red[64][64 + 4];
  const int cl = 4 * (threadIdx.x & 15), rl = threadIdx.x >> 4, c = blockIdx.x * 64 + cl;
  const size_t ld = rms_part_ld(H);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  if (c < H)
#pragma unroll 8
    for (int i = rl; i < n; i += 64) v += *reinterpret_cast<const f32x4*>(part + i * ld + c);
  *reinterpret_cast<f32x4*>(&red[rl][cl]) = v;
  __syncthreads();
  // 16 neighbouring lanes sum a column, four rows each
  const int col = threadIdx.x >> 4, q = threadIdx.x & 15;
  float s = (red[4 * q][col] + red[4 * q + 1][col]) + (red[4 * q + 2][col] + red[4 * q + 3][col]);
  s = row16_sum(s);
  if (q == 0 && blockIdx.x * 64 + col < H) dgamma[blockIdx.x * 64 + col] = s;
}

// Threads a row and pieces of 8 columns a thread: rows of up to 128 columns take
// 16 threads, up to 1024 a wave, then the fewest of 256, 512 and 1024 that hold the
// row in four pieces.  The 8-bit output of over 16384 columns (three and four pieces of
// 1024 threads, 128 registers to each) does not fit: three aligned pieces spill nothing,
// four 10 registers in bf16 and 21 in fp32; unaligned three 6, four 34 and 73.  In bf16
// 2048 x 24576 take 77 us (4.6 TB/s), 2048 x 32768 130 (3.6), 2048 x 32767 230 (2.0).
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
  else if (pieces <= 3 * 1024) f(integral_constant<int, 1024>{}, integral_constant<int, 3>{});
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
  rms_fold_kernel<<<(a.cols + 63) / 64, kFoldThreads, 0, s>>>(a.part, n, a.cols, a.dgamma);
}

}  // namespace

// Workgroups of the backward.  Each holds the CU's registers for long, so there are as
// many as run at once, 2 of 256 threads to a CU or 1 of 512 and more.
constexpr int kParts = 512, kPartsWide = 256;
int rms_backward_parts(long long rows, int cols) {
  long long n = 0;
  by_width(cols, [&](auto tpr, auto) {
    constexpr int TPR = decltype(tpr)::value;
    constexpr int per = TPR < 256 ? 256 / TPR : 1;
    const long long sets = (rows + per - 1) / per, most = TPR > 256 ? kPartsWide : kParts;
    const long long each = (sets + most - 1) / most;  // sets of rows a workgroup
    n = sets ? (sets + each - 1) / each : 0;
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

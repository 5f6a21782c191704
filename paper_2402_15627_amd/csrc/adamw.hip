// One AdamW step over many fp32 tensors at once, states in 32 bits or in 8.
//
//   g = grad_scale grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
//   w = w (1 - lr decay) - lr (m c1) / (sqrt(v c2) + eps)
//
// Bound by HBM: each element of w, g and the states is read once and written
// once (30 bytes with a bf16 copy of w, 18 with states of 8 bits), so the
// arithmetic is free as long as it stays under about a hundred instructions an
// element: 226.5 M parameters 1180 us (5.8 TB/s), in 8 bits 667 (6.1).  A launch
// takes up to kAdamMax tensors, cut into chunks of 1024 elements, a workgroup
// each (2048: 1191 us, 4096: 1195); a thread has four elements, a wave the 256
// that share the scales of an 8-bit state.
//
// Every operation is rounded by itself (no contraction into fused products; a quotient
// in 2^32 is off by a step, see sqrt_near): a value that decides an 8-bit code is then the
// one that elementary operations give, codes do not depend on how a compiler groups
// them, and an element's result on no other element but by its block's scales.
#include "common.h"
#include "kernels.h"

namespace pb {
namespace {

// Tensors need the alignment of their elements only: gfx950 loads and stores
// vectors at any address.
typedef float f32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_a1 __attribute__((aligned(1)));

PB_DEV f32x4 load_stream(const float* p) {
  return __builtin_nontemporal_load(reinterpret_cast<const f32x4_a4*>(p));
}
PB_DEV void store_stream(float* p, const f32x4& v) {
  __builtin_nontemporal_store((f32x4_a4)v, reinterpret_cast<f32x4_a4*>(p));
}

// 32 random bits of element e: two rounds of shift and product.
PB_DEV uint32_t random_bits(uint64_t seed, uint64_t e) {
  uint32_t x = (uint32_t)e * 0x9E3779B1u + (uint32_t)seed;
  x = (x ^ (x >> 16)) * 0x6A09E667u;
  x += (uint32_t)(e >> 32) * 0x9E3779B1u + (uint32_t)(seed >> 32);
  x = (x ^ (x >> 15)) * 0xBB67AE85u;
  return x ^ (x >> 16);
}

// Largest of the wave's 64 unsigned words, in every lane.
template <int CTRL>
PB_DEV uint32_t umax_dpp(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true));
}
PB_DEV uint32_t wave_umax(uint32_t v) {
  v = umax_dpp<0x128>(v);  // rotations within 16 lanes
  v = umax_dpp<0x124>(v);
  v = umax_dpp<0x122>(v);
  v = umax_dpp<0x121>(v);
  const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
  v = max(a[0], a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return max(b[0], b[1]);
}

// e4m3 code of |y| <= 448 rounded up or down as `rnd` (16 bits, and 4 zeros) says: to a
// neighbour as often as y is near it.  Bits of the fp32 value below the code's
// last place meet the random ones in an integer sum; below 2^-6, where codes
// are multiples of 2^-9, the value itself takes the place of its bits.
PB_DEV uint32_t code_e4m3(float a, uint32_t rnd) {
  const uint32_t bits = a < 0x1p-6f ? (uint32_t)(a * 0x1p29f)
                                    : __float_as_uint(a) - (120u << 23);
  return min((bits + rnd) >> 20, 0x7eu);
}

// Four elements' updated state x (lane's part of its wave's 256) as codes; their
// scale is the largest magnitude over 448 (its product with the rounded 1/448),
// at least 2^-126.  A value that is not finite makes the scale so (magnitudes are
// compared as words, where NaN is above all).  bits: random, of each element; the upper
// half, or with KEEP the lower.  KEEP (x >= 0): what is above zero keeps a code above zero.
template <bool KEEP>
PB_DEV uint32_t quantise(const f32x4& x, const uint32_t (&bits)[4], float& scale) {
#pragma clang fp contract(off)
  uint32_t top = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) top = max(top, __float_as_uint(fabsf(x[k])));
  const float s = __uint_as_float(wave_umax(top)) * (1.0f / 448.0f);
  scale = s < 0x1p-126f ? 0x1p-126f : s;
  const float inv = 1.0f / scale;
  uint32_t word = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float y = x[k] * inv;
    uint32_t c = code_e4m3(fabsf(y), KEEP ? (bits[k] & 0xffffu) << 4 : bits[k] >> 16 << 4);
    if (KEEP) c = c == 0 && x[k] > 0.f ? 1u : c;
    else c |= (__float_as_uint(y) >> 24) & 0x80u;
    word |= c << (8 * k);
  }
  return word;
}
PB_DEV void dequantise(uint32_t word, float scale, f32x4& x) {
#pragma clang fp contract(off)
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8(word, false);
  const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
  x[0] = lo[0] * scale, x[1] = lo[1] * scale, x[2] = hi[0] * scale, x[3] = hi[1] * scale;
}

// Square root and quotient from the hardware's approximations and an exact remainder each.
// Beside the correctly rounded ones: roots the same for all 2^24 values of 1 .. 4 (other
// powers of four scale them), quotients but for one of 2^32, off by a step.  Half the
// instructions of the general ones, which also take care of values whose squares or
// reciprocals leave fp32.  x: 0, or 2^-90 .. 2^90; d: 2^-90 .. 2^90.
PB_DEV float sqrt_near(float x) {
  const float y = __builtin_amdgcn_rsqf(fmaxf(x, 0x1p-90f)), s = x * y;
  return __builtin_fmaf(__builtin_fmaf(-s, s, x), 0.5f * y, s);
}
PB_DEV float div_near(float n, float d) {
  const float y = __builtin_amdgcn_rcpf(d), q = n * y;
  return __builtin_fmaf(__builtin_fmaf(-d, q, n), y, q);
}
PB_DEV bool in_range(float x) { return x >= 0x1p-90f && x <= 0x1p90f; }

// One step of four elements; r: the root of the new v, where ROOT.
template <bool ROOT>
PB_DEV void update(const AdamScalars& c, float decay, const f32x4& grad, f32x4& w, f32x4& m,
                   f32x4& v, f32x4& r) {
#pragma clang fp contract(off)
  f32x4 vh;
  bool plain[4], all = true;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float g = grad[k] * c.grad_scale;
    m[k] = m[k] * c.beta1 + g * c.rest1;
    v[k] = v[k] * c.beta2 + (g * g) * c.rest2;
    vh[k] = v[k] * c.c2;
    plain[k] = c.eps_in_range && (v[k] == 0.f || (in_range(v[k]) && in_range(vh[k])));
    all = all && plain[k];
  }
  f32x4 u;
  if (__builtin_amdgcn_ballot_w64(!all) == 0) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      u[k] = div_near(m[k] * c.c1, sqrt_near(vh[k]) + c.eps);
      if (ROOT) r[k] = sqrt_near(v[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // (an element in range has the same bits beside one that is not)
      const float n = m[k] * c.c1, d = (plain[k] ? sqrt_near(vh[k]) : __builtin_sqrtf(vh[k])) + c.eps;
      u[k] = plain[k] ? div_near(n, d) : n / d;
      if (ROOT) r[k] = plain[k] ? sqrt_near(v[k]) : __builtin_sqrtf(v[k]);
    }
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) w[k] = w[k] * decay - u[k] * c.lr;
}

// n of four values (the tensor's end may be in between); WHOLE: all four.
template <bool WHOLE>
PB_DEV f32x4 load_some(const float* p, int n) {
  if (WHOLE || n == 4) return load_stream(p);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) v[k] = p[k];
  return v;
}
template <bool WHOLE>
PB_DEV void store_some(float* p, int n, const f32x4& v) {
  if (WHOLE || n == 4) return store_stream(p, v);
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) p[k] = v[k];
}
template <bool WHOLE>
PB_DEV void store_copy(bf16* p, int n, const f32x4& w) {
  if (WHOLE || n == 4)
    __builtin_nontemporal_store((u32x2_a2)u32x2{pack_bf2(w[0], w[1]), pack_bf2(w[2], w[3])},
                                reinterpret_cast<u32x2_a2*>(p));
  else
    for (int k = 0; k < n; ++k) p[k] = (bf16)w[k];
}
template <bool WHOLE>
PB_DEV void store_copy(float* p, int n, const f32x4& w) {
  store_some<WHOLE>(p, n, w);
}
template <bool WHOLE>
PB_DEV uint32_t load_codes(const uint8_t* p, int n) {
  if (WHOLE || n == 4) return *reinterpret_cast<const u32_a1*>(p);
  uint32_t v = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) v |= (uint32_t)p[k] << (8 * k);
  return v;
}
template <bool WHOLE>
PB_DEV void store_codes(uint8_t* p, int n, uint32_t v) {
  if (WHOLE || n == 4) {
    *reinterpret_cast<u32_a1*>(p) = v;
    return;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
    if (k < n) p[k] = (uint8_t)(v >> (8 * k));
}

// The tensor of a chunk: the last whose chunks begin at or before it.
PB_DEV int tensor_of(const AdamTable& t, int chunk) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (chunk >= t.chunk0[mid]) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// Elements e .. e + n - 1 of tensor i (n <= 4, a wave's lanes side by side).
template <bool E4M3, typename CT, bool WHOLE>
PB_DEV void step(const AdamTable& t, const AdamScalars& c, int i, long long e, int n) {
  f32x4 w = load_some<WHOLE>(t.w[i] + e, n), r;
  const f32x4 g = load_some<WHOLE>(t.g[i] + e, n);
  if constexpr (!E4M3) {
    float *mp = (float*)t.m[i] + e, *vp = (float*)t.v[i] + e;
    f32x4 m = load_some<WHOLE>(mp, n), v = load_some<WHOLE>(vp, n);
    update<false>(c, t.decay[i], g, w, m, v, r);
    store_some<WHOLE>(mp, n, m);
    store_some<WHOLE>(vp, n, v);
  } else {
#pragma clang fp contract(off)
    uint8_t *mp = (uint8_t*)t.m[i] + e, *vp = (uint8_t*)t.v[i] + e;
    float *ms = t.m_scale[i] + e / kAdamBlock, *vs = t.v_scale[i] + e / kAdamBlock;
    const uint32_t cm = load_codes<WHOLE>(mp, n), cv = load_codes<WHOLE>(vp, n);
    f32x4 m, v;
    dequantise(cm, *ms, m);
    dequantise(cv, *vs, v);
    v *= v;
    update<true>(c, t.decay[i], g, w, m, v, r);
    uint32_t bits[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      bits[k] = random_bits(t.seed[i], (uint64_t)(e + k));
      if (!WHOLE && k >= n) m[k] = r[k] = 0.f;
    }
    float s;
    store_codes<WHOLE>(mp, n, quantise<false>(m, bits, s));
    if ((threadIdx.x & 63) == 0) *ms = s;
    store_codes<WHOLE>(vp, n, quantise<true>(r, bits, s));
    if ((threadIdx.x & 63) == 0) *vs = s;
  }
  store_some<WHOLE>(t.w[i] + e, n, w);
  if (t.copy[i]) store_copy<WHOLE>((CT*)t.copy[i] + e, n, w);
}

template <bool E4M3, typename CT>
__global__ __launch_bounds__(256) void adamw_kernel(AdamTable t, AdamScalars c) {
  const int chunk = blockIdx.x, i = tensor_of(t, chunk);
  const long long e0 = (long long)(chunk - t.chunk0[i]) * kAdamChunk, e = e0 + 4 * threadIdx.x;
  if (e0 + kAdamChunk <= t.numel[i]) {
    step<E4M3, CT, true>(t, c, i, e, 4);
  } else {
    const int n = (int)max(0LL, min(4LL, t.numel[i] - e));
    // (a wave with any element stays whole, for its scales)
    if (e / kAdamBlock * kAdamBlock < t.numel[i]) step<E4M3, CT, false>(t, c, i, e, n);
  }
}

}  // namespace

void launch_adamw(const AdamTable& t, const AdamScalars& c, bool e4m3, Dt copy_dt, hipStream_t s) {
  static_assert(kAdamChunk == 1024 && kAdamBlock == 256, "four elements a thread, a wave a block");
  const int n = t.chunk0[t.n];
  if (e4m3) {
    if (copy_dt == Dt::BF16) adamw_kernel<true, bf16><<<n, 256, 0, s>>>(t, c);
    else adamw_kernel<true, float><<<n, 256, 0, s>>>(t, c);
  } else {
    if (copy_dt == Dt::BF16) adamw_kernel<false, bf16><<<n, 256, 0, s>>>(t, c);
    else adamw_kernel<false, float><<<n, 256, 0, s>>>(t, c);
  }
}

}  // namespace pb

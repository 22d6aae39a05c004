// 8-bit blocks and GeLU: what the kernels that make them and those that use them share (device), and the checks of their
// descriptors (host).
//
// A block's scale is 2^e, e the smallest integer >= -126 with amax <= 448 * 2^e.  Dividing by a power of two is exact (what
// falls below fp32's normal range rounds to zero in e4m3 either way), so each element is rounded once, and e comes from the bits of
// amax: 448 = 1.75 * 2^8, so amax = 1.m * 2^E needs e = E - 8 where 1.m <= 1.75 and E - 7 where it is above.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "bounds_check.h"
#include "sbp_internal.h"

namespace sbp {

constexpr int kBlock8 = 128;                 // elements of a block along the last axis, rows of a tile

inline int64_t blocks8(int64_t n) { return (n + kBlock8 - 1) / kBlock8; }

// Like check_tensor, and SBP_E4M3 is a dtype (sbp_api.cu).
sbp_status check_tensor8(const sbp_tensor* t, const char* name, bool need_ptrs);
// values / scales as the header describes them; tiles: -1 = either (told apart by the first extent, the answer goes to *is_tiles).
sbp_status check_blocks8(const sbp_tensor* values, const sbp_tensor* scales, const char* name, int tiles, bool need_ptrs, bool* is_tiles);

// Bits of a block's scale from the bits of its largest finite magnitude; those of 1 / scale are kInvBits less it.
constexpr unsigned kInvBits = 254u << 23;
__device__ __forceinline__ unsigned scale_bits(unsigned amax) {
  const int e = (int)(amax >> 23) - 8 + ((amax & 0x7fffffu) > 0x600000u ? 1 : 0);      // biased
  return amax == 0u ? 127u << 23 : (unsigned)max(e, 1) << 23;
}

// Two numbers as e4m3, to nearest even; their magnitudes are at most 448, or NaN.
__device__ __forceinline__ unsigned e4m3_two(float lo, float hi) {
  unsigned short r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ unsigned e4m3_four(const float* v) { return e4m3_two(v[0], v[1]) | e4m3_two(v[2], v[3]) << 16; }

// The number an e4m3 pair stands for.
__device__ __forceinline__ void two_of_e4m3(unsigned v, float& lo, float& hi) {
  unsigned h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)v));
  asm("{\n\t.reg .b16 a, b;\n\tmov.b32 {a, b}, %2;\n\tcvt.f32.f16 %0, a;\n\tcvt.f32.f16 %1, b;\n\t}" : "=f"(lo), "=f"(hi) : "r"(h));
}

// Magnitude bits of a number; what is not finite counts as zero.
__device__ __forceinline__ unsigned finite_bits(float v) {
  const unsigned b = __float_as_uint(v) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0u;
}
// v, its sign too where it is zero, or NaN where it is infinite (the conversion would saturate it)
__device__ __forceinline__ float inf_to_nan(float v) { return v - (v - v); }

// Eight elements of a row as they were loaded, so that loads may be ahead of their use at no more registers than the bytes need.
// VEC: they follow one another, all are there and the first is 16-byte aligned; else the first `n` are there, `step` elements apart (so that
// neighbouring lanes may take neighbouring ones).
template <typename T, bool VEC>
struct Eight;
template <>
struct Eight<float, true> {
  float4 a, b;
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p, int, int) {
    clear();
    if (SBP_GUARD(p, 32)) {
      a = __ldcs(reinterpret_cast<const float4*>(p));
      b = __ldcs(reinterpret_cast<const float4*>(p + 4));
    }
  }
  __device__ __forceinline__ void get(float* v) const {
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
};
template <>
struct Eight<__nv_bfloat16, true> {
  uint4 a;
  __device__ __forceinline__ void clear() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p, int, int) {
    clear();
    if (SBP_GUARD(p, 16)) a = __ldcs(reinterpret_cast<const uint4*>(p));
  }
  __device__ __forceinline__ void get(float* v) const {
    const unsigned w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
  }
};
template <typename T>
struct Eight<T, false> {
  float v_[8];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) v_[e] = 0.f;
  }
  __device__ __forceinline__ void load(const T* p, int n, int step) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v_[e] = e < n && SBP_GUARD(p + e * step, sizeof(T)) ? (float)p[e * step] : 0.f;
  }
  __device__ __forceinline__ void get(float* v) const {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v_[e];
  }
};

// Bits of the largest magnitude of eight numbers; infinities and NaN are larger than all numbers.
template <typename T, bool VEC>
__device__ __forceinline__ unsigned largest_bits(const Eight<T, VEC>& x) {
  float v[8];
  x.get(v);
  unsigned m = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
  return m;
}
__device__ __forceinline__ unsigned largest_bits(const Eight<__nv_bfloat16, true>& x) {      // in pairs
  constexpr unsigned kMag = 0x7fff7fffu;
  const unsigned m = __vmaxs2(__vimax3_s16x2(x.a.x & kMag, x.a.y & kMag, x.a.z & kMag), x.a.w & kMag);
  return max(m << 16, m & 0xffff0000u);
}

template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, float* v, int n = 8, int step = 1) {
  Eight<T, VEC> x;
  x.load(p, n, step);
  x.get(v);
}
__device__ __forceinline__ unsigned bf16_two(float lo, float hi) {
  unsigned r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, const float* v, int n = 8, int step = 1) {
  if constexpr (VEC) {
    if (SBP_GUARD(p, 32)) {
      __stcs(reinterpret_cast<float4*>(p), make_float4(v[0], v[1], v[2], v[3]));
      __stcs(reinterpret_cast<float4*>(p + 4), make_float4(v[4], v[5], v[6], v[7]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n && SBP_GUARD(p + e * step, 4)) p[e * step] = v[e];
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* v, int n = 8, int step = 1) {
  if constexpr (VEC) {
    if (SBP_GUARD(p, 16))
      __stcs(reinterpret_cast<uint4*>(p), make_uint4(bf16_two(v[0], v[1]), bf16_two(v[2], v[3]), bf16_two(v[4], v[5]), bf16_two(v[6], v[7])));
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < n && SBP_GUARD(p + e * step, 2)) p[e * step] = __float2bfloat16_rn(v[e]);
  }
}

__device__ __forceinline__ unsigned long long pair_of(float x, float y) {
  unsigned long long v;
  asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
  return v;
}
__device__ __forceinline__ unsigned long long pair_of(float x) { return pair_of(x, x); }
__device__ __forceinline__ float pair_lo(unsigned long long v) { return __uint_as_float((unsigned)v); }
__device__ __forceinline__ float pair_hi(unsigned long long v) { return __uint_as_float((unsigned)(v >> 32)); }
__device__ __forceinline__ unsigned long long pair_fma(unsigned long long a, unsigned long long b, unsigned long long c) {
  unsigned long long v;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
  return v;
}
__device__ __forceinline__ unsigned long long pair_add(unsigned long long a, unsigned long long b) {
  unsigned long long v;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}
__device__ __forceinline__ unsigned long long pair_mul(unsigned long long a, unsigned long long b) {
  unsigned long long v;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
  return v;
}

// Of two numbers t = min(|z|, 16), e = exp(-t^2 / 2) and q = Phi(-t), the normal distribution's tail.  Phi(-t) = e v(t), where v(t) = erfcx(t / sqrt 2) / 2
// falls off as 1 / t: it is k times a polynomial in k = 1 / (1 + 0.304 t) fitted to it for the smallest relative error (6e-8, over t up to
// 13.6; with its roundings 4e-7), so the tail keeps its digits until e underflows.
// From t = 16 on e is zero: what is larger, infinities too, is taken for 16.  NaN stays NaN.
// FINITE: there are no infinities, and t is |z| itself (e is zero all the same).  EXACT: z^2 is taken with what its rounding leaves, else its rounding is z^2 / 2 units in the last place of e (none for bf16 numbers).
// Cost: two special functions and some eleven instructions a number, for which erfcf and expf take about sixty.
template <bool EXACT, bool FINITE>
__device__ __forceinline__ void tail_two(float a, float b, unsigned long long& t, unsigned long long& q, unsigned long long& e) {
  float ta = fabsf(a), tb = fabsf(b);
  if constexpr (!FINITE) {
    asm("min.NaN.f32 %0, %0, 0f41800000;" : "+f"(ta));
    asm("min.NaN.f32 %0, %0, 0f41800000;" : "+f"(tb));
  }
  t = pair_of(ta, tb);
  const unsigned long long d = pair_fma(t, pair_of(0.30405593f), pair_of(1.0f));
  float ka, kb;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(ka) : "f"(pair_lo(d)));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(kb) : "f"(pair_hi(d)));
  const unsigned long long k = pair_of(ka, kb), c = pair_of(-0.72134752f), s = pair_mul(t, t);      // -log2(e) / 2
  unsigned long long x;
  if constexpr (EXACT) x = pair_fma(s, c, pair_mul(pair_fma(t, t, s ^ 0x8000000080000000ull), c));
  else x = pair_mul(s, c);
  float ea, eb;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(ea) : "f"(pair_lo(x)));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(eb) : "f"(pair_hi(x)));
  e = pair_of(ea, eb);
  unsigned long long v = pair_fma(k, pair_of(0.036719587f), pair_of(-0.15461463f));
  v = pair_fma(v, k, pair_of(0.19085145f));
  v = pair_fma(v, k, pair_of(-0.041933011f));
  v = pair_fma(v, k, pair_of(0.12292960f));
  v = pair_fma(v, k, pair_of(0.10262408f));
  v = pair_fma(v, k, pair_of(0.12216413f));
  v = pair_fma(v, k, pair_of(0.12125883f));
  q = pair_mul(pair_mul(v, k), e);
}

// GeLU(z) = z Phi(z) = max(z, 0) - |z| Phi(-|z|): below zero the tail alone, with its digits.  (Minus infinity gives 0.)
template <bool EXACT, bool FINITE>
__device__ __forceinline__ void gelu_two(float& a, float& b) {
  unsigned long long t, q, e;
  tail_two<EXACT, FINITE>(a, b, t, q, e);
  const unsigned long long y = pair_fma(t ^ 0x8000000080000000ull, q, pair_of(fmaxf(a, 0.f), fmaxf(b, 0.f)));
  a = pair_lo(y);
  b = pair_hi(y);
}

// Its slope Phi(z) + z phi(z), phi(z) = e / sqrt(2 pi): with r = Phi(-t) - t phi(t), that is r below zero and 1 - r above.
__device__ __forceinline__ void gelu_slope_two(float& a, float& b) {
  unsigned long long t, q, e;
  tail_two<false, false>(a, b, t, q, e);
  const unsigned long long r = pair_fma(pair_mul(t, e), pair_of(-0.39894228f), q);
  a = a < 0.f ? pair_lo(r) : 1.0f - pair_lo(r);
  b = b < 0.f ? pair_hi(r) : 1.0f - pair_hi(r);
}

}  // namespace sbp

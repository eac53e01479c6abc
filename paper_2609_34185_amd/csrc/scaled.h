// Element types of the 8-bit quantisers, their scales, division by a scale and codes.
#pragma once
#include <cstdint>

namespace ep {

struct Bf16 { uint16_t bits; };
struct Fp16 { _Float16 h; };

__device__ __forceinline__ float as_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float as_float(Fp16 x) { return (float)x.h; }
__device__ __forceinline__ float as_float(float x) { return x; }

// x / s rounded to FP32, for many x of one s.  From the correctly rounded r = 1 / s, q0 = x r and
// q = q0 + r (x - q0 s): one correction of a quotient that is within one unit gives the correctly
// rounded one (Markstein), as long as neither r nor the residual leaves the normal range.  Outside
// it the quotient is divided out, and clamped to `top`, since a subnormal scale may be off by half.
// A NaN stays one.
struct Divider {
  float s, r, top;
  bool fast;
  __device__ __forceinline__ Divider(float scale, float largest) : s(scale), top(largest) {
    fast = s >= 0x1p-60f && s < 0x1p126f;
    r = 1.0f / s;
  }
  __device__ __forceinline__ float operator()(float x) const {
    if (fast) {
      const float q0 = x * r;
      return __builtin_fmaf(__builtin_fmaf(-q0, s, x), r, q0);
    }
    const float q = x / s;
    return q > top ? top : q < -top ? -top : q;
  }
};

// ---- eight consecutive elements ---------------------------------------------------
__device__ __forceinline__ void load8(const Bf16* p, float (&v)[8]) {
  typedef uint32_t v4u __attribute__((ext_vector_type(4)));
  const v4u w = *reinterpret_cast<const v4u*>(p);
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void load8(const Fp16* p, float (&v)[8]) {
  typedef _Float16 v8h __attribute__((ext_vector_type(8)));
  const v8h w = *reinterpret_cast<const v8h*>(p);
#pragma unroll
  for (int i = 0; i < 8; i++) v[i] = (float)w[i];
}
__device__ __forceinline__ void load8(const float* p, float (&v)[8]) {
  typedef float v4f __attribute__((ext_vector_type(4)));
  const v4f a = reinterpret_cast<const v4f*>(p)[0], b = reinterpret_cast<const v4f*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}

// Largest magnitude as bits: the order of the bits of |x| is the order of |x|, an infinity
// above every finite value and a NaN above that, so neither is lost in a maximum.
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8]) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) t = max(t, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return t;
}

// The scale of values whose largest magnitude has these bits, `most` being the largest code.
constexpr float kE4m3Max = 448.0f, kI8Max = 127.0f;
__device__ __forceinline__ float scale_of(uint32_t top, float most) {
  const float s = __uint_as_float(top) * (1.0f / most);
  return s == 0.0f ? 1.0f : s;
}

// E4M3(x / s) of eight values.
typedef uint32_t codes_v2u __attribute__((ext_vector_type(2)));
__device__ __forceinline__ codes_v2u codes8(const float (&v)[8], const Divider& by) {
  codes_v2u out;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(by(v[4 * i]), by(v[4 * i + 1]), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(by(v[4 * i + 2]), by(v[4 * i + 3]), w, true);
    out[i] = (uint32_t)w;
  }
  return out;
}

}  // namespace ep

// Element types of the 8-bit quantisers and their division by a scale.
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

}  // namespace ep

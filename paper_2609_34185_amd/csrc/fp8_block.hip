// FP8 with a scale for each block of 128: the quantiser of activations (and weights), and the
// product Y = X W^T that reads its output next to FP8 weights, such as an entropy-coded FP8
// container decodes to.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"

namespace ep {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kE4m3Max = 448.0f;

// ---- element types -------------------------------------------------------------
struct Bf16 { uint16_t bits; };
struct Fp16 { _Float16 h; };

// Eight consecutive elements as floats.
__device__ __forceinline__ void load8(const Bf16* p, float (&v)[8]) {
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
  const v4f a = reinterpret_cast<const v4f*>(p)[0], b = reinterpret_cast<const v4f*>(p)[1];
#pragma unroll
  for (int i = 0; i < 4; i++) {
    v[i] = a[i];
    v[4 + i] = b[i];
  }
}

// ---- quantiser -------------------------------------------------------------------
// Largest magnitude as bits: the order of the bits of |x| is the order of |x|, an infinity
// above every finite value and a NaN above that, so neither is lost in a maximum.
__device__ __forceinline__ uint32_t top_bits(const float (&v)[8]) {
  uint32_t t = 0;
#pragma unroll
  for (int i = 0; i < 8; i++) t = max(t, __float_as_uint(v[i]) & 0x7FFFFFFFu);
  return t;
}

__device__ __forceinline__ float scale_of(uint32_t top) {
  const float s = __uint_as_float(top) / kE4m3Max;
  return s == 0.0f ? 1.0f : s;
}

// E4M3(x / s) of eight values.  x / s rounded to FP32 is formed from the correctly rounded
// r = 1 / s as q0 = x r, q = q0 + r (x - q0 s): one correction of a quotient that is within
// one unit gives the correctly rounded one (Markstein), as long as neither r nor the residual
// leaves the normal range.  Outside it the quotient is divided out, and clamped since a
// subnormal scale may be off by half.  A NaN stays one.
__device__ __forceinline__ v2u codes8(const float (&v)[8], float s) {
  float q[8];
  if (s >= 0x1p-60f && s < 0x1p126f) {
    const float r = 1.0f / s;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float q0 = v[i] * r;
      q[i] = __builtin_fmaf(__builtin_fmaf(-q0, s, v[i]), r, q0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float d = v[i] / s;
      q[i] = d > kE4m3Max ? kE4m3Max : d < -kE4m3Max ? -kE4m3Max : d;
    }
  }
  v2u out;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i], q[4 * i + 1], 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(q[4 * i + 2], q[4 * i + 3], w, true);
    out[i] = (uint32_t)w;
  }
  return out;
}

constexpr int kQuantThreads = 256;
constexpr int kLanes = 16;                 // lanes on one 128-column block, eight columns each

// One row's block of 128 for each 16 lanes.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quant_rows_kernel(const T* __restrict__ x,
                                                                   uint8_t* __restrict__ q,
                                                                   float* __restrict__ scale,
                                                                   uint32_t units, uint32_t kb,
                                                                   int64_t k, int64_t x_row) {
  const uint32_t unit = blockIdx.x * (kQuantThreads / kLanes) + threadIdx.x / kLanes;
  if (unit >= units) return;
  const uint32_t row = unit / kb, col = (unit - row * kb) * 128 + 8 * (threadIdx.x % kLanes);
  float v[8] = {};
  if (col < k) load8(x + row * x_row + col, v);
  uint32_t top = top_bits(v);
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const float s = scale_of(top);
  if (col < k) *reinterpret_cast<v2u*>(q + row * k + col) = codes8(v, s);
  if (threadIdx.x % kLanes == 0) scale[unit] = s;
}

// One 128 x 128 block for each workgroup.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quant_blocks_kernel(const T* __restrict__ x,
                                                                     uint8_t* __restrict__ q,
                                                                     float* __restrict__ scale,
                                                                     uint32_t kb, int64_t m, int64_t k,
                                                                     int64_t x_row) {
  constexpr int kRows = kQuantThreads / kLanes, kPasses = 128 / kRows;
  __shared__ uint32_t wave_top[kQuantThreads / 64];
  const uint32_t bi = blockIdx.x / kb, col = (blockIdx.x - bi * kb) * 128 + 8 * (threadIdx.x % kLanes);
  const int64_t r0 = (int64_t)bi * 128 + threadIdx.x / kLanes;
  float v[kPasses][8] = {};
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < kPasses; p++) {
    if (col < k && r0 + kRows * p < m) load8(x + (r0 + kRows * p) * x_row + col, v[p]);
    top = max(top, top_bits(v[p]));
  }
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if (threadIdx.x % 64 == 0) wave_top[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kQuantThreads / 64; w++) top = max(top, wave_top[w]);
  const float s = scale_of(top);
#pragma unroll
  for (int p = 0; p < kPasses; p++)
    if (col < k && r0 + kRows * p < m)
      *reinterpret_cast<v2u*>(q + (r0 + kRows * p) * k + col) = codes8(v[p], s);
  if (threadIdx.x == 0) scale[blockIdx.x] = s;
}

template <typename T>
void quant_launch(const void* x, uint8_t* q, float* scale, int64_t m, int64_t k, int64_t x_row,
                  int block_rows, uint32_t kb, hipStream_t stream) {
  if (block_rows == 1) {
    const uint32_t units = (uint32_t)(m * kb), per = kQuantThreads / kLanes;
    hipLaunchKernelGGL(quant_rows_kernel<T>, dim3((units + per - 1) / per), dim3(kQuantThreads), 0, stream,
                       static_cast<const T*>(x), q, scale, units, kb, k, x_row);
  } else {
    hipLaunchKernelGGL(quant_blocks_kernel<T>, dim3((uint32_t)((m + 127) / 128 * kb)), dim3(kQuantThreads), 0,
                       stream, static_cast<const T*>(x), q, scale, kb, m, k, x_row);
  }
}

// ---- product -----------------------------------------------------------------------
struct Product {
  const uint8_t* x;
  const float* x_scale;
  const uint8_t* w;
  const float* w_scale;
  void* y;
  int64_t m, n, k;
  uint32_t kb;         // blocks of 128 along k
  uint32_t w_scales;   // ep_scale_layout
  uint32_t y_dtype;
};

// Scale of W's row j in block b.
__device__ __forceinline__ float w_scale_at(const Product& P, int64_t j, uint32_t b) {
  if (P.w_scales == EP_SCALE_ROW) return P.w_scale[j];
  return P.w_scale[(P.w_scales == EP_SCALE_BLOCK ? j / 128 : j) * P.kb + b];
}

__device__ __forceinline__ uint16_t bf16_of(float f) {
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);   // a NaN stays one
  return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
}

__device__ __forceinline__ void store_y(const Product& P, int64_t at, float f) {
  if (P.y_dtype == EP_FP32) static_cast<float*>(P.y)[at] = f;
  else if (P.y_dtype == EP_FP16) static_cast<_Float16*>(P.y)[at] = (_Float16)f;
  else static_cast<uint16_t*>(P.y)[at] = bf16_of(f);
}

// One 16 x 16 tile of Y for each wave.  v_mfma_f32_16x16x128_f8f6f4 multiplies 16 rows of W by
// 16 rows of X over one whole block: lane l supplies 32 bytes of row l mod 16 of both, and gets
// the products of W rows 4 (l / 16) + 0 .. 3 with X row l mod 16.  Which 32 of the block's 128
// bytes a quarter of the wave supplies does not matter as long as both operands agree.
//
// The FP8 instructions add their products in fewer bits than FP32: measured against 64 bits, a
// block of Gaussian codes is off by 1.4e-5 of its size (root mean square), which disappears in the
// rounding to BF16 (1.7e-3) or FP16 (2.1e-4).  FP32 outputs (EXACT) take FP16 instructions
// instead, into which both FP8 types widen without rounding, at half the rate: 8e-8.
template <int WFMT>
__device__ __forceinline__ v8h widen8(int lo, int hi) {
  v2h a, b, c, d;
  if (WFMT == 0) {
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(lo, 1.0f, true);
    c = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.0f, false);
    d = __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(hi, 1.0f, true);
  }
  return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int WFMT, bool EXACT>
__device__ __forceinline__ v4f block_product(const v8i& w, const v8i& x) {
  if (!EXACT) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, v4f{}, WFMT, 0, 0, 0, 0, 0);
  v4f part = {};
#pragma unroll
  for (int i = 0; i < 4; i++)
    part = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<WFMT>(w[2 * i], w[2 * i + 1]), widen8<0>(x[2 * i], x[2 * i + 1]), part, 0, 0, 0);
  return part;
}

template <int WFMT, bool EXACT>
__global__ __launch_bounds__(256) void product_kernel(Product P) {
  const int lane = threadIdx.x & 63, row = lane & 15, quarter = lane >> 4;
  const int64_t tn = (P.n + 15) / 16, tile = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t i0 = tile / tn * 16, j0 = tile % tn * 16;
  if (i0 >= P.m) return;
  const int64_t i = i0 + row, j = j0 + row;
  v4f acc = {};
  for (uint32_t b = 0; b < P.kb; b++) {
    v8i xw[2] = {};
    const uint8_t* src[2] = {P.w + j * P.k, P.x + i * P.k};
    const bool in[2] = {j < P.n, i < P.m};
#pragma unroll
    for (int o = 0; o < 2; o++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int64_t at = (int64_t)b * 128 + 64 * h + 16 * quarter;
        if (in[o] && at < P.k) {
          const v4i t = *reinterpret_cast<const v4i*>(src[o] + at);
#pragma unroll
          for (int e = 0; e < 4; e++) xw[o][4 * h + e] = t[e];
        }
      }
    const v4f part = block_product<WFMT, EXACT>(xw[0], xw[1]);
    const float xs = i < P.m ? P.x_scale[i * P.kb + b] : 0.0f;
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int64_t jr = j0 + 4 * quarter + r;
      const float ws = jr < P.n ? w_scale_at(P, jr, b) : 0.0f;
      acc[r] = __builtin_fmaf(part[r], xs * ws, acc[r]);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int64_t jr = j0 + 4 * quarter + r;
    if (i < P.m && jr < P.n) store_y(P, i * P.n + jr, acc[r]);
  }
}

template <int WFMT>
void product_launch(const Product& P, uint32_t groups, hipStream_t stream) {
  if (P.y_dtype == EP_FP32)
    hipLaunchKernelGGL((product_kernel<WFMT, true>), dim3(groups), dim3(256), 0, stream, P);
  else
    hipLaunchKernelGGL((product_kernel<WFMT, false>), dim3(groups), dim3(256), 0, stream, P);
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

}  // namespace
}  // namespace ep

extern "C" int ep_quant_fp8_block(const void* d_x, int x_dtype, int64_t m, int64_t k, int64_t x_row,
                                  int block_rows, void* d_q, float* d_scale, void* hip_stream) {
  if (m < 0 || k <= 0 || k % 16) return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: need m >= 0, k > 0 and k % 16 == 0");
  if (x_row < k) return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: x_row below k");
  if (block_rows != 1 && block_rows != 128)
    return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: block_rows must be 1 or 128");
  if (x_dtype != EP_BF16 && x_dtype != EP_FP16 && x_dtype != EP_FP32)
    return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: x_dtype must be BF16, FP16 or FP32");
  if (x_row % (x_dtype == EP_FP32 ? 4 : 8))
    return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: rows of x must be 16-byte aligned");
  if (m == 0) return EP_OK;
  if (!d_x || !d_q || !d_scale) return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: null pointer");
  if (ep::misaligned(d_x) || ep::misaligned(d_q))
    return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: x and q must be 16-byte aligned");
  const int64_t kb = (k + 127) / 128;
  if (kb > 0x7FFFFFFF || m > 0x7FFFFFFF / kb)
    return ep::fail(EP_ERR_ARG, "ep_quant_fp8_block: more than 2^31 - 1 blocks");
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  uint8_t* const q = static_cast<uint8_t*>(d_q);
  if (x_dtype == EP_BF16) ep::quant_launch<ep::Bf16>(d_x, q, d_scale, m, k, x_row, block_rows, (uint32_t)kb, stream);
  else if (x_dtype == EP_FP16) ep::quant_launch<ep::Fp16>(d_x, q, d_scale, m, k, x_row, block_rows, (uint32_t)kb, stream);
  else ep::quant_launch<float>(d_x, q, d_scale, m, k, x_row, block_rows, (uint32_t)kb, stream);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_quant_fp8_block: launch failed");
  return EP_OK;
}

extern "C" int ep_gemm_fp8_block(const void* d_x, const float* d_x_scale, const void* d_w, int w_dtype,
                                 const float* d_w_scale, int w_scales, void* d_y, int y_dtype, int64_t m,
                                 int64_t n, int64_t k, void* hip_stream) {
  constexpr int64_t kMost = 1 << 24;
  if (m < 0 || n <= 0 || k <= 0 || k % 16 || m > kMost || n > kMost || k > kMost)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: need m >= 0, n, k > 0, k % 16 == 0, none above 2^24");
  if (w_dtype != EP_FP8_E4M3 && w_dtype != EP_FP8_E5M2)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: w_dtype must be FP8_E4M3 or FP8_E5M2");
  if (w_scales < EP_SCALE_BLOCK || w_scales > EP_SCALE_ROW)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: unknown layout of the weights' scales");
  if (y_dtype != EP_BF16 && y_dtype != EP_FP16 && y_dtype != EP_FP32)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: y_dtype must be BF16, FP16 or FP32");
  if (m == 0) return EP_OK;
  if (!d_x || !d_x_scale || !d_w || !d_w_scale || !d_y)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: null pointer");
  if (ep::misaligned(d_x) || ep::misaligned(d_w))
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: operands must be 16-byte aligned");
  const ep::Product P = {static_cast<const uint8_t*>(d_x), d_x_scale, static_cast<const uint8_t*>(d_w), d_w_scale,
                         d_y, m, n, k, (uint32_t)((k + 127) / 128), (uint32_t)w_scales, (uint32_t)y_dtype};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const int64_t tiles = (m + 15) / 16 * ((n + 15) / 16), groups = (tiles + 3) / 4;
  if (groups > 0x7FFFFFFF) return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: matrix too large");
  if (w_dtype == EP_FP8_E4M3) ep::product_launch<0>(P, (uint32_t)groups, stream);
  else ep::product_launch<1>(P, (uint32_t)groups, stream);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_gemm_fp8_block: launch failed");
  return EP_OK;
}

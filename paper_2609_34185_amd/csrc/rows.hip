// Operators on rows between a layer's products: norms with the residual sum and its gate, the
// gated activation, and the INT8 quantiser.  A row is read once, held in registers as FP32 while
// its statistics are summed, and written once, rounded or quantised for the next product.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"
#include "scaled.h"

namespace ep {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v8f __attribute__((ext_vector_type(8)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr int64_t kMostRow = 65536;   // elements: 1024 threads of eight vectors of eight

// ---- eight elements of a type that is known at run time ----------------------------------
// Loads do not depend on the type but by its size, so that several rows' loads are in flight
// before the first one's values are needed.
struct Raw8 {
  v4u lo, hi;
};
__device__ __forceinline__ Raw8 raw8(const void* row, int dtype, uint32_t vec) {
  Raw8 r = {};
  if (dtype == EP_FP32) {
    const v4u* const p = static_cast<const v4u*>(row) + 2 * (size_t)vec;
    r.lo = p[0];
    r.hi = p[1];
  } else {
    r.lo = static_cast<const v4u*>(row)[vec];
  }
  return r;
}
__device__ __forceinline__ void widen8(const Raw8& r, int dtype, float (&v)[8]) {
  if (dtype == EP_BF16) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[2 * i] = __uint_as_float(r.lo[i] << 16);
      v[2 * i + 1] = __uint_as_float(r.lo[i] & 0xFFFF0000u);
    }
  } else if (dtype == EP_FP16) {
    const v8h h = __builtin_bit_cast(v8h, r.lo);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)h[i];
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      v[i] = __uint_as_float(r.lo[i]);
      v[4 + i] = __uint_as_float(r.hi[i]);
    }
  }
}
__device__ __forceinline__ void load8(const void* row, int dtype, uint32_t vec, float (&v)[8]) {
  widen8(raw8(row, dtype, vec), dtype, v);
}
__device__ __forceinline__ void store8(void* row, int dtype, uint32_t vec, const float (&v)[8]) {
  const v8f f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
  if (dtype == EP_BF16) {
    static_cast<v8b*>(row)[vec] = __builtin_convertvector(f, v8b);
  } else if (dtype == EP_FP16) {
    static_cast<v8h*>(row)[vec] = __builtin_convertvector(f, v8h);
  } else {
    static_cast<v4f*>(row)[2 * (size_t)vec] = v4f{v[0], v[1], v[2], v[3]};
    static_cast<v4f*>(row)[2 * (size_t)vec + 1] = v4f{v[4], v[5], v[6], v[7]};
  }
}
// The row that lies `row` rows of `ld` elements of a type after p.
__device__ __forceinline__ const void* row_at(const void* p, int dtype, int64_t row, int64_t ld) {
  return static_cast<const uint8_t*>(p) + row * ld * (dtype == EP_FP32 ? 4 : 2);
}
__device__ __forceinline__ void* row_at(void* p, int dtype, int64_t row, int64_t ld) {
  return static_cast<uint8_t*>(p) + row * ld * (dtype == EP_FP32 ? 4 : 2);
}

// INT8 round(x / s) of eight values, halves to even.
__device__ __forceinline__ v2u codes8_i8(const float (&v)[8], const Divider& by) {
  v2u out;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    uint32_t w = 0;
#pragma unroll
    for (int j = 0; j < 4; j++) {
      const float q = fminf(fmaxf(rintf(by(v[4 * i + j])), -kI8Max), kI8Max);
      w |= ((uint32_t)(int)q & 0xFFu) << (8 * j);
    }
    out[i] = w;
  }
  return out;
}

// ---- a row's threads ---------------------------------------------------------------------
// L lanes of a wave hold a row (L is 16, 32 or 64, several rows to a workgroup), or the whole
// workgroup (L is 0); thread t holds vectors t, t + lanes, ...: V of them, eight elements each.
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
struct Top {
  __device__ __forceinline__ uint32_t operator()(uint32_t a, uint32_t b) const { return max(a, b); }
};

template <int L>
struct RowThreads {
  uint32_t* lds;   // two buffers of 16, used in turn: a reduction's reads end before the next one's barrier
  uint32_t turn = 0;
  __device__ __forceinline__ explicit RowThreads(uint32_t* mem) : lds(mem) {}
  __device__ __forceinline__ static uint32_t lanes() { return L ? L : blockDim.x; }
  __device__ __forceinline__ static uint32_t at() { return L ? threadIdx.x % (L ? L : 1) : threadIdx.x; }
  // The row's reduction in every thread of it, in an order that the sizes alone decide.
  template <typename T, typename F>
  __device__ __forceinline__ T all(T x, F f) {
    static_assert(sizeof(T) == 4, "one word");
#pragma unroll
    for (int d = 1; d < (L ? L : 64); d *= 2) x = f(x, __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, x), d)));
    if (L) return x;
    uint32_t* const slot = lds + 16 * turn;
    turn ^= 1;
    if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = __builtin_bit_cast(uint32_t, x);
    __syncthreads();
    x = __builtin_bit_cast(T, slot[0]);
    for (uint32_t w = 1; w < blockDim.x / 64; w++) x = f(x, __builtin_bit_cast(T, slot[w]));
    return x;
  }
  __device__ __forceinline__ float sum(float x) { return all(x, Sum{}); }
  __device__ __forceinline__ uint32_t top(uint32_t x) { return all(x, Top{}); }
};

// Subtracts the mean (layer norm) and returns the factor that makes the row's mean square 1.  A row
// whose sums pass FP32's range is scaled down by a power of two first, and v with it.
template <int L, int V>
__device__ __forceinline__ float normed(RowThreads<L>& row, float (&v)[V][8], int kind, uint32_t vecs, uint32_t n, float eps) {
  bool scaled = false;
  for (;;) {
    float mean = 0.0f, part = 0.0f;
    if (kind == EP_NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int j = 0; j < V; j++)
#pragma unroll
        for (int i = 0; i < 8; i++) s += v[j][i];
      mean = row.sum(s) / (float)n;
    }
#pragma unroll
    for (int j = 0; j < V; j++)
      if (row.at() + j * row.lanes() < vecs) {
#pragma unroll
        for (int i = 0; i < 8; i++) {
          const float d = v[j][i] - mean;
          part = __builtin_fmaf(d, d, part);
        }
      }
    const float total = row.sum(part);
    if (total < INFINITY || scaled) {
      if (kind == EP_NORM_LAYER) {
#pragma unroll
        for (int j = 0; j < V; j++)
#pragma unroll
          for (int i = 0; i < 8; i++) v[j][i] -= mean;
      }
      return 1.0f / __builtin_sqrtf(total / (float)n + eps);
    }
    // all threads of a row come here together; those of a wave's other rows take part in its shuffles
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < V; j++) top = max(top, top_bits(v[j]));
    top = row.top(top);
    // 2^-e with 2^e the power of two below the largest (a NaN or infinity stays what it is)
    const int e = (int)(top >> 23) - 127;
    const float down = __builtin_ldexpf(1.0f, -e);
#pragma unroll
    for (int j = 0; j < V; j++)
#pragma unroll
      for (int i = 0; i < 8; i++) v[j][i] *= down;
    eps = fmaxf(__builtin_ldexpf(eps, -2 * e), 0x1p-126f);   // above 0, for a row whose deviations are
    scaled = true;
  }
}

// Rounds or quantises the row and writes it; vectors at or past `vecs` hold zeros.
template <int L, int V>
__device__ __forceinline__ void write_row(RowThreads<L>& row, const float (&v)[V][8], uint32_t vecs, void* y, int dtype, float* scale) {
  if (dtype == EP_INT8) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < V; j++) top = max(top, top_bits(v[j]));
    const float s = scale_of(row.top(top), kI8Max);
    const Divider by(s, kI8Max);
#pragma unroll
    for (int j = 0; j < V; j++) {
      const uint32_t vec = row.at() + j * row.lanes();
      if (vec < vecs) static_cast<v2u*>(y)[vec] = codes8_i8(v[j], by);
    }
    if (row.at() == 0) *scale = s;
    return;
  }
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = row.at() + j * row.lanes();
    if (dtype == EP_FP8_E4M3) {   // sixteen lanes hold a block of 128
      uint32_t top = top_bits(v[j]);
#pragma unroll
      for (int d = 1; d < 16; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
      const float s = scale_of(top, kE4m3Max);
      if (vec < vecs) {
        static_cast<v2u*>(y)[vec] = codes8(v[j], Divider(s, kE4m3Max));
        if (vec % 16 == 0) scale[vec / 16] = s;
      }
    } else if (vec < vecs) {
      store8(y, dtype, vec, v[j]);
    }
  }
}

// Where row i of y and of its scales begin.
struct RowOut {
  void* y;
  float* scale;
  int64_t y_row;
  int dtype;
  uint32_t n;
  __device__ __forceinline__ void* row(int64_t i) const {
    return static_cast<uint8_t*>(y) + i * y_row * (dtype == EP_FP32 ? 4 : dtype == EP_BF16 || dtype == EP_FP16 ? 2 : 1);
  }
  __device__ __forceinline__ float* scale_row(int64_t i) const {
    return dtype == EP_FP8_E4M3 ? scale + i * ((n + 127) / 128) : dtype == EP_INT8 ? scale + i : nullptr;
  }
};

__device__ __forceinline__ int64_t row_of(uint32_t lanes) {
  return ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (blockDim.x / lanes) + threadIdx.x / lanes;
}

// ---- norm ----------------------------------------------------------------------------------
template <int L, int V>
__global__ __launch_bounds__(L ? 256 : 1024) void norm_kernel(ep_norm_call C) {
  __shared__ uint32_t lds[32];
  RowThreads<L> row(lds);
  const int64_t i = row_of(row.lanes());
  if (i >= C.m) return;   // whole rows: threads of a row leave together
  const uint32_t n = (uint32_t)C.n, vecs = n / 8;
  const uint32_t group = C.group_rows && i >= C.group_rows ? (uint32_t)i / (uint32_t)C.group_rows : 0;   // both below 2^31 where divided
  const void* const x = row_at(C.d_x, C.x_dtype, i, C.x_row);
  const void* const res = C.d_res ? row_at(C.d_res, C.res_dtype, i, C.res_row) : nullptr;
  const void* const gate = C.d_gate ? row_at(C.d_gate, C.w_dtype, group, C.gate_ld) : nullptr;
  const void* const w = C.d_w ? row_at(C.d_w, C.w_dtype, group, C.w_ld) : nullptr;
  const void* const b = C.d_b ? row_at(C.d_b, C.w_dtype, group, C.b_ld) : nullptr;

  float v[V][8];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = row.at() + j * row.lanes();
#pragma unroll
    for (int e = 0; e < 8; e++) v[j][e] = 0.0f;
    if (vec < vecs) load8(x, C.x_dtype, vec, v[j]);
  }
  if (C.post != EP_NORM_NONE) {
    const float r = normed<L, V>(row, v, C.post, vecs, n, C.eps);
#pragma unroll
    for (int j = 0; j < V; j++) {
      const uint32_t vec = row.at() + j * row.lanes();
      if (vec >= vecs) continue;
      float f[8];
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= r;
      if (C.d_post_w) {
        load8(C.d_post_w, C.w_dtype, vec, f);
#pragma unroll
        for (int e = 0; e < 8; e++) v[j][e] *= f[e];
      }
      if (C.d_post_b) {
        load8(C.d_post_b, C.w_dtype, vec, f);
#pragma unroll
        for (int e = 0; e < 8; e++) v[j][e] += f[e];
      }
    }
  }
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = row.at() + j * row.lanes();
    if (vec >= vecs) {
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = 0.0f;
      continue;
    }
    float f[8];
    if (gate) {
      load8(gate, C.w_dtype, vec, f);
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= f[e];
    }
    if (res) {
      load8(res, C.res_dtype, vec, f);
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = __builtin_fmaf(C.alpha, v[j][e], f[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= C.alpha;
    }
    if (C.d_res_out) store8(row_at(C.d_res_out, C.res_dtype, i, C.res_out_row), C.res_dtype, vec, v[j]);
  }
  if (C.pre == EP_NORM_NONE) return;
  const float r = normed<L, V>(row, v, C.pre, vecs, n, C.eps);
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = row.at() + j * row.lanes();
    if (vec >= vecs) {
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = 0.0f;
      continue;
    }
    float f[8], a[8] = {};
    if (b) load8(b, C.w_dtype, vec, a);
    if (w) {
      load8(w, C.w_dtype, vec, f);
      if (C.w_plus_one) {
#pragma unroll
        for (int e = 0; e < 8; e++) f[e] += 1.0f;
      }
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = __builtin_fmaf(v[j][e] * r, f[e], a[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = __builtin_fmaf(v[j][e], r, a[e]);
    }
  }
  const RowOut out = {C.d_y, C.d_y_scale, C.y_row, C.y_dtype, n};
  write_row<L, V>(row, v, vecs, out.row(i), C.y_dtype, out.scale_row(i));
}

// ---- activation and quantiser -----------------------------------------------------------------
struct ActCall {
  const void* a;
  const void* b;   // nullable
  int64_t m, a_row, b_row;
  int x_dtype, act;
  RowOut out;
};

constexpr int kActNone = 0;

// a / (1 + exp(-z)), by the exponential that does not overflow: far out on the negative side it falls
// to 0 through FP32's subnormal values.
__device__ __forceinline__ float gated(float a, float z) {
  const float e = expf(-fabsf(z));
  return (z < 0.0f ? a * e : a) / (1.0f + e);
}
__device__ __forceinline__ float activated(float a, int act) {
  if (act == EP_ACT_SILU) return gated(a, a);
  if (act == EP_ACT_GELU) return 0.5f * a * erfcf(-0.70710678118654752f * a);
  // (1 + tanh z) / 2 is 1 / (1 + exp(-2 z))
  return gated(a, 1.5957691216057308f * __builtin_fmaf(0.044715f * a * a, a, a));
}

template <int L, int V>
__global__ __launch_bounds__(L ? 256 : 1024) void act_kernel(ActCall C) {
  __shared__ uint32_t lds[32];
  RowThreads<L> row(lds);
  const int64_t i = row_of(row.lanes());
  if (i >= C.m) return;
  const uint32_t vecs = C.out.n / 8;
  const void* const a = row_at(C.a, C.x_dtype, i, C.a_row);
  const void* const b = C.b ? row_at(C.b, C.x_dtype, i, C.b_row) : nullptr;
  float v[V][8];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = row.at() + j * row.lanes();
#pragma unroll
    for (int e = 0; e < 8; e++) v[j][e] = 0.0f;
    if (vec >= vecs) continue;
    load8(a, C.x_dtype, vec, v[j]);
    if (C.act != kActNone) {
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] = activated(v[j][e], C.act);
    }
    if (b) {
      float f[8];
      load8(b, C.x_dtype, vec, f);
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= f[e];
    }
  }
  write_row<L, V>(row, v, vecs, C.out.row(i), C.out.dtype, C.out.scale_row(i));
}

// ---- launches --------------------------------------------------------------------------------
struct Shape {
  int lanes, vectors;   // of a row; lanes 0: a workgroup of `threads`
  int threads;
};
Shape shape_of(int64_t n) {
  const int64_t vecs = n / 8;
  if (vecs <= 16) return {16, 1, 256};
  if (vecs <= 32) return {32, 1, 256};
  if (vecs <= 64) return {64, 1, 256};
  const int v = vecs <= 1024 ? 1 : vecs <= 2048 ? 2 : vecs <= 4096 ? 4 : 8;
  return {0, v, (int)(((vecs + v - 1) / v + 63) / 64 * 64)};
}
// Workgroups in one or more rows of a grid, whose x dimension holds fewer than 2^32 threads.
dim3 row_grid(int64_t m, const Shape& s) {
  const int64_t per = s.lanes ? s.threads / s.lanes : 1, groups = (m + per - 1) / per;
  const int64_t x = std::min<int64_t>(groups, 1 << 21);
  return dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x));
}

#define EP_ROW_LAUNCH(kernel, L, V, call) hipLaunchKernelGGL((kernel<L, V>), grid, dim3(s.threads), 0, stream, call)
#define EP_ROW_LAUNCHES(kernel, call)                           \
  do {                                                          \
    if (s.lanes == 16) EP_ROW_LAUNCH(kernel, 16, 1, call);      \
    else if (s.lanes == 32) EP_ROW_LAUNCH(kernel, 32, 1, call); \
    else if (s.lanes == 64) EP_ROW_LAUNCH(kernel, 64, 1, call); \
    else if (s.vectors == 1) EP_ROW_LAUNCH(kernel, 0, 1, call); \
    else if (s.vectors == 2) EP_ROW_LAUNCH(kernel, 0, 2, call); \
    else if (s.vectors == 4) EP_ROW_LAUNCH(kernel, 0, 4, call); \
    else EP_ROW_LAUNCH(kernel, 0, 8, call);                     \
  } while (0)

void act_launch(const ActCall& C, hipStream_t stream) {
  const Shape s = shape_of(C.out.n);
  const dim3 grid = row_grid(C.m, s);
  EP_ROW_LAUNCHES(act_kernel, C);
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }
bool wide_type(int t) { return t == EP_BF16 || t == EP_FP16 || t == EP_FP32; }
bool off_row(int64_t row, int64_t n, int t) { return row < n || row % (t == EP_FP32 ? 4 : t == EP_BF16 || t == EP_FP16 ? 8 : 16); }

// The distance of rows or vectors that are apart at all, in bytes, stays far from 2^63.
constexpr int64_t kMostLd = (int64_t)1 << 40, kMostRows = 0x7FFFFFFF;

}  // namespace
}  // namespace ep

extern "C" int ep_quant_i8_row(const void* d_x, int x_dtype, int64_t m, int64_t k, int64_t x_row, int8_t* d_q,
                               float* d_scale, void* hip_stream) {
  using namespace ep;
  if (m < 0 || m > kMostRows || k <= 0 || k > kMostRow || k % 16)
    return fail(EP_ERR_ARG, "ep_quant_i8_row: need 0 <= m < 2^31, 0 < k <= 65536 and k % 16 == 0");
  if (!wide_type(x_dtype)) return fail(EP_ERR_ARG, "ep_quant_i8_row: x_dtype must be BF16, FP16 or FP32");
  if (x_row > kMostLd || off_row(x_row, k, x_dtype))
    return fail(EP_ERR_ARG, "ep_quant_i8_row: rows of x must hold k elements and be 16-byte aligned");
  if (m == 0) return EP_OK;
  if (!d_x || !d_q || !d_scale) return fail(EP_ERR_ARG, "ep_quant_i8_row: null pointer");
  if (misaligned(d_x) || misaligned(d_q) || reinterpret_cast<uintptr_t>(d_scale) & 3)
    return fail(EP_ERR_ARG, "ep_quant_i8_row: x and q must be 16-byte aligned, scale by its elements");
  const ActCall C = {d_x, nullptr, m, x_row, 0, x_dtype, kActNone, {d_q, d_scale, k, EP_INT8, (uint32_t)k}};
  act_launch(C, static_cast<hipStream_t>(hip_stream));
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_quant_i8_row: launch failed");
  return EP_OK;
}

extern "C" int ep_glu(const void* d_a, const void* d_b, int x_dtype, int64_t m, int64_t n, int64_t a_row,
                      int64_t b_row, int act, void* d_y, int y_dtype, float* d_y_scale, void* hip_stream) {
  using namespace ep;
  const bool codes = y_dtype == EP_FP8_E4M3 || y_dtype == EP_INT8;
  if (!wide_type(x_dtype)) return fail(EP_ERR_ARG, "ep_glu: x_dtype must be BF16, FP16 or FP32");
  if (!wide_type(y_dtype) && !codes) return fail(EP_ERR_ARG, "ep_glu: y_dtype must be BF16, FP16, FP32, FP8_E4M3 or INT8");
  if (act < EP_ACT_SILU || act > EP_ACT_GELU_TANH) return fail(EP_ERR_ARG, "ep_glu: unknown activation");
  if (m < 0 || m > kMostRows || n <= 0 || n > kMostRow || n % (codes ? 16 : 8))
    return fail(EP_ERR_ARG, "ep_glu: need 0 <= m < 2^31, 0 < n <= 65536, n % 8 == 0, and n % 16 == 0 for an 8-bit y");
  if (a_row > kMostLd || off_row(a_row, n, x_dtype) || (d_b && (b_row > kMostLd || off_row(b_row, n, x_dtype))))
    return fail(EP_ERR_ARG, "ep_glu: rows of a and b must hold n elements and be 16-byte aligned");
  if (m == 0) return EP_OK;
  if (!d_a || !d_y || (codes && !d_y_scale)) return fail(EP_ERR_ARG, "ep_glu: null pointer");
  if (misaligned(d_a) || misaligned(d_b) || misaligned(d_y) || (codes && reinterpret_cast<uintptr_t>(d_y_scale) & 3))
    return fail(EP_ERR_ARG, "ep_glu: a, b and y must be 16-byte aligned, scales by their elements");
  const ActCall C = {d_a, d_b, m, a_row, b_row, x_dtype, act, {d_y, d_y_scale, n, y_dtype, (uint32_t)n}};
  act_launch(C, static_cast<hipStream_t>(hip_stream));
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_glu: launch failed");
  return EP_OK;
}

extern "C" int ep_norm(const ep_norm_call* call, void* hip_stream) {
  using namespace ep;
  if (!call) return fail(EP_ERR_ARG, "ep_norm: null call");
  ep_norm_call C = *call;
  const bool codes = C.y_dtype == EP_FP8_E4M3 || C.y_dtype == EP_INT8, normed = C.pre != EP_NORM_NONE;
  if (C.post < EP_NORM_NONE || C.post > EP_NORM_LAYER || C.pre < EP_NORM_NONE || C.pre > EP_NORM_LAYER)
    return fail(EP_ERR_ARG, "ep_norm: unknown kind of norm");
  if (!wide_type(C.x_dtype) || ((C.d_res || C.d_res_out) && !wide_type(C.res_dtype)))
    return fail(EP_ERR_ARG, "ep_norm: x_dtype and res_dtype must be BF16, FP16 or FP32");
  const bool vectors = C.d_post_w || C.d_post_b || C.d_gate || C.d_w || C.d_b;
  if (vectors && !wide_type(C.w_dtype)) return fail(EP_ERR_ARG, "ep_norm: w_dtype must be BF16, FP16 or FP32");
  if (normed && !wide_type(C.y_dtype) && !codes)
    return fail(EP_ERR_ARG, "ep_norm: y_dtype must be BF16, FP16, FP32, FP8_E4M3 or INT8");
  if (C.m < 0 || C.m > kMostRows || C.n <= 0 || C.n > kMostRow || C.n % (normed && codes ? 16 : 8))
    return fail(EP_ERR_ARG, "ep_norm: need 0 <= m < 2^31, 0 < n <= 65536, n % 8 == 0, and n % 16 == 0 for an 8-bit y");
  if (!(C.eps > 0.0f) || !std::isfinite(C.eps) || !std::isfinite(C.alpha))
    return fail(EP_ERR_ARG, "ep_norm: eps must be above 0, alpha and eps finite");
  for (int64_t* p : {&C.x_row, &C.res_row, &C.res_out_row, &C.y_row})
    if (*p == 0) *p = C.n;
  if (C.x_row > kMostLd || off_row(C.x_row, C.n, C.x_dtype) ||
      (C.d_res && (C.res_row > kMostLd || off_row(C.res_row, C.n, C.res_dtype))) ||
      (C.d_res_out && (C.res_out_row > kMostLd || off_row(C.res_out_row, C.n, C.res_dtype))) ||
      (normed && (C.y_row > kMostLd || off_row(C.y_row, C.n, C.y_dtype))))
    return fail(EP_ERR_ARG, "ep_norm: rows must hold n elements and be 16-byte aligned");
  if (C.group_rows < 0 || C.gate_ld < 0 || C.w_ld < 0 || C.b_ld < 0 || C.gate_ld > kMostLd || C.w_ld > kMostLd || C.b_ld > kMostLd)
    return fail(EP_ERR_ARG, "ep_norm: negative group size or distance");
  if (vectors && (C.gate_ld | C.w_ld | C.b_ld) % (C.w_dtype == EP_FP32 ? 4 : 8))
    return fail(EP_ERR_ARG, "ep_norm: vectors of groups must be 16-byte aligned");
  if (C.m == 0) return EP_OK;
  if (!C.d_x || (normed && (!C.d_y || (codes && !C.d_y_scale)))) return fail(EP_ERR_ARG, "ep_norm: null pointer");
  if (!normed && !C.d_res_out) return fail(EP_ERR_ARG, "ep_norm: nothing to write");
  if (C.d_res && C.d_res == C.d_res_out && C.res_row != C.res_out_row)
    return fail(EP_ERR_ARG, "ep_norm: a residual stream in place needs one distance of rows");
  for (const void* p : {C.d_x, C.d_res, static_cast<const void*>(C.d_res_out), static_cast<const void*>(C.d_y), C.d_post_w, C.d_post_b,
                        C.d_gate, C.d_w, C.d_b})
    if (misaligned(p)) return fail(EP_ERR_ARG, "ep_norm: rows and vectors must be 16-byte aligned");
  if (normed && codes && reinterpret_cast<uintptr_t>(C.d_y_scale) & 3)
    return fail(EP_ERR_ARG, "ep_norm: scales must be aligned by their elements");
  const Shape s = shape_of(C.n);
  const dim3 grid = row_grid(C.m, s);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  EP_ROW_LAUNCHES(norm_kernel, C);
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_norm: launch failed");
  return EP_OK;
}

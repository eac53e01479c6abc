// Operators on rows between a layer's products: norms with the residual sum and its gate, the
// gated activation, and the INT8 quantiser.  A row is read once, held in registers as FP32 while
// its statistics are summed, and written once, rounded or quantised for the next product.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

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

// ---- rows of a type that is known at run time ----------------------------------------------
// V vectors of eight elements from places `at`, `at` + step, ... of a row of `vecs` of them, as they lie
// in memory.  All loads go out before the first value is needed: those past the row's end read its
// last vector, and are not waited for one by one.  A 16-bit vector takes four registers until it is
// widened.
template <int V>
struct RawRow {
  v4u lo[V], hi[V];   // hi: FP32 only
  __device__ __forceinline__ void load(const void* row, int dtype, uint32_t at, uint32_t step, uint32_t vecs) {
    if (dtype == EP_FP32) {
#pragma unroll
      for (int j = 0; j < V; j++) {
        const v4u* const p = static_cast<const v4u*>(row) + 2 * (size_t)min(at + j * step, vecs - 1);
        lo[j] = p[0];
        hi[j] = p[1];
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; j++) {
        lo[j] = static_cast<const v4u*>(row)[min(at + j * step, vecs - 1)];
        hi[j] = v4u{};
      }
    }
  }
  // Vector j as floats, 0 past the row's end.
  __device__ __forceinline__ void get(int j, int dtype, uint32_t at, uint32_t step, uint32_t vecs, float (&v)[8]) const {
    if (dtype == EP_BF16) {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        v[2 * i] = __uint_as_float(lo[j][i] << 16);
        v[2 * i + 1] = __uint_as_float(lo[j][i] & 0xFFFF0000u);
      }
    } else if (dtype == EP_FP16) {
      const v8h h = __builtin_bit_cast(v8h, lo[j]);
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = (float)h[i];
    } else {
#pragma unroll
      for (int i = 0; i < 4; i++) {
        v[i] = __uint_as_float(lo[j][i]);
        v[4 + i] = __uint_as_float(hi[j][i]);
      }
    }
    if (at + j * step >= vecs) {
#pragma unroll
      for (int i = 0; i < 8; i++) v[i] = 0.0f;
    }
  }
};
template <int V>
__device__ __forceinline__ void load_row(const void* row, int dtype, uint32_t at, uint32_t step, uint32_t vecs, float (&v)[V][8]) {
  const auto of = [&](auto type) {   // the type's branch once for all vectors
    constexpr int G = V > 4 ? 4 : V;
#pragma unroll
    for (int g = 0; g < V; g += G) {
      RawRow<G> raw;
      raw.load(row, type(), at + g * step, step, vecs);
#pragma unroll
      for (int j = 0; j < G; j++) raw.get(j, type(), at + g * step, step, vecs, v[g + j]);
    }
  };
  if (dtype == EP_BF16) of(std::integral_constant<int, EP_BF16>{});
  else if (dtype == EP_FP16) of(std::integral_constant<int, EP_FP16>{});
  else of(std::integral_constant<int, EP_FP32>{});
}
template <int V>
__device__ __forceinline__ void store_row(void* row, int dtype, uint32_t at, uint32_t step, uint32_t vecs, const float (&v)[V][8]) {
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t vec = at + j * step;
    if (vec >= vecs) continue;
    const v8f f = {v[j][0], v[j][1], v[j][2], v[j][3], v[j][4], v[j][5], v[j][6], v[j][7]};
    if (dtype == EP_BF16) {
      static_cast<v8b*>(row)[vec] = __builtin_convertvector(f, v8b);
    } else if (dtype == EP_FP16) {
      static_cast<v8h*>(row)[vec] = __builtin_convertvector(f, v8h);
    } else {
      static_cast<v4f*>(row)[2 * (size_t)vec] = v4f{f[0], f[1], f[2], f[3]};
      static_cast<v4f*>(row)[2 * (size_t)vec + 1] = v4f{f[4], f[5], f[6], f[7]};
    }
  }
}
// The row that lies `row` rows of `ld` elements of a type after p.
__device__ __forceinline__ const void* row_at(const void* p, int dtype, int64_t row, int64_t ld) {
  return static_cast<const uint8_t*>(p) + row * ld * (dtype == EP_FP32 ? 4 : 2);
}
__device__ __forceinline__ void* row_at(void* p, int dtype, int64_t row, int64_t ld) {
  return static_cast<uint8_t*>(p) + row * ld * (dtype == EP_FP32 ? 4 : 2);
}

// INT8 round(x / s) of eight values, halves to even: added to 1.5 2^23 a quotient of at most 127 (and a
// rounding) is rounded to a whole number, whose low eight bits are the code.
__device__ __forceinline__ v2u codes8_i8(const float (&v)[8], const Divider& by) {
  v2u out;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    uint32_t q[4];
#pragma unroll
    for (int j = 0; j < 4; j++) q[j] = __float_as_uint(by(v[4 * i + j]) + 12582912.0f);
    const uint32_t lo = __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), hi = __builtin_amdgcn_perm(q[3], q[2], 0x04000C0Cu);
    out[i] = lo | hi;
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
// The reduction over 16 lanes in every one of them: each adds what the lanes 8, 4, 2 and 1 after it
// hold, by moves inside the vector unit.
template <int N, typename T>
__device__ __forceinline__ T rotated(T x) {
  const int v = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(v, v, 0x120 + N, 0xF, 0xF, false));
}
template <typename T, typename F>
__device__ __forceinline__ T all16(T x, F f) {
  x = f(x, rotated<8>(x));
  x = f(x, rotated<4>(x));
  x = f(x, rotated<2>(x));
  return f(x, rotated<1>(x));
}
template <typename T>
__device__ __forceinline__ T lane_of(T x, int lane) {
  return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane));
}

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
    x = all16(x, f);
    if (L == 16) return x;
    if (L == 32) return f(x, __builtin_bit_cast(T, __shfl_xor(__builtin_bit_cast(int, x), 16)));
    x = f(f(lane_of(x, 0), lane_of(x, 16)), f(lane_of(x, 32), lane_of(x, 48)));
    if (L) return x;
    uint32_t* const slot = lds + 16 * turn;
    turn ^= 1;
    if (threadIdx.x % 64 == 0) slot[threadIdx.x / 64] = __builtin_bit_cast(uint32_t, x);
    __syncthreads();
    // a lane for each wave's; 0 is neutral to both reductions
    const uint32_t w = threadIdx.x % 16;
    return all16(__builtin_bit_cast(T, w < blockDim.x / 64 ? slot[w] : 0u), f);
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
          for (int i = 0; i < 8; i++) v[j][i] = row.at() + j * row.lanes() < vecs ? v[j][i] - mean : 0.0f;
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
  if (dtype != EP_INT8 && dtype != EP_FP8_E4M3) {
    store_row<V>(y, dtype, row.at(), row.lanes(), vecs, v);
    return;
  }
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
  for (int j = 0; j < V; j++) {   // sixteen lanes hold a block of 128
    const uint32_t vec = row.at() + j * row.lanes();
    const float s = scale_of(all16(top_bits(v[j]), Top{}), kE4m3Max);
    if (vec < vecs) {
      static_cast<v2u*>(y)[vec] = codes8(v[j], Divider(s, kE4m3Max));
      if (vec % 16 == 0) scale[vec / 16] = s;
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

// v = f(v), and v = f(v, row), a few vectors of the row at a time; past its end the row is 0.
template <int V, typename F>
__device__ __forceinline__ void each(F f, float (&v)[V][8]) {
#pragma unroll
  for (int j = 0; j < V; j++)
#pragma unroll
    for (int i = 0; i < 8; i++) v[j][i] = f(v[j][i]);
}
template <int V, typename F>
__device__ __forceinline__ void with_row(F f, const void* row, int dtype, uint32_t at, uint32_t step, uint32_t vecs, float (&v)[V][8]) {
  constexpr int G = V > 4 ? 2 : V;
#pragma unroll
  for (int g = 0; g < V; g += G) {
    float t[G][8];
    load_row<G>(row, dtype, at + g * step, step, vecs, t);
#pragma unroll
    for (int j = 0; j < G; j++)
      if (g + j < V) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[g + j][i] = f(v[g + j][i], t[j][i]);
      }
  }
}

// ---- norm ----------------------------------------------------------------------------------
// h = res + alpha gate N_post(x) and y = N_pre(h) of a row, one pass over memory: the row stays in registers
// as FP32 from its loads to its stores, and each norm sums it once or twice (the mean first, so that no
// digits of a row far from zero are lost) in lanes, then over waves through LDS.  Bound by memory:
// 8192 x 5120 of BF16 with both norms and the residual stream in 64 us, 5.3 TB/s of reads and writes; 8222 x
// 3840 gated, with an FP32 stream, in 74 us, 5.1 TB/s.  One row takes 4.3 us, a chain of loads and
// reductions: with all loads sent before the first reduction it is 4.3 as well, and 8192 rows take 78.
// Rows of more than 32768 hold 64 values a thread, which leaves one workgroup on a CU and spills a few of
// them: 2.5 TB/s.
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

  const uint32_t at = row.at(), step = row.lanes();
  float v[V][8];
  load_row<V>(x, C.x_dtype, at, step, vecs, v);
  if (C.post != EP_NORM_NONE) {
    const float r = normed<L, V>(row, v, C.post, vecs, n, C.eps);
    each<V>([&](float a) { return a * r; }, v);
    if (C.d_post_w) with_row<V>([](float a, float f) { return a * f; }, C.d_post_w, C.w_dtype, at, step, vecs, v);
    if (C.d_post_b) with_row<V>([](float a, float f) { return a + f; }, C.d_post_b, C.w_dtype, at, step, vecs, v);
  }
  if (gate) with_row<V>([](float a, float f) { return a * f; }, gate, C.w_dtype, at, step, vecs, v);
  const float alpha = C.alpha;
  if (res) with_row<V>([=](float a, float f) { return __builtin_fmaf(alpha, a, f); }, res, C.res_dtype, at, step, vecs, v);
  else each<V>([=](float a) { return alpha * a; }, v);
  if (C.d_res_out) store_row<V>(row_at(C.d_res_out, C.res_dtype, i, C.res_out_row), C.res_dtype, at, step, vecs, v);
  if (C.pre == EP_NORM_NONE) return;
  const float r = normed<L, V>(row, v, C.pre, vecs, n, C.eps);
  each<V>([=](float a) { return a * r; }, v);
  const float one = C.w_plus_one ? 1.0f : 0.0f;
  if (w) with_row<V>([=](float a, float f) { return a * (f + one); }, w, C.w_dtype, at, step, vecs, v);
  if (b) with_row<V>([](float a, float f) { return a + f; }, b, C.w_dtype, at, step, vecs, v);
  const RowOut out = {C.d_y, C.d_y_scale, C.y_row, C.y_dtype, n};
  write_row<L, V>(row, v, vecs, out.row(i), C.y_dtype, out.scale_row(i));
}

// ---- activation and quantiser -----------------------------------------------------------------
// exp(x) for x <= 0: 2^n 2^f with n the whole number nearest to x log2(e) and f what is left of it, in
// two parts of log2(e) so that no bit of the product is lost; results fall to 0 through the
// subnormal values, and are 0 long before -150.
__device__ __forceinline__ float exp_negative(float x) {
  x = fmaxf(x, -150.0f);
  const float n = rintf(x * 1.44269504f);
  const float f = __builtin_fmaf(x, 1.925963033e-8f, __builtin_fmaf(x, 1.44269502f, -n));
  return __builtin_ldexpf(__builtin_amdgcn_exp2f(f), (int)n);
}
// 1 / d for d from 1 to 2^8, by one step of Newton's on the instruction's, which is within a unit.
__device__ __forceinline__ float reciprocal(float d) {
  const float r = __builtin_amdgcn_rcpf(d);
  return __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r);
}
// a / (1 + exp(-z)), by the exponential that does not overflow.
__device__ __forceinline__ float gated(float a, float z) {
  const float e = exp_negative(-fabsf(z));
  return (z < 0.0f ? a * e : a) * reciprocal(1.0f + e);
}
// a Phi(a) = max(a, 0) - z Phi(-z) with z = |a|, and Phi(-z) = exp(-z^2 / 2) M(z).  M falls smoothly from
// 1/2 to 1 / (z sqrt(2 pi)): t Q(t) with t = 1 / (1 + 0.24 z) and Q of degree 9, fitted for the least
// relative error over 0 .. 14.6, where the exponential ends; with its constants in FP32 it is within 3e-8.  The
// result was within 7.2 2^-24 of itself at 66 thousand values in each of five ranges from -12.9 to 6 (SiLU 3.8); by the
// bounds of the steps it could be 17.9 off.  What z^2 loses when it is rounded moves the exponential by as much.  max(a, 0) takes a negative a times -0: of -inf
// the product is the NaN that the formula's -inf 0 is, where z and h, which are bounded, would make it 0.
__device__ __forceinline__ float gelu(float a) {
  const float z = fminf(fabsf(a), 20.0f), sq = z * z, lost = __builtin_fmaf(z, z, -sq);
  const float e = exp_negative(-0.5f * sq), t = reciprocal(__builtin_fmaf(0.24f, z, 1.0f));
  float q = __builtin_fmaf(0.0255265534f, t, -0.124637879f);
  q = __builtin_fmaf(q, t, 0.205476031f);
  q = __builtin_fmaf(q, t, -0.144257292f);
  q = __builtin_fmaf(q, t, 0.141432092f);
  q = __builtin_fmaf(q, t, 0.028170027f);
  q = __builtin_fmaf(q, t, 0.0877551958f);
  q = __builtin_fmaf(q, t, 0.0889361501f);
  q = __builtin_fmaf(q, t, 0.0958570391f);
  q = __builtin_fmaf(q, t, 0.0957420841f);
  const float h = q * t * __builtin_fmaf(e, -0.5f * lost, e);
  return __builtin_fmaf(-z, h, a < 0.0f ? a * -0.0f : a);
}
// (1 + tanh z) / 2 is 1 / (1 + exp(-2 z))
__device__ __forceinline__ float gelu_tanh(float a) { return gated(a, 1.5957691216057308f * __builtin_fmaf(0.044715f * a * a, a, a)); }


struct ActCall {
  const void* a;
  const void* b;
  int64_t m, a_row, b_row;
  int act;         // 0: none
  RowOut out;
};

__device__ __forceinline__ void activate(int act, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 8; i++) {
    if (act == EP_ACT_SILU) v[i] = gated(v[i], v[i]);
    else if (act == EP_ACT_GELU) v[i] = gelu(v[i]);
    else if (act == EP_ACT_GELU_TANH) v[i] = gelu_tanh(v[i]);
  }
}

// INT8 rows: the whole row is in registers until its largest value is known, so that it crosses the memory
// once.  Bound by memory: 8192 x 17408 of BF16 to codes in 74 us, 5.7 TB/s; with SiLU and the other half in
// 139 us, 5.1 TB/s.  One row of 17408 takes 3.5 us.
template <int L, int V, int TYPE, bool GATED>
__global__ __launch_bounds__(L ? 256 : 1024) void act_rows_kernel(ActCall C) {
  __shared__ uint32_t lds[32];
  RowThreads<L> row(lds);
  const int64_t i = row_of(row.lanes());
  if (i >= C.m) return;
  const uint32_t vecs = C.out.n / 8, at = row.at(), step = row.lanes();
  RawRow<V> a, b;
  a.load(row_at(C.a, TYPE, i, C.a_row), TYPE, at, step, vecs);
  if (GATED) b.load(row_at(C.b, TYPE, i, C.b_row), TYPE, at, step, vecs);
  float v[V][8];
#pragma unroll
  for (int j = 0; j < V; j++) {
    a.get(j, TYPE, at, step, vecs, v[j]);
    activate(C.act, v[j]);
    if (GATED) {
      float f[8];
      b.get(j, TYPE, at, step, vecs, f);
#pragma unroll
      for (int e = 0; e < 8; e++) v[j][e] *= f[e];
    }
  }
  write_row<L, V>(row, v, vecs, C.out.row(i), EP_INT8, C.out.scale_row(i));
}

// Other outputs, where no more than 128 of a row's values belong together: the rows' vectors one after
// the other, each row padded to whole blocks, V of them for a thread.  8192 x 17408 of BF16, gated by SiLU: to
// E4M3 in 136 us, 5.3 TB/s (199 by whole rows), to BF16 in 148 us, 5.8 TB/s.  The vector unit is close behind
// the memory: some 27 operations a value for SiLU and a code, of the 34 that fit beside 5 bytes; with the
// math library's exponential and a division for a reciprocal it was the bound, and GELU's polynomial
// makes it so again (178 us; 212 with the library's function).
constexpr int kFlatThreads = 256;
template <int V, int TYPE, bool GATED>
__global__ __launch_bounds__(kFlatThreads) void act_flat_kernel(ActCall C) {
  const uint32_t vecs = C.out.n / 8, padded = (vecs + 15) / 16 * 16;
  const uint64_t first = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * (V * kFlatThreads);
  const int64_t row0 = (int64_t)(first / padded);
  const uint32_t in0 = (uint32_t)(first - (uint64_t)row0 * padded);
  const float inverse = 1.0f / (float)padded;
  RawRow<1> a[V], b[V];
  int64_t row[V];
  uint32_t vec[V];
#pragma unroll
  for (int j = 0; j < V; j++) {
    const uint32_t x = in0 + threadIdx.x + j * kFlatThreads;
    const uint32_t r = (uint32_t)(((float)x + 0.5f) * inverse);   // x / padded: x is below 2^17, so that half a unit outweighs both roundings
    row[j] = row0 + r;
    vec[j] = x - r * padded;
    const int64_t i = min(row[j], C.m - 1);   // past the end the last row is read for nothing
    a[j].load(row_at(C.a, TYPE, i, C.a_row), TYPE, vec[j], 16, vecs);
    if (GATED) b[j].load(row_at(C.b, TYPE, i, C.b_row), TYPE, vec[j], 16, vecs);
  }
#pragma unroll
  for (int j = 0; j < V; j++) {
    float v[1][8];
    a[j].get(0, TYPE, vec[j], 16, vecs, v[0]);
    activate(C.act, v[0]);
    if (GATED) {
      float f[8];
      b[j].get(0, TYPE, vec[j], 16, vecs, f);
#pragma unroll
      for (int e = 0; e < 8; e++) v[0][e] *= f[e];
    }
    const bool mine = row[j] < C.m && vec[j] < vecs;
    if (C.out.dtype == EP_FP8_E4M3) {
      const float s = scale_of(all16(top_bits(v[0]), Top{}), kE4m3Max);
      if (mine) {
        static_cast<v2u*>(C.out.row(row[j]))[vec[j]] = codes8(v[0], Divider(s, kE4m3Max));
        if (vec[j] % 16 == 0) C.out.scale_row(row[j])[vec[j] / 16] = s;
      }
    } else if (mine) {
      store_row<1>(C.out.row(row[j]), C.out.dtype, vec[j], 16, vecs, v);
    }
  }
}

// ---- launches --------------------------------------------------------------------------------
struct Shape {
  int lanes, vectors;   // of a row; lanes 0: a workgroup of `threads`
  int threads;
};
// Two vectors a thread where a row has enough of them: one leaves each thread too little in flight
// (8192 x 5120 with both norms in 94 us, 64 with two, 64 and 65 with four and three), and eight leave
// too few threads on a CU; longer rows take three (8192 x 17408 to INT8 in 75 us, 86 with four) and
// more only where 1024 threads do not hold them else.
Shape shape_of(int64_t n) {
  const int64_t vecs = n / 8;
  if (vecs <= 16) return {16, 1, 256};
  if (vecs <= 32) return {32, 1, 256};
  if (vecs <= 64) return {64, 1, 256};
  const int v = vecs <= 2048 ? 2 : vecs <= 3072 ? 3 : vecs <= 4096 ? 4 : 8;
  return {0, v, (int)(((vecs + v - 1) / v + 63) / 64 * 64)};
}
// Workgroups in one or more rows of a grid, whose x dimension holds fewer than 2^32 threads.
dim3 row_grid(int64_t m, const Shape& s) {
  const int64_t per = s.lanes ? s.threads / s.lanes : 1, groups = (m + per - 1) / per;
  const int64_t x = std::min<int64_t>(groups, 1 << 21);
  return dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x));
}

// f<L, V>() for the row's shape.
template <typename F>
void by_shape(const Shape& s, F f) {
  using std::integral_constant;
#define EP_SHAPE_CASE(L, V) \
  if (s.lanes == L && s.vectors == V) return f(integral_constant<int, L>{}, integral_constant<int, V>{})
  EP_SHAPE_CASE(16, 1);
  EP_SHAPE_CASE(32, 1);
  EP_SHAPE_CASE(64, 1);
  EP_SHAPE_CASE(0, 2);
  EP_SHAPE_CASE(0, 3);
  EP_SHAPE_CASE(0, 4);
  EP_SHAPE_CASE(0, 8);
#undef EP_SHAPE_CASE
}

template <int TYPE, bool GATED>
void act_launch(const ActCall& C, hipStream_t stream) {
  if (C.out.dtype == EP_INT8) {
    const Shape s = shape_of(C.out.n);
    by_shape(s, [&](auto l, auto v) {
      hipLaunchKernelGGL((act_rows_kernel<l(), v(), TYPE, GATED>), row_grid(C.m, s), dim3(s.threads), 0, stream, C);
    });
    return;
  }
  constexpr int kVectors = 2;
  const int64_t vectors = C.m * ((C.out.n + 127) / 128 * 16), groups = (vectors + kVectors * kFlatThreads - 1) / (kVectors * kFlatThreads);
  const int64_t x = std::min<int64_t>(groups, 1 << 23);
  hipLaunchKernelGGL((act_flat_kernel<kVectors, TYPE, GATED>), dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x)), dim3(kFlatThreads), 0,
                     stream, C);
}
template <bool GATED>
void act_launch(const ActCall& C, int x_dtype, hipStream_t stream) {
  if (x_dtype == EP_BF16) act_launch<EP_BF16, GATED>(C, stream);
  else if (x_dtype == EP_FP16) act_launch<EP_FP16, GATED>(C, stream);
  else act_launch<EP_FP32, GATED>(C, stream);
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }
bool wide_type(int t) { return t == EP_BF16 || t == EP_FP16 || t == EP_FP32; }
bool off_row(int64_t row, int64_t n, int t) { return row < n || row % (t == EP_FP32 ? 4 : t == EP_BF16 || t == EP_FP16 ? 8 : 16); }

int64_t size_of(int t) { return t == EP_FP32 ? 4 : t == EP_BF16 || t == EP_FP16 ? 2 : 1; }
// Rows of an output of a call, or of an input.
struct Rows {
  const void* p;
  int type;
  int64_t row;   // elements from one to the next
};
// Whether an output at an input's address would be written over values that are still to be read: those
// of another row, where the rows' distances in bytes differ, or of the same row by another thread, where
// the types' sizes differ and a row is not read as a whole before any of it is written.
bool clash(const Rows& out, const Rows& in, int64_t m, bool whole_first) {
  if (!out.p || out.p != in.p) return false;
  const int64_t a = size_of(out.type), b = size_of(in.type);
  return (m > 1 && out.row * a != in.row * b) || (!whole_first && a != b);
}

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
  if (clash({d_q, EP_INT8, k}, {d_x, x_dtype, x_row}, m, true)) return fail(EP_ERR_ARG, "ep_quant_i8_row: q at x, whose rows lie otherwise");
  const ActCall C = {d_x, nullptr, m, x_row, 0, 0, {d_q, d_scale, k, EP_INT8, (uint32_t)k}};
  act_launch<false>(C, x_dtype, static_cast<hipStream_t>(hip_stream));
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
  const Rows y = {d_y, y_dtype, n};
  const bool whole = y_dtype == EP_INT8;
  if (clash(y, {d_a, x_dtype, a_row}, m, whole) || clash(y, {d_b, x_dtype, b_row}, m, whole))
    return fail(EP_ERR_ARG, "ep_glu: y at a or b, whose rows lie otherwise");
  const ActCall C = {d_a, d_b, m, a_row, b_row, act, {d_y, d_y_scale, n, y_dtype, (uint32_t)n}};
  if (d_b) act_launch<true>(C, x_dtype, static_cast<hipStream_t>(hip_stream));
  else act_launch<false>(C, x_dtype, static_cast<hipStream_t>(hip_stream));
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
  const Rows h = {C.d_res_out, C.res_dtype, C.res_out_row}, y = {normed ? C.d_y : nullptr, C.y_dtype, C.y_row};
  for (const Rows& in : {Rows{C.d_x, C.x_dtype, C.x_row}, Rows{C.d_res, C.res_dtype, C.res_row}})
    if (clash(h, in, C.m, false) || clash(y, in, C.m, true)) return fail(EP_ERR_ARG, "ep_norm: an output at an input whose rows lie otherwise");
  if (y.p && y.p == h.p) return fail(EP_ERR_ARG, "ep_norm: y and the new stream in one place");
  const Shape s = shape_of(C.n);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  by_shape(s, [&](auto l, auto v) { hipLaunchKernelGGL((norm_kernel<l(), v()>), row_grid(C.m, s), dim3(s.threads), 0, stream, C); });
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_norm: launch failed");
  return EP_OK;
}

// FP8 with a scale for each block of 128: the quantiser of activations (and weights), and the
// product Y = X W^T that reads its output next to FP8 weights, such as an entropy-coded FP8
// container decodes to.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"
#include "scaled.h"
#include "tile_order.h"

namespace ep {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v4b __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kE4m3Max = 448.0f;

// ---- element types -------------------------------------------------------------
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
  const float s = __uint_as_float(top) * (1.0f / kE4m3Max);
  return s == 0.0f ? 1.0f : s;
}

// E4M3(x / s) of eight values.
__device__ __forceinline__ v2u codes8(const float (&v)[8], const Divider& by) {
  v2u out;
#pragma unroll
  for (int i = 0; i < 2; i++) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(by(v[4 * i]), by(v[4 * i + 1]), 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(by(v[4 * i + 2]), by(v[4 * i + 3]), w, true);
    out[i] = (uint32_t)w;
  }
  return out;
}

constexpr int kQuantThreads = 256;
constexpr int kLanes = 16;                 // lanes on one 128-column block, eight columns each

// Workgroups in one or more rows of a grid, whose x dimension holds fewer than 2^32 threads.
dim3 quant_grid(int64_t groups) {
  const int64_t x = std::min<int64_t>(groups, 1 << 22);
  return dim3((uint32_t)x, (uint32_t)((groups + x - 1) / x));
}
__device__ __forceinline__ uint32_t quant_group() { return blockIdx.y * gridDim.x + blockIdx.x; }

// One row's block of 128 for each 16 lanes: a wave reads four blocks of a row in one load of up to
// 32 bytes a lane and keeps them in registers until the codes are made, so that X crosses the memory
// once.  Bound by memory: 8192 x 17408 of BF16 in 80 us, 5.3 TB/s of reads and writes; a row of
// 5120 takes 2.2 us, which is the launch.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quant_rows_kernel(const T* __restrict__ x,
                                                                   uint8_t* __restrict__ q,
                                                                   float* __restrict__ scale,
                                                                   uint32_t units, uint32_t kb,
                                                                   int64_t k, int64_t x_row) {
  const uint32_t unit = quant_group() * (kQuantThreads / kLanes) + threadIdx.x / kLanes;   // below 2^32
  if (unit >= units) return;
  const uint32_t row = unit / kb, col = (unit - row * kb) * 128 + 8 * (threadIdx.x % kLanes);
  float v[8] = {};
  if (col < k) load8(x + row * x_row + col, v);
  uint32_t top = top_bits(v);
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const float s = scale_of(top);
  if (col < k) *reinterpret_cast<v2u*>(q + row * k + col) = codes8(v, Divider(s, kE4m3Max));
  if (threadIdx.x % kLanes == 0) scale[unit] = s;
}

// One 128 x 128 block for each workgroup, in registers between the maximum and the codes.  Bound by
// memory: 17408 x 5120 of BF16 in 52 us, 5.1 TB/s.
template <typename T>
__global__ __launch_bounds__(kQuantThreads) void quant_blocks_kernel(const T* __restrict__ x,
                                                                     uint8_t* __restrict__ q,
                                                                     float* __restrict__ scale,
                                                                     uint32_t blocks, uint32_t kb, int64_t m,
                                                                     int64_t k, int64_t x_row) {
  constexpr int kRows = kQuantThreads / kLanes, kPasses = 128 / kRows;
  __shared__ uint32_t wave_top[kQuantThreads / 64];
  const uint32_t block = quant_group();
  if (block >= blocks) return;
  const uint32_t bi = block / kb, col = (block - bi * kb) * 128 + 8 * (threadIdx.x % kLanes);
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
  const Divider by(s, kE4m3Max);
#pragma unroll
  for (int p = 0; p < kPasses; p++)
    if (col < k && r0 + kRows * p < m)
      *reinterpret_cast<v2u*>(q + (r0 + kRows * p) * k + col) = codes8(v[p], by);
  if (threadIdx.x == 0) scale[block] = s;
}

template <typename T>
void quant_launch(const void* x, uint8_t* q, float* scale, int64_t m, int64_t k, int64_t x_row,
                  int block_rows, uint32_t kb, hipStream_t stream) {
  if (block_rows == 1) {
    const uint32_t units = (uint32_t)(m * kb), per = kQuantThreads / kLanes;
    hipLaunchKernelGGL(quant_rows_kernel<T>, quant_grid(((int64_t)units + per - 1) / per), dim3(kQuantThreads), 0, stream,
                       static_cast<const T*>(x), q, scale, units, kb, k, x_row);
  } else {
    const int64_t blocks = (m + 127) / 128 * kb;
    hipLaunchKernelGGL(quant_blocks_kernel<T>, quant_grid(blocks), dim3(kQuantThreads), 0, stream,
                       static_cast<const T*>(x), q, scale, (uint32_t)blocks, kb, m, k, x_row);
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
  uint32_t wide;       // four values of a row of Y from a multiple of four on lie aligned as one store's
};

// Y's element types: ep_dtype codes as template arguments.
template <int OUT>
__device__ __forceinline__ void store_y(void* y, int64_t at, float f) {
  if (OUT == EP_FP32) static_cast<float*>(y)[at] = f;
  else if (OUT == EP_FP16) static_cast<_Float16*>(y)[at] = (_Float16)f;
  else static_cast<__bf16*>(y)[at] = (__bf16)f;
}

// Four values of row i from column j, a multiple of four, on; in one store where it is aligned.
template <int OUT>
__device__ __forceinline__ void store_y4(const Product& P, int64_t i, int64_t j, const v4f& v) {
  const int64_t at = i * P.n + j;
  if (P.wide && j + 4 <= P.n) {
    if (OUT == EP_FP32) {
      *reinterpret_cast<v4f*>(static_cast<float*>(P.y) + at) = v;
    } else if (OUT == EP_FP16) {
      *reinterpret_cast<v4h*>(static_cast<_Float16*>(P.y) + at) = __builtin_convertvector(v, v4h);
    } else {
      *reinterpret_cast<v4b*>(static_cast<__bf16*>(P.y) + at) = __builtin_convertvector(v, v4b);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; r++)
      if (j + r < P.n) store_y<OUT>(P.y, at + r, v[r]);
  }
}

// Workgroup barrier for direct loads: this wave's LDS reads have returned and at most N of its
// direct loads are still in flight, then s_barrier.  The scheduling barriers keep the compiler
// from moving LDS accesses across it.
template <int N>
__device__ __forceinline__ void stage_barrier() {
  static_assert(N >= 0 && N < 64, "vmcnt");
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4));   // vmcnt(N) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// One block of 128 of a 16 x 16 tile.  v_mfma_f32_16x16x128_f8f6f4 multiplies 16 rows of W by 16
// rows of X: lane l supplies 32 bytes of row l mod 16 of both, and gets the products of W rows
// 4 (l / 16) + 0 .. 3 with X row l mod 16.  Which 32 of the block's 128 bytes a quarter of the
// wave supplies does not matter as long as both operands agree: here two pieces of 16, so that
// the four quarters of a load cover 64 bytes of a row.
//
// The FP8 instructions add their products in fewer bits than FP32.  Measured: of every eight
// products, aligned along k, each is cut towards zero to a multiple of 2^-13 of the power of two that
// the largest has by its factors' exponents (a subnormal's being the least normal one); the eight are
// then added, and the groups of eight in FP32.  So a block is off by at most 7 2^-13 of the sum of its
// products' magnitudes, subnormal codes counted as the smallest normal one: 1.4e-5 of its size for
// Gaussian codes (root mean square), below the rounding to BF16 (1.7e-3) or FP16 (2.1e-4), but all of
// it where two large products cancel beside small ones.  16-bit outputs take them, at twice the rate.
// FP32 outputs (EXACT) take FP16 instructions, into which both FP8 types widen without rounding: 8e-8.
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

// ---- product in tiles, operands through LDS --------------------------------------------
typedef __attribute__((address_space(3))) uint8_t lds_u8;

// LDS rows of 128 bytes: chunk j (16 bytes) of row r lies at place j ^ swz(r).  A 16-byte read is
// served to 16 lanes at a time, of the first 32 lanes 0-3, 12-15 and 20-27 together and then the
// others (measured), and is free of conflicts if they meet 16 different columns of a 256-byte bank
// row.  Where lane l reads chunk q + l / 16 of row l mod 16, rows 0-3 and 12-15 are read at one
// chunk together with rows 4-11 at the next: with r / 2 as the key, their eight places in either
// half of the bank row are different.
__device__ __forceinline__ uint32_t swz(uint32_t r) { return (r >> 1) & 7; }

constexpr uint32_t kOutside = 0x80000000u;   // past the end of every buffer below (2^30 bytes at most), also with a row's offset added

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_of(const void* p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}

// Few rows of X.  A workgroup owns `height` <= 16 NW rows of W and 16 NX rows of X; its KW waves
// take blocks of 128 along k in turn, each through NS stages of LDS of its own, and add their sums
// in the order of the waves at the end.  No wave waits for another before that, and what bounds the
// kernel is what a CU reads, at about 50 GB/s for each whatever the shape of the workgroup: W once by
// as many CUs as there are, and X again for every strip of W, which of 61 rows is 0.56 of a CU's 1.25
// MB.  Taller strips over a share of k would read less of X; they are not built.  (Fragments loaded into
// registers, 16 rows of 64 bytes a load instead of 8 of 128, took 94 us where this takes 28:
// 61 x 5120 x 17408.)  Measured: 1 x 17408 x 5120 in 15.4 us, 5.8 TB/s of W; 61 x 5120 x 17408 with
// FP32 outputs in 30 us, 3.0 TB/s.
template <int WFMT, int OUT, int LAYOUT, int NW, int NX, int KW, int NS>
__global__ __launch_bounds__(64 * KW) void product_ring_kernel(Product P, uint32_t height, uint32_t per_xcd) {
  constexpr bool EXACT = OUT == EP_FP32;
  constexpr int TW = 16 * NW, TX = 16 * NX;
  // scales come as the operands do: a row of X or W for a lane, or (blocks) the one or two blocks of
  // 128 rows that the strip lies in
  constexpr int kXScaleLoads = (TX + 63) / 64,
                kWScaleLoads = LAYOUT == EP_SCALE_ROW ? 0 : LAYOUT == EP_SCALE_BLOCK ? 1 : (TW + 63) / 64;
  constexpr int kPerStep = (TW + TX) / 8 + kXScaleLoads + kWScaleLoads;
  constexpr int kScales = (TW + TX) * 128, kStage = kScales + 256 * (kXScaleLoads + kWScaleLoads);
  constexpr int kTiles = NW * NX;
  constexpr int kLds = NS * kStage * KW > KW * kTiles * 1024 ? NS * kStage * KW : KW * kTiles * 1024;
  static_assert(kLds <= 160 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[kLds];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  lds_u8* const lds = (lds_u8*)lds_mem + NS * kStage * wave;
  const uint32_t xcd = blockIdx.x % kXcds, turn = blockIdx.x / kXcds;
  const int64_t j0 = (int64_t)(turn % per_xcd * kXcds + xcd) * height, i0 = (int64_t)(turn / per_xcd) * TX;
  if (j0 >= P.n) return;
  const int64_t rows_x = min(P.m - i0, (int64_t)TX), rows_w = min(P.n - j0, (int64_t)height);
  const uint32_t k = (uint32_t)P.k, kb = P.kb;
  const __amdgpu_buffer_rsrc_t rx = rsrc_of(P.x + i0 * P.k, rows_x * P.k), rw = rsrc_of(P.w + j0 * P.k, rows_w * P.k);
  const __amdgpu_buffer_rsrc_t rxs = rsrc_of(P.x_scale + i0 * kb, rows_x * kb * 4);
  const int64_t block0 = j0 / 128, blocks = (j0 + rows_w - 1) / 128 - block0 + 1;
  const __amdgpu_buffer_rsrc_t rws = LAYOUT == EP_SCALE_BLOCK ? rsrc_of(P.w_scale + block0 * kb, blocks * kb * 4)
                                                              : rsrc_of(P.w_scale + j0 * kb, LAYOUT == EP_SCALE_ROW ? 0 : rows_w * kb * 4);

  // direct loads: segments of 8 rows, lane l writing chunk (l mod 8) ^ swz(row) of row l / 8
  const uint32_t seg_row = lane >> 3;
  const uint32_t even = 16 * ((lane & 7) ^ swz(seg_row)), odd = 16 * ((lane & 7) ^ swz(seg_row + 8));
  auto fetch = [&](uint32_t b, uint32_t stage) {
    lds_u8* const dst = lds + kStage * stage;
    const uint32_t at[2] = {128 * b + even, 128 * b + odd};
    uint32_t off[2];
#pragma unroll
    for (int h = 0; h < 2; h++) off[h] = b < kb && at[h] < k ? seg_row * k + at[h] : kOutside;
#pragma unroll
    for (int q = 0; q < TX / 8; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, dst + 1024 * q, 16, off[q & 1] + 8 * q * k, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < TW / 8; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, dst + TX * 128 + 1024 * q, 16, off[q & 1] + 8 * q * k, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < kXScaleLoads; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rxs, dst + kScales + 256 * q, 4,
                                               b < kb ? 4 * ((64 * q + lane) * kb + b) : kOutside, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < kWScaleLoads; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rws, dst + kScales + 256 * (kXScaleLoads + q), 4,
                                               b < kb ? 4 * ((64 * q + lane) * kb + b) : kOutside, 0, 0, 0);
  };

  v4f acc[NW][NX];
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) acc[i][t] = v4f{};
  const int first_rows = (int)(128 - j0 % 128);   // of the strip before a multiple of 128
  const uint32_t fs = swz(col), fo0 = 128 * col + 16 * (quarter ^ fs), fo1 = 128 * col + 16 * ((4 + quarter) ^ fs);
  auto fragment = [&](const lds_u8* p) {
    const v4i a = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo0);
    const v4i b = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo1);
    return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  };

#pragma unroll
  for (int s = 0; s < NS - 1; s++) fetch(wave + KW * s, s);
  uint32_t stage = 0;
  for (uint32_t b = wave; b < kb; b += KW) {
    // the stage read last time is free: its reads have returned
    fetch(b + KW * (NS - 1), stage == 0 ? NS - 1 : stage - 1);
    __builtin_amdgcn_sched_barrier(0);
    constexpr int kLater = (NS - 1) * kPerStep;   // loads of the stages after this one
    static_assert(kLater < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((kLater & 15) | ((kLater >> 4) << 14) | (7 << 4) | (15 << 8));   // vmcnt(kLater)
    __builtin_amdgcn_sched_barrier(0);
    const lds_u8* const p = lds + kStage * stage;
    const __attribute__((address_space(3))) float* const sc = (const __attribute__((address_space(3))) float*)(p + kScales);
    v8i xf[NX];
    float xs[NX];
#pragma unroll
    for (int t = 0; t < NX; t++) {
      xf[t] = fragment(p + 2048 * t);
      xs[t] = sc[16 * t + col];
    }
#pragma unroll
    for (int i = 0; i < NW; i++) {
      const v8i wf = fragment(p + TX * 128 + 2048 * i);
      const float wblock = LAYOUT == EP_SCALE_BLOCK ? sc[64 * kXScaleLoads + (16 * i + 4 * quarter < first_rows ? 0 : 1)] : 1.0f;
      v4f ws;
      if (LAYOUT == EP_SCALE_ROW_BLOCK)
        ws = *reinterpret_cast<const __attribute__((address_space(3))) v4f*>(sc + 64 * kXScaleLoads + 16 * i + 4 * quarter);
#pragma unroll
      for (int t = 0; t < NX; t++) {
        const v4f part = block_product<WFMT, EXACT>(wf, xf[t]);
        const float s = LAYOUT == EP_SCALE_BLOCK ? xs[t] * wblock : xs[t];
#pragma unroll
        for (int r = 0; r < 4; r++)
          acc[i][t][r] = __builtin_fmaf(LAYOUT == EP_SCALE_ROW_BLOCK ? part[r] * ws[r] : part[r], s, acc[i][t][r]);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // lgkmcnt(0): this stage is read
    __builtin_amdgcn_sched_barrier(0);
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
  __builtin_amdgcn_s_waitcnt(0);   // direct loads still in flight land before LDS is used again
  __syncthreads();
  v4f* const join = (v4f*)lds_mem;
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) join[(wave * kTiles + NX * i + t) * 64 + lane] = acc[i][t];
  __syncthreads();
  for (int u = wave; u < kTiles; u += KW) {
    v4f v = join[u * 64 + lane];
#pragma unroll
    for (int w = 1; w < KW; w++) v += join[(w * kTiles + u) * 64 + lane];
    const int64_t j = j0 + 16 * (u / NX) + 4 * quarter, row = i0 + 16 * (u % NX) + col;
    if (row >= P.m || j >= j0 + rows_w) continue;
    if (LAYOUT == EP_SCALE_ROW)
#pragma unroll
      for (int r = 0; r < 4; r++) v[r] *= P.w_scale[min(j + r, P.n - 1)];
    store_y4<OUT>(P, row, j, v);
  }
}

// The tile of Y at row i0 of X and j0 of W.  Wave (ww, wx) of WW x WX owns NW x NX tiles of
// 16 x 16; NS stages of operands (and their scales) are in LDS, written by direct loads while the
// stage before is multiplied.  The sum of a block of 128 comes out of the matrix instruction and is
// added to acc with its scale by the vector unit, one multiply-add for 128 products of a lane, which
// runs beside the matrix unit.  The tile of 256 x 256 by eight waves (128 x 64 each)
// reads 24 fragments of LDS for 32 tiles of products; smaller tiles, which read more, are for
// launches that have too few of the large ones to go round.
// Measured: 8192 x 17408 x 5120, scales in blocks, BF16 outputs: 763 us, 1.91 PFLOP/s; the matrix unit
// is busy 43 % of the cycles at 2.1 GHz, which is where power holds the clock.  FP32 outputs: 1284 us.
template <int WFMT, int OUT, int LAYOUT, int NW, int NX, int WW, int WX, int NS>
__device__ __forceinline__ void tile_product(const Product& P, int64_t i0, int64_t j0, lds_u8* lds) {
  constexpr bool EXACT = OUT == EP_FP32;
  constexpr int kWaves = WW * WX, TW = 16 * NW * WW, TX = 16 * NX * WX;
  constexpr int kSegsW = TW / 8 / kWaves, kSegsX = TX / 8 / kWaves;   // 1 KiB loads of a wave and step
  constexpr int kScaleLoads = (TW + TX) / 64;
  constexpr int kPerStep = kSegsW + kSegsX + (kScaleLoads + kWaves - 1) / kWaves;
  constexpr int kStage = (TW + TX) * 128, kScaleStage = (TW + TX) * 4;
  static_assert(TW % (8 * kWaves) == 0 && TX % (8 * kWaves) == 0 && TW % 64 == 0 && TX % 64 == 0, "tile");
  static_assert(LAYOUT != EP_SCALE_BLOCK || 128 % (16 * NW) == 0, "a wave's rows of W lie in one block of 128");
  static_assert(kScaleLoads <= kWaves, "one scale load for each wave");
  lds_u8* const lds_scales = lds + NS * kStage;

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int ww = wave % WW, wx = wave / WW;
  const int64_t rows_x = min(P.m - i0, (int64_t)TX), rows_w = min(P.n - j0, (int64_t)TW);
  const uint32_t k = (uint32_t)P.k, kb = P.kb;
  const __amdgpu_buffer_rsrc_t rx = rsrc_of(P.x + i0 * P.k, rows_x * P.k), rw = rsrc_of(P.w + j0 * P.k, rows_w * P.k);
  const __amdgpu_buffer_rsrc_t rxs = rsrc_of(P.x_scale + i0 * kb, rows_x * kb * 4);
  const __amdgpu_buffer_rsrc_t rws =
      LAYOUT == EP_SCALE_BLOCK ? rsrc_of(P.w_scale + j0 / 128 * kb, (rows_w + 127) / 128 * kb * 4)
                               : rsrc_of(P.w_scale + j0 * kb, LAYOUT == EP_SCALE_ROW ? 0 : rows_w * kb * 4);

  // direct loads: a wave instruction fills one segment of 8 rows; lane l writes the 16 bytes at
  // 16 l, the place of chunk (l mod 8) ^ swz(row) of row l / 8
  const uint32_t seg_row = 8 * wave + (lane >> 3);
  const uint32_t chunk = 16 * ((lane & 7) ^ swz(seg_row & 15));
  static_assert(8 * kWaves % 16 == 0, "rows of a lane's segments share their swizzle");
  const uint32_t scale_at = [&] {   // this lane's scale of a step, in floats from the step's first
    const uint32_t s = 64 * (wave % kScaleLoads) + lane;
    return s < TX ? s * kb : LAYOUT == EP_SCALE_BLOCK ? ((s - TX) >> 7) * kb : (s - TX) * kb;
  }();
  auto fetch = [&](uint32_t b, uint32_t stage) {
    lds_u8* const dst = lds + kStage * stage + 1024 * wave;
    const uint32_t at = 128 * b + chunk;
    const uint32_t off = at < k ? seg_row * k + at : kOutside;
#pragma unroll
    for (int q = 0; q < kSegsX; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, dst + 1024 * kWaves * q, 16, off + 8 * kWaves * q * k, 0, 0, 0);
#pragma unroll
    for (int q = 0; q < kSegsW; q++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rw, dst + TX * 128 + 1024 * kWaves * q, 16, off + 8 * kWaves * q * k, 0, 0, 0);
    const bool of_x = wave % kScaleLoads < TX / 64;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(of_x ? rxs : rws, lds_scales + kScaleStage * stage + 256 * (wave % kScaleLoads), 4,
                                             b < kb ? 4 * (scale_at + b) : kOutside, 0, 0, 0);
  };

  v4f acc[NW][NX];
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) acc[i][t] = v4f{};

  // fragments: row col of a 16-row tile, chunks quarter and 4 + quarter
  const uint32_t fs = swz(col);
  const uint32_t fo0 = 16 * (quarter ^ fs), fo1 = 16 * ((4 + quarter) ^ fs);
  const uint32_t fx = (16 * NX * wx + col) * 128, fw = (TX + 16 * NW * ww + col) * 128;
  auto fragment = [&](const lds_u8* p) {
    const v4i a = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo0);
    const v4i b = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo1);
    return v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  };

#pragma unroll
  for (int s = 0; s < NS - 1; s++) fetch(s, s);
  stage_barrier<(NS - 2) * kPerStep>();
  uint32_t stage = 0;
  for (uint32_t b = 0; b < kb; b++) {
    const lds_u8* const p = lds + kStage * stage;
    const __attribute__((address_space(3))) float* const sc =
        (const __attribute__((address_space(3))) float*)(lds_scales + kScaleStage * stage);
    const uint32_t ahead = stage == 0 ? NS - 1 : stage - 1;
    fetch(b + NS - 1, ahead);
    v8i xf[NX];
    float xs[NX];
#pragma unroll
    for (int t = 0; t < NX; t++) {
      xf[t] = fragment(p + fx + 16 * 128 * t);
      xs[t] = sc[16 * NX * wx + 16 * t + col];
    }
    if (LAYOUT == EP_SCALE_BLOCK) {
      const float ws = sc[TX + 16 * NW * ww];
#pragma unroll
      for (int t = 0; t < NX; t++) xs[t] *= ws;
    }
#pragma unroll
    for (int i = 0; i < NW; i++) {
      const v8i wf = fragment(p + fw + 16 * 128 * i);
      v4f ws;
      if (LAYOUT == EP_SCALE_ROW_BLOCK)
        ws = *reinterpret_cast<const __attribute__((address_space(3))) v4f*>(sc + TX + 16 * NW * ww + 16 * i + 4 * quarter);
#pragma unroll
      for (int t = 0; t < NX; t++) {
        const v4f part = block_product<WFMT, EXACT>(wf, xf[t]);
#pragma unroll
        for (int r = 0; r < 4; r++)
          acc[i][t][r] = __builtin_fmaf(LAYOUT == EP_SCALE_ROW_BLOCK ? part[r] * ws[r] : part[r], xs[t], acc[i][t][r]);
      }
    }
    stage_barrier<(NS - 2) * kPerStep>();
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
  __builtin_amdgcn_s_waitcnt(0);   // direct loads still in flight land before the wave ends

#pragma unroll
  for (int i = 0; i < NW; i++) {
    const int64_t j = j0 + 16 * (NW * ww + i) + 4 * quarter;
    v4f ws = {1.0f, 1.0f, 1.0f, 1.0f};
    if (LAYOUT == EP_SCALE_ROW) {
#pragma unroll
      for (int r = 0; r < 4; r++) ws[r] = P.w_scale[min(j + r, P.n - 1)];
    }
#pragma unroll
    for (int t = 0; t < NX; t++) {
      const int64_t row = i0 + 16 * (NX * wx + t) + col;
      if (row < P.m) store_y4<OUT>(P, row, j, LAYOUT == EP_SCALE_ROW ? acc[i][t] * ws : acc[i][t]);
    }
  }
}

// Workgroups [0, full) take whole tiles; the `split` last tiles are taken as two halves of W's
// rows each by the others, so that a last round of few tiles takes half as long
// (8192 x 17408 x 5120: 765 us for 785).
template <int WFMT, int OUT, int LAYOUT, int NW, int NX, int WW, int WX, int NS>
__global__ __launch_bounds__(64 * WW * WX) void product_tiles_kernel(Product P, uint32_t tw, uint32_t tx,
                                                                     uint32_t full, uint32_t split) {
  constexpr int TW = 16 * NW * WW, TX = 16 * NX * WX;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[NS * (TW + TX) * 132];
  lds_u8* const lds = (lds_u8*)lds_mem;
  uint32_t ti, tj;
  if (blockIdx.x < full) {
    tile_of(xcd_spread(blockIdx.x, full), tx, tw, ti, tj);
    tile_product<WFMT, OUT, LAYOUT, NW, NX, WW, WX, NS>(P, (int64_t)ti * TX, (int64_t)tj * TW, lds);
  } else {
    const uint32_t u = xcd_spread(blockIdx.x - full, 2 * split);
    tile_of(full + u / 2, tx, tw, ti, tj);
    const int64_t j0 = (int64_t)tj * TW + TW / 2 * (u & 1);
    if (j0 < P.n) tile_product<WFMT, OUT, LAYOUT, NW / 2, NX, WW, WX, NS>(P, (int64_t)ti * TX, j0, lds);
  }
}

template <int WFMT, int OUT, int LAYOUT, int NW, int NX, int WW, int WX, int NS>
void tiles_launch(const Product& P, int cus, hipStream_t stream) {
  constexpr int TW = 16 * NW * WW, TX = 16 * NX * WX;
  const uint32_t tx = (uint32_t)((P.m + TX - 1) / TX), tw = (uint32_t)((P.n + TW - 1) / TW);
  const uint32_t tiles = tx * tw, last = tiles % cus, split = 2 * last <= (uint32_t)cus ? last : 0;
  hipLaunchKernelGGL((product_tiles_kernel<WFMT, OUT, LAYOUT, NW, NX, WW, WX, NS>), dim3(tiles + split), dim3(64 * WW * WX),
                     0, stream, P, tw, tx, tiles - split, split);
}

// ---- which kernel -----------------------------------------------------------------------
// Workgroups of a launch, and how many of them a CU takes in all.
int64_t rounds(int64_t groups, int cus) { return (groups + cus - 1) / cus; }

// Rows of W for a workgroup of the streaming kernel: the multiple of 8 up to 16 NW that makes the
// CU with the most work read the fewest rows.
template <int NW, int NX>
uint32_t ring_height(const Product& P, int cus) {
  const int64_t tx = (P.m + 16 * NX - 1) / (16 * NX), rows_x = std::min<int64_t>(P.m, 16 * NX);
  int64_t best = 16 * NW, least = INT64_MAX;
  for (int64_t h = 16 * NW; h >= 8; h -= 8) {
    const int64_t read = rounds((P.n + h - 1) / h * tx, cus) * (h + rows_x);
    if (read < least) {
      least = read;
      best = h;
    }
  }
  return (uint32_t)best;
}

template <int NX>
int64_t ring_groups(const Product& P, uint32_t height) {
  return (P.n + height - 1) / height * ((P.m + 16 * NX - 1) / (16 * NX));
}

template <int WFMT, int OUT, int LAYOUT, int NW, int NX, int KW, int NS>
void ring_launch(const Product& P, uint32_t height, hipStream_t stream) {
  const uint32_t strips = (uint32_t)((P.n + height - 1) / height), tx = (uint32_t)((P.m + 16 * NX - 1) / (16 * NX));
  const uint32_t per_xcd = (strips + kXcds - 1) / kXcds;
  hipLaunchKernelGGL((product_ring_kernel<WFMT, OUT, LAYOUT, NW, NX, KW, NS>), dim3(per_xcd * kXcds * tx), dim3(64 * KW), 0,
                     stream, P, height, per_xcd);
}

// Time of a launch on its busiest CU, in ns: what a step along k takes, and what a workgroup takes
// besides (its first loads, its stores).  Measured with n from 438 to 17408, k from 512 to 17408 and
// m from 64 to 4441, for outputs of 16 bits (FP8 instructions) and FP32 (FP16 instructions).
constexpr int kBesides = 1500;

// Tiles: a CU with half a tile (of W's rows), with one, and with more, for each of them.
struct TileCost {
  int rows_w, rows_x, half, one, each;
};
constexpr TileCost kSmallTile[2] = {{128, 64, 510, 750, 490}, {128, 64, 640, 900, 660}},
                   kMidTile[2] = {{128, 128, 780, 1170, 850}, {128, 128, 900, 1400, 1090}},
                   kLargeTile[2] = {{256, 256, 1310, 1970, 1970}, {256, 256, 2200, 3650, 3650}};

int64_t tile_cost(const TileCost& c, const Product& P, int cus) {
  const int64_t tiles = (P.m + c.rows_x - 1) / c.rows_x * ((P.n + c.rows_w - 1) / c.rows_w);
  const int64_t halves = (2 * tiles + cus - 1) / cus;     // of the busiest CU
  const int64_t step = halves == 1 ? c.half : std::max<int64_t>(c.one, c.each * halves / 2);
  return step * P.kb + kBesides * ((halves + 1) / 2);
}

// Workgroups of the streaming kernel, by rounds of the chip.
int64_t ring_cost(int step, int64_t groups, const Product& P, int cus) {
  return (step * (int64_t)P.kb + kBesides) * rounds(groups, cus);
}

// Up to 16 rows of X the launch is W's stream from memory: 1 x 17408 x 5120 in 15.6 us with four
// waves a workgroup, 18.0 with eight; 1 x 5120 x 17408, which has too few strips for several
// workgroups on a CU, in 27.2 and 16.6.  Beyond, the kernel with the least estimate.  The streaming
// ones read X again for every strip of W, and are left out where X is what there is most of (4441 x
// 438 x 14800: 194 us for the small tile's 88).
template <int WFMT, int OUT, int LAYOUT>
void product_launch(const Product& P, int cus, hipStream_t stream) {
  constexpr bool EXACT = OUT == EP_FP32;
  if (P.m <= 16) {
    const uint32_t h = ring_height<2, 1>(P, cus);
    if (rounds(ring_groups<1>(P, h), cus) > 1) ring_launch<WFMT, OUT, LAYOUT, 2, 1, 4, 2>(P, h, stream);
    else ring_launch<WFMT, OUT, LAYOUT, 2, 1, 8, 2>(P, h, stream);
    return;
  }
  const uint32_t h2 = ring_height<3, 2>(P, cus), h4 = ring_height<3, 4>(P, cus);
  const int64_t never = P.m > 512 ? INT64_MAX : 0;
  const int64_t ring2 = std::max(never, ring_cost(210, ring_groups<2>(P, h2), P, cus)),
                ring4 = std::max(never, ring_cost(EXACT ? 320 : 270, ring_groups<4>(P, h4), P, cus));
  const int64_t small = tile_cost(kSmallTile[EXACT], P, cus), mid = tile_cost(kMidTile[EXACT], P, cus),
                large = tile_cost(kLargeTile[EXACT], P, cus);
  const int64_t least = std::min({ring2, ring4, small, mid, large});
  if (least == large) tiles_launch<WFMT, OUT, LAYOUT, 8, 4, 2, 4, 2>(P, cus, stream);
  else if (least == mid) tiles_launch<WFMT, OUT, LAYOUT, 4, 4, 2, 2, 2>(P, cus, stream);
  else if (least == small) tiles_launch<WFMT, OUT, LAYOUT, 4, 2, 2, 2, 3>(P, cus, stream);
  else if (least == ring4) ring_launch<WFMT, OUT, LAYOUT, 3, 4, 5, 2>(P, h4, stream);
  else ring_launch<WFMT, OUT, LAYOUT, 3, 2, 6, 2>(P, h2, stream);
}

template <int WFMT, int OUT>
void product_launch(const Product& P, int w_scales, int cus, hipStream_t stream) {
  if (w_scales == EP_SCALE_BLOCK) product_launch<WFMT, OUT, EP_SCALE_BLOCK>(P, cus, stream);
  else if (w_scales == EP_SCALE_ROW_BLOCK) product_launch<WFMT, OUT, EP_SCALE_ROW_BLOCK>(P, cus, stream);
  else product_launch<WFMT, OUT, EP_SCALE_ROW>(P, cus, stream);
}

template <int WFMT>
void product_launch(const Product& P, int w_scales, int y_dtype, int cus, hipStream_t stream) {
  if (y_dtype == EP_FP32) product_launch<WFMT, EP_FP32>(P, w_scales, cus, stream);
  else if (y_dtype == EP_FP16) product_launch<WFMT, EP_FP16>(P, w_scales, cus, stream);
  else product_launch<WFMT, EP_BF16>(P, w_scales, cus, stream);
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
  constexpr int64_t kMost = 1 << 24, kMostK = 1 << 22;   // 256 rows of k bytes stay below 2^31
  if (m < 0 || n <= 0 || k <= 0 || k % 16 || m > kMost || n > kMost || k > kMostK)
    return ep::fail(EP_ERR_ARG, "ep_gemm_fp8_block: need m >= 0, n, k > 0, k % 16 == 0, m and n up to 2^24, k to 2^22");
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
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return ep::fail(EP_ERR_HIP, "ep_gemm_fp8_block: no device");
  const uintptr_t quad = y_dtype == EP_FP32 ? 16 : 8;
  const ep::Product P = {static_cast<const uint8_t*>(d_x), d_x_scale, static_cast<const uint8_t*>(d_w), d_w_scale,
                         d_y, m, n, k, (uint32_t)((k + 127) / 128), n % 4 == 0 && reinterpret_cast<uintptr_t>(d_y) % quad == 0};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (w_dtype == EP_FP8_E4M3) ep::product_launch<0>(P, w_scales, y_dtype, cus, stream);
  else ep::product_launch<1>(P, w_scales, y_dtype, cus, stream);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_gemm_fp8_block: launch failed");
  return EP_OK;
}

// INT8 product with a scale for each row of X and of W: Y = xs ws (X W^T) + bias, the sums exact in
// 32-bit integers, for any number of rows of X.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"
#include "product_tiles.h"
#include "tile_order.h"

namespace ep {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

struct Product {
  const uint8_t* x;
  const float* x_scale;
  const uint8_t* w;
  const float* w_scale;
  const float* bias;   // nullable
  void* y;
  int64_t m, n, k;
  uint32_t kb;         // steps of 128 along k
  uint32_t wide;       // four values of a row of Y from a multiple of four on lie aligned as one store's
};

// Scales, bias and the rounding to Y's type of four sums of row i (below m) from column j on.
template <int OUT>
__device__ __forceinline__ void finish(const Product& P, int64_t i, int64_t j, const v4i& sum) {
  const float xs = P.x_scale[i];
  v4f v;
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int64_t c = min(j + r, P.n - 1);
    v[r] = (float)sum[r] * xs * P.w_scale[c];
    if (P.bias) v[r] += P.bias[c];
  }
  store_y4<OUT>(P.y, P.n, P.wide, i, j, v);
}

// A 16 x 16 tile over 128 of k: v_mfma_i32_16x16x64_i8 multiplies 16 rows of W by 16 rows of X, lane l
// supplying 16 bytes of row l mod 16 of both and getting the sums of W rows 4 (l / 16) + 0 .. 3 with
// X row l mod 16.  Which bytes a quarter of the wave supplies does not matter as long as both agree.
struct Fragment {
  v4i a, b;
};
__device__ __forceinline__ v4i tile_step(const Fragment& w, const Fragment& x, v4i acc) {
  acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(w.a, x.a, acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(w.b, x.b, acc, 0, 0, 0);
}

// Few rows of X.  A workgroup owns `height` <= 16 NW rows of W and 16 NX rows of X; its KW waves
// take steps of 128 along k in turn, each through NS stages of LDS of its own, and add their sums
// at the end.  No wave waits for another before that.
template <int OUT, int NW, int NX, int KW, int NS>
__global__ __launch_bounds__(64 * KW) void ring_kernel(Product P, uint32_t height, uint32_t per_xcd) {
  constexpr int TW = 16 * NW, TX = 16 * NX;
  constexpr int kPerStep = (TW + TX) / 8;
  constexpr int kStage = (TW + TX) * 128;
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
  };

  v4i acc[NW][NX];
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) acc[i][t] = v4i{};
  const uint32_t fs = swz(col), fo0 = 128 * col + 16 * (quarter ^ fs), fo1 = 128 * col + 16 * ((4 + quarter) ^ fs);
  auto fragment = [&](const lds_u8* p) {
    return Fragment{*reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo0),
                    *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo1)};
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
    Fragment xf[NX];
#pragma unroll
    for (int t = 0; t < NX; t++) xf[t] = fragment(p + 2048 * t);
#pragma unroll
    for (int i = 0; i < NW; i++) {
      const Fragment wf = fragment(p + TX * 128 + 2048 * i);
#pragma unroll
      for (int t = 0; t < NX; t++) acc[i][t] = tile_step(wf, xf[t], acc[i][t]);
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(15 | (3 << 14) | (7 << 4));   // lgkmcnt(0): this stage is read
    __builtin_amdgcn_sched_barrier(0);
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
  __builtin_amdgcn_s_waitcnt(0);   // direct loads still in flight land before LDS is used again
  __syncthreads();
  v4i* const join = (v4i*)lds_mem;
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) join[(wave * kTiles + NX * i + t) * 64 + lane] = acc[i][t];
  __syncthreads();
  for (int u = wave; u < kTiles; u += KW) {
    v4i v = join[u * 64 + lane];
#pragma unroll
    for (int w = 1; w < KW; w++) v += join[(w * kTiles + u) * 64 + lane];
    const int64_t j = j0 + 16 * (u / NX) + 4 * quarter, row = i0 + 16 * (u % NX) + col;
    if (row >= P.m || j >= j0 + rows_w) continue;
    finish<OUT>(P, row, j, v);
  }
}

// The tile of Y at row i0 of X and j0 of W.  Wave (ww, wx) of WW x WX owns NW x NX tiles of
// 16 x 16; NS stages of operands are in LDS, written by direct loads while the stage before is
// multiplied.
template <int OUT, int NW, int NX, int WW, int WX, int NS>
__device__ __forceinline__ void tile_product(const Product& P, int64_t i0, int64_t j0, lds_u8* lds) {
  constexpr int kWaves = WW * WX, TW = 16 * NW * WW, TX = 16 * NX * WX;
  constexpr int kSegsW = TW / 8 / kWaves, kSegsX = TX / 8 / kWaves;   // 1 KiB loads of a wave and step
  constexpr int kPerStep = kSegsW + kSegsX;
  constexpr int kStage = (TW + TX) * 128;
  static_assert(TW % (8 * kWaves) == 0 && TX % (8 * kWaves) == 0, "tile");

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int ww = wave % WW, wx = wave / WW;
  const int64_t rows_x = min(P.m - i0, (int64_t)TX), rows_w = min(P.n - j0, (int64_t)TW);
  const uint32_t k = (uint32_t)P.k, kb = P.kb;
  const __amdgpu_buffer_rsrc_t rx = rsrc_of(P.x + i0 * P.k, rows_x * P.k), rw = rsrc_of(P.w + j0 * P.k, rows_w * P.k);

  // direct loads: a wave instruction fills one segment of 8 rows; lane l writes the 16 bytes at
  // 16 l, the place of chunk (l mod 8) ^ swz(row) of row l / 8
  const uint32_t seg_row = 8 * wave + (lane >> 3);
  const uint32_t chunk = 16 * ((lane & 7) ^ swz(seg_row & 15));
  static_assert(8 * kWaves % 16 == 0, "rows of a lane's segments share their swizzle");
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
  };

  v4i acc[NW][NX];
#pragma unroll
  for (int i = 0; i < NW; i++)
#pragma unroll
    for (int t = 0; t < NX; t++) acc[i][t] = v4i{};

  // fragments: row col of a 16-row tile, chunks quarter and 4 + quarter
  const uint32_t fs = swz(col);
  const uint32_t fo0 = 16 * (quarter ^ fs), fo1 = 16 * ((4 + quarter) ^ fs);
  const uint32_t fx = (16 * NX * wx + col) * 128, fw = (TX + 16 * NW * ww + col) * 128;
  auto fragment = [&](const lds_u8* p) {
    return Fragment{*reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo0),
                    *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fo1)};
  };

#pragma unroll
  for (int s = 0; s < NS - 1; s++) fetch(s, s);
  stage_barrier<(NS - 2) * kPerStep>();
  uint32_t stage = 0;
  for (uint32_t b = 0; b < kb; b++) {
    const lds_u8* const p = lds + kStage * stage;
    fetch(b + NS - 1, stage == 0 ? NS - 1 : stage - 1);
    Fragment xf[NX];
#pragma unroll
    for (int t = 0; t < NX; t++) xf[t] = fragment(p + fx + 16 * 128 * t);
#pragma unroll
    for (int i = 0; i < NW; i++) {
      const Fragment wf = fragment(p + fw + 16 * 128 * i);
#pragma unroll
      for (int t = 0; t < NX; t++) acc[i][t] = tile_step(wf, xf[t], acc[i][t]);
    }
    stage_barrier<(NS - 2) * kPerStep>();
    stage = stage + 1 == NS ? 0 : stage + 1;
  }
  __builtin_amdgcn_s_waitcnt(0);   // direct loads still in flight land before the wave ends

#pragma unroll
  for (int i = 0; i < NW; i++) {
    const int64_t j = j0 + 16 * (NW * ww + i) + 4 * quarter;
    if (j >= P.n) continue;
#pragma unroll
    for (int t = 0; t < NX; t++) {
      const int64_t row = i0 + 16 * (NX * wx + t) + col;
      if (row < P.m) finish<OUT>(P, row, j, acc[i][t]);
    }
  }
}

// Workgroups [0, full) take whole tiles; the `split` last tiles are taken as two halves of W's
// rows each by the others, so that a last round of few tiles takes half as long.
template <int OUT, int NW, int NX, int WW, int WX, int NS>
__global__ __launch_bounds__(64 * WW * WX) void tiles_kernel(Product P, uint32_t tw, uint32_t tx, uint32_t full, uint32_t split) {
  constexpr int TW = 16 * NW * WW, TX = 16 * NX * WX;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[NS * (TW + TX) * 128];
  lds_u8* const lds = (lds_u8*)lds_mem;
  uint32_t ti, tj;
  if (blockIdx.x < full) {
    tile_of(xcd_spread(blockIdx.x, full), tx, tw, ti, tj);
    tile_product<OUT, NW, NX, WW, WX, NS>(P, (int64_t)ti * TX, (int64_t)tj * TW, lds);
  } else {
    const uint32_t u = xcd_spread(blockIdx.x - full, 2 * split);
    tile_of(full + u / 2, tx, tw, ti, tj);
    const int64_t j0 = (int64_t)tj * TW + TW / 2 * (u & 1);
    if (j0 < P.n) tile_product<OUT, NW / 2, NX, WW, WX, NS>(P, (int64_t)ti * TX, j0, lds);
  }
}

template <int OUT, int NW, int NX, int WW, int WX, int NS>
void tiles_launch(const Product& P, int cus, hipStream_t stream) {
  constexpr int TW = 16 * NW * WW, TX = 16 * NX * WX;
  const uint32_t tx = (uint32_t)((P.m + TX - 1) / TX), tw = (uint32_t)((P.n + TW - 1) / TW);
  const uint32_t tiles = tx * tw, last = tiles % cus, split = 2 * last <= (uint32_t)cus ? last : 0;
  hipLaunchKernelGGL((tiles_kernel<OUT, NW, NX, WW, WX, NS>), dim3(tiles + split), dim3(64 * WW * WX), 0, stream, P, tw, tx,
                     tiles - split, split);
}

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

template <int OUT, int NW, int NX, int KW, int NS>
void ring_launch(const Product& P, uint32_t height, hipStream_t stream) {
  const uint32_t strips = (uint32_t)((P.n + height - 1) / height), tx = (uint32_t)((P.m + 16 * NX - 1) / (16 * NX));
  const uint32_t per_xcd = (strips + kXcds - 1) / kXcds;
  hipLaunchKernelGGL((ring_kernel<OUT, NW, NX, KW, NS>), dim3(per_xcd * kXcds * tx), dim3(64 * KW), 0, stream, P, height, per_xcd);
}

template <int OUT>
void product_launch(const Product& P, int cus, hipStream_t stream) {
  if (P.m <= 16) {
    const uint32_t h = ring_height<2, 1>(P, cus);
    if (rounds((P.n + h - 1) / h, cus) > 1) ring_launch<OUT, 2, 1, 4, 2>(P, h, stream);
    else ring_launch<OUT, 2, 1, 8, 2>(P, h, stream);
    return;
  }
  const int64_t large = rounds(((P.m + 255) / 256) * ((P.n + 255) / 256), cus);
  if (P.m > 512 && large >= 1) tiles_launch<OUT, 8, 4, 2, 4, 2>(P, cus, stream);
  else tiles_launch<OUT, 4, 2, 2, 2, 3>(P, cus, stream);
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

constexpr int64_t kMost = 1 << 24, kMostK = 131071;   // sums of k products of two codes stay below 2^31
bool bad_sizes(int64_t m, int64_t n, int64_t k) { return m < 0 || n <= 0 || k <= 0 || k % 16 || m > kMost || n > kMost || k > kMostK; }

}  // namespace
}  // namespace ep

extern "C" uint64_t ep_gemm_i8_scaled_workspace(int64_t m, int64_t n, int64_t k) {
  if (ep::bad_sizes(m, n, k)) return 0;
  return 0;
}

extern "C" int ep_gemm_i8_scaled(const int8_t* d_x, const float* d_x_scale, const int8_t* d_w, const float* d_w_scale,
                                 const float* d_bias, void* d_y, int y_dtype, int64_t m, int64_t n, int64_t k,
                                 void* d_workspace, uint64_t ws_bytes, void* hip_stream) {
  using namespace ep;
  if (bad_sizes(m, n, k))
    return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: need m >= 0, n > 0, 0 < k <= 131071, k % 16 == 0, m and n up to 2^24");
  if (y_dtype != EP_BF16 && y_dtype != EP_FP16 && y_dtype != EP_FP32)
    return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: y_dtype must be BF16, FP16 or FP32");
  if (m == 0) return EP_OK;
  if (!d_x || !d_x_scale || !d_w || !d_w_scale || !d_y) return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: null pointer");
  const uintptr_t size = y_dtype == EP_FP32 ? 4 : 2;
  if (misaligned(d_x) || misaligned(d_w) || reinterpret_cast<uintptr_t>(d_y) % size ||
      (reinterpret_cast<uintptr_t>(d_x_scale) | reinterpret_cast<uintptr_t>(d_w_scale) | reinterpret_cast<uintptr_t>(d_bias)) % 4)
    return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: operands must be 16-byte aligned, scales, bias and y by their elements");
  const uint64_t need = ep_gemm_i8_scaled_workspace(m, n, k);
  if (need && (!d_workspace || misaligned(d_workspace) || ws_bytes < need))
    return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: a workspace that is missing, misaligned or short");
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return fail(EP_ERR_HIP, "ep_gemm_i8_scaled: no device");
  const Product P = {reinterpret_cast<const uint8_t*>(d_x), d_x_scale, reinterpret_cast<const uint8_t*>(d_w), d_w_scale, d_bias, d_y, m, n, k,
                     (uint32_t)((k + 127) / 128), n % 4 == 0 && reinterpret_cast<uintptr_t>(d_y) % (4 * size) == 0};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (y_dtype == EP_FP32) product_launch<EP_FP32>(P, cus, stream);
  else if (y_dtype == EP_FP16) product_launch<EP_FP16>(P, cus, stream);
  else product_launch<EP_BF16>(P, cus, stream);
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_gemm_i8_scaled: launch failed");
  return EP_OK;
}

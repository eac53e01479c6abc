// INT8 x INT8 -> INT32 matrix product on gfx950 MFMA, for decode-then-GEMM:
// Y[M x N] = A[M x K] * B[N x K]^T, both operands K-contiguous (row-major A,
// row-major B = the decoded weight matrix as stored), exact int32 accumulation,
// in the tiles of i8_tile.h.
//
// Tile order: workgroups are dealt to the 8 XCDs round-robin, so the
// workgroup id is remapped so that each XCD runs a contiguous range of tiles,
// walked in groups of four tile rows (the 32 tiles an XCD holds at once share
// 4 A panels and 8 B panels in its L2).  When the last round of whole tiles
// would occupy at most half of the CUs, its tiles are issued as twice as many
// 256 x 128 halves instead, so that round takes about half as long.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"
#include "i8_tile.h"
#include "tile_order.h"

namespace ep {
namespace {

using i8::kGemmThreads;
using i8::kOutside;
using i8::kSlotBytes;
using i8::kSlots;
using i8::kTileK;
using i8::kTileM;
using i8::kTileN;
using i8::lds_u8;

// Stores a wave's sums of the tile at (m0, n0), TN columns wide; with ADD they are added to Y by atomics (a
// K range of a split tile).
template <int TN, bool ADD>
__device__ __forceinline__ void tile_to(const int8_t* a, const int8_t* b, int32_t* y, int64_t m, int64_t n,
                                        int64_t k, int64_t m0, int64_t n0, int64_t k_lo, int64_t k_hi, lds_u8* lds) {
  i8::tile_product<TN>(a, b, m, n, k, m0, n0, k_lo, k_hi, lds, [=](const auto& acc, int wm, int wn, int lane) {
    constexpr int kBlocksM = i8::kBlocksM, kWaveM = i8::kWaveM, kWaveN = TN / 2, kBlocksN = kWaveN / 32;
    const int half = lane >> 5, fr = lane & 31;
#pragma unroll
    for (int i = 0; i < kBlocksM; i++)
#pragma unroll
      for (int j = 0; j < kBlocksN; j++) {
        const int64_t col = n0 + kWaveN * wn + 32 * j + fr;
#pragma unroll
        for (int r = 0; r < 16; r++) {
          const int64_t row = m0 + kWaveM * wm + 32 * i + 8 * (r >> 2) + 4 * half + (r & 3);
          if (row < m && col < n) {
            EP_GLOBAL int32_t* const p = (EP_GLOBAL int32_t*)y + row * n + col;
            if (ADD) __hip_atomic_fetch_add(p, acc[i][j][r], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            else *p = acc[i][j][r];
          }
        }
      }
  });
}

// Workgroups [0, full) take whole 256 x 256 tiles; when the last round of
// whole tiles would fill at most half the CUs, its `split` tiles are instead
// taken as 2 * split half-width (256 x 128) tiles by workgroups [full, ..),
// so that round lasts about half as long.  With parts > 1 (a launch of few
// tiles) each of those units is taken by `parts` workgroups, each summing a
// range of `part_steps` K steps into Y with atomics (Y cleared before).
template <bool ADD>
__device__ __forceinline__ void gemm_unit(const int8_t* a, const int8_t* b, int32_t* y, int64_t m,
                                          int64_t n, int64_t k, uint32_t tm, uint32_t tn,
                                          uint32_t full, uint32_t split, uint32_t id, int64_t k_lo,
                                          int64_t k_hi, lds_u8* lds) {
  uint32_t ti, tj;
  if (id < full) {
    tile_of(xcd_spread(id, full), tm, tn, ti, tj);
    tile_to<kTileN, ADD>(a, b, y, m, n, k, (int64_t)ti * kTileM, (int64_t)tj * kTileN, k_lo,
                              k_hi, lds);
  } else {
    const uint32_t u = xcd_spread(id - full, 2 * split);
    tile_of(full + u / 2, tm, tn, ti, tj);
    tile_to<kTileN / 2, ADD>(a, b, y, m, n, k, (int64_t)ti * kTileM,
                                  (int64_t)tj * kTileN + (kTileN / 2) * (u & 1), k_lo, k_hi, lds);
  }
}

__global__ __launch_bounds__(kGemmThreads) void gemm_i8_nt_kernel(const int8_t* __restrict__ a,
                                                                  const int8_t* __restrict__ b,
                                                                  int32_t* __restrict__ y,
                                                                  int64_t m, int64_t n, int64_t k,
                                                                  uint32_t tm, uint32_t tn,
                                                                  uint32_t full, uint32_t split,
                                                                  uint32_t parts, uint32_t part_steps) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[kSlots * kSlotBytes];
  lds_u8* const lds = (lds_u8*)lds_mem;
  if (parts == 1) {
    gemm_unit<false>(a, b, y, m, n, k, tm, tn, full, split, blockIdx.x, 0, k, lds);
  } else {
    const uint32_t unit = blockIdx.x / parts, part = blockIdx.x % parts;
    const int64_t k_lo = (int64_t)part * part_steps * kTileK;
    const int64_t k_hi = k_lo + (int64_t)part_steps * kTileK < k ? k_lo + (int64_t)part_steps * kTileK : k;
    if (k_lo < k_hi) gemm_unit<true>(a, b, y, m, n, k, tm, tn, full, split, unit, k_lo, k_hi, lds);
  }
}

__global__ void zero_i32_kernel(int32_t* __restrict__ y, int64_t count) {
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count;
       i += (int64_t)gridDim.x * blockDim.x)
    ((EP_GLOBAL int32_t*)y)[i] = 0;
}

}  // namespace
}  // namespace ep

extern "C" int ep_gemm_i8_nt(const int8_t* d_a, const int8_t* d_b, int32_t* d_y, int64_t m,
                             int64_t n, int64_t k, void* hip_stream) {
  if (!d_a || !d_b || !d_y) return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: null pointer");
  if (m <= 0 || n <= 0 || k <= 0 || k % 16)
    return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: need m, n, k > 0 and k % 16 == 0");
  if ((reinterpret_cast<uintptr_t>(d_a) | reinterpret_cast<uintptr_t>(d_b)) & 15)
    return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: operands must be 16-byte aligned");
  // |a * b| <= 128 * 128 = 2^14, so a K-term sum stays below 2^31 for K <= 131071
  if (k > 131071)
    return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: k above 131071 may overflow the int32 sums");
  if (m * k >= (int64_t)ep::kOutside || n * k >= (int64_t)ep::kOutside)
    return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: an operand above 2^31 bytes");
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0)
    return ep::fail(EP_ERR_HIP, "ep_gemm_i8_nt: no device");
  const int64_t tm = (m + ep::kTileM - 1) / ep::kTileM, tn = (n + ep::kTileN - 1) / ep::kTileN;
  const int64_t tiles = tm * tn, last = tiles % cus;
  if (tiles + last > 0x7FFFFFFF) return ep::fail(EP_ERR_ARG, "ep_gemm_i8_nt: matrix too large");
  const int64_t split = (last > 0 && 2 * last <= cus) ? last : 0;   // one workgroup per CU
  // A launch of at most half as many units (whole or half tiles) as CUs splits
  // K over `parts` workgroups per unit, at least four 128-byte steps each.
  const int64_t units = tiles + split, steps = (k + ep::kTileK - 1) / ep::kTileK;
  int64_t parts = 1;
  if (2 * units <= cus) parts = std::max<int64_t>(1, std::min<int64_t>(cus / units, steps / 4));
  const int64_t part_steps = (steps + parts - 1) / parts;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (parts > 1) {
    const int64_t count = m * n;
    const unsigned blocks = (unsigned)std::min<int64_t>((count + 255) / 256, 4096);
    hipLaunchKernelGGL(ep::zero_i32_kernel, dim3(blocks), dim3(256), 0, stream, d_y, count);
  }
  hipLaunchKernelGGL(ep::gemm_i8_nt_kernel, dim3((unsigned)(units * parts)), dim3(ep::kGemmThreads), 0,
                     stream, d_a, d_b, d_y, m, n, k, (uint32_t)tm, (uint32_t)tn,
                     (uint32_t)(tiles - split), (uint32_t)split, (uint32_t)parts, (uint32_t)part_steps);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_gemm_i8_nt: launch failed");
  return EP_OK;
}

// Pieces of the products of 8-bit operands in tiles: direct loads to LDS, places there, stores.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/entropack.h"

namespace ep {
namespace {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef __bf16 v4b __attribute__((ext_vector_type(4)));

// Y's element types: ep_dtype codes as template arguments.
template <int OUT>
__device__ __forceinline__ void store_y(void* y, int64_t at, float f) {
  if (OUT == EP_FP32) static_cast<float*>(y)[at] = f;
  else if (OUT == EP_FP16) static_cast<_Float16*>(y)[at] = (_Float16)f;
  else static_cast<__bf16*>(y)[at] = (__bf16)f;
}

// Four values of row i from column j, a multiple of four, on; in one store where it is aligned.
template <int OUT>
__device__ __forceinline__ void store_y4(void* y, int64_t n, uint32_t wide, int64_t i, int64_t j, const v4f& v) {
  const int64_t at = i * n + j;
  if (wide && j + 4 <= n) {
    if (OUT == EP_FP32) {
      *reinterpret_cast<v4f*>(static_cast<float*>(y) + at) = v;
    } else if (OUT == EP_FP16) {
      *reinterpret_cast<v4h*>(static_cast<_Float16*>(y) + at) = __builtin_convertvector(v, v4h);
    } else {
      *reinterpret_cast<v4b*>(static_cast<__bf16*>(y) + at) = __builtin_convertvector(v, v4b);
    }
  } else {
#pragma unroll
    for (int r = 0; r < 4; r++)
      if (j + r < n) store_y<OUT>(y, at + r, v[r]);
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

}  // namespace
}  // namespace ep

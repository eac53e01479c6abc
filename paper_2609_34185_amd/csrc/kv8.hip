// The paged 8-bit key/value cache: places for the new tokens of a step (block tables and slot
// maps), and the writer that quantises keys and values into them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "../../include/entropack.h"
#include "common.h"
#include "kv8.h"

namespace ep {
namespace {

// ---- block tables and slot maps ------------------------------------------------------
constexpr int kSlotThreads = 1024;
constexpr int kSlotWaves = kSlotThreads / 64;
constexpr int kSlotTokens = 2048;    // slots that one workgroup writes

struct Slots {
  const int32_t *cached, *fresh, *free_pages, *n_free;
  int32_t* table;
  int32_t *len, *cu;
  int64_t* slots;
  int32_t *used, *status;
  int64_t n_req, table_ld, n_slots;
  int shift;           // log2 of a page's tokens
};

// Sums of a and b over the threads before this one; ta and tb get the workgroup's.
__device__ __forceinline__ void scan2(int64_t& a, int64_t& b, int64_t& ta, int64_t& tb,
                                      int64_t (*wave_sums)[2]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t a0 = a, b0 = b;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t pa = __shfl_up(a, d), pb = __shfl_up(b, d);
    if (lane >= d) {
      a += pa;
      b += pb;
    }
  }
  __syncthreads();   // the last use of wave_sums is over
  if (lane == 63) {
    wave_sums[wave][0] = a;
    wave_sums[wave][1] = b;
  }
  __syncthreads();
  a -= a0;
  b -= b0;
  ta = tb = 0;
#pragma unroll
  for (int w = 0; w < kSlotWaves; w++) {
    if (w == wave) {
      a += ta;
      b += tb;
    }
    ta += wave_sums[w][0];
    tb += wave_sums[w][1];
  }
}

// Every workgroup walks all requests in tiles of 1024, carrying the sums of their tokens and
// pages, and writes the slots of its own 2048 tokens; tile t's lengths, table entries and sums
// are written by workgroup t mod the grid's size.  Walking them again in every workgroup costs
// eight bytes a request from the caches, and saves a second launch and any waiting between
// workgroups: 256 requests are one tile.
__global__ __launch_bounds__(kSlotThreads) void slots_kernel(Slots S) {
  __shared__ int64_t wave_sums[kSlotWaves][2];
  __shared__ int64_t first_tok[kSlotThreads + 1];   // of the tile's requests
  __shared__ int32_t first_page[kSlotThreads], held[kSlotThreads];
  __shared__ int32_t old_tokens[kSlotThreads];      // cached, or -1 of a refused request
  const int t = threadIdx.x;
  const int64_t n_free = max(*S.n_free, 0);
  const int64_t lo = (int64_t)blockIdx.x * kSlotTokens;
  const int64_t hi = lo + kSlotTokens < S.n_slots ? lo + kSlotTokens : S.n_slots;
  const int64_t page = (int64_t)1 << S.shift;
  int64_t tok = 0, pages = 0;      // before the tile
  int32_t bits = 0;
  for (int64_t tile = 0, b0 = 0; b0 < S.n_req; tile++, b0 += kSlotThreads) {
    const int64_t b = b0 + t;
    int64_t cached = 0, fresh = 0;
    if (b < S.n_req) {
      cached = max(S.cached[b], 0);
      fresh = max(S.fresh[b], 0);
    }
    const int64_t have = (cached + page - 1) >> S.shift, want = (cached + fresh + page - 1) >> S.shift;
    // tokens first: a request whose tokens do not fit the slot map asks for no pages
    int64_t my_tok = fresh, my_page = 0, tile_tok, tile_pages, none;
    scan2(my_tok, my_page, tile_tok, none, wave_sums);
    my_tok += tok;
    const bool row_fits = want <= S.table_ld, slots_fit = my_tok + fresh <= S.n_slots;
    const int64_t need = row_fits && slots_fit ? want - have : 0;
    int64_t off = need, dummy = 0;
    scan2(off, dummy, tile_pages, none, wave_sums);
    off += pages;
    const bool paged = need == 0 || off + need <= n_free;
    const bool ok = row_fits && slots_fit && paged;
    first_tok[t] = my_tok;
    first_page[t] = (int32_t)(off < 0x7FFFFFFF ? off : 0x7FFFFFFF);
    held[t] = (int32_t)have;
    old_tokens[t] = ok ? (int32_t)cached : -1;
    if (t == 0) first_tok[kSlotThreads] = tok + tile_tok;
    const bool mine = tile % gridDim.x == blockIdx.x;
    if (mine && b < S.n_req) {
      S.len[b] = (int32_t)(ok ? cached + fresh : cached);
      const int64_t most = 0x7FFFFFFF;
      S.cu[b] = (int32_t)(my_tok < most ? my_tok : most);
      if (b == S.n_req - 1) S.cu[b + 1] = (int32_t)(my_tok + fresh < most ? my_tok + fresh : most);
      bits |= (row_fits ? 0 : EP_STATUS_TABLE_FULL) | (slots_fit ? 0 : EP_STATUS_SLOTS_FULL) |
              (paged ? 0 : EP_STATUS_NO_PAGES);
      // pages taken: all that is needed, or what is needed before the first request that they
      // do not suffice for
      if (need > 0 && off <= n_free && off + need > n_free) *S.used = (int32_t)off;
      if (b == S.n_req - 1 && off + need <= n_free) *S.used = (int32_t)(off + need);
    }
    __syncthreads();
    // the tile's tokens in this workgroup's range; a token at the start of a page that its
    // request did not hold puts the page into the table
    const int64_t from = max(lo, tok), to = min(hi, tok + tile_tok);
    for (int64_t at = from + t; at < to; at += kSlotThreads) {
      int r = 0;   // the last request of the tile whose first token is not after `at`
#pragma unroll
      for (int d = kSlotThreads / 2; d > 0; d /= 2)
        if (first_tok[r + d] <= at) r += d;
      int64_t slot = -1;
      if (old_tokens[r] >= 0) {
        const int64_t pos = old_tokens[r] + (at - first_tok[r]), j = pos >> S.shift;
        int32_t* const entry = S.table + (b0 + r) * S.table_ld + j;
        int32_t p;
        if (j < held[r]) {
          p = *entry;
        } else {
          p = S.free_pages[first_page[r] + (j - held[r])];
          if ((pos & (page - 1)) == 0) *entry = p;
        }
        slot = (int64_t)p * page + (pos & (page - 1));
      }
      S.slots[at] = slot;
    }
    tok += tile_tok;
    pages += tile_pages;
    __syncthreads();
  }
  for (int64_t at = max(lo, tok) + t; at < hi; at += kSlotThreads) S.slots[at] = -1;
  if (bits && S.status) __hip_atomic_fetch_or(S.status, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- append --------------------------------------------------------------------------
struct Bf16 { uint16_t bits; };
struct Fp16 { _Float16 h; };
__device__ __forceinline__ float as_float(Bf16 x) { return __uint_as_float((uint32_t)x.bits << 16); }
__device__ __forceinline__ float as_float(Fp16 x) { return (float)x.h; }
__device__ __forceinline__ float as_float(float x) { return x; }

struct Append {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  const void *new_k, *new_v;
  const int64_t* slots;
  int64_t k_row, v_row, n_tokens, n_slots;
  int heads, shift;
};

// Nearest code of x / s (0 where s is 0).
template <bool INT8>
__device__ __forceinline__ uint8_t code_of(float x, float s) {
  const float top = INT8 ? 127.0f : 448.0f;
  float q = s == 0.0f ? 0.0f : x / s;
  q = q > top ? top : q < -top ? -top : q;   // a NaN stays one
  if (INT8) return (uint8_t)(int8_t)(int)rintf(q);
  return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(q, q, 0, false) & 0xFF);
}

template <bool INT8>
__device__ __forceinline__ float value_of(uint8_t c) {
  if (INT8) return (float)(int8_t)c;
  return __builtin_amdgcn_cvt_f32_fp8(c, 0);
}

// One workgroup for each token, head and array (keys, values); those whose token is not the
// first of its page's tokens have nothing to do.
constexpr int kAppendThreads = 256;

template <typename T, int D, bool INT8>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Append A) {
  __shared__ uint32_t wave_top[kAppendThreads / 64];
  const int64_t t0 = blockIdx.x;
  const int head = blockIdx.y;
  const bool values = blockIdx.z;
  const int64_t slot = A.slots[t0];
  if (slot < 0 || slot >= A.n_slots) return;
  const int64_t page = slot >> A.shift;
  const int tokens = 1 << A.shift, at = (int)(slot & (tokens - 1));
  if (t0 > 0 && A.slots[t0 - 1] >= 0 && A.slots[t0 - 1] >> A.shift == page) return;
  int count = 1;
  while (at + count < tokens && t0 + count < A.n_tokens && A.slots[t0 + count] == slot + count) count++;

  const T* const x = static_cast<const T*>(values ? A.new_v : A.new_k) + (int64_t)head * D;
  const int64_t row = values ? A.v_row : A.k_row;
  uint8_t* const codes = (values ? A.v : A.k) + (page * A.heads + head) * ((int64_t)tokens * D);
  float* const scale = (values ? A.v_scale : A.k_scale) + page * A.heads + head;
  uint32_t top = 0;
  for (int e = threadIdx.x; e < count * D; e += kAppendThreads)
    top = max(top, __float_as_uint(as_float(x[(t0 + e / D) * row + e % D])) & 0x7FFFFFFFu);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  if (threadIdx.x % 64 == 0) wave_top[threadIdx.x / 64] = top;
  const float before = at > 0 ? *scale : 0.0f;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kAppendThreads / 64; w++) top = max(top, wave_top[w]);
  const float fresh = __uint_as_float(top) / (INT8 ? 127.0f : 448.0f);
  // a NaN of either side stays
  const float now = fresh > before || fresh != fresh ? fresh : before;
  if (threadIdx.x == 0) *scale = now;
  // code (p, c) lies at p D + c of a key page, c tokens + p of a value page
  if (now != before)
    for (int e = threadIdx.x; e < at * D; e += kAppendThreads) {
      const int p = e / D, c = e % D;
      uint8_t* const q = codes + (values ? c * tokens + p : p * D + c);
      *q = code_of<INT8>(value_of<INT8>(*q) * before, now);
    }
  for (int e = threadIdx.x; e < count * D; e += kAppendThreads) {
    const int p = e / D, c = e % D;
    codes[values ? c * tokens + at + p : (at + p) * D + c] = code_of<INT8>(as_float(x[(t0 + p) * row + c]), now);
  }
}

template <typename T, int D>
void append_launch(const Append& A, bool int8, hipStream_t stream) {
  const dim3 grid((uint32_t)A.n_tokens, A.heads, 2);
  if (int8) hipLaunchKernelGGL((append_kernel<T, D, true>), grid, dim3(kAppendThreads), 0, stream, A);
  else hipLaunchKernelGGL((append_kernel<T, D, false>), grid, dim3(kAppendThreads), 0, stream, A);
}

template <typename T>
void append_launch(const Append& A, int dim, bool int8, hipStream_t stream) {
  if (dim == 64) append_launch<T, 64>(A, int8, stream);
  else if (dim == 128) append_launch<T, 128>(A, int8, stream);
  else append_launch<T, 256>(A, int8, stream);
}

int fail_with(int code, const char* what, const char* why) { return fail(code, (std::string(what) + ": " + why).c_str()); }

}  // namespace
}  // namespace ep

extern "C" int ep_kv8_slots(const int32_t* d_cached, const int32_t* d_new, int64_t n_req, int page_tokens,
                            const int32_t* d_free, const int32_t* d_n_free, int32_t* d_table, int64_t table_ld,
                            int32_t* d_len, int32_t* d_cu, int64_t* d_slots, int64_t n_slots, int32_t* d_used,
                            int32_t* d_status, void* hip_stream) {
  const int shift = ep::page_shift(page_tokens);
  if (shift < 0) return ep::fail(EP_ERR_ARG, "ep_kv8_slots: page_tokens must be 16, 32, 64, 128 or 256");
  if (n_req <= 0 || n_req >= 0x7FFFFFFF || table_ld <= 0 || table_ld > 0x7FFFFFFF || n_slots < 0 || n_slots > 0x7FFFFFFF)
    return ep::fail(EP_ERR_ARG, "ep_kv8_slots: need n_req, table_ld > 0 and 0 <= n_slots < 2^31");
  if (!d_cached || !d_new || !d_free || !d_n_free || !d_table || !d_len || !d_cu || (!d_slots && n_slots) || !d_used)
    return ep::fail(EP_ERR_ARG, "ep_kv8_slots: null pointer");
  const ep::Slots S = {d_cached, d_new, d_free, d_n_free, d_table, d_len, d_cu, d_slots,
                       d_used, d_status, n_req, table_ld, n_slots, shift};
  const int64_t groups = std::max<int64_t>(1, (n_slots + ep::kSlotTokens - 1) / ep::kSlotTokens);
  hipLaunchKernelGGL(ep::slots_kernel, dim3((uint32_t)groups), dim3(ep::kSlotThreads), 0,
                     static_cast<hipStream_t>(hip_stream), S);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_kv8_slots: launch failed");
  return EP_OK;
}

extern "C" int ep_kv8_append(const ep_kv8_cache* cache, const void* d_k, const void* d_v, int dtype,
                             int64_t k_row, int64_t v_row, const int64_t* d_slots, int64_t n_tokens,
                             void* hip_stream) {
  if (const char* why = ep::cache_fault(cache)) return ep::fail_with(EP_ERR_ARG, "ep_kv8_append", why);
  if (dtype != EP_BF16 && dtype != EP_FP16 && dtype != EP_FP32)
    return ep::fail(EP_ERR_ARG, "ep_kv8_append: dtype must be BF16, FP16 or FP32");
  const int64_t width = (int64_t)cache->kv_heads * cache->head_dim, step = dtype == EP_FP32 ? 4 : 8;
  if (k_row < width || v_row < width || k_row % step || v_row % step)
    return ep::fail(EP_ERR_ARG, "ep_kv8_append: rows must hold kv_heads * head_dim elements and be 16-byte aligned");
  if (n_tokens < 0 || n_tokens > 0x7FFFFFFF)
    return ep::fail(EP_ERR_ARG, "ep_kv8_append: n_tokens outside 0 .. 2^31 - 1");
  if (n_tokens == 0) return EP_OK;
  if (!d_k || !d_v || !d_slots) return ep::fail(EP_ERR_ARG, "ep_kv8_append: null pointer");
  if ((reinterpret_cast<uintptr_t>(d_k) | reinterpret_cast<uintptr_t>(d_v)) & 15)
    return ep::fail(EP_ERR_ARG, "ep_kv8_append: keys and values must be 16-byte aligned");
  const int shift = ep::page_shift(cache->page_tokens);
  const ep::Append A = {static_cast<uint8_t*>(cache->d_k), static_cast<uint8_t*>(cache->d_v), cache->d_k_scale,
                        cache->d_v_scale, d_k, d_v, d_slots, k_row, v_row, n_tokens,
                        cache->n_pages << shift, cache->kv_heads, shift};
  const bool int8 = cache->dtype == EP_INT8;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (dtype == EP_BF16) ep::append_launch<ep::Bf16>(A, cache->head_dim, int8, stream);
  else if (dtype == EP_FP16) ep::append_launch<ep::Fp16>(A, cache->head_dim, int8, stream);
  else ep::append_launch<float>(A, cache->head_dim, int8, stream);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_kv8_append: launch failed");
  return EP_OK;
}

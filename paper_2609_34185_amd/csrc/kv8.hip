// The paged 8-bit key/value cache: places for the new tokens of a step (block tables and slot
// maps), and the writer that quantises keys and values into them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>

#include "../../include/entropack.h"
#include "common.h"
#include "kv8.h"
#include "scaled.h"

namespace ep {
namespace {

// ---- block tables and slot maps ------------------------------------------------------
constexpr int kSlotThreads = 512, kSlotWaves = kSlotThreads / 64;
constexpr int kEach = 8, kTile = kSlotThreads * kEach;   // requests of a thread, and of a tile
constexpr int kSlotTokens = 2048;                        // slots that one workgroup writes

// Where request r of a tile is kept: a word is left out after each thread's, so that threads that
// write theirs at once meet different banks.
constexpr int kPlaces = kTile + kTile / kEach;
__device__ __forceinline__ int place_of(int r) { return r + r / kEach; }

// A thread's counts, negative ones and those past the end as 0.
__device__ __forceinline__ void load_counts(const int32_t* p, int64_t first, int64_t n, int32_t (&v)[kEach]) {
  if (first + kEach <= n && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
#pragma unroll
    for (int i = 0; i < kEach; i += 4) {
      const int4 x = *reinterpret_cast<const int4*>(p + first + i);
      v[i] = max(x.x, 0);
      v[i + 1] = max(x.y, 0);
      v[i + 2] = max(x.z, 0);
      v[i + 3] = max(x.w, 0);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kEach; i++) v[i] = first + i < n ? max(p[first + i], 0) : 0;
  }
}

struct Slots {
  const int32_t *cached, *fresh, *free_pages, *n_free;
  int32_t* table;
  int32_t *len, *cu;
  int64_t* slots;
  int32_t *used, *status;
  int64_t n_req, table_ld, n_slots;
  int shift;           // log2 of a page's tokens
};

// Sum of x over the threads before this one; `all` gets the workgroup's.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t& all, int64_t* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t sum = x;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t up = __shfl_up(sum, d);
    if (lane >= d) sum += up;
  }
  __syncthreads();   // the last use of wave_sums is over
  if (lane == 63) wave_sums[wave] = sum;
  __syncthreads();
  int64_t before = sum - x;
  all = 0;
#pragma unroll
  for (int w = 0; w < kSlotWaves; w++) {
    if (w < wave) before += wave_sums[w];
    all += wave_sums[w];
  }
  return before;
}

// Every workgroup walks all requests in tiles of 4096, carrying the sums of their tokens and pages,
// and writes the slots of its own 2048 tokens; tile t's lengths and sums are written by workgroup
// t mod the grid's size.  Walking them again in every workgroup costs eight bytes a request from
// the caches, and saves a second launch and any waiting between workgroups.  What is left is
// latency: the counts, two scans, a search in LDS and a page number.  256 requests of one token take
// 7.6 us, 3001 with 775 thousand tokens 16.8.
__global__ __launch_bounds__(kSlotThreads) void slots_kernel(Slots S) {
  __shared__ int64_t wave_sums[kSlotWaves];
  // of the tile's requests, r at place_of(r)
  __shared__ int32_t first_tok[kPlaces];      // from this workgroup's first on
  __shared__ int32_t first_page[kPlaces], held[kPlaces];
  __shared__ int32_t old_tokens[kPlaces];     // cached, or -1 of a refused request
  const int t = threadIdx.x;
  const int64_t n_free = max(*S.n_free, 0), most = 0x7FFFFFFF;
  const int64_t lo = (int64_t)blockIdx.x * kSlotTokens;
  const int64_t hi = lo + kSlotTokens < S.n_slots ? lo + kSlotTokens : S.n_slots;
  const int32_t page = 1 << S.shift;
  int64_t tok = 0, pages = 0;      // before the tile
  int32_t bits = 0;
  for (int64_t tile = 0, b0 = 0; b0 < S.n_req; tile++, b0 += kTile) {
    const int64_t mine = b0 + (int64_t)t * kEach;
    int32_t cached[kEach], fresh[kEach];
    int64_t my_tok = 0;
    load_counts(S.cached, mine, S.n_req, cached);
    load_counts(S.fresh, mine, S.n_req, fresh);
#pragma unroll
    for (int i = 0; i < kEach; i++) my_tok += fresh[i];
    int64_t tile_tok, tile_pages;
    my_tok = tok + scan(my_tok, tile_tok, wave_sums);
    // pages that a request asks for: none if it does not fit its row of the table or the slot map
    auto pages_of = [&](int i, int64_t first, bool& row_fits, bool& slots_fit, int64_t& have) {
      have = ((int64_t)cached[i] + page - 1) >> S.shift;
      const int64_t want = ((int64_t)cached[i] + fresh[i] + page - 1) >> S.shift;
      row_fits = want <= S.table_ld && (int64_t)cached[i] + fresh[i] <= most;
      slots_fit = first + fresh[i] <= S.n_slots;
      return row_fits && slots_fit ? want - have : 0;
    };
    int64_t need = 0, first = my_tok, have;
    bool row_fits, slots_fit;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
      need += pages_of(i, first, row_fits, slots_fit, have);
      first += fresh[i];
    }
    int64_t off = pages + scan(need, tile_pages, wave_sums);
    const bool owner = tile % gridDim.x == blockIdx.x;
    first = my_tok;
#pragma unroll
    for (int i = 0; i < kEach; i++) {
      const int64_t b = mine + i;
      need = pages_of(i, first, row_fits, slots_fit, have);
      const bool paged = need == 0 || off + need <= n_free, ok = row_fits && slots_fit && paged;
      const int r = place_of(t * kEach + i);
      first_tok[r] = (int32_t)min(first - lo, most);
      first_page[r] = (int32_t)min(off, most);
      held[r] = (int32_t)have;
      old_tokens[r] = ok ? cached[i] : -1;
      if (owner && b < S.n_req) {
        S.len[b] = ok ? cached[i] + fresh[i] : cached[i];
        S.cu[b] = (int32_t)min(first, most);
        if (b == S.n_req - 1) S.cu[b + 1] = (int32_t)min(first + fresh[i], most);
        bits |= (row_fits ? 0 : EP_STATUS_TABLE_FULL) | (slots_fit ? 0 : EP_STATUS_SLOTS_FULL) |
                (paged ? 0 : EP_STATUS_NO_PAGES);
        // pages taken: all that is needed, or what is needed before the first request that they
        // do not suffice for
        if (need > 0 && off <= n_free && off + need > n_free) *S.used = (int32_t)off;
        if (b == S.n_req - 1 && off + need <= n_free) *S.used = (int32_t)(off + need);
      }
      first += fresh[i];
      off += need;
    }
    __syncthreads();
    // the tile's tokens in this workgroup's range; a token at the start of a page that its
    // request did not hold puts the page into the table
    const int from = (int)min(max(tok - lo, (int64_t)0), (int64_t)kSlotTokens), to = (int)(min(hi, tok + tile_tok) - lo);
    constexpr int kOwn = kSlotTokens / kSlotThreads;
    int r[kOwn] = {};   // the last request of the tile whose first token is not after this thread's
#pragma unroll
    for (int d = kTile / 2; d > 0; d /= 2)
#pragma unroll
      for (int u = 0; u < kOwn; u++)
        if (first_tok[place_of(r[u] + d)] <= t + kSlotThreads * u) r[u] += d;
    int32_t p[kOwn] = {}, in_page[kOwn], fill[kOwn];   // fill: the row's entry to write, or -1
#pragma unroll
    for (int u = 0; u < kOwn; u++) {
      const int at = t + kSlotThreads * u, l = place_of(r[u]);
      in_page[u] = fill[u] = -1;
      if (at >= from && at < to && old_tokens[l] >= 0) {
        const int32_t pos = old_tokens[l] + (at - first_tok[l]), j = pos >> S.shift;
        in_page[u] = pos & (page - 1);
        if (j >= held[l] && in_page[u] == 0) fill[u] = j;
        p[u] = *(j < held[l] ? S.table + (b0 + r[u]) * S.table_ld + j : S.free_pages + first_page[l] + (j - held[l]));
      }
    }
#pragma unroll
    for (int u = 0; u < kOwn; u++) {
      const int at = t + kSlotThreads * u;
      if (fill[u] >= 0) S.table[(b0 + r[u]) * S.table_ld + fill[u]] = p[u];
      if (at >= from && at < to) S.slots[lo + at] = in_page[u] < 0 ? -1 : (int64_t)p[u] * page + in_page[u];
    }
    tok += tile_tok;
    pages += tile_pages;
    if (b0 + kTile < S.n_req) __syncthreads();
  }
  for (int64_t at = max(lo, tok) + t; at < hi; at += kSlotThreads) S.slots[at] = -1;
  if (bits && S.status) __hip_atomic_fetch_or(S.status, bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---- append --------------------------------------------------------------------------
struct Append {
  uint8_t *k, *v;
  float *k_scale, *v_scale;
  const void *new_k, *new_v;
  const int64_t* slots;
  int64_t k_row, v_row, n_tokens, n_slots;
  int heads, shift;
};

// Codes of two values in the low bytes.  Rounding to nearest even; INT8's NaN becomes 0, and shows
// in the scale.
template <bool INT8>
__device__ __forceinline__ uint32_t codes2(float a, float b) {
  if (INT8) return ((uint32_t)(int)rintf(a) & 0xFFu) | ((uint32_t)(int)rintf(b) & 0xFFu) << 8;
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// The values of the four codes of a word, carried over from one scale to another.
template <bool INT8>
__device__ __forceinline__ uint32_t rescaled4(uint32_t c, float before, const Divider& by) {
  float x[4];
  if (INT8) {
#pragma unroll
    for (int i = 0; i < 4; i++) x[i] = (float)(int8_t)(c >> (8 * i));
  } else {
    x[0] = __builtin_amdgcn_cvt_f32_fp8((int)c, 0);
    x[1] = __builtin_amdgcn_cvt_f32_fp8((int)c, 1);
    x[2] = __builtin_amdgcn_cvt_f32_fp8((int)c, 2);
    x[3] = __builtin_amdgcn_cvt_f32_fp8((int)c, 3);
  }
#pragma unroll
  for (int i = 0; i < 4; i++) x[i] = by(x[i] * before);
  return codes2<INT8>(x[0], x[1]) | codes2<INT8>(x[2], x[3]) << 16;
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// Element e of a lane's channels of one token, from the words that hold them.
__device__ __forceinline__ float element(const Bf16*, const uint32_t* w, int e) {
  return __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
}
__device__ __forceinline__ float element(const Fp16*, const uint32_t* w, int e) {
  return (float)__builtin_bit_cast(_Float16, (uint16_t)(e & 1 ? w[e >> 1] >> 16 : w[e >> 1]));
}
__device__ __forceinline__ float element(const float*, const uint32_t* w, int e) { return __uint_as_float(w[e]); }

// W words (2, 4, 8 or 16) from an address aligned to as many bytes as a load takes.
template <int W>
__device__ __forceinline__ void load_words(const void* p, uint32_t* w) {
  if (W == 2) {
    const uint2 x = *static_cast<const uint2*>(p);
    w[0] = x.x;
    w[1] = x.y;
  } else {
#pragma unroll
    for (int i = 0; i < W / 4; i++) {
      const v4u x = static_cast<const v4u*>(p)[i];
#pragma unroll
      for (int j = 0; j < 4; j++) w[4 * i + j] = x[j];
    }
  }
}

// A run of tokens that take consecutive places of one page, for one head, keys or values.
struct Run {
  uint8_t* codes;
  float* scale;
  const void* x;       // the head's channels of the run's first token
  int64_t row;         // elements from one token to the next
  int at, count;       // first place, tokens
  bool values;
};

template <typename T, int D>
__device__ __forceinline__ Run run_of(const Append& A, int64_t t0, int64_t slot, int count, int item) {
  const int head = item >> 1, tokens = 1 << A.shift;
  Run R;
  R.values = item & 1;
  R.row = R.values ? A.v_row : A.k_row;
  R.x = static_cast<const T*>(R.values ? A.new_v : A.new_k) + t0 * R.row + head * D;
  const int64_t block = (slot >> A.shift) * A.heads + head;
  R.codes = (R.values ? A.v : A.k) + block * ((int64_t)tokens * D);
  R.scale = (R.values ? A.v_scale : A.k_scale) + block;
  R.at = (int)(slot & (tokens - 1));
  R.count = count;
  return R;
}

// The page's scale with the new tokens' largest magnitude among it; a NaN of either side stays.
template <bool INT8>
__device__ __forceinline__ float grown(float before, uint32_t top) {
  const float fresh = __uint_as_float(top) * (INT8 ? 1.0f / 127.0f : 1.0f / 448.0f);
  return fresh > before || fresh != fresh ? fresh : before;
}

// Carry the codes of places 0 .. at - 1 over to another scale, 16 codes for a lane at a time; done by
// one wave.
template <int D, bool INT8>
__device__ __forceinline__ void carry_over(uint8_t* codes, int at, bool values, int tokens, float before, const Divider& by) {
  const int lane = threadIdx.x & 63, per = values ? (at + 15) >> 4 : D / 16, all = values ? D * per : at * per;
#pragma unroll 4
  for (int i = lane; i < all; i += 64) {
    const int r = i / per, c = i - r * per;
    v4u* const p = reinterpret_cast<v4u*>(codes + (values ? r * tokens + 16 * c : 16 * i));
    const v4u old = *p;
    v4u w;
#pragma unroll
    for (int k = 0; k < 4; k++) {
      w[k] = rescaled4<INT8>(old[k], before, by);
      if (values) {   // what is not the page's yet stays
        const int mine = min(max(at - 16 * c - 4 * k, 0), 4);
        const uint32_t mask = mine == 4 ? 0xFFFFFFFFu : (1u << (8 * mine)) - 1u;
        w[k] = (w[k] & mask) | (old[k] & ~mask);
      }
    }
    *p = w;
  }
}

// C codes (a multiple of 4) of one token, four in a word.
template <typename T, int C, bool INT8>
__device__ __forceinline__ void codes_of(const uint32_t* w, const Divider& by, uint32_t (&q)[C / 4]) {
#pragma unroll
  for (int k = 0; k < C / 4; k++) {
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; e++) v[e] = by.s == 0.0f ? 0.0f : by(element(static_cast<const T*>(nullptr), w, 4 * k + e));
    q[k] = codes2<INT8>(v[0], v[1]) | codes2<INT8>(v[2], v[3]) << 16;
  }
}

// A long run, by one wave.  16 lanes hold a token's channels, D / 16 each, and the wave's four rows
// of lanes take four tokens each of a block of 16 places, so that a value channel's 16 codes can
// be gathered into one lane: bytes are transposed four by four within a lane, then words between
// the rows of lanes.  Up to kBlocks blocks stay in registers between the maximum and the codes;
// twice as many cost a wave of occupancy (58 us for 52 at 25 thousand tokens x 8 heads), and longer runs
// read their values again from the caches.
template <typename T, int D, bool INT8>
__device__ __forceinline__ void append_long(const Run& R, int tokens) {
  constexpr int C = D / 16, W = C * (int)sizeof(T) / 4, kBlocks = 256 / D;
  const int lane = threadIdx.x & 63, sub = lane & 15, quarter = lane >> 4;
  const int first = R.at & ~15, last = R.at + R.count;
  const bool once = last - first <= 16 * kBlocks;
  const T* const x = static_cast<const T*>(R.x) + C * sub;
  uint32_t w[kBlocks][4][W];
  auto load = [&](int place0, int blocks) {
#pragma unroll
    for (int n = 0; n < kBlocks; n++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int place = place0 + 16 * n + 4 * quarter + i;
#pragma unroll
        for (int j = 0; j < W; j++) w[n][i][j] = 0;
        if (n < blocks && place >= R.at && place < last) load_words<W>(x + (place - R.at) * R.row, w[n][i]);
      }
  };
  uint32_t top = 0;
  for (int place0 = first; place0 < last; place0 += 16 * kBlocks) {
    load(place0, kBlocks);
#pragma unroll
    for (int n = 0; n < kBlocks; n++)
#pragma unroll
      for (int i = 0; i < 4; i++)
#pragma unroll
        for (int e = 0; e < C; e++) top = max(top, __float_as_uint(element(x, w[n][i], e)) & 0x7FFFFFFFu);
  }
  const float before = R.at > 0 ? *R.scale : 0.0f;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const float now = grown<INT8>(before, top);
  const Divider by(now, INT8 ? 127.0f : 448.0f);
  if (now != before && R.at > 0) carry_over<D, INT8>(R.codes, R.at, R.values, tokens, before, by);
  if (lane == 0) *R.scale = now;
  for (int place0 = first; place0 < last; place0 += 16 * kBlocks) {
    if (!once) load(place0, kBlocks);
#pragma unroll
    for (int n = 0; n < kBlocks; n++) {
      const int p0 = place0 + 16 * n;
      if (p0 >= last) break;
      uint32_t q[4][C / 4];
#pragma unroll
      for (int i = 0; i < 4; i++) codes_of<T, C, INT8>(w[n][i], by, q[i]);
      if (!R.values) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const int place = p0 + 4 * quarter + i;
          if (place >= R.at && place < last) {
            uint32_t* const dst = reinterpret_cast<uint32_t*>(R.codes + place * D + C * sub);
#pragma unroll
            for (int k = 0; k < C / 4; k++) dst[k] = q[i][k];
          }
        }
        continue;
      }
#pragma unroll
      for (int k = 0; k < C / 4; k++) {
        // t[m]: the lane's four tokens of channel 4 k + m
        const uint32_t a = __builtin_amdgcn_perm(q[1][k], q[0][k], 0x05010400u), b = __builtin_amdgcn_perm(q[3][k], q[2][k], 0x05010400u),
                       c = __builtin_amdgcn_perm(q[1][k], q[0][k], 0x07030602u), d = __builtin_amdgcn_perm(q[3][k], q[2][k], 0x07030602u);
        uint32_t t[4] = {__builtin_amdgcn_perm(b, a, 0x05040100u), __builtin_amdgcn_perm(b, a, 0x07060302u),
                         __builtin_amdgcn_perm(d, c, 0x05040100u), __builtin_amdgcn_perm(d, c, 0x07060302u)};
        // word m of row r of lanes to word r of row m
#pragma unroll
        for (int m = 0; m < 4; m += 2) {
          const auto s = __builtin_amdgcn_permlane16_swap(t[m], t[m + 1], false, false);
          t[m] = s[0];
          t[m + 1] = s[1];
        }
#pragma unroll
        for (int m = 0; m < 2; m++) {
          const auto s = __builtin_amdgcn_permlane32_swap(t[m], t[m + 2], false, false);
          t[m] = s[0];
          t[m + 2] = s[1];
        }
        uint8_t* const dst = R.codes + (C * sub + 4 * k + quarter) * tokens + p0;
        if (p0 >= R.at && p0 + 16 <= last) {
          *reinterpret_cast<v4u*>(dst) = v4u{t[0], t[1], t[2], t[3]};
        } else {
#pragma unroll
          for (int e = 0; e < 16; e++)
            if (p0 + e >= R.at && p0 + e < last) dst[e] = (uint8_t)(t[e >> 2] >> (8 * (e & 3)));
        }
      }
    }
  }
}

// Short runs, several at a time: D / 8 lanes hold a token's channels, eight each, and take the run's
// tokens one after the other.  Lanes without a run have count 0.
template <typename T, int D, bool INT8>
__device__ __forceinline__ void append_short(const Run& R, int tokens) {
  constexpr int kLanes = D / 8, W = 8 * (int)sizeof(T) / 4;
  const int lane = threadIdx.x & 63, sub = lane % kLanes;
  const T* const x = static_cast<const T*>(R.x) + 8 * sub;
  uint32_t w[W], top = 0;
  float before = 0.0f;
  if (R.count && R.at > 0) before = *R.scale;
  for (int i = 0; i < R.count; i++) {
    load_words<W>(x + i * R.row, w);
#pragma unroll
    for (int e = 0; e < 8; e++) top = max(top, __float_as_uint(element(x, w, e)) & 0x7FFFFFFFu);
  }
#pragma unroll
  for (int d = 1; d < kLanes; d *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, d));
  const float now = grown<INT8>(before, top);
  const Divider by(now, INT8 ? 127.0f : 448.0f);
  // pages whose scale grew, one after the other by the whole wave
  uint64_t carry = __ballot(R.count && R.at > 0 && now != before && sub == 0);
  while (carry) {
    const int from = __builtin_ctzll(carry);
    carry &= carry - 1;
    const uint64_t p = (uint64_t)R.codes;
    uint8_t* const codes = (uint8_t*)((uint64_t)__builtin_amdgcn_readlane((int)(p >> 32), from) << 32 |
                                      (uint32_t)__builtin_amdgcn_readlane((int)p, from));
    const Divider to(__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(now), from)), by.top);
    carry_over<D, INT8>(codes, __builtin_amdgcn_readlane(R.at, from), __builtin_amdgcn_readlane(R.values, from), tokens,
                        __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(before), from)), to);
  }
  if (!R.count) return;
  if (sub == 0) *R.scale = now;
  for (int i = 0; i < R.count; i++) {
    if (R.count > 1) load_words<W>(x + i * R.row, w);
    uint32_t q[2];
    codes_of<T, 8, INT8>(w, by, q);
    const int place = R.at + i;
    if (!R.values) {
      *reinterpret_cast<uint2*>(R.codes + place * D + 8 * sub) = make_uint2(q[0], q[1]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; e++) R.codes[(8 * sub + e) * tokens + place] = (uint8_t)(q[e >> 2] >> (8 * (e & 3)));
    }
  }
}

// A workgroup takes, for kItems of the (head, keys or values) pairs, the runs that begin among
// WINDOW tokens.  Every wave finds them by itself from the slots; no wave waits for another.  A new
// token is read once and its codes written once; a page's older codes are read and written only
// where its scale grows.  128 requests of one token, 8 heads of 128: 7.9 us, the latency of slots,
// scale and codes one after the other; 25 thousand tokens of prompts: 52 us, 3.0 TB/s of reads and
// writes, bound by the latency of a long run in its wave: loads, maximum, transposition, stores (31 us
// for the bytes alone).  Windows of a page's tokens instead of 16 took 45 us for 48 with pages of 32,
// 62 for 57 with pages of 64, and 25 for 16 at 100 prompts of up to 40 tokens.
constexpr int kAppendThreads = 256, kItems = 4;
constexpr int kFew = 4;    // tokens of a run that a few lanes take one by one

template <typename T, int D, bool INT8, int WINDOW>
__global__ __launch_bounds__(kAppendThreads) void append_kernel(Append A) {
  constexpr int kShort = 64 / (D / 8);            // short runs of a wave at a time
  constexpr int kWaves = kAppendThreads / 64;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tokens = 1 << A.shift;
  const int item0 = blockIdx.y * kItems, items = min(2 * A.heads - item0, kItems);
  for (int64_t w0 = (int64_t)blockIdx.x * WINDOW; w0 < A.n_tokens; w0 += (int64_t)gridDim.x * WINDOW) {
    // lane i: token w0 - 1 + i, as far as the longest run that begins here may reach
    auto slot_at = [&](int64_t t) {   // -1: not a token of the cache
      const int64_t s = t >= 0 && t < A.n_tokens ? A.slots[t] : -1;
      return s >= 0 && s < A.n_slots ? s : (int64_t)-1;
    };
    const int64_t mine = slot_at(w0 + lane), prior = slot_at(w0 + lane - 1);
    const int64_t next = slot_at(w0 + lane + 1);
    const uint64_t in_window = WINDOW == 64 ? ~0ull : (1ull << WINDOW) - 1;
    const uint64_t leaders = __ballot(mine >= 0 && (prior < 0 || prior >> A.shift != mine >> A.shift)) & in_window;
    // lanes whose token is followed by the page's next place: a run ends at the first without
    const uint64_t goes_on = __ballot(mine >= 0 && next == mine + 1 && (next & (tokens - 1)) != 0);
    auto slot_of = [&](int from) {
      return (int64_t)((uint64_t)__builtin_amdgcn_readlane((int)(mine >> 32), from) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)mine, from));
    };
    // tokens of the run that begins at lane `from` of the window
    auto count_of = [&](int from) {
      const uint64_t ends = ~(goes_on >> from);
      int count = ends ? 1 + (int)__builtin_ctzll(ends) : 64;
      if (from + count < 64) return count;
      const int64_t slot = slot_of(from);
      const int most = (int)min((int64_t)(tokens - (int)(slot & (tokens - 1))), A.n_tokens - (w0 + from));
      while (count < most) {
        const uint64_t other = ~__ballot(count + lane < most && slot_at(w0 + from + count + lane) == slot + count + lane);
        if (other) return count + (int)__builtin_ctzll(other);
        count += 64;
      }
      return most;
    };
    uint64_t shorts = 0;
    for (uint64_t left = leaders; left; left &= left - 1) {
      const int from = __builtin_ctzll(left);
      if (count_of(from) <= kFew) shorts |= 1ull << from;
    }
    const int units = __popcll(shorts) * items;
    for (int u0 = wave * kShort; u0 < units; u0 += kWaves * kShort) {
      const int u = u0 + lane / (D / 8);
      Run R = {};
      uint64_t left = shorts;   // the runs of this wave's lanes, one after the other
      for (int v = 0; v * items < u0 + kShort && left; v++, left &= left - 1) {
        if ((v + 1) * items <= u0) continue;
        const int from = __builtin_ctzll(left);
        const Run one = run_of<T, D>(A, w0 + from, slot_of(from), count_of(from), item0 + max(u - v * items, 0) % items);
        if (u / items == v) R = one;
      }
      append_short<T, D, INT8>(R, tokens);
    }
    for (uint64_t left = leaders & ~shorts; left; left &= left - 1) {
      const int from = __builtin_ctzll(left);
      for (int i = wave; i < items; i += kWaves)
        append_long<T, D, INT8>(run_of<T, D>(A, w0 + from, slot_of(from), count_of(from), item0 + i), tokens);
    }
  }
}

template <typename T, int D>
void append_launch(const Append& A, bool int8, hipStream_t stream) {
  // Few tokens spread over more workgroups (8 heads of 128; windows of 4 and of 16): 128 requests of
  // one token 8.5 and 12.3 us, 4 runs of 686 tokens in all 13.1 and 16.5, of 2439 18.6 and 17.2.
  const bool few = A.n_tokens <= 1024;
  const int64_t window = few ? 4 : 16;
  const dim3 grid((uint32_t)std::min<int64_t>((A.n_tokens + window - 1) / window, 1 << 22), (2 * A.heads + kItems - 1) / kItems);
  if (few && int8) hipLaunchKernelGGL((append_kernel<T, D, true, 4>), grid, dim3(kAppendThreads), 0, stream, A);
  else if (few) hipLaunchKernelGGL((append_kernel<T, D, false, 4>), grid, dim3(kAppendThreads), 0, stream, A);
  else if (int8) hipLaunchKernelGGL((append_kernel<T, D, true, 16>), grid, dim3(kAppendThreads), 0, stream, A);
  else hipLaunchKernelGGL((append_kernel<T, D, false, 16>), grid, dim3(kAppendThreads), 0, stream, A);
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

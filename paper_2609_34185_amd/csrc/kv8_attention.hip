// Softmax attention over the paged 8-bit key/value cache on gfx950 matrix instructions.
//
// Both products run transposed, S^T = K Q^T and O^T = V^T P^T, so that a lane holds scores of
// one query only (its column l mod 16) and the weights it computes are already where the second
// product wants them.  With v_mfma_f32_16x16x32_f16, lane l supplies eight values along the sum
// of row (A) or column (B) l mod 16, quarter l / 16 of the 32, and gets rows 4 (l / 16) + 0 .. 3
// of column l mod 16.  A chunk is 64 tokens in four row tiles; row m of tile i is token
//   16 (m / 4) + 4 i + m mod 4,
// so the 16 scores of a lane belong to 16 consecutive tokens, 16 (l / 16) + 0 .. 15: one page,
// one scale, and one 16-byte load of a value channel holds the codes of exactly these tokens.
//
// Codes become FP16 or BF16 without rounding (E4M3 and INT8 fit both).  A query row is scaled by a
// power of two to a largest value in [2^14, 2^15) and enters as FP16: BF16 has 8 bits of FP16's
// 11, and what falls below FP16's range is less than 2^-39 of the largest.  The scale of a key page
// and the inverse power multiply the FP32 scores.  A weight exp2(s - m), times the scale of its
// value page, enters the second product as the sum of two BF16 numbers: 16 bits, and the range of
// FP32, so that neither small weights nor wide page scales are lost.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <string>
#include <type_traits>

#include "../../include/entropack.h"
#include "common.h"
#include "kv8.h"

namespace ep {
namespace {

typedef _Float16 v2h __attribute__((ext_vector_type(2)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRows = 16;            // query rows of a tile: (token, head of the group) pairs
constexpr int kChunk = 64;           // tokens of a wave's step
constexpr int kWaves = 4;

struct Attn {
  const uint8_t *k, *v;
  const float *k_scale, *v_scale;
  const uint16_t* q;
  uint16_t* out;
  float* lse;
  const int32_t *cu, *len, *table;
  float *part_out, *part_lse;        // [splits][total_q][q_heads][D], [splits][total_q][q_heads]
  int64_t table_ld, total_q, q_row, out_row, n_pages, n_req;
  int32_t heads, group, shift, causal, window, splits, split_tokens;
  float scale;
};

__device__ __forceinline__ float minus_inf() { return -__builtin_inff(); }

// ---- codes to FP16 -----------------------------------------------------------------
// Four codes.  INT8: the byte with its top bit flipped, n = code + 128, is the low byte of the
// FP16 number 1024 + n, and 1024 + n - 1152 is exact.
template <bool INT8>
__device__ __forceinline__ void widen4(uint32_t c, v2h& a, v2h& b) {
  if (INT8) {
    const uint32_t n = c ^ 0x80808080u;
    const v2h off = {(_Float16)1152.0f, (_Float16)1152.0f};
    a = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, n, 0x04010400u)) - off;
    b = __builtin_bit_cast(v2h, __builtin_amdgcn_perm(0x64646464u, n, 0x04030402u)) - off;
  } else {
    a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c, 1.0f, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)c, 1.0f, true);
  }
}

template <bool INT8>
__device__ __forceinline__ v8h widen8(uint32_t lo, uint32_t hi) {
  v2h a, b, c, d;
  widen4<INT8>(lo, a, b);
  widen4<INT8>(hi, c, d);
  return v8h{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The same as BF16.  INT8: the values, as floats, have their upper halves alone.
template <bool INT8>
__device__ __forceinline__ v8b widen8_bf16(uint32_t lo, uint32_t hi) {
  typedef uint32_t v4w __attribute__((ext_vector_type(4)));
  v4w out;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const uint32_t c = (i < 2 ? lo : hi) >> (i & 1 ? 16 : 0);
    if (INT8)
      out[i] = __builtin_amdgcn_perm(__float_as_uint((float)(int8_t)(c >> 8)), __float_as_uint((float)(int8_t)c), 0x07060302u);
    else
      out[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)(i < 2 ? lo : hi), 1.0f, true)
                                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)(i < 2 ? lo : hi), 1.0f, false));
  }
  return __builtin_bit_cast(v8b, out);
}

// Zero the bytes that are E4M3's not-a-number (0x7F and 0xFF).
__device__ __forceinline__ uint32_t without_nans(uint32_t c) {
  const uint32_t n = (((c & 0x7F7F7F7Fu) + 0x01010101u) >> 7) & 0x01010101u;   // 1 in such a byte
  return c & ~(n * 0xFFu);
}

// ---- element types of queries and outputs --------------------------------------------
template <bool FP16>
__device__ __forceinline__ float widen(uint16_t x) {
  if (FP16) return (float)__builtin_bit_cast(_Float16, x);
  return __uint_as_float((uint32_t)x << 16);
}

template <bool FP16>
__device__ __forceinline__ uint16_t narrow(float f) {
  if (FP16) return __builtin_bit_cast(uint16_t, (_Float16)f);
  return __builtin_bit_cast(uint16_t, (__bf16)f);
}

// Over the four lanes that share a query (l mod 16).
__device__ __forceinline__ float max4(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum4(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// exp2 of x - m for a running maximum m that may still be -infinity (then nothing was seen, and
// x is -infinity too).
__device__ __forceinline__ float exp2_from(float x, float m) {
  return __builtin_amdgcn_exp2f(x - (m == minus_inf() ? 0.0f : m));
}

// What one workgroup works on: a request's queries and keys, and one kv head.  Positions in a
// request fit 32 bits.
struct Work {
  const int32_t* table;
  int64_t q0;            // first query
  int32_t len, m, h;
  uint32_t rows;         // (query, head of the group) pairs
};

__device__ __forceinline__ Work work_of(const Attn& A, int64_t b, int32_t h) {
  Work W;
  W.h = h;
  W.len = (int32_t)min((int64_t)max(A.len[b], 0), min(A.table_ld << A.shift, (int64_t)0x7FFFF000));
  W.q0 = min((int64_t)max(A.cu[b], 0), A.total_q);
  W.m = (int32_t)max(min((int64_t)max(A.cu[b + 1], 0), A.total_q) - W.q0, (int64_t)0);
  W.rows = (uint32_t)W.m * A.group;      // total_q * q_heads is at most 2^29
  W.table = A.table + b * A.table_ld;
  return W;
}

// The table's entry for token t of a request that has tokens (past the last one, the last one's),
// and the page that it stands for: -1 where there is none to be seen.  Apart, so that an entry can
// be on its way while something else is done.
__device__ __forceinline__ int32_t entry_at(const Attn& A, const Work& W, int32_t t) {
  return W.table[min(t, W.len - 1) >> A.shift];
}
__device__ __forceinline__ int32_t page_of(const Attn& A, const Work& W, int32_t t, int32_t entry) {
  return t < W.len && (uint32_t)entry < (uint32_t)A.n_pages ? entry : -1;
}

// Splits of a request's keys.
__device__ __forceinline__ int splits_of(const Attn& A, int32_t len) {
  return min(max((len + A.split_tokens - 1) / A.split_tokens, 1), A.splits);
}

// Item `index` of all requests' items, count(request) of them each: sets its request and its number
// there, or returns false if there are fewer.  The request's head is the caller's to set.  Every
// workgroup counts for itself, a request for each of its 256 threads at a time, so that a launch
// holds no workgroups for items that short requests do not have but at its end.  (Workgroups without work, in turn with those that have
// some, take half of the CUs away from them: a prompt of 64 tokens next to one of 8192 cost
// 1485 us instead of 876.)
template <typename Count>
__device__ __forceinline__ bool find_item(const Attn& A, uint32_t index, Work& request, uint32_t& item, uint32_t& items,
                                          Count count) {
  __shared__ uint32_t wave_sum[kWaves], found[3];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (A.n_req <= 64) {     // every wave by itself
    Work W = work_of(A, min((int64_t)lane, A.n_req - 1), 0);
    const uint32_t mine = lane < A.n_req ? count(W) : 0;
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    const uint64_t hit = __ballot(index >= sum - mine && index < sum);
    if (!hit) return false;
    const int b = __builtin_ctzll(hit);
    items = __builtin_amdgcn_readlane(mine, b);
    item = index - (__builtin_amdgcn_readlane(sum, b) - items);
    // what lane b has read
    request.q0 = __builtin_amdgcn_readlane((int)W.q0, b);        // below 2^31
    request.len = __builtin_amdgcn_readlane(W.len, b);
    request.m = __builtin_amdgcn_readlane(W.m, b);
    request.rows = __builtin_amdgcn_readlane(W.rows, b);
    request.table = A.table + b * A.table_ld;
    return true;
  }
  uint32_t before = 0;     // items of the requests before this round's; below 2^31 in all
  int64_t round = 0;
  if (threadIdx.x == 0) found[2] = 0;
  for (int64_t b0 = 0; b0 < A.n_req && before <= index; b0 += 64 * kWaves) {
    const int64_t b = b0 + threadIdx.x;
    const uint32_t mine = b < A.n_req ? count(work_of(A, b, 0)) : 0;
    uint32_t sum = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const uint32_t up = __shfl_up(sum, d);
      if (lane >= d) sum += up;
    }
    __syncthreads();       // the last round's sums are read
    if (lane == 63) wave_sum[wave] = sum;
    __syncthreads();
    uint32_t all = 0, first = before + sum - mine;
#pragma unroll
    for (int w = 0; w < kWaves; w++) {
      if (w < wave) first += wave_sum[w];
      all += wave_sum[w];
    }
    if (index >= first && index < first + mine) {
      found[0] = (uint32_t)(b - b0);
      found[1] = index - first;
      found[2] = mine;
    }
    round = b0;
    before += all;
  }
  __syncthreads();
  items = __builtin_amdgcn_readfirstlane(found[2]);
  if (items == 0) return false;
  item = __builtin_amdgcn_readfirstlane(found[1]);
  request = work_of(A, round + __builtin_amdgcn_readfirstlane(found[0]), 0);
  return true;
}

// Keys [low, high) are seen by query row `row`; 0 <= low, high <= len.
struct Span {
  int32_t low, high;
};

__device__ __forceinline__ Span span_of(const Attn& A, const Work& W, uint32_t row) {
  if (!A.causal) return {0, W.len};
  const int32_t high = max(W.len - W.m + (int32_t)(row / (uint32_t)A.group) + 1, 0);   // at most len
  return {A.window > 0 ? max(high - A.window, 0) : 0, high};
}

// A query row in FP16 at its own power of two: 16 channels of each 64 for a lane, those that its
// key pieces hold.  Returns what a score is to be multiplied with.
template <int D, bool FP16>
__device__ __forceinline__ float load_query(const Attn& A, const Work& W, uint32_t row, int quarter,
                                            v8h (&q)[D / 64][2]) {
  const uint32_t i = row / (uint32_t)A.group, g = row - i * A.group;
  const uint16_t* const src = A.q + (W.q0 + i) * A.q_row + ((int64_t)W.h * A.group + g) * D + 16 * quarter;
  v4u w[D / 64][2];
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < D / 64; p++)
#pragma unroll
    for (int e = 0; e < 2; e++) {
      w[p][e] = *reinterpret_cast<const v4u*>(src + 64 * p + 8 * e);
#pragma unroll
      for (int c = 0; c < 4; c++) {
        top = max(top, __float_as_uint(widen<FP16>((uint16_t)w[p][e][c])) & 0x7FFFFFFFu);
        top = max(top, __float_as_uint(widen<FP16>((uint16_t)(w[p][e][c] >> 16))) & 0x7FFFFFFFu);
      }
    }
  top = max(top, (uint32_t)__shfl_xor((int)top, 16));
  top = max(top, (uint32_t)__shfl_xor((int)top, 32));
  const uint32_t ex = max(top >> 23, 15u);                        // biased exponent of the largest
  const float lift = __uint_as_float((268u - ex) << 23);          // 2^(14 - exponent)
#pragma unroll
  for (int p = 0; p < D / 64; p++)
#pragma unroll
    for (int e = 0; e < 2; e++)
#pragma unroll
      for (int c = 0; c < 4; c++) {
        q[p][e][2 * c] = (_Float16)(widen<FP16>((uint16_t)w[p][e][c]) * lift);
        q[p][e][2 * c + 1] = (_Float16)(widen<FP16>((uint16_t)(w[p][e][c] >> 16)) * lift);
      }
  return __uint_as_float((ex - 14u) << 23) * (A.scale * kLog2e);
}

// A tile of 16 query rows of one request and kv head, against one share of its tokens.  The
// workgroup's waves take chunks of 64 tokens in turn and join their results in LDS.  A wave's codes
// go from memory to the registers of the matrix instructions, each once, the next chunk's while one
// is used; all query heads of a kv head share them.  Bound by memory: 64 requests of up to 16384 tokens,
// 64 query and 8 kv heads of 128, E4M3: 150 us with the joining, 4.6 TB/s.  Three short requests:
// 11.0 us, two launches and the latency of lengths, table, keys and values one after the other.
template <int D, bool INT8, bool FP16>
__global__ __launch_bounds__(64 * kWaves) void attention_rows_kernel(Attn A, uint32_t tiles) {
  constexpr int kPieces = D / 64;    // 16-byte pieces of a key for each lane
  constexpr int kTiles = D / 16;     // tiles of 16 value channels
  __shared__ float join_m[kWaves][kRows], join_l[kWaves][kRows];
  __shared__ float join_o[kWaves][kRows][D + 4];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  // Up to 256 requests, one round of counting, a workgroup takes the item (tile of rows, split of
  // keys) of that number.  With more there is work enough everywhere: a request has the workgroups
  // of `tiles` row tiles and all splits, and they take every tiles-th tile.
  Work W;
  uint32_t tile, split, stride = tiles;
  if (A.n_req <= 64 * kWaves) {
    uint32_t item, items;
    if (!find_item(A, blockIdx.x / A.heads, W, item, items,
                   [&](const Work& R) { return (R.rows + kRows - 1) / kRows * splits_of(A, R.len); }))
      return;
    // the tiles of one split follow each other: they read the same keys and values
    const uint32_t row_tiles = (W.rows + kRows - 1) / kRows;
    tile = item % row_tiles;
    split = item / row_tiles;
    stride = 1u << 27;         // more than there are
  } else {
    W = work_of(A, blockIdx.x / A.heads, 0);
    tile = blockIdx.y % tiles;
    split = blockIdx.y / tiles;
  }
  W.h = blockIdx.x % A.heads;
  const uint32_t splits = splits_of(A, W.len), rows = W.rows;
  if (split >= splits) return;
  const int page_tokens = 1 << A.shift;
  const int64_t head_codes = (int64_t)page_tokens * D, q_heads = (int64_t)A.heads * A.group;

  for (; tile * kRows < rows; tile += stride) {
    const uint32_t row = min(tile * kRows + col, rows - 1);
    const Span mine = span_of(A, W, row), first = span_of(A, W, tile * kRows),
               last = span_of(A, W, min(tile * kRows + kRows - 1, rows - 1));
    // the split's share of the keys [first.low, last.high) that some row sees
    const int share = (int)split * A.split_tokens;
    const int begin = max(share, first.low & ~(kChunk - 1));
    const int end = split == splits - 1 ? last.high : min(share + A.split_tokens, last.high);

    v8h q[kPieces][2];
    const float row_scale = load_query<D, FP16>(A, W, row, quarter, q);

    v4f o[kTiles];
  #pragma unroll
    for (int t = 0; t < kTiles; t++) o[t] = v4f{};
    float top = minus_inf(), total = 0.0f;

    // the table's entries for the tokens whose keys this lane loads and for those whose scores it
    // holds, read a chunk ahead
    int32_t entry_k = -1, entry_v = -1;
    if (begin < end) {
      entry_k = entry_at(A, W, begin + kChunk * wave + 16 * (col >> 2));
      entry_v = entry_at(A, W, begin + kChunk * wave + 16 * quarter);
    }
    for (int t0 = begin + kChunk * wave; t0 < end; t0 += kChunk * kWaves) {
      const int tk = t0 + 16 * (col >> 2), tv = t0 + 16 * quarter;
      const int32_t pk = page_of(A, W, tk, entry_k), pv = page_of(A, W, tv, entry_v);
      entry_k = entry_at(A, W, tk + kChunk * kWaves);
      entry_v = entry_at(A, W, tv + kChunk * kWaves);
      float ks = 0.0f, vs = 0.0f;
      v4u kc[4][kPieces], vc[kTiles];
      if (pk >= 0) {
        const uint8_t* const src = A.k + ((int64_t)pk * A.heads + W.h) * head_codes +
                                   ((tk & (page_tokens - 1)) + (col & 3)) * D + 16 * quarter;
  #pragma unroll
        for (int t = 0; t < 4; t++)
  #pragma unroll
          for (int p = 0; p < kPieces; p++) kc[t][p] = *reinterpret_cast<const v4u*>(src + 4 * t * D + 64 * p);
      } else {
  #pragma unroll
        for (int t = 0; t < 4; t++)
  #pragma unroll
          for (int p = 0; p < kPieces; p++) kc[t][p] = v4u{};
      }
      if (pv >= 0) {
        const uint8_t* const src =
            A.v + ((int64_t)pv * A.heads + W.h) * head_codes + (tv & (page_tokens - 1)) + col * page_tokens;
        ks = A.k_scale[(int64_t)pv * A.heads + W.h];
        vs = A.v_scale[(int64_t)pv * A.heads + W.h];
  #pragma unroll
        for (int t = 0; t < kTiles; t++) vc[t] = *reinterpret_cast<const v4u*>(src + 16 * t * page_tokens);
      } else {
  #pragma unroll
        for (int t = 0; t < kTiles; t++) vc[t] = v4u{};
      }

      float s[16];
      const float f = ks * row_scale;
  #pragma unroll
      for (int t = 0; t < 4; t++) {
        v4f acc = {};
  #pragma unroll
        for (int p = 0; p < kPieces; p++) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<INT8>(kc[t][p][0], kc[t][p][1]), q[p][0], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(widen8<INT8>(kc[t][p][2], kc[t][p][3]), q[p][1], acc, 0, 0, 0);
        }
  #pragma unroll
        for (int r = 0; r < 4; r++) s[4 * t + r] = acc[r] * f;
      }
      // where a row of the tile does not see all of the chunk, or a page is missing
      const bool cut = __any(t0 + kChunk > first.high || t0 < last.low || pk < 0 || pv < 0);
      uint32_t seen = 0xFFFFu;
      if (cut) {
        seen = 0;
  #pragma unroll
        for (int e = 0; e < 16; e++) {
          const bool yes = pv >= 0 && tv + e < mine.high && tv + e >= mine.low;
          seen |= (uint32_t)yes << e;
          s[e] = yes ? s[e] : minus_inf();
        }
        if (!INT8) {
  #pragma unroll
          for (int t = 0; t < kTiles; t++)
  #pragma unroll
            for (int c = 0; c < 4; c++) vc[t][c] = without_nans(vc[t][c]);
        }
      }
      float mx = s[0];
  #pragma unroll
      for (int e = 1; e < 16; e++) mx = fmaxf(mx, s[e]);
      const float now = fmaxf(top, max4(mx));
      const float keep = exp2_from(top, now), base = now == minus_inf() ? 0.0f : now;
      float sum = 0.0f;
      v8b hi[2], lo[2];
  #pragma unroll
      for (int e = 0; e < 16; e++) {
        const float p = __builtin_amdgcn_exp2f(s[e] - base);
        sum += p;
        float w = p * vs;
        if (cut) w = (seen >> e) & 1u ? w : 0.0f;
        const __bf16 wh = (__bf16)w;
        hi[e >> 3][e & 7] = wh;
        lo[e >> 3][e & 7] = (__bf16)(w - (float)wh);
      }
      total = total * keep + sum;
      top = now;
  #pragma unroll
      for (int t = 0; t < kTiles; t++) {
        const v8b va = widen8_bf16<INT8>(vc[t][0], vc[t][1]), vb = widen8_bf16<INT8>(vc[t][2], vc[t][3]);
  #pragma unroll
        for (int r = 0; r < 4; r++) o[t][r] *= keep;
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, hi[0], o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, hi[1], o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, lo[0], o[t], 0, 0, 0);
        o[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vb, lo[1], o[t], 0, 0, 0);
      }
    }

    // join the waves, each at its own maximum
    total = sum4(total);
    if (quarter == 0) {
      join_m[wave][col] = top;
      join_l[wave][col] = total;
    }
  #pragma unroll
    for (int t = 0; t < kTiles; t++)
      *reinterpret_cast<v4f*>(&join_o[wave][col][16 * t + 4 * quarter]) = o[t];
    __syncthreads();
    constexpr int kPer = kRows * D / (64 * kWaves);   // outputs of a thread, in one row
    const int r = threadIdx.x / (D / kPer), c0 = threadIdx.x % (D / kPer) * kPer;
    const uint32_t out_row = tile * kRows + r;
    if (out_row < rows) {
      float all = minus_inf(), l = 0.0f, v[kPer] = {};
  #pragma unroll
      for (int w = 0; w < kWaves; w++) all = fmaxf(all, join_m[w][r]);
  #pragma unroll
      for (int w = 0; w < kWaves; w++) {
        const float f = exp2_from(join_m[w][r], all);
        l += f * join_l[w][r];
  #pragma unroll
        for (int c = 0; c < kPer; c++) v[c] += f * join_o[w][r][c0 + c];
      }
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const float lse2 = l == 0.0f ? minus_inf() : all + __builtin_amdgcn_logf(l);
      const int64_t token = W.q0 + out_row / (uint32_t)A.group, head = W.h * A.group + out_row % (uint32_t)A.group;
      if (A.splits > 1) {
        const int64_t at = ((int64_t)split * A.total_q + token) * q_heads + head;
  #pragma unroll
        for (int c = 0; c < kPer; c++) A.part_out[at * D + c0 + c] = v[c] * inv;
        if (c0 == 0) A.part_lse[at] = lse2;
      } else {
        uint16_t* const dst = A.out + token * A.out_row + head * D + c0;
  #pragma unroll
        for (int c = 0; c < kPer; c++) dst[c] = narrow<FP16>(v[c] * inv);
        if (c0 == 0 && A.lse) A.lse[token * q_heads + head] = lse2 * kLn2;
      }
    }
    __syncthreads();     // the joined results are read
  }
}

// ---- many query rows -----------------------------------------------------------------
// A workgroup's four waves hold 32 query rows each (two column tiles; 16 for 256 channels) and share the chunks of 64
// tokens, which direct loads bring to LDS as they lie in the cache, one chunk ahead.  Every wave
// widens the codes it reads, so LDS and its bandwidth hold 8 bits a value.
//
// A weight enters the second product with its page's value scale in the exponent, as FP16 of
//   2^(s + log2 vs - peak + 12),
// where a row's peak follows the largest s + log2 vs among the keys that it sees, whatever the scales
// of others are: 11 bits down to 2^-26 of the row's largest product of weight and scale, 0 below
// 2^-37 of it.  (Two BF16 numbers, as in the kernel for few rows, would keep those too, for half as
// many matrix instructions again: 1427 us for 1177, 929 for 744 with 64 channels.)  The peak moves only
// when it is passed by more than 3, so that the sums are rarely rescaled and FP16 holds 2^15.  The sum
// of the weights themselves, which pages of small values and of zeros count in all the same, is kept
// apart by each lane, at a maximum of its own.
//
// Bound by how little the two units work at once: the vector unit, which widens codes and makes
// weights, is busy 68 % of the cycles and the matrix unit 35 %, together about all of them.  What is
// left is to issue a chunk's K Q^T under the exponentials of the one before.  Two causal prompts of up
// to 8192 tokens, 40 query and 8 kv heads of 128, E4M3: 1055 us, 0.86 PFLOP/s.  Codes widened once for
// the workgroup and kept in LDS as FP16 take 16 % off the vector unit and are no faster (1104 us for
// 1109 in one run; 64 channels 793 for 726): LDS then moves twice the bytes.
constexpr int kPromptWaves = kWaves;
constexpr int col_tiles(int dim) { return dim <= 128 ? 2 : 1; }   // what 256 registers hold
constexpr int prompt_rows(int dim) { return kPromptWaves * col_tiles(dim) * 16; }
constexpr float kLift = 12.0f, kSlack = 3.0f, kSumSlack = 40.0f, kNothing = -40.0f;

typedef __attribute__((address_space(3))) uint8_t lds_u8;
typedef __attribute__((address_space(1))) const uint8_t global_u8;

// One instruction, without the steps that quiet an operand first; a NaN stays one.
__device__ __forceinline__ float max3(float a, float b, float c) {
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c);
}

// The largest over the four lanes that share a query, without LDS.
__device__ __forceinline__ float swap_max4(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = max3(__uint_as_float(a[0]), __uint_as_float(a[1]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return max3(__uint_as_float(a[0]), __uint_as_float(a[1]), __uint_as_float(a[1]));
}

// Places in LDS.  A 16-byte read is served to 16 lanes at a time, of the first 32 lanes 0-3, 12-15
// and 20-27 together and then the others (measured), and is free of conflicts if they meet 16
// different columns of a 256-byte bank row.
// Chunk j of token row r among its row's chunks; lane l reads chunk 4 p + l / 16 of row 16 (l / 4
// mod 4) + 4 i + l mod 4.
template <int D>
__device__ __forceinline__ uint32_t key_place(uint32_t j, uint32_t r) {
  if (D == 64) return j ^ (-(r >> 4) & 3);
  if (D == 128) return j ^ (((r >> 1) & 1) | ((r >> 4) & 3) << 1);
  return j ^ ((r & 3) | ((r >> 4) & 3) << 2);
}
// Run j (of 16 tokens) of value channel d among its four; lane l reads run l / 16 of channel l mod 16.
__device__ __forceinline__ uint32_t value_place(uint32_t j, uint32_t d) { return j ^ (-(d >> 2) & 3); }

template <int D, bool INT8, bool FP16>
__global__ __launch_bounds__(64 * kPromptWaves, 2) void attention_prompt_kernel(Attn A) {
  constexpr int kColTiles = col_tiles(D), kPromptRows = prompt_rows(D);
  constexpr int kPieces = D / 64, kTiles = D / 16;
  constexpr int kBytes = kChunk * D;                       // of a chunk's keys, and of its values
  constexpr int kLoads = kBytes / 1024 / kPromptWaves;     // direct loads of a wave for each
  constexpr int kPass = D <= 128 ? 2 : 1;                  // chunks between two barriers
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[2 * kPass][2 * kBytes];

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  Work W;
  uint32_t tile, tiles;
  if (!find_item(A, blockIdx.x / A.heads, W, tile, tiles, [&](const Work& R) { return (R.rows + kPromptRows - 1) / kPromptRows; }))
    return;
  W.h = blockIdx.x % A.heads;
  tile = tiles - 1 - tile;     // the longest rows of a causal request first
  const int split = blockIdx.y, page_tokens = 1 << A.shift;
  const int64_t q_heads = (int64_t)A.heads * A.group;
  // the run of 16 tokens that this lane's value loads are of (a KiB of values is 16 channels of
  // four runs)
  const uint32_t v_run = value_place(lane & 3, lane >> 2);

  const uint32_t tile_first = tile * kPromptRows, wave_first = tile_first + 16 * kColTiles * wave;
  const Span first = span_of(A, W, tile_first), last = span_of(A, W, min(tile_first + kPromptRows - 1, W.rows - 1));
  const int splits = splits_of(A, W.len);
  if (split >= splits) return;
  const int share = split * A.split_tokens;
  const int begin = max(share, first.low & ~(kChunk - 1));
  const int end = split == splits - 1 ? last.high : min(share + A.split_tokens, last.high);
  // keys [wave_a.low, wave_end) are seen by some row of this wave, [wave_b.low, wave_a.high) by all
  const Span wave_a = span_of(A, W, min(wave_first, W.rows - 1)),
             wave_b = span_of(A, W, min(wave_first + 16 * kColTiles - 1, W.rows - 1));
  const int wave_end = wave_first < W.rows ? wave_b.high : 0;

  Span span[kColTiles];
  // peak: of s + log2 vs, the row's; sums of weights 2^(s - top): this lane's tokens'
  float row_scale[kColTiles], peak[kColTiles], top[kColTiles], total[kColTiles];
  v8h q[kColTiles][kPieces][2];
  v4f o[kTiles][kColTiles];
#pragma unroll
  for (int n = 0; n < kColTiles; n++) {
    const uint32_t row = min(wave_first + 16 * n + col, W.rows - 1);
    span[n] = span_of(A, W, row);
    row_scale[n] = load_query<D, FP16>(A, W, row, quarter, q[n]);
    peak[n] = top[n] = minus_inf();
    total[n] = 0.0f;
#pragma unroll
    for (int t = 0; t < kTiles; t++) o[t][n] = v4f{};
  }

  // Direct loads of chunk t0, whose run `quarter` lies in `page`: this wave takes every fourth KiB
  // of the keys and of the values.  Runs with nothing to fetch take page 0, whose scores are
  // masked and whose codes are cleaned.
  uint32_t k_off[kLoads];    // of this lane's 16 bytes in a run of 16 tokens
#pragma unroll
  for (int i = 0; i < kLoads; i++) {
    const uint32_t at = 1024 * (kPromptWaves * i + wave) + 16 * lane, r = at / D;
    k_off[i] = r % 16 * D + 16 * key_place<D>(at % D / 16, r);
  }
  const uint32_t v_off = (16 * wave + (lane >> 2)) * page_tokens;
  const int code_shift = A.shift + (D == 64 ? 6 : D == 128 ? 7 : 8);   // log2 of a page and head's codes
  auto fetch = [&](int t0, int32_t page, uint32_t stage) {
    lds_u8* const dst = (lds_u8*)lds_mem[stage] + 1024 * wave;
    const int32_t in = max(page, 0);
    // of the four runs: where their page and head begins
    int64_t from[4];
#pragma unroll
    for (int j = 0; j < 4; j++)
      from[j] = (int64_t)((uint32_t)__builtin_amdgcn_readlane(in, 16 * j) * (uint32_t)A.heads + W.h) << code_shift;
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
      const uint32_t run = 1024 * (kPromptWaves * i + wave) / (16 * D);   // the same in all lanes
      const int64_t at = run < 2 ? (run < 1 ? from[0] : from[1]) : (run < 3 ? from[2] : from[3]);
      const uint8_t* const src = A.k + at + ((t0 + 16 * (int)run) & (page_tokens - 1)) * D;
      __builtin_amdgcn_global_load_lds((global_u8*)(src + k_off[i]), dst + 1024 * kPromptWaves * i, 16, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < 4; j++) from[j] += (t0 + 16 * j) & (page_tokens - 1);
    const int64_t at = v_run & 2 ? (v_run & 1 ? from[3] : from[2]) : (v_run & 1 ? from[1] : from[0]);
    const uint8_t* const src = A.v + (at + v_off);
#pragma unroll
    for (int i = 0; i < kLoads; i++)
      __builtin_amdgcn_global_load_lds((global_u8*)(src + 16 * kPromptWaves * i * page_tokens),
                                       dst + kBytes + 1024 * kPromptWaves * i, 16, 0, 0);
  };

  // One chunk.  cut: some row of the wave does not see all of it.
  auto chunk = [&](int t0, uint32_t stage, int32_t page, float ks, float vs, bool cut) {
    const lds_u8* const keys = (const lds_u8*)lds_mem[stage];
    const lds_u8* const values = keys + kBytes;
    v4f s[4][kColTiles];
#pragma unroll
    for (int t = 0; t < 4; t++) {
#pragma unroll
      for (int n = 0; n < kColTiles; n++) s[t][n] = v4f{};
      const uint32_t r = 16 * (col >> 2) + 4 * t + (col & 3);
#pragma unroll
      for (int p = 0; p < kPieces; p++) {
        const v4u c = *reinterpret_cast<const __attribute__((address_space(3))) v4u*>(
            keys + r * D + 16 * key_place<D>(4 * p + quarter, r));
        const v8h a = widen8<INT8>(c[0], c[1]), b = widen8<INT8>(c[2], c[3]);
#pragma unroll
        for (int n = 0; n < kColTiles; n++) {
          s[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, q[n][p][0], s[t][n], 0, 0, 0);
          s[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, q[n][p][1], s[t][n], 0, 0, 0);
        }
      }
    }
    // the values' codes are on their way while the weights are made
    v4u vc[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; t++) {
      const uint32_t d = 16 * t + col;
      vc[t] = *reinterpret_cast<const __attribute__((address_space(3))) v4u*>(
          values + d * kChunk + 16 * value_place(quarter, d));
    }
    float f[kColTiles];
#pragma unroll
    for (int n = 0; n < kColTiles; n++) f[n] = ks * row_scale[n];
    if (cut) {
      if (!INT8) {
#pragma unroll
        for (int t = 0; t < kTiles; t++)
#pragma unroll
          for (int i = 0; i < 4; i++) vc[t][i] = without_nans(vc[t][i]);
      }
      // scores as they are, -infinity where unseen; a value scale that is not finite makes the
      // rows that see its page not-a-number, and no others
      const int tv = t0 + 16 * quarter;
      const bool bad = !(fabsf(vs) < __builtin_inff());
#pragma unroll
      for (int n = 0; n < kColTiles; n++) {
        const int low = page >= 0 ? span[n].low - tv : 16, high = span[n].high - tv;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const float x = bad ? __builtin_nanf("") : s[e >> 2][n][e & 3] * f[n];
          s[e >> 2][n][e & 3] = e >= low && e < high ? x : minus_inf();
        }
        f[n] = 1.0f;
      }
      if (bad) vs = 0.0f;
    }
    // log2 of the page's value scale, -infinity for one of zeros
    const float log_vs = vs < 0x1p-100f ? __builtin_amdgcn_logf(vs * 0x1p100f) - 100.0f : __builtin_amdgcn_logf(vs);
    v8h w[2][kColTiles];
#pragma unroll
    for (int n = 0; n < kColTiles; n++) {
      float mx = max3(s[0][n][0], s[0][n][1], s[0][n][2]);
      mx = max3(mx, s[0][n][3], s[1][n][0]);
      mx = max3(mx, s[1][n][1], s[1][n][2]);
      mx = max3(mx, s[1][n][3], s[2][n][0]);
      mx = max3(mx, s[2][n][1], s[2][n][2]);
      mx = max3(mx, s[2][n][3], s[3][n][0]);
      mx = max3(mx, s[3][n][1], s[3][n][2]);
      mx = max3(mx, s[3][n][3], s[3][n][3]) * f[n];
      const float high = swap_max4(mx + log_vs);
      if (__any(high > peak[n] + kSlack)) {
        const float now = high > peak[n] + kSlack ? high : peak[n];
        const float keep = exp2_from(peak[n], now);
#pragma unroll
        for (int t = 0; t < kTiles; t++) o[t][n] *= keep;
        peak[n] = now;
      }
      if (__any(mx > top[n] + kSumSlack)) {
        const float now = mx > top[n] + kSumSlack ? mx : top[n];
        total[n] *= exp2_from(top[n], now);
        top[n] = now;
      }
      // where the lane's weights are nothing in FP16 (as those of a page of zeros are) they still have
      // to be summed, and are lifted until the largest is 2^-40
      const float lift = log_vs + (kLift - (peak[n] == minus_inf() ? 0.0f : peak[n]));
      const float least = kNothing - max3(mx, -0x1p126f, -0x1p126f);
      const float base = max3(lift, least, least);
      const float back = __builtin_amdgcn_exp2f(-(top[n] == minus_inf() ? 0.0f : top[n]) - base);
      float sum = 0.0f;
#pragma unroll
      for (int t = 0; t < 4; t++)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][n][r], f[n], base));
          sum += e;
          w[t >> 1][n][4 * (t & 1) + r] = (_Float16)e;
        }
      total[n] = __builtin_fmaf(sum, back, total[n]);
    }
#pragma unroll
    for (int t = 0; t < kTiles; t++) {
      const v8h a = widen8<INT8>(vc[t][0], vc[t][1]), b = widen8<INT8>(vc[t][2], vc[t][3]);
#pragma unroll
      for (int n = 0; n < kColTiles; n++) {
        o[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a, w[0][n], o[t][n], 0, 0, 0);
        o[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b, w[1][n], o[t][n], 0, 0, 0);
      }
    }
  };

  // pages and scales of the lane's runs of 16 tokens, and the table's entries of the next pass's:
  // loaded a pass before they are used, as the codes are
  int32_t page[kPass], entry[kPass];
  float ks[kPass], vs[kPass];
  auto scales = [&](int32_t p, float& k, float& v) {
    const uint32_t at = (uint32_t)max(p, 0) * (uint32_t)A.heads + W.h;
    k = A.k_scale[at];
    v = A.v_scale[at];
  };
#pragma unroll
  for (int g = 0; g < kPass; g++) {
    const int t = begin + kChunk * g;
    page[g] = entry[g] = -1;
    ks[g] = vs[g] = 0.0f;
    if (t < end) {
      page[g] = page_of(A, W, t + 16 * quarter, entry_at(A, W, t + 16 * quarter));
      fetch(t, page[g], g);
      scales(page[g], ks[g], vs[g]);
      entry[g] = entry_at(A, W, t + kChunk * kPass + 16 * quarter);
    }
  }
  uint32_t stage = 0;
  for (int t0 = begin; t0 < end; t0 += kChunk * kPass) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0x70);   // vmcnt(0) lgkmcnt(0): this pass has landed, the last one is read
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    int32_t next[kPass], after[kPass];
    float next_ks[kPass], next_vs[kPass];
#pragma unroll
    for (int g = 0; g < kPass; g++) {
      const int t = t0 + kChunk * (kPass + g);
      next[g] = after[g] = -1;
      next_ks[g] = next_vs[g] = 0.0f;
      if (t < end) {
        next[g] = page_of(A, W, t + 16 * quarter, entry[g]);
        fetch(t, next[g], (stage ^ kPass) + g);
        scales(next[g], next_ks[g], next_vs[g]);
        after[g] = entry_at(A, W, t + kChunk * kPass + 16 * quarter);
      }
    }
#pragma unroll 1
    for (int g = 0; g < kPass; g++) {
      const int t = t0 + kChunk * g;
      if (t < min(wave_end, end) && t + kChunk > wave_a.low) {
        const int32_t p = kPass > 1 && g ? page[kPass - 1] : page[0];
        const float k = kPass > 1 && g ? ks[kPass - 1] : ks[0], v = kPass > 1 && g ? vs[kPass - 1] : vs[0];
        const bool cut = t + kChunk > wave_a.high || t < wave_b.low || __any(p < 0);
        chunk(t, stage + g, p, p < 0 ? 0.0f : k, p < 0 ? 0.0f : v, cut);
      }
    }
#pragma unroll
    for (int g = 0; g < kPass; g++) {
      page[g] = next[g];
      entry[g] = after[g];
      ks[g] = next_ks[g];
      vs[g] = next_vs[g];
    }
    stage ^= kPass;
  }
#pragma unroll
  for (int n = 0; n < kColTiles; n++) {
    const uint32_t row = wave_first + 16 * n + col;
    const float all = swap_max4(top[n]), l = sum4(total[n] * exp2_from(top[n], all));
    if (row >= W.rows) continue;
    // o 2^(peak - 12) / (l 2^all), in two steps since small pages' powers may lie outside FP32
    const float half = 0.5f * (peak[n] - kLift - all), inv = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(half) / l;
    const float rest = l == 0.0f ? 0.0f : __builtin_amdgcn_exp2f(half);
    const float lse2 = l == 0.0f ? minus_inf() : all + __builtin_amdgcn_logf(l);
    const int64_t token = W.q0 + row / (uint32_t)A.group, head = W.h * A.group + row % (uint32_t)A.group;
    if (A.splits > 1) {
      const int64_t at = ((int64_t)split * A.total_q + token) * q_heads + head;
#pragma unroll
      for (int t = 0; t < kTiles; t++)
        *reinterpret_cast<v4f*>(A.part_out + at * D + 16 * t + 4 * quarter) = o[t][n] * inv * rest;
      if (quarter == 0) A.part_lse[at] = lse2;
    } else {
      uint16_t* const dst = A.out + token * A.out_row + head * D + 4 * quarter;
#pragma unroll
      for (int t = 0; t < kTiles; t++) {
        typedef uint16_t v4s __attribute__((ext_vector_type(4)));
        v4s x;
#pragma unroll
        for (int r = 0; r < 4; r++) x[r] = narrow<FP16>(o[t][n][r] * inv * rest);
        *reinterpret_cast<v4s*>(dst + 16 * t) = x;
      }
      if (quarter == 0 && A.lse) A.lse[token * q_heads + head] = lse2 * kLn2;
    }
  }
}

// Joins the splits of a query row, a workgroup for each: sum_s 2^(lse_s - max) o_s / sum_s 2^(lse_s -
// max).  D / 4 lanes hold a row's channels, and the workgroup's groups of so many lanes take the
// splits in turn; their sums meet in LDS in a fixed order.  64 requests of 64 heads in 5 splits: 9 us,
// three of 40 heads 3.6, which is a launch.
template <int D, bool FP16>
__global__ __launch_bounds__(256) void attention_join_kernel(Attn A) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes;
  __shared__ float sums[kGroups][D + 4];     // a group's o, then its sum of weights
  const int64_t q_heads = (int64_t)A.heads * A.group, all_rows = A.total_q * q_heads;
  const Work W = work_of(A, blockIdx.x, 0);
  const int group = threadIdx.x / kLanes, c0 = threadIdx.x % kLanes * 4, splits = splits_of(A, W.len);
  for (int64_t row = W.q0 * q_heads + blockIdx.y; row < (W.q0 + W.m) * q_heads; row += gridDim.y) {
    float all = minus_inf(), l = 0.0f;
    for (int s = threadIdx.x & 63; s < splits; s += 64) all = fmaxf(all, A.part_lse[s * all_rows + row]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all = fmaxf(all, __shfl_xor(all, d));
    v4f v = {};
#pragma unroll 4
    for (int s = group; s < splits; s += kGroups) {
      const float f = exp2_from(A.part_lse[s * all_rows + row], all);
      const v4f o = *reinterpret_cast<const v4f*>(A.part_out + (s * all_rows + row) * D + c0);
      l += f;
#pragma unroll
      for (int c = 0; c < 4; c++) v[c] += f == 0.0f ? 0.0f : f * o[c];
    }
    *reinterpret_cast<v4f*>(&sums[group][c0]) = v;
    if (c0 == 0) sums[group][D] = l;
    __syncthreads();
    if (group == 0) {
#pragma unroll
      for (int g = 1; g < kGroups; g++) {
        v += *reinterpret_cast<const v4f*>(&sums[g][c0]);
        l += sums[g][D];
      }
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      uint16_t* const dst = A.out + row / q_heads * A.out_row + row % q_heads * D + c0;
#pragma unroll
      for (int c = 0; c < 4; c++) dst[c] = narrow<FP16>(v[c] * inv);
      if (c0 == 0 && A.lse) A.lse[row] = l == 0.0f ? minus_inf() : (all + __builtin_amdgcn_logf(l)) * kLn2;
    }
    __syncthreads();
  }
}

// ---- host ------------------------------------------------------------------------------
const char* call_fault(const ep_kv8_cache* c, const ep_kv8_attn* a) {
  if (const char* why = cache_fault(c)) return why;
  if (!a) return "null call";
  if (a->q_heads <= 0 || a->q_heads > 1 << 20 || a->q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads";
  if (a->dtype != EP_BF16 && a->dtype != EP_FP16) return "queries must be BF16 or FP16";
  // a grid holds less than 2^32 threads: one workgroup for each (request, head) and each full tile
  if (a->n_req <= 0 || a->n_req > (1 << 22) / c->kv_heads) return "n_req * kv_heads outside 1 .. 2^22";
  if (a->table_ld <= 0 || a->table_ld > 0x7FFFFFFF) return "table_ld outside 1 .. 2^31 - 1";
  if (a->total_q < 0 || a->total_q > 0x7FFFFFFF) return "total_q outside 0 .. 2^31 - 1";
  if (a->total_q * a->q_heads > 1 << 29) return "total_q * q_heads above 2^29";
  if (a->window < 0 || (a->window && !a->causal)) return "a window needs causal, and must not be negative";
  if (!(a->scale >= 0.0f && a->scale < __builtin_inff())) return "scale must be finite and not negative";
  if (a->max_q <= 0 || a->max_len < 0) return "max_q must be positive and max_len not negative";
  const int64_t width = (int64_t)a->q_heads * c->head_dim;
  if ((a->q_row && a->q_row < width) || (a->out_row && a->out_row < width) || a->q_row % 8 || a->out_row % 8)
    return "rows must hold q_heads * head_dim elements and be 16-byte aligned";
  if (a->total_q && (!a->d_q || !a->d_out || !a->d_cu_q || !a->d_len || !a->d_table)) return "null pointer";
  if ((reinterpret_cast<uintptr_t>(a->d_q) | reinterpret_cast<uintptr_t>(a->d_out)) & 15)
    return "queries and outputs must be 16-byte aligned";
  return nullptr;
}

// How a call's keys are shared out.  Workgroups are (request and head, split, row tile).
struct Plan {
  int64_t tiles;         // row tiles of a launch: of all requests, or (not counted) of each
  int64_t splits, split_tokens, max_q;
  bool prompt, counted;
};

constexpr int64_t kMostGroups = (1 << 24) - 1;   // of 256 threads in one row of a grid

Plan plan_of(const ep_kv8_cache& c, const ep_kv8_attn& a) {
  Plan P;
  const int64_t group = a.q_heads / c.kv_heads, rows = a.max_q * group;
  P.max_q = a.max_q;
  // At 8 kv heads, few-row kernel and prompt kernel: 16 rows 29 and 59 us (16 requests of up to 8000
  // tokens), 36 and 37 (64 of up to 1000); 32 rows 45 and 63, 56 and 37; 48 rows 52 and 66, 76 and 42.
  // (Also with far more queries than max_q says, whose tiles of 16 rows would not fit a grid.)
  P.prompt = rows > 32 || (a.n_req <= 64 * kWaves && (a.total_q * group / kRows + a.n_req) * c.kv_heads > kMostGroups);
  // the tiles of all requests are at most those that total_q would fill, and one more for each
  const int64_t tile_rows = P.prompt ? prompt_rows(c.head_dim) : kRows;
  P.counted = P.prompt || a.n_req <= 64 * kWaves;
  P.tiles = P.counted ? a.total_q * group / tile_rows + a.n_req : std::min<int64_t>((rows + kRows - 1) / kRows, 64);
  const int64_t max_len = std::min(std::max(a.max_len, 1), 1 << 30);   // the last split takes what is past it
  // Up to ten workgroups for a CU of at least 1024 tokens (64 requests of up to 16384 tokens in 5
  // splits: 150 us, in 2 168, in 10 158), but of 256 where that leaves less than four (3 requests
  // of up to 1999 tokens, 8 kv heads: 11.3 us in 8 splits, 26.5 in one).  Of few rows, a request's tiles
  // share what they read and count once.  Of many, partial results cost more the more rows there are:
  // 512 queries after 15872 tokens, 40 query heads, 306 us in 15 splits, 288 in 8, 319 in 4, 478 in
  // one; 128 after 16256 100, 108, 137 and 467.
  const int64_t groups = (P.prompt ? P.tiles : a.n_req) * c.kv_heads;
  P.splits = std::min(2560 / groups, std::max(max_len / 1024, std::min(1024 / groups, (max_len + 255) / 256)));
  if (P.counted && !P.prompt) P.splits = std::min(P.splits, kMostGroups / (P.tiles * c.kv_heads));
  P.splits = std::min<int64_t>(std::max<int64_t>(P.splits, 1), 256);
  P.split_tokens = (max_len + P.splits - 1) / P.splits;
  P.split_tokens = (P.split_tokens + kChunk - 1) / kChunk * kChunk;
  return P;
}

uint64_t plan_bytes(const Plan& P, const ep_kv8_cache& c, const ep_kv8_attn& a) {
  if (P.splits == 1) return 0;
  return (uint64_t)P.splits * a.total_q * a.q_heads * (c.head_dim + 1) * sizeof(float);
}

template <int D, bool INT8, bool FP16>
void attention_launch(const Attn& A, const Plan& P, int64_t n_req, hipStream_t stream) {
  if (P.prompt)
    hipLaunchKernelGGL((attention_prompt_kernel<D, INT8, FP16>), dim3((uint32_t)(P.tiles * A.heads), (uint32_t)P.splits),
                       dim3(64 * kPromptWaves), 0, stream, A);
  else
    hipLaunchKernelGGL((attention_rows_kernel<D, INT8, FP16>),
                       P.counted ? dim3((uint32_t)(P.tiles * P.splits * A.heads))
                                 : dim3((uint32_t)(n_req * A.heads), (uint32_t)(P.splits * P.tiles)),
                       dim3(64 * kWaves), 0, stream, A, (uint32_t)P.tiles);
  if (P.splits > 1) {
    const int64_t rows = P.max_q * A.heads * A.group;
    hipLaunchKernelGGL((attention_join_kernel<D, FP16>),
                       dim3((uint32_t)n_req, (uint32_t)std::min<int64_t>(rows, 65535)), dim3(256), 0,
                       stream, A);
  }
}

template <int D>
void attention_launch(const Attn& A, const Plan& P, int64_t n_req, bool int8, bool fp16, hipStream_t stream) {
  if (int8 && fp16) attention_launch<D, true, true>(A, P, n_req, stream);
  else if (int8) attention_launch<D, true, false>(A, P, n_req, stream);
  else if (fp16) attention_launch<D, false, true>(A, P, n_req, stream);
  else attention_launch<D, false, false>(A, P, n_req, stream);
}

}  // namespace
}  // namespace ep

extern "C" uint64_t ep_kv8_attention_workspace(const ep_kv8_cache* cache, const ep_kv8_attn* call) {
  if (ep::call_fault(cache, call)) return 0;
  return ep::plan_bytes(ep::plan_of(*cache, *call), *cache, *call);
}

extern "C" int ep_kv8_attention(const ep_kv8_cache* cache, const ep_kv8_attn* call, void* d_workspace,
                                uint64_t ws_bytes, void* hip_stream) {
  if (const char* why = ep::call_fault(cache, call))
    return ep::fail(EP_ERR_ARG, (std::string("ep_kv8_attention: ") + why).c_str());
  if (call->total_q == 0) return EP_OK;
  const ep::Plan P = ep::plan_of(*cache, *call);
  const uint64_t bytes = ep::plan_bytes(P, *cache, *call);
  if (bytes && (!d_workspace || ws_bytes < bytes || (reinterpret_cast<uintptr_t>(d_workspace) & 15)))
    return ep::fail(EP_ERR_ARG, "ep_kv8_attention: workspace missing, short or misaligned");
  const int64_t width = (int64_t)call->q_heads * cache->head_dim;
  ep::Attn A = {};
  A.k = static_cast<const uint8_t*>(cache->d_k);
  A.v = static_cast<const uint8_t*>(cache->d_v);
  A.k_scale = cache->d_k_scale;
  A.v_scale = cache->d_v_scale;
  A.q = static_cast<const uint16_t*>(call->d_q);
  A.out = static_cast<uint16_t*>(call->d_out);
  A.lse = call->d_lse;
  A.cu = call->d_cu_q;
  A.len = call->d_len;
  A.table = call->d_table;
  A.part_out = static_cast<float*>(d_workspace);
  A.part_lse = A.part_out + P.splits * call->total_q * width;
  A.table_ld = call->table_ld;
  A.total_q = call->total_q;
  A.q_row = call->q_row ? call->q_row : width;
  A.out_row = call->out_row ? call->out_row : width;
  A.n_pages = cache->n_pages;
  A.n_req = call->n_req;
  A.heads = cache->kv_heads;
  A.group = call->q_heads / cache->kv_heads;
  A.shift = ep::page_shift(cache->page_tokens);
  A.causal = call->causal;
  A.window = call->window;
  A.splits = (int32_t)P.splits;
  A.split_tokens = (int32_t)std::min<int64_t>(P.split_tokens, 0x7FFFFFFF);
  A.scale = call->scale;
  const bool int8 = cache->dtype == EP_INT8, fp16 = call->dtype == EP_FP16;
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (cache->head_dim == 64) ep::attention_launch<64>(A, P, call->n_req, int8, fp16, stream);
  else if (cache->head_dim == 128) ep::attention_launch<128>(A, P, call->n_req, int8, fp16, stream);
  else ep::attention_launch<256>(A, P, call->n_req, int8, fp16, stream);
  if (hipGetLastError() != hipSuccess) return ep::fail(EP_ERR_HIP, "ep_kv8_attention: launch failed");
  return EP_OK;
}

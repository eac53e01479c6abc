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
  int64_t table_ld, total_q, q_row, out_row, n_pages;
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
  const uint32_t u = __float_as_uint(f);
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return (uint16_t)((u >> 16) | 0x40u);
  return (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
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

// A tile of 16 query rows of one request and kv head, against one share of its tokens.  The
// workgroup's waves take chunks of 64 tokens in turn and join their results in LDS.
template <int D, bool INT8, bool FP16>
__global__ __launch_bounds__(64 * kWaves) void attention_rows_kernel(Attn A) {
  constexpr int kPieces = D / 64;    // 16-byte pieces of a key for each lane
  constexpr int kTiles = D / 16;     // tiles of 16 value channels
  __shared__ float join_m[kWaves][kRows], join_l[kWaves][kRows];
  __shared__ float join_o[kWaves][kRows][D + 4];

  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int col = lane & 15, quarter = lane >> 4;
  const int h = blockIdx.x % A.heads;
  const int64_t b = blockIdx.x / A.heads;
  const int split = blockIdx.y;
  const int64_t page_tokens = (int64_t)1 << A.shift;
  const int64_t q_heads = (int64_t)A.heads * A.group;
  const int64_t len = min((int64_t)max(A.len[b], 0), A.table_ld << A.shift);
  const int64_t q0 = min((int64_t)max(A.cu[b], 0), A.total_q), q1 = min((int64_t)max(A.cu[b + 1], 0), A.total_q);
  const int64_t m = q1 - q0, rows = m * A.group;
  const int32_t* const table = A.table + b * A.table_ld;
  const int64_t head_codes = page_tokens * D;

  for (int64_t tile = blockIdx.z; tile * kRows < rows; tile += gridDim.z) {
    const int64_t row = tile * kRows + col;
    const bool live = row < rows;
    const int64_t i = min(row, rows - 1) / A.group, g = min(row, rows - 1) % A.group;
    // keys [low, high) are seen by this row, [tile_low, tile_high) by any row of the tile
    int64_t high = len, low = 0, tile_high = len, tile_low = 0, all_high = len, all_low = 0;
    if (A.causal) {
      const int64_t first = tile * kRows / A.group, last = min(tile * kRows + kRows - 1, rows - 1) / A.group;
      high = len - m + i + 1;
      tile_high = len - m + last + 1;
      all_high = len - m + first + 1;
      if (A.window > 0) {
        low = high - A.window;
        tile_low = max(all_high - A.window, (int64_t)0);
        all_low = tile_high - A.window;
      }
    }
    // this split's share of them
    const int64_t share = (int64_t)split * A.split_tokens;
    const int64_t begin = max(share, tile_low & ~(int64_t)(kChunk - 1));
    const int64_t end = split == A.splits - 1 ? tile_high : min(share + A.split_tokens, tile_high);

    // the row's query: 16 channels of each 64 for a lane, in FP16 at the row's power of two
    v8h q[kPieces][2];
    float row_scale;
    {
      const uint16_t* const src = A.q + (q0 + i) * A.q_row + (h * A.group + g) * D + 16 * quarter;
      v4u w[kPieces][2];
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < kPieces; p++)
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
      row_scale = __uint_as_float((ex - 14u) << 23) * (A.scale * kLog2e);
#pragma unroll
      for (int p = 0; p < kPieces; p++)
#pragma unroll
        for (int e = 0; e < 2; e++)
#pragma unroll
          for (int c = 0; c < 4; c++) {
            q[p][e][2 * c] = (_Float16)(widen<FP16>((uint16_t)w[p][e][c]) * lift);
            q[p][e][2 * c + 1] = (_Float16)(widen<FP16>((uint16_t)(w[p][e][c] >> 16)) * lift);
          }
    }

    v4f o[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; t++) o[t] = v4f{};
    float top = minus_inf(), total = 0.0f;

    for (int64_t t0 = begin + kChunk * wave; t0 < end; t0 += kChunk * kWaves) {
      // pages of the tokens whose keys this lane loads, and of the tokens whose scores it holds
      const int64_t tk = t0 + 16 * (col >> 2), tv = t0 + 16 * quarter;
      uint32_t pk = tk < len ? (uint32_t)table[tk >> A.shift] : ~0u;
      uint32_t pv = tv < len ? (uint32_t)table[tv >> A.shift] : ~0u;
      const bool in_k = pk < A.n_pages, in_v = pv < A.n_pages;
      float ks = 0.0f, vs = 0.0f;
      v4u kc[4][kPieces], vc[kTiles];
      if (in_k) {
        const uint8_t* const src = A.k + ((int64_t)pk * A.heads + h) * head_codes +
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
      if (in_v) {
        const uint8_t* const src = A.v + ((int64_t)pv * A.heads + h) * head_codes + (tv & (page_tokens - 1)) +
                                   (int64_t)col * page_tokens;
        ks = A.k_scale[(int64_t)pv * A.heads + h];
        vs = A.v_scale[(int64_t)pv * A.heads + h];
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
      const bool cut = __any(t0 + kChunk > all_high || t0 < all_low || t0 + kChunk > len || !in_k || !in_v);
      uint32_t seen = 0xFFFFu;
      if (cut) {
        seen = 0;
#pragma unroll
        for (int e = 0; e < 16; e++) {
          const bool yes = in_v && live && tv + e < high && tv + e >= low && tv + e < len;
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
    const int64_t out_row = tile * kRows + r;
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
      const int64_t token = q0 + out_row / A.group, head = h * A.group + out_row % A.group;
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
    __syncthreads();
  }
}

// Joins the splits of each query row: sum_s 2^(lse_s - max) o_s / sum_s 2^(lse_s - max).
template <int D, bool FP16>
__global__ __launch_bounds__(256) void attention_join_kernel(Attn A) {
  constexpr int kLanes = D / 4, kPer = 256 / kLanes;
  const int64_t b = blockIdx.x, q_heads = (int64_t)A.heads * A.group, all_rows = A.total_q * q_heads;
  const int64_t q0 = min((int64_t)max(A.cu[b], 0), A.total_q), q1 = min((int64_t)max(A.cu[b + 1], 0), A.total_q);
  const int c0 = threadIdx.x % kLanes * 4;
  for (int64_t row = q0 * q_heads + blockIdx.y * kPer + threadIdx.x / kLanes; row < q1 * q_heads;
       row += (int64_t)gridDim.y * kPer) {
    float all = minus_inf(), l = 0.0f;
    for (int s = 0; s < A.splits; s++) all = fmaxf(all, A.part_lse[s * all_rows + row]);
    v4f v = {};
    for (int s = 0; s < A.splits; s++) {
      const float lse = A.part_lse[s * all_rows + row], f = exp2_from(lse, all);
      l += f;
      if (f != 0.0f) v += f * *reinterpret_cast<const v4f*>(A.part_out + (s * all_rows + row) * D + c0);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t* const dst = A.out + row / q_heads * A.out_row + row % q_heads * D + c0;
#pragma unroll
    for (int c = 0; c < 4; c++) dst[c] = narrow<FP16>(v[c] * inv);
    if (c0 == 0 && A.lse) A.lse[row] = l == 0.0f ? minus_inf() : (all + __builtin_amdgcn_logf(l)) * kLn2;
  }
}

// ---- host ------------------------------------------------------------------------------
const char* call_fault(const ep_kv8_cache* c, const ep_kv8_attn* a) {
  if (const char* why = cache_fault(c)) return why;
  if (!a) return "null call";
  if (a->q_heads <= 0 || a->q_heads > 1 << 20 || a->q_heads % c->kv_heads) return "q_heads must be a multiple of kv_heads";
  if (a->dtype != EP_BF16 && a->dtype != EP_FP16) return "queries must be BF16 or FP16";
  if (a->n_req <= 0 || a->n_req > 0xFFFFFF / c->kv_heads) return "n_req * kv_heads outside 1 .. 2^24 - 1";
  if (a->table_ld <= 0 || a->table_ld > 0x7FFFFFFF) return "table_ld outside 1 .. 2^31 - 1";
  if (a->total_q < 0 || a->total_q > 0x7FFFFFFF) return "total_q outside 0 .. 2^31 - 1";
  if (a->window < 0 || (a->window && !a->causal)) return "a window needs causal, and must not be negative";
  if (a->max_q <= 0 || a->max_len < 0) return "max_q must be positive and max_len not negative";
  const int64_t width = (int64_t)a->q_heads * c->head_dim;
  if ((a->q_row && a->q_row < width) || (a->out_row && a->out_row < width) || a->q_row % 8 || a->out_row % 8)
    return "rows must hold q_heads * head_dim elements and be 16-byte aligned";
  if (a->total_q && (!a->d_q || !a->d_out || !a->d_cu_q || !a->d_len || !a->d_table)) return "null pointer";
  if ((reinterpret_cast<uintptr_t>(a->d_q) | reinterpret_cast<uintptr_t>(a->d_out)) & 15)
    return "queries and outputs must be 16-byte aligned";
  return nullptr;
}

// How a call's keys are shared out.  Workgroups are (row tile, request and head, split).
struct Plan {
  int64_t tiles, splits, split_tokens, max_q;
};

constexpr int64_t kWantGroups = 4096;
constexpr int64_t kLeastTokens = kChunk * kWaves;

Plan plan_of(const ep_kv8_cache& c, const ep_kv8_attn& a) {
  Plan P;
  const int64_t group = a.q_heads / c.kv_heads;
  P.tiles = std::min<int64_t>((a.max_q * group + kRows - 1) / kRows, 65535);
  P.max_q = a.max_q;
  const int64_t base = P.tiles * a.n_req * c.kv_heads;   // below 2^40
  const int64_t most = std::max<int64_t>(1, (a.max_len + kLeastTokens - 1) / kLeastTokens);
  P.splits = std::min<int64_t>({std::max<int64_t>(1, kWantGroups / base), most, 256});
  P.split_tokens = (std::max<int64_t>(a.max_len, 1) + P.splits - 1) / P.splits;
  P.split_tokens = (P.split_tokens + kChunk - 1) / kChunk * kChunk;
  return P;
}

uint64_t plan_bytes(const Plan& P, const ep_kv8_cache& c, const ep_kv8_attn& a) {
  if (P.splits == 1) return 0;
  return (uint64_t)P.splits * a.total_q * a.q_heads * (c.head_dim + 1) * sizeof(float);
}

template <int D, bool INT8, bool FP16>
void attention_launch(const Attn& A, const Plan& P, int64_t n_req, hipStream_t stream) {
  hipLaunchKernelGGL((attention_rows_kernel<D, INT8, FP16>),
                     dim3((uint32_t)(n_req * A.heads), (uint32_t)P.splits, (uint32_t)P.tiles), dim3(64 * kWaves), 0,
                     stream, A);
  if (P.splits > 1) {
    const int64_t rows = P.max_q * A.heads * A.group, per = 256 / (D / 4);
    hipLaunchKernelGGL((attention_join_kernel<D, FP16>),
                       dim3((uint32_t)n_req, (uint32_t)std::min<int64_t>((rows + per - 1) / per, 65535)), dim3(256), 0,
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

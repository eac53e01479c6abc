// INT8 product with a scale for each row of X and of W: Y = xs ws (X W^T) + bias, the sums exact in
// 32-bit integers, for any number of rows of X.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <type_traits>

#include "../../include/entropack.h"
#include "common.h"
#include "i8_plan.h"
#include "i8_tile.h"
#include "product_tiles.h"
#include "tile_order.h"

namespace ep {
namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// A launch's operands and, where it shares k out over workgroups, the sums that it leaves for another.
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
  int32_t* sums;       // [parts][m][sums_ld], or null: one part, which writes Y
  int64_t sums_ld;     // n, rounded up to a multiple of 4
  uint32_t parts, part_steps;   // of k, and the steps of 128 of each
};

// What a tile's sums become: Y's element types by their ep_dtype codes, or the sums themselves.
constexpr int kSums = 0;
template <int OUT>
constexpr int kSize = OUT == EP_BF16 || OUT == EP_FP16 ? 2 : 4;

// Four values of row i (below m) from column j, a multiple of four below n, on.
template <int OUT>
__device__ __forceinline__ v4f scaled(const v4i& sum, float xs, const v4f& ws, const v4f& bias) {
  v4f v;
#pragma unroll
  for (int r = 0; r < 4; r++) v[r] = (float)sum[r] * xs * ws[r] + bias[r];
  return v;
}
template <int OUT>
__device__ __forceinline__ void finish(const Product& P, int64_t i, int64_t j, const v4i& sum) {
  v4f ws, bias = {};
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int64_t c = min(j + r, P.n - 1);
    ws[r] = P.w_scale[c];
    if (P.bias) bias[r] = P.bias[c];
  }
  store_y4<OUT>(P.y, P.n, P.wide, i, j, scaled<OUT>(sum, P.x_scale[i], ws, bias));
}

// The scales and biases of a tile's `count` columns of Y from j0 on, in LDS that nothing else uses any more
// or yet; all threads of the workgroup take part.
template <int OUT>
__device__ __forceinline__ void stage_scales(const Product& P, int64_t j0, int count, lds_u8* lds) {
  __attribute__((address_space(3))) float* const to = (__attribute__((address_space(3))) float*)lds;
  __syncthreads();
  if (OUT != kSums)
    for (int c = threadIdx.x; c < count; c += blockDim.x) {
      const int64_t j = min(j0 + c, P.n - 1);
      to[c] = P.w_scale[j];
      to[count + c] = P.bias ? P.bias[j] : 0.0f;
    }
  __syncthreads();
}

// A wave's ROWS x COLS block of Y goes through LDS of its own, so that its stores are whole lines of rows
// instead of the pieces of 8 or 16 bytes that a lane holds.  Rows there are padded by 16 bytes.
template <int OUT, int ROWS, int COLS>
struct Block {
  static constexpr int kPitch = COLS * kSize<OUT> + 16, kBytes = ROWS * kPitch;
  lds_u8* lds;
  // four values of a row from column c, a multiple of four, on
  __device__ __forceinline__ void put(int row, int c, const v4i& sum, float xs, const v4f& ws, const v4f& bias) const {
    typedef __attribute__((address_space(3))) v2u* two;
    typedef __attribute__((address_space(3))) v4u* four;
    lds_u8* const at = lds + row * kPitch + c * kSize<OUT>;
    if (OUT == kSums) {
      *(four)at = __builtin_bit_cast(v4u, sum);
      return;
    }
    const v4f v = scaled<OUT>(sum, xs, ws, bias);
    if (OUT == EP_FP32) *(four)at = __builtin_bit_cast(v4u, v);
    else if (OUT == EP_FP16) *(two)at = __builtin_bit_cast(v2u, __builtin_convertvector(v, v4h));
    else *(two)at = __builtin_bit_cast(v2u, __builtin_convertvector(v, v4b));
  }
  // the block's rows below m and columns below n to row i and column j of Y, or of the part's sums
  __device__ __forceinline__ void store(const Product& P, uint32_t part, int64_t i, int64_t j, int lane) const {
    constexpr int kPerRow = COLS * kSize<OUT> / 16, kEach = 16 / kSize<OUT>;   // pieces of 16 bytes
    asm volatile("" ::: "memory");
    const int64_t ld = OUT == kSums ? P.sums_ld : P.n;
    uint8_t* const to = (OUT == kSums ? reinterpret_cast<uint8_t*>(P.sums + (int64_t)part * P.m * ld) : static_cast<uint8_t*>(P.y)) +
                        (i * ld + j) * kSize<OUT>;
    typedef typename std::conditional<kSize<OUT> == 2, uint16_t, uint32_t>::type element;
#pragma unroll
    for (int r = 0; r < ROWS * kPerRow; r += 64) {
      const int row = 64 % kPerRow ? (r + lane) / kPerRow : r / kPerRow + lane / kPerRow, c = 64 % kPerRow ? (r + lane) % kPerRow : lane % kPerRow;
      if ((ROWS * kPerRow % 64 && r + lane >= ROWS * kPerRow) || i + row >= P.m) continue;
      const lds_u8* const from = lds + row * kPitch + 16 * c;
      uint8_t* const at = to + row * ld * kSize<OUT> + 16 * c;
      const int64_t left = ld - j - kEach * c;   // columns from this lane's on
      if (left >= kEach) {
        const v4u v = *(const __attribute__((address_space(3))) v4u*)from;
        __builtin_memcpy(reinterpret_cast<element*>(at), &v, 16);   // rows of Y begin at any element
      } else {
        for (int e = 0; e < left; e++)
          reinterpret_cast<element*>(at)[e] = *(const __attribute__((address_space(3))) element*)(from + e * kSize<OUT>);
      }
    }
    asm volatile("" ::: "memory");
  }
};
__device__ __forceinline__ v4f staged4(const lds_u8* lds, int c) { return *(const __attribute__((address_space(3))) v4f*)(lds + 4 * c); }

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
// at the end.  No wave waits for another before that.  Bound by W's way from memory: 1 x 17408 x 5120 in
// 14.8 us, 6.0 TB/s; 32 x 17408 x 5120 in 21 us.
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
// 16 x 16; NS stages of operands are in LDS, written by direct loads.  203 x 5120 x 17408 in tiles of
// 192 x 128 and 4 shares of k, on a card where the whole call takes 37.6 us: 30, of which 25 are the 131 MB that come from
// memory (W, X for each XCD, and some of W for its second tile of X) and 3 the sums' 17 MB; the matrix unit is busy a quarter of the cycles and LDS 15 %.
// More of W in flight and less of X, by waves of their own for each, takes 5 us more.
template <int OUT, int NW, int NX, int WW, int WX, int NS>
__device__ __forceinline__ void tile_product(const Product& P, uint32_t part, int64_t i0, int64_t j0, lds_u8* lds) {
  constexpr int kWaves = WW * WX, TW = 16 * NW * WW, TX = 16 * NX * WX;
  constexpr int kSegsW = TW / 8 / kWaves, kSegsX = TX / 8 / kWaves;   // 1 KiB loads of a wave and step
  constexpr int kPerStep = kSegsW + kSegsX;
  constexpr int kStage = (TW + TX) * 128;
  static_assert(TW % (8 * kWaves) == 0 && TX % (8 * kWaves) == 0, "tile");

  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, quarter = lane >> 4;
  const int ww = wave % WW, wx = wave / WW;
  const int64_t rows_x = min(P.m - i0, (int64_t)TX), rows_w = min(P.n - j0, (int64_t)TW);
  const uint32_t k = (uint32_t)P.k, b0 = part * P.part_steps, b1 = min(b0 + P.part_steps, P.kb);
  const __amdgpu_buffer_rsrc_t rx = rsrc_of(P.x + i0 * P.k, rows_x * P.k), rw = rsrc_of(P.w + j0 * P.k, rows_w * P.k);

  // direct loads: a wave instruction fills one segment of 8 rows; lane l writes the 16 bytes at
  // 16 l, the place of chunk (l mod 8) ^ swz(row) of row l / 8
  const uint32_t seg_row = 8 * wave + (lane >> 3);
  const uint32_t chunk = 16 * ((lane & 7) ^ swz(seg_row & 15));
  static_assert(8 * kWaves % 16 == 0, "rows of a lane's segments share their swizzle");
  auto fetch = [&](uint32_t b, uint32_t stage) {
    lds_u8* const dst = lds + kStage * stage + 1024 * wave;
    const uint32_t at = 128 * b + chunk;
    const uint32_t off = b < b1 && at < k ? seg_row * k + at : kOutside;
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
  // The fragments of half a step (64 of k) are read while the half before is multiplied: without that the
  // waves, which meet at a barrier every step, all read LDS and then all multiply.
  struct Half {
    v4i x[NX], w[NW];
  };
  const auto read = [&](Half& h, const lds_u8* p, uint32_t fo) {
#pragma unroll
    for (int t = 0; t < NX; t++) h.x[t] = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fx + fo + 16 * 128 * t);
#pragma unroll
    for (int i = 0; i < NW; i++) h.w[i] = *reinterpret_cast<const __attribute__((address_space(3))) v4i*>(p + fw + fo + 16 * 128 * i);
  };
  const auto multiply = [&](const Half& h) {
#pragma unroll
    for (int i = 0; i < NW; i++)
#pragma unroll
      for (int t = 0; t < NX; t++) acc[i][t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(h.w[i], h.x[t], acc[i][t], 0, 0, 0);
  };

#pragma unroll
  for (int s = 0; s < NS; s++) fetch(b0 + s, s);
  stage_barrier<(NS - 1) * kPerStep>();
  Half first, second;
  read(first, lds, fo0);
  uint32_t stage = 0;
  for (uint32_t b = b0; b < b1; b++) {
    const uint32_t next = stage + 1 == NS ? 0 : stage + 1;
    read(second, lds + kStage * stage, fo1);
    multiply(first);
    // every wave has read this step, and the next one has landed; its place is free for the one NS later
    stage_barrier<(NS - 2) * kPerStep>();
    fetch(b + NS, stage);
    read(first, lds + kStage * next, fo0);   // zeros after the last step
    multiply(second);
    stage = next;
  }
  __builtin_amdgcn_s_waitcnt(0);   // direct loads still in flight land before LDS is used again
  stage_scales<OUT>(P, j0, TW, lds);
  typedef Block<OUT, 16, 16 * NW> Strip;
  static_assert(8 * TW + kWaves * Strip::kBytes <= NS * kStage, "LDS");
  const Strip strip = {lds + 8 * TW + wave * Strip::kBytes};
#pragma unroll
  for (int t = 0; t < NX; t++) {
    const int64_t row = i0 + 16 * (NX * wx + t);
    const float xs = OUT == kSums ? 0.0f : P.x_scale[min(row + col, P.m - 1)];
#pragma unroll
    for (int i = 0; i < NW; i++) {
      const int c = 16 * (NW * ww + i) + 4 * quarter;
      strip.put(col, 16 * i + 4 * quarter, acc[i][t], xs, staged4(lds, c), staged4(lds, TW + c));
    }
    strip.store(P, part, row, j0 + 16 * NW * ww, lane);
  }
}

// Units [0, full) are whole tiles; the `split` last tiles are taken in `cut` pieces each, so that a last round
// of few tiles is a short one: halves of W's rows, or quarters of half the rows of both.  Every unit is taken by
// `parts` workgroups, one for each share of k, which follow each other on one XCD.  They read other columns of the same
// rows, so that nothing is shared between them, and every XCD reads all of X.
struct Units {
  uint32_t tw, tx, full, split, cut;
  // The unit and the share of k of this workgroup; whole tiles and pieces are spread over the XCDs apart.
  __device__ __forceinline__ void mine(uint32_t parts, uint32_t& unit, uint32_t& part) const {
    const uint32_t whole = full * parts;
    const uint32_t id = blockIdx.x < whole ? xcd_spread(blockIdx.x, whole) : whole + xcd_spread(blockIdx.x - whole, cut * split * parts);
    unit = id / parts;
    part = id - unit * parts;
  }
};
template <int OUT, int NW, int NX, int WW, int WX, int NS>
__global__ __launch_bounds__(64 * WW * WX) void tiles_kernel(Product P, Units U) {
  constexpr int TW = 16 * NW * WW, TX = 16 * NX * WX;
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[NS * (TW + TX) * 128];
  lds_u8* const lds = (lds_u8*)lds_mem;
  uint32_t unit, part, ti, tj;
  U.mine(P.parts, unit, part);
  if (unit < U.full) {
    tile_of(unit, U.tx, U.tw, ti, tj);
    tile_product<OUT, NW, NX, WW, WX, NS>(P, part, (int64_t)ti * TX, (int64_t)tj * TW, lds);
  } else {
    constexpr bool kW = kCutW<NW, NX, WW, WX>, kX = kCutX<NW, NX, WW, WX>;
    const uint32_t u = unit - U.full, piece = u % U.cut;
    tile_of(U.full + u / U.cut, U.tx, U.tw, ti, tj);
    const int64_t i0 = (int64_t)ti * TX + (kX ? TX / 2 * (kW ? piece >> 1 : piece) : 0), j0 = (int64_t)tj * TW + (kW ? TW / 2 * (piece & 1) : 0);
    if (i0 >= P.m || j0 >= P.n) return;
    if constexpr (kW && kX) {   // stages of half the size, twice as many
      if (U.cut == 4) return tile_product<OUT, NW / 2, NX / 2, WW, WX, 2 * NS>(P, part, i0, j0, lds);
    }
    if constexpr (kW) tile_product<OUT, NW / 2, NX, WW, WX, NS>(P, part, i0, j0, lds);
    else if constexpr (kX) tile_product<OUT, NW, NX / 2, WW, WX, NS>(P, part, i0, j0, lds);
  }
}

// Many rows: tiles of 256 x 256 by four waves (i8_tile.h), W's rows as A so that a lane has four columns
// of a row of Y side by side; halves are of X's rows, quarters of 128 x 128 and eighths of 128 x 64.  Bound by power: 8192 x 5120 x 17408 to BF16 in 583 to
// 600 us, 2.5 POP/s, as the product to int32 in the same tiles; the matrix unit is busy 70 % of the cycles.
// Stores of a lane's four columns instead of whole lines take 604, with a load of its scales for each 680;
// eight waves of 128 x 64, whose tiles of 16 x 16 read half as much LDS again for a product, 593.
template <int OUT, int TN>
__device__ __forceinline__ void large_tile(const Product& P, uint32_t part, int64_t i0, int64_t j0, lds_u8* lds) {
  const int64_t k_lo = (int64_t)part * P.part_steps * 128, k_hi = min(k_lo + (int64_t)P.part_steps * 128, P.k);
  i8::tile_product<TN>(reinterpret_cast<const int8_t*>(P.w), reinterpret_cast<const int8_t*>(P.x), P.n, P.m, P.k, j0, i0, k_lo, k_hi,
                       (i8::lds_u8*)lds, [&](const auto& acc, int ww, int wx, int lane) {
    constexpr int kWaveX = TN / 2;
    const int half = lane >> 5, col = lane & 31;
    stage_scales<OUT>(P, j0, 256, lds);
    typedef Block<OUT, 32, i8::kWaveM> Strip;
    static_assert(8 * 256 + 4 * Strip::kBytes <= i8::kSlots * i8::kSlotBytes, "LDS");
    const Strip strip = {lds + 8 * 256 + (2 * ww + wx) * Strip::kBytes};
#pragma unroll
    for (int t = 0; t < kWaveX / 32; t++) {
      const int64_t row = i0 + kWaveX * wx + 32 * t;
      const float xs = OUT == kSums ? 0.0f : P.x_scale[min(row + col, P.m - 1)];
#pragma unroll
      for (int i = 0; i < i8::kBlocksM; i++)
#pragma unroll
        for (int g = 0; g < 4; g++) {
          const int c = 32 * i + 8 * g + 4 * half, at = i8::kWaveM * ww + c;
          const v4i v = {acc[i][t][4 * g], acc[i][t][4 * g + 1], acc[i][t][4 * g + 2], acc[i][t][4 * g + 3]};
          strip.put(col, c, v, xs, staged4(lds, at), staged4(lds, 256 + at));
        }
      strip.store(P, part, row, j0 + i8::kWaveM * ww, lane);
    }
  });
}
template <int OUT>
__global__ __launch_bounds__(i8::kGemmThreads) void large_kernel(Product P, Units U) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds_mem[i8::kSlots * i8::kSlotBytes];
  lds_u8* const lds = (lds_u8*)lds_mem;
  uint32_t unit, part, ti, tj;
  U.mine(P.parts, unit, part);
  if (unit < U.full) {
    tile_of(unit, U.tw, U.tx, tj, ti);
    return large_tile<OUT, 256>(P, part, (int64_t)ti * 256, (int64_t)tj * 256, lds);
  }
  const uint32_t u = unit - U.full, piece = u % U.cut;
  tile_of(U.full + u / U.cut, U.tw, U.tx, tj, ti);
  int64_t i0 = (int64_t)ti * 256, j0 = (int64_t)tj * 256;
  if (U.cut == 2) return large_tile<OUT, 128>(P, part, i0 + 128 * piece, j0, lds);
  j0 += 128 * (piece & 1);
  i0 += 256 / (U.cut / 2) * (piece >> 1);
  if (i0 >= P.m || j0 >= P.n) return;
  if (U.cut == 4) tile_product<OUT, 4, 4, 2, 2, 5>(P, part, i0, j0, lds);
  else tile_product<OUT, 4, 2, 2, 2, 6>(P, part, i0, j0, lds);
}

// The parts' sums, scales, bias and rounding: a thread for four columns of a row.  Four parts of 203 x 5120, 17 MB,
// in 6 us, most of it the launch.  What a workspace held before the call does not matter, so that there is no cleared
// counter by which the last workgroup of a tile could know itself and join in the same launch.
template <int OUT>
__global__ __launch_bounds__(256) void join_kernel(Product P) {
  const uint32_t per_row = (uint32_t)(P.sums_ld / 4), id = blockIdx.x * 256 + threadIdx.x;   // below 2^31
  const int64_t i = id / per_row, j = 4 * (int64_t)(id - (uint32_t)i * per_row);
  if (i >= P.m) return;
  const v4i* p = reinterpret_cast<const v4i*>(P.sums + i * P.sums_ld + j);
  const int64_t next = P.m * P.sums_ld / 4;
  v4i v = {};
  for (uint32_t s = 0; s < P.parts; s += 4) {
    v4i part[4];
#pragma unroll
    for (uint32_t e = 0; e < 4; e++) part[e] = p[min(s + e, P.parts - 1) * next];
#pragma unroll
    for (uint32_t e = 0; e < 4; e++)
      if (s + e < P.parts) v += part[e];
  }
  finish<OUT>(P, i, j, v);
}

Units units_of(const Product& P, int tw, int tx, uint32_t most, int cus) {
  const uint32_t x = (uint32_t)((P.m + tx - 1) / tx), w = (uint32_t)((P.n + tw - 1) / tw), tiles = x * w;
  const uint32_t cut = P.parts > 1 ? 1 : cut_of(tiles, most, cus), split = cut > 1 ? tiles % cus : 0;
  return {w, x, tiles - split, split, cut};
}
template <int OUT, int NW, int NX, int WW, int WX, int NS>
void tiles_launch(const Product& P, int cus, hipStream_t stream) {
  const Units U = units_of(P, 16 * NW * WW, 16 * NX * WX, kMostCut<NW, NX, WW, WX>, cus);
  hipLaunchKernelGGL((tiles_kernel<OUT, NW, NX, WW, WX, NS>), dim3((U.full + U.cut * U.split) * P.parts), dim3(64 * WW * WX), 0, stream, P, U);
}
template <int OUT>
void large_launch(const Product& P, int cus, hipStream_t stream) {
  const Units U = units_of(P, 256, 256, kMostLarge, cus);
  hipLaunchKernelGGL(large_kernel<OUT>, dim3((U.full + U.cut * U.split) * P.parts), dim3(i8::kGemmThreads), 0, stream, P, U);
}

template <int OUT, int NW, int NX, int KW, int NS>
void ring_launch(const Product& P, uint32_t height, hipStream_t stream) {
  const uint32_t strips = (uint32_t)((P.n + height - 1) / height), tx = (uint32_t)((P.m + 16 * NX - 1) / (16 * NX));
  const uint32_t per_xcd = (strips + kXcds - 1) / kXcds;
  hipLaunchKernelGGL((ring_kernel<OUT, NW, NX, KW, NS>), dim3(per_xcd * kXcds * tx), dim3(64 * KW), 0, stream, P, height, per_xcd);
}

template <int OUT>
void tile_launch(Kernel kernel, const Product& P, int cus, hipStream_t stream) {
  if (kernel == kTile64) tiles_launch<OUT, 4, 2, 2, 2, 3>(P, cus, stream);
  else if (kernel == kTile128) tiles_launch<OUT, 4, 4, 2, 2, 4>(P, cus, stream);
  else if (kernel == kWideX) tiles_launch<OUT, 4, 4, 2, 4, 3>(P, cus, stream);
  else if (kernel == kWideW) tiles_launch<OUT, 4, 4, 4, 2, 3>(P, cus, stream);
  else if (kernel == kWideW64) tiles_launch<OUT, 4, 2, 4, 2, 4>(P, cus, stream);
  else if (kernel == k192x128) tiles_launch<OUT, 3, 4, 4, 2, 4>(P, cus, stream);
  else if (kernel == k192x192) tiles_launch<OUT, 6, 3, 2, 4, 3>(P, cus, stream);
  else large_launch<OUT>(P, cus, stream);
}

// Up to 16 rows the launch is W's stream from memory: by four waves a workgroup, or eight where W has too
// few strips for several workgroups on a CU.
template <int OUT>
void product_launch(const Plan& plan, const Product& P, int cus, hipStream_t stream) {
  if (plan.kernel == kRing16) {
    if (rounds((P.n + plan.height - 1) / plan.height, cus) > 1) ring_launch<OUT, 2, 1, 4, 2>(P, plan.height, stream);
    else ring_launch<OUT, 2, 1, 8, 2>(P, plan.height, stream);
  } else if (plan.kernel == kRing32) {
    ring_launch<OUT, 3, 2, 6, 2>(P, plan.height, stream);
  } else if (plan.kernel == kRing64) {
    ring_launch<OUT, 3, 4, 5, 2>(P, plan.height, stream);
  } else if (P.parts == 1) {
    tile_launch<OUT>(plan.kernel, P, cus, stream);
  } else {
    tile_launch<kSums>(plan.kernel, P, cus, stream);
    const int64_t threads = P.m * (P.sums_ld / 4);   // of fewer tiles than CUs: below 2^31
    hipLaunchKernelGGL(join_kernel<OUT>, dim3((uint32_t)((threads + 255) / 256)), dim3(256), 0, stream, P);
  }
}

bool misaligned(const void* p) { return reinterpret_cast<uintptr_t>(p) & 15; }

int compute_units() {
  int dev = 0, cus = 0;
  if (hipGetDevice(&dev) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
  return cus;
}

constexpr int64_t kMost = 1 << 24, kMostK = 131071;   // sums of k products of two codes stay below 2^31
bool bad_sizes(int64_t m, int64_t n, int64_t k) { return m < 0 || n <= 0 || k <= 0 || k % 16 || m > kMost || n > kMost || k > kMostK; }

}  // namespace
}  // namespace ep

extern "C" uint64_t ep_gemm_i8_scaled_workspace(int64_t m, int64_t n, int64_t k) {
  const int cus = ep::compute_units();
  return ep::bad_sizes(m, n, k) || m == 0 || cus <= 0 ? 0 : ep::workspace_of(ep::plan_of(m, n, k, cus), m, n);
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
  const int cus = compute_units();
  if (cus <= 0) return fail(EP_ERR_HIP, "ep_gemm_i8_scaled: no device");
  const Plan plan = plan_of(m, n, k, cus);
  if (workspace_of(plan, m, n) && (!d_workspace || misaligned(d_workspace) || ws_bytes < workspace_of(plan, m, n)))
    return fail(EP_ERR_ARG, "ep_gemm_i8_scaled: a workspace that is missing, misaligned or short");
  const Product P = {reinterpret_cast<const uint8_t*>(d_x), d_x_scale, reinterpret_cast<const uint8_t*>(d_w), d_w_scale, d_bias, d_y, m, n, k,
                     (uint32_t)((k + 127) / 128), n % 4 == 0 && reinterpret_cast<uintptr_t>(d_y) % (4 * size) == 0,
                     plan.parts > 1 ? static_cast<int32_t*>(d_workspace) : nullptr, (n + 3) / 4 * 4, plan.parts, plan.part_steps};
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (y_dtype == EP_FP32) product_launch<EP_FP32>(plan, P, cus, stream);
  else if (y_dtype == EP_FP16) product_launch<EP_FP16>(plan, P, cus, stream);
  else product_launch<EP_BF16>(plan, P, cus, stream);
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_gemm_i8_scaled: launch failed");
  return EP_OK;
}

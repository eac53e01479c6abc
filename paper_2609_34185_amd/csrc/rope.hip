// Rotary positions: pairs of a head's channels are turned by position times the pair's frequency.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "../../include/entropack.h"
#include "common.h"

namespace ep {
namespace {

constexpr int kThreads = 256;

// Cosine and sine of `phase` / 2^32 of a turn.  The nearest quarter is taken off as an integer, which
// leaves at most an eighth of a turn either way; there the Taylor series to x^11 and x^10 are within
// 7e-11 and 2e-10, so that what is left is the rounding of x and of the sums.
__device__ __forceinline__ void turn(uint32_t phase, float& c, float& s) {
  const uint32_t quarter = (phase + 0x20000000u) >> 30;
  const float x = (float)(int32_t)(phase - (quarter << 30)) * 1.4629180792671596e-9f;   // 2 pi / 2^32
  const float q = x * x;
  float si = __builtin_fmaf(q, -2.5052108e-8f, 2.7557319e-6f);
  si = __builtin_fmaf(q, si, -1.9841270e-4f);
  si = __builtin_fmaf(q, si, 8.3333333e-3f);
  si = __builtin_fmaf(q, si, -1.6666667e-1f);
  si = __builtin_fmaf(q * x, si, x);
  float co = __builtin_fmaf(q, -2.7557319e-7f, 2.4801587e-5f);
  co = __builtin_fmaf(q, co, -1.3888889e-3f);
  co = __builtin_fmaf(q, co, 4.1666667e-2f);
  co = __builtin_fmaf(q, co, -0.5f);
  co = __builtin_fmaf(q, co, 1.0f);
  const bool swap = quarter & 1;
  c = swap ? si : co;
  s = swap ? co : si;
  if ((quarter + 1) & 2) c = -c;   // quarters 1 and 2
  if (quarter & 2) s = -s;         // quarters 2 and 3
}

template <typename T>
__device__ __forceinline__ float value(T x) { return (float)x; }

// VEC elements at a time: one load where they lie aligned.
template <typename T, int VEC>
struct Pack {
  T v[VEC];
} __attribute__((aligned(sizeof(T) * VEC < 16 ? sizeof(T) * VEC : 16)));

// What is one for all threads, computed on the host.
struct Rope {
  ep_rope_call c;
  uint32_t rotated, copied;   // units of a head: of VEC pairs, and of VEC channels outside the rotated part
  uint32_t heads, lanes;      // of queries and keys; threads that share a token's heads, for each unit
};

// The last request that begins at or before token t, by whole waves: a lane for every 64th part of those
// that are left, so that 64 requests take one load and 4096 two.
__device__ __forceinline__ uint32_t request_of(const int32_t* cu, uint32_t n, int64_t t) {
  const uint32_t lane = threadIdx.x & 63;
  uint32_t lo = 0;
  while (n > 1) {
    const uint32_t step = (n + 63) / 64, at = lane * step;
    const uint64_t begun = __ballot(at < n && cu[lo + min(at, n - 1)] <= t);
    const uint32_t part = begun ? 63 - __builtin_clzll(begun) : 0;
    lo += part * step;
    n = min(step, n - part * step);
  }
  return lo;
}

// A thread turns one unit (VEC pairs) of every lanes-th head of a token: its cosines and sines are
// made once for all of them, the angle by one 64-bit product that wraps at whole turns.  Bound by memory:
// 14.5 thousand tokens of 40 + 8 heads of 128 in BF16, positions from lengths, in 68 us, 5.2 TB/s; channels
// side by side or FP32 at 4.7 to 5.0.  One token takes 3.3 us, the launch and the chain length, position,
// store.
template <typename T, int VEC, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rope_kernel(Rope R) {
  const ep_rope_call& C = R.c;
  const uint32_t units = R.rotated + R.copied, per_token = units * R.lanes;
  const uint64_t first = ((uint64_t)blockIdx.y * gridDim.x + blockIdx.x) * kThreads;
  const int64_t t0 = (int64_t)(first / per_token);
  if (t0 >= C.n_tokens) return;
  const uint32_t into = (uint32_t)(first - (uint64_t)t0 * per_token) + threadIdx.x, ahead = into / per_token;
  const int64_t t = t0 + ahead;
  uint32_t b = 0, end = 1;   // the token's request is one of these
  if (!C.d_pos) {
    b = request_of(C.d_cu, (uint32_t)C.n_req, t0);
    const int64_t t1 = t0 + (kThreads - 1 + per_token - 1) / per_token;
    end = b + 1 + (t1 > t0 && b + 1 < (uint32_t)C.n_req ? request_of(C.d_cu + b, (uint32_t)C.n_req - b, t1) : 0);
  }
  if (t >= C.n_tokens) return;
  const uint32_t in = into - ahead * per_token, lane = in / units, unit = in - lane * units;

  // what does not wait for the position: frequencies and the first head's values
  const bool turns = unit < R.rotated;
  uint32_t one, two;   // channels
  uint64_t freq[VEC];
  if (turns) {
    one = C.rot_first + (PAIRS ? 2 : 1) * VEC * unit;
    two = PAIRS ? one + VEC : one + C.rot_dim / 2;
#pragma unroll
    for (int i = 0; i < VEC; i++) freq[i] = C.d_freqs[VEC * unit + i];
  } else {
    one = VEC * (unit - R.rotated);
    if (one >= (uint32_t)C.rot_first) one += C.rot_dim;
    two = one;
  }
  typedef Pack<T, VEC> P;
  const auto load = [&](uint32_t h, P& x, P& y) {
    const bool key = h >= (uint32_t)C.q_heads;
    const T* const from = static_cast<const T*>(key ? C.d_k : C.d_q) + t * (key ? C.k_row : C.q_row) +
                          (int64_t)(key ? h - C.q_heads : h) * C.head_dim;
    x = *reinterpret_cast<const P*>(from + one);
    if (turns) y = *reinterpret_cast<const P*>(from + two);
  };
  P x, y;
  load(lane, x, y);

  int32_t pos;
  if (C.d_pos) {
    pos = C.d_pos[t];
  } else {
    while (end - b > 1) {
      const uint32_t mid = (b + end) / 2;
      if (C.d_cu[mid] <= t) b = mid;
      else end = mid;
    }
    const int32_t past = C.d_cu[b + 1];
    if (t >= past || t < C.d_cu[b]) return;   // a row after the last token
    pos = C.d_len[b] - past + (int32_t)t;
  }

  float co[VEC], si[VEC];
  if (turns) {
#pragma unroll
    for (int i = 0; i < VEC; i++) {
      const uint64_t phase = freq[i] * (uint64_t)(int64_t)pos;
      turn((uint32_t)((phase + 0x80000000u) >> 32), co[i], si[i]);
      co[i] *= C.amplitude;
      si[i] *= C.inverse ? -C.amplitude : C.amplitude;
    }
  }
  for (uint32_t h = lane; h < R.heads; h += R.lanes) {
    P next_x, next_y;
    if (h + R.lanes < R.heads) load(h + R.lanes, next_x, next_y);   // heads lie apart, in place too
    const bool key = h >= (uint32_t)C.q_heads;
    T* const to = static_cast<T*>(key ? C.d_k_out : C.d_q_out) + t * (key ? C.k_out_row : C.q_out_row) +
                  (int64_t)(key ? h - C.q_heads : h) * C.head_dim;
    if (turns) {
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        // pairs side by side: x holds the first half of 2 VEC channels, y the second
        const int k = 2 * i;
        T& pa = !PAIRS || k < VEC ? x.v[PAIRS ? k % VEC : i] : y.v[k % VEC];
        T& pb = PAIRS && k + 1 < VEC ? x.v[(k + 1) % VEC] : y.v[PAIRS ? (k + 1) % VEC : i];
        const float a = value(pa), b = value(pb);
        pa = (T)__builtin_fmaf(a, co[i], -(b * si[i]));
        pb = (T)__builtin_fmaf(a, si[i], b * co[i]);
      }
    }
    *reinterpret_cast<P*>(to + one) = x;
    if (turns) *reinterpret_cast<P*>(to + two) = y;
    x = next_x;
    y = next_y;
  }
}

// A thread takes as many heads as make 96 bytes in and out, three at least, as long as there are threads
// for 1024 on each of 256 CUs: its position and its cosines and sines are made once for them, and the
// next head's values are on their way while one is turned.  14.5 thousand tokens of 40 + 8 heads of 128 in
// BF16: 68 us with 2.7 or 3 heads a thread, 77 with 16; 4.3 thousand of 40 + 8 heads of 64, half of them
// rotated: 14 us with 3, 20 with one.
constexpr int64_t kEnough = 256 * 1024, kBytes = 96;

template <typename T, int VEC>
void launch(Rope& R, hipStream_t stream) {
  const ep_rope_call& C = R.c;
  const bool in_place = C.d_q == C.d_q_out && (C.k_heads == 0 || C.d_k == C.d_k_out);
  R.rotated = C.rot_dim / 2 / VEC;
  R.copied = in_place ? 0 : (C.head_dim - C.rot_dim) / VEC;
  const int64_t each = C.n_tokens * (R.rotated + R.copied);
  constexpr int64_t kHeads = std::max<int64_t>(3, kBytes / (2 * VEC * sizeof(T)));
  R.lanes = (uint32_t)std::min<int64_t>(R.heads, std::max((R.heads + kHeads - 1) / kHeads, (kEnough + each - 1) / each));
  const int64_t groups = (each * R.lanes + kThreads - 1) / kThreads, x = std::min<int64_t>(groups, 1 << 22);
  const dim3 grid((uint32_t)x, (uint32_t)((groups + x - 1) / x));
  if (C.layout == EP_ROPE_PAIRS) hipLaunchKernelGGL((rope_kernel<T, VEC, true>), grid, dim3(kThreads), 0, stream, R);
  else hipLaunchKernelGGL((rope_kernel<T, VEC, false>), grid, dim3(kThreads), 0, stream, R);
}

// Eight channels at a time where every unit lies aligned for one load, else as many as do.
template <typename T>
void launch(Rope& R, hipStream_t stream) {
  const ep_rope_call& C = R.c;
  uint64_t bytes = reinterpret_cast<uintptr_t>(C.d_q) | reinterpret_cast<uintptr_t>(C.d_q_out);
  uint64_t counts = C.rot_dim / 2 | C.rot_first | C.head_dim | C.q_row | C.q_out_row;
  if (C.k_heads) {
    bytes |= reinterpret_cast<uintptr_t>(C.d_k) | reinterpret_cast<uintptr_t>(C.d_k_out);
    counts |= C.k_row | C.k_out_row;
  }
  const auto aligned = [&](int vec) { return counts % vec == 0 && bytes % std::min<size_t>(16, vec * sizeof(T)) == 0; };
  if (aligned(8)) launch<T, 8>(R, stream);
  else if (aligned(4)) launch<T, 4>(R, stream);
  else if (aligned(2)) launch<T, 2>(R, stream);
  else launch<T, 1>(R, stream);
}

}  // namespace
}  // namespace ep

extern "C" int ep_rope_freqs(int rot_dim, double base, int stretch, double factor, double trained_len, double low,
                             double high, uint64_t* freqs) {
  using ep::fail;
  if (!freqs) return fail(EP_ERR_ARG, "ep_rope_freqs: null pointer");
  if (rot_dim < 2 || rot_dim > 1024 || rot_dim % 2) return fail(EP_ERR_ARG, "ep_rope_freqs: rot_dim must be even and within 2 .. 1024");
  if (!(base >= 1.0 && base <= 1e18)) return fail(EP_ERR_ARG, "ep_rope_freqs: base outside 1 .. 1e18");
  if (stretch < EP_ROPE_PLAIN || stretch > EP_ROPE_INDEX) return fail(EP_ERR_ARG, "ep_rope_freqs: unknown kind of stretching");
  if (stretch != EP_ROPE_PLAIN && !(factor >= 1.0 && factor <= 1e9)) return fail(EP_ERR_ARG, "ep_rope_freqs: factor outside 1 .. 1e9");
  if (stretch == EP_ROPE_BASE && rot_dim == 2) return fail(EP_ERR_ARG, "ep_rope_freqs: a stretched base needs rot_dim above 2");
  if (stretch >= EP_ROPE_TURNS && !(trained_len >= 1.0 && trained_len <= 2147483648.0 && low > 0.0 && high > low && high <= 1e9))
    return fail(EP_ERR_ARG, "ep_rope_freqs: trained_len outside 1 .. 2^31, or low and high outside 0 < low < high <= 1e9");
  if (stretch == EP_ROPE_INDEX && base == 1.0) return fail(EP_ERR_ARG, "ep_rope_freqs: pairs of base 1 all make the same turns");
  // in 64 bits of mantissa, so that a frequency's own rounding, times a position of 31 bits, stays
  // below 2^-32 of a turn
  const long double turn = 6.283185307179586476925286766559L;
  const long double b = stretch == EP_ROPE_BASE ? (long double)base * powl(factor, (long double)rot_dim / (rot_dim - 2)) : base;
  long double from = 0, to = 1;
  if (stretch == EP_ROPE_INDEX) {
    const long double per = rot_dim / (2 * logl(base));
    from = std::max(floorl(per * logl(trained_len / (turn * high))), 0.0L);
    to = std::min(ceill(per * logl(trained_len / (turn * low))), (long double)(rot_dim - 1));
  }
  for (int i = 0; i < rot_dim / 2; i++) {
    long double theta = powl(b, -2.0L * i / rot_dim), keep = 1;
    if (stretch == EP_ROPE_LINEAR) theta /= factor;
    else if (stretch == EP_ROPE_TURNS) keep = (trained_len * theta / turn - low) / ((long double)high - low);
    else if (stretch == EP_ROPE_INDEX) keep = 1 - (i - from) / std::max(to - from, 0.001L);
    if (stretch >= EP_ROPE_TURNS) {
      keep = std::min(std::max(keep, 0.0L), 1.0L);
      theta *= keep + (1 - keep) / factor;
    }
    freqs[i] = (uint64_t)llrintl(theta / turn * 18446744073709551616.0L);   // below 2^62
  }
  return EP_OK;
}

extern "C" int ep_rope(const ep_rope_call* call, void* hip_stream) {
  using namespace ep;
  if (!call) return fail(EP_ERR_ARG, "ep_rope: null call");
  Rope R = {*call, 0, 0, 0, 0};
  ep_rope_call& C = R.c;
  if (C.dtype != EP_BF16 && C.dtype != EP_FP16 && C.dtype != EP_FP32) return fail(EP_ERR_ARG, "ep_rope: dtype must be BF16, FP16 or FP32");
  if (C.layout != EP_ROPE_HALF && C.layout != EP_ROPE_PAIRS) return fail(EP_ERR_ARG, "ep_rope: unknown layout");
  if (C.n_tokens < 0 || C.n_tokens > 0x7FFFFFFF) return fail(EP_ERR_ARG, "ep_rope: n_tokens outside 0 .. 2^31 - 1");
  if (C.q_heads <= 0 || C.q_heads > 65536 || C.k_heads < 0 || C.k_heads > 65536) return fail(EP_ERR_ARG, "ep_rope: heads out of range");
  if (C.head_dim < 2 || C.head_dim > 1024 || C.rot_dim < 2 || C.rot_dim % 2 || C.rot_first < 0 || C.rot_dim > C.head_dim - C.rot_first)
    return fail(EP_ERR_ARG, "ep_rope: head_dim outside 2 .. 1024, or a rotated part that is odd, empty or beyond it");
  const int64_t q = (int64_t)C.q_heads * C.head_dim, k = (int64_t)C.k_heads * C.head_dim, most = (int64_t)1 << 31;
  for (int64_t* p : {&C.q_row, &C.q_out_row})
    if (*p == 0) *p = q;
  for (int64_t* p : {&C.k_row, &C.k_out_row})
    if (*p == 0) *p = k;
  if (C.q_row < q || C.q_out_row < q || C.q_row > most || C.q_out_row > most ||
      (C.k_heads && (C.k_row < k || C.k_out_row < k || C.k_row > most || C.k_out_row > most)))
    return fail(EP_ERR_ARG, "ep_rope: rows shorter than their heads, or above 2^31 elements");
  if (!std::isfinite(C.amplitude)) return fail(EP_ERR_ARG, "ep_rope: amplitude is not finite");
  if (!C.d_pos && (C.n_req < 1 || C.n_req > 0x7FFFFFFE)) return fail(EP_ERR_ARG, "ep_rope: n_req out of range");
  if (C.n_tokens == 0) return EP_OK;
  if (!C.d_q || !C.d_q_out || !C.d_freqs || (C.k_heads && (!C.d_k || !C.d_k_out)) || (!C.d_pos && (!C.d_cu || !C.d_len)))
    return fail(EP_ERR_ARG, "ep_rope: null pointer");
  const uintptr_t size = C.dtype == EP_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(C.d_q) | reinterpret_cast<uintptr_t>(C.d_q_out)) % size ||
      (C.k_heads && (reinterpret_cast<uintptr_t>(C.d_k) | reinterpret_cast<uintptr_t>(C.d_k_out)) % size) ||
      reinterpret_cast<uintptr_t>(C.d_freqs) % 8 ||
      (reinterpret_cast<uintptr_t>(C.d_pos) | reinterpret_cast<uintptr_t>(C.d_cu) | reinterpret_cast<uintptr_t>(C.d_len)) % 4)
    return fail(EP_ERR_ARG, "ep_rope: pointers off their elements");
  if ((C.d_q == C.d_q_out && C.q_row != C.q_out_row) || (C.k_heads && C.d_k == C.d_k_out && C.k_row != C.k_out_row))
    return fail(EP_ERR_ARG, "ep_rope: a rotation in place needs one distance of rows");
  if (C.k_heads && (C.d_q_out == C.d_k || C.d_k_out == C.d_q || C.d_q_out == C.d_k_out))
    return fail(EP_ERR_ARG, "ep_rope: an output at the other's input or output");
  R.heads = (uint32_t)(C.q_heads + C.k_heads);
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  if (C.dtype == EP_BF16) launch<__bf16>(R, stream);
  else if (C.dtype == EP_FP16) launch<_Float16>(R, stream);
  else launch<float>(R, stream);
  if (hipGetLastError() != hipSuccess) return fail(EP_ERR_HIP, "ep_rope: launch failed");
  return EP_OK;
}

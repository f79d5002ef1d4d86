// wm_cache_device.h -- device code that the paged cache's kernels share: the
// places of ragged requests, the 8-bit codes, the tiles of an attention call.
#pragma once
#include <hip/hip_runtime.h>

#include "wm_cache_internal.h"

namespace wm {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kNegInf = -__builtin_huge_valf();

__device__ __forceinline__ int lane_id() { return threadIdx.x & 63; }

// Lists of places shared by ragged requests: request r has q = q_start[r+1] -
// q_start[r] tokens and needs at most q mul / div + 1 + more places, so its
// places begin at q_start[r] mul / div + r (1 + more): no prefix sum is needed
// to find them.
struct Places {
  const int32_t *q_start;
  uint32_t n, mul, div, per;  // per: places per request beyond the quotient
  __device__ __forceinline__ int64_t first(uint32_t r) const {
    const int64_t q = q_start[r] > 0 ? q_start[r] : 0;
    return q * mul / div + (int64_t)r * per;
  }
  // The request that place x belongs to: 64 candidates at a time, so that a
  // search over 64 requests costs one load's latency and over 4096 two.
  __device__ __forceinline__ uint32_t find(int64_t x) const {
    uint32_t lo = 0, left = n;
    while (left > 1) {
      const uint32_t stride = (left + 63u) / 64u;
      const uint32_t i = (uint32_t)lane_id() * stride;
      const bool le = i < left && first(lo + i) <= x;
      uint32_t c = (uint32_t)__popcll(__ballot(le));
      c = c ? c - 1u : 0u;
      const uint32_t skip = c * stride < left ? c * stride : 0u;
      lo += skip;
      left = left - skip < stride ? left - skip : stride;
    }
    return lo;
  }
};

// ---- 8-bit codes --------------------------------------------------------------

template <int FMT>
struct Code;
template <>
struct Code<WM_E4M3> {
  static constexpr float kLargest = 448.0f;
  static constexpr bool kInfinities = false;
  // bit 7 of each byte that is a code with no finite value: the NaN of either sign
  static __device__ __forceinline__ uint32_t special(uint32_t w) {
    return (w & 0x7F7F7F7Fu) + 0x01010101u;
  }
  static __device__ __forceinline__ uint32_t two(float x, float y) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x, y, 0, false) & 0xFFFFu;
  }
  static __device__ __forceinline__ float value(uint32_t b) {
    return __builtin_amdgcn_cvt_f32_fp8((int)b, 0);
  }
  // exact: three mantissa bits, exponents of -9..8
  template <bool HI>
  static __device__ __forceinline__ bf16x2 bf(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HI);
  }
  template <bool HI>
  static __device__ __forceinline__ f16x2 half(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, HI);
  }
};
template <>
struct Code<WM_E5M2> {
  static constexpr float kLargest = 57344.0f;
  static constexpr bool kInfinities = true;
  static __device__ __forceinline__ uint32_t special(uint32_t w) {
    return (w & 0x7F7F7F7Fu) + 0x04040404u;  // infinities too
  }
  static __device__ __forceinline__ uint32_t two(float x, float y) {
    return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(x, y, 0, false) & 0xFFFFu;
  }
  static __device__ __forceinline__ float value(uint32_t b) {
    return __builtin_amdgcn_cvt_f32_bf8((int)b, 0);
  }
  template <bool HI>
  static __device__ __forceinline__ bf16x2 bf(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, 1.0f, HI);
  }
  template <bool HI>
  static __device__ __forceinline__ f16x2 half(uint32_t w) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_bf8(w, 1.0f, HI);
  }
};

// A sum's part with the weight f: a weight that is rounded to 0 takes all but
// infinities and NaN away.
__device__ __forceinline__ float weighed(float f, float y) {
  return f != 0.0f ? f * y : (fabsf(y) <= 3.4028234e38f ? 0.0f : y);
}

// Makes those of the wave's codes x zero that have no finite value; was there
// one?
template <int FMT, int N>
__device__ __forceinline__ bool take_special(u32x4 (&x)[N]) {
  uint32_t any = 0;
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t sp = Code<FMT>::special(x[i][j]) & 0x80808080u;
      x[i][j] &= ~((sp >> 7) * 0xFFu);
      any |= sp;
    }
  return __any(any != 0);
}

// A request as attention sees it.  Its query rows that share a key head are its
// tokens times the heads of the group, row = token * group + head; tiles of
// `rows` of them are worked on together.  Its sequence is cut into parts of
// 2^cut tokens (512, or more where the span that some row sees has over 30 of
// them), at multiples of that: the cut depends on the request alone, so a
// request of one tile gives the same bits whatever else the call holds.
struct Request {
  int64_t q0;             // its first query row's token
  uint32_t n_rows, tiles;
  int32_t len, pos0;      // its length, position of its first new token
  uint32_t cut, part0, parts;
};

__device__ __forceinline__ Request request_of(const AttendArgs &a, uint32_t r, bool tell) {
  Request x = {0, 0, 0, 0, 0, a.plan.cut, 0, 1};
  int64_t q0 = a.q_start[r], q1 = a.q_start[r + 1], len = a.len[r];
  const int64_t end = q1;  // rows that are not there keep their positions
  if (tell && a.verdict && (q0 < 0 || q1 > (int64_t)a.n_tokens)) atomicOr(a.verdict, WM_C_SLOTS);
  q0 = q0 > 0 ? q0 : 0;
  q1 = q1 < (int64_t)a.n_tokens ? q1 : (int64_t)a.n_tokens;
  if (q0 >= q1) return x;
  const int64_t cap = (int64_t)a.max_blocks << a.bt_log2;
  if (tell && a.verdict && (len < 0 || len > cap)) atomicOr(a.verdict, WM_C_LENGTH);
  len = len < cap ? len : cap;
  len = len > 0 ? len : 0;
  // (below -2^30 none of up to 2^30 rows sees anything, and differences of
  // positions stay within 32 bits)
  int64_t p0 = len - (end - q0);
  p0 = p0 > -(1ll << 30) ? p0 : -(1ll << 30);
  const uint32_t lo =
      a.window && p0 + 1 > (int64_t)a.window ? (uint32_t)(p0 + 1 - a.window) : 0u;
  const uint32_t hi = (uint32_t)len;
  x.q0 = q0;
  x.n_rows = (uint32_t)((q1 - q0) * a.group);
  x.tiles = (x.n_rows + a.plan.rows - 1) / a.plan.rows;
  x.len = (int32_t)len;
  x.pos0 = (int32_t)p0;
  while (((hi - lo) >> x.cut) >= 31u) ++x.cut;
  auto parts = [&]() {
    return (uint32_t)(((uint64_t)hi + (1u << x.cut) - 1) >> x.cut) - (lo >> x.cut);
  };
  while (parts() > a.plan.splits) ++x.cut;  // longer than the caller's longest
  x.part0 = lo >> x.cut;
  x.parts = parts();
  x.parts = x.parts ? x.parts : 1u;
  return x;
}

// The tokens [lo, hi) that some row of a tile sees, and its parts.
struct Tile {
  uint32_t row0, lo, hi, part0, part1;
};

__device__ __forceinline__ Tile tile_of(const AttendArgs &a, const Request &x, uint32_t i) {
  Tile t;
  t.row0 = i * a.plan.rows;
  const uint32_t last = t.row0 + a.plan.rows < x.n_rows ? t.row0 + a.plan.rows - 1 : x.n_rows - 1;
  const int64_t p_lo = (int64_t)x.pos0 + t.row0 / a.group;
  const int64_t p_hi = (int64_t)x.pos0 + last / a.group;
  const int64_t lo = a.window && p_lo + 1 > (int64_t)a.window ? p_lo + 1 - a.window : 0;
  t.hi = p_hi + 1 > 0 ? (uint32_t)(p_hi + 1) : 0u;
  t.lo = (uint32_t)(lo < (int64_t)t.hi ? lo : t.hi);
  t.part0 = t.lo >> x.cut;
  t.part1 = (uint32_t)(((uint64_t)t.hi + (1u << x.cut) - 1) >> x.cut);
  if (t.hi == t.lo) t.part1 = t.part0;
  return t;
}

// Where a row's parts lie in the workspace: side by side, so that joining them
// reads one stretch.
__device__ __forceinline__ uint64_t part_place(const AttendArgs &a, uint64_t token, uint32_t hq) {
  return (token * (a.group * a.c.n_heads) + hq) * a.plan.splits;
}

// The same request in every lane of a wave, told to the compiler.
__device__ __forceinline__ Request uniform(const Request &x) {
  Request y = x;
  y.q0 = (int64_t)__builtin_amdgcn_readfirstlane((int)x.q0);  // a row of n_tokens: 31 bits
  y.n_rows = __builtin_amdgcn_readfirstlane(x.n_rows);
  y.tiles = __builtin_amdgcn_readfirstlane(x.tiles);
  y.len = __builtin_amdgcn_readfirstlane(x.len);
  y.pos0 = __builtin_amdgcn_readfirstlane(x.pos0);
  y.cut = __builtin_amdgcn_readfirstlane(x.cut);
  y.part0 = __builtin_amdgcn_readfirstlane(x.part0);
  y.parts = __builtin_amdgcn_readfirstlane(x.parts);
  return y;
}

// Query element types: the key codes are exact in either, so the product with
// the queries is exact and the sum is the matrix core's, in 32 bits.
template <int DT, int FMT>
struct Qk;
template <int FMT>
struct Qk<WM_BF16, FMT> {
  typedef bf16x8 frag;
  static __device__ __forceinline__ frag key(uint32_t x, uint32_t y) {
    const bf16x2 p = Code<FMT>::template bf<false>(x), q = Code<FMT>::template bf<true>(x);
    const bf16x2 r = Code<FMT>::template bf<false>(y), s = Code<FMT>::template bf<true>(y);
    return frag{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
  }
  static __device__ __forceinline__ f32x4 mma(frag k, frag q, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q, c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t two(float x, float y) {
    const bf16x2 v = {(__bf16)x, (__bf16)y};
    return __builtin_bit_cast(uint32_t, v);
  }
};
template <int FMT>
struct Qk<WM_FP16, FMT> {
  typedef f16x8 frag;
  static __device__ __forceinline__ frag key(uint32_t x, uint32_t y) {
    const f16x2 p = Code<FMT>::template half<false>(x), q = Code<FMT>::template half<true>(x);
    const f16x2 r = Code<FMT>::template half<false>(y), s = Code<FMT>::template half<true>(y);
    return frag{p[0], p[1], q[0], q[1], r[0], r[1], s[0], s[1]};
  }
  static __device__ __forceinline__ f32x4 mma(frag k, frag q, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(k, q, c, 0, 0, 0);
  }
  static __device__ __forceinline__ uint32_t two(float x, float y) {
    const f16x2 v = {(_Float16)x, (_Float16)y};
    return __builtin_bit_cast(uint32_t, v);
  }
};

}  // namespace
}  // namespace wm

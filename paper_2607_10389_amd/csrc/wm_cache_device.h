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
  // codes with no finite value: the NaN of either sign
  static __device__ __forceinline__ bool special(uint32_t b) { return (b & 0x7Fu) == 0x7Fu; }
  static __device__ __forceinline__ bool infinite(uint32_t) { return false; }
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
  static __device__ __forceinline__ bool special(uint32_t b) { return (b & 0x7Fu) >= 0x7Cu; }
  static __device__ __forceinline__ bool infinite(uint32_t b) { return (b & 0x7Fu) == 0x7Cu; }
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

template <int DT>
__device__ __forceinline__ float load_elem(const void *p, uint64_t i) {
  if (DT == WM_BF16)
    return __uint_as_float((uint32_t) static_cast<const uint16_t *>(p)[i] << 16);
  return (float)static_cast<const _Float16 *>(p)[i];
}

// ---- attention ----------------------------------------------------------------

// Tiles.  A request's query rows that share a key head are its tokens times the
// heads of the group, row = token * group + head; a tile is 16 NQ of them.
struct Tile {
  uint32_t r, row0, n_rows;  // request, its first row, its rows in all
  int64_t q0;                // its first token
  int32_t len, pos0;         // its length, position of its first new token
  uint32_t lo, hi;           // tokens that some row of the tile sees: [lo, hi)
};

__device__ __forceinline__ bool tile_of(const AttendArgs &a, uint32_t place, Tile *t) {
  const uint32_t rows = a.plan.rows;
  const Places pl = {a.q_start, a.n_requests, a.group, rows, 1u};
  const uint32_t r = __builtin_amdgcn_readfirstlane(pl.find(place));
  int64_t q0 = a.q_start[r], q1 = a.q_start[r + 1];
  q0 = q0 > 0 ? q0 : 0;
  q1 = q1 < (int64_t)a.n_tokens ? q1 : (int64_t)a.n_tokens;
  const int64_t nth = (int64_t)place - pl.first(r);
  if (nth < 0 || q0 >= q1) return false;
  const uint64_t n_rows = (uint64_t)(q1 - q0) * a.group;
  if ((uint64_t)nth * rows >= n_rows) return false;
  const int64_t cap = (int64_t)a.max_blocks << a.bt_log2;
  int64_t len = a.len[r];
  if (len > cap) {
    len = cap;
    if (threadIdx.x == 0 && a.verdict) atomicOr(a.verdict, WM_C_LENGTH);
  }
  len = len > 0 ? len : 0;
  t->r = r;
  t->row0 = (uint32_t)nth * rows;
  t->n_rows = (uint32_t)n_rows;
  t->q0 = q0;
  t->len = (int32_t)len;
  t->pos0 = (int32_t)(len - (q1 - q0));
  const uint32_t last = t->row0 + rows < t->n_rows ? t->row0 + rows - 1 : t->n_rows - 1;
  const int64_t p_lo = (int64_t)t->pos0 + t->row0 / a.group;
  const int64_t p_hi = (int64_t)t->pos0 + last / a.group;
  int64_t lo = 0;
  if (a.window && p_lo + 1 > (int64_t)a.window) lo = p_lo + 1 - a.window;
  t->hi = p_hi + 1 > 0 ? (uint32_t)(p_hi + 1) : 0u;
  t->lo = (uint32_t)(lo < (int64_t)t->hi ? lo : t->hi);
  return true;
}

__device__ __forceinline__ uint32_t splits_of(const AttendArgs &a, const Tile &t) {
  const uint32_t s0 = t.lo >> 6, s1 = (t.hi + 63u) >> 6;
  return (s1 - s0 + a.plan.steps - 1) / a.plan.steps;
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

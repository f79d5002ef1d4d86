// wm_attend.h -- the attention kernel of the paged 8-bit cache, and its launch
// for one head size (each head size is compiled in a file of its own).
#pragma once
#include "wm_cache_device.h"

namespace wm {
namespace {

// exponent that weights (times their values' scales, in the row's unit) are
// raised by before they are rounded to half precision: at most 2^15 then, and
// one of 2^-29 of the largest still has all its bits (2^-40 its last one)
constexpr float kLift = 15.0f;
constexpr float kUnitLeast = -125.0f;  // 2^125 and 2^-125 are both normal numbers

// What a wave holds of its 16 NQ rows.  A lane has one row of each 16 (column
// lane % 16 of the matrix core's result) and of the output the dimensions
// 16 i + 4 (lane / 16) + 0..3.
template <int D, int NQ>
struct Rows {
  f32x4 o[NQ][D / 16];
  float m[NQ], l[NQ];  // maximum of the scores (base 2) and sum of the weights
  float most[NQ];      // maximum of weight times scale (base 2, from m on)
  bool special;        // (the whole wave's) values that are not finite were added
};

template <int D, int NQ>
__device__ __forceinline__ void clear(Rows<D, NQ> *w) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    w->m[n] = kNegInf;
    w->l[n] = 0.0f;
    w->most[n] = kNegInf;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) w->o[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  w->special = false;
}

__device__ __forceinline__ float or_zero(float x) { return x == kNegInf ? 0.0f : x; }

// The unit of a row's value sums, 2^(unit - kLift) with a whole number, where
// `most` is the largest weight times scale of what the row has seen (base 2, as
// scores are, and taken from the largest score, or scores of millions would
// leave it no bits).  So the parts that make up the sum are rounded to half
// precision with all their bits, whether the weight is large or the scale, and
// what the row does not see has no say in it.
__device__ __forceinline__ float unit_of(float most) {
  return fminf(fmaxf(ceilf(most), kUnitLeast), 127.0f);
}

// The maximum over the four lane groups that share a row.
__device__ __forceinline__ float group_max(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto p = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const float y = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  const uint32_t v = __float_as_uint(y);
  const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(q[0]), __uint_as_float(q[1]));
}

// Queries as the first product's right operand (column = row of the tile), the
// head's dimensions in the order in which the keys' 16-byte loads give them,
// and the rows' positions (-1: no row).
template <int DT, int FMT, int D, int NQ>
__device__ __forceinline__ void load_queries(const AttendArgs &a, const Request &x, uint32_t row0,
                                             uint32_t h,
                                             typename Qk<DT, FMT>::frag (&q)[NQ][D / 32],
                                             int (&pos)[NQ]) {
  typedef typename Qk<DT, FMT>::frag frag;
  const int lane = lane_id(), c16 = lane & 15, g = lane >> 4;
  const bool wide = (((uintptr_t)a.q.ptr >> 1 | a.q.row_stride | a.q.head_stride) & 7u) == 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t row = row0 + 16 * n + c16;
    const bool in = row < x.n_rows;
    const uint32_t tok = in ? row / a.group : 0u, hq = h * a.group + (in ? row % a.group : 0u);
    pos[n] = in ? x.pos0 + (int)tok : -1;
    const uint16_t *qp = (const uint16_t *)a.q.ptr + (uint64_t)(x.q0 + tok) * a.q.row_stride +
                         (uint64_t)hq * a.q.head_stride + g * 16;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const uint16_t *p = qp + (c >> 1) * 64 + (c & 1) * 8;
      u32x4 e;
      if (wide) {
        e = *(const u32x4 *)p;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = (uint32_t)p[2 * j] | (uint32_t)p[2 * j + 1] << 16;
      }
      q[n][c] = __builtin_bit_cast(frag, e);
    }
  }
}

// The last token before those that a row at `pos` sees, -1 if there is none.
__device__ __forceinline__ int before_window(const AttendArgs &a, int pos) {
  return a.window && pos >= (int)a.window ? pos - (int)a.window : -1;
}

// A wave's rows into the output, or as part `part` into the workspace if the
// tile has several.
template <int DT, int FMT, int D, int NQ>
__device__ __forceinline__ void store_rows(const AttendArgs &a, const Request &x, uint32_t row0,
                                           uint32_t h, const Rows<D, NQ> &w, float lift,
                                           bool whole, uint32_t part) {
  const int lane = lane_id(), c16 = lane & 15, g = lane >> 4;
  const bool wide = (((uintptr_t)a.out.ptr >> 1 | a.out.row_stride | a.out.head_stride) & 3u) == 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t row = row0 + 16 * n + c16;
    if (row >= x.n_rows) continue;
    const uint64_t tok = (uint64_t)x.q0 + row / a.group;
    const uint32_t hq = h * a.group + row % a.group;
    const float inv = w.l[n] > 0.0f || w.l[n] != w.l[n] ? ldexpf(1.0f / w.l[n], (int)unit_of(w.most[n])) : 0.0f;
    const float lse2 = w.l[n] == 0.0f ? kNegInf : w.m[n] + __builtin_amdgcn_logf(w.l[n]) - lift;
    if (!whole) {
      const uint64_t to = part_place(a, tok, hq) + part;
      float *po = a.part_out + to * D + 4 * g;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) *(f32x4 *)(po + 16 * j) = w.o[n][j] * inv;
      if (g == 0) a.part_lse[to] = lse2;
      continue;
    }
    uint16_t *op = (uint16_t *)a.out.ptr + tok * a.out.row_stride +
                   (uint64_t)hq * a.out.head_stride + 4 * g;
#pragma unroll
    for (int j = 0; j < D / 16; ++j) {
      uint32_t u = Qk<DT, FMT>::two(w.o[n][j][0] * inv, w.o[n][j][1] * inv);
      uint32_t v = Qk<DT, FMT>::two(w.o[n][j][2] * inv, w.o[n][j][3] * inv);
      // (or the compiler would round product and half apart for one kind of store
      // and at once for the other, and the bits would depend on the address)
      asm("" : "+v"(u), "+v"(v));
      if (wide) {
        *(u32x2 *)(op + 16 * j) = u32x2{u, v};
      } else {
        op[16 * j] = (uint16_t)u;
        op[16 * j + 1] = (uint16_t)(u >> 16);
        op[16 * j + 2] = (uint16_t)v;
        op[16 * j + 3] = (uint16_t)(v >> 16);
      }
    }
    if (g == 0 && a.lse)
      a.lse[tok * (a.group * a.c.n_heads) + hq] = lse2 * 0.6931471805599453f;
  }
}

// The work items of a call: a part of a tile of a request, for one key head.
// They are counted on the device, by a scan over the requests' lengths that
// every wave makes for itself, 64 requests at a time (a load, six shuffles and
// no barrier): lengths as different as 1 and 100,000 in one call leave no
// workgroup without work.
struct Item {
  uint32_t r, h, tile, part;
  Request x;
};

struct ItemWalk {
  Request *mine;        // LDS: the wave's 64 requests
  bool tell;            // say so of lengths and starts that are out of range
  uint64_t base = 0;    // items before them
  uint32_t r0 = 0, n = 0, sum = 0, all = 0;  // a lane's items, with those before it, all 64's

  __device__ __forceinline__ void scan(const AttendArgs &a) {
    const uint32_t r = r0 + lane_id();
    Request x = {};
    if (r < a.n_requests) x = request_of(a, r, tell);
    mine[lane_id()] = x;
    n = x.tiles * x.parts;
    sum = n;
    for (int i = 1; i < 64; i <<= 1) {
      const uint32_t y = __shfl_up(sum, i);
      if (lane_id() >= i) sum += y;
    }
    all = __builtin_amdgcn_readlane(sum, 63);
  }

  // Item `at` (ascending from call to call); false behind the last one.  A
  // request's last tiles come first: later rows see more.
  __device__ __forceinline__ bool find(const AttendArgs &a, uint64_t at, Item *it) {
    const uint64_t item = at / a.c.n_heads;
    it->h = (uint32_t)(at - item * a.c.n_heads);
    while (item - base >= all) {
      base += all;
      r0 += 64;
      if (r0 >= a.n_requests) return false;
      scan(a);
    }
    const uint32_t j = (uint32_t)(item - base);
    const uint32_t i = (uint32_t)__popcll(__ballot(sum <= j));
    if (i > 63) return false;  // starts that do not ascend
    const uint32_t k = j - (__builtin_amdgcn_readlane(sum, i) - __builtin_amdgcn_readlane(n, i));
    it->r = r0 + i;
    it->x = uniform(mine[i]);
    it->tile = it->x.tiles - 1 - k / it->x.parts;
    it->part = it->x.part0 + k % it->x.parts;
    return true;
  }
};

// The values of steps [first, last] that are not finite, for the rows that see
// them (a NaN may be added twice, which changes nothing).  A cache of finite
// values never gets here.
template <int FMT, int D, int NQ>
__device__ __forceinline__ void add_special(const AttendArgs &a, const Tile &t, uint32_t h,
                                            const int32_t *row, uint32_t first, uint32_t last,
                                            const int (&pos)[NQ], const int (&low)[NQ],
                                            Rows<D, NQ> *w) {
  const uint32_t bt = 1u << a.bt_log2;
  const int g = lane_id() >> 4;
  uint32_t j = first << 6, end = (last + 1) << 6;
  j = j < t.lo ? t.lo : j;
  end = end < t.hi ? end : t.hi;
#pragma unroll 1
  for (; j < end; ++j) {
    const int32_t id = row[j >> a.bt_log2];
    if ((uint32_t)id >= a.c.n_blocks) continue;
    const uint8_t *v = (const uint8_t *)a.c.v + (uint64_t)id * a.c.v_stride +
                       ((uint64_t)h * D + 4 * g) * bt + (j & (bt - 1));
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const uint32_t b = v[(uint64_t)(16 * i + k) * bt];
        const float y = Code<FMT>::special(b) & 0x80u ? Code<FMT>::value(b) : 0.0f;
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          w->o[n][i][k] += (int)j <= pos[n] && (int)j > low[n] ? y : 0.0f;
      }
  }
}

// Attention over a range of 64-token steps.  The scores are computed
// transposed, S^T = K Q^T, with key row 4 a + b of tile t being token 16 a +
// 4 t + b of the step: the result then leaves lane group a the weights of the
// 16 consecutive tokens from 16 a on, in the order in which the second
// product O^T = V^T P^T wants them as its right operand, and V^T's left
// operand is 16 consecutive codes of the transposed values.  So the weights
// never leave their lane, both operands come from memory in 16-byte loads
// without a detour through LDS, and 16 tokens never cross a block's end.
template <int DT, int FMT, int D, int NQ>
__device__ __forceinline__ void attend_steps(const AttendArgs &a, uint32_t r, const Request &x,
                                             const Tile &t, uint32_t h, uint32_t step0,
                                             uint32_t step1, Rows<D, NQ> *w) {
  typedef Qk<DT, FMT> T;
  typedef typename T::frag frag;
  constexpr int KC = D / 64, VT = D / 16;
  const int lane = lane_id(), c16 = lane & 15, g = lane >> 4, ka = c16 >> 2, kb = c16 & 3;
  const uint32_t bt = 1u << a.bt_log2;
  frag q[NQ][2 * KC];
  int pos[NQ];
  load_queries<DT, FMT, D, NQ>(a, x, t.row0, h, q, pos);
  // the lane's part of a block's keys and values
  const uint8_t *kbase = (const uint8_t *)a.c.k + ((uint64_t)h * bt + kb) * D + g * 16;
  const uint8_t *vbase = (const uint8_t *)a.c.v + ((uint64_t)h * D + c16) * bt;
  const int32_t *row = a.table + (uint64_t)r * a.table_stride;
  int low[NQ];  // the last token before those that a row sees
#pragma unroll
  for (int n = 0; n < NQ; ++n) low[n] = before_window(a, pos[n]);
  bool bad_page = false;
  // the table's entry for token j (a multiple of 16), and the block that it is:
  // -1 if no row sees its 16 tokens.  (The entry is looked at a step later,
  // when it is needed: looking at once would wait for it.)
  auto entry_of = [&](uint32_t j) {
    return row[(j < t.hi && j + 16 > t.lo ? j : t.lo) >> a.bt_log2];
  };
  auto block_of = [&](int32_t id, uint32_t j) -> int32_t {
    const bool in = j < t.hi && j + 16 > t.lo, out = in && (uint32_t)id >= a.c.n_blocks;
    bad_page |= out;
    return in && !out ? id : -1;
  };
  // A step's keys are loaded while the step before is between its two
  // products, its values while its own scores are computed: each load has a
  // product and a softmax to arrive in, with one step's registers.  (256
  // dimensions have none left for that; 192 spill about 60 for it, and 256
  // about 24 without.)
  constexpr bool kAhead = D < 256;
  u32x4 kr[4][KC], vr[VT];
  float ks = 0.0f, vs = 0.0f;
  // blocks that are not there are read at block 0 and masked
  auto load_keys = [&](int32_t id, uint32_t t0) {
    const uint8_t *kp = kbase + (uint64_t)(id < 0 ? 0 : id) * a.c.k_stride +
                        ((t0 + 16 * ka) & (bt - 1)) * D;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < KC; ++c) kr[i][c] = *(const u32x4 *)(kp + i * 4 * D + c * 64);
  };
  auto load_values = [&](int32_t id, uint32_t t0) {
    const uint8_t *vp = vbase + (uint64_t)(id < 0 ? 0 : id) * a.c.v_stride +
                        ((t0 + 16 * g) & (bt - 1));
#pragma unroll
    for (int i = 0; i < VT; ++i) vr[i] = *(const u32x4 *)(vp + (uint64_t)i * 16 * bt);
    ks = a.c.k_scale[(uint64_t)(id < 0 ? 0 : id) * a.c.k_scale_stride + h];
    vs = a.c.v_scale[(uint64_t)(id < 0 ? 0 : id) * a.c.v_scale_stride + h];
    vs = id < 0 ? 0.0f : vs;
  };
  int32_t idk = -1, idv = -1;  // the step's blocks
  int32_t ek = 0, ev = 0;      // the next one's entries
  auto entries = [&](uint32_t s) {
    ek = entry_of((s << 6) + 16 * ka);
    ev = entry_of((s << 6) + 16 * g);
  };
  auto blocks = [&](uint32_t s) {
    idk = block_of(ek, (s << 6) + 16 * ka);
    idv = block_of(ev, (s << 6) + 16 * g);
  };
  if (step0 < step1) entries(step0);
  if (kAhead && step0 < step1) {
    blocks(step0);
    entries(step0 + 4);
    load_keys(idk, step0 << 6);
    load_values(idv, step0 << 6);
  }
  uint32_t sp_first = ~0u, sp_last = 0;  // steps with values that were taken out
  for (uint32_t s = step0; s < step1; s += 4) {
    const uint32_t t0 = s << 6;
    const bool more = s + 4 < step1;
    if (!kAhead) {
      blocks(s);
      load_keys(idk, t0);
      load_values(idv, t0);
      entries(s + 4);
    }
    f32x4 sc[NQ][4];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[n][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        const frag k0 = T::key(kr[i][c][0], kr[i][c][1]), k1 = T::key(kr[i][c][2], kr[i][c][3]);
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          sc[n][i] = T::mma(k0, q[n][2 * c], sc[n][i]);
          sc[n][i] = T::mma(k1, q[n][2 * c + 1], sc[n][i]);
        }
      }
    if (kAhead && more) load_keys(block_of(ek, t0 + 256 + 16 * ka), t0 + 256);
    // masks: only where some row of the tile does not see some of the 64 tokens
    // (places behind the request's last row see none, so a tile that is not
    // full masks every step)
    const float cs = ks * a.scale_log2;
    const int first = (int)(t0 + 16 * g);  // the lane's first token
    bool partial = idv < 0;
#pragma unroll
    for (int n = 0; n < NQ; ++n) partial |= first + 15 > pos[n] || first <= low[n];
    const bool masked = __any(partial);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[n][i] *= cs;
    if (masked) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int end = idv < 0 ? -1 : pos[n] - first, begin = low[n] - first;
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (i > end || i <= begin) sc[n][i >> 2][i & 3] = kNegInf;
      }
    }
    const float vlog = __builtin_amdgcn_logf(vs);
    f16x8 p[NQ][2], p_low[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mine = kNegInf;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) mine = fmaxf(mine, sc[n][i][j]);
      const float top = fmaxf(w->m[n], group_max(mine));
      const float use = or_zero(top);  // nothing seen yet: every weight is 0
      const float most = fmaxf(w->most[n] + (w->m[n] - use), group_max(mine - use + vlog));
      const float was = unit_of(w->most[n]), unit = unit_of(most);
      const float keep = __builtin_amdgcn_exp2f(w->m[n] - use);
      const float shrink = ldexpf(keep, (int)(was - unit));
      // (finite, for the weights of 0 where the row does not see the block)
      const float vscale = fminf(ldexpf(vs, -(int)unit), 3.4028234e38f);
      w->m[n] = top;
      w->most[n] = most;
      w->l[n] *= keep;
#pragma unroll
      for (int i = 0; i < VT; ++i) w->o[n][i] *= shrink;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = __builtin_amdgcn_exp2f(sc[n][i][j] - use + kLift);
          w->l[n] += e;
          const float x = e * vscale;
          // weights in half precision (11 bits): a bf16 result loses nothing
          // to them; for half precision results a second term keeps the rest
          const _Float16 hi = (_Float16)x;
          p[n][i >> 1][(i & 1) * 4 + j] = hi;
          if (DT == WM_FP16) p_low[n][i >> 1][(i & 1) * 4 + j] = (_Float16)(x - (float)hi);
        }
    }
    // o + V^T P^T
    auto accumulate = [&](int n, int i, u32x4 codes) -> f32x4 {
      typedef Qk<WM_FP16, FMT> V;
      const f16x8 v0 = V::key(codes[0], codes[1]), v1 = V::key(codes[2], codes[3]);
      f32x4 o = w->o[n][i];
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][0], o, 0, 0, 0);
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][1], o, 0, 0, 0);
      if (DT == WM_FP16) {
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p_low[n][0], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p_low[n][1], o, 0, 0, 0);
      }
      return o;
    };
    // values that are not finite: a weight of 0 would not keep those that a
    // row does not see out of the product, and an infinity would meet weights
    // that are rounded to 0 or (the second term) below it.  They are taken out
    // here, and the rows that see them get them at the end.
    if ((masked || Code<FMT>::kInfinities) && take_special<FMT>(vr)) {
      sp_first = s < sp_first ? s : sp_first;
      sp_last = s;
    }
#pragma unroll
    for (int i = 0; i < VT; ++i)
#pragma unroll
      for (int n = 0; n < NQ; ++n) w->o[n][i] = accumulate(n, i, vr[i]);
    if (kAhead && more) {
      idv = block_of(ev, t0 + 256 + 16 * g);
      load_values(idv, t0 + 256);
      entries(s + 8);
    }
  }
  w->special = sp_first <= sp_last;
  if (w->special) add_special<FMT, D, NQ>(a, t, h, row, sp_first, sp_last, pos, low, w);
  // a lane has summed its own tokens: the rows' sums over the lane groups
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    w->l[n] += __shfl_xor(w->l[n], 16);
    w->l[n] += __shfl_xor(w->l[n], 32);
  }
  if (__any(bad_page) && lane == 0 && a.verdict) atomicOr(a.verdict, WM_C_PAGE);
}

// Four waves share a tile and take its steps in turn; then their parts are
// joined through LDS, two at a time (a lane's rows are the same in each wave).
template <int D, int NQ>
struct Parked {
  float o[NQ * (D / 4)][64], m[NQ][64], l[NQ][64], most[NQ][64];
  uint32_t special;
};

template <int D, int NQ>
__device__ __forceinline__ void park(const Rows<D, NQ> &w, Parked<D, NQ> *x, int lane) {
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) x->o[n * (D / 4) + 4 * i + j][lane] = w.o[n][i][j];
    x->m[n][lane] = w.m[n];
    x->l[n][lane] = w.l[n];
    x->most[n][lane] = w.most[n];
  }
  if (lane == 0) x->special = w.special;
}

template <int D, int NQ>
__device__ __forceinline__ void join(Rows<D, NQ> *w, const Parked<D, NQ> &x, int lane) {
  w->special |= __builtin_amdgcn_readfirstlane(x.special) != 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float mx = x.m[n][lane], top = fmaxf(w->m[n], mx);
    const float use = or_zero(top), r0 = w->most[n], r1 = x.most[n][lane];
    const float most = fmaxf(r0 + (w->m[n] - use), r1 + (mx - use));
    const float u0 = unit_of(r0), u1 = unit_of(r1), unit = unit_of(most);
    const float f0 = __builtin_amdgcn_exp2f(w->m[n] - use), f1 = __builtin_amdgcn_exp2f(mx - use);
    w->m[n] = top;
    w->l[n] = w->l[n] * f0 + x.l[n][lane] * f1;
    const float g0 = ldexpf(f0, (int)(u0 - unit)), g1 = ldexpf(f1, (int)(u1 - unit));
    w->most[n] = most;
    if (w->special) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w->o[n][i][j] = weighed(g0, w->o[n][i][j]) +
                          weighed(g1, x.o[n * (D / 4) + 4 * i + j][lane]);
      continue;
    }
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w->o[n][i][j] = w->o[n][i][j] * g0 + x.o[n * (D / 4) + 4 * i + j][lane] * g1;
  }
}

// Workgroups of a CU: two or three waves a SIMD, with a step each under way.
constexpr int resident(int d, int nq) {
  return d * nq <= 64 ? 3 : 2;
}

// Few rows: the grid is as large as the GPU holds, its workgroups take the
// items in turn.  HBM bounds it: 32 sessions of 24,576 to 32,768 tokens, 8 key
// heads of 128, read 1.9 GB in 374 us (5.1 TB/s); eight of 7,296 tokens and 16
// heads 239 MB in 52 us (4.6); 64 of 1 to 8,192 tokens 118 MB in 32 us (3.7),
// where parts of 512 tokens share 512 workgroups unevenly.  One session of 512
// tokens takes 9.1 us: the chain lengths, table, keys, softmax, join.
template <int DT, int FMT, int D, int NQ>
__global__ __launch_bounds__(kAttThreads, resident(D, NQ)) void k_attend(AttendArgs a) {
  __shared__ Parked<D, NQ> parked[2];
  __shared__ Request requests[kAttThreads];
  const int wave = threadIdx.x >> 6, lane = lane_id();
  ItemWalk walk;
  walk.mine = requests + 64 * wave;
  walk.tell = blockIdx.x == 0 && wave == 0;  // it goes through all requests
  walk.scan(a);
  Item it;
  for (uint64_t at = blockIdx.x; walk.find(a, at, &it); at += gridDim.x) {
    const Request &x = it.x;
    const Tile t = tile_of(a, x, it.tile);
    const bool none = t.part0 == t.part1;  // no row sees anything: the first item says so
    if (none ? it.part != x.part0 : (it.part < t.part0 || it.part >= t.part1)) continue;
    Rows<D, NQ> w;
    clear(&w);
    // steps of the part, wave w those that are w modulo 4
    uint32_t s0 = it.part << (x.cut - 6), s1 = (uint32_t)(((uint64_t)t.hi + 63) >> 6);
    if (s1 > s0 + (1u << (x.cut - 6))) s1 = s0 + (1u << (x.cut - 6));
    if (s0 < t.lo >> 6) s0 += ((t.lo >> 6) - s0) & ~3u;
    if (!none) attend_steps<DT, FMT, D, NQ>(a, it.r, x, t, it.h, s0 + wave, s1, &w);
    __syncthreads();  // wave 0 has read the item before's
    if (wave >= 2) park(w, &parked[wave - 2], lane);
    __syncthreads();
    if (wave < 2) join(&w, parked[wave], lane);
    __syncthreads();
    if (wave == 1) park(w, &parked[0], lane);
    __syncthreads();
    if (wave) continue;
    join(&w, parked[0], lane);
    const bool whole = t.part1 - t.part0 <= 1;
    store_rows<DT, FMT, D, NQ>(a, x, t.row0, it.h, w, kLift, whole, it.part - t.part0);
  }
}

// ---- many rows --------------------------------------------------------------
//
// Prompts: a tile of 128 rows, 16 NQ of them per wave, and every wave goes
// through all of the tile's steps.  A step's keys and values are converted
// once for all waves, each a share, and lie in LDS as the matrix instructions'
// left operands, 16 bytes a lane in lane order: reads and writes without bank
// conflicts.  Two steps' worth, so one barrier a step.
//
// Up to 128 dimensions four waves have two row blocks each.  Two leave room
// for a second wave on the SIMD, whose products run beside this one's
// exponentials (three or four blocks read LDS less often, but were slower:
// 288 and 524 us where two took 256).  192 dimensions and more: eight waves
// with a block each, so that the sums still fit into 256 registers; the tile
// is 128 rows either way.  (Spilled: 46 and 55 registers at 128 dimensions, 81
// and 105 over e5m2; up to 9 at 192, 32 to 45 at 256, none at 64.)
//
// What bounds it is the vector ALU beside the matrix cores (half a maximum, an
// exponential, two fused products and a rounding per score), so little else
// is done per score: scores are scaled within the exponent's product, which
// also takes the values' scale (the sum of the weights takes it out again), a
// row's maxima move only when one has grown 2^4 fold (weights are at most
// 2^15 all the same: the lift is 4 less), and steps that every row sees whole
// run in a loop without masks.
//
// Measured: 2,048 new tokens over 16,384 for four sessions, 32 query heads of
// 128, in 2,486 us, 940 TFLOP/s (a bf16 library product of 8192^3: 1300); 1,500
// to 2,048 over 1 to 4,096 in 228 us, 640 TFLOP/s.  A step takes 1.15 us a workgroup,
// of which the matrix cores are busy 0.43; a tile's start and end take about
// 10 us, a third of it for 64 KiB of queries and results.
constexpr float kSlack = 4.0f, kLiftMany = 11.0f;

constexpr int many_waves(int d) { return d <= 128 ? 4 : 8; }

// (Written out: fmaxf would first turn each operand's signalling NaN quiet.
// The compiler does not see that this reads its operands, so it does not keep
// the distance that a matrix instruction's result needs: settled() does, and
// a maximum that lanes exchange ends with an fmaxf.)
__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(y), "v"(z));
  return r;
}

// Results of matrix instructions that max3() may read: 16 wait states after
// the last of them, where the 16 x 16 ones need 11 at most.
template <int NQ>
__device__ __forceinline__ void settled(f32x4 (&x)[NQ][4]) {
  static_assert(NQ <= 2, "named below");
  if (NQ == 1)
    asm volatile("s_nop 15" : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[0][2]), "+v"(x[0][3]));
  else
    asm volatile("s_nop 15"
                 : "+v"(x[0][0]), "+v"(x[0][1]), "+v"(x[0][2]), "+v"(x[0][3]),
                   "+v"(x[NQ - 1][0]), "+v"(x[NQ - 1][1]), "+v"(x[NQ - 1][2]),
                   "+v"(x[NQ - 1][3]));
}

// The item of a workgroup.  Above 512 requests counting would take longer than
// the work, and an item's place alone says whose it is; some workgroups then
// have none (with few requests that would leave CUs idle: the ones with work
// would not be spread evenly).
__device__ __forceinline__ bool find_item(const AttendArgs &a, Request *mine, uint32_t at,
                                          Item *it) {
  if (a.n_requests <= 512) {
    ItemWalk walk;
    walk.mine = mine;
    walk.tell = false;
    walk.scan(a);
    return walk.find(a, at, it);
  }
  const uint32_t item = at / a.c.n_heads;
  it->h = at - item * a.c.n_heads;
  const Places pl = {a.q_start, a.n_requests, a.group, a.plan.rows, 1u};
  const uint32_t place = item / a.plan.splits, nth = item % a.plan.splits;
  it->r = __builtin_amdgcn_readfirstlane(pl.find(place));
  it->x = uniform(request_of(a, it->r, false));
  const uint32_t tile = place - __builtin_amdgcn_readfirstlane((uint32_t)pl.first(it->r));
  if (tile >= it->x.tiles || nth >= it->x.parts) return false;
  it->tile = it->x.tiles - 1 - tile;
  it->part = it->x.part0 + nth;
  return true;
}

struct Yes {
  static constexpr bool value = true;
};
struct No {
  static constexpr bool value = false;
};

template <int DT, int FMT, int D>
__global__ __launch_bounds__(64 * many_waves(D), 2) void k_attend_many(AttendArgs a) {
  typedef Qk<DT, FMT> T;
  typedef Qk<WM_FP16, FMT> V;
  typedef typename T::frag frag;
  constexpr int kWaves = many_waves(D), NQ = 8 / kWaves, KC = D / 64, VT = D / 16;
  // a wave's share of a step: of key tile wave % 4 every KS-th 64 dimensions,
  // and every kWaves-th value tile
  constexpr int KS = kWaves / 4, KW = (KC + KS - 1) / KS, VW = (VT + kWaves - 1) / kWaves;
  __shared__ u32x4 kf[2][8 * KC][64];  // [step][4 tiles x 2 KC][lane]
  __shared__ u32x4 vf[2][2 * VT][64];
  __shared__ uint32_t special[2][kWaves];  // the waves' sp_first and sp_last
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = lane_id();
  const int c16 = lane & 15, g = lane >> 4, ka = c16 >> 2, kb = c16 & 3;
  const uint32_t bt = 1u << a.bt_log2;
  __shared__ Request requests[64 * kWaves];
  Item it;
  const uint32_t place = blockIdx.y * gridDim.x + blockIdx.x;
  // (starts ascend: those beyond the rows show at either end)
  if (place == 0 && threadIdx.x == 0 && a.verdict &&
      (a.q_start[0] < 0 || (int64_t)a.q_start[a.n_requests] > (int64_t)a.n_tokens))
    atomicOr(a.verdict, WM_C_SLOTS);
  if (!find_item(a, requests + 64 * wave, place, &it)) return;
  // (every request with new tokens has an item, whose workgroup speaks for it)
  if (threadIdx.x == 0 && a.verdict &&
      (a.len[it.r] < 0 || (int64_t)a.len[it.r] > (int64_t)a.max_blocks << a.bt_log2))
    atomicOr(a.verdict, WM_C_LENGTH);
  const Request &x = it.x;
  const Tile t = tile_of(a, x, it.tile);
  const bool none = t.part0 == t.part1;
  if (none ? it.part != x.part0 : (it.part < t.part0 || it.part >= t.part1)) return;
  const uint32_t h = it.h, row0 = t.row0 + wave * 16 * NQ;
  frag q[NQ][2 * KC];
  int pos[NQ], low[NQ];
  load_queries<DT, FMT, D, NQ>(a, x, row0, h, q, pos);
#pragma unroll
  for (int n = 0; n < NQ; ++n) low[n] = before_window(a, pos[n]);
  // a negative factor of the scores goes into the queries
  const float scale = fabsf(a.scale_log2);
  if (a.scale_log2 < 0.0f) {
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int c = 0; c < 2 * KC; ++c)
        q[n][c] = __builtin_bit_cast(frag, __builtin_bit_cast(u32x4, q[n][c]) ^ 0x80008000u);
  }
  // tokens [w_lo, w_hi) are seen by some row of the wave (rows behind the
  // request's last are not stored: what they see does not matter)
  const uint32_t row1 = row0 + 16 * NQ - 1 < x.n_rows ? row0 + 16 * NQ - 1 : x.n_rows - 1;
  const int p_first = x.pos0 + (int)(row0 / a.group), p_last = x.pos0 + (int)(row1 / a.group);
  const bool idle = row0 >= x.n_rows;
  const int w_hi = idle ? 0 : p_last + 1;
  const int w_lo = a.window && p_first + 1 > (int)a.window ? p_first + 1 - (int)a.window : 0;
  Rows<D, NQ> w;
  clear(&w);
  const uint32_t s_part = it.part << (x.cut - 6);
  uint32_t s0 = t.lo >> 6, s1 = none ? 0u : (uint32_t)(((uint64_t)t.hi + 63) >> 6);
  if (s0 < s_part) s0 = s_part;
  if (s1 > s_part + (1u << (x.cut - 6))) s1 = s_part + (1u << (x.cut - 6));

  // the lane's place in a step's keys and values
  const uint32_t k_lane = (kb + 4 * (wave & 3)) * D + (wave >> 2) * 64 + g * 16;
  const uint32_t v_lane = (16 * wave + c16) * bt;
  const int32_t *row = a.table + (uint64_t)it.r * a.table_stride;
  bool bad_page = false;
  // the table's entry for the n tokens from j on, which lie in one block, and
  // the block that it is: -1 if no row sees its 16 tokens.  (The entry is
  // looked at a step later, when it is needed: looking at once would wait.)
  auto entry_of = [&](uint32_t j, uint32_t n) {
    return row[(j < t.hi && j + n > t.lo ? j : t.lo) >> a.bt_log2];
  };
  auto block_of = [&](int32_t id, uint32_t j) -> int32_t {
    const bool in = j < t.hi && j + 16 > t.lo, out = in && (uint32_t)id >= a.c.n_blocks;
    bad_page |= out;
    return in && !out ? id : -1;
  };
  // does the wave have share j of the keys, of the values?
  auto has_k = [&](int j) { return KC % KS == 0 || (wave >> 2) + KS * j < KC; };
  auto has_v = [&](int j) { return VT % kWaves == 0 || wave + kWaves * j < VT; };
  u32x4 kg[KW], vg[VW] = {};
  float ks1 = 0.0f, vs1 = 0.0f;
  int32_t idk1 = -1, idv1 = -1;  // blocks of the step that is loaded
  int32_t ek = 0, ev = 0;        // entries of the one after
  auto blocks = [&](uint32_t s) {
    if (a.bt_log2 >= 6) {
      ev = entry_of(s << 6, 64);
    } else {
      ek = entry_of((s << 6) + 16 * ka, 16);
      ev = entry_of((s << 6) + 16 * g, 16);
    }
  };
  auto load_from = [&](const uint8_t *kp, uint32_t k_off, const uint8_t *vp, uint32_t v_off) {
#pragma unroll
    for (int j = 0; j < KW; ++j)
      if (has_k(j)) kg[j] = *(const u32x4 *)(kp + (k_off + j * KS * 64));
#pragma unroll
    for (int j = 0; j < VW; ++j)
      if (has_v(j)) vg[j] = *(const u32x4 *)(vp + (uint64_t)j * kWaves * 16 * bt + v_off);
  };
  auto load = [&](uint32_t s) {
    const uint32_t t0 = s << 6;
    const uint8_t *kh = (const uint8_t *)a.c.k + (uint64_t)h * bt * D;
    const uint8_t *vh = (const uint8_t *)a.c.v + (uint64_t)h * bt * D;
    if (a.bt_log2 >= 6) {
      // a step lies in one block: one address for the wave, and 32-bit places
      const int32_t id = __builtin_amdgcn_readfirstlane(ev);
      const bool out = (uint32_t)id >= a.c.n_blocks;
      bad_page |= out;
      idk1 = idv1 = out ? -1 : id;
      const uint64_t at = out ? 0u : (uint64_t)id;
      load_from(kh + at * a.c.k_stride + (t0 & (bt - 1)) * D, k_lane + 16 * ka * D,
                vh + at * a.c.v_stride + (t0 & (bt - 1)), v_lane + 16 * g);
    } else {
      idk1 = block_of(ek, t0 + 16 * ka);
      idv1 = block_of(ev, t0 + 16 * g);
      load_from(kh + (uint64_t)(idk1 < 0 ? 0 : idk1) * a.c.k_stride +
                    ((t0 + 16 * ka) & (bt - 1)) * D, k_lane,
                vh + (uint64_t)(idv1 < 0 ? 0 : idv1) * a.c.v_stride + ((t0 + 16 * g) & (bt - 1)),
                v_lane);
    }
    ks1 = a.c.k_scale[(uint64_t)(idv1 < 0 ? 0 : idv1) * a.c.k_scale_stride + h];
    vs1 = a.c.v_scale[(uint64_t)(idv1 < 0 ? 0 : idv1) * a.c.v_scale_stride + h];
  };
  uint32_t sp_first = ~0u, sp_last = 0;  // steps with values that the wave took out
  bool far = false;  // maxima of the wave's rows beyond 2^20
  auto step = [&](uint32_t s, auto mask_tag) {
    constexpr bool kMasked = decltype(mask_tag)::value;
    const int b = s & 1;
    const int32_t idv = idv1;
    // a block that is not there: no codes that could be NaN, scales of 0
    const float ks = idv < 0 ? 0.0f : ks1, vs = idv < 0 ? 0.0f : vs1;
    const uint32_t k_there = idk1 < 0 ? 0u : ~0u, v_there = idv < 0 ? 0u : ~0u;
#pragma unroll
    for (int j = 0; j < KW; ++j)
      if (has_k(j)) {
        kg[j] &= k_there;
        const int at = (wave & 3) * 2 * KC + 2 * ((wave >> 2) + KS * j);
        kf[b][at][lane] = __builtin_bit_cast(u32x4, T::key(kg[j][0], kg[j][1]));
        kf[b][at + 1][lane] = __builtin_bit_cast(u32x4, T::key(kg[j][2], kg[j][3]));
      }
    // (a place without a share is 0 from the start)
#pragma unroll
    for (int j = 0; j < VW; ++j) vg[j] &= v_there;
    if (kMasked && take_special<FMT>(vg)) {  // as in attend_steps()
      sp_first = s < sp_first ? s : sp_first;
      sp_last = s;
    }
#pragma unroll
    for (int j = 0; j < VW; ++j)
      if (has_v(j)) {
        const int at = 2 * (wave + kWaves * j);
        vf[b][at][lane] = __builtin_bit_cast(u32x4, V::key(vg[j][0], vg[j][1]));
        vf[b][at + 1][lane] = __builtin_bit_cast(u32x4, V::key(vg[j][2], vg[j][3]));
      }
    if (s + 1 < s1) {
      load(s + 1);
      blocks(s + 2);
    }
    __syncthreads();
    const int t0 = (int)(s << 6);
    if (kMasked && (t0 >= w_hi || t0 + 63 < w_lo)) return;  // nothing for this wave
    f32x4 sc[NQ][4];
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[n][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // LDS is read four operands ahead of the products: the barriers keep the
    // compiler from putting a read right before its use
    u32x4 ahead[2][4];
#pragma unroll
    for (int c = 0; c < 4; ++c) ahead[0][c] = kf[b][c][lane];
#pragma unroll
    for (int j = 0; j < 2 * KC; ++j) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        ahead[(j + 1) & 1][c] = j + 1 < 2 * KC ? kf[b][4 * (j + 1) + c][lane] : vf[b][c][lane];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int i = (4 * j + c) / (2 * KC), d = (4 * j + c) % (2 * KC);
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          sc[n][i] = T::mma(__builtin_bit_cast(frag, ahead[j & 1][c]), q[n][d], sc[n][i]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    settled<NQ>(sc);
    const float cs = ks * scale;  // not negative: a row's largest score is its largest sum
    const int first = t0 + 16 * g;
    if (kMasked) {
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const int end = idv < 0 ? -1 : pos[n] - first, begin = low[n] - first;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float y = sc[n][i >> 2][i & 3] * cs;
          sc[n][i >> 2][i & 3] = i > end || i <= begin ? kNegInf : y;
        }
      }
    }
    const float f = kMasked ? 1.0f : cs;
    const float vlog = __builtin_amdgcn_logf(vs);
    float mine[NQ];  // the lane's largest score
    bool grows = false;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float y = max3(sc[n][0][0], sc[n][0][1], sc[n][0][2]);
#pragma unroll
      for (int i = 3; i < 15; i += 2)
        y = max3(y, sc[n][i >> 2][i & 3], sc[n][(i + 1) >> 2][(i + 1) & 3]);
      y = fmaxf(y, sc[n][3][3]) * f;
      mine[n] = !kMasked && idv < 0 ? kNegInf : y;
      const float d = mine[n] - w.m[n];
      grows |= d > kSlack || d + vlog > w.most[n] + kSlack;
    }
    if (__any(grows)) {
      bool high = false;
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float m = fmaxf(w.m[n], group_max(mine[n]));
        const float use = or_zero(m);
        const float most = fmaxf(w.most[n] + (w.m[n] - use), group_max(mine[n] - use + vlog));
        const float keep = __builtin_amdgcn_exp2f(w.m[n] - use);
        const float shrink = ldexpf(keep, (int)(unit_of(w.most[n]) - unit_of(most)));
        w.m[n] = m;
        w.most[n] = most;
        w.l[n] *= keep;
        high |= fabsf(use) > 0x1p20f;
#pragma unroll
        for (int i = 0; i < VT; ++i) w.o[n][i] *= shrink;
      }
      far = __any(high);
    }
    // Scores of a million and more leave the sum of exponents that follows no
    // bits: their maximum is taken off first, as they were rounded for it.
    if (far) {
#pragma clang fp contract(off)
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float y = sc[n][i >> 2][i & 3] * f;
          sc[n][i >> 2][i & 3] = y - or_zero(w.m[n]);
        }
    }
    const float fs = far ? 1.0f : f;
    f16x8 p[NQ][2], p_low[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      // the scale in the row's unit: far below it, it stays in the sum of the
      // weights alone.  (The empty asm keeps the compiler from carrying the unit
      // through the branch above, which took 100 registers.)
      float most = w.most[n];
      asm("" : "+v"(most));
      const int unit = (int)unit_of(most);
      const float ratio = fminf(fmaxf(ldexpf(vs, -unit), 0x1p-60f), 0x1p126f);
      const float back = __builtin_amdgcn_rcpf(ratio);
      float add = kLiftMany + __builtin_amdgcn_logf(ratio) - or_zero(far ? 0.0f : w.m[n]);
      if (!kMasked) add = idv < 0 ? kNegInf : add;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][i >> 2][i & 3], fs, add));
        w.l[n] = __builtin_fmaf(y, back, w.l[n]);
        const _Float16 hi = (_Float16)y;
        p[n][i >> 3][i & 7] = hi;
        if (DT == WM_FP16) p_low[n][i >> 3][i & 7] = (_Float16)(y - (float)hi);
      }
    }
    auto accumulate = [&](int n, f32x4 o, f16x8 v0, f16x8 v1) -> f32x4 {
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][0], o, 0, 0, 0);
      o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][1], o, 0, 0, 0);
      if (DT == WM_FP16) {
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p_low[n][0], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p_low[n][1], o, 0, 0, 0);
      }
      return o;
    };
#pragma unroll
    for (int i = 0; i < VT / 2; ++i) {
      if (i + 1 < VT / 2) {
#pragma unroll
        for (int c = 0; c < 4; ++c) ahead[(i + 1) & 1][c] = vf[b][4 * (i + 1) + c][lane];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int n = 0; n < NQ; ++n)
          w.o[n][2 * i + k] = accumulate(n, w.o[n][2 * i + k],
                                         __builtin_bit_cast(f16x8, ahead[i & 1][2 * k]),
                                         __builtin_bit_cast(f16x8, ahead[i & 1][2 * k + 1]));
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // steps [s_a, s_b) are seen whole by every row of the tile
  uint32_t s_a = s0, s_b = s1;
  {
    const uint32_t last = t.row0 + 127 < x.n_rows ? t.row0 + 127 : x.n_rows - 1;
    const int t_first = x.pos0 + (int)(t.row0 / a.group), t_last = x.pos0 + (int)(last / a.group);
    const uint32_t whole = t_first < 0 ? 0u : (uint32_t)(t_first + 1) >> 6;
    if (a.window && t_last + 1 > (int)a.window)
      s_a = (uint32_t)(t_last + 1 - (int)a.window + 63) >> 6;
    s_a = s_a < s0 ? s0 : (s_a > s1 ? s1 : s_a);
    s_b = whole < s_a ? s_a : (whole > s1 ? s1 : whole);
  }
  for (;;) {
    if (s0 < s1) {
      blocks(s0);
      load(s0);
      blocks(s0 + 1);
    }
    for (uint32_t s = s0; s < s1;) {
      const bool masked = s < s_a || s >= s_b;
      const uint32_t end = s < s_a ? s_a : (s < s_b ? s_b : s1);
      if (masked)
        for (; s < end; ++s) step(s, Yes{});
      else
        for (; s < end; ++s) step(s, No{});
    }
    // An infinity that met its weight (see attend_steps()) has left none of its
    // dimension's sums finite.  Then all steps go again as masked ones, which
    // take infinities out: looking for them in every step took 5% to 14%.
    if (!Code<FMT>::kInfinities || s_a >= s_b) break;
    float none = 0.0f;
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) none = __builtin_fmaf(w.o[n][i][j], 0.0f, none);
    if (!__syncthreads_or(!(none == 0.0f))) break;
    clear(&w);
    far = false;
    sp_first = ~0u;
    sp_last = 0;
    s_b = s_a = s0;
  }
  // each wave took out of its share, for the rows of all
  if (lane == 0) {
    special[0][wave] = sp_first;
    special[1][wave] = sp_last;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const uint32_t x = __builtin_amdgcn_readfirstlane(special[0][i]);
    const uint32_t y = __builtin_amdgcn_readfirstlane(special[1][i]);
    sp_first = x < sp_first ? x : sp_first;
    sp_last = y > sp_last ? y : sp_last;
  }
  if (sp_first <= sp_last)
    add_special<FMT, D, NQ>(a, t, h, row, sp_first, sp_last, pos, low, &w);
  if (__any(bad_page) && lane == 0 && a.verdict) atomicOr(a.verdict, WM_C_PAGE);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    w.l[n] += __shfl_xor(w.l[n], 16);
    w.l[n] += __shfl_xor(w.l[n], 32);
  }
  if (idle) return;
  const bool whole = t.part1 - t.part0 <= 1;
  store_rows<DT, FMT, D, NQ>(a, x, row0, h, w, kLiftMany, whole, it.part - t.part0);
}

template <int DT, int FMT, int D>
int attend_rows(const AttendArgs &a, hipStream_t st) {
  const uint64_t most = (uint64_t)a.plan.tiles * a.c.n_heads * a.plan.splits;
  if (a.plan.rows > 32) {
    // (fewer than 2^26: of the 2^30 rows and heads at most, requests have over 32
    // on average, and where they are many no sequence is cut)
    const dim3 grid(grid_x((uint32_t)most), grid_y((uint32_t)most));
    k_attend_many<DT, FMT, D><<<grid, 64 * many_waves(D), 0, st>>>(a);
    return (int)hipGetLastError();
  }
  const uint64_t room = (uint64_t)a.n_cu * resident(D, a.plan.rows / 16);
  const uint32_t grid = (uint32_t)(most < room ? most : room);
  if constexpr (D <= 64) {
    if (a.plan.rows == 32) {
      k_attend<DT, FMT, D, 2><<<grid, kAttThreads, 0, st>>>(a);
      return (int)hipGetLastError();
    }
  }
  k_attend<DT, FMT, D, 1><<<grid, kAttThreads, 0, st>>>(a);
  return (int)hipGetLastError();
}

template <int D>
int attend_dim(const AttendArgs &a, void *stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool e4 = a.c.format == WM_E4M3;
  if (a.q.dtype == WM_BF16)
    return e4 ? attend_rows<WM_BF16, WM_E4M3, D>(a, st) : attend_rows<WM_BF16, WM_E5M2, D>(a, st);
  return e4 ? attend_rows<WM_FP16, WM_E4M3, D>(a, st) : attend_rows<WM_FP16, WM_E5M2, D>(a, st);
}

}  // namespace
}  // namespace wm

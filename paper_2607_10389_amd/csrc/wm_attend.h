// wm_attend.h -- the attention kernel of the paged 8-bit cache, and its launch
// for one head size (each head size is compiled in a file of its own).
#pragma once
#include "wm_cache_device.h"

namespace wm {
namespace {

// exponent that weights are raised by before they are rounded to half
// precision: at most 2^15 then, and a weight of 2^-29 of the largest still has
// all its bits (2^-40 its last one)
constexpr float kLift = 15.0f;

// What a wave holds of its 16 NQ rows.  A lane has one row of each 16 (column
// lane % 16 of the matrix core's result) and of the output the dimensions
// 16 i + 4 (lane / 16) + 0..3.
template <int D, int NQ>
struct Rows {
  f32x4 o[NQ][D / 16];
  float m[NQ], l[NQ];  // maximum of the scores (base 2) and sum of the weights
  float vref;          // o is in units of vref 2^-kLift
};

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
  // queries: right operand, column = row of the tile, the same order of the
  // head's dimensions as the keys' loads give
  frag q[NQ][2 * KC];
  int pos[NQ];
  const bool wide = (((uintptr_t)a.q.ptr >> 1 | a.q.row_stride | a.q.head_stride) & 7u) == 0;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t row = t.row0 + 16 * n + c16;
    const bool in = row < x.n_rows;
    const uint32_t tok = in ? row / a.group : 0u, hq = h * a.group + (in ? row % a.group : 0u);
    pos[n] = in ? x.pos0 + (int)tok : -1;
    const uint16_t *qp = (const uint16_t *)a.q.ptr + (uint64_t)(x.q0 + tok) * a.q.row_stride +
                         (uint64_t)hq * a.q.head_stride + g * 16;
    if (wide) {
#pragma unroll
      for (int c = 0; c < 2 * KC; ++c)
        q[n][c] = __builtin_bit_cast(frag, *(const u32x4 *)(qp + (c >> 1) * 64 + (c & 1) * 8));
    } else {
#pragma unroll
      for (int c = 0; c < 2 * KC; ++c) {
        u32x4 e;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint16_t *p = qp + (c >> 1) * 64 + (c & 1) * 8 + 2 * j;
          e[j] = (uint32_t)p[0] | (uint32_t)p[1] << 16;
        }
        q[n][c] = __builtin_bit_cast(frag, e);
      }
    }
  }
  // the lane's part of a block's keys and values
  const uint8_t *kbase = (const uint8_t *)a.c.k + ((uint64_t)h * bt + kb) * D + g * 16;
  const uint8_t *vbase = (const uint8_t *)a.c.v + ((uint64_t)h * D + c16) * bt;
  const int32_t *row = a.table + (uint64_t)r * a.table_stride;
  int low[NQ];  // the last token before those that a row sees
#pragma unroll
  for (int n = 0; n < NQ; ++n) low[n] = a.window ? pos[n] - (int)a.window : -1;
  bool bad_page = false;
  // the block of token j (j a multiple of 16), -1 if no row sees its 16 tokens
  auto block_of = [&](uint32_t j) -> int32_t {
    const bool in = j < t.hi && j + 16 > t.lo;
    const int32_t id = row[(in ? j : t.lo) >> a.bt_log2];  // lo < hi: an entry of the table
    const bool out = in && (uint32_t)id >= a.c.n_blocks;
    bad_page |= out;
    return in && !out ? id : -1;
  };
  // A step's keys are loaded while the step before is between its two
  // products, its values while its own scores are computed: each load has a
  // product and a softmax to arrive in, with one step's registers.  (256
  // dimensions have none left for that.)
  constexpr bool kAhead = D * NQ <= 256 && D < 256;
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
  int32_t idk = -1, idv = -1, idk1 = -1, idv1 = -1;  // this step's, and the next one's blocks
  auto blocks = [&](uint32_t s) {
    idk1 = block_of((s << 6) + 16 * ka);
    idv1 = block_of((s << 6) + 16 * g);
  };
  if (step0 < step1) blocks(step0);
  if (kAhead && step0 < step1) {
    idk = idk1;
    idv = idv1;
    blocks(step0 + 4);
    load_keys(idk, step0 << 6);
    load_values(idv, step0 << 6);
  }
  for (uint32_t s = step0; s < step1; s += 4) {
    const uint32_t t0 = s << 6;
    const bool more = s + 4 < step1;
    if (!kAhead) {
      idk = idk1;
      idv = idv1;
      load_keys(idk, t0);
      load_values(idv, t0);
      blocks(s + 4);
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
    if (kAhead && more) load_keys(idk1, t0 + 256);
    // masks: only where some row does not see some of the 64 tokens
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
    // the values' unit: the largest scale so far
    float vmax = fabsf(vs);
    vmax = fmaxf(vmax, __shfl_xor(vmax, 16));
    vmax = fmaxf(vmax, __shfl_xor(vmax, 32));
    const float vref = fmaxf(w->vref, vmax);
    const float vscale = vs / vref, shrink = w->vref / vref;
    w->vref = vref;
    f16x8 p[NQ][2], p_low[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float top = w->m[n];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, sc[n][i][j]);
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const float use = top == kNegInf ? 0.0f : top;  // nothing seen yet: every weight is 0
      const float keep = __builtin_amdgcn_exp2f(w->m[n] - use);
      w->m[n] = top;
      w->l[n] *= keep;
#pragma unroll
      for (int i = 0; i < VT; ++i) w->o[n][i] *= keep * shrink;
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
    // values that are not finite and that some row does not see: a weight of
    // 0 would not keep them out of the product
    bool special = false;
    if (masked) {
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) any |= Code<FMT>::special(vr[i][j]);
      special = __any((any & 0x80808080u) != 0);
    }
    if (special) {
      // a row at a time, with only the codes that it sees (a loop that a cache
      // of finite values never enters); a weight below half precision counts
      // as its smallest, so that an infinity stays one
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (sc[n][i >> 2][i & 3] > kNegInf && p[n][i >> 3][i & 7] == (_Float16)0.0f)
            p[n][i >> 3][i & 7] = (_Float16)copysignf(0x1p-24f, vscale);
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll 1
        for (int c = 0; c < 16; ++c) {
          // the places that row c sees (every lane asks lane c)
          const int last = __shfl(pos[n], c) - first, begin = __shfl(low[n], c) - first;
          const int end = idv < 0 ? -1 : last;
          u32x4 m;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            m[i] = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (4 * i + j <= end && 4 * i + j > begin) m[i] |= 0xFFu << (8 * j);
          }
#pragma unroll
          for (int i = 0; i < VT; ++i) {
            const f32x4 o = accumulate(n, i, vr[i] & m);
            if (c16 == c) w->o[n][i] = o;
          }
        }
    } else {
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int n = 0; n < NQ; ++n) w->o[n][i] = accumulate(n, i, vr[i]);
    }
    if (kAhead && more) {
      idv = idv1;
      load_values(idv, t0 + 256);
      blocks(s + 8);
    }
  }
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
  float o[NQ * (D / 4)][64], m[NQ][64], l[NQ][64], vref[64];
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
  }
  x->vref[lane] = w.vref;
}

template <int D, int NQ>
__device__ __forceinline__ void join(Rows<D, NQ> *w, const Parked<D, NQ> &x, int lane) {
  const float vx = x.vref[lane], vref = fmaxf(w->vref, vx);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const float mx = x.m[n][lane], top = fmaxf(w->m[n], mx);
    const float use = top == kNegInf ? 0.0f : top;
    const float f0 = __builtin_amdgcn_exp2f(w->m[n] - use), f1 = __builtin_amdgcn_exp2f(mx - use);
    w->m[n] = top;
    w->l[n] = w->l[n] * f0 + x.l[n][lane] * f1;
    const float g0 = f0 * (w->vref / vref), g1 = f1 * (vx / vref);
#pragma unroll
    for (int i = 0; i < D / 16; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        w->o[n][i][j] = w->o[n][i][j] * g0 + x.o[n * (D / 4) + 4 * i + j][lane] * g1;
  }
  w->vref = vref;
}

// Workgroups of a CU: two or three waves a SIMD, with a step each under way.
constexpr int resident(int d, int nq) {
  return d * nq <= 64 ? 3 : 2;
}

// The grid is as large as the GPU holds; its workgroups take the work items
// (a part of a tile of a request, for one key head) in turn.  The items are counted on the
// device, by a scan over the requests' lengths that every workgroup makes
// for itself, 256 requests at a time: lengths as different as 1 and 100,000
// in one call leave no workgroup without work and none with a long rest.
template <int DT, int FMT, int D, int NQ>
__global__ __launch_bounds__(kAttThreads, resident(D, NQ)) void k_attend(AttendArgs a) {
  __shared__ Parked<D, NQ> parked[2];
  __shared__ uint64_t pre[kAttThreads + 1], sums[kAttThreads / 64];
  __shared__ Request req[kAttThreads];
  const int wave = threadIdx.x >> 6, lane = lane_id();
  const uint32_t heads = a.c.n_heads;
  uint64_t base = 0;  // items before the requests in pre
  uint32_t r0 = 0;
  auto scan = [&]() {
    const uint32_t r = r0 + threadIdx.x;
    Request x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (r < a.n_requests) x = request_of(a, r, blockIdx.x == 0);
    uint64_t n = (uint64_t)x.tiles * x.parts;
    for (int i = 1; i < 64; i <<= 1) {
      const uint64_t y = __shfl_up(n, i);
      if (lane >= i) n += y;
    }
    __syncthreads();  // pre's readers are done
    if (lane == 63) sums[wave] = n;
    __syncthreads();
    for (int i = 0; i < wave; ++i) n += sums[i];
    pre[threadIdx.x + 1] = n;
    if (threadIdx.x == 0) pre[0] = 0;
    req[threadIdx.x] = x;
    __syncthreads();
  };
  scan();
  for (uint64_t at = blockIdx.x;; at += gridDim.x) {
    const uint64_t item = at / heads;
    const uint32_t h = (uint32_t)(at - item * heads);
    while (item - base >= pre[kAttThreads]) {
      base += pre[kAttThreads];
      r0 += kAttThreads;
      if (r0 >= a.n_requests) return;
      scan();
    }
    uint32_t i = 0;
#pragma unroll
    for (int k = kAttThreads / 2; k; k >>= 1)
      if (pre[i + k] <= item - base) i += k;
    i = __builtin_amdgcn_readfirstlane(i);
    const uint32_t r = r0 + i;
    const Request x = uniform(req[i]);
    const uint32_t k = (uint32_t)(item - base - pre[i]);
    const uint32_t tile = __builtin_amdgcn_readfirstlane(k / x.parts);
    const uint32_t part = __builtin_amdgcn_readfirstlane(x.part0 + k % x.parts);
    const Tile t = tile_of(a, x, tile);
    const bool none = t.part0 == t.part1;  // no row sees anything: the first item says so
    if (none ? part != x.part0 : (part < t.part0 || part >= t.part1)) continue;
    Rows<D, NQ> w;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      w.m[n] = kNegInf;
      w.l[n] = 0.0f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) w.o[n][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    w.vref = 0x1p-125f;  // below it a scale has no exact reciprocal
    // steps of the part, wave w those that are w modulo 4
    uint32_t s0 = part << (x.cut - 6), s1 = (uint32_t)(((uint64_t)t.hi + 63) >> 6);
    if (s1 > s0 + (1u << (x.cut - 6))) s1 = s0 + (1u << (x.cut - 6));
    if (s0 < t.lo >> 6) s0 += ((t.lo >> 6) - s0) & ~3u;
    if (!none) attend_steps<DT, FMT, D, NQ>(a, r, x, t, h, s0 + wave, s1, &w);
    __syncthreads();  // wave 0 has read the item before's
    if (wave >= 2) park(w, &parked[wave - 2], lane);
    __syncthreads();
    if (wave < 2) join(&w, parked[wave], lane);
    __syncthreads();
    if (wave == 1) park(w, &parked[0], lane);
    __syncthreads();
    if (wave) continue;
    join(&w, parked[0], lane);
    const int c16 = lane & 15, g = lane >> 4;
    const uint32_t n_parts = t.part1 - t.part0;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const uint32_t row = t.row0 + 16 * n + c16;
      if (row >= x.n_rows) continue;
      const float inv = w.l[n] > 0.0f || w.l[n] != w.l[n] ? w.vref / w.l[n] : 0.0f;
      const float lse2 = w.l[n] == 0.0f ? kNegInf : w.m[n] + __builtin_amdgcn_logf(w.l[n]) - kLift;
      if (n_parts > 1) {
        const uint64_t to = part_place(a, x, r, tile, part - t.part0, h) + 16 * n + c16;
        float *po = a.part_out + to * D + 4 * g;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) *(f32x4 *)(po + 16 * j) = w.o[n][j] * inv;
        if (g == 0) a.part_lse[to] = lse2;
      } else {
        const uint32_t tok = row / a.group, hq = h * a.group + row % a.group;
        uint16_t *op = (uint16_t *)a.out.ptr + (uint64_t)(x.q0 + tok) * a.out.row_stride +
                       (uint64_t)hq * a.out.head_stride + 4 * g;
        const bool wide =
            (((uintptr_t)a.out.ptr >> 1 | a.out.row_stride | a.out.head_stride) & 3u) == 0;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          const uint32_t u = Qk<DT, FMT>::two(w.o[n][j][0] * inv, w.o[n][j][1] * inv);
          const uint32_t v = Qk<DT, FMT>::two(w.o[n][j][2] * inv, w.o[n][j][3] * inv);
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
          a.lse[(uint64_t)(x.q0 + tok) * (a.group * heads) + hq] = lse2 * 0.6931471805599453f;
      }
    }
  }
}

template <int DT, int FMT, int D>
int attend_rows(const AttendArgs &a, hipStream_t st) {
  const uint64_t most = (uint64_t)a.plan.tiles * a.c.n_heads * a.plan.splits;
  const uint64_t room = (uint64_t)a.n_cu * resident(D, a.plan.rows / 16);
  const uint32_t grid = (uint32_t)(most < room ? most : room);
  if (a.plan.rows == 16)
    k_attend<DT, FMT, D, 1><<<grid, kAttThreads, 0, st>>>(a);
  else
    k_attend<DT, FMT, D, 2><<<grid, kAttThreads, 0, st>>>(a);
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

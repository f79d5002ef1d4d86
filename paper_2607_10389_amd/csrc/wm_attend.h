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
__device__ __forceinline__ void attend_steps(const AttendArgs &a, const Tile &t, uint32_t h,
                                             uint32_t step0, uint32_t step1, uint32_t stride,
                                             Rows<D, NQ> *w) {
  typedef Qk<DT, FMT> T;
  typedef typename T::frag frag;
  constexpr int KC = D / 64, VT = D / 16;
  const int lane = lane_id(), c16 = lane & 15, g = lane >> 4, ka = c16 >> 2, kb = c16 & 3;
  const uint32_t bt = 1u << a.bt_log2;
  // queries: right operand, column = row of the tile, the same order of the
  // head's dimensions as the keys' loads give
  frag q[NQ][2 * KC];
  int pos[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t row = t.row0 + 16 * n + c16;
    const bool in = row < t.n_rows;
    const uint32_t tok = in ? row / a.group : 0u, hq = h * a.group + (in ? row % a.group : 0u);
    pos[n] = in ? t.pos0 + (int)tok : -1;
    const uint16_t *qp = (const uint16_t *)a.q.ptr + (uint64_t)(t.q0 + tok) * a.q.row_stride +
                         (uint64_t)hq * a.q.head_stride + g * 16;
#pragma unroll
    for (int c = 0; c < 2 * KC; ++c) {
      uint16_t e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) e[j] = qp[(c >> 1) * 64 + (c & 1) * 8 + j];
      u32x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = (uint32_t)e[2 * j] | (uint32_t)e[2 * j + 1] << 16;
      q[n][c] = __builtin_bit_cast(frag, x);
    }
  }
  const uint8_t *kbase = (const uint8_t *)a.c.k + (uint64_t)h * bt * D;
  const uint8_t *vbase = (const uint8_t *)a.c.v + (uint64_t)h * bt * D;
  const int32_t *row = a.table + (uint64_t)t.r * a.table_stride;
  bool bad_page = false;
  // the block of token j (j a multiple of 16), -1 if no row sees its 16 tokens
  auto block_of = [&](uint32_t j) -> int32_t {
    if (j >= t.hi || j + 16 <= t.lo) return -1;
    const int32_t id = row[j >> a.bt_log2];
    if ((uint32_t)id >= a.c.n_blocks) {
      bad_page = true;
      return -1;
    }
    return id;
  };
  for (uint32_t s = step0; s < step1; s += stride) {
    const uint32_t t0 = s << 6;
    const int32_t idk = block_of(t0 + 16 * ka), idv = block_of(t0 + 16 * g);
    // blocks that are not there are read at block 0 and masked
    const uint8_t *kp = kbase + (uint64_t)(idk < 0 ? 0 : idk) * a.c.k_stride +
                        (((t0 + 16 * ka) & (bt - 1)) + kb) * D + g * 16;
    const uint8_t *vp = vbase + (uint64_t)(idv < 0 ? 0 : idv) * a.c.v_stride + (uint64_t)c16 * bt +
                        ((t0 + 16 * g) & (bt - 1));
    u32x4 kr[4][KC], vr[VT];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int c = 0; c < KC; ++c) kr[i][c] = *(const u32x4 *)(kp + i * 4 * D + c * 64);
#pragma unroll
    for (int i = 0; i < VT; ++i) vr[i] = *(const u32x4 *)(vp + (uint64_t)i * 16 * bt);
    float ks = 0.0f, vs = 0.0f;
    if (idv >= 0) {
      ks = a.c.k_scale[(uint64_t)idv * a.c.k_scale_stride + h];
      vs = a.c.v_scale[(uint64_t)idv * a.c.v_scale_stride + h];
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
    // masks: only where some row does not see some of the 64 tokens
    const float cs = ks * a.scale_log2;
    const int first = (int)(t0 + 16 * g);  // the lane's first token
    bool partial = idv < 0;
#pragma unroll
    for (int n = 0; n < NQ; ++n)
      partial |= first + 15 > pos[n] || (a.window && first <= pos[n] - (int)a.window);
    const bool masked = __any(partial);
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sc[n][i] *= cs;
        if (masked) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int tok = first + 4 * i + j;
            const bool seen = idv >= 0 && tok <= pos[n] &&
                              (!a.window || tok > pos[n] - (int)a.window);
            sc[n][i][j] = seen ? sc[n][i][j] : kNegInf;
          }
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
    // values that are not finite and that some row does not see: a weight of
    // 0 would not keep them out of the product
    bool special = false;
    if (masked) {
#pragma unroll
      for (int i = 0; i < VT; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          special |= Code<FMT>::special((vr[i][j >> 2] >> (8 * (j & 3))) & 0xFFu);
      special = __any(special);
    }
    if (special) {
      // the rows' count of NaN, +inf and -inf that they see (1, 2^7 and 2^14
      // each, at most 64 of them: exact) in place of those codes
      f16x8 seen[NQ][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int j = 0; j < 16; ++j)
          seen[n][j >> 3][j & 7] = sc[n][j >> 2][j & 3] == kNegInf ? (_Float16)0.0f : (_Float16)1.0f;
#pragma unroll
      for (int i = 0; i < VT; ++i) {
        f16x8 mark[2];
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t sh = 8 * (j & 3), b = (vr[i][j >> 2] >> sh) & 0xFFu;
          const bool sp = Code<FMT>::special(b);
          mark[j >> 3][j & 7] = !sp ? (_Float16)0.0f
                                    : (!Code<FMT>::infinite(b) ? (_Float16)1.0f
                                                               : (b & 0x80u ? (_Float16)16384.0f
                                                                            : (_Float16)128.0f));
          if (sp) vr[i][j >> 2] &= ~(0xFFu << sh);
        }
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          f32x4 cnt = {0.0f, 0.0f, 0.0f, 0.0f};
          cnt = __builtin_amdgcn_mfma_f32_16x16x32_f16(mark[0], seen[n][0], cnt, 0, 0, 0);
          cnt = __builtin_amdgcn_mfma_f32_16x16x32_f16(mark[1], seen[n][1], cnt, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t u = (uint32_t)cnt[j];
            const bool nan = (u & 127u) || (((u >> 7) & 127u) && (u >> 14));
            if (nan)
              w->o[n][i][j] = __builtin_nanf("");
            else if (u >> 14)
              w->o[n][i][j] += kNegInf;
            else if ((u >> 7) & 127u)
              w->o[n][i][j] -= kNegInf;
          }
        }
      }
    }
#pragma unroll
    for (int i = 0; i < VT; ++i) {
      typedef Qk<WM_FP16, FMT> V;
      const f16x8 v0 = V::key(vr[i][0], vr[i][1]), v1 = V::key(vr[i][2], vr[i][3]);
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        f32x4 o = w->o[n][i];
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p[n][0], o, 0, 0, 0);
        o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p[n][1], o, 0, 0, 0);
        if (DT == WM_FP16) {
          o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, p_low[n][0], o, 0, 0, 0);
          o = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, p_low[n][1], o, 0, 0, 0);
        }
        w->o[n][i] = o;
      }
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

template <int DT, int FMT, int D, int NQ>
__global__ __launch_bounds__(kAttThreads) void k_attend(AttendArgs a) {
  __shared__ Parked<D, NQ> parked[2];
  Tile t;
  if (!tile_of(a, blockIdx.x, &t)) return;
  const uint32_t h = blockIdx.y, z = blockIdx.z;
  uint32_t n_split = splits_of(a, t);
  n_split = n_split < gridDim.z ? n_split : gridDim.z;
  if (z && z >= n_split) return;
  const int wave = threadIdx.x >> 6, lane = lane_id();
  Rows<D, NQ> w;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    w.m[n] = kNegInf;
    w.l[n] = 0.0f;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) w.o[n][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  w.vref = 0x1p-125f;  // below it a scale has no exact reciprocal
  const uint32_t first = (t.lo >> 6) + z * a.plan.steps, all = (t.hi + 63u) >> 6;
  uint32_t last = first + a.plan.steps;
  // the last split place takes what a longer sequence than max_len has left
  if (last > all || z + 1 == gridDim.z) last = all;
  attend_steps<DT, FMT, D, NQ>(a, t, h, first + wave, last, 4, &w);
  if (wave >= 2) park(w, &parked[wave - 2], lane);
  __syncthreads();
  if (wave < 2) join(&w, parked[wave], lane);
  __syncthreads();
  if (wave == 1) park(w, &parked[0], lane);
  __syncthreads();
  if (wave) return;
  join(&w, parked[0], lane);
  const int c16 = lane & 15, g = lane >> 4;
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const uint32_t row = t.row0 + 16 * n + c16;
    if (row >= t.n_rows) continue;
    const float inv = w.l[n] > 0.0f || w.l[n] != w.l[n] ? w.vref / w.l[n] : 0.0f;
    const float lse2 = w.l[n] == 0.0f ? kNegInf : w.m[n] + __builtin_amdgcn_logf(w.l[n]) - kLift;
    if (n_split > 1) {
      const uint64_t at = (((uint64_t)blockIdx.x * gridDim.y + h) * gridDim.z + z) * (16 * NQ) +
                          (16 * n + c16);
      float *po = a.part_out + at * D + 4 * g;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) *(f32x4 *)(po + 16 * i) = w.o[n][i] * inv;
      if (g == 0) a.part_lse[at] = lse2;
    } else {
      const uint32_t tok = row / a.group, hq = h * a.group + row % a.group;
      uint16_t *op = (uint16_t *)a.out.ptr + (uint64_t)(t.q0 + tok) * a.out.row_stride +
                     (uint64_t)hq * a.out.head_stride + 4 * g;
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        const uint32_t x = Qk<DT, FMT>::two(w.o[n][i][0] * inv, w.o[n][i][1] * inv);
        const uint32_t y = Qk<DT, FMT>::two(w.o[n][i][2] * inv, w.o[n][i][3] * inv);
        op[16 * i] = (uint16_t)x;
        op[16 * i + 1] = (uint16_t)(x >> 16);
        op[16 * i + 2] = (uint16_t)y;
        op[16 * i + 3] = (uint16_t)(y >> 16);
      }
      if (g == 0 && a.lse)
        a.lse[(uint64_t)(t.q0 + tok) * (a.group * a.c.n_heads) + hq] = lse2 * 0.6931471805599453f;
    }
  }
}

template <int DT, int FMT, int D>
int attend_rows(const AttendArgs &a, hipStream_t st) {
  const dim3 grid(a.plan.tiles, a.c.n_heads, a.plan.splits);
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

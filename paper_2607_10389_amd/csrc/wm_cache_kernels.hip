// wm_cache_kernels.hip -- the paged 8-bit attention cache on gfx950: block
// tables and slot maps, the store of new keys and values, attention over the
// cache, and a session's blocks to and from the flat state.
//
// Every index that comes from the device (lengths, starts, blocks, slots) is
// checked against the buffers before it is used.
#include "wm_cache_device.h"

namespace wm {
namespace {

// ---- block tables and slot maps ---------------------------------------------

// A scan over the requests: every workgroup scans all lengths (8 bytes a
// request, from L2 but for the first) and so knows by itself, before it
// writes, whether the step is possible and where each request's blocks and
// tokens lie; the writes are then divided over the grid.  No workgroup waits
// for another.  What is written is never read by the same call: taken and
// returned places of the ring are disjoint (count + returns <= capacity), and
// a table entry is read only where it was in use before.
constexpr int kTabThreads = 1024;

struct Step {
  int32_t o, n;
  uint32_t b, c, tokens, need, give;
};

__device__ __forceinline__ Step step_of(const TablesArgs &a, uint32_t r) {
  Step s = {0, 0, 0, 0, 0, 0, 0};
  if (r >= a.n_requests) return s;
  s.o = a.old_len[r];
  s.n = a.new_len[r];
  const uint32_t round = (1u << a.bt_log2) - 1u;
  // a negative length becomes a large count that fails the check
  s.b = (uint32_t)(((uint64_t)(uint32_t)s.o + round) >> a.bt_log2);
  s.c = (uint32_t)(((uint64_t)(uint32_t)s.n + round) >> a.bt_log2);
  s.tokens = s.n > s.o ? (uint32_t)(s.n - s.o) : 0u;
  s.need = s.c > s.b ? s.c - s.b : 0u;
  s.give = s.b > s.c ? s.b - s.c : 0u;
  return s;
}

__global__ __launch_bounds__(kTabThreads) void k_page_tables(TablesArgs a) {
  __shared__ uint64_t sum[3][kTabThreads / 64];
  __shared__ uint64_t pre[3][kTabThreads + 1];
  __shared__ Step st[kTabThreads];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t head = a.pool_in[0], count = a.pool_in[1];
  // pass 1: totals
  uint64_t tok = 0, need = 0, give = 0;
  bool bad = false;
  for (uint32_t r = tid; r < a.n_requests; r += kTabThreads) {
    const Step s = step_of(a, r);
    bad |= s.o < 0 || s.n < 0 || s.b > a.max_blocks || s.c > a.max_blocks;
    tok += s.tokens;
    need += s.need;
    give += s.give;
  }
  for (int i = 32; i; i >>= 1) {
    tok += __shfl_xor(tok, i);
    need += __shfl_xor(need, i);
    give += __shfl_xor(give, i);
  }
  if (lane == 0) {
    sum[0][wave] = tok;
    sum[1][wave] = need;
    sum[2][wave] = give;
  }
  bad = __syncthreads_or(bad);
  tok = need = give = 0;
  for (int i = 0; i < kTabThreads / 64; ++i) {
    tok += sum[0][i];
    need += sum[1][i];
    give += sum[2][i];
  }
  uint32_t v = 0;
  if (need > count || count + give > a.ring_cap || head >= a.ring_cap) v |= WM_C_POOL;
  if (tok > a.slot_cap) v |= WM_C_SLOTS;
  if (bad) v = WM_C_LENGTH;  // the other counts mean nothing then
  if (blockIdx.x == 0 && tid == 0) {
    *a.verdict = v;
    a.pool_out[0] = v ? head : (uint32_t)((head + need) % a.ring_cap);
    a.pool_out[1] = v ? count : (uint32_t)(count - need + give);
    if (!v) a.q_start[a.n_requests] = (int32_t)tok;
  }
  if (v) return;
  // pass 2: a tile of requests at a time
  const uint64_t step = (uint64_t)gridDim.x * kTabThreads;
  const uint64_t at = (uint64_t)blockIdx.x * kTabThreads + tid;
  const uint32_t bt = 1u << a.bt_log2;
  uint64_t base[3] = {0, 0, 0};
  for (uint32_t r0 = 0; r0 < a.n_requests; r0 += kTabThreads) {
    __syncthreads();  // the tile before is done with the shared arrays
    const uint32_t r = r0 + tid;
    const Step s = step_of(a, r);
    st[tid] = s;
    uint64_t x[3] = {s.tokens, s.need, s.give};
    for (int i = 1; i < 64; i <<= 1)
      for (int k = 0; k < 3; ++k) {
        const uint64_t y = __shfl_up(x[k], i);
        if (lane >= i) x[k] += y;
      }
    if (lane == 63)
      for (int k = 0; k < 3; ++k) sum[k][wave] = x[k];
    __syncthreads();
    for (int k = 0; k < 3; ++k) {
      uint64_t w = base[k];
      for (int i = 0; i < wave; ++i) w += sum[k][i];
      pre[k][tid + 1] = w + x[k];
      if (tid == 0) pre[k][0] = base[k];
    }
    __syncthreads();
    if (blockIdx.x == 0 && r < a.n_requests) a.q_start[r] = (int32_t)pre[0][tid];
    auto owner = [&](int k, uint64_t j) {  // the last request whose part begins at or before j
      int lo = 0, hi = kTabThreads;
      while (hi - lo > 1) {
        const int m = (lo + hi) >> 1;
        if (pre[k][m] <= j)
          lo = m;
        else
          hi = m;
      }
      return lo;
    };
    for (uint64_t j = pre[1][0] + at; j < pre[1][kTabThreads]; j += step) {
      const int i = owner(1, j);
      a.table[(uint64_t)(r0 + i) * a.table_stride + st[i].b + (uint32_t)(j - pre[1][i])] =
          a.ring[(head + j) % a.ring_cap];
    }
    for (uint64_t j = pre[2][0] + at; j < pre[2][kTabThreads]; j += step) {
      const int i = owner(2, j);
      a.ring[(head + count + j) % a.ring_cap] =
          a.table[(uint64_t)(r0 + i) * a.table_stride + st[i].c + (uint32_t)(j - pre[2][i])];
    }
    for (uint64_t j = pre[0][0] + at; j < pre[0][kTabThreads]; j += step) {
      const int i = owner(0, j);
      const uint32_t p = (uint32_t)st[i].o + (uint32_t)(j - pre[0][i]);
      const uint32_t blk = p >> a.bt_log2;
      const int32_t id = blk < st[i].b
                             ? a.table[(uint64_t)(r0 + i) * a.table_stride + blk]
                             : a.ring[(head + pre[1][i] + (blk - st[i].b)) % a.ring_cap];
      a.slots[j] = (int64_t)id * bt + (p & (bt - 1u));
    }
    for (int k = 0; k < 3; ++k) base[k] = pre[k][kTabThreads];
  }
}

// ---- store new keys and values -----------------------------------------------

constexpr int kAppThreads = 256;

// The scale of a block that gets values of magnitude up to amax.  448 = 0.875
// 2^9 and 57344 = 0.875 2^16, and products with a 24-bit scale are exact in
// 64 bits, so comparing mantissas gives the smallest power of two exactly.
template <int FMT>
__device__ __forceinline__ float raise_scale(float was, float amax, bool fresh) {
  const double base = fresh ? 1.0 : (double)was;
  int e, e0;
  const double m = frexp((double)amax, &e), m0 = frexp(base * Code<FMT>::kLargest, &e0);
  int k = amax == 0.0f ? -100000 : e - e0 + (m > m0 ? 1 : 0);
  const int low = fresh ? -100 : 0;
  k = k > low ? k : low;
  return (float)ldexp(base, k);
}

template <int FMT>
__device__ __forceinline__ uint32_t code_of(float x, float scale) {
  float y = x / scale;  // a power of two unless the caller's own scale is kept: then rounded
  const float big = Code<FMT>::kLargest;
  y = y > big ? big : (y < -big ? -big : y);  // NaN passes
  return Code<FMT>::two(y, 0.0f) & 0xFFu;
}

// A workgroup takes one block that gets tokens, one head, keys or values:
// the largest magnitude first, then the codes.  Keys are stored as they come,
// values transposed.
template <int DT, int FMT>
__global__ __launch_bounds__(kAppThreads) void k_cache_append(AppendArgs a) {
  const uint32_t bt = 1u << a.bt_log2, dim = a.c.head_dim;
  const int tid = threadIdx.x;
  const Places pl = {a.q_start, a.n_requests, 1u, bt, 2u};
  const uint32_t r = pl.find(blockIdx.x);
  const uint32_t h = blockIdx.y;
  const bool value = blockIdx.z != 0;
  int64_t q0 = a.q_start[r], q1 = a.q_start[r + 1];
  if (q1 > (int64_t)a.n_tokens) {
    if (tid == 0 && a.verdict) atomicOr(a.verdict, WM_C_SLOTS);
    q1 = a.n_tokens;
  }
  const int64_t nth = (int64_t)blockIdx.x - pl.first(r);
  if (q0 < 0 || nth < 0 || q0 >= q1) return;
  // the block's tokens: nth * bt - at .. of the request's, at being the place
  // of the first new token in its block
  const int64_t s0 = a.slots[q0];
  const int64_t at = s0 >= 0 ? (s0 & (bt - 1)) : 0;
  const int64_t begin = nth ? q0 + nth * bt - at : q0;
  if (begin >= q1) return;
  int64_t end = q0 + (nth + 1) * bt - at;
  end = end < q1 ? end : q1;
  const uint32_t off = nth ? 0u : (uint32_t)at, n_new = (uint32_t)(end - begin);
  const int64_t slot = a.slots[begin];
  if (slot < 0) return;
  const uint64_t page = (uint64_t)slot >> a.bt_log2;
  if (page >= a.c.n_blocks) {
    if (tid == 0 && a.verdict) atomicOr(a.verdict, WM_C_PAGE);
    return;
  }
  const bool fresh = off == 0;
  const wm_rows &src = value ? a.v : a.k;
  const uint64_t row0 = (uint64_t)begin * src.row_stride + (uint64_t)h * src.head_stride;
  const uint32_t n_elem = n_new * dim;
  float amax = 0.0f;
  for (uint32_t i = tid; i < n_elem; i += kAppThreads) {
    const float x = fabsf(load_elem<DT>(src.ptr, row0 + (uint64_t)(i / dim) * src.row_stride + i % dim));
    if (x <= 3.4028234e38f && x > amax) amax = x;
  }
  __shared__ float part[kAppThreads / 64];
  for (int i = 32; i; i >>= 1) amax = fmaxf(amax, __shfl_xor(amax, i));
  if ((tid & 63) == 0) part[tid >> 6] = amax;
  __syncthreads();
  for (int i = 0; i < kAppThreads / 64; ++i) amax = fmaxf(amax, part[i]);
  float *sp = (value ? a.c.v_scale + page * a.c.v_scale_stride
                     : a.c.k_scale + page * a.c.k_scale_stride) + h;
  const float was = *sp;
  const float now = raise_scale<FMT>(was, amax, fresh);
  __syncthreads();  // every thread has read the scale
  if (tid == 0 && now != was) *sp = now;
  uint8_t *codes = value ? (uint8_t *)a.c.v + page * a.c.v_stride : (uint8_t *)a.c.k + page * a.c.k_stride;
  codes += (uint64_t)h * bt * dim;
  const bool again = !fresh && now != was;
  const float ratio = again ? was / now : 1.0f;
  for (uint32_t i = tid; i < bt * dim; i += kAppThreads) {
    const uint32_t t = value ? i & (bt - 1) : i / dim;  // token of the block
    const uint32_t d = value ? i >> a.bt_log2 : i % dim;
    uint32_t b;
    if (t >= off && t < off + n_new) {
      b = code_of<FMT>(load_elem<DT>(src.ptr, row0 + (uint64_t)(t - off) * src.row_stride + d), now);
    } else if (fresh) {
      b = 0;
    } else if (again) {
      b = Code<FMT>::two(Code<FMT>::value(codes[i]) * ratio, 0.0f) & 0xFFu;
    } else {
      continue;
    }
    codes[i] = (uint8_t)b;
  }
}

// ---- attention: the parts of a split sequence joined ---------------------------

// A wave takes one query row: its parts' sums in one load (a lane each), then
// the weighted sum of the parts in their order.
template <int DT, int KD>
__global__ __launch_bounds__(kAttThreads) void k_attend_join(AttendArgs a) {
  const uint32_t hq_all = a.group * a.c.n_heads;
  const uint64_t at = (uint64_t)blockIdx.x * (kAttThreads / 64) + (threadIdx.x >> 6);
  const uint64_t token = at / hq_all;
  if (token >= a.n_tokens) return;
  const uint32_t hq = (uint32_t)(at - token * hq_all), h = hq / a.group;
  const Places pl = {a.q_start, a.n_requests, 1u, 1u, 0u};
  const uint32_t r = __builtin_amdgcn_readfirstlane(pl.find((int64_t)token));
  const Request x = request_of(a, r, false);
  if ((int64_t)token < x.q0) return;
  const uint64_t row = (token - (uint64_t)x.q0) * a.group + (hq - h * a.group);
  if (row >= x.n_rows) return;
  const uint32_t tile = (uint32_t)row / a.plan.rows;
  const Tile t = tile_of(a, x, tile);
  const uint32_t n = t.part1 - t.part0;
  if (n <= 1) return;
  const int lane = lane_id();
  const uint64_t p0 = part_place(a, x, r, tile, 0, h) + row % a.plan.rows;
  const uint64_t step = (uint64_t)a.c.n_heads * a.plan.rows;  // from a part to the next
  const float z = (uint32_t)lane < n ? a.part_lse[p0 + lane * step] : kNegInf;
  float top = z;
  for (int i = 32; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i));
  const float use = top == kNegInf ? 0.0f : top;
  const float weight = __builtin_amdgcn_exp2f(z - use);
  float sum = weight;
  for (int i = 32; i; i >>= 1) sum += __shfl_xor(sum, i);
  // eight parts in flight; a lane has KD neighbouring dimensions
  float o[KD];
#pragma unroll
  for (int j = 0; j < KD; ++j) o[j] = 0.0f;
  const float *p = a.part_out + p0 * (64 * KD) + lane * KD;
  for (uint32_t k0 = 0; k0 < n; k0 += 8) {
    float y[8][KD];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t kk = k0 + k < n ? k0 + k : n - 1;
#pragma unroll
      for (int j = 0; j < KD; ++j) y[k][j] = p[kk * step * (64 * KD) + j];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      // a weight of 0 behind the last part
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), k0 + k));
#pragma unroll
      for (int j = 0; j < KD; ++j) o[j] += f == 0.0f ? 0.0f : f * y[k][j];
    }
  }
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t *op = (uint16_t *)a.out.ptr + token * a.out.row_stride +
                 (uint64_t)hq * a.out.head_stride + lane * KD;
#pragma unroll
  for (int j = 0; j < KD; ++j) op[j] = (uint16_t)Qk<DT, WM_E4M3>::two(o[j] * inv, 0.0f);
  if (lane == 0 && a.lse)
    a.lse[token * hq_all + hq] =
        (sum == 0.0f ? kNegInf : use + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// ---- a session's blocks and the flat state -----------------------------------

__global__ void k_check_pages(const int32_t *pages, uint32_t n, uint64_t least, uint32_t *verdict) {
  bool bad = false;
  for (uint32_t i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x)
    bad |= pages[i] < 0 || (uint64_t)pages[i] >= least;
  if (bad) atomicOr(verdict, WM_C_PAGE);
}

constexpr int kPageThreads = 256;

// A workgroup copies pieces of up to 16 KiB of one page of one pool.
template <bool GATHER, typename T>
__global__ __launch_bounds__(kPageThreads) void k_pages(PoolBatch b, uint8_t *flat,
                                                        const int32_t *pages, uint32_t n_pages,
                                                        const uint32_t *verdict) {
  if (*verdict) return;
  for (uint64_t x = blockIdx.x; x < b.pieces; x += gridDim.x) {
    uint32_t lo = 0, hi = b.n;
    while (hi - lo > 1) {
      const uint32_t m = (lo + hi) / 2;
      if (b.p[m].first <= x)
        lo = m;
      else
        hi = m;
    }
    const uint64_t bytes = b.p[lo].page_bytes, per = (bytes + kPiece - 1) / kPiece;
    const uint64_t page = (x - b.p[lo].first) / per, at = (x - b.p[lo].first) % per * kPiece;
    const uint64_t n = bytes - at < kPiece ? bytes - at : kPiece;
    uint8_t *side = (uint8_t *)b.p[lo].ptr + (uint64_t)pages[page] * b.p[lo].stride + at;
    uint8_t *f = flat + b.p[lo].off + page * bytes + at;
    const T *src = (const T *)(GATHER ? side : f);
    T *dst = (T *)(GATHER ? f : side);
    for (uint64_t i = threadIdx.x; i < n / sizeof(T); i += kPageThreads) dst[i] = src[i];
    if (GATHER && page + 1 == n_pages && at + n == bytes) {  // the gap behind the pool's last page
      const uint64_t end = n_pages * bytes, gap = (16u - (end & 15u)) & 15u;
      if (threadIdx.x < gap) flat[b.p[lo].off + end + threadIdx.x] = 0;
    }
  }
}

int last_error() { return (int)hipGetLastError(); }

}  // namespace

int launch_page_tables(const TablesArgs &a, void *stream) {
  // a workgroup for each 4096 slots, at most two per CU
  uint64_t n = (a.slot_cap + 4095) / 4096;
  n = n < 1 ? 1 : (n > 512 ? 512 : n);
  k_page_tables<<<(uint32_t)n, kTabThreads, 0, reinterpret_cast<hipStream_t>(stream)>>>(a);
  return last_error();
}

int launch_cache_append(const AppendArgs &a, void *stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const uint32_t places = (a.n_tokens >> a.bt_log2) + 2u * a.n_requests;
  const dim3 grid(places, a.c.n_heads, 2);
  const bool e4 = a.c.format == WM_E4M3;
  if (a.k.dtype == WM_BF16 && e4)
    k_cache_append<WM_BF16, WM_E4M3><<<grid, kAppThreads, 0, st>>>(a);
  else if (a.k.dtype == WM_BF16)
    k_cache_append<WM_BF16, WM_E5M2><<<grid, kAppThreads, 0, st>>>(a);
  else if (e4)
    k_cache_append<WM_FP16, WM_E4M3><<<grid, kAppThreads, 0, st>>>(a);
  else
    k_cache_append<WM_FP16, WM_E5M2><<<grid, kAppThreads, 0, st>>>(a);
  return last_error();
}

int launch_cache_attend(const AttendArgs &a, void *stream) {
  const uint32_t d = a.c.head_dim;
  int e = d == 64    ? launch_attend_64(a, stream)
          : d == 128 ? launch_attend_128(a, stream)
          : d == 192 ? launch_attend_192(a, stream)
                     : launch_attend_256(a, stream);
  if (e || a.plan.splits <= 1) return e;
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const uint64_t waves = (uint64_t)a.n_tokens * a.group * a.c.n_heads;
  const uint32_t grid = (uint32_t)((waves + kAttThreads / 64 - 1) / (kAttThreads / 64));
  const bool bf = a.q.dtype == WM_BF16;
  switch (d / 64) {
#define WM_JOIN(kd)                                                      \
  case kd:                                                               \
    if (bf)                                                              \
      k_attend_join<WM_BF16, kd><<<grid, kAttThreads, 0, st>>>(a);       \
    else                                                                 \
      k_attend_join<WM_FP16, kd><<<grid, kAttThreads, 0, st>>>(a);       \
    break;
    WM_JOIN(1) WM_JOIN(2) WM_JOIN(3) WM_JOIN(4)
#undef WM_JOIN
  }
  return last_error();
}

int launch_check_pages(const int32_t *pages, uint32_t n_pages, uint64_t least_blocks,
                       uint32_t *verdict, void *stream) {
  const uint32_t n = (n_pages + 1023u) / 1024u;
  k_check_pages<<<n < 256u ? n : 256u, 256, 0, reinterpret_cast<hipStream_t>(stream)>>>(
      pages, n_pages, least_blocks, verdict);
  return last_error();
}

int launch_pages(bool gather, const PoolBatch &b, uint8_t *flat, const int32_t *pages,
                 uint32_t n_pages, uint64_t least_blocks, uint32_t *verdict, bool wide, int n_cu,
                 void *stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  (void)least_blocks;
  const uint64_t most = (uint64_t)n_cu * 8;
  const uint32_t grid = (uint32_t)(b.pieces < most ? b.pieces : most);
  if (gather && wide)
    k_pages<true, u32x4><<<grid, kPageThreads, 0, st>>>(b, flat, pages, n_pages, verdict);
  else if (gather)
    k_pages<true, uint32_t><<<grid, kPageThreads, 0, st>>>(b, flat, pages, n_pages, verdict);
  else if (wide)
    k_pages<false, u32x4><<<grid, kPageThreads, 0, st>>>(b, flat, pages, n_pages, verdict);
  else
    k_pages<false, uint32_t><<<grid, kPageThreads, 0, st>>>(b, flat, pages, n_pages, verdict);
  return last_error();
}

}  // namespace wm

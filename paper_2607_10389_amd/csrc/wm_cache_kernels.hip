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
// a table entry is read only where it was in use before.  256 or 2048 requests
// need one scan, more a first pass for the totals.
// What bounds it is the chain lengths - scan - search - ring - store: 3.8 us
// for a step of 64 requests; 10 to 11 us for 1500 requests with 1.08 M new
// tokens (8.7 MB of slots, 0.8 TB/s), of which an empty kernel takes about 3.  Shared
// arrays are written in 16-byte pieces and sums kept in 32 bits (saturating):
// both together took 4 of 15 us off that.
struct Step {
  int32_t o, n;   // lengths and
  uint32_t b, c;  // blocks before and after
  __device__ __forceinline__ uint32_t tokens() const { return n > o ? (uint32_t)(n - o) : 0u; }
  __device__ __forceinline__ uint32_t need() const { return c > b ? c - b : 0u; }
  __device__ __forceinline__ uint32_t give() const { return b > c ? b - c : 0u; }
  __device__ __forceinline__ bool bad(const TablesArgs &a) const {
    return o < 0 || n < 0 || b > a.max_blocks || c > a.max_blocks;
  }
};

__device__ __forceinline__ Step step_of(const TablesArgs &a, int32_t o, int32_t n) {
  const uint32_t round = (1u << a.bt_log2) - 1u;
  return Step{o, n, (uint32_t)(((uint64_t)(uint32_t)o + round) >> a.bt_log2),
              (uint32_t)(((uint64_t)(uint32_t)n + round) >> a.bt_log2)};
}

// Sums stop at 2^32 - 1: more than any pool or slot map holds.
__device__ __forceinline__ uint32_t add(uint32_t x, uint32_t y) {
  return __builtin_elementwise_add_sat(x, y);
}

// PER lengths from request r on; 0 behind the last request.
template <int PER>
__device__ __forceinline__ void load_lengths(const int32_t *p, uint32_t r, uint32_t n, bool wide,
                                             int32_t *x) {
  if (PER == 8 && wide && r + PER <= n) {
    const u32x4 u = *(const u32x4 *)(p + r), v = *(const u32x4 *)(p + r + 4);
#pragma unroll
    for (int i = 0; i < PER; ++i) x[i] = (int32_t)(i < 4 ? u[i & 3] : v[i & 3]);
    return;
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) x[i] = r + i < n ? p[r + i] : 0;
}

template <int PER>
__device__ __forceinline__ void store_entries(uint32_t *to, const uint32_t *x) {
  if (PER % 4) {
#pragma unroll
    for (int i = 0; i < PER; ++i) to[i] = x[i];
  } else {
#pragma unroll
    for (int i = 0; i < PER / 4; ++i)
      ((u32x4 *)to)[i] = u32x4{x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
  }
}

// A thread scans PER neighbouring requests by itself before the waves do.
constexpr int kTabThreads = 256;

// Neighbouring slots that a workgroup writes: eight a thread, one where there
// are few (a step's single tokens: latency).
__host__ __device__ __forceinline__ uint32_t slot_run(uint64_t slot_cap) {
  return slot_cap <= 8192 ? kTabThreads : 8 * kTabThreads;
}
template <int N>
struct Copies {
  static constexpr int value = N;
};

template <int PER>
__global__ __launch_bounds__(kTabThreads) void k_page_tables(TablesArgs a) {
  constexpr int NT = kTabThreads, kTile = NT * PER;
  __shared__ uint32_t sum[3][NT / 64];
  // lengths before and after, and what stands before a request; a thread's PER
  // entries are written in 16-byte pieces
  __shared__ __attribute__((aligned(16))) uint32_t st[2][kTile];
  __shared__ __attribute__((aligned(16))) uint32_t pre[3][kTile + 4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const uint32_t head = a.pool_in[0], count = a.pool_in[1];
  // tokens, blocks taken and blocks returned in all
  uint32_t total[3] = {0, 0, 0};
  auto decide = [&](bool bad) -> bool {
    uint32_t v = 0;
    if (total[1] > count || (uint64_t)count + total[2] > a.ring_cap || head >= a.ring_cap)
      v |= WM_C_POOL;
    if (total[0] > a.slot_cap) v |= WM_C_SLOTS;
    if (bad) v = WM_C_LENGTH;  // the other counts mean nothing then
    if (blockIdx.x == 0 && tid == 0) {
      *a.verdict = v;
      a.pool_out[0] = v ? head : (uint32_t)(((uint64_t)head + total[1]) % a.ring_cap);
      a.pool_out[1] = v ? count : count - total[1] + total[2];
      if (!v) a.q_start[a.n_requests] = (int32_t)total[0];
    }
    return v == 0;
  };
  const bool once = a.n_requests <= kTile;
  if (!once) {
    uint32_t x[3] = {0, 0, 0};
    bool bad = false;
    for (uint32_t r = tid; r < a.n_requests; r += NT) {
      const Step s = step_of(a, a.old_len[r], a.new_len[r]);
      bad |= s.bad(a);
      x[0] = add(x[0], s.tokens());
      x[1] = add(x[1], s.need());
      x[2] = add(x[2], s.give());
    }
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      for (int i = 32; i; i >>= 1) x[k] = add(x[k], __shfl_xor(x[k], i));
      if (lane == 0) sum[k][wave] = x[k];
    }
    bad = __syncthreads_or(bad);
    for (int k = 0; k < 3; ++k)
      for (int i = 0; i < NT / 64; ++i) total[k] = add(total[k], sum[k][i]);
    if (!decide(bad)) return;
  }
  const uint64_t step = (uint64_t)gridDim.x * NT;
  const uint64_t at = (uint64_t)blockIdx.x * NT + tid;
  const uint32_t bt = 1u << a.bt_log2;
  // a place of the ring: less than two rounds
  auto place = [&](uint64_t x) { return (uint32_t)(x >= a.ring_cap ? x - a.ring_cap : x); };
  const bool wide = (((uintptr_t)a.old_len | (uintptr_t)a.new_len) & 15u) == 0;
  uint32_t base[3] = {0, 0, 0};
  for (uint32_t r0 = 0; r0 < a.n_requests || (once && r0 == 0); r0 += kTile) {
    __syncthreads();  // the tile before is done with the shared arrays
    Step s[PER];
    int32_t o[PER], n[PER];
    load_lengths<PER>(a.old_len, r0 + PER * tid, a.n_requests, wide, o);
    load_lengths<PER>(a.new_len, r0 + PER * tid, a.n_requests, wide, n);
    uint32_t x[3] = {0, 0, 0};
    bool bad = false;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      s[i] = step_of(a, o[i], n[i]);
      bad |= s[i].bad(a);
      x[0] = add(x[0], s[i].tokens());
      x[1] = add(x[1], s[i].need());
      x[2] = add(x[2], s[i].give());
    }
    store_entries<PER>(&st[0][PER * tid], (const uint32_t *)o);
    store_entries<PER>(&st[1][PER * tid], (const uint32_t *)n);
    const uint32_t own[3] = {x[0], x[1], x[2]};
    for (int i = 1; i < 64; i <<= 1)
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const uint32_t y = __shfl_up(x[k], i);
        x[k] = lane >= i ? add(x[k], y) : x[k];
      }
    if (lane == 63)
#pragma unroll
      for (int k = 0; k < 3; ++k) sum[k][wave] = x[k];
    bad = __syncthreads_or(bad);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      uint32_t before = base[k], all = base[k];
#pragma unroll
      for (int i = 0; i < NT / 64; ++i) {
        if (i < wave) before = add(before, sum[k][i]);
        all = add(all, sum[k][i]);
      }
      // (exact once decide() has passed)
      uint32_t p = before + x[k] - own[k], e[PER];
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        e[i] = p;
        p += k == 0 ? s[i].tokens() : (k == 1 ? s[i].need() : s[i].give());
      }
      store_entries<PER>(&pre[k][PER * tid], e);
      if (tid == NT - 1) pre[k][kTile] = p;
      if (once) total[k] = all;
      base[k] = all;
    }
    if (once && !decide(bad)) return;
    __syncthreads();
    if (blockIdx.x == 0)
      for (uint32_t i = tid; i < kTile && r0 + i < a.n_requests; i += NT)
        a.q_start[r0 + i] = (int32_t)pre[0][i];
    // blocks of a length (as in step_of)
    auto blocks_of = [&](uint32_t n) { return (n + (bt - 1u)) >> a.bt_log2; };
    auto owner = [&](int k, uint32_t j) {  // the last request whose part begins at or before j
      int lo = 0;
#pragma unroll
      for (int m = kTile / 2; m; m >>= 1)
        if (pre[k][lo + m] <= j) lo += m;
      return lo;
    };
    for (uint64_t j = pre[1][0] + at; j < pre[1][kTile]; j += step) {
      const int i = owner(1, (uint32_t)j);
      a.table[(uint64_t)(r0 + i) * a.table_stride + blocks_of(st[0][i]) +
              ((uint32_t)j - pre[1][i])] =
          a.ring[place(head + j)];
    }
    for (uint64_t j = pre[2][0] + at; j < pre[2][kTile]; j += step) {
      const int i = owner(2, (uint32_t)j);
      a.ring[place((uint64_t)place((uint64_t)head + count) + j)] =
          a.table[(uint64_t)(r0 + i) * a.table_stride + blocks_of(st[1][i]) +
                  ((uint32_t)j - pre[2][i])];
    }
    // the same for the wave: 64 candidates at a time
    auto owner_of = [&](uint32_t j) {
      constexpr int kStride = kTile / 64;
      const int c = __popcll(__ballot(pre[0][lane * kStride] <= j)) - 1;
      const bool le = lane < kStride && pre[0][c * kStride + lane % kStride] <= j;
      return c * kStride + __popcll(__ballot(le)) - 1;
    };
    // a run of neighbouring slots belongs to few of many requests: a slot's
    // is searched among those
    const uint32_t slots1 = pre[0][kTile], n_run = slot_run(a.slot_cap);
    for (uint64_t run = pre[0][0] + (uint64_t)blockIdx.x * n_run; run < slots1;
         run += (uint64_t)gridDim.x * n_run) {
      const uint32_t j0 = (uint32_t)run;
      const uint32_t j1 = slots1 - j0 < n_run ? slots1 - 1 : j0 + n_run - 1;
      int lo = 0, hi = kTile - 1, half = kTile / 2;
      if (PER > 1) {
        lo = owner_of(j0);
        hi = owner_of(j1);
        half = hi > lo ? 1 << (31 - __clz(hi - lo)) : 0;
      }
      auto write = [&](auto copies) {  // so many slots a thread, side by side
        constexpr int N = decltype(copies)::value;
        uint32_t j[N], p[N];
        int l[N];
        int32_t id[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          j[i] = j0 + i * NT + tid < j1 ? j0 + i * NT + tid : j1;
          l[i] = lo;
        }
        for (int m = half; m; m >>= 1)
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (l[i] + m <= hi && pre[0][l[i] + m] <= j[i]) l[i] += m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t o = st[0][l[i]], b = blocks_of(o);
          p[i] = o + (j[i] - pre[0][l[i]]);
          const uint32_t blk = p[i] >> a.bt_log2;
          id[i] = *(blk < b ? a.table + (uint64_t)(r0 + l[i]) * a.table_stride + blk
                            : a.ring + place((uint64_t)head + pre[1][l[i]] + (blk - b)));
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (j0 + i * NT + tid <= j1) a.slots[j[i]] = (int64_t)id[i] * bt + (p[i] & (bt - 1u));
      };
      if (j1 - j0 < NT)
        write(Copies<1>{});
      else
        write(Copies<8>{});
    }
  }
}

// ---- store new keys and values -----------------------------------------------

constexpr int kAppThreads = 256;
constexpr uint32_t kPlacesY = 32768;  // a grid's second axis

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

// Four codes; inv: 1 / scale, a power of two, so that the product is exact.
template <int FMT>
__device__ __forceinline__ uint32_t codes_of(const float *x, float inv) {
  const float big = Code<FMT>::kLargest;
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = x[i] * inv;
    y[i] = y[i] > big ? big : (y[i] < -big ? -big : y[i]);  // NaN passes
  }
  return Code<FMT>::two(y[0], y[1]) | Code<FMT>::two(y[2], y[3]) << 16;
}

// Four codes whose scale was raised by 1 / ratio, a power of two.
template <int FMT>
__device__ __forceinline__ uint32_t moved_codes(uint32_t w, float ratio) {
  float y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = Code<FMT>::value(w >> (8 * i) & 0xFFu) * ratio;
  return Code<FMT>::two(y[0], y[1]) | Code<FMT>::two(y[2], y[3]) << 16;
}

template <int DT>
__device__ __forceinline__ float element(uint16_t h) {
  return DT == WM_BF16 ? __uint_as_float((uint32_t)h << 16)
                       : (float)__builtin_bit_cast(_Float16, h);
}

// Eight neighbouring elements of a row.
template <int DT, bool WIDE>
__device__ __forceinline__ void load_eight(const void *p, uint64_t at, float *x) {
  const uint16_t *e = static_cast<const uint16_t *>(p) + at;
  u32x4 w;
  if (WIDE) {
    w = *(const u32x4 *)e;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (uint32_t)e[2 * i] | (uint32_t)e[2 * i + 1] << 16;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t h = w[i >> 1] >> (16 * (i & 1)) & 0xFFFFu;
    x[i] = element<DT>((uint16_t)h);
  }
}

// A block that gets tokens, a head, keys or values: the largest magnitude
// first, then the codes, from the same 16-byte loads (the second time from
// L2).  NT threads work on it: a workgroup where blocks get many tokens, a wave
// where they get a few (a step's single tokens: no barrier, and four times as
// many blocks on their way).  Keys are stored as they come.  Values are
// transposed in registers: a thread takes four tokens of eight dimensions and
// stores eight words of four tokens, its neighbours the next four tokens, so
// that 16 threads read 64 bytes of a row and write 64 bytes of one.
// What bounds it: HBM for prompts (24 of them into 16 heads of 128: 227 MB in
// 59 us, 3.9 TB/s, where a plain copy reaches 4.8); for single tokens a chain
// of four loads (starts, slot, row and scale, codes): 64 of them in 7.2 us.
// (Pieces of 16 tokens held in registers from the first pass to the second
// took 83 us and 160 us: too few threads with a load under way.)
template <int DT, int FMT, int NT, bool WIDE>
__global__ __launch_bounds__(kAppThreads) void k_cache_append(AppendArgs a) {
  __shared__ float part[kAppThreads / 64];
  const uint32_t bt = 1u << a.bt_log2, dim = a.c.head_dim, d8 = dim / 8;
  const uint32_t tid = NT == 64 ? (uint32_t)lane_id() : threadIdx.x;
  // neighbouring workgroups take neighbouring heads: of a token's row they
  // read one stretch
  const uint32_t unit = blockIdx.z * kPlacesY + blockIdx.y;
  const uint32_t place = __builtin_amdgcn_readfirstlane(
      NT == 64 ? unit * (kAppThreads / 64) + (threadIdx.x >> 6) : unit);
  const Places pl = {a.q_start, a.n_requests, 1u, bt, 2u};
  const uint32_t r = __builtin_amdgcn_readfirstlane(pl.find(place));
  const bool value = blockIdx.x >= a.c.n_heads;
  const uint32_t h = blockIdx.x - (value ? a.c.n_heads : 0u);
  int64_t q0 = a.q_start[r], q1 = a.q_start[r + 1];
  if (q1 > (int64_t)a.n_tokens) {
    if (tid == 0 && a.verdict) atomicOr(a.verdict, WM_C_SLOTS);
    q1 = a.n_tokens;
  }
  const int64_t nth = (int64_t)place - pl.first(r);
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
  const int64_t slot = nth ? a.slots[begin] : s0, last = a.slots[end - 1];
  if (slot < 0) return;
  const uint64_t page = (uint64_t)slot >> a.bt_log2;
  // (a later block begins at its first place)
  if (page >= a.c.n_blocks || (nth && (slot & (bt - 1)))) {
    if (tid == 0 && a.verdict) atomicOr(a.verdict, WM_C_PAGE);
    return;
  }
  const wm_rows &src = value ? a.v : a.k;
  const uint64_t row0 = (uint64_t)begin * src.row_stride + (uint64_t)h * src.head_stride;
  float *sp = (value ? a.c.v_scale + page * a.c.v_scale_stride
                     : a.c.k_scale + page * a.c.k_scale_stride) + h;
  const float was = *sp;
  const bool fresh = off == 0 || !(was >= 0x1p-126f && was <= 3.4028234e38f);
  float amax = 0.0f;
  // (several loads under way: one more of the last piece changes nothing)
  constexpr int U = NT == 64 ? 1 : 4;
  for (uint32_t i0 = tid; i0 < n_new * d8; i0 += U * NT) {
    float x[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = i0 + u * NT < n_new * d8 ? i0 + u * NT : n_new * d8 - 1;
      load_eight<DT, WIDE>(src.ptr, row0 + (uint64_t)(i / d8) * src.row_stride + i % d8 * 8, x[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = fabsf(x[u][j]);
        if (y <= 3.4028234e38f && y > amax) amax = y;
      }
  }
  for (int i = 32; i; i >>= 1) amax = fmaxf(amax, __shfl_xor(amax, i));
  if (NT > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = amax;
    __syncthreads();  // (and every thread has read the scale)
    for (int i = 0; i < kAppThreads / 64; ++i) amax = fmaxf(amax, part[i]);
  }
  // The last token stands where slots that follow each other put it?  (Asked
  // here, its slot has come while the rows did.)
  if ((uint64_t)last - (uint64_t)slot != n_new - 1u) {
    if (tid == 0 && a.verdict) atomicOr(a.verdict, WM_C_PAGE);
    return;
  }
  const float now = raise_scale<FMT>(was, amax, fresh);
  if (tid == 0 && now != was) *sp = now;
  const bool again = !fresh && now != was;
  const float ratio = again ? was / now : 1.0f;
  const uint64_t base = (uint64_t)h * bt * dim;
  if ((__float_as_uint(now) & 0x7FFFFFu) != 0) {
    // the caller's own scale, no power of two: true quotients, a byte at a time
    uint8_t *codes = (value ? (uint8_t *)a.c.v + page * a.c.v_stride
                            : (uint8_t *)a.c.k + page * a.c.k_stride) + base;
#pragma unroll 1
    for (uint32_t i = tid; i < bt * dim; i += NT) {
      const uint32_t t = value ? i & (bt - 1) : i / dim, d = value ? i >> a.bt_log2 : i % dim;
      const uint16_t *e =
          (const uint16_t *)src.ptr + row0 + (uint64_t)(t - off) * src.row_stride + d;
      if (t >= off && t < off + n_new) {
        float y = element<DT>(*e) / now;
        const float big = Code<FMT>::kLargest;
        y = y > big ? big : (y < -big ? -big : y);
        codes[i] = (uint8_t)Code<FMT>::two(y, 0.0f);
      } else if (again) {
        codes[i] = (uint8_t)Code<FMT>::two(Code<FMT>::value(codes[i]) * ratio, 0.0f);
      }
    }
    return;
  }
  const float inv = 1.0f / now;
  if (!value) {
    uint8_t *codes = (uint8_t *)a.c.k + page * a.c.k_stride + base;
    // only the new rows, unless all of the block's change
    const bool all = fresh || again;
    const uint32_t t0 = all ? 0u : off, t1 = all ? bt : off + n_new;
    for (uint32_t i0 = t0 * d8 + tid; i0 < t1 * d8; i0 += U * NT) {
      float x[U][8];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (a place that gets no token takes one of those that do, unused)
        const uint32_t i = i0 + u * NT;
        uint32_t t = i / d8;
        t = t < off ? 0u : (t < off + n_new ? t - off : n_new - 1);
        load_eight<DT, WIDE>(src.ptr, row0 + (uint64_t)t * src.row_stride + i % d8 * 8, x[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint32_t i = i0 + u * NT, t = i / d8;
        if (i >= t1 * d8) break;
        u32x2 *to = (u32x2 *)(codes + (uint64_t)i * 8);
        u32x2 w = {0, 0};
        if (t >= off && t < off + n_new) {
          w = u32x2{codes_of<FMT>(x[u], inv), codes_of<FMT>(x[u] + 4, inv)};
        } else if (again) {
          const u32x2 y = *to;
          w = u32x2{moved_codes<FMT>(y[0], ratio), moved_codes<FMT>(y[1], ratio)};
        }
        *to = w;
      }
    }
    return;
  }
  uint8_t *codes = (uint8_t *)a.c.v + page * a.c.v_stride + base;
  const bool all = fresh || again;
  // groups of four tokens
  const uint32_t g0 = all ? 0u : off / 4, g1 = all ? bt / 4 : (off + n_new + 3) / 4;
  const uint32_t ng = g1 - g0;
  for (uint32_t i = tid; i < ng * d8; i += NT) {
    const uint32_t t = (g0 + i % ng) * 4, d = i / ng * 8;
    uint32_t *to = (uint32_t *)(codes + (uint64_t)d * bt + t);
    uint32_t w[8], mine = 0;  // mine: bytes of the words that are new tokens
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (t + j >= off && t + j < off + n_new) mine |= 0xFFu << (8 * j);
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = 0;
    if (!fresh && mine != ~0u) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        w[j] = to[(uint64_t)j * (bt / 4)];
        if (again) w[j] = moved_codes<FMT>(w[j], ratio);
      }
    }
    if (mine) {
      uint32_t c[4][2];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        // a place that gets no token takes its codes from one that does; they
        // are not used
        uint32_t tok = t + j < off ? off : t + j;
        tok = tok < off + n_new ? tok - off : n_new - 1;
        float x[8];
        load_eight<DT, WIDE>(src.ptr, row0 + (uint64_t)tok * src.row_stride + d, x);
        c[j][0] = codes_of<FMT>(x, inv);
        c[j][1] = codes_of<FMT>(x + 4, inv);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int k = j >> 2, sel = j & 3;
        // byte sel of four words into one
        const uint32_t lo = __builtin_amdgcn_perm(c[1][k], c[0][k], 0x0C0C0400u + 0x0101u * sel);
        const uint32_t hi = __builtin_amdgcn_perm(c[3][k], c[2][k], 0x0C0C0400u + 0x0101u * sel);
        w[j] = (w[j] & ~mine) | ((lo | hi << 16) & mine);
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) to[(uint64_t)j * (bt / 4)] = w[j];
  }
}

// ---- attention: the parts of a split sequence joined ---------------------------

// A wave takes one query row: its parts' sums in one load (a lane each), then
// the weighted sum of the parts in their order.  Eight parts are loaded at
// once, or the chain of loads would bound it: 4.7 us for 128 rows of 15 parts,
// 9.9 us for 2048 rows of 16 to 31.
template <int DT, int KD>
__global__ __launch_bounds__(kAttThreads) void k_attend_join(AttendArgs a) {
  const uint32_t hq_all = a.group * a.c.n_heads;
  const uint64_t unit = (uint64_t)blockIdx.y * gridDim.x + blockIdx.x;
  const uint64_t at = unit * (kAttThreads / 64) + (threadIdx.x >> 6);
  const uint64_t token = at / hq_all;
  if (token >= a.n_tokens) return;
  const uint32_t hq = (uint32_t)(at - token * hq_all);
  const Places pl = {a.q_start, a.n_requests, 1u, 1u, 0u};
  const uint32_t r = __builtin_amdgcn_readfirstlane(pl.find((int64_t)token));
  const Request x = request_of(a, r, false);
  if ((int64_t)token < x.q0) return;
  const uint64_t row = (token - (uint64_t)x.q0) * a.group + hq % a.group;
  if (row >= x.n_rows) return;
  const uint32_t tile = (uint32_t)row / a.plan.rows;
  const Tile t = tile_of(a, x, tile);
  const uint32_t n = t.part1 - t.part0;
  if (n <= 1) return;
  const int lane = lane_id();
  const uint64_t p0 = part_place(a, token, hq);
  const float z = (uint32_t)lane < n ? a.part_lse[p0 + lane] : kNegInf;
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
      for (int j = 0; j < KD; ++j) y[k][j] = p[(uint64_t)kk * (64 * KD) + j];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      // (behind the last part it comes again, with a weight of 0)
      const float f = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), k0 + k));
#pragma unroll
      for (int j = 0; j < KD; ++j) o[j] += weighed(f, y[k][j]);
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

// A workgroup copies pieces of up to 16 KiB of one page of one pool.  HBM bounds
// it: 1.67 GB of 28 layers in 319 us (read and written, 5.2 TB/s); 37.8 MB in
// 7.2 us, with a part of it in the caches.
template <bool GATHER, typename T>
__global__ __launch_bounds__(kPageThreads) void k_pages(PoolBatch b, uint8_t *flat,
                                                        const int32_t *pages, uint32_t n_pages,
                                                        uint64_t least, uint32_t *verdict) {
  if (n_pages <= kPagesLooked) {
    // every workgroup looks at the whole list, so that none writes if one
    // block is bad
    bool bad = false;
    for (uint32_t i = threadIdx.x; i < n_pages; i += kPageThreads)
      bad |= pages[i] < 0 || (uint64_t)pages[i] >= least;
    if (__syncthreads_or(bad)) {
      if (threadIdx.x == 0) atomicOr(verdict, WM_C_PAGE);
      return;
    }
  }
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
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  // a workgroup for each run of slots, at most as many as 256 CUs hold at once
  // (40 KiB of LDS each); one scan for up to 256 or 2048 requests
  const uint64_t per = slot_run(a.slot_cap);
  uint64_t n = (a.slot_cap + per - 1) / per;
  n = n < 1 ? 1 : (n > 768 ? 768 : n);
  if (a.n_requests <= 256)
    k_page_tables<1><<<(uint32_t)n, kTabThreads, 0, st>>>(a);
  else
    k_page_tables<8><<<(uint32_t)n, kTabThreads, 0, st>>>(a);
  return last_error();
}

namespace {

template <int DT, int FMT>
int append_types(const AppendArgs &a, hipStream_t st) {
  const uint32_t places = (a.n_tokens >> a.bt_log2) + 2u * a.n_requests;
  // a wave for a block's few tokens: up to eight a request on average
  const bool few = a.n_tokens <= 8ull * a.n_requests;
  const bool wide = (((uintptr_t)a.k.ptr >> 1 | (uintptr_t)a.v.ptr >> 1 | a.k.row_stride |
                      a.k.head_stride | a.v.row_stride | a.v.head_stride) & 7u) == 0;
  const uint32_t units = few ? (places + 3) / 4 : places;
  const dim3 grid(2 * a.c.n_heads, units < kPlacesY ? units : kPlacesY,
                  (units + kPlacesY - 1) / kPlacesY);
  if (few && wide)
    k_cache_append<DT, FMT, 64, true><<<grid, kAppThreads, 0, st>>>(a);
  else if (few)
    k_cache_append<DT, FMT, 64, false><<<grid, kAppThreads, 0, st>>>(a);
  else if (wide)
    k_cache_append<DT, FMT, kAppThreads, true><<<grid, kAppThreads, 0, st>>>(a);
  else
    k_cache_append<DT, FMT, kAppThreads, false><<<grid, kAppThreads, 0, st>>>(a);
  return last_error();
}

}  // namespace

int launch_cache_append(const AppendArgs &a, void *stream) {
  hipStream_t st = reinterpret_cast<hipStream_t>(stream);
  const bool e4 = a.c.format == WM_E4M3;
  if (a.k.dtype == WM_BF16)
    return e4 ? append_types<WM_BF16, WM_E4M3>(a, st) : append_types<WM_BF16, WM_E5M2>(a, st);
  return e4 ? append_types<WM_FP16, WM_E4M3>(a, st) : append_types<WM_FP16, WM_E5M2>(a, st);
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
  const uint32_t units = (uint32_t)((waves + kAttThreads / 64 - 1) / (kAttThreads / 64));
  const dim3 grid(grid_x(units), grid_y(units));
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
  const uint64_t most = (uint64_t)n_cu * 8;
  const uint32_t grid = (uint32_t)(b.pieces < most ? b.pieces : most);
  const auto kernel = gather ? (wide ? k_pages<true, u32x4> : k_pages<true, uint32_t>)
                             : (wide ? k_pages<false, u32x4> : k_pages<false, uint32_t>);
  kernel<<<grid, kPageThreads, 0, st>>>(b, flat, pages, n_pages, least_blocks, verdict);
  return last_error();
}

}  // namespace wm

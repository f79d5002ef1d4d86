// wm_cache_api.cpp -- the C ABI of the paged 8-bit cache (include/wm_cache.h).
//
// Host side only: argument checks (before anything is enqueued), the split of
// an attention call and the launches.  Nothing is allocated or kept.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>

#include "wm_cache_internal.h"

using namespace wm;

namespace {

bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

wm_status hip_status(int e) { return e == 0 ? WM_OK : WM_ERR_HIP; }

bool log2_of(uint32_t block_tokens, uint32_t *l) {
  for (uint32_t i = 4; i <= 8; ++i)
    if (block_tokens == 1u << i) {
      *l = i;
      return true;
    }
  return false;
}

wm_status check_cache(const wm_cache *c, uint32_t *bt_log2) {
  if (!c || c->flags || !c->n_blocks || c->n_blocks > 0x7FFFFFFFu || !c->n_heads ||
      c->n_heads > 65535u || (c->format != WM_E4M3 && c->format != WM_E5M2))
    return WM_ERR_INVALID_ARG;
  if (!log2_of(c->block_tokens, bt_log2)) return WM_ERR_UNSUPPORTED;
  const uint32_t d = c->head_dim;
  if (d != 64 && d != 128 && d != 192 && d != 256) return WM_ERR_UNSUPPORTED;
  const uint64_t page = (uint64_t)c->n_heads * c->block_tokens * d;
  if (!c->k || !c->v || !c->k_scale || !c->v_scale || !aligned(c->k, 16) || !aligned(c->v, 16) ||
      !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4))
    return WM_ERR_INVALID_ARG;
  if (c->k_stride < page || c->v_stride < page || (c->k_stride & 15u) || (c->v_stride & 15u) ||
      c->k_scale_stride < c->n_heads || c->v_scale_stride < c->n_heads)
    return WM_ERR_INVALID_ARG;
  return WM_OK;
}

bool check_rows(const wm_rows *r) {
  return r && !r->flags && (r->dtype == WM_BF16 || r->dtype == WM_FP16) && aligned(r->ptr, 2);
}

// CUs of the current device (0: none); asked of the runtime once per device.
int cus() {
  static std::atomic<int> known[64];
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0) return 0;
  if (dev < 64 && (n = known[dev].load(std::memory_order_relaxed)) != 0) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess)
    return 0;
  if (dev < 64) known[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Offsets of the pools in the flat state and its size; false for a table
// that is not valid.
bool pool_layout(const wm_pool *p, uint32_t n, uint32_t n_pages, uint64_t *total) {
  *total = 0;
  if (n && !p) return false;
  for (uint32_t i = 0; i < n; ++i) {
    if (n_pages && p[i].page_bytes > (1ull << 62) / n_pages) return false;
    *total += (p[i].page_bytes * n_pages + 15u) & ~15ull;
    if (*total > (1ull << 62)) return false;
  }
  return true;
}

wm_status pages_call(bool gather, const wm_pool *pools, uint32_t n_pools, const int32_t *pages,
                     uint32_t n_pages, uint8_t *flat, uint64_t flat_cap, uint32_t *verdict,
                     void *stream) {
  uint64_t total = 0, least = ~0ull;
  if (n_pools > WM_MAX_POOLS || !verdict || !aligned(verdict, 4) ||
      !pool_layout(pools, n_pools, n_pages, &total))
    return WM_ERR_INVALID_ARG;
  for (uint32_t i = 0; i < n_pools; ++i) {
    const wm_pool &p = pools[i];
    if (!p.page_bytes || (p.page_bytes & 3u) || (p.stride & 3u) || p.stride < p.page_bytes ||
        !p.n_blocks || p.n_blocks > 0x7FFFFFFFull || !p.ptr || !aligned(p.ptr, 4))
      return WM_ERR_INVALID_ARG;
    least = std::min(least, p.n_blocks);
  }
  if (total && (!flat || !aligned(flat, 16) || !pages || !aligned(pages, 4)))
    return WM_ERR_INVALID_ARG;
  if (flat_cap < total) return WM_ERR_CAPACITY;
  if (!total) return WM_OK;
  const int n_cu = cus();
  if (!n_cu) return WM_ERR_HIP;
  if (n_pages > kPagesLooked && launch_check_pages(pages, n_pages, least, verdict, stream) != 0)
    return WM_ERR_HIP;
  uint64_t off = 0;
  for (uint32_t i = 0; i < n_pools;) {
    PoolBatch b;
    std::memset(&b, 0, sizeof(b));
    bool wide = true;
    for (; i < n_pools && b.n < kPoolsPerLaunch; ++i, ++b.n) {
      const wm_pool &p = pools[i];
      auto &o = b.p[b.n];
      o.ptr = reinterpret_cast<uint64_t>(p.ptr);
      o.stride = p.stride;
      o.off = off;
      o.page_bytes = p.page_bytes;
      o.n_blocks = p.n_blocks;
      o.first = b.pieces;
      b.pieces += (uint64_t)n_pages * ((p.page_bytes + kPiece - 1) / kPiece);
      off += (p.page_bytes * n_pages + 15u) & ~15ull;
      wide = wide && ((o.ptr | p.stride | p.page_bytes) & 15u) == 0;
    }
    if (launch_pages(gather, b, flat, pages, n_pages, least, verdict, wide, n_cu, stream) != 0)
      return WM_ERR_HIP;
  }
  return WM_OK;
}

}  // namespace

namespace wm {

AttendPlan attend_plan(uint32_t n_requests, uint32_t n_tokens, uint32_t n_heads,
                       uint32_t n_q_heads, uint32_t head_dim, uint32_t max_len) {
  AttendPlan p = {16, 1, 1, 9};
  if (!n_requests || !n_tokens || !n_heads || n_q_heads < n_heads) return p;
  const uint64_t rows = (uint64_t)n_tokens * (n_q_heads / n_heads), each = rows / n_requests;
  const uint64_t len = std::max<uint64_t>(1, max_len);
  // The mean of the rows per request decides, requests without rows counted:
  // lengths of rows are known on the device alone.  (So a prompt beside many
  // single tokens, or among many empty places, takes the others' kernel.)
  // Tiles of 128 rows read the cache once for all of a request's rows and keep
  // the matrix cores busier; small tiles spread it over the CUs in parts.  With
  // 64 rows per request and head 64 requests of 4112 tokens, 8 heads of 128,
  // take 237 us in the first and 395 in the second, but 8 of them 74 and 56: up
  // to 64 rows, where the large tiles would leave half of 256 CUs idle, the
  // second is the faster one (with 128 rows it is not: 73 against 79 us).
  const uint64_t busy = std::max<uint64_t>(rows / 128, n_requests) * n_heads;
  if (each > 64 || (each > 32 && busy > 128))
    p.rows = 128;
  else if (each > 16 && head_dim <= 64)
    p.rows = 32;  // (larger heads: two tiles of 16 read twice, but 617 -> 428 us at 256
                  // dimensions, 220 -> 209 at 128; at 64 it is 103 -> 113)
  p.tiles = (uint32_t)(rows / p.rows + n_requests);
  if (p.rows > 32) {
    // a sequence is cut only where its tiles leave more than half of 256 CUs idle
    const uint64_t want = std::max<uint64_t>(1, std::min<uint64_t>(256 / busy, 31));
    while (((len - 1) >> p.cut) + 1 > want) ++p.cut;
  }
  // parts of 512 tokens, or of more so that there are at most 32
  p.splits = (uint32_t)std::min<uint64_t>(32, ((len - 1) >> p.cut) + 1);
  return p;
}

}  // namespace wm

extern "C" {

wm_status wm_page_tables(const int32_t *old_len, const int32_t *new_len, uint32_t n_requests,
                         uint32_t block_tokens, int32_t *block_table, uint64_t table_stride,
                         uint32_t max_blocks, int32_t *free_ring, uint32_t ring_cap,
                         const uint32_t *pool_in, uint32_t *pool_out, int64_t *slot_map,
                         uint64_t slot_cap, int32_t *q_start, uint32_t *verdict, void *stream) {
  TablesArgs a;
  if (!log2_of(block_tokens, &a.bt_log2)) return WM_ERR_UNSUPPORTED;
  if (!pool_in || !pool_out || pool_in == pool_out || !q_start || !verdict || !free_ring ||
      !ring_cap || ring_cap > 0x7FFFFFFFu)
    return WM_ERR_INVALID_ARG;
  if (n_requests && (!old_len || !new_len || !block_table)) return WM_ERR_INVALID_ARG;
  if (n_requests > 0x7FFFFFFFu || table_stride < max_blocks ||
      (uint64_t)max_blocks * block_tokens > 0x7FFFFFFFull || slot_cap > 0x7FFFFFFFull)
    return WM_ERR_INVALID_ARG;
  if (slot_cap && !slot_map) return WM_ERR_INVALID_ARG;
  if (!aligned(old_len, 4) || !aligned(new_len, 4) || !aligned(block_table, 4) ||
      !aligned(free_ring, 4) || !aligned(pool_in, 4) || !aligned(pool_out, 4) ||
      !aligned(slot_map, 8) || !aligned(q_start, 4) || !aligned(verdict, 4))
    return WM_ERR_INVALID_ARG;
  a.old_len = old_len;
  a.new_len = new_len;
  a.table = block_table;
  a.table_stride = table_stride;
  a.ring = free_ring;
  a.pool_in = pool_in;
  a.pool_out = pool_out;
  a.slots = slot_map;
  a.slot_cap = slot_cap;
  a.q_start = q_start;
  a.verdict = verdict;
  a.n_requests = n_requests;
  a.max_blocks = max_blocks;
  a.ring_cap = ring_cap;
  return hip_status(launch_page_tables(a, stream));
}

wm_status wm_cache_append(const wm_cache *cache, const wm_rows *k, const wm_rows *v,
                          const int64_t *slot_map, const int32_t *q_start, uint32_t n_requests,
                          uint32_t n_tokens, uint32_t *verdict, void *stream) {
  AppendArgs a;
  const wm_status s = check_cache(cache, &a.bt_log2);
  if (s != WM_OK) return s;
  if (!check_rows(k) || !check_rows(v) || k->dtype != v->dtype || !aligned(verdict, 4))
    return WM_ERR_INVALID_ARG;
  if (n_requests > 0x3FFFFFFFu || n_tokens > 0x7FFFFFFFu) return WM_ERR_INVALID_ARG;
  if (!n_requests || !n_tokens) return WM_OK;
  if (!k->ptr || !v->ptr || !slot_map || !q_start || !aligned(slot_map, 8) || !aligned(q_start, 4))
    return WM_ERR_INVALID_ARG;
  a.c = *cache;
  a.k = *k;
  a.v = *v;
  a.slots = slot_map;
  a.q_start = q_start;
  a.verdict = verdict;
  a.n_requests = n_requests;
  a.n_tokens = n_tokens;
  return hip_status(launch_cache_append(a, stream));
}

uint64_t wm_attend_ws_bytes(uint32_t n_requests, uint32_t n_tokens, uint32_t n_heads,
                            uint32_t n_q_heads, uint32_t head_dim, uint32_t max_len) {
  const AttendPlan p = attend_plan(n_requests, n_tokens, n_heads, n_q_heads, head_dim, max_len);
  if (p.splits <= 1) return 0;
  return (uint64_t)n_tokens * n_q_heads * p.splits * (head_dim + 1u) * 4u;
}

wm_status wm_cache_attend(const wm_cache *cache, const wm_rows *q, const wm_rows *out, float *lse,
                          uint32_t n_q_heads, const int32_t *block_table, uint64_t table_stride,
                          uint32_t max_blocks, const int32_t *len, const int32_t *q_start,
                          uint32_t n_requests, uint32_t n_tokens, uint32_t max_len, float scale,
                          uint32_t window, uint32_t *verdict, void *ws, uint64_t ws_bytes,
                          void *stream) {
  AttendArgs a;
  const wm_status s = check_cache(cache, &a.bt_log2);
  if (s != WM_OK) return s;
  if (!check_rows(q) || !check_rows(out) || q->dtype != out->dtype || !aligned(lse, 4) ||
      !aligned(verdict, 4) || !std::isfinite(scale))
    return WM_ERR_INVALID_ARG;
  if (!n_q_heads || n_q_heads % cache->n_heads || n_requests > 0x3FFFFFFFu ||
      (uint64_t)n_tokens * n_q_heads > 0x3FFFFFFFull || max_len > 0x7FFFFFFFu ||
      window > 0x7FFFFFFFu || table_stride < max_blocks ||
      (uint64_t)max_blocks * cache->block_tokens > 0x7FFFFFFFull)
    return WM_ERR_INVALID_ARG;
  if (!n_requests || !n_tokens) return WM_OK;
  if (!q->ptr || !out->ptr || !len || !q_start || (max_blocks && !block_table) ||
      !aligned(block_table, 4) || !aligned(len, 4) || !aligned(q_start, 4))
    return WM_ERR_INVALID_ARG;
  a.plan = attend_plan(n_requests, n_tokens, cache->n_heads, n_q_heads, cache->head_dim, max_len);
  const uint64_t vectors = (uint64_t)n_tokens * n_q_heads * a.plan.splits;
  a.part_out = a.part_lse = nullptr;
  if (a.plan.splits > 1) {
    if (!ws || !aligned(ws, 16) || ws_bytes < vectors * (cache->head_dim + 1u) * 4u)
      return WM_ERR_WORKSPACE;
    a.part_out = static_cast<float *>(ws);
    a.part_lse = a.part_out + vectors * cache->head_dim;
  }
  a.c = *cache;
  a.q = *q;
  a.out = *out;
  a.lse = lse;
  a.table = block_table;
  a.table_stride = table_stride;
  a.len = len;
  a.q_start = q_start;
  a.verdict = verdict;
  a.n_requests = n_requests;
  a.n_tokens = n_tokens;
  a.group = n_q_heads / cache->n_heads;
  a.max_blocks = max_blocks;
  a.window = window;
  a.n_cu = (uint32_t)cus();
  if (!a.n_cu) return WM_ERR_HIP;
  a.scale_log2 = (float)((double)scale * 1.4426950408889634);
  return hip_status(launch_cache_attend(a, stream));
}

uint64_t wm_flat_pages_bytes(const wm_pool *pools, uint32_t n_pools, uint32_t n_pages) {
  uint64_t total = 0;
  return pool_layout(pools, n_pools, n_pages, &total) ? total : 0;
}

wm_status wm_flatten_pages(const wm_pool *pools, uint32_t n_pools, const int32_t *pages,
                           uint32_t n_pages, void *flat, uint64_t flat_cap, uint32_t *verdict,
                           void *stream) {
  return pages_call(true, pools, n_pools, pages, n_pages, static_cast<uint8_t *>(flat), flat_cap,
                    verdict, stream);
}

wm_status wm_rehydrate_pages(const void *flat, uint64_t flat_cap, const wm_pool *pools,
                             uint32_t n_pools, const int32_t *pages, uint32_t n_pages,
                             uint32_t *verdict, void *stream) {
  return pages_call(false, pools, n_pools, pages, n_pages,
                    static_cast<uint8_t *>(const_cast<void *>(flat)), flat_cap, verdict, stream);
}

}  // extern "C"

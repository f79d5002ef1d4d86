// wm_cache_internal.h -- launch interfaces of the paged 8-bit cache
// (declared in include/wm_cache.h).
#pragma once
#include <cstdint>

#include "wm_cache.h"

namespace wm {

struct TablesArgs {
  const int32_t *old_len, *new_len;
  int32_t *table;
  uint64_t table_stride;
  int32_t *ring;
  const uint32_t *pool_in;
  uint32_t *pool_out;
  int64_t *slots;
  uint64_t slot_cap;
  int32_t *q_start;
  uint32_t *verdict;
  uint32_t n_requests, bt_log2, max_blocks, ring_cap;
};
int launch_page_tables(const TablesArgs &a, void *stream);

struct AppendArgs {
  wm_cache c;
  wm_rows k, v;
  const int64_t *slots;
  const int32_t *q_start;
  uint32_t *verdict;
  uint32_t n_requests, n_tokens, bt_log2;
};
int launch_cache_append(const AppendArgs &a, void *stream);

// How an attention call is laid out (a function of host numbers alone).
struct AttendPlan {
  uint32_t rows;    // query rows (tokens x group) of a tile
  uint32_t tiles;   // tile places: at least the tiles of every request
  uint32_t splits;  // most parts that a tile's sequence is cut into: 1..32
  uint32_t cut;     // a part has 2^cut tokens at least
};
AttendPlan attend_plan(uint32_t n_requests, uint32_t n_tokens, uint32_t n_heads,
                       uint32_t n_q_heads, uint32_t head_dim, uint32_t max_len);

struct AttendArgs {
  wm_cache c;
  wm_rows q, out;
  float *lse;
  const int32_t *table;
  uint64_t table_stride;
  const int32_t *len, *q_start;
  uint32_t *verdict;
  float *part_out, *part_lse;  // workspace: [tokens][query heads][splits] vectors, numbers
  AttendPlan plan;
  uint32_t n_requests, n_tokens, group, max_blocks, bt_log2, window, n_cu;
  float scale_log2;  // scale * log2(e)
};
int launch_cache_attend(const AttendArgs &a, void *stream);
// A grid of n workgroups and more on two axes: one axis holds 2^32 threads.
inline uint32_t grid_x(uint32_t n) { return n < 1u << 22 ? n : 1u << 22; }
inline uint32_t grid_y(uint32_t n) { return (n - 1u) / (1u << 22) + 1u; }
// The tiles of one head size (a file each).
int launch_attend_64(const AttendArgs &a, void *stream);
int launch_attend_128(const AttendArgs &a, void *stream);
int launch_attend_192(const AttendArgs &a, void *stream);
int launch_attend_256(const AttendArgs &a, void *stream);
constexpr int kAttThreads = 256;

// Pools whose addresses travel in a launch's arguments: no copy of the
// caller's host table, so the call may be captured.
constexpr uint32_t kPoolsPerLaunch = 64;
struct PoolBatch {
  struct {
    uint64_t ptr, stride, off;  // off: of the pool's first page in flat
    uint64_t page_bytes, n_blocks;
    uint64_t first;             // first piece of this pool in the launch
  } p[kPoolsPerLaunch];
  uint64_t pieces;
  uint32_t n;
};
int launch_pages(bool gather, const PoolBatch &b, uint8_t *flat, const int32_t *pages,
                 uint32_t n_pages, uint64_t least_blocks, uint32_t *verdict, bool wide, int n_cu,
                 void *stream);
// A list of up to this many blocks is looked at by the copy's workgroups
// themselves (one launch less: 1.3 of 8.5 us); a longer one by a launch before.
constexpr uint32_t kPagesLooked = 1024;
// ORs WM_C_PAGE into *verdict if a page is outside [0, least_blocks).
int launch_check_pages(const int32_t *pages, uint32_t n_pages, uint64_t least_blocks,
                       uint32_t *verdict, void *stream);
constexpr uint64_t kPiece = 16384;  // bytes of a page that a workgroup takes at once

}  // namespace wm

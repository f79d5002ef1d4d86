/*
 * wm_cache.h -- C ABI of libwm's paged 8-bit attention cache on MI355X.
 *
 * A session that the mover (wm.h) installs answers from its cache; a server
 * holds that cache in blocks of tokens shared by many requests.  These calls
 * are what such a session needs around its move:
 *
 *   wm_page_tables      block tables and slot maps from request lengths
 *   wm_cache_append     new keys and values into the cache, in 8 bits
 *   wm_cache_attend     attention over the cache
 *   wm_flatten_pages    a session's blocks into the mover's flat state
 *   wm_rehydrate_pages  the flat state into blocks of another pool
 *
 * Conventions, beyond wm.h's:
 *   - Every pointer is a DEVICE pointer of the caller's unless a comment says
 *     "host".  The calls only enqueue kernels on `stream` and return; they
 *     allocate and keep nothing, copy nothing from the host and may be
 *     captured into a graph.  Lengths stay on the device.
 *   - Argument errors are found on the host, before anything is enqueued.
 *   - What only the device can see (a length, a block or a slot out of
 *     range) never leaves the buffers: it becomes a bit of the caller's
 *     device word `verdict`, as documented for each call.
 *   - Results are the same on every run: no output depends on the order in
 *     which workgroups run, nor on which blocks a session was given.
 *   - Calls on different streams that write the same buffers, workspace or
 *     verdict word must be ordered.
 *   - Types: lengths, block ids and row starts are int32, slots are int64.
 */
#ifndef WM_CACHE_H
#define WM_CACHE_H

#include <stdint.h>

#include "wm.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bits of the device verdict word of these calls. */
#define WM_C_LENGTH 1u /* a length below 0 or beyond the block table */
#define WM_C_POOL 2u   /* fewer free blocks than needed, or more than fit */
#define WM_C_SLOTS 4u  /* more new tokens than the slot map or the rows hold */
#define WM_C_PAGE 8u   /* a block or slot outside the pool */

/* Element types of queries, keys, values and outputs. */
#define WM_BF16 1
#define WM_FP16 2

/* Code types of the cache: OCP 8-bit floats. */
#define WM_E4M3 1 /* largest value 448, no infinities */
#define WM_E5M2 2 /* largest value 57344 */

/* One layer's cache in a pool of n_blocks blocks of block_tokens tokens:
 *   keys    [n_blocks][n_heads][block_tokens][head_dim] codes
 *   values  [n_blocks][n_heads][head_dim][block_tokens] codes (transposed:
 *           the matrix cores read one head dimension of several tokens)
 *   scales  [n_blocks][n_heads] float: a value is its code times the scale
 * The strides are those from a block to the next (codes: bytes, a multiple
 * of 16; scales: floats), so that one pool may hold every layer's blocks side
 * by side; everything inside a block is dense.  k and v are 16-byte aligned.
 * Scales are finite and not negative. */
typedef struct wm_cache {
  void *k, *v;
  float *k_scale, *v_scale;
  uint64_t k_stride, v_stride;
  uint64_t k_scale_stride, v_scale_stride;
  uint32_t n_blocks;     /* 1..2^31-1 */
  uint32_t n_heads;      /* 1..65535 */
  uint32_t block_tokens; /* 16, 32, 64, 128 or 256 */
  uint32_t head_dim;     /* 64, 128, 192 or 256 */
  uint32_t format;       /* WM_E4M3 or WM_E5M2 */
  uint32_t flags;        /* must be 0 */
} wm_cache;

/* A matrix of vectors: row (token) t, head h begins at
 * ptr + t * row_stride + h * head_stride elements; the vector is dense. */
typedef struct wm_rows {
  void *ptr;
  uint64_t row_stride, head_stride;
  uint32_t dtype; /* WM_BF16 or WM_FP16 */
  uint32_t flags; /* must be 0 */
} wm_rows;

/* ---- block tables and slot maps -------------------------------------------
 * One step of a scheduler: request r goes from old_len[r] to new_len[r]
 * tokens.  A request that grows takes blocks from the front of the free
 * ring; one that shrinks (0: it is done) gives its last ones back at the
 * ring's end, where this call does not take them.  With b and c the block
 * counts before and after, and takes and returns ordered by request, then by
 * place in the request:
 *   block_table[r][b + j] = the next block taken          (c > b)
 *   the next place returned to = block_table[r][c + j]    (b > c)
 *   q_start[r]  = sum over requests before r of max(0, new - old);
 *                 n_requests + 1 entries, the last the number of new tokens
 *   slot_map[q_start[r] + i] = block_table[r][p / bt] * bt + p % bt, with
 *                 p = old_len[r] + i: where new token i of r is stored
 * Other entries of the tables, and slots behind the last new token, are left
 * as they were.
 *   old_len, new_len : n_requests each
 *   block_table : n_requests rows of max_blocks entries, table_stride apart
 *   free_ring   : ring_cap block ids, of which `count` from place `head` on
 *                 (round the end) are free
 *   pool_in     : {head, count} before; pool_out: the same after.  Two
 *                 different buffers: a call that is repeated with the same
 *                 inputs gives the same outputs
 *   slot_map    : slot_cap entries
 *   verdict     : 1 u32, written: 0, or WM_C_LENGTH alone, or WM_C_POOL and
 *                 WM_C_SLOTS; then no table, ring, slot or start changed and
 *                 pool_out is pool_in
 * n_requests 0 is allowed (pool_out is pool_in, q_start[0] is 0).
 * Errors: WM_ERR_INVALID_ARG, WM_ERR_UNSUPPORTED (block_tokens not listed
 *         above), WM_ERR_HIP. */
wm_status wm_page_tables(const int32_t *old_len, const int32_t *new_len,
                         uint32_t n_requests, uint32_t block_tokens,
                         int32_t *block_table, uint64_t table_stride,
                         uint32_t max_blocks, int32_t *free_ring,
                         uint32_t ring_cap, const uint32_t *pool_in,
                         uint32_t *pool_out, int64_t *slot_map,
                         uint64_t slot_cap, int32_t *q_start,
                         uint32_t *verdict, void *stream);

/* ---- store new keys and values ----------------------------------------------
 * Rows q_start[r] .. q_start[r + 1] - 1 of k and v are request r's new tokens,
 * in order, and slot_map says where each is stored (wm_page_tables).  For each
 * block and head that gets tokens, with F the format's largest value and a the
 * largest finite magnitude of what it gets (keys and values apart):
 *   a block whose first place gets a token, or whose scale is no positive
 *   finite (and normal) number, is fresh: its scale becomes 2^e
 *   with the smallest e >= -100 such that a <= F 2^e, and its places that
 *   get no token become zero;
 *   any other block keeps its scale s if a <= F s, else the scale becomes
 *   s 2^n with the smallest n that is enough and its older codes are rounded
 *   again to it (a power of two: exact but for values that get subnormal).
 *   code = x / scale, rounded to nearest, ties to even (a quotient that is not
 *   exact, by a scale of the caller's that is no power of two, to 32 bits
 *   first); an infinity becomes the largest value of its sign, a NaN stays one.
 *   slot_map : n_tokens entries; where the first new token of a block has a
 *              slot below 0 (padding) or beyond the pool (sets WM_C_PAGE), or
 *              where the slots of a block's first and last new token do not fit
 *              consecutive places (sets it too), the block's are not stored
 *   n_tokens : rows that k, v and slot_map have; q_start beyond it sets
 *              WM_C_SLOTS and those tokens are not stored.  Rows behind the
 *              last request's are not read
 *   verdict  : 1 u32 that bits are ORed into, or NULL
 * A request's new tokens have consecutive places, as wm_page_tables gives
 * them, and no block belongs to two requests that get tokens in one call.
 * Errors: WM_ERR_INVALID_ARG, WM_ERR_UNSUPPORTED (block_tokens or head_dim
 *         not listed above), WM_ERR_HIP. */
wm_status wm_cache_append(const wm_cache *cache, const wm_rows *k,
                          const wm_rows *v, const int64_t *slot_map,
                          const int32_t *q_start, uint32_t n_requests,
                          uint32_t n_tokens, uint32_t *verdict, void *stream);

/* ---- attention ------------------------------------------------------------
 * Query row q_start[r] + i of request r stands at position
 * p = len[r] - (q_start[r+1] - q_start[r]) + i of its sequence (len counts the
 * new tokens, which are in the cache already) and sees the tokens
 * j <= p, and with window > 0 only j > p - window.  Query head h reads key
 * head h / (n_q_heads / n_heads).
 *   s_j = scale * <q, K_j>,  out = sum_j softmax(s)_j V_j,
 *   lse = log sum_j exp s_j
 * A row that sees nothing (p < 0, a length of 0) gets zeros and lse = -inf.
 * What a row does not see has no influence on it, infinities and NaN
 * included; a value that is not finite reaches every row that sees it, however
 * small its weight.  Scores, softmax and sums are in 32 bits.  One query row per
 * request is the form for single tokens; many are a prompt or a chunk of it.
 * (The kernel goes by the mean of rows per request: a prompt and many single
 * tokens are faster in two calls than in one.)
 * With up to 32 query heads to a key head, a single token gets the same bits
 * in any call of single tokens whose max_len is not below its length.
 * Weights, times the scales of their values, are rounded to 11 bits for bf16
 * outputs and 22 for fp16 ones before they meet the codes; those far below the
 * row's largest to 2^-35 of it.
 *   q, out      : n_tokens rows of n_q_heads heads, the same type, fewer
 *                 than 2^30 vectors; rows behind the last request's are
 *                 neither read nor written
 *   lse         : n_tokens x n_q_heads float, dense, or NULL
 *   block_table : as for wm_page_tables; entries that no row sees are not
 *                 used.  A block outside the pool is not read: its tokens
 *                 count as unseen and WM_C_PAGE is set
 *   q_start     : n_requests + 1, ascending.  Starts below 0 or beyond n_tokens
 *                 set WM_C_SLOTS: the rows that are there stand where the
 *                 formula says, the others are not computed
 *   len         : n_requests; where a request has rows, a length below 0 or
 *                 beyond the table's max_blocks sets WM_C_LENGTH and counts as
 *                 0 or as that many tokens
 *   max_len     : host: the longest length, for the split of the work; the
 *                 outputs stay right if a length is larger
 *   verdict     : 1 u32 that bits are ORed into, or NULL
 *   ws          : ws_bytes >= wm_attend_ws_bytes() of the same numbers,
 *                 16-byte aligned (NULL if that is 0)
 * Errors: WM_ERR_INVALID_ARG, WM_ERR_UNSUPPORTED, WM_ERR_WORKSPACE,
 *         WM_ERR_HIP. */
wm_status wm_cache_attend(const wm_cache *cache, const wm_rows *q,
                          const wm_rows *out, float *lse, uint32_t n_q_heads,
                          const int32_t *block_table, uint64_t table_stride,
                          uint32_t max_blocks, const int32_t *len,
                          const int32_t *q_start, uint32_t n_requests,
                          uint32_t n_tokens, uint32_t max_len, float scale,
                          uint32_t window, uint32_t *verdict, void *ws,
                          uint64_t ws_bytes, void *stream);

/* Workspace of wm_cache_attend (partial results where few rows read a long
 * cache); the same on every device.  0: none is needed. */
uint64_t wm_attend_ws_bytes(uint32_t n_requests, uint32_t n_tokens,
                            uint32_t n_heads, uint32_t n_q_heads,
                            uint32_t head_dim, uint32_t max_len);

/* ---- a session's blocks and the flat state ----------------------------------
 * wm_flatten and wm_rehydrate for state that lies in pools: pool i holds
 * n_blocks pages of page_bytes, `stride` bytes from one to the next (a cache's
 * codes or scales, of one layer or of all; of any type, also 16-bit caches).
 * Flat layout: pool i's listed pages in the list's order, dense, from off_i on;
 * off_0 = 0, off_{i+1} = off_i + round_up(n_pages * page_bytes, 16); flatten
 * writes zeros into the gaps. */
typedef struct wm_pool {
  void *ptr;           /* 4-byte aligned */
  uint64_t page_bytes; /* a multiple of 4 */
  uint64_t stride;     /* >= page_bytes, a multiple of 4 */
  uint64_t n_blocks;   /* 1..2^31-1 */
} wm_pool;

#define WM_MAX_POOLS 4096

/* Flat size of n_pages pages of each pool; 0 for a NULL table with n_pools
 * above 0 or a sum beyond 2^62.  pools: host array. */
uint64_t wm_flat_pages_bytes(const wm_pool *pools, uint32_t n_pools,
                             uint32_t n_pages);

/* Gather (flatten) and scatter (rehydrate).
 *   pools   : host array of n_pools entries (read before returning)
 *   pages   : n_pages block ids, those of the session in order (a row of the
 *             block table).  They must differ from each other for rehydrate
 *   flat    : flat_cap >= wm_flat_pages_bytes() bytes, 16-byte aligned
 *   verdict : 1 u32.  The call does its work only if it is 0: the install
 *             after wm_decode_verify may be enqueued behind it with the same
 *             word.  A block id outside any of the pools sets WM_C_PAGE, and
 *             then nothing is written
 * flat must not overlap the pools.
 * Errors: WM_ERR_INVALID_ARG, WM_ERR_CAPACITY, WM_ERR_HIP. */
wm_status wm_flatten_pages(const wm_pool *pools, uint32_t n_pools,
                           const int32_t *pages, uint32_t n_pages, void *flat,
                           uint64_t flat_cap, uint32_t *verdict, void *stream);
wm_status wm_rehydrate_pages(const void *flat, uint64_t flat_cap,
                             const wm_pool *pools, uint32_t n_pools,
                             const int32_t *pages, uint32_t n_pages,
                             uint32_t *verdict, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* WM_CACHE_H */

/*
 * Upkeep of a paged cache (plora_paged.h) between steps: requests that are continued
 * by several others, cut short, reordered or ended, with their pages shared, copied
 * and given back; and keys moved inside the caches of all layers.
 *
 *   plora_kv_remap    the block table of a new batch from that of an old one
 *   plora_kv_copy     the pages that a remap has to copy, in all layers
 *   plora_kv_compact  the keys of an accepted path (plora_tree.h), in all layers
 *
 * A page is held by every request whose table row names it among its first
 * ceil(length / page_size) entries, and by whoever else keeps it (an adapter's prompt,
 * a request that waits).  shares int32 [n_pages] counts the holders of a page beyond
 * the first: 0 for a page as plora_kv_plan hands it out, and for a free one, so an
 * array of zeros goes with a new pool.  A holder outside the batches is counted by the
 * caller, who adds 1 for it; and plora_kv_remap is all that is needed to drop one (a
 * batch of one, continued by none).
 *
 * Free pages are free_pages[*free_head ..], as plora_kv_plan takes them.  Pages that
 * come free are put before the head, so a list with room for all pages of the pool
 * never overflows.
 *
 * Types, errors, streams and determinism are those of plora_paged.h; a failed launch
 * is reported by plora_paged_last_hip_error.
 */
#ifndef PLORA_PAGES_H
#define PLORA_PAGES_H

#include <stddef.h>
#include <stdint.h>

#include "plora_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most layers of one call. */
#define PLORA_CACHE_MAX_LAYERS 1024

/* A pool's pages and who holds them. */
typedef struct {
  int32_t n_pages;
  int32_t n_free;       /* entries of free_pages */
  int32_t* shares;      /* [n_pages], updated */
  int32_t* free_pages;  /* [n_free], entries before the head are written */
  int32_t* scratch;     /* [n_pages][2], 8-byte aligned, no contents needed */
} plora_page_pool;

/* A batch before or after a remap. */
typedef struct {
  int32_t batch;
  int32_t max_pages;
  int32_t* table;       /* [batch][max_pages] */
  int32_t* kv_len;      /* [batch] */
} plora_kv_batch;

/*
 * Request i of the new batch holds the first n_i keys of request src_i of the old one:
 * n_i = kv_len_old[src_i], or less if keep (int32, may be NULL) says so, and 0 where
 * src_i is no request of the old batch.  Any number of requests may continue one, with
 * lengths of their own; an old request that none continues has ended.
 *
 * With P_i = ceil(n_i / page_size), new request i's row names the pages of its first
 * P_i entries (the rest of the row is left as it was) and is one holder of each; the
 * old requests hold nothing any more.  Then
 *   - a page that nobody holds is put into the free list: in the order of the old
 *     batch's requests and their entries, so that they lie from the new head on, and
 *   - where a new request's last page is partly filled and has other holders, who might
 *     write behind its keys or whose keys lie there, the request gets a page of its own
 *     from the list, and copies tells what to copy: looked at in the order of the
 *     requests, so the last of those that hold nothing else of it keeps the page itself.
 * *free_next = *free_head - pages put there + pages taken.  If the list has no page to
 * give, the request (and every later one that needs one) ends at its last whole page,
 * kv_len saying so, and is counted.
 *
 *   src     int32 [new->batch]
 *   copies  int32 [new->batch][3]: page, new page, keys of it; -1 behind the last
 *   meta    int32 [8]: pages put into the list, pages taken (copies), requests ended
 *           at a whole page for want of one, pages that came free for which the list
 *           had no room before its head (lost to it), 0...
 * A page outside the pool is held by nobody and not copied.  Lengths below 0 count as
 * 0, and above max_pages page_size as that.  A row names no page twice among those
 * that it holds.  The two batches' arrays, src, keep, free_head, free_next, copies and
 * meta must not overlap.  The old batch's rows, of 1024 requests, have up to 2^31 - 2^14
 * entries.  ws: plora_kv_remap_workspace_bytes, 16-byte aligned, no contents needed.
 * One launch for small batches, two or three for larger ones.
 */
size_t plora_kv_remap_workspace_bytes(int32_t old_batch, int32_t new_batch);
plora_status plora_kv_remap(const plora_kv_batch* old_batch, const int32_t* src,
                            const int32_t* keep, int32_t page_size,
                            const plora_page_pool* pool, const int32_t* free_head,
                            int32_t* free_next, const plora_kv_batch* new_batch,
                            int32_t* copies, int32_t* meta, void* ws, size_t ws_bytes,
                            hipStream_t stream);

/*
 * The first keys of pages copied to others, in the k and v of every layer, as a remap
 * lists them: copies [cap][3], *n_copies of them (device; &meta[1] of the remap; at
 * most cap count).  caches: the layers' caches (host array), all of one shape and
 * strides.  Entries of pages outside the pool are left out; keys are cut off at
 * page_size.  No page is both copied to and from, and none copied to twice.
 */
plora_status plora_kv_copy(const plora_kv_cache* caches, int32_t layers, const int32_t* copies,
                           int32_t cap, const int32_t* n_copies, hipStream_t stream);

/*
 * The keys of accepted paths moved together: for each request b of the step and
 * i < count_b, in this order, the key and value at the slot of its new token
 * path[q_start_b + i] are stored at the slot of its new token i (path and count as
 * plora_tree_accept leaves them), in the k and v of every layer.  A number outside the
 * request's tokens, or a slot outside the pool, moves nothing; slots of the step's
 * tokens differ.
 */
plora_status plora_kv_compact(const plora_kv_cache* caches, int32_t layers,
                              const plora_kv_step* step, const int32_t* path,
                              const int32_t* count, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PLORA_PAGES_H */

/*
 * What a serving step on one MI355X needs between a layer's q, k, v
 * projections (plora.h) and its output projection, over a paged cache:
 *
 *   plora_kv_plan      once a step: token starts, positions, block table
 *                      entries for new pages and cache slots, from the
 *                      request lengths, on the GPU
 *   plora_rope         rotary positions of one tensor, or (inverse) its gradient
 *   plora_rope_append  rotary positions of q and k, k and v stored in the cache
 *   plora_attn_plan    once a step: the work of the attention, balanced over
 *                      the chip; groups of requests that share a prefix
 *   plora_attn_paged   per layer: attention over the cache
 *
 * The batch of a step: request b (0 <= b < batch) has past_b keys in the cache
 * and brings n_b >= 0 new tokens, which lie one after another in request order
 * in the T rows of the step's activations.  Token t of request b:
 *
 *   q_start_b = n_0 + ... + n_(b-1),   kv_len_b = past_b + n_b
 *   pos_t  = past_b + t - q_start_b
 *   slot_t = table[b][pos_t / page_size] page_size + pos_t % page_size
 *
 * Layouts (row-major, device memory owned by the caller; strides in elements):
 *   q, k, v  [T][heads][head_dim] with a token stride and a head stride
 *   cache    pages of page_size keys: element d of key o of head h of page p at
 *            p page_stride + h head_stride + o token_stride + d, in k and in v
 *   table    int32 [batch][max_pages]: page ids, in the order of the keys
 * Types: bf16 or fp16 bits (plora_dtype), fp32 arithmetic, one rounding to
 * nearest even at each store (and that of the softmax weights named under
 * plora_attn_paged).  Every call is asynchronous on stream, allocates nothing,
 * keeps no pointer, and is bitwise deterministic.
 *
 * Errors, before anything is launched: PLORA_ERR_INVALID_ARG for a null required
 * pointer, a negative size or stride, or sizes that do not fit each other;
 * PLORA_ERR_UNSUPPORTED for what lies outside the stated ranges or alignments;
 * PLORA_ERR_WORKSPACE_TOO_SMALL; PLORA_ERR_HIP for a failed launch.  T, batch or
 * heads of 0 is a no-op, with these exceptions: plora_kv_plan still writes its
 * per-request outputs, and plora_rope_append with heads of 0 has no q to turn but
 * stores k and v (with kv_heads of 0 it turns q alone).
 * What only the device can see never faults: a request that cannot be served is
 * left out and counted, a slot or page id outside the pool is not written and
 * reads as zeros.
 */
#ifndef PLORA_PAGED_H
#define PLORA_PAGED_H

#include <stddef.h>
#include <stdint.h>

#include "plora.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { PLORA_BF16 = 0, PLORA_FP16 = 1 } plora_dtype;
typedef enum { PLORA_ROPE_HALF = 0, PLORA_ROPE_INTERLEAVED = 1 } plora_rope_layout;

/* Most requests of a step, and most tokens (as for plora_segment). */
#define PLORA_PAGED_MAX_BATCH 16384
#define PLORA_PAGED_MAX_TOKENS 1048576
/* Most keys a row of the block table may name (max_pages page_size). */
#define PLORA_PAGED_MAX_KEYS (1 << 30)
/* Pages hold a power of two of keys in this range. */
#define PLORA_PAGE_MIN 16
#define PLORA_PAGE_MAX 256
/* Longest head plora_rope takes. */
#define PLORA_ROPE_MAX_DIM 512

/* One layer's cache.  head_dim is 64 or 128 for plora_attn_paged, any even
 * number up to PLORA_ROPE_MAX_DIM for plora_rope_append. */
typedef struct {
  int32_t n_pages;
  int32_t page_size;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t dtype;
  int32_t reserved;
  void* k;
  void* v;
  int64_t page_stride;
  int64_t head_stride;
  int64_t token_stride;
} plora_kv_cache;

/* A step's buffers.  T is the number of rows of its activations; rows past the
 * requests' tokens are padding: req -1, pos 0, slot -1. */
typedef struct {
  int32_t batch;
  int32_t T;
  int32_t page_size;
  int32_t max_pages;
  int32_t* table;    /* [batch][max_pages], entries of held pages set; new ones are written */
  int32_t* q_start;  /* [batch + 1], clamped to T */
  int32_t* kv_len;   /* [batch] */
  int32_t* pos;      /* [T] */
  int32_t* req;      /* [T] */
  int64_t* slot;     /* [T] */
  int32_t* meta;     /* [8]: rows of requests' tokens, pages taken, requests left out, 0... */
} plora_kv_step;

/*
 * Fill the step from past [batch] and n_new [batch] (int32).  New pages are
 * taken from free_pages [n_free] (int32 page ids), from *free_head on, in
 * request order: request b takes ceil(kv_len_b / page_size) -
 * ceil(past_b / page_size) of them, into the entries of its row that follow the
 * held ones.  *free_next = *free_head + the pages taken.  Inputs and outputs
 * must not overlap (a loop hands kv_len and free_next to the next step as past
 * and free_head).  The pages of a request that has ended are the caller's to put
 * behind the list's end or into a later step's list.  A request is left out if
 * past or n_new is negative, its length passes max_pages page_size, its tokens
 * pass T, or the free list is too short for it (then every later request that
 * needs a page is left out too): it takes no pages, its kv_len is max(past, 0),
 * its tokens are padding.
 * Requests of n_new 0 keep their length.  One launch.
 */
plora_status plora_kv_plan(const int32_t* past, const int32_t* n_new,
                           const int32_t* free_pages, int32_t n_free,
                           const int32_t* free_head, int32_t* free_next,
                           const plora_kv_step* step, hipStream_t stream);

/*
 * Rotary positions.  The first rot elements of each head are pairs (a, b),
 * pair i being elements (i, rot/2 + i) (PLORA_ROPE_HALF) or (2i, 2i + 1)
 * (PLORA_ROPE_INTERLEAVED); with the angle f = 2 pi frac(pos turns_i / 2^64),
 *
 *   a' = scale (a cos f - b sin f),   b' = scale (a sin f + b cos f)
 *
 * and elements rot.. are copied unscaled.  turns: uint64 [rot/2] in device
 * memory, turns per position in units of 2^-64 (a frequency w in radians per
 * position gives w / (2 pi) 2^64): the part of a turn is exact in whole numbers
 * at any position, where a product of floats loses it in long contexts.
 * inverse: the transposed map (f -> -f), the gradient of the input from that of
 * the output.  rot is even, 0 <= rot <= head_dim; head_dim is even, up to
 * PLORA_ROPE_MAX_DIM; pos int32 [T].  out may be x itself (with its strides),
 * and must not overlap it otherwise.
 */
plora_status plora_rope(const void* x, int64_t x_token, int64_t x_head, const int32_t* pos,
                        const uint64_t* turns, int32_t T, int32_t heads, int32_t head_dim,
                        int32_t rot, int32_t layout, float scale, int32_t inverse, int32_t dtype,
                        void* out, int64_t out_token, int64_t out_head, hipStream_t stream);

/*
 * q rotated into q_out (which may be q itself), k rotated into the cache and v
 * copied there, token t at slot[t]; a token whose slot is negative or outside
 * the pool is not stored (its q is rotated all the same).  Either may be absent:
 * heads of 0 (q and q_out NULL) or kv_heads of 0 (k and v NULL).  cache gives the
 * key heads, the head dimension and the type of all four.  slots of one call
 * must differ.
 */
plora_status plora_rope_append(const void* q, int64_t q_token, int64_t q_head,
                               const void* k, int64_t k_token, int64_t k_head,
                               const void* v, int64_t v_token, int64_t v_head,
                               const int32_t* pos, const int64_t* slot, const uint64_t* turns,
                               int32_t T, int32_t heads, int32_t rot, int32_t layout, float scale,
                               const plora_kv_cache* cache, void* q_out, int64_t out_token,
                               int64_t out_head, hipStream_t stream);

/*
 * The shape of a step's attention: sizes known to the host.
 *   batch, T   as in the step
 *   heads      query heads, a multiple of kv_heads; query head h reads key head
 *              h / (heads / kv_heads)
 *   head_dim   64 or 128
 *   max_q      an upper bound on every request's new tokens (a request with
 *              more gets zeros, and plora_attn_plan counts it)
 *   shared     nonzero if plora_attn_plan will be given groups
 */
typedef struct {
  int32_t batch;
  int32_t T;
  int32_t heads;
  int32_t kv_heads;
  int32_t head_dim;
  int32_t max_q;
  int32_t shared;
  int32_t reserved;
} plora_attn_shape;

/* Host.  Bytes of a plan, and of the workspace one plora_attn_paged call uses;
 * 0 for an empty or unsupported shape. */
size_t plora_attn_plan_bytes(const plora_attn_shape* shape);
size_t plora_attn_paged_workspace_bytes(const plora_attn_shape* shape);

/*
 * The work of the step's attention, from the lengths in the step (as
 * plora_kv_plan left them): which query rows read which keys, cut into work
 * groups of about equal work.  Serves every layer of the step.
 *
 * Groups (shape->shared): seg is plora_segment's grouping of the batch, T =
 * batch, by an int32 group id per request (for a prompt that belongs to an
 * adapter: the request's adapter id; -1 for none), over n_groups groups;
 * prefix_len int32 [n_groups] (device) gives the leading keys that all requests
 * of a group have in common.  Their tables must name the same pages for the
 * whole pages of that prefix; those pages are then read once for the group.  A
 * request shares if its new tokens lie behind the prefix, it has at most
 * PLORA_ATTN_SHARE_ROWS query rows per key head (one with more fills the matrix
 * units by itself), and another request of its group does.  Without groups seg
 * and prefix_len are NULL; with n_groups of 0 prefix_len may be.  One launch.
 *
 * int32 word PLORA_ATTN_PLAN_LEFT_OUT of the plan is the number of requests that
 * have tokens in the step and are left out here, their outputs zeros: those of
 * more than max_q tokens, and those whose lengths do not agree with the step's
 * or the shape's bounds.  (Requests that plora_kv_plan left out are counted in
 * its meta.)
 */
#define PLORA_ATTN_SHARE_ROWS 128
#define PLORA_ATTN_PLAN_LEFT_OUT 6
plora_status plora_attn_plan(const plora_kv_step* step, const plora_attn_shape* shape,
                             const plora_segments* seg, const int32_t* prefix_len,
                             int32_t n_groups, void* plan, size_t plan_bytes,
                             hipStream_t stream);

/*
 * out[t][h] = sum_j p_j v_j,  p = softmax_j(scale <q[t][h], k_j>),  over the keys
 * j <= pos_t of token t's request.  A row with no key (padding, a request left
 * out) gets zeros; a key that a row does not see has no part in it, whatever its
 * values.  q_token, q_head, out_token, out_head: element strides (multiples of
 * 8), pointers 16-byte aligned, cache strides multiples of 8, the token stride
 * from head_dim to below 2^25 (a pool may have its pages, heads and keys in any
 * order).  Scores, weights and sums are fp32; the weights enter the product with
 * v as two values of the type (bf16: 16 bits) for requests of up to 16 query rows
 * per key head, and for others over a prefix that they share; as one (bf16: 8
 * bits) over the own keys of a request of more rows, where that product bounds
 * the call.  So a request's own size says how its weights are rounded, and the
 * batch that it is in never rounds them more.  out must not overlap q.  plan: as
 * plora_attn_plan wrote it for the same step and shape; ws: at least
 * plora_attn_paged_workspace_bytes bytes, 16-byte aligned, no contents needed.
 */
plora_status plora_attn_paged(const void* q, int64_t q_token, int64_t q_head,
                              const plora_kv_cache* cache, const plora_kv_step* step,
                              const plora_attn_shape* shape, float scale, const void* plan,
                              size_t plan_bytes, void* out, int64_t out_token, int64_t out_head,
                              void* ws, size_t ws_bytes, hipStream_t stream);

/* Test hook: the hipError_t of the most recent launch of this header's calls
 * that returned PLORA_ERR_HIP in this process, 0 if none did. */
int32_t plora_paged_last_hip_error(void);

#ifdef __cplusplus
}
#endif

#endif /* PLORA_PAGED_H */

/*
 * Trees of drafted tokens in a step over a paged cache (plora_paged.h): a request
 * brings several guesses of its next tokens at once, the model looks at all of
 * them in one step, and the longest path that it agrees with is kept.
 *
 *   plora_tree_plan    once a step: positions and descendants of the trees' nodes
 *   plora_attn_tree    per layer: attention in which a node sees the cached keys
 *                      and its own ancestors
 *   plora_tree_accept  once a step: the accepted path of every tree
 *
 * (plora_kv_compact in plora_pages.h then moves the accepted keys together, and
 * plora_kv_remap gives back the pages behind them.)
 *
 * The new tokens of a request are the nodes of its tree, numbered 0 .. n_b - 1 in
 * the order of its rows in the step (row q_start_b + i); several roots are allowed.
 * parent int32 [T] names, for row q_start_b + i, the node's parent by its number,
 * less than i, or -1 for a root.  A prompt, or a single token, is the tree in which
 * every parent is the node before ("a chain"), so a step holds any mix of prompts,
 * single tokens and trees.  The keys of the nodes lie in the cache in the order of
 * their numbers, as plora_kv_plan places them (step->slot); for their rotation a
 * node's position is past_b + its depth, which step->pos is not.
 *
 * A node is cut if its parent is out of range, if one of its ancestors is cut, or if
 * its request, not being a chain, has more than PLORA_TREE_MAX_NODES nodes.  A cut
 * node's position is 0, no node sees it, its attention is zeros, and it is not
 * accepted; the others of its request are as without it.  Rows of no request, or of a
 * request that the step left out, are as cut nodes.
 *
 * Types, errors, streams and determinism are those of plora_paged.h; a failed launch
 * is reported by plora_paged_last_hip_error.  With T of 0 the outputs of the requests
 * are written, with batch of 0 those of the rows, except by plora_attn_tree, for which
 * both are a no-op.
 */
#ifndef PLORA_TREE_H
#define PLORA_TREE_H

#include <stddef.h>
#include <stdint.h>

#include "plora_paged.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Most nodes of a request's tree (a chain may have any number). */
#define PLORA_TREE_MAX_NODES 1024

/* What a step knows of its trees. */
typedef struct {
  int32_t batch;
  int32_t T;
  int32_t* pos;   /* [T]: past + depth, for plora_rope and plora_rope_append */
  int32_t* span;  /* [T][2], 8-byte aligned: the first and last preorder number
                     (siblings in the order of their numbers) of the node and its
                     descendants; node j is i or an ancestor of i if
                     span[j][0] <= span[i][0] <= span[j][1].  -1, -2 of a cut one */
  int32_t* info;  /* [batch][2]: 1 for a tree that is no chain, else 0; nodes cut */
} plora_tree;

/* Fill the tree from parent and the step (as plora_kv_plan left it).  One launch. */
plora_status plora_tree_plan(const int32_t* parent, const plora_kv_step* step,
                             const plora_tree* tree, hipStream_t stream);

/*
 * As plora_attn_paged, with the same plan (plora_attn_plan, made for the same step and
 * shape, groups with shared prefixes included), but a new token sees, beside the
 * request's keys before past, the new keys of its ancestors and its own, and no other
 * new key.  The weights enter the product with v as there, and a chain, with or without a
 * shared prefix, has plora_attn_paged's outputs to the bit.
 */
plora_status plora_attn_tree(const void* q, int64_t q_token, int64_t q_head,
                             const plora_kv_cache* cache, const plora_kv_step* step,
                             const plora_attn_shape* shape, const plora_tree* tree, float scale,
                             const void* plan, size_t plan_bytes, void* out, int64_t out_token,
                             int64_t out_head, void* ws, size_t ws_bytes, hipStream_t stream);

/*
 * Which path of its tree each request keeps.  drafted [T] are the nodes' tokens,
 * target [T] the model's choice of the token behind each node (its most likely one, or
 * one drawn from its distribution: the kept tokens then have that distribution); both
 * of token_bytes 4 or 8, any values.  The first given_b nodes (given int32 [batch], or
 * NULL for 1 each; at most n_b) are certain: the root, which the step before chose, or
 * the tokens of a prompt.  Those of them that are not cut are the path's start; from its
 * last node on, the path goes to the child whose token is the node's target, of several
 * to the one with the lowest number, until there is none (without a start: to no node).
 * Of a request whose nodes are all cut, as those of a tree of too many, nothing is kept:
 * count is 0 and kv_len what it was before the step.
 *
 *   path   [T]      row q_start_b + i: the number of the path's i-th node, -1 behind
 *   count  [batch]  nodes on the path
 *   token  [batch]  the target behind its last node (of drafted's type), -1 if it is
 *                   empty
 *   kv_len [batch]  kv_len of the step, less the new tokens that are not on the path:
 *                   the keys to keep
 * Rows of no request have path -1.  The outputs must not overlap the inputs (kv_len
 * not the step's).  One launch.
 */
plora_status plora_tree_accept(const int32_t* parent, const void* drafted, const void* target,
                               int32_t token_bytes, const int32_t* given,
                               const plora_kv_step* step, int32_t* path, int32_t* count,
                               void* token, int32_t* kv_len, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PLORA_TREE_H */

// The layout of a step's attention plan and of the workspace, shared by the
// plan kernel and the attention's kernels, and the bounds that size both.
#ifndef PLORA_ATTN_PLAN_H
#define PLORA_ATTN_PLAN_H

#include <algorithm>

#include "paged_dev.h"

namespace paged {

// Rows of an item: a "few" item has up to kFew query rows of one key head, a
// "tile" up to kTile.
constexpr int kFew = 16;
constexpr int kTile = 128;
// Keys that a few item's four wavefronts, and a tile item, take at a time.
constexpr int kFewStep = 128;
constexpr int kTileStep = 64;

// The most pieces that cutting adds, over the whole launch (see attn_plan_kernel).
constexpr int kFewTarget = 4096;
constexpr int kTileTarget = 1024;

// Requests for which the plan's kernel keeps what it needs in LDS, and its arrays.
constexpr int kHere = 1024;
constexpr int kKeptArrays = 12;

// A set of query rows that read the same keys: the tokens of one request
// ("self"), or those of a group's members (its prefix).  Rows are numbered
// (token, head in the key head's group), token first; an item is a run of a
// set's rows against a range of its keys.
struct Item {
  int32_t tok;        // first token of the set: an index of the batch's rows, or of order
  int32_t row;        // first row of the item in the set
  int32_t rows;
  int32_t req;        // the request whose table row names the pages
  int32_t lo, hi;     // keys
  int32_t part;       // first row of the item's partials, -1: writes the output
  int32_t gathered;   // tok indexes order
};
static_assert(sizeof(Item) == 32, "two 16-byte loads");

// What the merge needs of a request.
struct ReqInfo {
  int32_t part, splits, rows;       // its own partials: part -1 if none, and its rows
  int32_t pre_part, pre_splits, pre_rows, pre_row;  // its prefix's: pre_part -1 if none
  int32_t state;                    // 0: no rows (zeros), 1: partials to merge, 2: written
};
static_assert(sizeof(ReqInfo) == 32, "");

struct Bounds {
  int32_t r;             // query heads per key head
  int32_t few_cap, tile_cap;
  int64_t part_rows;     // partial rows per key head
};

// The most items of each kind and the most partial rows a step of this shape can
// have.  The plan cuts a kind's sets into pieces of at least C keys, C >= work /
// (target / kv_heads), work = the sum over sets of tiles x keys, so the cuts add at
// most target / kv_heads items to one per tile.
inline Bounds bounds(const plora_attn_shape& s) {
  Bounds b{};
  b.r = s.heads / s.kv_heads;
  const int64_t rows = (int64_t)s.T * b.r;
  const int64_t few_more = (kFewTarget + s.kv_heads - 1) / s.kv_heads;
  const int64_t tile_more = (kTileTarget + s.kv_heads - 1) / s.kv_heads;
  const bool tiles = s.shared || (int64_t)s.max_q * b.r > kFew;
  const int64_t sharing = s.shared ? std::min(rows, (int64_t)s.batch * PLORA_ATTN_SHARE_ROWS) : 0;
  const int64_t groups = s.shared ? s.batch / 2 : 0;
  b.few_cap = (int32_t)(s.batch + groups + few_more);
  if (tiles) {
    const int64_t own = rows / kTile + std::min((int64_t)s.batch, rows / (kFew + 1));
    b.tile_cap = (int32_t)(own + sharing / kTile + groups + tile_more);
  }
  // rows with partials: those that share, twice; and those of sets cut in two or
  // more, at most two rows for each added item's
  const int64_t few_rows = std::min<int64_t>(kFew, s.shared ? kFew : (int64_t)s.max_q * b.r);
  b.part_rows = 2 * sharing + 2 * (few_rows * few_more + (tiles ? kTile * tile_more : 0));
  return b;
}

// Bytes of the plan: a header, the items, the gathered tokens, the requests, and what
// the plan's kernel keeps of many requests.
struct PlanLayout {
  size_t few, tile, order, req, kept, bytes;
};
inline PlanLayout plan_layout(const plora_attn_shape& s, const Bounds& b) {
  PlanLayout l{};
  l.few = 256;
  l.tile = l.few + align256((size_t)b.few_cap * sizeof(Item));
  l.order = l.tile + align256((size_t)b.tile_cap * sizeof(Item));
  l.req = l.order + align256(s.shared ? (size_t)s.T * 4 : 0);
  l.kept = l.req + align256((size_t)s.batch * sizeof(ReqInfo));
  l.bytes = l.kept + align256(s.batch > kHere ? (size_t)(s.batch + 1) * kKeptArrays * 4 : 0);
  return l;
}
struct PlanHeader {
  int32_t few, tiles;          // items: of few rows, from their list's start; of more
  int32_t part_rows;
  int32_t few_keys, tile_keys; // keys per piece
  int32_t later;               // short items of few rows, from their list's end
  int32_t left;                // requests whose tokens get zeros
};
static_assert(offsetof(PlanHeader, left) == 4 * PLORA_ATTN_PLAN_LEFT_OUT, "");

inline bool shape_ok(const plora_attn_shape& s) {
  return s.batch >= 0 && s.T >= 0 && s.heads >= 0 && s.kv_heads >= 0 && s.max_q >= 0 &&
         s.batch <= PLORA_PAGED_MAX_BATCH && s.T <= PLORA_PAGED_MAX_TOKENS &&
         s.kv_heads <= 1024 && s.heads <= 65536 &&
         (s.kv_heads == 0 || (s.heads % s.kv_heads == 0 && s.heads / s.kv_heads <= 1024)) &&
         (s.head_dim == 64 || s.head_dim == 128);
}
inline bool shape_empty(const plora_attn_shape& s) {
  return s.batch == 0 || s.T == 0 || s.heads == 0 || s.kv_heads == 0;
}

}  // namespace paged

#endif  // PLORA_ATTN_PLAN_H

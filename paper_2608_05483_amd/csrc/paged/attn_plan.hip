// The work of a step's attention, built on the GPU (include/plora_paged.h,
// plora_attn_plan): which query rows read which keys, in items of about equal work.

#include "attn_plan.h"

namespace paged {
namespace {

constexpr int kNT = 512;
constexpr int kWaves = kNT / 64;

struct PlanArgs {
  int32_t batch, T, r, kv_heads, max_q, page_size;
  int64_t max_keys;
  const int32_t *q_start, *kv_len, *req;
  // groups
  int32_t shared, n_groups, cap;
  const int32_t *perm, *seg_ptr, *seg_id, *meta, *prefix_len;
  // plan
  PlanHeader* head;
  Item *few, *tile;
  int32_t* order;
  ReqInfo* info;
  int32_t* kept;             // kKeptArrays x [batch + 1], steps of more than kHere requests
  int32_t few_cap, tile_cap, part_cap;
};

// What is found out once about each request and each group, in LDS or, for steps
// of more than kHere requests, in the plan.
struct Kept {
  // requests: new tokens (0: none, or the step left it out), the first, keys, keys
  // that it shares, its group, the place of its first token in the groups' order
  int32_t *n, *q0, *kv, *u, *seg, *place;
  // entries of perm: tokens of members before it
  int32_t* moff;
  // groups: first entry of perm, keys of the prefix, who could share (then the
  // prefix's first partial row), its pieces, its first member
  int32_t *begin, *pre, *part, *splits, *req;
};
static_assert(sizeof(Kept) == kKeptArrays * sizeof(int32_t*), "");

// Counts, none below 0, are kept to 2^30, above every cap.
constexpr uint32_t kMany = 1u << 30;
struct AddCount {
  __device__ uint32_t operator()(uint32_t a, uint32_t b) const { return min(a + b, kMany); }
};
struct Max {
  __device__ int operator()(int a, int b) const { return max(a, b); }
};

// Exclusive scans of N counts a thread over the work group, from carry on, which
// then holds the sums.
template <int N>
__device__ __forceinline__ void scan(uint32_t (&x)[N], uint32_t (&carry)[N],
                                     uint32_t (&red)[kWaves][N]) {
  const AddCount add;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  uint32_t inc[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    inc[i] = wave_scan(x[i], add);
    if (lane == 63) red[wv][i] = inc[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    uint32_t before = carry[i], all = carry[i];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const uint32_t y = red[w][i];
      if (w < wv) before = add(before, y);
      all = add(all, y);
    }
    // (what is before this lane; exact below kMany, and not below it otherwise)
    x[i] = add(before, inc[i] < kMany ? inc[i] - x[i] : kMany);
    carry[i] = all;
  }
  __syncthreads();
}

// How sets of rows x keys are cut.
struct Cut {
  int tiles, pieces, keys;   // keys per piece
  bool few;
};
__device__ __forceinline__ Cut cut(int rows, int keys, int few_keys, int tile_keys) {
  Cut c;
  c.few = rows <= kFew;
  c.tiles = c.few ? 1 : (rows + kTile - 1) / kTile;
  const uint32_t last = keys - 1;                        // keys >= 1
  const uint32_t n = last / (uint32_t)(c.few ? few_keys : tile_keys) + 1;
  const uint32_t step = c.few ? kFewStep : kTileStep;
  c.keys = (int)((last / n + step) & -step);
  c.pieces = (int)(last / (uint32_t)c.keys + 1);         // <= n
  return c;
}
static_assert(pow2(kFewStep) && pow2(kTileStep), "");

struct Set {
  int32_t tok, rows, req, lo, hi, part, gathered;
  Cut c;
  int32_t base, items;       // first item, items that the list has room for
};

__device__ __forceinline__ void emit(const PlanArgs& a, const Set& x, int j, int tile,
                                     int piece) {
  Item it;
  it.tok = x.tok;
  it.row = tile * kTile;
  it.rows = min(x.rows - it.row, kTile);                 // none if the set did not fit
  it.req = x.req;
  it.lo = x.lo + piece * x.c.keys;
  it.hi = min(x.hi, it.lo + x.c.keys);
  it.part = x.part < 0 ? -1 : x.part + piece * x.rows + it.row;
  it.gathered = x.gathered;
  (x.c.few ? a.few : a.tile)[x.base + j] = it;
}

// One work group.  Passes over the requests: what is known of each; the members of
// the groups and their tokens in group order; the work of each kind, which sets the
// keys per piece; the items (a scan gives each set its place; its thread writes up
// to kOwn items, a wavefront a set's where there are more).  Sums of whole numbers
// only, or of as many in 64-bit floats, which hold them: no order changes them.
//
// Few items are cut into pieces of work / (kFewTarget / kv_heads) keys, at least
// kMinFew: at 4096 work groups, five rounds over the chip, the last round's idle
// ones cost little (64 requests x 32 heads x 512..4096 keys: 402 us at 768, 392 at
// 2048, 380 at 4096), and pieces of less than 512 keys pay more for their start and
// their partials than they gain (one request of 30011 keys on 8 heads, both
// kernels: 32 us at 256, 28 at 512).  Sets of at most half of that come last, so that
// what is begun last is short (256 requests of 33..543 keys on 8 heads: 67 us in the
// requests' order, 63 so; 180 of 9..708 on 40: 230 and 223).
// Tile items: the number of pieces changes how many rounds the chip's kTileSlots
// work groups (two per compute unit, at a head dimension of 128; at 64 three fit, for
// which the rounds are then counted too many) take, so several cuts are tried, a
// wavefront each, and the one whose rounds x (longest piece + kTileStart) is least is
// taken (256 requests in 6 groups x 64 heads over 8, prefixes of 4000 keys: 608 work
// groups, two rounds, 81 us; 456, one, 64; the tile items alone, with weights of one
// value).  kTileStart is what a piece costs beside its keys, most of it the writing and
// reading of its partials.
//
// Once a step and bound by latency: dependent loads, barriers, and code that is
// fetched for the first time.
constexpr int kMinFew = 512, kMinTile = 256;
constexpr int kTileSlots = 512, kTileStart = 512;
constexpr int kTries = kWaves;
__constant__ const int kTry[kTries] = {256, 320, 384, 448, 512, 640, 768, 1024};
static_assert(kTileTarget == 1024, "the finest cut tried bounds the items");
constexpr int kOwn = 8;
// Tile items are listed by the length of their keys, in quarters of the longest's, the
// longest first: a long one that is begun last is waited for.  (Where one round takes
// all, their order is none, and nothing is spent on it.  A step of several rounds pays
// 1.3 us for a pass and a scan more; 20 requests of 1..128 tokens over 380..640 keys, 16
// heads: a layer's attention 36.9 us for 40.5.)
constexpr int kClasses = 4;
__device__ __forceinline__ int class_of(int keys, int longest) {
  const int64_t k = 4 * (int64_t)keys;
  return k > 3 * (int64_t)longest ? 0 : k > 2 * (int64_t)longest ? 1 : k > longest ? 2 : 3;
}

// Keys per piece so that work is cut into target / kv_heads pieces.  (Both are whole
// numbers below 2^53 and the result, where it is not cut off, below 2^30: the
// division in 64-bit floats rounds to a whole number only where it is one.)
__device__ __forceinline__ int per_piece(double work, int target, int kv_heads, int least,
                                         int step) {
  const int t = (target + kv_heads - 1) / kv_heads;
  const double c = min(max(ceil(work / t), (double)least), (double)PLORA_PAGED_MAX_KEYS);
  return min(((int)c + step - 1) & -step, PLORA_PAGED_MAX_KEYS);
}

__global__ __launch_bounds__(kNT) void attn_plan_kernel(PlanArgs a) {
  __shared__ int32_t s_kept[kKeptArrays * (kHere + 1)];
  __shared__ Set s_sets[kNT];
  __shared__ int s_keys[kNT], s_tiles[kNT], s_big[kNT], s_bigs, s_left;
  __shared__ uint32_t red1[kWaves][1], red4[kWaves][4];
  __shared__ double s_work[kWaves][2];
  __shared__ int64_t s_cost[kTries];
  __shared__ int s_per[kTries], s_long[kTries];  // (longest piece; 0: one round takes all)
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  Kept y;
  {
    int32_t* p = a.batch <= kHere ? s_kept : a.kept;
    const int n = a.batch <= kHere ? kHere + 1 : a.batch + 1;
    y = Kept{p, p + n, p + 2 * n, p + 3 * n, p + 4 * n, p + 5 * n, p + 6 * n,
             p + 7 * n, p + 8 * n, p + 9 * n, p + 10 * n, p + 11 * n};
  }
  int n_seg = 0, n_valid = 0, b0 = -1, left = 0;
  if (tid == 0) s_left = 0;
  if (a.shared) {
    n_seg = min(max(a.meta[0], 0), a.cap);
    n_valid = min(max(a.meta[1], 0), a.batch);
    if (tid < a.batch) b0 = a.perm[tid];
  }
  for (int b = tid; b < a.batch; b += kNT) {
    const int q0 = a.q_start[b], q1 = a.q_start[b + 1], kv = a.kv_len[b];
    int n = 0;
    if (q0 >= 0 && q0 < q1 && q1 <= a.T && a.req[q0] == b) n = q1 - q0;
    const bool fits = n <= a.max_q && kv >= n && kv <= a.max_keys;
    left += n > 0 && !fits;
    y.n[b] = fits ? n : 0;
    y.q0[b] = q0;
    y.kv[b] = kv;
    y.u[b] = 0;
  }
  if (a.shared) {
    for (int i = tid; i <= n_seg; i += kNT) {
      const int g = i < n_seg ? a.seg_id[i] : -1;
      y.begin[i] = min(max(a.seg_ptr[i], 0), n_valid);
      // the whole pages of the prefix
      int64_t u = 0;
      if (g >= 0 && g < a.n_groups) u = min((int64_t)a.prefix_len[g], a.max_keys);
      y.pre[i] = u <= 0 ? 0 : (int)(u & -(int64_t)a.page_size);
      y.part[i] = 0;
      y.req[i] = INT32_MAX;
    }
    __syncthreads();
    // who could share
    for (int p = tid; p < n_valid; p += kNT) {
      const int b = p == tid ? b0 : a.perm[p];
      if (b < 0 || b >= a.batch || n_seg == 0) continue;
      int s = 0, z = n_seg;                              // the segment that holds p
      while (z - s > 1) {
        const int mid = (s + z) >> 1;
        if (y.begin[mid] <= p) s = mid;
        else z = mid;
      }
      const int n = y.n[b], u = y.pre[s];
      y.seg[b] = s;
      if (n > 0 && u > 0 && (int64_t)n * a.r <= PLORA_ATTN_SHARE_ROWS && y.kv[b] - n >= u) {
        y.u[b] = u;
        atomicAdd(&y.part[s], 1);
        atomicMin(&y.req[s], b);
      }
    }
    __syncthreads();
    // members: not alone in their group; their tokens in group order
    uint32_t carry[1] = {0};
    for (int p0 = 0; p0 < n_valid; p0 += kNT) {
      const int p = p0 + tid;
      int b = p >= n_valid ? -1 : p == tid ? b0 : a.perm[p], n = 0;
      if (b < 0 || b >= a.batch) b = -1;
      if (b >= 0 && y.u[b] > 0) {
        if (y.part[y.seg[b]] >= 2) n = y.n[b];
        else y.u[b] = 0;
      }
      uint32_t at[1] = {(uint32_t)n};
      scan(at, carry, red1);
      if (p < n_valid) y.moff[p] = at[0];
      if (n > 0) {
        y.place[b] = at[0];
        for (int j = 0; j < n && (int)at[0] + j < a.T; ++j) a.order[at[0] + j] = y.q0[b] + j;
      }
    }
    if (tid == 0) y.moff[n_valid] = carry[0];
  }
  __syncthreads();
  // the sets: the groups' prefixes, then the requests' own keys
  const int n_sets = n_seg + a.batch;
  const auto members = [&](int s, int& tok) {            // a group's tokens
    tok = y.moff[y.begin[s]];
    return y.moff[y.begin[s + 1]] - tok;
  };
  const auto set_of = [&](int i, int& rows, int& keys) {
    int64_t n;
    int tok;
    if (i < n_seg) {
      n = members(i, tok);
      keys = y.pre[i];
    } else {
      n = y.n[i - n_seg];
      keys = y.kv[i - n_seg] - y.u[i - n_seg];
    }
    n *= a.r;
    rows = n > 0 && n <= INT32_MAX && keys > 0 ? (int)n : 0;
  };
  // work of each kind, in tiles x keys
  double few_work = 0, tile_work = 0;
  for (int i = tid; i < n_sets; i += kNT) {
    int rows, keys;
    set_of(i, rows, keys);
    if (rows > kFew) tile_work += (double)((rows + kTile - 1) / kTile) * keys;
    else if (rows > 0) few_work += keys;
  }
  few_work = wave_scan(few_work, Add{});
  tile_work = wave_scan(tile_work, Add{});
  if (lane == 63) s_work[wv][0] = few_work, s_work[wv][1] = tile_work;
  __syncthreads();
  few_work = tile_work = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) few_work += s_work[w][0], tile_work += s_work[w][1];
  const int few_keys = per_piece(few_work, kFewTarget, a.kv_heads, kMinFew, kFewStep);
  int tile_keys = PLORA_PAGED_MAX_KEYS;
  // several rounds of tile items: the longest piece, and where this thread's next item of
  // each class goes
  int longest_tile = 0;
  uint32_t next[kClasses] = {};
  if (tile_work > 0) {
    const int per = per_piece(tile_work, kTry[wv], a.kv_heads, kMinTile, kTileStep);
    int64_t items = 0;
    int longest = 0;
    for (int i0 = 0; i0 < n_sets; i0 += kNT) {
      const int m = min(kNT, n_sets - i0);
      int rows = 0, keys = 0;
      if (tid < m) set_of(i0 + tid, rows, keys);
      s_tiles[tid] = rows > kFew ? (rows + kTile - 1) / kTile : 0;
      s_keys[tid] = keys;
      __syncthreads();
      for (int j = lane; j < m; j += 64) {
        const int t = s_tiles[j];
        if (t == 0) continue;
        const Cut c = cut(kTile, s_keys[j], 1, per);
        items += (int64_t)t * c.pieces;
        longest = max(longest, c.keys);
      }
      __syncthreads();
    }
    items = wave_scan(items, Add{});
    longest = wave_scan(longest, Max{});
    if (lane == 63) {
      s_cost[wv] = (items * a.kv_heads + kTileSlots - 1) / kTileSlots * (longest + kTileStart);
      s_per[wv] = per;
      s_long[wv] = items * a.kv_heads > kTileSlots ? longest : 0;
    }
    __syncthreads();
    int64_t least = INT64_MAX;
#pragma unroll
    for (int k = 0; k < kTries; ++k)
      if (s_cost[k] < least) least = s_cost[k], tile_keys = s_per[k], longest_tile = s_long[k];
    if (longest_tile > 0) {
      for (int i = tid; i < n_sets; i += kNT) {
        int rows, keys;
        set_of(i, rows, keys);
        if (rows <= kFew) continue;
        const Cut c = cut(rows, keys, 1, tile_keys);
        const uint32_t z = (uint32_t)min((int64_t)c.tiles * c.pieces, (int64_t)kMany);
        const int k = class_of(c.keys, longest_tile);
#pragma unroll
        for (int j = 0; j < kClasses; ++j) next[j] = k == j ? AddCount{}(next[j], z) : next[j];
      }
      uint32_t all[kClasses] = {}, at = 0;
      scan(next, all, red4);
#pragma unroll
      for (int j = 0; j < kClasses; ++j) {
        next[j] = AddCount{}(at, next[j]);
        at = AddCount{}(at, all[j]);
      }
    }
  }
  // items
  uint32_t sum[4] = {0, 0, 0, 0};                        // few, tiles, rows of partials, later
  for (int i0 = 0; i0 < n_sets; i0 += kNT) {
    const int i = i0 + tid, b = i - n_seg;
    const bool own = i < n_sets && b >= 0;
    Set x{};
    x.req = -1;
    int u = 0, rows, keys;
    if (tid == 0) s_bigs = 0;
    if (i < n_sets) {
      set_of(i, rows, keys);
      x.rows = rows;
    }
    if (own) {
      u = y.u[b];
      x.tok = y.q0[b];
      x.req = b;
      x.lo = u;
      x.hi = y.kv[b];
    } else if (i < n_sets) {
      members(i, x.tok);
      x.hi = y.pre[i];
      x.gathered = 1;
      x.req = y.req[i];
    }
    int64_t items = 0, part = 0;
    if (x.rows > 0) {
      x.c = cut(x.rows, x.hi - x.lo, few_keys, tile_keys);
      items = (int64_t)x.c.tiles * x.c.pieces;
      if (!own || u > 0 || x.c.pieces > 1) part = (int64_t)x.rows * x.c.pieces;
    }
    const bool later = x.rows > 0 && x.c.few && x.c.pieces == 1 && x.c.keys <= few_keys / 2;
    uint32_t at[4] = {(uint32_t)min(x.c.few && !later ? items : 0, (int64_t)kMany),
                      (uint32_t)min(x.c.few ? 0 : items, (int64_t)kMany),
                      (uint32_t)min(part, (int64_t)kMany), later};
    const uint32_t tiles = at[1];
    scan(at, sum, red4);
    if (longest_tile > 0 && tiles > 0) {
      const int k = class_of(x.c.keys, longest_tile);
#pragma unroll
      for (int j = 0; j < kClasses; ++j)
        if (k == j) at[1] = next[j], next[j] = AddCount{}(next[j], tiles);
    }
    x.base = later ? a.few_cap - 1 - (int)at[3] : x.c.few ? at[0] : at[1];
    x.part = part > 0 ? (int)at[2] : -1;
    // (never past the caps for lengths that agree with the shape)
    const int cap = x.c.few ? a.few_cap : a.tile_cap;
    if (x.base < 0 || x.base + items > cap || at[2] + part > a.part_cap) x.rows = 0;
    x.items = x.base < 0 ? 0 : (int)min(items, (int64_t)max(cap - x.base, 0));
    if (i < n_seg) {
      y.part[i] = x.rows > 0 ? x.part : -1;
      y.splits[i] = x.c.pieces;
    }
    if (x.items > kOwn) {
      s_sets[tid] = x;
      s_big[atomicAdd(&s_bigs, 1)] = tid;
    } else {
      int tile = x.c.tiles - 1, piece = 0;
      for (int j = 0; j < x.items; ++j) {
        emit(a, x, j, tile, piece);
        if (++piece == x.c.pieces) piece = 0, --tile;
      }
    }
    __syncthreads();
    if (own) {
      ReqInfo f{};
      f.part = x.part;
      f.splits = x.c.pieces;
      f.rows = x.rows;
      f.pre_part = -1;
      f.state = x.rows == 0 ? 0 : x.part < 0 ? 2 : 1;
      if (u > 0 && x.rows > 0) {
        const int s = y.seg[b];
        int tok;
        f.pre_rows = members(s, tok) * a.r;
        f.pre_part = y.part[s];
        f.pre_splits = y.splits[s];
        f.pre_row = (y.place[b] - tok) * a.r;
        if (f.pre_part < 0) f.state = 0;
      }
      left += y.n[b] > 0 && f.state == 0;
      a.info[b] = f;
    }
    const int bigs = s_bigs;
    for (int k = wv; k < bigs; k += kWaves) {
      const Set& z = s_sets[s_big[k]];
      // the last rows, which see the most keys, first
      for (int j = lane; j < z.items; j += 64)
        emit(a, z, j, z.c.tiles - 1 - j / z.c.pieces, j % z.c.pieces);
    }
    __syncthreads();
  }
  if (left > 0) atomicAdd(&s_left, left);
  __syncthreads();
  if (tid == 0) {
    PlanHeader h{};
    h.left = s_left;
    h.few = min((int)sum[0], a.few_cap);
    h.later = min((int)sum[3], a.few_cap - h.few);
    h.tiles = min((int)sum[1], a.tile_cap);
    h.part_rows = min((int)sum[2], a.part_cap);
    h.few_keys = few_keys;
    h.tile_keys = tile_keys;
    *a.head = h;
  }
}

}  // namespace
}  // namespace paged

extern "C" size_t plora_attn_plan_bytes(const plora_attn_shape* shape) {
  using namespace paged;
  if (!shape || !shape_ok(*shape) || shape_empty(*shape)) return 0;
  return plan_layout(*shape, bounds(*shape)).bytes;
}

extern "C" plora_status plora_attn_plan(const plora_kv_step* step, const plora_attn_shape* shape,
                                        const plora_segments* seg, const int32_t* prefix_len,
                                        int32_t n_groups, void* plan, size_t plan_bytes,
                                        hipStream_t stream) {
  using namespace paged;
  if (!step || !shape || step->batch != shape->batch || step->T != shape->T || n_groups < 0 ||
      step->max_pages < 0 || (seg && !shape->shared) || (seg && seg->T != shape->batch))
    return PLORA_ERR_INVALID_ARG;
  if (shape->batch < 0 || shape->T < 0 || shape->heads < 0 || shape->kv_heads < 0 ||
      shape->max_q < 0)
    return PLORA_ERR_INVALID_ARG;
  if (!shape_ok(*shape) || !page_size_ok(step->page_size)) return PLORA_ERR_UNSUPPORTED;
  if (shape_empty(*shape)) return PLORA_OK;
  if (!step->q_start || !step->kv_len || !step->req || !plan) return PLORA_ERR_INVALID_ARG;
  if (seg && ((n_groups > 0 && !prefix_len) || !seg->perm || !seg->seg_ptr || !seg->seg_id || !seg->meta ||
              seg->cap != std::min(seg->T, n_groups)))
    return PLORA_ERR_INVALID_ARG;
  if (!aligned(plan, 16)) return PLORA_ERR_UNSUPPORTED;
  const Bounds b = bounds(*shape);
  const PlanLayout l = plan_layout(*shape, b);
  if (plan_bytes < l.bytes) return PLORA_ERR_WORKSPACE_TOO_SMALL;
  char* base = static_cast<char*>(plan);
  PlanArgs a{};
  a.batch = shape->batch;
  a.T = shape->T;
  a.r = b.r;
  a.kv_heads = shape->kv_heads;
  a.max_q = shape->max_q;
  a.page_size = step->page_size;
  a.max_keys = std::min((int64_t)step->max_pages * step->page_size,
                        (int64_t)PLORA_PAGED_MAX_KEYS);
  a.q_start = step->q_start;
  a.kv_len = step->kv_len;
  a.req = step->req;
  a.head = reinterpret_cast<PlanHeader*>(base);
  a.few = reinterpret_cast<Item*>(base + l.few);
  a.tile = reinterpret_cast<Item*>(base + l.tile);
  a.order = reinterpret_cast<int32_t*>(base + l.order);
  a.info = reinterpret_cast<ReqInfo*>(base + l.req);
  a.few_cap = b.few_cap;
  a.tile_cap = b.tile_cap;
  a.part_cap = (int32_t)b.part_rows;
  a.kept = reinterpret_cast<int32_t*>(base + l.kept);
  if (seg && n_groups > 0) {
    a.shared = 1;
    a.n_groups = n_groups;
    a.cap = seg->cap;
    a.perm = seg->perm;
    a.seg_ptr = seg->seg_ptr;
    a.seg_id = seg->seg_id;
    a.meta = seg->meta;
    a.prefix_len = prefix_len;
  }
  clear_error();
  hipLaunchKernelGGL(attn_plan_kernel, dim3(1), dim3(kNT), 0, stream, a);
  return launch_status();
}

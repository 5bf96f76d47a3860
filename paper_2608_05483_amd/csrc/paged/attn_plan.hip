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
  int32_t *u_len, *place, *seg_of, *moff, *seg_part;   // [batch + 1] each, groups only
  int32_t few_cap, tile_cap;
  int64_t part_cap;
};

// Exclusive scan of one value a thread over the work group; total is the sum.
__device__ __forceinline__ int64_t scan(int64_t x, int64_t* red, int64_t& total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int64_t inc = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(inc, d, 64);
    if (lane >= d) inc += y;
  }
  if (lane == 63) red[wv] = inc;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wv) before += red[w];
    all += red[w];
  }
  __syncthreads();
  total = all;
  return before + inc - x;
}

// A request's new tokens, 0 if it has none or the step left it out.
__device__ __forceinline__ int tokens(const PlanArgs& a, int b, int& q0, int& kv) {
  q0 = a.q_start[b];
  kv = a.kv_len[b];
  const int q1 = a.q_start[b + 1];
  if (q0 < 0 || q0 >= q1 || q1 > a.T || a.req[q0] != b) return 0;
  const int n = q1 - q0;
  return n > a.max_q || kv < n || kv > a.max_keys ? 0 : n;
}

// The whole pages of a group's prefix, in keys.
__device__ __forceinline__ int prefix(const PlanArgs& a, int seg) {
  const int g = a.seg_id[seg];
  if (g < 0 || g >= a.n_groups) return 0;
  const int64_t u = min((int64_t)a.prefix_len[g], a.max_keys);
  return u <= 0 ? 0 : (int)(u & -(int64_t)a.page_size);
}

// How sets of rows x keys are cut.
struct Rule {
  int few_keys, tile_keys;   // most keys per piece
};
struct Cut {
  int tiles, pieces, keys;   // keys per piece
  bool few;
};
__device__ __forceinline__ Cut cut(int rows, int keys, const Rule& r) {
  Cut c;
  c.few = rows <= kFew;
  c.tiles = c.few ? 1 : (rows + kTile - 1) / kTile;
  const int most = c.few ? r.few_keys : r.tile_keys, step = c.few ? kFewStep : kTileStep;
  const int n = (keys - 1) / most + 1;                   // keys >= 1
  c.keys = ((keys - 1) / n + 1 + step - 1) / step * step;
  c.pieces = (keys - 1) / c.keys + 1;                    // <= n
  return c;
}

// First place of a segment in perm.
__device__ __forceinline__ int seg_begin(const PlanArgs& a, int s, int n_valid) {
  return min(max(a.seg_ptr[s], 0), n_valid);
}

struct Set {
  int32_t tok, rows, req, lo, hi, part, gathered;
  Cut c;
  int64_t base;              // first item
};

// One work group.  Passes over the requests: the members of the groups and their
// tokens in group order; the work of each kind, which sets the keys per piece;
// the items (scans give each set its place, then a wavefront a set writes them).
// Integer sums only, in a fixed order (the counts of members are sums by atomics,
// whose order does not matter).
//
// Few items are cut into pieces of work / (kFewTarget / kv_heads) keys, at least
// kMinFew: at 4096 work groups, five rounds over the chip, the last round's idle
// ones cost little (64 requests x 32 heads x 512..4096 keys: 402 us at 768, 392 at
// 2048, 380 at 4096), and pieces of less than 512 keys pay more for their start and
// their partials than they gain (one request of 30011 keys on 8 heads, both
// kernels: 42 us at 256, 33 at 512).
// Tile items: the number of pieces changes how many rounds the chip's kTileSlots
// work groups (two per compute unit) take, so several cuts are tried and the one
// whose rounds x (longest piece + kTileStart) is least is taken (256 requests in 6
// groups x 64 heads over 8, prefixes of 4000 keys: 608 work groups, two rounds, 81
// us; 456, one, 64; the tile items alone).
// Once a step and bound by latency: its dependent loads and its scans.
constexpr int kMinFew = 512, kMinTile = 256;
constexpr int kTileSlots = 512, kTileStart = 128;
constexpr int kTries = 8;
__constant__ const int kTry[kTries] = {256, 320, 384, 448, 512, 640, 768, 1024};
static_assert(kTileTarget == 1024, "the finest cut tried bounds the items");

__global__ __launch_bounds__(kNT) void attn_plan_kernel(PlanArgs a) {
  __shared__ int64_t red[kWaves];
  __shared__ Set sets[kNT];
  __shared__ Rule s_rule;
  __shared__ int64_t s_items[kTries][kWaves];
  __shared__ int s_longest[kTries][kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  int n_seg = 0, n_valid = 0;
  int64_t total;
  if (a.shared) {
    n_seg = min(max(a.meta[0], 0), a.cap);
    n_valid = min(max(a.meta[1], 0), a.batch);
    for (int i = tid; i <= a.batch; i += kNT) a.u_len[i] = 0, a.seg_part[i] = 0;
    __syncthreads();
    // who could share
    for (int p = tid; p < n_valid; p += kNT) {
      const int b = a.perm[p];
      if (b < 0 || b >= a.batch) continue;
      int s = 0, z = n_seg;                              // the segment that holds p
      while (z - s > 1) {
        const int mid = (s + z) >> 1;
        if (a.seg_ptr[mid] <= p) s = mid;
        else z = mid;
      }
      int q0, kv;
      const int n = tokens(a, b, q0, kv), u = n_seg > 0 ? prefix(a, s) : 0;
      a.seg_of[b] = s;
      if (n > 0 && u > 0 && (int64_t)n * a.r <= PLORA_ATTN_SHARE_ROWS && kv - n >= u) {
        a.u_len[b] = u;
        atomicAdd(&a.seg_part[s], 1);
      }
    }
    __syncthreads();
    // members: not alone in their group; their tokens in group order
    int64_t carry = 0;
    for (int p0 = 0; p0 < n_valid; p0 += kNT) {
      const int p = p0 + tid;
      int b = p < n_valid ? a.perm[p] : -1, q0 = 0, kv, n = 0;
      if (b < 0 || b >= a.batch) b = -1;
      if (b >= 0 && a.u_len[b] > 0) {
        if (a.seg_part[a.seg_of[b]] >= 2) n = tokens(a, b, q0, kv);
        else a.u_len[b] = 0;
      }
      const int64_t at = carry + scan(n, red, total);
      carry += total;
      if (p < n_valid) a.moff[p] = (int)at;
      if (n > 0) {
        a.place[b] = (int)at;
        for (int j = 0; j < n; ++j)
          if (at + j < a.T) a.order[at + j] = q0 + j;
      }
    }
    if (tid == 0) a.moff[n_valid] = (int)carry;
    __syncthreads();
  }
  // a set's rows and keys: the groups' prefixes, then the requests' own
  const auto set_of = [&](int i, int& rows, int& keys) {
    int64_t n;
    if (i < n_seg) {
      n = a.moff[seg_begin(a, i + 1, n_valid)] - a.moff[seg_begin(a, i, n_valid)];
      keys = prefix(a, i);
    } else {
      int q0, kv;
      n = tokens(a, i - n_seg, q0, kv);
      keys = kv - (a.shared ? a.u_len[i - n_seg] : 0);
    }
    n *= a.r;
    rows = n > 0 && n <= INT32_MAX && keys > 0 ? (int)n : 0;
  };
  const int n_sets = n_seg + a.batch;
  // work of each kind, in tiles x keys
  int64_t few_work = 0, tile_work = 0;
  for (int i = tid; i < n_sets; i += kNT) {
    int rows, keys;
    set_of(i, rows, keys);
    if (rows == 0) continue;
    if (rows > kFew) tile_work += (int64_t)((rows + kTile - 1) / kTile) * keys;
    else few_work += keys;
  }
  int64_t all_few, all_tile;
  scan(few_work, red, all_few);
  scan(tile_work, red, all_tile);
  const auto per_piece = [&](int64_t work, int target, int least, int step) {
    const int64_t t = (target + a.kv_heads - 1) / a.kv_heads;
    const int64_t c = max((work + t - 1) / t, (int64_t)least);
    return (int)min((c + step - 1) / step * step, (int64_t)PLORA_PAGED_MAX_KEYS);
  };
  Rule rule;
  rule.few_keys = per_piece(all_few, kFewTarget, kMinFew, kFewStep);
  rule.tile_keys = PLORA_PAGED_MAX_KEYS;
  if (all_tile > 0) {
    int64_t items[kTries] = {};
    int longest[kTries] = {}, per[kTries];
#pragma unroll
    for (int k = 0; k < kTries; ++k) per[k] = per_piece(all_tile, kTry[k], kMinTile, kTileStep);
    for (int i = tid; i < n_sets; i += kNT) {
      int rows, keys;
      set_of(i, rows, keys);
      if (rows <= kFew) continue;
#pragma unroll
      for (int k = 0; k < kTries; ++k) {
        const Cut c = cut(rows, keys, Rule{1, per[k]});
        items[k] += (int64_t)c.tiles * c.pieces;
        longest[k] = max(longest[k], c.keys);
      }
    }
#pragma unroll
    for (int k = 0; k < kTries; ++k) {
      for (int d = 32; d; d >>= 1) {
        items[k] += __shfl_xor(items[k], d, 64);
        longest[k] = max(longest[k], __shfl_xor(longest[k], d, 64));
      }
      if (lane == 0) s_items[k][wv] = items[k], s_longest[k][wv] = longest[k];
    }
    __syncthreads();
    if (tid == 0) {
      int64_t least = INT64_MAX;
#pragma unroll
      for (int k = 0; k < kTries; ++k) {
        int64_t n = 0;
        int len = 0;
        for (int w = 0; w < kWaves; ++w) n += s_items[k][w], len = max(len, s_longest[k][w]);
        const int64_t cost = (n * a.kv_heads + kTileSlots - 1) / kTileSlots * (len + kTileStart);
        if (cost < least) least = cost, rule.tile_keys = per[k];
      }
    }
  }
  if (tid == 0) s_rule = rule;
  __syncthreads();
  rule = s_rule;
  // items: the groups' prefixes first, then the requests' own keys
  int64_t few_n = 0, tile_n = 0, part_n = 0;
  for (int pass = a.shared ? 0 : 1; pass < 2; ++pass) {
    const int count = pass == 0 ? n_seg : a.batch;
    for (int i0 = 0; i0 < count; i0 += kNT) {
      const int i = i0 + tid, m = min(kNT, count - i0);
      Set x{};
      x.req = -1;
      int64_t rows = 0;
      int u = 0;
      if (i < count && pass == 0) {
        const int p0 = seg_begin(a, i, n_valid), p1 = seg_begin(a, i + 1, n_valid);
        x.tok = a.moff[p0];
        rows = (int64_t)(a.moff[p1] - x.tok) * a.r;
        x.hi = prefix(a, i);
        x.gathered = 1;
        if (rows > 0) x.req = a.req[a.order[min(x.tok, a.T - 1)]];
      } else if (i < count) {
        int q0, kv;
        const int n = tokens(a, i, q0, kv);
        u = a.shared ? a.u_len[i] : 0;
        rows = (int64_t)n * a.r;
        x.tok = q0;
        x.req = i;
        x.lo = u;
        x.hi = kv;
      }
      if (rows <= 0 || rows > INT32_MAX || x.hi <= x.lo) rows = 0;
      x.rows = (int)rows;
      int64_t items = 0, part = 0;
      if (rows > 0) {
        x.c = cut(x.rows, x.hi - x.lo, rule);
        items = (int64_t)x.c.tiles * x.c.pieces;
        part = pass == 0 || u > 0 || x.c.pieces > 1 ? rows * x.c.pieces : 0;
      }
      int64_t few_total, tile_total, part_total;
      const int64_t fb = few_n + scan(x.c.few ? items : 0, red, few_total);
      const int64_t tb = tile_n + scan(x.c.few ? 0 : items, red, tile_total);
      const int64_t pb = part_n + scan(part, red, part_total);
      x.base = x.c.few ? fb : tb;
      // (never past the caps for lengths that agree with the shape)
      const int64_t cap = x.c.few ? a.few_cap : a.tile_cap;
      if (x.base + items > cap || pb + part > a.part_cap) x.rows = 0;
      x.part = part > 0 ? (int)pb : -1;
      if (i < count && pass == 0) a.seg_part[i] = x.rows > 0 ? x.part : -1;
      if (i < count && pass == 1) {
        ReqInfo f{};
        f.part = x.part;
        f.splits = x.c.pieces;
        f.rows = x.rows;
        f.pre_part = -1;
        f.state = x.rows == 0 ? 0 : x.part < 0 ? 2 : 1;
        if (u > 0 && x.rows > 0) {
          const int s = a.seg_of[i], t0 = a.moff[seg_begin(a, s, n_valid)];
          const int all = (a.moff[seg_begin(a, s + 1, n_valid)] - t0) * a.r;
          f.pre_part = a.seg_part[s];
          f.pre_rows = all;
          f.pre_splits = cut(all, u, rule).pieces;
          f.pre_row = (a.place[i] - t0) * a.r;
          if (f.pre_part < 0) f.state = 0;
        }
        a.info[i] = f;
      }
      sets[tid] = x;
      __syncthreads();
      for (int k = wv; k < m; k += kWaves) {
        const Set& y = sets[k];
        Item* list = y.c.few ? a.few : a.tile;
        const int64_t cap = y.c.few ? a.few_cap : a.tile_cap;
        const int64_t items = min((int64_t)y.c.tiles * y.c.pieces, cap - y.base);
        for (int j = lane; j < items; j += 64) {
          // the last rows, which see the most keys, first
          const int tile = y.c.tiles - 1 - j / y.c.pieces, piece = j % y.c.pieces;
          Item it;
          it.tok = y.tok;
          it.row = tile * kTile;
          it.rows = min(y.rows - it.row, kTile);      // none if the set did not fit
          it.req = y.req;
          it.lo = y.lo + piece * y.c.keys;
          it.hi = min(y.hi, it.lo + y.c.keys);
          it.part = y.part < 0 ? -1 : y.part + piece * y.rows + it.row;
          it.gathered = y.gathered;
          list[y.base + j] = it;
        }
      }
      __syncthreads();
      few_n += few_total;
      tile_n += tile_total;
      part_n += part_total;
    }
  }
  if (tid == 0) {
    PlanHeader h{};
    h.few = (int)min(few_n, (int64_t)a.few_cap);
    h.tiles = (int)min(tile_n, (int64_t)a.tile_cap);
    h.part_rows = (int)min(part_n, a.part_cap);
    h.few_keys = rule.few_keys;
    h.tile_keys = rule.tile_keys;
    // rounded up: all tiles have come by the last work group, at most one an eight
    const uint64_t few8 = ((uint64_t)h.few * a.kv_heads + 7) / 8;
    const uint64_t tile8 = ((uint64_t)h.tiles * a.kv_heads + 7) / 8;
    h.tile_rate = tile8 ? ((tile8 << 32) + few8 + tile8 - 1) / (few8 + tile8) : 0;
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
  if (seg && (!prefix_len || !seg->perm || !seg->seg_ptr || !seg->seg_id || !seg->meta ||
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
  a.part_cap = b.part_rows;
  if (seg && n_groups > 0) {
    a.shared = 1;
    a.n_groups = n_groups;
    a.cap = seg->cap;
    a.perm = seg->perm;
    a.seg_ptr = seg->seg_ptr;
    a.seg_id = seg->seg_id;
    a.meta = seg->meta;
    a.prefix_len = prefix_len;
    int32_t* s = reinterpret_cast<int32_t*>(base + l.scratch);
    const int32_t n = shape->batch + 1;
    a.u_len = s;
    a.place = s + n;
    a.seg_of = s + 2 * n;
    a.moff = s + 3 * n;
    a.seg_part = s + 4 * n;
  }
  clear_error();
  hipLaunchKernelGGL(attn_plan_kernel, dim3(1), dim3(kNT), 0, stream, a);
  return launch_status();
}

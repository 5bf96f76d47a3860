// Upkeep of a paged cache (include/plora_pages.h): plora_kv_remap, plora_kv_copy,
// plora_kv_compact.

#include <algorithm>

#include "paged_dev.h"
#include "plora_pages.h"

namespace paged {
namespace {

constexpr int kNT = 256;

struct RemapArgs {
  const int32_t *old_table, *old_len, *src, *keep, *free_head;
  int32_t *new_table, *new_len, *shares, *free_pages, *free_next, *copies, *meta;
  int32_t old_batch, new_batch, old_max, new_max, log_page, n_pages, n_free;
  // workspace: a new request's partly filled page (-1: none), and the entries that an
  // old one drops; scratch: for such pages who holds them so (how many, the last)
  int32_t* part;
  int2 *drop, *last;
};

__device__ __forceinline__ int old_length(const RemapArgs& a, int b) {
  return (int)min((int64_t)max(a.old_len[b], 0), (int64_t)a.old_max << a.log_page);
}
// Keys that new request i holds.
__device__ __forceinline__ int new_length(const RemapArgs& a, int i, int b) {
  if (b < 0 || b >= a.old_batch) return 0;
  int n = old_length(a, b);
  if (a.keep) n = min(n, max(a.keep[i], 0));
  return (int)min((int64_t)n, (int64_t)a.new_max << a.log_page);
}
__device__ __forceinline__ int pages_of(const RemapArgs& a, int keys) {
  return (keys + (1 << a.log_page) - 1) >> a.log_page;
}
__device__ __forceinline__ bool in_pool(const RemapArgs& a, int page) {
  return page >= 0 && page < a.n_pages;
}
__device__ __forceinline__ int now(const int32_t* p) {
  return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The lowest of a team's values: a wavefront's, or (red) a work group's of kNT threads.
template <int NT>
__device__ __forceinline__ int lowest(int x, int* red) {
#pragma unroll
  for (int d = 32; d; d >>= 1) x = min(x, __shfl_xor(x, d, 64));
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = x;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) x = min(x, red[w]);
  }
  return x;
}

// New request i, or old request i - new_batch, by a team of NT threads.  An old
// request's holds pass to the first new one that continues it, so only what changes is
// counted: that one's shorter tail and the pages of requests that none continues are
// dropped, the other continuations hold theirs in addition.  Sums of whole numbers, in
// any order.
template <int NT>
__device__ __forceinline__ void remap_row(const RemapArgs& a, int i, int* red) {
  const int tid = threadIdx.x % NT;
  if (i < a.new_batch) {
    const int b = a.src[i], n = new_length(a, i, b), pages = pages_of(a, n);
    if (tid == 0) {
      a.new_len[i] = n;
      if (pages == 0) a.part[i] = -1;
    }
    if (pages == 0) return;
    int first = i;
    for (int j = tid; j < i; j += NT)
      if (a.src[j] == b) first = min(first, j);
    first = lowest<NT>(first, red);
    const int32_t* from = a.old_table + (int64_t)b * a.old_max;
    int32_t* to = a.new_table + (int64_t)i * a.new_max;
    for (int j = tid; j < pages; j += NT) {
      const int page = from[j];
      const bool held = in_pool(a, page);
      to[j] = page;
      if (first < i && held) atomicAdd(&a.shares[page], 1);
      if (j == pages - 1) {
        const bool part = held && (n & ((1 << a.log_page) - 1));
        a.part[i] = part ? page : -1;
        if (part) a.last[page] = int2{0, -1};
      }
    }
  } else {
    const int b = i - a.new_batch;
    int first = a.new_batch;
    for (int j = tid; j < a.new_batch; j += NT)
      if (a.src[j] == b) first = min(first, j);
    first = lowest<NT>(first, red);
    const int kept = first < a.new_batch ? pages_of(a, new_length(a, first, b)) : 0;
    const int held = pages_of(a, old_length(a, b));
    if (tid == 0) a.drop[b] = int2{kept, held - kept};
    const int32_t* from = a.old_table + (int64_t)b * a.old_max;
    for (int j = kept + tid; j < held; j += NT) {
      const int page = from[j];
      if (in_pool(a, page)) atomicAdd(&a.shares[page], -1);
    }
  }
}

__global__ __launch_bounds__(kNT) void remap_rows_kernel(RemapArgs a) {
  __shared__ int red[kNT / 64];
  remap_row<kNT>(a, blockIdx.x, red);
}

// A dropped page that nobody holds carries the number of the lowest request that dropped
// it, as a mark below all counts.
constexpr int kMark = INT32_MIN / 2;     // (the number is added)

// An old request's dropped entries by a work group: the marks, and what of the entries
// has to be looked at again, from the first page without a holder to the last.  Of a page
// that others go on with there is no more to do: where forks of long contexts end
// together, of each only its last page or two.
__global__ __launch_bounds__(kNT) void remap_mark_kernel(RemapArgs a) {
  __shared__ int red[2][kNT / 64];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int2 d = a.drop[b];
  if (d.y == 0) return;
  const int32_t* from = a.old_table + (int64_t)b * a.old_max;
  int first = INT32_MAX, last = -1;
  for (int j = d.x + tid; j < d.x + d.y; j += kNT) {
    const int page = from[j];
    if (in_pool(a, page) && now(&a.shares[page]) < 0) {
      atomicMin(&a.shares[page], kMark + b);
      first = min(first, j);
      last = max(last, j);
    }
  }
  first = lowest<kNT>(first, red[0]);
  last = -lowest<kNT>(-last, red[1]);
  if (tid == 0) a.drop[b] = last < 0 ? int2{0, 0} : int2{first, last - first + 1};
}

constexpr int kFT = 1024;                // threads, and requests looked at together
constexpr int kFW = kFT / 64;

// Exclusive sum over the work group's threads; total is the sum of all.
__device__ __forceinline__ int block_sum(int x, int* red, int& total) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int inc = wave_scan(x, Add{});
  __syncthreads();
  if (lane == 63) red[wv] = inc;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kFW; ++w) {
    if (w < wv) before += red[w];
    total += red[w];
  }
  return before + inc - x;
}

// One work group.  The entries that old requests drop, of 1024 requests at a time: of
// those whose page nobody holds (its count is below 0) the lowest request puts its mark
// there, and the marked ones go before the list's head, from the last to the first.  Then
// the new requests' partly filled pages that others hold too: how many hold a page so and
// which is the last of them are known after one pass, so each can tell whether it has to
// take a page of its own; a scan numbers those that do.
// Bound by latency, dependent loads and barriers: what there is nothing of is left out, a
// thread asks for kEach entries in a row together, and what it has found of them, and of
// its new request, stays in registers where all fits (the usual case).
// ROWS: the requests as well, a wavefront each.  MARKED: remap_mark_kernel was before.
constexpr int kEach = 8;
constexpr int kTurn = kFT * kEach;
template <bool ROWS, bool MARKED>
__global__ __launch_bounds__(kFT) void remap_finish_kernel(RemapArgs a) {
  __shared__ int s_first[kFT], s_from[kFT];
  __shared__ int red[kFW];
  const int tid = threadIdx.x;
  const int chunks = (a.old_batch + kFT - 1) / kFT;
  const int32_t head = *a.free_head;
  if constexpr (ROWS) {
    for (int i = tid >> 6; i < a.new_batch + a.old_batch; i += kFW) remap_row<64>(a, i, nullptr);
    __syncthreads();
  }
  // (asked for beside the drops)
  const int part0 = tid < a.new_batch ? a.part[tid] : -1;
  const int n0 = tid < a.new_batch ? a.new_len[tid] : 0;
  const bool list = head >= 0 && head <= a.n_free;
  int room = list ? head : 0, freed = 0;
  // a chunk's requests: where their entries begin in order, and in their rows
  const auto open = [&](int c) {
    const int b = c * kFT + tid;
    const int2 d = b < a.old_batch ? a.drop[b] : int2{0, 0};
    int total;
    const int at = block_sum(d.y, red, total);
    s_first[tid] = at;
    s_from[tid] = d.x;
    __syncthreads();
    return total;
  };
  // this thread's entries of a turn: their requests and pages (-1: none)
  struct Entries {
    int b[kEach], page[kEach];
  } x;
  const auto get = [&](int c, int turn, int total) {
    const int e0 = turn * kTurn + tid * kEach, m = min(kFT, a.old_batch - c * kFT);
#pragma unroll
    for (int k = 0; k < kEach; ++k) x.b[k] = x.page[k] = -1;
    if (e0 >= total) return;
    int lo = 0, hi = m;
    while (hi - lo > 1) {                // the last request that starts at or before e0
      const int mid = (lo + hi) >> 1;
      if (s_first[mid] <= e0) lo = mid;
      else hi = mid;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
      if (e0 + k >= total) break;
      while (lo + 1 < m && s_first[lo + 1] <= e0 + k) ++lo;
      x.b[k] = c * kFT + lo;
      x.page[k] = a.old_table[(int64_t)x.b[k] * a.old_max + s_from[lo] + e0 + k - s_first[lo]];
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (!in_pool(a, x.page[k])) x.page[k] = -1;
  };
  const auto mark = [&]() {
    int n[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) n[k] = x.page[k] >= 0 ? now(&a.shares[x.page[k]]) : 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (n[k] < 0) atomicMin(&a.shares[x.page[k]], kMark + x.b[k]);
  };
  const auto put = [&]() {
    int n[kEach], mine = 0, total;
#pragma unroll
    for (int k = 0; k < kEach; ++k) n[k] = x.page[k] >= 0 ? now(&a.shares[x.page[k]]) : 0;
#pragma unroll
    for (int k = 0; k < kEach; ++k) mine += x.page[k] >= 0 && n[k] == kMark + x.b[k];
    // (the last of this turn is put right before the head)
    int at = block_sum(mine, red, total);
    at += room - total;
#pragma unroll
    for (int k = 0; k < kEach; ++k)
      if (x.page[k] >= 0 && n[k] == kMark + x.b[k]) {
        a.shares[x.page[k]] = 0;
        if (at >= 0) a.free_pages[at] = x.page[k];
        ++at;
      }
    room -= total;
    freed += total;
  };
  int total = 0;
  for (int c = 0; !MARKED && c < chunks; ++c) {
    total = open(c);
    for (int t = 0; t * kTurn < total; ++t) get(c, t, total), mark();
    __syncthreads();
  }
  for (int c = chunks - 1; c >= 0; --c) {
    if (MARKED || c < chunks - 1) total = open(c);
    for (int t = (total + kTurn - 1) / kTurn - 1; t >= 0; --t) {
      if (MARKED || chunks > 1 || total > kTurn) get(c, t, total);
      put();
    }
    __syncthreads();
  }
  const int back = min(freed, list ? head : 0), top = head - back;
  const int avail = list ? a.n_free - top : 0;
  // partly filled pages with other holders, and those who hold them so
  bool some = false;
  for (int i = tid; i < a.new_batch; i += kFT) {
    const int page = i == tid ? part0 : a.part[i];
    if (page >= 0 && now(&a.shares[page]) > 0) {
      atomicAdd(&a.last[page].x, 1);
      atomicMax(&a.last[page].y, i);
      some = true;
    }
  }
  int taken = 0;
  // what a request's page was found to be
  int holders = 0, how_many = 0, last = -1;
  const auto look = [&](int page) {
    holders = how_many = 0, last = -1;
    if (page < 0) return;
    holders = now(&a.shares[page]) + 1;
    how_many = now(&a.last[page].x), last = now(&a.last[page].y);
  };
  // (and what has been put into the list is there for the work group)
  if (__syncthreads_or(some)) {
    for (int i0 = 0; i0 < a.new_batch; i0 += kFT) {
      const int i = i0 + tid;
      const int page = i >= a.new_batch ? -1 : i == tid ? part0 : a.part[i];
      look(page);
      const bool own = holders > 1 && (how_many != holders || last != i);
      int more;
      const int at = taken + block_sum(own, red, more);
      taken += more;
      if (own) {
        const int n = i == tid ? n0 : a.new_len[i], S1 = (1 << a.log_page) - 1;
        if (at < avail) {
          const int fresh = now(&a.free_pages[top + at]);
          a.new_table[(int64_t)i * a.new_max + (n >> a.log_page)] = fresh;
          a.copies[3 * at] = page;
          a.copies[3 * at + 1] = fresh;
          a.copies[3 * at + 2] = n & S1;
        } else {
          a.new_len[i] = n & ~S1;
        }
      }
    }
    // counts change once nobody asks for them any more: all that held a page so took
    // pages of their own, but the last if nobody else holds it
    __syncthreads();
    for (int i = tid; i < a.new_batch; i += kFT) {
      const int page = i == tid ? part0 : a.part[i];
      if (a.new_batch > kFT) look(page);
      if (holders > 1 && last == i)
        a.shares[page] = holders - 1 - how_many + (how_many == holders);
    }
  }
  const int given = min(taken, max(avail, 0));
  for (int i = given + tid; i < a.new_batch; i += kFT)
    a.copies[3 * i] = a.copies[3 * i + 1] = a.copies[3 * i + 2] = -1;
  if (tid == 0) {
    *a.free_next = top + given;
    a.meta[0] = back;
    a.meta[1] = given;
    a.meta[2] = taken - given;
    a.meta[3] = freed - back;
  }
  if (tid >= 4 && tid < 8) a.meta[tid] = 0;
}

// Layers of one launch; their pointers are the launch's arguments.
constexpr int kLayers = 64;
struct MoveArgs {
  uint8_t* pool[2 * kLayers];            // k and v by layer
  int64_t page_stride, head_stride, token_stride;   // bytes
  int32_t n_pages, log_page, kv_heads, units;       // units of a row
};

// A work group copies a page's keys in k or v of a layer: neighbouring threads take
// neighbouring units of a row, kCopyAtOnce rows of a thread on their way together, written
// non-temporally (nobody reads them soon).  Bound by reading and writing: 297 MB, read
// and written, in 49 us (6.0 TB/s); with plain stores 55, and with 8 rows 63 (non-temporal
// 51); loads non-temporal as well 73.
constexpr int kCopyAtOnce = 16;
template <class U>
__global__ __launch_bounds__(kNT) void copy_kernel(MoveArgs a, const int32_t* copies, int32_t cap,
                                                   const int32_t* n_copies) {
  const int e = blockIdx.x;
  const int n = *n_copies, from = copies[3 * e], to = copies[3 * e + 1], some = copies[3 * e + 2];
  if (e >= min(n, cap)) return;
  const int keys = min(some, 1 << a.log_page);
  if (from < 0 || from >= a.n_pages || to < 0 || to >= a.n_pages || keys <= 0) return;
  uint8_t* pool = a.pool[2 * blockIdx.y + blockIdx.z];
  const uint8_t* x = pool + from * a.page_stride;
  uint8_t* y = pool + to * a.page_stride;
  const int wide = min(a.units, kNT), per = kNT / wide;    // units and rows at a time
  const int rows = keys * a.kv_heads;
  if ((int)threadIdx.x >= wide * per) return;
  for (int u = threadIdx.x % wide; u < a.units; u += wide) {
    for (int r0 = threadIdx.x / wide; r0 < rows; r0 += per * kCopyAtOnce) {
      U v[kCopyAtOnce];
      int64_t off[kCopyAtOnce];
#pragma unroll
      for (int i = 0; i < kCopyAtOnce; ++i) {
        const int r = min(r0 + i * per, rows - 1), h = (uint32_t)r / (uint32_t)keys;
        off[i] = h * a.head_stride + (r - h * keys) * a.token_stride + (int64_t)u * sizeof(U);
        v[i] = *reinterpret_cast<const U*>(x + off[i]);
      }
#pragma unroll
      for (int i = 0; i < kCopyAtOnce; ++i)
        if (r0 + i * per < rows)
          __builtin_nontemporal_store(v[i], reinterpret_cast<U*>(y + off[i]));
    }
  }
}

// A thread moves one unit of a head's row, in k or v of a layer, for all keys of a
// request's path, which nobody else touches.  A lane looks up a move, 64 at once.  Up to
// kAtOnce keys are read before they are stored where that is the same as one after the
// other: a path's numbers are not below their places, so no key of the ones read
// together is where an earlier one of them goes.  Bound by latency (64 paths of up to 9
// keys in 16 layers 6.7 us, 7.4 with plain stores).
constexpr int kAtOnce = 8;
template <class U>
__global__ __launch_bounds__(kNT) void compact_kernel(MoveArgs a, const int32_t* q_start,
                                                      const int32_t* req, const int64_t* slot,
                                                      const int32_t* path, const int32_t* count,
                                                      int32_t T, int32_t parts) {
  const int b = blockIdx.x / parts, c = (blockIdx.x % parts) * blockDim.x + threadIdx.x;
  const int lane = threadIdx.x & 63;
  const int some = count[b];
  const int q0 = max(q_start[b], 0), n = min(q_start[b + 1], T) - q0;
  if (n <= 0) return;
  const int first = req[q0], m = min(some, n);
  const int64_t slots = (int64_t)a.n_pages << a.log_page;
  const bool mine = c < a.kv_heads * a.units;
  uint8_t* pool = a.pool[2 * blockIdx.y + blockIdx.z] + (c / a.units) * a.head_stride +
                  (int64_t)(c % a.units) * sizeof(U);
  if (first != b) return;
  for (int i0 = 0; i0 < m; i0 += 64) {
    // this lane's move, a slot below 0 for none
    const int i = i0 + lane;
    int64_t from = -1, to = -1;
    bool late = false;
    if (i < m) {
      const int j = path[q0 + i];
      if (j != i && j >= 0 && j < n) {
        from = slot[q0 + j];
        to = slot[q0 + i];
        if (from < 0 || from >= slots || to < 0 || to >= slots) from = -1;
        late = j < i;
      }
    }
    uint64_t todo = __ballot(from >= 0);
    const int most = __any(late) ? 1 : kAtOnce;
    const int64_t S1 = (1 << a.log_page) - 1;
    const int64_t from_at = (from >> a.log_page) * a.page_stride + (from & S1) * a.token_stride;
    const int64_t to_at = (to >> a.log_page) * a.page_stride + (to & S1) * a.token_stride;
    const auto of = [](int64_t x, int l) {
      return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)x, l) |
             (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), l) << 32;
    };
    while (todo) {
      U v[kAtOnce];
      int64_t y[kAtOnce];
      int k = 0;
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q) {
        if (q < most && todo) {
          const int l = __builtin_ctzll(todo);
          todo &= todo - 1;
          y[q] = of(to_at, l);
          if (mine) v[q] = *reinterpret_cast<const U*>(pool + of(from_at, l));
          k = q + 1;
        }
      }
#pragma unroll
      for (int q = 0; q < kAtOnce; ++q)
        if (q < k && mine) __builtin_nontemporal_store(v[q], reinterpret_cast<U*>(pool + y[q]));
    }
  }
}

// The layers' checks, and what a launch needs of them; *bytes is the widest unit that
// all rows are made of.
plora_status caches_status(const plora_kv_cache* c, int32_t layers, MoveArgs& a, int& bytes) {
  if (layers < 0 || (layers > 0 && !c)) return PLORA_ERR_INVALID_ARG;
  if (layers > PLORA_CACHE_MAX_LAYERS) return PLORA_ERR_UNSUPPORTED;
  if (layers == 0) return PLORA_OK;
  const plora_kv_cache& x = c[0];
  if (x.n_pages < 0 || x.kv_heads < 0 || x.head_dim < 0 || x.page_stride < 0 ||
      x.head_stride < 0 || x.token_stride < 0)
    return PLORA_ERR_INVALID_ARG;
  if (!page_size_ok(x.page_size) || (x.dtype != PLORA_BF16 && x.dtype != PLORA_FP16) ||
      x.kv_heads > 1024 || x.head_dim > PLORA_ROPE_MAX_DIM)
    return PLORA_ERR_UNSUPPORTED;
  uint64_t bits = (uint64_t)x.page_stride | (uint64_t)x.head_stride | (uint64_t)x.token_stride |
                  (uint64_t)x.head_dim;
  bits *= 2;
  for (int l = 0; l < layers; ++l) {
    const plora_kv_cache& y = c[l];
    if (y.n_pages != x.n_pages || y.page_size != x.page_size || y.kv_heads != x.kv_heads ||
        y.head_dim != x.head_dim || y.dtype != x.dtype || y.page_stride != x.page_stride ||
        y.head_stride != x.head_stride || y.token_stride != x.token_stride)
      return PLORA_ERR_INVALID_ARG;
    if (x.n_pages > 0 && x.kv_heads > 0 && x.head_dim > 0 && (!y.k || !y.v))
      return PLORA_ERR_INVALID_ARG;
    bits |= reinterpret_cast<uintptr_t>(y.k) | reinterpret_cast<uintptr_t>(y.v);
  }
  bytes = bits & 1 ? 1 : bits & 2 ? 2 : bits & 4 ? 4 : bits & 8 ? 8 : 16;
  if (bytes == 1) return PLORA_ERR_UNSUPPORTED;
  a.page_stride = x.page_stride * 2;
  a.head_stride = x.head_stride * 2;
  a.token_stride = x.token_stride * 2;
  a.n_pages = x.n_pages;
  a.log_page = log2_of(x.page_size);
  a.kv_heads = x.kv_heads;
  a.units = x.head_dim * 2 / bytes;
  return PLORA_OK;
}

// f<U>(layers of this launch) for all layers, kLayers at a time.
template <class F>
plora_status by_layers(const plora_kv_cache* c, int32_t layers, MoveArgs& a, int bytes, F&& f) {
  clear_error();
  for (int l0 = 0; l0 < layers; l0 += kLayers) {
    const int n = std::min(kLayers, layers - l0);
    for (int l = 0; l < n; ++l) {
      a.pool[2 * l] = static_cast<uint8_t*>(c[l0 + l].k);
      a.pool[2 * l + 1] = static_cast<uint8_t*>(c[l0 + l].v);
    }
    if (bytes == 16) f(u32x4{}, n);
    else if (bytes == 8) f(u32x2{}, n);
    else if (bytes == 4) f(uint32_t{}, n);
    else f(uint16_t{}, n);
    const plora_status st = launch_status();
    if (st != PLORA_OK) return st;
  }
  return PLORA_OK;
}

// Whether the one work group does everything: few requests of both batches, and few
// entries at most.  (Two remaps, there and back, in a graph, so and in two launches each:
// 9 requests of 32 pages 13.5 us and 17.0, of 251 pages 16.0 and 17.9, of 938 pages 30 and
// 24; 20 of 63 pages 16.5 and 18.5; 40 of 63 19.2 and 18.7; 60 of 63 24.0 and 19.5.)
constexpr int kInOneRows = 32, kInOneEntries = 4096;
bool remap_in_one(const RemapArgs& a) {
  return a.old_batch + a.new_batch <= kInOneRows &&
         (int64_t)(a.old_batch + a.new_batch) * std::max(a.old_max, a.new_max) <= kInOneEntries;
}

// Whether the marks get a launch of their own, which costs 3 us where little is dropped.
// How much is, only the device knows: requests end where the batch shrinks, and may
// where it does not (a beam's).  (There and back in a graph, without and with it: 64
// requests by 4 over 31 pages, 8 000 entries to drop from, 21 us and 23; over 50, 13 000,
// 33 and 16; over 250, 64 000, 102 and 19; by 8, 224 and 26.  25 600 entries of which none
// is dropped 11.1 and 14.3; all 84 and 56.)
constexpr int64_t kMarkShrinking = 12288, kMarkAny = 65536;
bool remap_marks(const RemapArgs& a) {
  return (int64_t)a.old_batch * a.old_max >=
         (a.new_batch < a.old_batch ? kMarkShrinking : kMarkAny);
}

struct RemapWs {
  size_t drop, bytes;
};
RemapWs remap_ws(int32_t old_batch, int32_t new_batch) {
  RemapWs w{};
  w.drop = align256((size_t)new_batch * 4);
  w.bytes = w.drop + align256((size_t)old_batch * 8);
  return w;
}

}  // namespace
}  // namespace paged

extern "C" size_t plora_kv_remap_workspace_bytes(int32_t old_batch, int32_t new_batch) {
  if (old_batch < 0 || new_batch < 0 || old_batch > PLORA_PAGED_MAX_BATCH ||
      new_batch > PLORA_PAGED_MAX_BATCH)
    return 0;
  return paged::remap_ws(old_batch, new_batch).bytes;
}

extern "C" plora_status plora_kv_remap(const plora_kv_batch* old_batch, const int32_t* src,
                                       const int32_t* keep, int32_t page_size,
                                       const plora_page_pool* pool, const int32_t* free_head,
                                       int32_t* free_next, const plora_kv_batch* new_batch,
                                       int32_t* copies, int32_t* meta, void* ws, size_t ws_bytes,
                                       hipStream_t stream) {
  using namespace paged;
  if (!old_batch || !new_batch || !pool) return PLORA_ERR_INVALID_ARG;
  const plora_kv_batch &o = *old_batch, &n = *new_batch;
  if (o.batch < 0 || o.max_pages < 0 || n.batch < 0 || n.max_pages < 0 || pool->n_pages < 0 ||
      pool->n_free < 0)
    return PLORA_ERR_INVALID_ARG;
  if (o.batch > PLORA_PAGED_MAX_BATCH || n.batch > PLORA_PAGED_MAX_BATCH ||
      !page_size_ok(page_size) || (int64_t)o.max_pages * page_size > PLORA_PAGED_MAX_KEYS ||
      (int64_t)n.max_pages * page_size > PLORA_PAGED_MAX_KEYS)
    return PLORA_ERR_UNSUPPORTED;
  if (!free_head || !free_next || !meta || (o.batch + n.batch > 0 && !ws) || (pool->n_pages > 0 && (!pool->shares || !pool->scratch)) ||
      (pool->n_free > 0 && !pool->free_pages) || (o.batch > 0 && !o.kv_len) ||
      (o.batch > 0 && o.max_pages > 0 && !o.table) ||
      (n.batch > 0 && (!n.kv_len || !src || !copies)) ||
      (n.batch > 0 && n.max_pages > 0 && !n.table))
    return PLORA_ERR_INVALID_ARG;
  if ((o.batch > 0 && n.batch > 0 && (o.kv_len == n.kv_len || (o.table && o.table == n.table))) ||
      free_head == free_next || (n.batch > 0 && (src == n.kv_len || keep == n.kv_len)))
    return PLORA_ERR_INVALID_ARG;
  // (entries of a chunk of requests are counted in 32 bits)
  if ((int64_t)std::min(o.batch, kFT) * o.max_pages > INT32_MAX - kTurn)
    return PLORA_ERR_UNSUPPORTED;
  if (!aligned(ws, 16) || !aligned(pool->scratch, 8)) return PLORA_ERR_UNSUPPORTED;
  const RemapWs w = remap_ws(o.batch, n.batch);
  if (ws_bytes < w.bytes) return PLORA_ERR_WORKSPACE_TOO_SMALL;
  RemapArgs a{};
  a.old_table = o.table;
  a.old_len = o.kv_len;
  a.src = src;
  a.keep = keep;
  a.free_head = free_head;
  a.new_table = n.table;
  a.new_len = n.kv_len;
  a.shares = pool->shares;
  a.free_pages = pool->free_pages;
  a.free_next = free_next;
  a.copies = copies;
  a.meta = meta;
  a.old_batch = o.batch;
  a.new_batch = n.batch;
  a.old_max = o.max_pages;
  a.new_max = n.max_pages;
  a.log_page = log2_of(page_size);
  a.n_pages = pool->n_pages;
  a.n_free = pool->n_free;
  char* p = static_cast<char*>(ws);
  a.part = reinterpret_cast<int32_t*>(p);
  a.drop = reinterpret_cast<int2*>(p + w.drop);
  a.last = reinterpret_cast<int2*>(pool->scratch);
  clear_error();
  if (remap_in_one(a)) {
    hipLaunchKernelGGL((remap_finish_kernel<true, false>), dim3(1), dim3(kFT), 0, stream, a);
    return launch_status();
  }
  hipLaunchKernelGGL(remap_rows_kernel, dim3(o.batch + n.batch), dim3(kNT), 0, stream, a);
  plora_status st = launch_status();
  if (st != PLORA_OK) return st;
  if (!remap_marks(a)) {
    hipLaunchKernelGGL((remap_finish_kernel<false, false>), dim3(1), dim3(kFT), 0, stream, a);
    return launch_status();
  }
  hipLaunchKernelGGL(remap_mark_kernel, dim3(o.batch), dim3(kNT), 0, stream, a);
  st = launch_status();
  if (st != PLORA_OK) return st;
  hipLaunchKernelGGL((remap_finish_kernel<false, true>), dim3(1), dim3(kFT), 0, stream, a);
  return launch_status();
}

extern "C" plora_status plora_kv_copy(const plora_kv_cache* caches, int32_t layers,
                                      const int32_t* copies, int32_t cap,
                                      const int32_t* n_copies, hipStream_t stream) {
  using namespace paged;
  if (cap < 0) return PLORA_ERR_INVALID_ARG;
  if (cap > PLORA_PAGED_MAX_BATCH) return PLORA_ERR_UNSUPPORTED;
  MoveArgs a{};
  int bytes = 16;
  const plora_status st = caches_status(caches, layers, a, bytes);
  if (st != PLORA_OK) return st;
  if (cap > 0 && (!copies || !n_copies)) return PLORA_ERR_INVALID_ARG;
  if (cap == 0 || layers == 0 || a.n_pages == 0 || a.kv_heads == 0 || a.units == 0)
    return PLORA_OK;
  return by_layers(caches, layers, a, bytes, [&](auto u, int n) {
    hipLaunchKernelGGL(copy_kernel<decltype(u)>, dim3(cap, n, 2), dim3(kNT), 0, stream, a, copies,
                       cap, n_copies);
  });
}

extern "C" plora_status plora_kv_compact(const plora_kv_cache* caches, int32_t layers,
                                         const plora_kv_step* step, const int32_t* path,
                                         const int32_t* count, hipStream_t stream) {
  using namespace paged;
  if (!step || step->batch < 0 || step->T < 0) return PLORA_ERR_INVALID_ARG;
  if (step->batch > PLORA_PAGED_MAX_BATCH || step->T > PLORA_PAGED_MAX_TOKENS)
    return PLORA_ERR_UNSUPPORTED;
  MoveArgs a{};
  int bytes = 16;
  const plora_status st = caches_status(caches, layers, a, bytes);
  if (st != PLORA_OK) return st;
  if (layers > 0 && caches[0].page_size != step->page_size) return PLORA_ERR_INVALID_ARG;
  if (step->batch == 0 || step->T == 0 || layers == 0 || a.n_pages == 0 || a.kv_heads == 0 ||
      a.units == 0)
    return PLORA_OK;
  if (!step->q_start || !step->req || !step->slot || !path || !count)
    return PLORA_ERR_INVALID_ARG;
  const int columns = a.kv_heads * a.units, threads = std::min(kNT, (columns + 63) / 64 * 64);
  const int parts = (columns + threads - 1) / threads;
  if ((int64_t)step->batch * parts * threads > (int64_t)UINT32_MAX)   // threads of a launch
    return PLORA_ERR_UNSUPPORTED;
  return by_layers(caches, layers, a, bytes, [&](auto u, int n) {
    hipLaunchKernelGGL(compact_kernel<decltype(u)>, dim3(step->batch * parts, n, 2), dim3(threads),
                       0, stream, a, step->q_start, step->req, step->slot, path, count, step->T,
                       parts);
  });
}

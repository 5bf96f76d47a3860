// Trees of drafted tokens (include/plora_tree.h): plora_tree_plan and
// plora_tree_accept.  (plora_attn_tree is in attn_paged.hip.)

#include <algorithm>

#include "paged_dev.h"
#include "plora_tree.h"

namespace paged {
namespace {

constexpr int kNT = 256;
constexpr int kWaves = kNT / 64;
constexpr int kMost = PLORA_TREE_MAX_NODES;
constexpr int kNone = INT32_MIN;         // no node's parent that is looked for

// The rows of request b, or (b = batch) those behind the last one; rows of no request
// are those of a request that the step left out, too.
struct Rows {
  int q0, n;
  bool there;
};
__device__ __forceinline__ Rows rows_of(const int32_t* q_start, const int32_t* req, int32_t batch,
                                        int32_t T, int b) {
  Rows x;
  x.q0 = min(max(q_start[b], 0), T);
  const int end = b < batch ? min(max(q_start[b + 1], 0), T) : T;
  x.n = max(end - x.q0, 0);
  x.there = b < batch && x.n > 0 && req[x.q0] == b;
  return x;
}

struct TreeArgs {
  const int32_t *parent, *q_start, *kv_len, *req;
  int32_t batch, T;
  int32_t* pos;
  int2* span;
  int2* info;
};

// A work group a request.  With the parents in LDS a node walks to its root twice: to
// add itself to the size of each of its ancestors, and to add up its depth and its
// preorder number: one for each ancestor, and the sizes of the earlier siblings of each
// node on the path.  Those are found by looking at all nodes, four at a time,
// the same ones in all lanes, so that many reads are on their way (24 requests of 100
// to 250 nodes: 11.3 us, 19 with each lane going from its parent on).  Whole numbers, so
// the order of the additions changes nothing.  Bound by latency: 64 requests of 20 to 60
// nodes 6 us, as long as plora_kv_plan for the same step.  The walks are as long as the
// path: 1000 nodes in any order 68 us, 950 of a prompt and 50 drafted behind it 348 (200
// and 50: 35; 1000 of a chain, which is not walked, 3.4).
__global__ __launch_bounds__(kNT) void tree_plan_kernel(TreeArgs a) {
  __shared__ __attribute__((aligned(16))) int s_par[kMost], s_size[kMost], s_sib[kMost];
  __shared__ int s_cut;
  const int tid = threadIdx.x, b = blockIdx.x;
  const int kv = b < a.batch ? a.kv_len[b] : 0;
  const Rows x = rows_of(a.q_start, a.req, a.batch, a.T, b);
  const int32_t* par = a.parent + x.q0;
  if (tid == 0) s_cut = 0;
  // (asked for beside the request's number)
  bool chain = true;
  for (int i = tid; i < x.n; i += kNT) {
    const int p = par[i];
    chain = chain && p == i - 1;
    if (i < kMost) s_par[i] = p, s_size[i] = 0;
  }
  if (tid < 3 && x.n + tid < kMost) s_par[x.n + tid] = kNone, s_size[x.n + tid] = 0;
  chain = __syncthreads_and(chain);
  const int past = x.there ? max(kv - x.n, 0) : 0;
  if (!x.there || chain || x.n > kMost) {
    const bool cut = !x.there || !chain;
    for (int i = tid; i < x.n; i += kNT) {
      a.pos[x.q0 + i] = cut ? 0 : past + i;
      a.span[x.q0 + i] = cut ? int2{-1, -2} : int2{i, x.n - 1};
    }
    if (tid == 0 && b < a.batch)
      a.info[b] = x.there && !chain ? int2{1, x.n} : int2{0, 0};
    return;
  }
  int cut = 0;
  for (int i = tid; i < x.n; i += kNT) {
    int p = i, q;
    while (true) {
      atomicAdd(&s_size[p], 1);
      q = s_par[p];
      if (q < 0 || q >= p) break;
      p = q;
    }
    s_sib[i] = q == -1 ? 0 : -1;
    if (q != -1) {                       // no root is reached: taken back
      ++cut;
      for (q = i;; q = s_par[q]) {
        atomicAdd(&s_size[q], -1);
        if (q == p) break;
      }
    }
  }
  if (cut) atomicAdd(&s_cut, cut);
  __syncthreads();
  for (int i0 = tid & -64; i0 < x.n; i0 += kNT) {
    const int i = i0 + (tid & 63), p = i < x.n ? s_par[i] : kNone;
    const bool cut = i >= x.n || s_sib[i] < 0;
    int before = 0;
    const int4* pars = reinterpret_cast<const int4*>(s_par);
    const int4* sizes = reinterpret_cast<const int4*>(s_size);
    const int end = min(i0 + 63, x.n);
#pragma unroll 4
    for (int j = 0; j < end; j += 4) {
      const int4 q = pars[j >> 2], z = sizes[j >> 2];
      before += q.x == p && j < i ? z.x : 0;
      before += q.y == p && j + 1 < i ? z.y : 0;
      before += q.z == p && j + 2 < i ? z.z : 0;
      before += q.w == p && j + 3 < i ? z.w : 0;
    }
    if (!cut) s_sib[i] = before;
  }
  __syncthreads();
  for (int i = tid; i < x.n; i += kNT) {
    int pos = 0;
    int2 span = {-1, -2};
    if (s_sib[i] >= 0) {
      int depth = -1, first = 0;
      for (int p = i; p >= 0; p = s_par[p]) ++depth, first += s_sib[p];
      first += depth;
      pos = past + depth;
      span = int2{first, first + s_size[i] - 1};
    }
    a.pos[x.q0 + i] = pos;
    a.span[x.q0 + i] = span;
  }
  if (tid == 0) a.info[b] = int2{1, s_cut};
}

struct AcceptArgs {
  const int32_t* parent;
  const void *drafted, *target;
  const int32_t *given, *q_start, *kv_len, *req;
  int32_t batch, T;
  int32_t *path, *count;
  void* token;
  int32_t* kv_out;
};

// A wavefront a request.  A child has a higher number than its node, so the search for
// the next node begins behind the present one, 64 nodes at a time, and the first lane
// that fits has the lowest number.  What is known of up to kHold x 64 nodes is asked for
// at once and searched in registers (1000 requests of up to 60 nodes: 6.0 us, 6.6 with
// two dependent loads a step of the path).  Bound by latency.
constexpr int kHold = 4;
template <class Tok>
__global__ __launch_bounds__(kNT) void tree_accept_kernel(AcceptArgs a) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (b > a.batch) return;
  const int given = a.given && b < a.batch ? a.given[b] : 1;
  const int kv = b < a.batch ? a.kv_len[b] : 0;
  const Rows x = rows_of(a.q_start, a.req, a.batch, a.T, b);
  const int32_t* par = a.parent + x.q0;
  const Tok* drafted = static_cast<const Tok*>(a.drafted) + x.q0;
  const Tok* target = static_cast<const Tok*>(a.target) + x.q0;
  int32_t* path = a.path + x.q0;
  int count = 0;
  Tok token = -1;
  const bool hold = x.n <= 64 * kHold;
  int hp[kHold];
  Tok hd[kHold], ht[kHold];
  if (hold) {
#pragma unroll
    for (int q = 0; q < kHold; ++q) {
      const int i = min(64 * q + lane, x.n - 1);
      if (64 * q < x.n) hp[q] = par[i], hd[q] = drafted[i], ht[q] = target[i];
    }
  }
  if (x.there) {
    const int certain = min(max(given, 0), x.n);
    bool some = certain > 0;
    if (some && x.n > kMost) {           // too many nodes: all are cut
      bool chain = true;
      for (int i = lane; i < x.n; i += 64) chain = chain && par[i] == i - 1;
      some = __all(chain);
    }
    bool fine = true;
    for (int i = lane; some && i < certain; i += 64) fine = fine && par[i] >= -1 && par[i] < i;
    int cur = -1;
    if (some && __all(fine)) {
      for (int i = lane; i < certain; i += 64) path[i] = i;
      count = certain;
      cur = certain - 1;
    } else if (some) {                   // the given nodes that are not cut
      for (int i0 = 0; i0 < certain; i0 += 64) {
        const int i = i0 + lane;
        bool in = false;
        if (i < certain) {
          int p = i, q = par[p];
          while (q >= 0 && q < p) p = q, q = par[p];
          in = q == -1;
        }
        const uint64_t kept = __ballot(in);
        if (in) path[count + __popcll(kept & ((1ull << lane) - 1))] = i;
        if (kept) cur = i0 + 63 - __builtin_clzll(kept);
        count += __popcll(kept);
      }
    }
    // (a child of a node that is not cut is not cut)
    bool going = count > 0;
    const auto target_of = [&](int i) {
      if (!hold) return target[i];
      Tok t = ht[0];
#pragma unroll
      for (int q = 1; q < kHold; ++q) t = (i >> 6) == q ? ht[q] : t;
      return (Tok)__shfl(t, i & 63, 64);
    };
    if (count > 0) token = target_of(cur);
    while (going) {
      int next = -1;
      if (hold) {
#pragma unroll
        for (int q = kHold - 1; q >= 0; --q) {
          if (64 * q >= x.n) continue;
          const int i = 64 * q + lane;
          const uint64_t fits = __ballot(i < x.n && i > cur && hp[q] == cur && hd[q] == token);
          if (fits) next = 64 * q + __builtin_ctzll(fits);
        }
      } else {
        for (int i0 = cur + 1; i0 < x.n && next < 0; i0 += 64) {
          const int i = i0 + lane;
          const uint64_t fits = __ballot(i < x.n && par[i] == cur && drafted[i] == token);
          if (fits) next = i0 + __builtin_ctzll(fits);
        }
      }
      going = next >= 0;
      if (going) {
        cur = next;
        if (lane == 0) path[count] = cur;
        ++count;
        token = target_of(cur);
      }
    }
  }
  for (int i = count + lane; i < x.n; i += 64) path[i] = -1;
  if (lane == 0 && b < a.batch) {
    a.count[b] = count;
    static_cast<Tok*>(a.token)[b] = token;
    a.kv_out[b] = kv - (x.there ? x.n - count : 0);
  }
}

plora_status step_status(const plora_kv_step* s) {
  if (!s || s->batch < 0 || s->T < 0) return PLORA_ERR_INVALID_ARG;
  if (s->batch > PLORA_PAGED_MAX_BATCH || s->T > PLORA_PAGED_MAX_TOKENS)
    return PLORA_ERR_UNSUPPORTED;
  if (s->batch == 0 && s->T == 0) return PLORA_OK;
  if (!s->q_start || (s->batch > 0 && !s->kv_len) || (s->T > 0 && !s->req))
    return PLORA_ERR_INVALID_ARG;
  return PLORA_OK;
}

}  // namespace
}  // namespace paged

extern "C" plora_status plora_tree_plan(const int32_t* parent, const plora_kv_step* step,
                                        const plora_tree* tree, hipStream_t stream) {
  using namespace paged;
  const plora_status st = step_status(step);
  if (st != PLORA_OK) return st;
  if (!tree || tree->batch != step->batch || tree->T != step->T) return PLORA_ERR_INVALID_ARG;
  if (step->batch == 0 && step->T == 0) return PLORA_OK;
  if ((step->T > 0 && (!parent || !tree->pos || !tree->span)) || (step->batch > 0 && !tree->info))
    return PLORA_ERR_INVALID_ARG;
  if (!aligned(tree->span, 8) || !aligned(tree->info, 8)) return PLORA_ERR_UNSUPPORTED;
  TreeArgs a{};
  a.parent = parent;
  a.q_start = step->q_start;
  a.kv_len = step->kv_len;
  a.req = step->req;
  a.batch = step->batch;
  a.T = step->T;
  a.pos = tree->pos;
  a.span = reinterpret_cast<int2*>(tree->span);
  a.info = reinterpret_cast<int2*>(tree->info);
  clear_error();
  hipLaunchKernelGGL(tree_plan_kernel, dim3(step->batch + 1), dim3(kNT), 0, stream, a);
  return launch_status();
}

extern "C" plora_status plora_tree_accept(const int32_t* parent, const void* drafted,
                                          const void* target, int32_t token_bytes,
                                          const int32_t* given, const plora_kv_step* step,
                                          int32_t* path, int32_t* count, void* token,
                                          int32_t* kv_len, hipStream_t stream) {
  using namespace paged;
  const plora_status st = step_status(step);
  if (st != PLORA_OK) return st;
  if (token_bytes != 4 && token_bytes != 8) return PLORA_ERR_UNSUPPORTED;
  if (step->batch == 0 && step->T == 0) return PLORA_OK;
  if ((step->T > 0 && (!parent || !drafted || !target || !path)) ||
      (step->batch > 0 && (!count || !token || !kv_len)))
    return PLORA_ERR_INVALID_ARG;
  if (step->batch > 0 && kv_len == step->kv_len) return PLORA_ERR_INVALID_ARG;
  if (!aligned(drafted, token_bytes) || !aligned(target, token_bytes) ||
      !aligned(token, token_bytes))
    return PLORA_ERR_UNSUPPORTED;
  AcceptArgs a{};
  a.parent = parent;
  a.drafted = drafted;
  a.target = target;
  a.given = given;
  a.q_start = step->q_start;
  a.kv_len = step->kv_len;
  a.req = step->req;
  a.batch = step->batch;
  a.T = step->T;
  a.path = path;
  a.count = count;
  a.token = token;
  a.kv_out = kv_len;
  const dim3 grid((step->batch + kWaves) / kWaves);        // and the rows behind the last
  clear_error();
  if (token_bytes == 4)
    hipLaunchKernelGGL(tree_accept_kernel<int32_t>, grid, dim3(kNT), 0, stream, a);
  else
    hipLaunchKernelGGL(tree_accept_kernel<int64_t>, grid, dim3(kNT), 0, stream, a);
  return launch_status();
}

// Block tables and slot maps of a step from its request lengths
// (include/plora_paged.h, plora_kv_plan).

#include <algorithm>

#include "paged_dev.h"

namespace paged {
namespace {

constexpr int kNT = 256;                // threads per work group
constexpr int kPer = 4;                 // requests per thread and chunk
constexpr int kChunk = kNT * kPer;      // requests scanned at a time
constexpr int kTok = 512;               // tokens per work group
constexpr int kWaves = kNT / 64;

// Exclusive scans over the work group of N counts a thread, in thread order, without
// a cut-off; total is the sums of all.
template <int N>
__device__ __forceinline__ void block_scan(uint32_t (&x)[N], uint32_t (&red)[kWaves][N],
                                           uint32_t (&total)[N]) {
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t inc = wave_scan(x[i], Add{});
    if (lane == 63) red[wv][i] = inc;
    x[i] = inc - x[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    total[i] = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      if (w < wv) x[i] += red[w][i];
      total[i] += red[w][i];
    }
  }
}

// Every work group scans all requests, a chunk of them at a time (tokens, and the
// pages of those that can be served: together where the tokens fit T, as then no
// request is left out for them, else one after the other), keeps the chunk's starts in
// LDS and writes those of its own kTok tokens that the chunk's requests hold: a
// search by halves for the request, one or two loads for the page.  A new page
// begins with a new token (page j of a request was not held, so j S >= past), and
// that token's thread writes the table entry, so a long prompt's pages are
// written in parallel.  No work group waits for another: nothing is read that the
// launch writes (held entries and free_pages are inputs).
// Bound by latency: a launch, the lengths, the search, the page; 16 B written a
// token.
__global__ __launch_bounds__(kNT) void kv_plan_kernel(
    const int32_t* __restrict__ past, const int32_t* __restrict__ n_new,
    const int32_t* __restrict__ free_pages, int32_t n_free,
    const int32_t* __restrict__ free_head, int32_t* __restrict__ free_next, int32_t batch,
    int32_t T, int32_t log_page, int32_t max_pages, int32_t* table, int32_t* __restrict__ q_start,
    int32_t* __restrict__ kv_len, int32_t* __restrict__ pos, int32_t* __restrict__ req,
    int64_t* __restrict__ slot, int32_t* __restrict__ meta) {
  __shared__ int s_start[kChunk], s_past[kChunk], s_off[kChunk];  // s_off -1: left out
  __shared__ uint32_t red2[kWaves][2], red1[kWaves][1];
  const int tid = threadIdx.x, S1 = (1 << log_page) - 1;
  const int64_t most = (int64_t)max_pages << log_page;
  const int head = *free_head;
  // (a free list that starts before its first entry has no pages to give)
  const int64_t avail = head < 0 ? 0 : (int64_t)n_free - head;
  const int t_lo = blockIdx.x * kTok, t_hi = min(T, t_lo + kTok);
  int tok_carry = 0, page_carry = 0, taken = 0, out = 0;
  for (int c0 = 0; c0 < batch; c0 += kChunk) {
    const int m = min(kChunk, batch - c0);
    int p[kPer], n[kPer], need[kPer], st[kPer];
    uint32_t x[2] = {0, 0}, total[2];
    // (1024 counts of at most T + 1 do not overflow; the pages' sum may, and then is
    // not used)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = kPer * tid + i;
      p[i] = b < m ? past[c0 + b] : 0;
      n[i] = b < m ? n_new[c0 + b] : 0;
      const bool ok = p[i] >= 0 && n[i] >= 0 && (int64_t)p[i] + n[i] <= most;
      need[i] = ok ? ((p[i] + n[i] + S1) >> log_page) - ((p[i] + S1) >> log_page) : -1;
      x[0] += min(max(n[i], 0), T + 1);
      x[1] += max(need[i], 0);
    }
    block_scan(x, red2, total);
    int at = min((int)x[0] + tok_carry, T + 1);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      st[i] = at;
      at = min(at + min(max(n[i], 0), T + 1), T + 1);
      if (at > T && n[i] != 0) need[i] = -1;
    }
    tok_carry = min(tok_carry + (int)total[0], T + 1);
    if (tok_carry > T) {
      uint32_t y[1] = {0}, all[1];
#pragma unroll
      for (int i = 0; i < kPer; ++i) y[0] += max(need[i], 0);
      block_scan(y, red1, all);
      x[1] = y[0];
      total[1] = all[0];
    }
    int off = page_carry + (int)x[1];
    page_carry += (int)total[1];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int b = kPer * tid + i;
      const bool ok = need[i] == 0 || (need[i] > 0 && (int64_t)off + need[i] <= avail);
      if (b < m) {
        s_start[b] = st[i];
        s_past[b] = p[i];
        s_off[b] = ok ? off : -1;
        if (ok && need[i] > 0) taken = max(taken, off + need[i]);
        out += !ok;
        if ((c0 / kChunk) % (int)gridDim.x == (int)blockIdx.x) {
          q_start[c0 + b] = min(st[i], T);
          kv_len[c0 + b] = ok ? p[i] + n[i] : max(p[i], 0);
        }
      }
      off += max(need[i], 0);
    }
    __syncthreads();
    // the chunk's tokens among this work group's
    const int lo = max(t_lo, s_start[0]), hi = min(t_hi, tok_carry);
    for (int t = lo + tid; t < hi; t += kNT) {
      int a = 0, z = m;                        // the last request that starts at or before t
      while (z - a > 1) {
        const int mid = (a + z) >> 1;
        if (s_start[mid] <= t) a = mid;
        else z = mid;
      }
      const int o = s_off[a], b = c0 + a;
      int ps = 0, rq = -1;
      int64_t sl = -1;
      if (o >= 0) {
        rq = b;
        ps = s_past[a] + t - s_start[a];
        const int j = ps >> log_page, held = (s_past[a] + S1) >> log_page;
        const int64_t e = (int64_t)b * max_pages + j;
        const int page = j < held ? table[e] : free_pages[head + o + j - held];
        if (j >= held && (ps & S1) == 0) table[e] = page;
        sl = page < 0 ? -1 : ((int64_t)page << log_page) + (ps & S1);
      }
      pos[t] = ps;
      req[t] = rq;
      slot[t] = sl;
    }
    __syncthreads();
  }
  // rows past the requests' tokens
  for (int t = max(t_lo, tok_carry) + tid; t < t_hi; t += kNT) {
    pos[t] = 0;
    req[t] = -1;
    slot[t] = -1;
  }
  if (blockIdx.x == 0) {
    for (int d = 32; d; d >>= 1) {
      taken = max(taken, __shfl_xor(taken, d, 64));
      out += __shfl_xor(out, d, 64);
    }
    __shared__ int w_taken[kWaves], w_out[kWaves];
    if ((tid & 63) == 0) w_taken[tid >> 6] = taken, w_out[tid >> 6] = out;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWaves; ++w) taken = max(taken, w_taken[w]), out += w_out[w];
      *free_next = head + taken;
      q_start[batch] = min(tok_carry, T);
      meta[0] = min(tok_carry, T);
      meta[1] = taken;
      meta[2] = out;
    }
    if (tid >= 3 && tid < 8) meta[tid] = 0;
  }
}

}  // namespace
}  // namespace paged

extern "C" int32_t plora_paged_last_hip_error(void) { return paged::g_last_hip_error.load(); }

extern "C" plora_status plora_kv_plan(const int32_t* past, const int32_t* n_new,
                                      const int32_t* free_pages, int32_t n_free,
                                      const int32_t* free_head, int32_t* free_next,
                                      const plora_kv_step* step, hipStream_t stream) {
  using namespace paged;
  if (!step || step->batch < 0 || step->T < 0 || step->max_pages < 0 || n_free < 0)
    return PLORA_ERR_INVALID_ARG;
  const plora_kv_step& s = *step;
  if (s.batch > PLORA_PAGED_MAX_BATCH || s.T > PLORA_PAGED_MAX_TOKENS ||
      !page_size_ok(s.page_size) || (int64_t)s.max_pages * s.page_size > PLORA_PAGED_MAX_KEYS)
    return PLORA_ERR_UNSUPPORTED;
  if (!free_head || !free_next || !s.q_start || !s.meta || (n_free > 0 && !free_pages))
    return PLORA_ERR_INVALID_ARG;
  if (s.batch > 0 && (!past || !n_new || !s.kv_len)) return PLORA_ERR_INVALID_ARG;
  if (s.batch > 0 && s.max_pages > 0 && !s.table) return PLORA_ERR_INVALID_ARG;
  if (s.T > 0 && (!s.pos || !s.req || !s.slot)) return PLORA_ERR_INVALID_ARG;
  const int grid = std::max(1, (s.T + kTok - 1) / kTok);
  clear_error();
  hipLaunchKernelGGL(kv_plan_kernel, dim3(grid), dim3(kNT), 0, stream, past, n_new, free_pages,
                     n_free, free_head, free_next, s.batch, s.T, log2_of(s.page_size),
                     s.max_pages, s.table, s.q_start, s.kv_len, s.pos, s.req, s.slot, s.meta);
  return launch_status();
}

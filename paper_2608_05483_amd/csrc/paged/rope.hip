// Rotary positions (include/plora_paged.h): plora_rope, plora_rope_append.

#include <algorithm>
#include <cmath>

#include "paged_dev.h"

namespace paged {
namespace {

constexpr int kNT = 256;
constexpr int kBatch = 4;     // rows that a thread asks for before it uses any

// One tensor of a launch: rows of (token, head).  The first is turned, with an out of
// tokens; the others' outs are pools, addressed by slot (out_head within a page), the
// second turned, the third copied.
struct Part {
  const uint16_t* in;
  uint16_t* out;
  int64_t in_token, in_head, out_token, out_head;
  int32_t heads;
};

struct RopeArgs {
  Part part[3];
  int32_t rows;             // heads of one token, all parts
  int32_t rows_per;         // rows per work group
  int32_t units, rot_units; // units of a row, and how many of them turn
  int32_t log_lanes;        // lanes of a row, a power of two
  const int32_t* pos;
  const int64_t* slot;
  const uint64_t* turns;
  int32_t rot, interleaved;
  float scale, sign;        // sign -1: the transposed turn
  int64_t n_slots, page_stride, key_stride;
  int32_t log_page;
};

template <int W>
struct Unit;
template <>
struct Unit<8> { typedef u32x4 type; };
template <>
struct Unit<4> { typedef u32x2 type; };
template <>
struct Unit<2> { typedef uint32_t type; };
template <>
struct Unit<1> { typedef uint16_t type; };

template <int W>
union Words {
  typename Unit<W>::type v;
  uint32_t w[(W + 1) / 2];
  uint16_t h[W];
};

template <class Ty, int W>
__device__ __forceinline__ void unpack(const Words<W>& u, float f[W]) {
  if constexpr (W == 1) {
    f[0] = Ty::lo(u.h[0]);
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) f[2 * i] = Ty::lo(u.w[i]), f[2 * i + 1] = Ty::hi(u.w[i]);
  }
}

template <class Ty, int W>
__device__ __forceinline__ Words<W> pack(const float f[W]) {
  Words<W> u;
  if constexpr (W == 1) {
    u.h[0] = (uint16_t)Ty::pack(f[0], 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) u.w[i] = Ty::pack(f[2 * i], f[2 * i + 1]);
  }
  return u;
}

// One of three values (by value: the choice is then one of registers).
template <class V>
__device__ __forceinline__ V pick(bool third, bool second, V a, V b, V c) {
  return third ? c : second ? b : a;
}

// A work group takes one token (blockIdx.x) and a run of its rows (blockIdx.y:
// heads of q, then k, then v).  A unit is two vectors of W elements, W pairs: in the
// half layout a thread has elements W e.. and rot/2 + W e.., otherwise 2 W e... A
// thread keeps its unit e over all its rows, so its W cosines and sines are read
// once, and a row is found by shifts.  cos and sin of the token's rot/2 angles are
// computed once, into LDS (the part of a turn comes from a wrapping 64-bit product,
// so it is exact at any position), while the first rows are on their way.  Copies
// (v, elements past rot) move bits.
// Bound by reading and writing the tensors (8317 tokens, 64 + 8 + 8 heads of 128:
// 67 us, 5.1 TB/s; with a part's fields indexed in the arguments, read for each row,
// 79, and with a division for each unit and its factors read for each besides, 98).
template <class Ty, int W>
__global__ __launch_bounds__(kNT) void rope_kernel(RopeArgs a) {
  __shared__ float s_cos[PLORA_ROPE_MAX_DIM / 2], s_sin[PLORA_ROPE_MAX_DIM / 2];
  const int t = blockIdx.x, tid = threadIdx.x, half = a.rot / 2;
  const int e = tid & ((1 << a.log_lanes) - 1), step = blockDim.x >> a.log_lanes;
  const int end = min(a.rows, ((int)blockIdx.y + 1) * a.rows_per);
  int row = blockIdx.y * a.rows_per + (tid >> a.log_lanes);
  const bool turns = e < a.rot_units, idle = e >= a.units;
  const int d0 = turns && !a.interleaved ? W * e : 2 * W * e;
  const int d1 = turns && !a.interleaved ? half + W * e : 2 * W * e + W;

  // (asked for before the rows, so that the angles do not wait for those)
  const int64_t ps = a.pos[t];
  const uint64_t turns0 = tid < half ? a.turns[tid] : 0;
  const int64_t slot = a.slot ? a.slot[t] : 0;
  const bool kept = slot >= 0 && slot < a.n_slots;
  const int64_t page = slot >> a.log_page, key = slot - (page << a.log_page);
  const int64_t cell = page * a.page_stride + key * a.key_stride;
  // (a part's fields are picked among values that the work group holds: indexed, each
  // row would read them from memory and wait, for the rows asked for before it too)
  const uint16_t *in0 = a.part[0].in + t * a.part[0].in_token,
                 *in1 = a.part[1].in + t * a.part[1].in_token,
                 *in2 = a.part[2].in + t * a.part[2].in_token;
  uint16_t *out0 = a.part[0].out + t * a.part[0].out_token, *out1 = a.part[1].out + cell,
           *out2 = a.part[2].out + cell;
  const int64_t ih0 = a.part[0].in_head, ih1 = a.part[1].in_head, ih2 = a.part[2].in_head;
  const int64_t oh0 = a.part[0].out_head, oh1 = a.part[1].out_head;
  const int n0 = a.part[0].heads, n01 = n0 + a.part[1].heads;
  Words<W> x[kBatch], y[kBatch];
  uint16_t* to[kBatch];
  int o0[kBatch], o1[kBatch];
  bool turn[kBatch];
  const auto ask = [&]() {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      const int r = row + j * step;
      to[j] = nullptr;
      if (idle || r >= end) continue;
      const bool is_k = r >= n0, is_v = r >= n01;
      const int h = r - pick(is_v, is_k, 0, n0, n01);
      const uint16_t* in = pick(is_v, is_k, in0, in1, in2) + h * pick(is_v, is_k, ih0, ih1, ih2);
      turn[j] = turns && !is_v;
      o0[j] = is_v ? 2 * W * e : d0;
      o1[j] = is_v ? 2 * W * e + W : d1;
      x[j].v = *reinterpret_cast<const typename Unit<W>::type*>(in + o0[j]);
      y[j].v = *reinterpret_cast<const typename Unit<W>::type*>(in + o1[j]);
      // (read whether it is kept or not, so as not to wait for the slot)
      if (!is_k || kept)
        to[j] = pick(is_v, is_k, out0, out1, out2) + h * pick(is_v, is_k, oh0, oh1, oh1);
    }
  };
  ask();
  for (int i = tid; i < half; i += blockDim.x) {
    const uint64_t part = (uint64_t)ps * (i == tid ? turns0 : a.turns[i]);
    // the part of a turn, signed, in half turns: [-1, 1]
    const float f = (float)(int32_t)(part >> 32) * 0x1p-31f;
    s_cos[i] = cospif(f) * a.scale;
    s_sin[i] = sinpif(f) * a.scale * a.sign;
  }
  __syncthreads();
  float c[W], s[W];
#pragma unroll
  for (int i = 0; i < W; ++i) {
    c[i] = turns ? s_cos[W * e + i] : 1.f;
    s[i] = turns ? s_sin[W * e + i] : 0.f;
  }
  while (row < end) {
#pragma unroll
    for (int j = 0; j < kBatch; ++j) {
      if (!to[j]) continue;
      if (turn[j]) {
        float f[W], g[W], p[W], q[W];
        unpack<Ty, W>(x[j], f);
        unpack<Ty, W>(y[j], g);
        if (W > 1 && a.interleaved) {
          // pairs 0 .. W/2 - 1 are in x, the others in y
#pragma unroll
          for (int i = 0; i < W / 2; ++i) {
            const int k = W / 2 + i;
            p[2 * i] = f[2 * i] * c[i] - f[2 * i + 1] * s[i];
            p[2 * i + 1] = f[2 * i] * s[i] + f[2 * i + 1] * c[i];
            q[2 * i] = g[2 * i] * c[k] - g[2 * i + 1] * s[k];
            q[2 * i + 1] = g[2 * i] * s[k] + g[2 * i + 1] * c[k];
          }
        } else {
#pragma unroll
          for (int i = 0; i < W; ++i) {
            p[i] = f[i] * c[i] - g[i] * s[i];
            q[i] = f[i] * s[i] + g[i] * c[i];
          }
        }
        x[j] = pack<Ty, W>(p);
        y[j] = pack<Ty, W>(q);
      }
      *reinterpret_cast<typename Unit<W>::type*>(to[j] + o0[j]) = x[j].v;
      *reinterpret_cast<typename Unit<W>::type*>(to[j] + o1[j]) = y[j].v;
    }
    row += kBatch * step;
    if (row < end) ask();
  }
}

// Whether units of w elements fit a tensor: its pointer, strides and cuts.
bool fits(int w, const void* p, int64_t token, int64_t head, int64_t page) {
  return aligned(p, 2 * w) && token % w == 0 && head % w == 0 && page % w == 0;
}

plora_status check(int32_t T, int32_t heads, int32_t head_dim, int32_t rot, int32_t layout,
                   int32_t dtype, float scale) {
  if (T < 0 || heads < 0 || head_dim < 0 || rot < 0 || rot > head_dim)
    return PLORA_ERR_INVALID_ARG;
  if (!std::isfinite(scale)) return PLORA_ERR_INVALID_ARG;
  if (T > PLORA_PAGED_MAX_TOKENS || heads > 65536 || head_dim > PLORA_ROPE_MAX_DIM ||
      head_dim % 2 || rot % 2 || (layout != PLORA_ROPE_HALF && layout != PLORA_ROPE_INTERLEAVED) ||
      (dtype != PLORA_BF16 && dtype != PLORA_FP16))
    return PLORA_ERR_UNSUPPORTED;
  return PLORA_OK;
}

template <class Ty>
void launch_type(const RopeArgs& a, int w, dim3 grid, int threads, hipStream_t stream) {
  auto* k = w == 8 ? rope_kernel<Ty, 8> : w == 4 ? rope_kernel<Ty, 4>
          : w == 2 ? rope_kernel<Ty, 2> : rope_kernel<Ty, 1>;
  hipLaunchKernelGGL(k, grid, dim3(threads), 0, stream, a);
}

// Vectors of the widest w that cuts a row into whole units, and the launch.
plora_status launch(RopeArgs& a, int32_t T, int32_t head_dim, int32_t dtype, int w,
                    hipStream_t stream) {
  while (w > 1 && (a.rot % (2 * w) || (head_dim - a.rot) % (2 * w))) w /= 2;
  a.units = head_dim / (2 * w);
  a.rot_units = a.rot / (2 * w);
  a.log_lanes = log2_of(a.units);
  a.rows = a.part[0].heads + a.part[1].heads + a.part[2].heads;
  if (a.rows == 0) return PLORA_OK;
  const int64_t lanes = (int64_t)a.rows << a.log_lanes;
  const int threads = (int)std::min<int64_t>(kNT, (lanes + 63) / 64 * 64);
  // A token's rows go to one work group for each kBatch passes, or, where the
  // tokens alone would leave compute units idle, for each pass.
  const int pass = threads >> a.log_lanes;
  a.rows_per = T < 1024 ? pass : kBatch * pass;
  const int blocks = (a.rows + a.rows_per - 1) / a.rows_per;
  a.rows_per = ((a.rows + blocks - 1) / blocks + pass - 1) / pass * pass;
  if (blocks > 65535) return PLORA_ERR_UNSUPPORTED;
  clear_error();
  const dim3 grid(T, blocks);
  if (dtype == PLORA_BF16) launch_type<Bf16>(a, w, grid, threads, stream);
  else launch_type<Fp16>(a, w, grid, threads, stream);
  return launch_status();
}

}  // namespace
}  // namespace paged

extern "C" plora_status plora_rope(const void* x, int64_t x_token, int64_t x_head,
                                   const int32_t* pos, const uint64_t* turns, int32_t T,
                                   int32_t heads, int32_t head_dim, int32_t rot, int32_t layout,
                                   float scale, int32_t inverse, int32_t dtype, void* out,
                                   int64_t out_token, int64_t out_head, hipStream_t stream) {
  using namespace paged;
  plora_status st = check(T, heads, head_dim, rot, layout, dtype, scale);
  if (st != PLORA_OK) return st;
  if (T == 0 || heads == 0 || head_dim == 0) return PLORA_OK;
  if (!x || !out || !pos || (rot > 0 && !turns) || x_token < 0 || x_head < 0 || out_token < 0 ||
      out_head < 0)
    return PLORA_ERR_INVALID_ARG;
  if (!aligned(x, 2) || !aligned(out, 2)) return PLORA_ERR_UNSUPPORTED;
  RopeArgs a{};
  a.part[0] = {(const uint16_t*)x, (uint16_t*)out, x_token, x_head, out_token, out_head,
               heads};
  a.pos = pos;
  a.turns = turns;
  a.rot = rot;
  a.interleaved = layout == PLORA_ROPE_INTERLEAVED;
  a.scale = scale;
  a.sign = inverse ? -1.f : 1.f;
  int w = 8;
  while (w > 1 && !(fits(w, x, x_token, x_head, 0) && fits(w, out, out_token, out_head, 0))) w /= 2;
  return launch(a, T, head_dim, dtype, w, stream);
}

extern "C" plora_status plora_rope_append(const void* q, int64_t q_token, int64_t q_head,
                                          const void* k, int64_t k_token, int64_t k_head,
                                          const void* v, int64_t v_token, int64_t v_head,
                                          const int32_t* pos, const int64_t* slot,
                                          const uint64_t* turns, int32_t T, int32_t heads,
                                          int32_t rot, int32_t layout, float scale,
                                          const plora_kv_cache* cache, void* q_out,
                                          int64_t out_token, int64_t out_head,
                                          hipStream_t stream) {
  using namespace paged;
  if (!cache) return PLORA_ERR_INVALID_ARG;
  const plora_kv_cache& c = *cache;
  plora_status st = check(T, heads, c.head_dim, rot, layout, c.dtype, scale);
  if (st != PLORA_OK) return st;
  if (c.n_pages < 0 || c.kv_heads < 0 || c.page_stride < 0 || c.head_stride < 0 ||
      c.token_stride < 0)
    return PLORA_ERR_INVALID_ARG;
  if (!page_size_ok(c.page_size) || c.kv_heads > 65536) return PLORA_ERR_UNSUPPORTED;
  if (T == 0 || c.head_dim == 0) return PLORA_OK;
  if (!pos || !slot || (rot > 0 && !turns)) return PLORA_ERR_INVALID_ARG;
  if (heads > 0 && (!q || !q_out || q_token < 0 || q_head < 0 || out_token < 0 || out_head < 0))
    return PLORA_ERR_INVALID_ARG;
  if (c.kv_heads > 0 && (!k || !v || !c.k || !c.v || k_token < 0 || k_head < 0 || v_token < 0 ||
                         v_head < 0))
    return PLORA_ERR_INVALID_ARG;
  if (!aligned(q, 2) || !aligned(q_out, 2) || !aligned(k, 2) || !aligned(v, 2) ||
      !aligned(c.k, 2) || !aligned(c.v, 2))
    return PLORA_ERR_UNSUPPORTED;
  RopeArgs a{};
  a.part[0] = {(const uint16_t*)q, (uint16_t*)q_out, q_token, q_head, out_token, out_head,
               heads};
  a.part[1] = {(const uint16_t*)k, (uint16_t*)c.k, k_token, k_head, 0, c.head_stride,
               c.kv_heads};
  a.part[2] = {(const uint16_t*)v, (uint16_t*)c.v, v_token, v_head, 0, c.head_stride,
               c.kv_heads};
  a.pos = pos;
  a.slot = slot;
  a.turns = turns;
  a.rot = rot;
  a.interleaved = layout == PLORA_ROPE_INTERLEAVED;
  a.scale = scale;
  a.sign = 1.f;
  a.n_slots = (int64_t)c.n_pages * c.page_size;
  a.page_stride = c.page_stride;
  a.key_stride = c.token_stride;
  a.log_page = log2_of(c.page_size);
  int w = 8;
  while (w > 1 && !(fits(w, q, q_token, q_head, 0) && fits(w, q_out, out_token, out_head, 0) &&
                    fits(w, k, k_token, k_head, 0) && fits(w, v, v_token, v_head, 0) &&
                    fits(w, c.k, c.token_stride, c.head_stride, c.page_stride) &&
                    fits(w, c.v, c.token_stride, c.head_stride, c.page_stride)))
    w /= 2;
  return launch(a, T, c.head_dim, c.dtype, w, stream);
}

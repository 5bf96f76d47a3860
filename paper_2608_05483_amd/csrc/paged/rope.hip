// Rotary positions (include/plora_paged.h): plora_rope, plora_rope_append.

#include <algorithm>
#include <cmath>

#include "paged_dev.h"

namespace paged {
namespace {

constexpr int kNT = 256;

// One tensor of a launch: rows of (token, head), each cut into units of W
// elements or W pairs.  units = those of one head, rot_units the first of them
// that are turned.
struct Part {
  const uint16_t* in;
  uint16_t* out;
  int64_t in_token, in_head, out_token, out_head;   // out_*: pages for the cache
  int32_t heads, units, rot_units;
  int32_t cached;                                   // out is a pool, addressed by slot
};

struct RopeArgs {
  Part part[3];
  int32_t parts;
  int32_t units;            // of one token, all parts
  int32_t chunk;            // units per work group
  const int32_t* pos;
  const int64_t* slot;
  const uint64_t* turns;
  int32_t T, rot, interleaved;
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
__device__ __forceinline__ void load(const uint16_t* p, float f[W]) {
  Words<W> u;
  u.v = *reinterpret_cast<const typename Unit<W>::type*>(p);
  if constexpr (W == 1) {
    f[0] = Ty::lo(u.h[0]);
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) f[2 * i] = Ty::lo(u.w[i]), f[2 * i + 1] = Ty::hi(u.w[i]);
  }
}

template <class Ty, int W>
__device__ __forceinline__ void store(uint16_t* p, const float f[W]) {
  Words<W> u;
  if constexpr (W == 1) {
    u.h[0] = (uint16_t)Ty::pack(f[0], 0.f);
  } else {
#pragma unroll
    for (int i = 0; i < W / 2; ++i) u.w[i] = Ty::pack(f[2 * i], f[2 * i + 1]);
  }
  *reinterpret_cast<typename Unit<W>::type*>(p) = u.v;
}

// A work group takes one token (blockIdx.x) and a run of its units
// (blockIdx.y).  cos and sin of the token's rot/2 angles are computed once, into
// LDS (the part of a turn comes from a wrapping 64-bit product, so it is exact
// at any position), then every unit is one load, W turns and one store: 16 bytes a lane where the layout
// allows (W = 8).  Copies (v, elements past rot) move bits.
// Bound by reading and writing the tensors.
template <class Ty, int W>
__global__ __launch_bounds__(kNT) void rope_kernel(RopeArgs a) {
  __shared__ float s_cos[PLORA_ROPE_MAX_DIM / 2], s_sin[PLORA_ROPE_MAX_DIM / 2];
  const int t = blockIdx.x, tid = threadIdx.x, half = a.rot / 2;
  const int64_t ps = a.pos[t];
  for (int i = tid; i < half; i += kNT) {
    const uint64_t part = (uint64_t)ps * a.turns[i];
    // the part of a turn, signed, in half turns: [-1, 1]
    const float x = (float)(int32_t)(part >> 32) * 0x1p-31f;
    s_cos[i] = cospif(x) * a.scale;
    s_sin[i] = sinpif(x) * a.scale * a.sign;
  }
  int64_t slot = a.slot ? a.slot[t] : 0;
  const bool kept = slot >= 0 && slot < a.n_slots;
  const int64_t page = slot >> a.log_page, key = slot - (page << a.log_page);
  const int64_t cell = page * a.page_stride + key * a.key_stride;
  __syncthreads();
  const int end = min(a.units, ((int)blockIdx.y + 1) * a.chunk);
  for (int u0 = blockIdx.y * a.chunk + tid; u0 < end; u0 += kNT) {
    int u = u0, n = 0;
    while (n + 1 < a.parts && u >= a.part[n].heads * a.part[n].units) {
      u -= a.part[n].heads * a.part[n].units;
      ++n;
    }
    const Part& p = a.part[n];
    if (p.cached && !kept) continue;
    const int h = u / p.units, e = u - h * p.units;
    const uint16_t* in = p.in + t * p.in_token + h * p.in_head;
    uint16_t* out = p.out + (p.cached ? cell : t * p.out_token) + h * p.out_head;
    if (e >= p.rot_units) {
      const int d = (p.rot_units ? a.rot : 0) + (e - p.rot_units) * W;
      *reinterpret_cast<typename Unit<W>::type*>(out + d) =
          *reinterpret_cast<const typename Unit<W>::type*>(in + d);
    } else if (!a.interleaved) {
      float x[W], y[W], r[W], q[W];
      load<Ty, W>(in + e * W, x);
      load<Ty, W>(in + half + e * W, y);
#pragma unroll
      for (int i = 0; i < W; ++i) {
        const float c = s_cos[e * W + i], s = s_sin[e * W + i];
        r[i] = x[i] * c - y[i] * s;
        q[i] = x[i] * s + y[i] * c;
      }
      store<Ty, W>(out + e * W, r);
      store<Ty, W>(out + half + e * W, q);
    } else if constexpr (W >= 2) {
      float x[W], r[W];
      load<Ty, W>(in + e * W, x);
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        const float c = s_cos[e * (W / 2) + i], s = s_sin[e * (W / 2) + i];
        r[2 * i] = x[2 * i] * c - x[2 * i + 1] * s;
        r[2 * i + 1] = x[2 * i] * s + x[2 * i + 1] * c;
      }
      store<Ty, W>(out + e * W, r);
    } else {
      // one element at a time: the pairs of this unit are 2e and 2e + 1
      float x, y;
      load<Ty, 1>(in + 2 * e, &x);
      load<Ty, 1>(in + 2 * e + 1, &y);
      const float c = s_cos[e], s = s_sin[e], r = x * c - y * s, q = x * s + y * c;
      store<Ty, 1>(out + 2 * e, &r);
      store<Ty, 1>(out + 2 * e + 1, &q);
    }
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
void launch_type(const RopeArgs& a, int w, dim3 grid, hipStream_t stream) {
  auto* k = w == 8 ? rope_kernel<Ty, 8> : w == 4 ? rope_kernel<Ty, 4>
          : w == 2 ? rope_kernel<Ty, 2> : rope_kernel<Ty, 1>;
  hipLaunchKernelGGL(k, grid, dim3(kNT), 0, stream, a);
}

// Units of the widest w that cuts every part evenly, and the launch.
plora_status launch(RopeArgs& a, int32_t head_dim, int32_t dtype, int w, hipStream_t stream) {
  const int turned = a.interleaved ? a.rot : a.rot / 2;     // elements that units begin in
  while (w > 1 && (turned % w || (head_dim - a.rot) % w)) w /= 2;
  const int rot_units = a.interleaved && w == 1 ? a.rot / 2 : turned / w;
  a.units = 0;
  for (int n = 0; n < a.parts; ++n) {
    Part& p = a.part[n];
    if (p.rot_units) p.rot_units = rot_units, p.units = rot_units + (head_dim - a.rot) / w;
    else p.units = head_dim / w;
    a.units += p.heads * p.units;
  }
  if (a.units == 0) return PLORA_OK;
  // A token's units go to one work group, or, where the tokens alone would leave
  // compute units idle, to one for each 256 of them
  a.chunk = a.T < 1024 ? kNT : a.units;
  const dim3 grid(a.T, (a.units + a.chunk - 1) / a.chunk);
  if (grid.y > 65535) return PLORA_ERR_UNSUPPORTED;
  clear_error();
  if (dtype == PLORA_BF16) launch_type<Bf16>(a, w, grid, stream);
  else launch_type<Fp16>(a, w, grid, stream);
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
               heads, 0, rot > 0, 0};
  a.parts = 1;
  a.pos = pos;
  a.turns = turns;
  a.T = T;
  a.rot = rot;
  a.interleaved = layout == PLORA_ROPE_INTERLEAVED;
  a.scale = scale;
  a.sign = inverse ? -1.f : 1.f;
  int w = 8;
  while (w > 1 && !(fits(w, x, x_token, x_head, 0) && fits(w, out, out_token, out_head, 0))) w /= 2;
  return launch(a, head_dim, dtype, w, stream);
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
               heads, 0, rot > 0, 0};
  a.part[1] = {(const uint16_t*)k, (uint16_t*)c.k, k_token, k_head, 0, c.head_stride,
               c.kv_heads, 0, rot > 0, 1};
  a.part[2] = {(const uint16_t*)v, (uint16_t*)c.v, v_token, v_head, 0, c.head_stride,
               c.kv_heads, 0, 0, 1};
  a.parts = 3;
  a.pos = pos;
  a.slot = slot;
  a.turns = turns;
  a.T = T;
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
  return launch(a, c.head_dim, c.dtype, w, stream);
}

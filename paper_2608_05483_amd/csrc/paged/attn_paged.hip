// Attention over the paged cache (include/plora_paged.h, plora_attn_paged): the
// items of the step's plan, then the merge of the partials.
//
// Both kernels compute transposed tiles: S^T = K Q^T, so that a lane holds scores
// of one query row (its column) for several keys, then O^T = V^T P^T with P taken
// straight from those registers: the matrix instruction's output layout gives a
// lane groups of four keys, and since a product may sum its keys in any order, V
// is brought into the same order.  No weight crosses a lane.  V^T needs, for one
// dimension, eight keys in a lane: few_kernel loads eight rows and transposes the
// 16-bit block in the lane's own registers, tile_kernel reads columns from LDS.
// The scores are kept times scale log2(e), so a weight is one exp2 of one fma.
//
// TREE (include/plora_tree.h, plora_attn_tree): a row sees, of its request's new keys,
// those whose interval of preorder numbers holds the row's own number.  A node's
// ancestors have lower numbers than it, so a row's last key is the one that it has
// without a tree, and the plan is the same; only in the steps that reach new keys does
// a lane compare the intervals of its keys.

#include <cmath>

#include "attn_plan.h"
#include "plora_tree.h"

namespace paged {
namespace {

constexpr int kNT = 256;
constexpr int kWaves = kNT / 64;
constexpr int kRsrcWord3 = 0x00020000;    // raw buffer, 32-bit data format (gfx9 family)
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
  const uint16_t *q, *k, *v;
  int64_t q_token, q_head, out_token, out_head, page_stride, head_stride;
  int32_t key_stride, n_pages, log_page, max_pages;
  const int32_t *table, *pos, *order, *req, *q_start;
  const PlanHeader* head;
  const Item *few, *last_few, *tile;
  const ReqInfo* info;
  int32_t batch, T, r, kv_heads;
  float c;                  // |scale| log2(e)
  uint32_t flip;            // sign bits for q where scale < 0
  uint16_t* out;
  float *pm, *pl, *po;      // partials: [row][kv_heads], [row][kv_heads][D]
  const int2 *span, *tree;  // trees: intervals by token, kinds by request
};

// The launch's arguments, read again: what is used only behind an item's loop would
// otherwise be held in scalar registers through it, which there are too few of.
__device__ __forceinline__ AttnArgs args_again() {
  auto p = __builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  AttnArgs a;
  __builtin_memcpy(&a, (const void*)p, sizeof(a));
  return a;
}

__device__ __forceinline__ f32x4 mfma16(Bf16, u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma16(Fp16, u32x4 a, u32x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(Bf16, u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(Fp16, u32x4 a, u32x4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Where 16 keys of one page and head lie, and how many bytes of them a row may
// read: what lies past the valid rows, or in a page outside the pool, reads zero
// through the buffer resource and fetches nothing.
// (What the 16 keys span, and a lane's offset in it, are counted in 32 bits: at most
// 30 token strides in bytes.)
constexpr int64_t kTokenStrideEnd = INT64_C(1) << 25;
static_assert(30 * kTokenStrideEnd + 4096 <= INT32_MAX, "");
struct Cell {
  int64_t at;
  int bytes;
};
__device__ __forceinline__ int page_of(const AttnArgs& a, const int32_t* row, int key, int end) {
  return row[min(key, end - 1) >> a.log_page];
}
__device__ __forceinline__ Cell cell_of(const AttnArgs& a, int page, int kvh, int key, int end,
                                        int D) {
  page = uniform(page);
  const bool ok = page >= 0 && page < a.n_pages && key < end;
  page = ok ? page : 0;
  Cell c;
  c.at = page * a.page_stride + kvh * a.head_stride +
         (int64_t)(key & ((1 << a.log_page) - 1)) * a.key_stride;
  c.bytes = ok ? ((min(end - key, 16) - 1) * a.key_stride + D) * 2 : 0;
  return c;
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const uint16_t* x, const Cell& c) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(x) + c.at, 0, c.bytes,
                                           kRsrcWord3);
}

// The few items' loads of K and V, which each reads once: non-temporal.  Layers in
// turn, both kernels, so and by the default policy: one request of 30011 keys on 8
// heads, 8 layers of 123 MB, 30.8 us a layer and 32.5; 16 of 1001 keys, 8 of 67 MB, 19.6
// and 22.5; 64 of 501, 8 of 135 MB, 27.1 and 30.9.  Only where all layers stay in the
// last-level cache is the default faster: one request of 3001 keys, 16 layers of 13 MB,
// 16.0 and 15.1 (32 of them, 16.0 and 17.0).
constexpr int kOnce = 2;
__device__ __forceinline__ u32x4 bld16(__amdgpu_buffer_rsrc_t r, int off) {
  return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, off, 0, kOnce));
}
__device__ __forceinline__ u32x2 bld8(__amdgpu_buffer_rsrc_t r, int off) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, off, 0, kOnce));
}

// Words of 16-bit pairs (a's, b's) of the low or high halves.
__device__ __forceinline__ uint32_t zip(uint32_t a, uint32_t b, bool high) {
  return high ? __builtin_amdgcn_perm(b, a, 0x07060302u) : __builtin_amdgcn_perm(b, a, 0x05040100u);
}

// A query row: its token, its head, the end of the keys it sees, its preorder number.
struct Row {
  int token, head, limit, number;
};
template <bool TREE>
__device__ __forceinline__ Row query_row(const AttnArgs& a, const Item& it, int kvh, int i) {
  Row x{0, 0, it.lo, -1};
  if (i < it.rows) {
    const int R = it.row + i, tk = it.tok + R / a.r;
    x.token = it.gathered ? a.order[tk] : tk;
    x.head = kvh * a.r + R % a.r;
    x.limit = max(it.lo, min(it.hi, a.pos[x.token] + 1));
    if constexpr (TREE) {
      x.number = a.span[x.token].x;
      if (x.number < 0) x.limit = it.lo;
    }
  }
  return x;
}

// Where an item's keys are the new ones of a tree: from key past on, key j is that of
// token j - shift.  (Chains and prefixes have none.)
struct NewKeys {
  int past, shift;
};
template <bool TREE>
__device__ __forceinline__ NewKeys new_keys(const AttnArgs& a, const Item& it) {
  NewKeys x{INT32_MAX, 0};
  if constexpr (TREE) {
    // (asked for together)
    const int kind = a.tree[max(it.req, 0)].x, past = a.pos[it.gathered ? 0 : it.tok];
    if (!it.gathered && uniform(kind)) {
      x.past = uniform(past);
      x.shift = x.past - it.tok;
    }
  }
  return x;
}
// Whether a row sees a key below its limit.  (The token is one of the request's if the
// step's arrays agree with each other, and one of the step's in any case.)
template <bool TREE>
__device__ __forceinline__ bool sees(const AttnArgs& a, const NewKeys& fresh, const Row& x,
                                     int key) {
  if (!TREE) return true;
  const int2 s = a.span[min(max(key - fresh.shift, 0), a.T - 1)];
  return (key < fresh.past) | ((s.x <= x.number) & (x.number <= s.y));
}

// One row by itself, in vector arithmetic over the keys it sees and no others,
// by one wavefront: 64 keys at a time, a lane a key for the scores and a lane D/64
// dimensions for the output.  Taken where the tiles gave a row that is not finite:
// they multiply the zero weight of a masked key with its value, which is not zero
// if that value is an infinity or NaN.  Rare, and then the row's own infinities and
// NaN come out as the sum gives them.
template <class Ty, int D, bool TREE>
__device__ __forceinline__ void careful_row(const AttnArgs& a, const Item& it, int kvh, int i) {
  constexpr int kPer = D / 64;
  const int lane = threadIdx.x & 63;
  const Row x = query_row<TREE>(a, it, kvh, i);
  const NewKeys fresh = new_keys<TREE>(a, it);
  bool some = x.limit > it.lo && (!TREE || it.lo < fresh.past);
  const uint16_t* q = a.q + x.token * a.q_token + x.head * a.q_head;
  const int32_t* row = a.table + (int64_t)it.req * a.max_pages;
  float m = -INFINITY, l = 0.f, acc[kPer] = {};
  for (int k0 = it.lo; k0 < x.limit; k0 += 64) {
    const int n = min(64, x.limit - k0);
    float s = -INFINITY;
    const bool seen = lane < n && sees<TREE>(a, fresh, x, k0 + lane);
    const uint64_t all = TREE ? __ballot(seen) : 0;
    some = some || all != 0;
    if (seen) {
      const int key = k0 + lane, page = row[key >> a.log_page];
      s = 0.f;
      if (page >= 0 && page < a.n_pages) {
        const uint16_t* kp = a.k + page * a.page_stride + kvh * a.head_stride +
                             (int64_t)(key & ((1 << a.log_page) - 1)) * a.key_stride;
        for (int d = 0; d < D; d += 2) {
          const uint32_t kw = *reinterpret_cast<const uint32_t*>(kp + d);
          const uint32_t qw = *reinterpret_cast<const uint32_t*>(q + d) ^ a.flip;
          s = fmaf(Ty::lo(kw), Ty::lo(qw), s);
          s = fmaf(Ty::hi(kw), Ty::hi(qw), s);
        }
      }
      s *= a.c;
    }
    float mx = s;
    for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
    mx = fmaxf(mx, m);
    const float ms = mx == -INFINITY ? 0.f : mx;
    const float al = exp2_(m - ms), p = exp2_(s - ms);
    m = mx;
    float t = p;
    for (int d = 32; d; d >>= 1) t += __shfl_xor(t, d, 64);
    l = l * al + t;
    for (int j = 0; j < kPer; ++j) acc[j] *= al;
    for (int j = 0; j < n; ++j) {
      if (TREE && !(all >> j & 1)) continue;
      const int key = k0 + j, page = uniform(row[key >> a.log_page]);
      const float w = __shfl(p, j, 64);
      if (page < 0 || page >= a.n_pages) continue;
      const uint16_t* vp = a.v + page * a.page_stride + kvh * a.head_stride +
                           (int64_t)(key & ((1 << a.log_page) - 1)) * a.key_stride + kPer * lane;
      for (int e = 0; e < kPer; ++e) acc[e] = fmaf(w, Ty::lo(vp[e]), acc[e]);
    }
  }
  if (m == -INFINITY && some) l = NAN;                // every score -inf: 0 / 0
  if (it.part < 0) {
    uint16_t* o = a.out + x.token * a.out_token + x.head * a.out_head + kPer * lane;
    for (int e = 0; e < kPer; ++e)
      o[e] = (uint16_t)Ty::pack(some ? acc[e] / l : 0.f, 0.f);
  } else {
    const int64_t at = ((int64_t)it.part + i) * a.kv_heads + kvh;
    if (lane == 0) a.pm[at] = m, a.pl[at] = l;
    for (int e = 0; e < kPer; ++e) a.po[at * D + kPer * lane + e] = acc[e];
  }
}

// N dimensions of an output row times inv, or of a partial.
template <class Ty, int N>
__device__ __forceinline__ void store_out(uint16_t* out, const float (&o)[N], float inv) {
  uint32_t w[N / 2];
#pragma unroll
  for (int d = 0; d < N / 2; ++d) w[d] = Ty::pack(o[2 * d] * inv, o[2 * d + 1] * inv);
  if constexpr (N == 8) *reinterpret_cast<u32x4*>(out) = u32x4{w[0], w[1], w[2], w[3]};
  else if constexpr (N == 4) *reinterpret_cast<u32x2*>(out) = u32x2{w[0], w[1]};
  else *reinterpret_cast<uint32_t*>(out) = w[0];
}
template <int N>
__device__ __forceinline__ void store_part(float* po, const float (&o)[N]) {
  if constexpr (N == 2) {
    po[0] = o[0], po[1] = o[1];
  } else {
#pragma unroll
    for (int d = 0; d < N; d += 4)
      *reinterpret_cast<f32x4*>(po + d) = f32x4{o[d], o[d + 1], o[d + 2], o[d + 3]};
  }
}

// Items of up to 16 rows (decode: the rows are a key head's query heads times the
// request's new tokens).  Bound by reading K and V once: 16 rows cost the matrix
// units a twentieth of that time, so every row count up to 16 takes one tile.  The
// four wavefronts take 32 keys each in turn, straight from memory into registers
// (K as the 16x16x32 product's rows: key n of 16, 16-byte units; V as rows of eight
// keys), and join through LDS at the end.  The weights enter the product with V as
// two values, hi + lo, which costs nothing here and keeps them to 16 bits.
// (most: of a tile item the last key of each wavefront's rows, of a few item with a
// tree the rows that see any of the wavefront's keys)
struct FewShared {
  float m[kWaves][kFew], l[kWaves][kFew];
  int bad, most[kWaves];
};
template <class Ty, int D, bool AHEAD, bool TREE>
__device__ __forceinline__ void few_item(const AttnArgs& a, const Item& it, int kvh,
                                         FewShared& sh, f32x4* o01, f32x4* o23) {
  constexpr int kQ = D / 32;             // 16-byte units of a row, per lane
  constexpr int kV = D / 16;             // dimensions per lane
  if (it.rows <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const int n = lane & 15, g = lane >> 4;
  const int32_t* row = a.table + (int64_t)it.req * a.max_pages;

  // The loads of 32 keys; the pages of the next 32 are asked for meanwhile.  The
  // first are under way before the query rows are known.
  struct Keys {
    u32x4 k[2][kQ];
    uint32_t v[8][kV / 2];
  } ka, kb;
  int page0, page1;
  const auto ask = [&](int k0) {
    page0 = page_of(a, row, k0, it.hi);
    page1 = page_of(a, row, k0 + 16, it.hi);
  };
  const auto load = [&](Keys& x, int k0) {
    const Cell cell[2] = {cell_of(a, page0, kvh, k0, it.hi, D),
                          cell_of(a, page1, kvh, k0 + 16, it.hi, D)};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const auto rk = rsrc(a.k, cell[b]);
#pragma unroll
      for (int j = 0; j < kQ; ++j)
        x.k[b][j] = bld16(rk, (n * a.key_stride + 32 * j + 8 * g) * 2);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const auto rv = rsrc(a.v, cell[b]);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int off = ((4 * g + i) * a.key_stride + kV * n) * 2;
        if constexpr (kV == 8) {
          const u32x4 w = bld16(rv, off);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.v[4 * b + i][e] = w[e];
        } else {
          const u32x2 w = bld8(rv, off);
#pragma unroll
          for (int e = 0; e < 2; ++e) x.v[4 * b + i][e] = w[e];
        }
      }
    }
    ask(k0 + kFewStep);
  };
  int k0 = it.lo + 32 * wv;
  ask(k0);
  if (k0 < it.hi) load(ka, k0);

  const Row x = query_row<TREE>(a, it, kvh, n);
  const NewKeys fresh = new_keys<TREE>(a, it);
  bool some = x.limit > it.lo && (!TREE || it.lo < fresh.past);
  u32x4 qf[kQ];
#pragma unroll
  for (int j = 0; j < kQ; ++j) qf[j] = u32x4{0, 0, 0, 0};
  if (n < it.rows) {
    const uint16_t* q = a.q + x.token * a.q_token + x.head * a.q_head + 8 * g;
#pragma unroll
    for (int j = 0; j < kQ; ++j) qf[j] = *reinterpret_cast<const u32x4*>(q + 32 * j) ^ a.flip;
  }
  int least = n < it.rows ? min(x.limit, fresh.past) : INT32_MAX;
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) least = min(least, __shfl_xor(least, d, 64));
  least = uniform(least);
  if (tid == 0) sh.bad = 0;

  float m = -INFINITY, l = 0.f;
  f32x4 acc[kV];
#pragma unroll
  for (int d = 0; d < kV; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  const auto use = [&](const Keys& y, int k0) {
    f32x4 s[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      s[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 0; j < kQ; ++j) s[b] = mfma16(Ty{}, y.k[b][j], qf[j], s[b]);
    }
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = s[i >> 2][i & 3] * a.c;
    if (k0 + 32 > least) {               // some row does not see all 32
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = k0 + 16 * (i >> 2) + 4 * g + (i & 3);
        bool seen = key < x.limit;
        if constexpr (TREE) {
          const bool in = sees<TREE>(a, fresh, x, key);
          seen = seen & in;
          some = some | seen;
        }
        t[i] = seen ? t[i] : -INFINITY;
      }
    }
    float mx = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, t[i]);
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    float ms = mx == -INFINITY ? 0.f : mx;
    const float al = exp2_(m - ms);
    m = mx;
    l *= al;
    ms -= Ty::kLift;
    u32x4 ph, pl;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = exp2_(t[2 * i] - ms), p1 = exp2_(t[2 * i + 1] - ms);
      l += p0 + p1;
      ph[i] = Ty::pack(p0, p1);
      pl[i] = Ty::pack(p0 - Ty::lo(ph[i]), p1 - Ty::hi(ph[i]));
    }
#pragma unroll
    for (int d = 0; d < kV; ++d) {
      u32x4 vt;
#pragma unroll
      for (int i = 0; i < 4; ++i) vt[i] = zip(y.v[2 * i][d / 2], y.v[2 * i + 1][d / 2], d & 1);
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[d][i] *= al;
      acc[d] = mfma16(Ty{}, vt, ph, acc[d]);
      acc[d] = mfma16(Ty{}, vt, pl, acc[d]);
    }
  };
  if constexpr (AHEAD) {
    while (k0 < it.hi) {
      if (k0 + kFewStep < it.hi) load(kb, k0 + kFewStep);
      use(ka, k0);
      k0 += kFewStep;
      if (k0 >= it.hi) break;
      if (k0 + kFewStep < it.hi) load(ka, k0 + kFewStep);
      use(kb, k0);
      k0 += kFewStep;
    }
  } else {
    for (; k0 < it.hi; k0 += kFewStep) {
      use(ka, k0);
      if (k0 + kFewStep < it.hi) load(ka, k0 + kFewStep);
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (g == 0) sh.m[wv][n] = m, sh.l[wv][n] = l;
  if constexpr (TREE) {
    uint64_t w = __ballot(some);
    w |= w >> 32;
    w |= w >> 16;
    if (lane == 0) sh.most[wv] = (int)w & 0xffff;
  }
  // acc[d][i] is the output's dimension kV (4 g + i) + d of row n; in LDS the
  // 16-byte units of a row are turned by its number
  const auto place = [&](int w, int r, int unit) {
    return (w < 2 ? o01 : o23) + ((w & 1) * kFew + r) * (D / 4) + (unit ^ r);
  };
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int d = 0; d < kV; d += 4)
      *place(wv, n, (kV * (4 * g + i) + d) / 4) =
          f32x4{acc[d][i], acc[d + 1][i], acc[d + 2][i], acc[d + 3][i]};
  __syncthreads();
  const int i = tid >> 4, e = (tid & 15) * kV;
  if (i < it.rows) {
    const Row y = query_row<TREE>(a, it, kvh, i);
    float M = sh.m[0][i];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, sh.m[w][i]);
    const float Ms = M == -INFINITY ? 0.f : M;
    float L = 0.f, o[kV] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2_(sh.m[w][i] - Ms);
      L = fmaf(f, sh.l[w][i], L);
#pragma unroll
      for (int d = 0; d < kV; d += 4) {
        const f32x4 v = *place(w, i, (e + d) / 4);
#pragma unroll
        for (int c = 0; c < 4; ++c) o[d + c] = fmaf(f, v[c], o[d + c]);
      }
    }
    bool any = y.limit > it.lo;
    if constexpr (TREE) any = (sh.most[0] | sh.most[1] | sh.most[2] | sh.most[3]) >> i & 1;
    if (M == -INFINITY && any) L = NAN;
    bool fine = true;
#pragma unroll
    for (int d = 0; d < kV; ++d) fine = fine && fabsf(o[d]) < INFINITY;
    if (!fine) atomicOr(&sh.bad, 1 << i);
    if (it.part < 0) {
      store_out<Ty, kV>(a.out + y.token * a.out_token + y.head * a.out_head + e, o,
                        any ? 1.f / L : 0.f);
    } else {
      const int64_t at = ((int64_t)it.part + i) * a.kv_heads + kvh;
      if (e == 0) a.pm[at] = M - Ty::kLift, a.pl[at] = L;
      store_part<kV>(a.po + at * D + e, o);
    }
  }
  __syncthreads();
  for (int b = wv; b < it.rows; b += kWaves)
    if (sh.bad >> b & 1) careful_row<Ty, D, TREE>(a, it, kvh, b);
}

// The few items of a step that can have no others.
template <class Ty, int D, bool TREE>
__global__ __launch_bounds__(kNT, 3) void few_kernel(AttnArgs a) {
  __shared__ f32x4 o01[2 * kFew * D / 4], o23[2 * kFew * D / 4];
  __shared__ FewShared sh;
  // (the grid covers the items' cap, so the item may be read beside their number)
  const int item = blockIdx.x / a.kv_heads, first = a.head->few;
  if (item >= first + a.head->later) return;
  const Item it = item < first ? a.few[item] : a.last_few[first - item];
  few_item<Ty, D, false, TREE>(a, it, blockIdx.x % a.kv_heads, sh, o01, o23);
}

// Items of up to 128 rows: prompts, and prefixes that many rows share.  A wavefront
// has 32 rows; K and V go through LDS, 64 keys at a time, two buffers, loaded there
// directly: the next keys are on their way while the present ones are used.  Rows
// stay rows in LDS, their 16-byte units turned by the row number, which the loaders'
// addresses do: for K by row mod 16, so that a read of one unit of 32 rows meets no
// bank twice; for V in steps of four units, for reads that transpose (16 lanes take
// 16 dimensions of four keys and each gets one dimension's four).
// The weights are formed against the row's present maximum before it is known
// whether that still stands: it is only raised, the output rescaled and the weights
// formed again, if a lane's sum of 32 passes kBar (bf16 2^13; fp16 2^16, above which
// a weight becomes infinite and the sum with it).  So no maximum is looked for in
// most steps, and no weight is more than its type holds.
// A request's own keys (more than 16 rows): the weights enter the product with V as
// one value of the type and are summed as rounded so.  A second product for the rest
// would add half to the work that bounds the kernel (5 prompts of 1500..5000 tokens x
// 32 heads: 600 us, 815 with it; 32 of 1..512 x 64, fp16: 371, 498); with one, the
// output is off by 1.4 times its own rounding (2.3e-3 of its norm in bf16, 1.66e-3 with
// two).  TWO, for a prefix that requests share: two values, as in a few item, so that
// a request's weights do not count to fewer bits for the company that it is in (256
// requests in 6 groups x 64 heads over 8, both kernels: 180 us, 175 with one).
// Bound by the matrix units and what they cannot hide: for 64 keys and 32 rows 32
// products (1024 cycles), 64 vector instructions and 32 exponentials (512), 64 reads
// of LDS (about 600).  64 keys x 128 rows, two work groups on every compute unit:
// 2.1 us a step, of which products alone take 1.4 (1029 TFLOP/s where K and V come
// from L2; 16 requests of 256 tokens behind 8192 keys, 32 heads).  With the keys
// through registers into LDS and V transposed there 2.4 us; with a maximum each step
// and a sum by additions 2.7; eight wavefronts a work group in two phases, one
// side's products beside the other's exponentials, 2.8.
// Schedules n times P products, each time fed by r reads from LDS, four times' reads
// ahead.
template <int N, int R, int P = 1>
__device__ __forceinline__ void feed() {
  constexpr int kAhead = 4;
  __builtin_amdgcn_sched_group_barrier(0x100, R * kAhead, 0);
#pragma unroll
  for (int i = 0; i < N - kAhead; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, P, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, P * kAhead, 0);
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_quad;
typedef __attribute__((address_space(3))) void* lds_ptr;

// Four 16-bit values of a lane's column: lane i of each 16 names the address of four
// values of row i / 4 (columns 4 (i % 4)..), and gets column i of the four rows.
__device__ __forceinline__ u32x2 read_columns(const uint16_t* p) {
  return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_quad)p));
}

// Waits for this wavefront's loads (those into LDS among them).
__device__ __forceinline__ void loads_done() { __builtin_amdgcn_s_waitcnt(0x0f70); }

template <class Ty, int D, bool TWO, bool TREE>
__device__ __forceinline__ void tile_item(const AttnArgs& a, const Item& it, int kvh,
                                          int* s_most, u32x4* s_k0, u32x4* s_k1, u32x4* s_v0,
                                          u32x4* s_v1, int* s_n0, int* s_n1) {
  constexpr int kQ = D / 16;                // products over a row
  constexpr int kV = D / 32;                // tiles of the output's dimensions
  constexpr int kU = D / 8;                 // 16-byte units of a row
  constexpr int kRowsPer = kNT / kU;        // K rows loaded at a time
  constexpr int kKL = kTileStep / kRowsPer; // K units per thread
  if (it.rows <= 0) return;
  const int tid = threadIdx.x, lane = tid & 63, wv = uniform(tid >> 6);
  const int n = lane & 31, h = lane >> 5;
  // (the first pages, asked for beside the rows)
  const int32_t* row = a.table + (int64_t)it.req * a.max_pages;
  int page = 0, at_lo = 0, at_hi = 0, bytes = 0;
  const auto ask = [&](int k0) { page = row[min(k0 + 16 * lane, it.hi - 1) >> a.log_page]; };
  ask(it.lo);
  const Row x = query_row<TREE>(a, it, kvh, 32 * wv + n);
  const NewKeys fresh = new_keys<TREE>(a, it);
  bool any = x.limit > it.lo && (!TREE || it.lo < fresh.past);
  const bool mine = 32 * wv + n < it.rows;
  u32x4 qf[kQ];
#pragma unroll
  for (int j = 0; j < kQ; ++j) qf[j] = u32x4{0, 0, 0, 0};
  if (mine) {
    const uint16_t* q = a.q + x.token * a.q_token + x.head * a.q_head + 8 * h;
#pragma unroll
    for (int j = 0; j < kQ; ++j) qf[j] = *reinterpret_cast<const u32x4*>(q + 16 * j) ^ a.flip;
  }
  int most = x.limit, least = mine ? min(x.limit, fresh.past) : INT32_MAX;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    most = max(most, __shfl_xor(most, d, 64));
    least = min(least, __shfl_xor(least, d, 64));
  }
  most = uniform(most);                     // of this wavefront
  least = uniform(least);
  if (lane == 0) s_most[wv] = most;
  __syncthreads();
  int end = s_most[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) end = max(end, s_most[w]);
  end = uniform(end);
  const int tiles = (end - it.lo + kTileStep - 1) / kTileStep;
  const int my = (most - it.lo + kTileStep - 1) / kTileStep;

  // Where 16 keys lie is found out for 64 times 16 keys at once, a lane each
  // (their pages are asked for 16 steps ahead), and read from the lanes.
  const auto locate = [&](int k0) {
    const int key = k0 + 16 * lane;
    const bool ok = page >= 0 && page < a.n_pages && key < end;
    const int64_t at = (ok ? page : 0) * a.page_stride + kvh * a.head_stride +
                       (int64_t)(key & ((1 << a.log_page) - 1)) * a.key_stride;
    at_lo = (int)at, at_hi = (int)(at >> 32);
    bytes = ok ? ((min(end - key, 16) - 1) * a.key_stride + D) * 2 : 0;
    ask(k0 + 1024);
  };
  const auto cell = [&](int j) {
    Cell c;
    c.at = (int64_t)(uint32_t)__builtin_amdgcn_readlane(at_lo, j) |
           (int64_t)__builtin_amdgcn_readlane(at_hi, j) << 32;
    c.bytes = __builtin_amdgcn_readlane(bytes, j);
    return c;
  };
  const auto turn_v = [](int rw) { return (D == 128 ? rw & 3 : (rw >> 1) & 1) << 2; };
  // Rows kr + i kRowsPer, place ku of the row in LDS; a load's rows lie in 16 keys of
  // one page.
  const int kr = tid / kU, ku = tid % kU;
  const int kg = uniform(kr >> 4), ko = kr & 15;
  const int off_k = (ko * a.key_stride + 8 * (ku ^ (kr & (kU - 1)))) * 2;
  const int off_v = (ko * a.key_stride + 8 * (ku ^ turn_v(kr))) * 2;
  const auto fetch = [&](int t, u32x4* sk, u32x4* sv, int* sn) {
    if ((t & 15) == 0) locate(it.lo + t * kTileStep);
    if constexpr (TREE) {
      // the intervals of 64 keys, firsts and lasts (what is none of the step's tokens
      // reads zero, and is cached or behind the end)
      if (wv == 0 && it.lo + (t + 1) * kTileStep > fresh.past) {
        const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<int2*>(a.span), 0, a.T * 8,
                                                         kRsrcWord3);
        const int off = (it.lo + t * kTileStep + lane - fresh.shift) * 8;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)sn, 4, off, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_ptr)(sn + 64), 4, off + 4, 0, 0, 0);
      }
    }
    const int j0 = 4 * (t & 15);
#pragma unroll
    for (int i = 0; i < kKL; ++i) {
      const Cell c = cell(j0 + kg + i * (kRowsPer / 16));
      const int to = (i * kRowsPer + wv * (kRowsPer / kWaves)) * kU;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(a.k, c), (lds_ptr)(sk + to), 16, off_k, 0, 0,
                                               0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc(a.v, c), (lds_ptr)(sv + to), 16, off_v, 0, 0,
                                               0);
    }
  };

  // (a row that sees none of the item's keys never asks for a maximum, a row without
  // one yet always)
  const float first = x.limit > it.lo ? -1.f : INFINITY;
  float m = -INFINITY, l = 0.f, bar = first;
  f32x16 acc[kV];
#pragma unroll
  for (int d = 0; d < kV; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[d][i] = 0.f;
  if (tiles > 0) {
    fetch(0, s_k0, s_v0, s_n0);
    loads_done();
  }
  __syncthreads();
  const auto step = [&](int t, const u32x4* sk, const u32x4* sv, const int* sn, u32x4* nk,
                        u32x4* nv, int* nn) {
    const int k0 = it.lo + t * kTileStep;
    if (t + 1 < tiles) fetch(t + 1, nk, nv, nn);
    if (t < my) {
      const u32x4* kp = sk + n * kU;
      const int kx = h ^ (n & (kU - 1));
      const int vi = lane & 15, vrow = 4 * h + (vi >> 2);
      const uint16_t* vp = reinterpret_cast<const uint16_t*>(sv) + vrow * D +
                           16 * (lane >> 4 & 1) + 4 * (vi & 3);
      // s[b][i] is key 32 b + 8 (i / 4) + 4 h + i % 4 of row n
      f32x16 s[2];
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
      for (int j = 0; j < kQ; ++j)
#pragma unroll
        for (int b = 0; b < 2; ++b)
          s[b] = mfma32(Ty{}, kp[b * 32 * kU + (kx ^ (2 * j))], qf[j], s[b]);
      feed<2 * kQ, 1>();
      __builtin_amdgcn_sched_barrier(0);
      if (k0 + kTileStep > least) {
        const int lim = x.limit - k0 - 4 * h;
        if (!TREE || k0 + kTileStep <= fresh.past) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              s[b][i] = 32 * b + 8 * (i >> 2) + (i & 3) < lim ? s[b][i] : -INFINITY;
          if constexpr (TREE) any = any || lim > 0;
        } else {
          // (four keys at a time, and the comparisons with the limit made here: else the
          // masks of all keys are held in scalar registers, and what the loop needs there
          // is moved away and back in every step)
          int cached = fresh.past - k0 - 4 * h, own = lim;
          asm volatile("" : "+v"(cached), "+v"(own));
          const i32x4* np = reinterpret_cast<const i32x4*>(sn) + h;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const i32x4 first = np[2 * j], last = np[16 + 2 * j];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int at = 8 * j + e;
              const bool seen = (at < own) & ((at < cached) | ((first[e] <= x.number) &
                                                               (x.number <= last[e])));
              const int i = 4 * (j & 3) + e;
              s[j >> 2][i] = seen ? s[j >> 2][i] : -INFINITY;
              any |= seen;
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      u32x4 p[4], rest[TWO ? 4 : 1];
      const auto weights = [&]() {
        const float ms = (m == -INFINITY ? 0.f : m) - Ty::kTileLift;
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float p0 = exp2_(fmaf(s[b][2 * i], a.c, -ms)),
                        p1 = exp2_(fmaf(s[b][2 * i + 1], a.c, -ms));
            const uint32_t w = Ty::pack(p0, p1);
            p[2 * b + (i >> 2)][i & 3] = w;
            if constexpr (TWO) {
              rest[2 * b + (i >> 2)][i & 3] = Ty::pack(p0 - Ty::lo(w), p1 - Ty::hi(w));
              sum0 += p0, sum1 += p1;
            } else {
              if (i & 1) sum1 = Ty::sum2(w, sum1);
              else sum0 = Ty::sum2(w, sum0);
            }
          }
        return sum0 + sum1;
      };
      float sum = weights();
      if (__any(sum > bar)) {
        float mx = m;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[b][i] * a.c);
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float ms = mx == -INFINITY ? 0.f : mx;
        const float al = exp2_(m - ms);
        m = mx;
        bar = m == -INFINITY ? first : Ty::kBar;
        l *= al;
#pragma unroll
        for (int d = 0; d < kV; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[d][i] *= al;
        sum = weights();
      }
      l += sum;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int d = 0; d < kV; ++d) {
          const uint16_t* v = vp + 16 * b * D + ((32 * d) ^ (turn_v(vrow) * 8));
          const u32x2 v0 = read_columns(v), v1 = read_columns(v + 8 * D);
          const u32x4 vt = {v0[0], v0[1], v1[0], v1[1]};
          acc[d] = mfma32(Ty{}, vt, p[b], acc[d]);
          if constexpr (TWO) acc[d] = mfma32(Ty{}, vt, rest[b], acc[d]);
        }
      feed<4 * kV, 2, TWO ? 2 : 1>();
      __builtin_amdgcn_sched_barrier(0);
    }
    loads_done();
    __syncthreads();
  };
  for (int t = 0; t < tiles; t += 2) {
    step(t, s_k0, s_v0, s_n0, s_k1, s_v1, s_n1);
    if (t + 1 < tiles) step(t + 1, s_k1, s_v1, s_n1, s_k0, s_v0, s_n0);
  }
  if (32 * wv >= it.rows) return;
  const AttnArgs z = args_again();
  l += __shfl_xor(l, 32, 64);
  if constexpr (TREE) {
    const int other = __shfl_xor((int)any, 32, 64);   // (by all lanes)
    any = any || other;
  }
  if (m == -INFINITY && any) l = NAN;
  // acc[d][i] is the output's dimension 32 d + 8 (i / 4) + 4 h + i % 4 of row n
  bool fine = true;
#pragma unroll
  for (int d = 0; d < kV; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) fine = fine && fabsf(acc[d][i]) < INFINITY;
  // (a row's two lanes agree on it; careful_row's lanes, which are others, write it then)
  uint64_t bad = __ballot(mine && !fine);
  bad = (bad | bad >> 32) & 0xffffffffu;
  if (mine && !(bad >> n & 1)) {
    const float inv = any ? 1.f / l : 0.f;
    const int64_t at = ((int64_t)it.part + 32 * wv + n) * z.kv_heads + kvh;
    if (it.part >= 0 && h == 0) z.pm[at] = m - Ty::kTileLift, z.pl[at] = l;
#pragma unroll
    for (int d = 0; d < kV; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int e = 32 * d + 2 * i + 4 * h;
        const float o[4] = {acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
        if (it.part < 0)
          store_out<Ty, 4>(z.out + x.token * z.out_token + x.head * z.out_head + e, o, inv);
        else
          store_part<4>(z.po + at * D + e, o);
      }
  }
  while (bad) {
    const int i = __builtin_ctzll(bad);
    bad &= bad - 1;
    careful_row<Ty, D, TREE>(z, it, kvh, 32 * wv + i);
  }
}

// Both kinds of items in one launch, the one bound by reading, the other by the
// matrix units.  They come in turn, kRun eights of each until one kind is used up:
// a run is a work group for every compute unit, and each holds two, so that a tile
// item has one of another kind beside it, and the long tile items have begun early.
// Both kernels, 256 requests in 6 groups: 179 us; in turn by each eight 202.  (With
// weights of one value over the prefixes 163; spread in proportion over the launch 193,
// all tile items first 163; a layer of 45 requests in 3 groups x 40 heads 93, 99, 102.)
// Eight work groups in a row are of one kind, so that a head's items, which share K and
// V, stay on one XCD where the key heads are a multiple of 8.
// (Two work groups on a compute unit at D 128, three at 64, to which the fp16 form is
// held: 5 registers spilt; prompts of 1500..5000 tokens: 351 us, 367 with two.)
constexpr uint32_t kRun = 32;
template <class Ty, int D, bool TREE>
__global__ __launch_bounds__(kNT, D == 64 ? 3 : 2) void items_kernel(AttnArgs a) {
  // (buffers by name: reads of one are seen not to meet the loads into the other)
  __shared__ u32x4 s_k0[kTileStep * D / 8], s_k1[kTileStep * D / 8];
  __shared__ u32x4 s_v0[kTileStep * D / 8], s_v1[kTileStep * D / 8];
  __shared__ i32x4 s_n0[TREE ? 32 : 1], s_n1[TREE ? 32 : 1];
  __shared__ FewShared sh;
  static_assert(sizeof(s_k0) == 2 * kFew * D * sizeof(float), "two wavefronts' outputs");
  const uint32_t turn = blockIdx.x >> 3, in = blockIdx.x & 7;
  const int few = a.head->few, all_few = few + a.head->later;
  const uint32_t tiles = ((uint32_t)a.head->tiles * a.kv_heads + 7) / 8;
  const uint32_t fews = ((uint32_t)all_few * a.kv_heads + 7) / 8;
  // (of each kind before this one, while both last)
  const uint32_t t0 = turn / (2 * kRun) * kRun + min(turn % (2 * kRun), kRun), f0 = turn - t0;
  bool tile = turn % (2 * kRun) < kRun;
  if (f0 > fews || (f0 == fews && !tile)) tile = true;
  else if (t0 > tiles || (t0 == tiles && tile)) tile = false;
  const uint32_t index =
      (tile ? turn - min(f0, fews) : turn - min(t0, tiles)) * 8 + in, item = index / a.kv_heads;
  const int kvh = index % a.kv_heads;
  // (the work groups behind the last item would pass the lists' ends)
  if (item >= (uint32_t)(tile ? a.head->tiles : all_few)) return;
  const Item it = tile ? a.tile[item]
                       : (int)item < few ? a.few[item] : a.last_few[few - (int)item];
  if (tile && it.gathered)
    tile_item<Ty, D, true, TREE>(a, it, kvh, sh.most, s_k0, s_k1, s_v0, s_v1,
                                reinterpret_cast<int*>(s_n0), reinterpret_cast<int*>(s_n1));
  else if (tile)
    tile_item<Ty, D, false, TREE>(a, it, kvh, sh.most, s_k0, s_k1, s_v0, s_v1,
                                reinterpret_cast<int*>(s_n0), reinterpret_cast<int*>(s_n1));
  else
    few_item<Ty, D, true, TREE>(a, it, kvh, sh, reinterpret_cast<f32x4*>(s_k0),
                          reinterpret_cast<f32x4*>(s_k1));
}

// Joins a row's partials: its request's own pieces, then its prefix's.  D / 4 lanes
// a row, 64 / (D / 4) rows (heads of one token) a wavefront; the weights of up to
// D / 4 pieces are found at once, a lane a piece, then eight partials are asked for
// at a time.  WIDE: four wavefronts for the same rows, a quarter of the pieces each,
// joined in a fixed order (few rows, cut into many pieces: one request of 30011 keys
// x 64 heads, 59 pieces: 10.0 us with a wavefront a row, about 5 so).  Rows that the
// items wrote themselves are left, rows without a key get zeros.  Bound by reading
// the partials, or by the latency of its chain of loads.
template <class Ty, int D, bool WIDE, int kAt>
__device__ __forceinline__ void merge_token(const AttnArgs& a, int t, int32_t per) {
  constexpr int kL = D / 4, kRows = 64 / kL;
  __shared__ f32x4 s_o[WIDE ? kWaves : 1][64];
  __shared__ float s_m[WIDE ? kWaves : 1][kRows], s_l[WIDE ? kWaves : 1][kRows];
  const int lane = threadIdx.x & 63, wv = uniform(threadIdx.x >> 6);
  const int e = lane % kL, sub = lane / kL;
  const int b = a.req[t], heads = a.kv_heads * a.r;
  // (read together, of some request where there is none)
  const int bb = min(max(b, 0), a.batch - 1);
  const int t0 = a.q_start[bb], t1 = a.q_start[bb + 1], R0 = (t - t0) * a.r;
  ReqInfo f = a.info[bb];
  if (b != bb || t < t0 || t >= t1) f.state = 0;
  if (f.state == 2) return;
  const int own = f.state == 1 ? f.splits : 0;
  const int pieces = own + (f.state == 1 && f.pre_part >= 0 ? f.pre_splits : 0);
  // (WIDE: wavefront w has every fourth piece from w on)
  const int mine = WIDE ? (pieces - wv + kWaves - 1) / kWaves : pieces;
  const int end = min(heads, ((int)blockIdx.y + 1) * per);
  for (int h0 = blockIdx.y * per + (WIDE ? 0 : wv * kRows); h0 < end;
       h0 += WIDE ? kRows : kWaves * kRows) {
    const int hd = min(h0 + sub, heads - 1), kvh = hd / a.r, R = R0 + hd % a.r;
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    const auto place = [&](int p) {
      const int64_t at =
          p < own ? (int64_t)f.part + (int64_t)p * f.rows
                  : (int64_t)f.pre_part + (int64_t)(p - own) * f.pre_rows + f.pre_row;
      return (at + R) * a.kv_heads + kvh;
    };
    const auto piece = [&](int i) { return WIDE ? i * kWaves + wv : i; };
    for (int p0 = 0; p0 < mine; p0 += kL) {
      const int n = min(kL, mine - p0);
      float m = -INFINITY, l = 0.f;
      if (e < n) {
        const int64_t at = place(piece(p0 + e));
        m = a.pm[at], l = a.pl[at];
      }
      // eight at a time (past the last: the last again, not added), the first before
      // the weights are known
      f32x4 x[kAt];
      const auto ask = [&](int j0) {
#pragma unroll
        for (int j = 0; j < kAt; ++j)
          x[j] = *reinterpret_cast<const f32x4*>(
              a.po + place(piece(p0 + min(j0 + j, n - 1))) * D + 4 * e);
      };
      ask(0);
      float mx = m;
#pragma unroll
      for (int d = kL / 2; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d, 64));
      mx = fmaxf(mx, M);
      const float ms = mx == -INFINITY ? 0.f : mx, al = exp2_(M - ms);
      if (M == -INFINITY && mx > -INFINITY) L = 0.f;
      M = mx;
      // a piece whose scores are all -inf (its l is NaN) weighs nothing beside
      // others; alone it makes the row NaN
      const float w = exp2_(m - ms);
      float s = m > -INFINITY ? w * l : mx > -INFINITY ? 0.f : l;
#pragma unroll
      for (int d = kL / 2; d; d >>= 1) s += __shfl_xor(s, d, 64);
      L = (M > -INFINITY ? L * al : L) + s;
      o *= al;
      for (int j0 = 0;;) {
#pragma unroll
        for (int j = 0; j < kAt; ++j) {
          const float wj = __shfl(w, min(j0 + j, n - 1), kL);
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = j0 + j < n ? fmaf(wj, x[j][i], o[i]) : o[i];
        }
        j0 += kAt;
        if (j0 >= n) break;
        ask(j0);
      }
    }
    if constexpr (WIDE) {
      if (e == 0) s_m[wv][sub] = M, s_l[wv][sub] = L;
      s_o[wv][lane] = o;
      __syncthreads();
      if (wv == 0) {
        M = s_m[0][sub];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) M = fmaxf(M, s_m[w][sub]);
        L = 0.f;
        o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          // (without a maximum: scores of -inf, which weigh nothing beside others, or NaN,
          // which the sums below still carry through a weight of zero)
          const float mw = s_m[w][sub], lw = s_l[w][sub];
          const float g = mw == -INFINITY ? 0.f : exp2_(mw - M);
          if (mw > -INFINITY) L = fmaf(g, lw, L);
          else if (M == -INFINITY) L += lw;
          const f32x4 x = s_o[w][lane];
#pragma unroll
          for (int i = 0; i < 4; ++i) o[i] = fmaf(g, x[i], o[i]);
        }
      }
      __syncthreads();
      if (wv != 0) continue;
    }
    if (h0 + sub >= end) continue;
    const bool none = M == -INFINITY && L == 0.f;
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = none ? 0.f : o[i] / L;
    store_out<Ty, 4>(a.out + t * a.out_token + hd * a.out_head + 4 * e, v, 1.f);
  }
}

// kAt: partials of a row on their way together.  Many rows hide the latency among
// themselves, so four, for which twice the wavefronts fit, are faster there (69 000 rows
// of 3 pieces 32 us with eight, 21 with four; 33 000 of 2 13.4 and 11.4); few rows, which
// have more pieces, take eight (1536 rows of 42 pieces 7.5 us, 9.0 with four).
constexpr int64_t kManyRows = 16384;
// Many tokens are kMergeTokens work groups' in turn, which look at 64 of theirs at
// once, a lane each, for those that have something to merge: few do among the tokens
// of long prompts, and those of one request lie with different work groups (16247
// tokens, none of them: 10.3 us with a work group each, 4.8 so).
constexpr int kMergeTokens = 2048;
template <class Ty, int D, bool WIDE, int kAt>
__global__ __launch_bounds__(kNT, kAt == 8 ? 4 : 8) void merge_kernel(AttnArgs a, int32_t per) {
  const int n = gridDim.x, lane = threadIdx.x & 63;
  if (n >= a.T) return merge_token<Ty, D, WIDE, kAt>(a, blockIdx.x, per);
  for (int t0 = blockIdx.x; t0 < a.T; t0 += 64 * n) {
    const int t = t0 + lane * n;
    bool any = false;
    if (t < a.T) {
      const int b = a.req[t], bb = min(max(b, 0), a.batch - 1);
      any = b != bb || t < a.q_start[bb] || t >= a.q_start[bb + 1] || a.info[bb].state != 2;
    }
    uint64_t mask = __ballot(any);
    while (mask) {
      const int i = __builtin_ctzll(mask);
      mask &= mask - 1;
      merge_token<Ty, D, WIDE, kAt>(a, t0 + i * n, per);
    }
  }
}

struct WsLayout {
  size_t l, o, bytes;
};
WsLayout ws_layout(const plora_attn_shape& s, const Bounds& b) {
  WsLayout w{};
  const size_t n = (size_t)b.part_rows * s.kv_heads;
  w.l = align256(n * 4);
  w.o = w.l + align256(n * 4);
  w.bytes = w.o + align256(n * s.head_dim * 4);
  return w;
}

// Work groups for the caps of both kinds, in eights.
int64_t item_blocks(const Bounds& b, int32_t kv_heads) {
  const int64_t few = (int64_t)b.few_cap * kv_heads, tiles = (int64_t)b.tile_cap * kv_heads;
  return ((few + 7) / 8 + (tiles + 7) / 8) * 8;
}

template <class Ty, int D, bool TREE>
plora_status launch(const AttnArgs& a, const Bounds& b, hipStream_t stream) {
  clear_error();
  if (b.tile_cap > 0)
    hipLaunchKernelGGL((items_kernel<Ty, D, TREE>), dim3(item_blocks(b, a.kv_heads)), dim3(kNT), 0,
                       stream, a);
  else
    hipLaunchKernelGGL((few_kernel<Ty, D, TREE>), dim3(b.few_cap * a.kv_heads), dim3(kNT), 0, stream,
                       a);
  plora_status st = launch_status();
  if (st != PLORA_OK) return st;
  // Few rows: a work group for what otherwise is a wavefront's.  Else heads of a
  // token per work group: all, or one pass where the tokens are few.
  const int heads = a.kv_heads * a.r, rows = 256 / D;
  if ((int64_t)a.T * heads <= 1024) {
    hipLaunchKernelGGL((merge_kernel<Ty, D, true, 8>), dim3(a.T, (heads + rows - 1) / rows),
                       dim3(kNT), 0, stream, a, rows);
  } else {
    const int per = a.T < kMergeTokens ? kWaves * rows : heads;
    const dim3 grid(std::min(a.T, kMergeTokens), (heads + per - 1) / per);
    if ((int64_t)a.T * heads <= kManyRows)
      hipLaunchKernelGGL((merge_kernel<Ty, D, false, 8>), grid, dim3(kNT), 0, stream, a, per);
    else
      hipLaunchKernelGGL((merge_kernel<Ty, D, false, 4>), grid, dim3(kNT), 0, stream, a, per);
  }
  return launch_status();
}

template <bool TREE>
plora_status run(const AttnArgs& a, const Bounds& b, int32_t head_dim, int32_t dtype,
                 hipStream_t stream) {
  if (dtype == PLORA_BF16)
    return head_dim == 128 ? launch<Bf16, 128, TREE>(a, b, stream)
                           : launch<Bf16, 64, TREE>(a, b, stream);
  return head_dim == 128 ? launch<Fp16, 128, TREE>(a, b, stream)
                         : launch<Fp16, 64, TREE>(a, b, stream);
}

// The checks of both entry points, and their launches; tree is null for the one.
plora_status attend(const void* q, int64_t q_token, int64_t q_head, const plora_kv_cache* cache,
                    const plora_kv_step* step, const plora_attn_shape* shape,
                    const plora_tree* tree, float scale, const void* plan, size_t plan_bytes,
                    void* out, int64_t out_token, int64_t out_head, void* ws, size_t ws_bytes,
                    hipStream_t stream) {
  if (!cache || !step || !shape) return PLORA_ERR_INVALID_ARG;
  if (tree && (tree->batch != step->batch || tree->T != step->T)) return PLORA_ERR_INVALID_ARG;
  const plora_attn_shape& s = *shape;
  const plora_kv_cache& c = *cache;
  if (s.batch < 0 || s.T < 0 || s.heads < 0 || s.kv_heads < 0 || s.max_q < 0 ||
      step->batch != s.batch || step->T != s.T || c.kv_heads != s.kv_heads ||
      c.head_dim != s.head_dim || c.page_size != step->page_size || c.n_pages < 0 ||
      step->max_pages < 0 || q_token < 0 || q_head < 0 || out_token < 0 || out_head < 0 ||
      c.page_stride < 0 || c.head_stride < 0 || c.token_stride < 0 || !std::isfinite(scale))
    return PLORA_ERR_INVALID_ARG;
  if (!shape_ok(s) || !page_size_ok(c.page_size) ||
      (c.dtype != PLORA_BF16 && c.dtype != PLORA_FP16))
    return PLORA_ERR_UNSUPPORTED;
  if (shape_empty(s)) return PLORA_OK;
  if (c.token_stride < s.head_dim) return PLORA_ERR_INVALID_ARG;
  if (q_token % 8 || q_head % 8 || out_token % 8 || out_head % 8 || c.page_stride % 8 ||
      c.head_stride % 8 || c.token_stride % 8 || c.token_stride >= kTokenStrideEnd)
    return PLORA_ERR_UNSUPPORTED;
  if (!q || !out || !plan || !ws || !step->pos || !step->req || !step->q_start ||
      (c.n_pages > 0 && (!c.k || !c.v)) || (step->max_pages > 0 && !step->table) ||
      (tree && (!tree->span || !tree->info)))
    return PLORA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(plan, 16) || !aligned(ws, 16) ||
      !aligned(c.k, 16) || !aligned(c.v, 16) ||
      (tree && (!aligned(tree->span, 8) || !aligned(tree->info, 8))))
    return PLORA_ERR_UNSUPPORTED;
  const Bounds b = bounds(s);
  const PlanLayout l = plan_layout(s, b);
  const WsLayout w = ws_layout(s, b);
  if (plan_bytes < l.bytes || ws_bytes < w.bytes) return PLORA_ERR_WORKSPACE_TOO_SMALL;
  if (item_blocks(b, s.kv_heads) > (int64_t)(UINT32_MAX / kNT))   // threads of a launch
    return PLORA_ERR_UNSUPPORTED;
  const char* p = static_cast<const char*>(plan);
  AttnArgs a{};
  a.q = static_cast<const uint16_t*>(q);
  a.k = static_cast<const uint16_t*>(c.k);
  a.v = static_cast<const uint16_t*>(c.v);
  a.q_token = q_token;
  a.q_head = q_head;
  a.out_token = out_token;
  a.out_head = out_head;
  a.page_stride = c.page_stride;
  a.head_stride = c.head_stride;
  a.key_stride = (int32_t)c.token_stride;
  a.n_pages = c.n_pages;
  a.log_page = log2_of(c.page_size);
  a.max_pages = step->max_pages;
  a.table = step->table;
  a.pos = step->pos;
  a.req = step->req;
  a.q_start = step->q_start;
  a.head = reinterpret_cast<const PlanHeader*>(p);
  a.few = reinterpret_cast<const Item*>(p + l.few);
  a.last_few = a.few + b.few_cap - 1;
  a.tile = reinterpret_cast<const Item*>(p + l.tile);
  a.order = reinterpret_cast<const int32_t*>(p + l.order);
  a.info = reinterpret_cast<const ReqInfo*>(p + l.req);
  a.batch = s.batch;
  a.T = s.T;
  a.r = b.r;
  a.kv_heads = s.kv_heads;
  // (a scale of 0 keeps masked scores at -inf with the smallest factor instead)
  a.c = std::max(std::fabs(scale) * 1.44269504f, 1.17549435e-38f);
  a.flip = scale < 0.f ? 0x80008000u : 0u;
  a.out = static_cast<uint16_t*>(out);
  char* wp = static_cast<char*>(ws);
  a.pm = reinterpret_cast<float*>(wp);
  a.pl = reinterpret_cast<float*>(wp + w.l);
  a.po = reinterpret_cast<float*>(wp + w.o);
  if (tree) {
    a.span = reinterpret_cast<const int2*>(tree->span);
    a.tree = reinterpret_cast<const int2*>(tree->info);
    return run<true>(a, b, s.head_dim, c.dtype, stream);
  }
  return run<false>(a, b, s.head_dim, c.dtype, stream);
}

}  // namespace
}  // namespace paged

extern "C" size_t plora_attn_paged_workspace_bytes(const plora_attn_shape* shape) {
  using namespace paged;
  if (!shape || !shape_ok(*shape) || shape_empty(*shape)) return 0;
  return ws_layout(*shape, bounds(*shape)).bytes;
}

extern "C" plora_status plora_attn_paged(const void* q, int64_t q_token, int64_t q_head,
                                         const plora_kv_cache* cache, const plora_kv_step* step,
                                         const plora_attn_shape* shape, float scale,
                                         const void* plan, size_t plan_bytes, void* out,
                                         int64_t out_token, int64_t out_head, void* ws,
                                         size_t ws_bytes, hipStream_t stream) {
  return paged::attend(q, q_token, q_head, cache, step, shape, nullptr, scale, plan, plan_bytes,
                       out, out_token, out_head, ws, ws_bytes, stream);
}

extern "C" plora_status plora_attn_tree(const void* q, int64_t q_token, int64_t q_head,
                                        const plora_kv_cache* cache, const plora_kv_step* step,
                                        const plora_attn_shape* shape, const plora_tree* tree,
                                        float scale, const void* plan, size_t plan_bytes,
                                        void* out, int64_t out_token, int64_t out_head, void* ws,
                                        size_t ws_bytes, hipStream_t stream) {
  if (!tree) return PLORA_ERR_INVALID_ARG;
  return paged::attend(q, q_token, q_head, cache, step, shape, tree, scale, plan, plan_bytes,
                       out, out_token, out_head, ws, ws_bytes, stream);
}

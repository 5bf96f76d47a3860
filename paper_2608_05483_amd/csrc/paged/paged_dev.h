// Shared by the kernels of include/plora_paged.h: 16-bit types, checks, status.
#ifndef PLORA_PAGED_DEV_H
#define PLORA_PAGED_DEV_H

#include <hip/hip_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "plora_paged.h"

namespace paged {

typedef int32_t i32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The two 16-bit types: unpacking, rounding to nearest even.  kLift: the power of two
// by which softmax weights are raised where they are held in the type, kTileLift where
// they may grow to kBar in sum before the maximum is looked at again: fp16 loses what
// is below 2^-25, and many keys of such weights beside one of weight 1 still count.
struct Bf16 {
  static constexpr float kLift = 0.f, kTileLift = 0.f, kBar = 8192.f;
  __device__ static __forceinline__ float lo(uint32_t w) { return __uint_as_float(w << 16); }
  __device__ static __forceinline__ float hi(uint32_t w) {
    return __uint_as_float(w & 0xffff0000u);
  }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  // c + the word's two values
  __device__ static __forceinline__ float sum2(uint32_t w, float c) {
    const bf16x2 one = {(__bf16)1.f, (__bf16)1.f};
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), one, c, false);
  }
};
struct Fp16 {
  static constexpr float kLift = 15.f, kTileLift = 8.f, kBar = 65536.f;
  __device__ static __forceinline__ float lo(uint32_t w) {
    return (float)__builtin_bit_cast(f16x2, w)[0];
  }
  __device__ static __forceinline__ float hi(uint32_t w) {
    return (float)__builtin_bit_cast(f16x2, w)[1];
  }
  __device__ static __forceinline__ uint32_t pack(float a, float b) {
    const f16x2 v = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  __device__ static __forceinline__ float sum2(uint32_t w, float c) {
    const f16x2 one = {(_Float16)1.f, (_Float16)1.f};
    return __builtin_amdgcn_fdot2(__builtin_bit_cast(f16x2, w), one, c, false);
  }
};

// A value moved over lanes, 0 where none comes (all lanes active).
template <int CTRL, int ROWS, class V>
__device__ __forceinline__ V moved(V x) {
  if constexpr (sizeof(V) == 4) {
    return __builtin_bit_cast(
        V, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, ROWS, 0xf, false));
  } else {
    const i32x2 w = __builtin_bit_cast(i32x2, x);
    const i32x2 y = {__builtin_amdgcn_update_dpp(0, w[0], CTRL, ROWS, 0xf, false),
                     __builtin_amdgcn_update_dpp(0, w[1], CTRL, ROWS, 0xf, false)};
    return __builtin_bit_cast(V, y);
  }
}
// Inclusive scan over a wavefront: within rows of 16 lanes, then over the rows.
template <class V, class Op>
__device__ __forceinline__ V wave_scan(V x, Op op) {
  x = op(x, moved<0x111, 0xf>(x));
  x = op(x, moved<0x112, 0xf>(x));
  x = op(x, moved<0x114, 0xf>(x));
  x = op(x, moved<0x118, 0xf>(x));
  x = op(x, moved<0x142, 0xa>(x));
  return op(x, moved<0x143, 0xc>(x));
}
struct Add {
  template <class V>
  __device__ V operator()(V a, V b) const { return a + b; }
};

inline bool aligned(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) % n) == 0; }
inline size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
constexpr bool pow2(int32_t v) { return v > 0 && (v & (v - 1)) == 0; }
inline bool page_size_ok(int32_t s) {
  return pow2(s) && s >= PLORA_PAGE_MIN && s <= PLORA_PAGE_MAX;
}
inline int32_t log2_of(int32_t v) {
  int32_t l = 0;
  while ((1 << l) < v) ++l;
  return l;
}

// The status of the launch just made (an error left by earlier HIP calls is
// cleared before it by clear_error), its error kept for plora_paged_last_hip_error.
inline std::atomic<int32_t> g_last_hip_error{0};
inline void clear_error() { (void)hipGetLastError(); }
inline plora_status launch_status() {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return PLORA_OK;
  g_last_hip_error.store((int32_t)e);
  return PLORA_ERR_HIP;
}

}  // namespace paged

#endif  // PLORA_PAGED_DEV_H

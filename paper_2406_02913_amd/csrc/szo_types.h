// Element types of the calls between the linear layers: loads to fp32 and stores from it, and sums over a few lanes.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "szo.h"

namespace szo {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

inline bool valid_type(int t) { return t == SZO_F32 || t == SZO_BF16 || t == SZO_F16; }
inline size_t type_bytes(int t) { return t == SZO_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

template <int TYPE> struct TypeOf;
template <> struct TypeOf<SZO_F32> { typedef float type; };
template <> struct TypeOf<SZO_BF16> { typedef __bf16 type; };
template <> struct TypeOf<SZO_F16> { typedef _Float16 type; };

// N neighbours as one vector; VEC: they lie at a multiple of their own size, else element by element.
template <int TYPE, int N, bool VEC>
__device__ __forceinline__ void load_f32(const void* base, int64_t at, float (&v)[N]) {
  typedef typename TypeOf<TYPE>::type T;
  typedef T vec __attribute__((ext_vector_type(N)));
  const T* p = static_cast<const T*>(base) + at;
  if constexpr (VEC) {
    const vec x = *reinterpret_cast<const vec*>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)x[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)p[i];
  }
}

template <int TYPE, int N, bool VEC>
__device__ __forceinline__ void store_f32(void* base, int64_t at, const float (&v)[N]) {
  typedef typename TypeOf<TYPE>::type T;
  typedef T vec __attribute__((ext_vector_type(N)));
  T* p = static_cast<T*>(base) + at;
  if constexpr (VEC) {
    vec x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    *reinterpret_cast<vec*>(p) = x;
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = (T)v[i];
  }
}

// Each lane's partner by a row permutation, without LDS: 1, 2: exclusive or; 4, 8: the mirror image in 8 or 16 lanes, which holds the
// other half's sum once the halves agree.
template <int CTRL>
__device__ __forceinline__ float lane_permuted(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}
// Sum over groups of L neighbouring lanes (4, 8, 16, 32 or 64), in every lane.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  v += lane_permuted<0xB1>(v);          // lanes 1 apart
  v += lane_permuted<0x4E>(v);          // 2 apart
  if constexpr (L >= 8) v += lane_permuted<0x141>(v);         // halves of 8
  if constexpr (L >= 16) v += lane_permuted<0x140>(v);
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (L >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
  if constexpr (L >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
  }
#endif
  return v;
}
template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  v = fmaxf(v, lane_permuted<0xB1>(v));
  v = fmaxf(v, lane_permuted<0x4E>(v));
  if constexpr (L >= 8) v = fmaxf(v, lane_permuted<0x141>(v));
  if constexpr (L >= 16) v = fmaxf(v, lane_permuted<0x140>(v));
#if defined(__HIP_DEVICE_COMPILE__)
  if constexpr (L >= 32) {
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
  if constexpr (L >= 64) {
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
  }
#endif
  return v;
}

}  // namespace szo

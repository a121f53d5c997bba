// wdp_common.h — element types, conversions, wide loads of any alignment and lane reductions of the policy's
// operators (include/wdp.h).  Included by the wdp_*.hip files only.
#ifndef WDP_COMMON_H
#define WDP_COMMON_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <type_traits>

#include "../../include/wdp.h"

namespace wdp {

using bf16 = __bf16;
using f16 = _Float16;

constexpr float kTiny = 7.888609052210118e-31f;  // 2^-100: the least maximum that a block's scale is made for
constexpr float kLargestE4M3 = 448.0f, kLargestE5M2 = 57344.0f;

inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline int size_of(int type) { return type == WDP_F32 ? 4 : type == WDP_BF16 || type == WDP_F16 ? 2 : 1; }
inline bool is_float_type(int type) { return type == WDP_F32 || type == WDP_BF16 || type == WDP_F16; }
inline bool is_8bit(int type) { return type == WDP_E4M3 || type == WDP_E5M2; }

// One launch.  Its status is the launch's own: hipGetLastError would answer with what any earlier call of the program left.
template <typename... P> int enqueue(void (*kernel)(P...), dim3 grid, int threads, hipStream_t stream, std::common_type_t<P>... args) {
  void* list[] = {&args...};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(unsigned(threads)), list, 0, stream) == hipSuccess ? WD_OK : WD_E_HIP;
}

template <typename T> __device__ __forceinline__ float to_float(T v) { return static_cast<float>(v); }
template <typename T> __device__ __forceinline__ T from_float(float v) { return static_cast<T>(v); }

// N adjacent elements at p (any alignment that the elements have) as floats, and back, in accesses of sixteen bytes: global
// memory takes those at any address, so whole vectors need no aligned rows.  (A struct of elements would be split into
// whatever pieces the compiler likes, hence the words.)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
template <typename V> struct __attribute__((packed, aligned(1))) Unaligned {
  V v;
};
template <typename V> __device__ __forceinline__ V load_raw(const void* p) { return static_cast<const Unaligned<V>*>(p)->v; }
template <typename V> __device__ __forceinline__ void store_raw(void* p, V v) { static_cast<Unaligned<V>*>(p)->v = v; }

template <typename T> __device__ __forceinline__ void widen(uint32_t w, float v[2]);
template <> __device__ __forceinline__ void widen<bf16>(uint32_t w, float v[2]) { v[0] = __uint_as_float(w << 16), v[1] = __uint_as_float(w & 0xFFFF0000u); }
template <> __device__ __forceinline__ void widen<f16>(uint32_t w, float v[2]) {
  typedef f16 f16x2 __attribute__((ext_vector_type(2)));
  const f16x2 h = __builtin_bit_cast(f16x2, w);
  v[0] = float(h[0]), v[1] = float(h[1]);
}
template <typename T> __device__ __forceinline__ uint32_t narrow(float a, float b) {
  typedef T Tx2 __attribute__((ext_vector_type(2)));
  const Tx2 h = {static_cast<T>(a), static_cast<T>(b)};
  return __builtin_bit_cast(uint32_t, h);
}

template <typename T, int N> __device__ __forceinline__ void load_vec(const T* __restrict__ p, float v[N]) {
  if constexpr (sizeof(T) == 4) {
    static_assert(N % 4 == 0, "whole accesses");
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x4 w = load_raw<u32x4>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i + e] = __uint_as_float(w[e]);
    }
  } else if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8) {
      const u32x4 w = load_raw<u32x4>(p + i);
#pragma unroll
      for (int e = 0; e < 4; ++e) widen<T>(w[e], v + i + 2 * e);
    }
  } else {
    static_assert(N == 4, "whole accesses");
    const u32x2 w = load_raw<u32x2>(p);
    widen<T>(w[0], v), widen<T>(w[1], v + 2);
  }
}
template <typename T, int N> __device__ __forceinline__ void store_vec(T* __restrict__ p, const float v[N]) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < N; i += 4) store_raw(p + i, u32x4{__float_as_uint(v[i]), __float_as_uint(v[i + 1]), __float_as_uint(v[i + 2]), __float_as_uint(v[i + 3])});
  } else if constexpr (N % 8 == 0) {
#pragma unroll
    for (int i = 0; i < N; i += 8)
      store_raw(p + i, u32x4{narrow<T>(v[i], v[i + 1]), narrow<T>(v[i + 2], v[i + 3]), narrow<T>(v[i + 4], v[i + 5]), narrow<T>(v[i + 6], v[i + 7])});
  } else {
    store_raw(p, u32x2{narrow<T>(v[0], v[1]), narrow<T>(v[2], v[3])});
  }
}

// The same where only the first n of the N elements exist (the others read as zero, and are not written).
template <typename T, int N> __device__ __forceinline__ void load_some(const T* __restrict__ p, int n, float v[N]) {
  if (n >= N) {
    load_vec<T, N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < n ? to_float<T>(p[i]) : 0.0f;
  }
}
template <typename T, int N> __device__ __forceinline__ void store_some(T* __restrict__ p, int n, const float v[N]) {
  if (n >= N) {
    store_vec<T, N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i < n) p[i] = from_float<T>(v[i]);
  }
}

// Four floats (in range, or NaN) to four 8-bit codes, to nearest even.
__device__ __forceinline__ uint32_t to_codes(int type, float a, float b, float c, float d) {
  int w = 0;
  if (type == WDP_E4M3) {
    w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
  } else {
    w = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, w, false);
    w = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, w, true);
  }
  return static_cast<uint32_t>(w);
}

// Exchanges inside a row of sixteen lanes, without LDS: with the neighbour, the pair, the mirror images in eight
// and in sixteen lanes.  After the k-th step of a reduction every lane holds the result of its 2^k lanes.
template <int CTRL> __device__ __forceinline__ float dpp(float v) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
constexpr int kDppPair = 0xB1, kDppQuad = 0x4E, kDppEight = 0x141, kDppSixteen = 0x140;

// Sum / maximum over aligned groups of LANES (a power of two up to 64) lanes; every lane gets it.
template <int LANES> __device__ __forceinline__ float group_sum(float v) {
  if (LANES >= 2) v += dpp<kDppPair>(v);
  if (LANES >= 4) v += dpp<kDppQuad>(v);
  if (LANES >= 8) v += dpp<kDppEight>(v);
  if (LANES >= 16) v += dpp<kDppSixteen>(v);
  if (LANES >= 32) v += __shfl_xor(v, 16);
  if (LANES >= 64) v += __shfl_xor(v, 32);
  return v;
}
// (fmax ignores a NaN: a block's scale is made from its other elements, and the NaN's code is NaN by itself)
template <int LANES> __device__ __forceinline__ float group_max(float v) {
  if (LANES >= 2) v = fmaxf(v, dpp<kDppPair>(v));
  if (LANES >= 4) v = fmaxf(v, dpp<kDppQuad>(v));
  if (LANES >= 8) v = fmaxf(v, dpp<kDppEight>(v));
  if (LANES >= 16) v = fmaxf(v, dpp<kDppSixteen>(v));
  if (LANES >= 32) v = fmaxf(v, __shfl_xor(v, 16));
  if (LANES >= 64) v = fmaxf(v, __shfl_xor(v, 32));
  return v;
}

}  // namespace wdp
#endif  // WDP_COMMON_H

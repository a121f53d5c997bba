// wdp_common.h — element types, conversions, wide loads of any alignment and lane reductions of the policy's
// operators (include/wdp.h).  Included by the wdp_*.hip files only.
#ifndef WDP_COMMON_H
#define WDP_COMMON_H

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

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

// A launch that failed leaves nothing behind in the runtime's error state.
inline int launched() {
  const hipError_t err = hipGetLastError();
  return err == hipSuccess ? WD_OK : WD_E_HIP;
}

template <typename T> __device__ __forceinline__ float to_float(T v) { return static_cast<float>(v); }
template <typename T> __device__ __forceinline__ T from_float(float v) { return static_cast<T>(v); }

// N elements at p (any alignment that the elements have) as floats.  Global memory takes a 16-byte access at any
// address, so whole vectors need no aligned rows.
template <typename T, int N> __device__ __forceinline__ void load_vec(const T* __restrict__ p, float v[N]) {
  struct __attribute__((packed, aligned(alignof(T)))) Raw {
    T e[N];
  };
  const Raw raw = *reinterpret_cast<const Raw*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = to_float<T>(raw.e[i]);
}
template <typename T, int N> __device__ __forceinline__ void store_vec(T* __restrict__ p, const float v[N]) {
  struct __attribute__((packed, aligned(alignof(T)))) Raw {
    T e[N];
  };
  Raw raw;
#pragma unroll
  for (int i = 0; i < N; ++i) raw.e[i] = from_float<T>(v[i]);
  *reinterpret_cast<Raw*>(p) = raw;
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

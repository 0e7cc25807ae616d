// Device side of the cache formats: 32-channel blocks with a shared power of
// two 2^(x - 127) and codes in E4M3 or E2M1 (see wavefilter.h).
#pragma once

#include "wavefilter.h"
#include "wf_device.hpp"

namespace wf {

// Eight channels of a row as fp32 numbers, and back (rounded to nearest even).
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]);
template <>
__device__ __forceinline__ void load8<bf16_t>(const bf16_t* p, float (&v)[8]) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}
template <>
__device__ __forceinline__ void load8<float>(const float* p, float (&v)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x4 w = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[4 * i + e] = w[e];
  }
}
template <typename T>
__device__ __forceinline__ void put8(T* p, const float (&v)[8]);
template <>
__device__ __forceinline__ void put8<bf16_t>(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                       pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
template <>
__device__ __forceinline__ void put8<float>(float* p, const float (&v)[8]) {
  reinterpret_cast<f32x4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
  reinterpret_cast<f32x4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// Exponent byte of a block whose largest magnitude has the fp32 bits amax:
// the smallest x >= 1 with amax <= top 2^(x - 127).  With top = m 2^k the
// exponent field of amax less k is that x, one more where its mantissa is
// above m's (448 = 1.75 2^8, 6 = 1.5 2^2).  255 for a NaN or an infinity.
template <int FMT>
__device__ __forceinline__ uint32_t block_exponent(uint32_t amax) {
  constexpr uint32_t above = FMT == WF_CACHE_E4M3 ? 0x1fffffu : 0x3fffffu;
  constexpr int k = FMT == WF_CACHE_E4M3 ? 8 : 2;
  const int x = (int)((amax + above) >> 23) - k;
  return amax >= 0x7f800000u ? 255u : (uint32_t)max(x, 1);
}

// The float 2^(127 - x), which takes a block's channels to its codes.
__device__ __forceinline__ float block_unscale(uint32_t x) {
  return __uint_as_float((254u - x) << 23);  // (x = 255: unused)
}
// The float a block's codes are multiplied by: 0 for x = 0, inf for 255 (codes 0).
__device__ __forceinline__ float block_scale(uint32_t x) { return __uint_as_float(x << 23); }

// Eight channels to codes: 8 bytes (E4M3) or the low 4 (E2M1).
template <int FMT>
__device__ __forceinline__ u32x2 encode8(const float (&v)[8]) {
  u32x2 c = {0u, 0u};
  if constexpr (FMT == WF_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
      c[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
    }
  } else {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], 1.0f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.0f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.0f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.0f, 3);
    c[0] = w;
  }
  return c;
}

// Eight codes (w: the low 4 bytes for E2M1) to their fp32 numbers times s.
template <int FMT>
__device__ __forceinline__ void decode8(u32x2 w, float s, float (&v)[8]) {
  if constexpr (FMT == WF_CACHE_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const hw_f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false);
      const hw_f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
      v[4 * i] = lo[0] * s;
      v[4 * i + 1] = lo[1] * s;
      v[4 * i + 2] = hi[0] * s;
      v[4 * i + 3] = hi[1] * s;
    }
  } else {
    const hw_f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 0);
    const hw_f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 1);
    const hw_f32x2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 2);
    const hw_f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], 1.0f, 3);
    v[0] = a[0] * s;
    v[1] = a[1] * s;
    v[2] = b[0] * s;
    v[3] = b[1] * s;
    v[4] = c[0] * s;
    v[5] = c[1] * s;
    v[6] = d[0] * s;
    v[7] = d[1] * s;
  }
}

}  // namespace wf

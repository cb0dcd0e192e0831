// Device-side helpers of the operators between two layers: 16-byte pieces of fp16 or bf16 rows
// as eight floats and back, sums over a few neighbouring lanes.
#pragma once
#include <hip/hip_runtime.h>

#include "owq_device.h"

namespace owq {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned long long u64;

struct F16 {
  static __device__ __forceinline__ float lo(u32 w) { return half_lo(w); }
  static __device__ __forceinline__ float hi(u32 w) { return half_hi(w); }
  static __device__ __forceinline__ u32 pack(float a, float b) {
    const h2_t h = {(_Float16)a, (_Float16)b};
    return __builtin_bit_cast(u32, h);
  }
};

struct BF16 {
  static __device__ __forceinline__ float lo(u32 w) { return __builtin_bit_cast(float, w << 16); }
  static __device__ __forceinline__ float hi(u32 w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
  static __device__ __forceinline__ u32 pack(float a, float b) {
    typedef __bf16 b2_t __attribute__((ext_vector_type(2)));
    const b2_t h = {(__bf16)a, (__bf16)b};       // to nearest, ties to even, NaN stays NaN
    return __builtin_bit_cast(u32, h);
  }
};

template <class E>
__device__ __forceinline__ void unpack8(u32x4 v, float *f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = E::lo(v[i]);
    f[2 * i + 1] = E::hi(v[i]);
  }
}

template <class E>
__device__ __forceinline__ u32x4 pack8(const float *f) {
  return (u32x4){E::pack(f[0], f[1]), E::pack(f[2], f[3]), E::pack(f[4], f[5]), E::pack(f[6], f[7])};
}

template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false));
}

// Sum over L = 1, 2, 4, 8 or 16 neighbouring lanes (every lane gets the total), in a fixed order.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
  if (L >= 2) v += dpp<0xB1>(v);     // lanes ^1
  if (L >= 4) v += dpp<0x4E>(v);     // lanes ^2
  if (L >= 8) v += dpp<0x141>(v);    // mirror in 8
  if (L >= 16) v += dpp<0x140>(v);   // mirror in 16
  return v;
}

template <int L>
__device__ __forceinline__ float lanes_max(float v) {
  if (L >= 2) v = fmaxf(v, dpp<0xB1>(v));
  if (L >= 4) v = fmaxf(v, dpp<0x4E>(v));
  if (L >= 8) v = fmaxf(v, dpp<0x141>(v));
  if (L >= 16) v = fmaxf(v, dpp<0x140>(v));
  return v;
}

// A value from another lane of the wave, `none` where there is no such lane: the six steps of a scan over 64 lanes
// (1, 2, 4 and 8 lanes down within rows of 16, then the last lane of a row to the next row, and of the lower half to the upper).
template <int STEP>
__device__ __forceinline__ u32 from_lane(u32 v, u32 none) {
  constexpr int ctrl = STEP == 0 ? 0x111 : STEP == 1 ? 0x112 : STEP == 2 ? 0x114 : STEP == 3 ? 0x118 : STEP == 4 ? 0x142 : 0x143;
  constexpr int rows = STEP == 4 ? 0xa : STEP == 5 ? 0xc : 0xf;
  return (u32)__builtin_amdgcn_update_dpp((int)none, (int)v, ctrl, rows, 0xf, false);
}
template <int STEP>
__device__ __forceinline__ u64 from_lane(u64 v, u64 none) {
  return (u64)from_lane<STEP>((u32)(v >> 32), (u32)(none >> 32)) << 32 | from_lane<STEP>((u32)v, (u32)none);
}
template <int STEP>
__device__ __forceinline__ float from_lane(float v, float none) {
  return __builtin_bit_cast(float, from_lane<STEP>(__builtin_bit_cast(u32, v), __builtin_bit_cast(u32, none)));
}
// Inclusive scan over the wave's lanes; the last lane holds the result over all of them.
template <class T, class F>
__device__ __forceinline__ T wave_scan(T v, T none, F &&f) {
  v = f(v, from_lane<0>(v, none));
  v = f(v, from_lane<1>(v, none));
  v = f(v, from_lane<2>(v, none));
  v = f(v, from_lane<3>(v, none));
  v = f(v, from_lane<4>(v, none));
  return f(v, from_lane<5>(v, none));
}

}  // namespace owq

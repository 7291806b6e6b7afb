// Rows in 16-byte vectors that may begin at any element, and sums over neighbouring lanes: what the operators on single rows
// (row_norm.hip, embed_rows.hip) share.
#pragma once
#include "operators.h"

namespace dc {

typedef unsigned short u16;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
// global loads and stores of gfx950 take any alignment: one instruction wherever a row begins
typedef u32x4 u32x4_any __attribute__((aligned(2), may_alias));
typedef u32x2 u32x2_any __attribute__((aligned(1), may_alias));
typedef unsigned u32_any __attribute__((aligned(1), may_alias));

template <typename T>
constexpr int kVector = 16 / (int)sizeof(T);     // values of 16 bytes

__device__ __forceinline__ void narrow(float x, float& y) { y = x; }
__device__ __forceinline__ void narrow(float x, u16& y) { y = to_bf16(x); }

// The vector of a row's columns c .. c + kVector - 1, zeros behind column C.
template <typename T, bool kFull>
__device__ __forceinline__ u32x4 load_vector(const T* row, int c, int C) {
  constexpr int kV = kVector<T>;
  if (kFull || c + kV <= C) return *reinterpret_cast<const u32x4_any*>(row + c);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int k = 0; k < kV; ++k)
    if (c + k < C) {
      const T x = row[c + k];
      if constexpr (sizeof(T) == 4) v[k] = __float_as_uint(x);
      else v[k / 2] |= (unsigned)x << (16 * (k & 1));
    }
  return v;
}
template <typename T>
__device__ __forceinline__ void store_vector(T* row, int c, int C, u32x4 v) {
  constexpr int kV = kVector<T>;
  if (c + kV <= C) {
    *reinterpret_cast<u32x4_any*>(row + c) = v;
    return;
  }
#pragma unroll
  for (int k = 0; k < kV; ++k)
    if (c + k < C) {
      if constexpr (sizeof(T) == 4) row[c + k] = __uint_as_float(v[k]);
      else row[c + k] = (u16)(v[k / 2] >> (16 * (k & 1)));
    }
}
__device__ __forceinline__ void unpack(float (&x)[4], u32x4 v, float) {
#pragma unroll
  for (int k = 0; k < 4; ++k) x[k] = __uint_as_float(v[k]);
}
__device__ __forceinline__ void unpack(float (&x)[8], u32x4 v, u16) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    x[2 * k] = __uint_as_float(v[k] << 16);
    x[2 * k + 1] = __uint_as_float(v[k] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 pack(const float (&x)[4], float) {
  return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
__device__ __forceinline__ u32x4 pack(const float (&x)[8], u16) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
}

// x of the lane that a DPP control names: within a row of 16 lanes, without LDS.
template <int kControl>
__device__ __forceinline__ float dpp(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kControl, 0xF, 0xF, true));
}
// The sum over `lanes` neighbours (a power of two up to 64, the same for the wave), in all of them.  kLanes: their number where it
// is known when the kernel is built, else 0.
template <int kLanes = 0>
__device__ __forceinline__ float lane_sum(float x, int lanes = kLanes) {
  if (kLanes ? kLanes > 1 : lanes > 1) x += dpp<0xB1>(x);            // quad_perm 1 0 3 2
  if (kLanes ? kLanes > 2 : lanes > 2) x += dpp<0x4E>(x);            // quad_perm 2 3 0 1
  if (kLanes ? kLanes > 4 : lanes > 4) x += dpp<0x141>(x);           // row_half_mirror
  if (kLanes ? kLanes > 8 : lanes > 8) x += dpp<0x140>(x);           // row_mirror
  if (kLanes ? kLanes > 16 : lanes > 16) {
    const u32x2 h = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  }
  if (kLanes ? kLanes > 32 : lanes > 32) {
    const u32x2 h = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    x = __uint_as_float(h[0]) + __uint_as_float(h[1]);
  }
  return x;
}

}  // namespace dc

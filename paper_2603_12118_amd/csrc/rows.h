// Rows of bf16 or fp32 as a lane takes them, eight values at a time, and groups of 32 values in 4 bits.
#pragma once
#include "common.h"

#include <type_traits>

namespace cs {

typedef unsigned int cu32x4 __attribute__((ext_vector_type(4)));
typedef float cf32x2 __attribute__((ext_vector_type(2)));
typedef float cf32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 cbf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack2_c(float a, float b) {
  const cf32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, cbf16x2));
}

template <bool ONCE, class T>
__device__ __forceinline__ T fetch(const T* p) {
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  else return *p;
}
template <bool ONCE, class T>
__device__ __forceinline__ void put(T v, T* p) {
  if constexpr (ONCE) __builtin_nontemporal_store(v, p);
  else *p = v;
}
// eight consecutive values of either type
template <bool BF16, bool ONCE>
__device__ __forceinline__ void load8(const void* base, int64_t at, float (&x)[8]) {
  if constexpr (BF16) {
    const cu32x4 u = fetch<ONCE>(reinterpret_cast<const cu32x4*>(static_cast<const bf16_t*>(base) + at));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  } else {
    const cf32x4* p = reinterpret_cast<const cf32x4*>(static_cast<const float*>(base) + at);
    const cf32x4 a = fetch<ONCE>(p), b = fetch<ONCE>(p + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}
template <bool BF16, bool ONCE>
__device__ __forceinline__ void store8(void* base, int64_t at, const float (&x)[8]) {
  if constexpr (BF16) {
    cu32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = pack2_c(x[2 * i], x[2 * i + 1]);
    put<ONCE>(u, reinterpret_cast<cu32x4*>(static_cast<bf16_t*>(base) + at));
  } else {
    cf32x4* p = reinterpret_cast<cf32x4*>(static_cast<float*>(base) + at);
    put<ONCE>(cf32x4{x[0], x[1], x[2], x[3]}, p);
    put<ONCE>(cf32x4{x[4], x[5], x[6], x[7]}, p + 1);
  }
}

// largest magnitude of the values of a group, eight in each of four lanes NEXT apart, as bits (NaN above infinity above every number)
template <int NEXT = 1>
__device__ __forceinline__ uint32_t group_max_bits(const float (&x)[8]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = max(m, (uint32_t)__shfl_xor((int)m, NEXT));
  return max(m, (uint32_t)__shfl_xor((int)m, 2 * NEXT));
}

// Eight codes of a lane's values and the group's scale byte.  The byte: adding a quarter to the mantissa carries into the
// exponent from 1.75 on.  The conversion instruction divides by the scale exactly, rounds to nearest even and saturates.
template <int NEXT = 1>
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], int& byte, bool& odd_values) {
  uint32_t m = group_max_bits<NEXT>(x);
  odd_values = m >= 0x7f800000u;
  if (odd_values) {               // (the four lanes of a group take this together)
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = x[i] != x[i] ? 0.f : fminf(fmaxf(x[i], -3.4028234663852886e38f), 3.4028234663852886e38f);
    m = group_max_bits<NEXT>(x);
  }
  byte = (int)((m + 0x200000u) >> 23) - 2;
  byte = byte < 2 ? 2 : byte > 252 ? 252 : byte;
  const float scale = __uint_as_float((uint32_t)byte << 23);
  uint32_t w = 0;
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], scale, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
}

__device__ __forceinline__ void values8(uint32_t w, int byte, float (&x)[8]) {
  const float scale = __uint_as_float((uint32_t)byte << 23);
  const cf32x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0), p1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
  const cf32x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2), p3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
  x[0] = p0.x; x[1] = p0.y; x[2] = p1.x; x[3] = p1.y; x[4] = p2.x; x[5] = p2.y; x[6] = p3.x; x[7] = p3.y;
}

// v of the lanes of a wave, summed: within rows of 16 by DPP, whose every step gives both sides the same sum, across them by two
// exchanges (an exchange goes through LDS)
template <class T>
__device__ __forceinline__ T wave_sum(T v) {
  auto with = [](T x, auto ctrl) {
    constexpr int C = decltype(ctrl)::value;
    if constexpr (sizeof(T) == 8) {
      const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(x), C, 0xf, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, __double2hiint(x), C, 0xf, 0xf, false);
      return x + __hiloint2double(hi, lo);
    } else {
      return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), C, 0xf, 0xf, false));
    }
  };
  v = with(v, std::integral_constant<int, 0xb1>());      // lanes 1 0 3 2
  v = with(v, std::integral_constant<int, 0x4e>());      // lanes 2 3 0 1
  v = with(v, std::integral_constant<int, 0x141>());     // half a row mirrored
  v = with(v, std::integral_constant<int, 0x140>());     // a row mirrored
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// codes 2 SEL, 2 SEL + 1 of a word, times 2^(byte - 127) where the byte is in bits 23..30 of `scale`: two bf16
template <int SEL>
__device__ __forceinline__ uint32_t widen2(uint32_t w, uint32_t scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, __uint_as_float(scale), SEL));
}
// byte B of w in bits 23..30
template <int B>
__device__ __forceinline__ uint32_t scale_of(uint32_t w) {
  return (B == 3 ? w >> 1 : w << (B == 3 ? 0 : 23 - 8 * B)) & 0x7f800000u;
}

}  // namespace cs

// Device side of the paged cache: codes and scales.
//
// 8 bits.  A scale is a power of two (or 0: a block of zeros), the least one with max|x| <= 448 s for e4m3
// and 127 s for int8 over the block's finite values.  A value is code * s: exact in bf16, whatever the
// code, while it is a normal number (e4m3's smallest code at scales below 2^-117 is not: it may become 0).
// A power of two costs e4m3 nothing (its precision does not depend on the scale) and int8 up to one bit of
// its range; in return a block whose scale grows with a later row moves its codes by whole binades, so that
// e4m3's normal numbers stay as they were, and the codes of given rows are the same on every path.
//
// 4 bits.  e2m1 codes, +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}, element 2 i in a byte's low half, and for 32 elements of a row
// a byte b: the least scale 2^(b - 127) with max|x| <= 6 2^(b - 127), 2 <= b <= 252.  With a scale for each row and
// 32 elements no code depends on other rows, so that rows can be written in any order.  The bounds keep every code but 0
// times its scale a normal finite number, in bf16 as in fp32: a row that a mask leaves out can hold any byte and adds
// 0 times it, 0.  The conversions from and to four bits take a scale's exponent alone.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"
#include "paged.h"

namespace kv {

typedef __bf16 __attribute__((ext_vector_type(2))) bf16x2_t;
typedef uint32_t __attribute__((ext_vector_type(2))) u32x2_t;
typedef uint32_t __attribute__((ext_vector_type(4))) u32x4_t;

// Two floats as a bf16 pair, rounded to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  bf16x2_t r;
  r[0] = (__bf16)a;
  r[1] = (__bf16)b;
  return __builtin_bit_cast(uint32_t, r);
}

// The scale of a block whose largest finite |x| has these bits.
template <int QT> __device__ __forceinline__ float block_scale(uint32_t amax_bits) {
  // amax = (1 + f) 2^(x - 127): 448 = 1.75 2^8, 127 = 1.984375 2^6
  constexpr int kTop = QT == kQtE4m3 ? 8 : 6;
  constexpr uint32_t kFrac = QT == kQtE4m3 ? 0x600000u : 0x7E0000u;
  if (amax_bits == 0) return 0.f;
  const int e = (int)(amax_bits >> 23) - kTop + ((amax_bits & 0x7FFFFFu) > kFrac ? 1 : 0);
  return __uint_as_float((uint32_t)max(e, 1) << 23);
}

// 1 / s (exact for a scale as block_scale gives it); 1 for 0, whose block has no finite value but 0.
__device__ __forceinline__ float inv_scale(float s) { return s > 0.f ? 1.f / s : 1.f; }

// Whether s is a scale as block_scale gives it, and every code times it is finite in bf16: 448 2^119, 127 2^121 (blocks of
// values near fp32's largest have a larger one, and 256 2^120 and 64 2^122 are 2^128).
template <int QT> __device__ __forceinline__ bool is_bf16_scale(float s) {
  const uint32_t u = __float_as_uint(s);
  return (u & 0x807FFFFFu) == 0 && s <= (QT == kQtE4m3 ? 0x1p119f : 0x1p121f);
}

// Four values in units of the scale as codes, rounded to nearest even.  kFinite: the values are finite and
// at most the largest code; else infinities saturate, and a NaN stays one in e4m3 and becomes 0 in int8.
template <int QT, bool kFinite> __device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  float x[4] = {a, b, c, d};
  if constexpr (QT == kQtE4m3) {
    uint32_t nan = 0;
    if constexpr (!kFinite) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        nan |= x[i] != x[i] ? 0xFFu << (8 * i) : 0u;
        x[i] = __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);
      }
    }
    uint32_t u = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    u = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], (int)u, true);
    return kFinite ? u : (u & ~nan) | (0x7F7F7F7Fu & nan);
  } else {
    int y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (!kFinite) x[i] = x[i] == x[i] ? __builtin_amdgcn_fmed3f(x[i], -127.f, 127.f) : 0.f;
      y[i] = (int)__builtin_rintf(x[i]);
    }
    const uint32_t lo = __builtin_amdgcn_perm((uint32_t)y[1], (uint32_t)y[0], 0x0C0C0400u);
    const uint32_t hi = __builtin_amdgcn_perm((uint32_t)y[3], (uint32_t)y[2], 0x04000C0Cu);
    return lo | hi;
  }
}

// Four codes as fp32.
template <int QT> __device__ __forceinline__ void decode4(uint32_t u, float (&f)[4]) {
  if constexpr (QT == kQtE4m3) {
    f[0] = __builtin_amdgcn_cvt_f32_fp8((int)u, 0);
    f[1] = __builtin_amdgcn_cvt_f32_fp8((int)u, 1);
    f[2] = __builtin_amdgcn_cvt_f32_fp8((int)u, 2);
    f[3] = __builtin_amdgcn_cvt_f32_fp8((int)u, 3);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(u >> (8 * i));
  }
}

// Codes 2 H and 2 H + 1 of a word times a power of two as a bf16 pair: exact, every code has at most 8
// significant bits.
template <int QT, int H> __device__ __forceinline__ uint32_t decode2_bf16(uint32_t u, float scale = 1.f) {
  if constexpr (QT == kQtE4m3) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, scale, H != 0));
  } else {
    const float a = (float)(int8_t)(u >> (16 * H)) * scale, b = (float)(int8_t)(u >> (16 * H + 8)) * scale;
    return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  }
}

// ---- 4 bits

constexpr int kGroup4 = 32;      // elements that share a scale
constexpr uint32_t kTop4 = 252;  // the largest scale byte

// The scale byte of elements whose largest finite |x| has these bits: 6 = 1.5 2^2.
__device__ __forceinline__ uint32_t scale_byte4(uint32_t amax_bits) {
  const int e = (int)(amax_bits >> 23) - 2 + ((amax_bits & 0x7FFFFFu) > 0x400000u ? 1 : 0);
  return (uint32_t)min(max(e, 2), (int)kTop4);
}
__device__ __forceinline__ float scale4(uint32_t byte) { return __uint_as_float(min(byte, kTop4) << 23); }

// Two bf16 values (no NaN) as codes in units of the scale, rounded to nearest even, past 6, 6, in the byte SEL of u.
template <int SEL> __device__ __forceinline__ uint32_t encode2_bf16(uint32_t u, uint32_t pair, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(u, __builtin_bit_cast(bf16x2_t, pair), scale, SEL);
}
__device__ __forceinline__ uint32_t encode8_bf16(const u32x4_t& x, float scale) {
  return encode2_bf16<3>(encode2_bf16<2>(encode2_bf16<1>(encode2_bf16<0>(0u, x[0], scale), x[1], scale), x[2], scale), x[3], scale);
}
// The same of two fp32 values.
template <int SEL> __device__ __forceinline__ uint32_t encode2_f32(uint32_t u, float a, float b, float scale) {
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(u, a, b, scale, SEL);
}
// The two codes of byte SEL times the scale as a bf16 pair, and as fp32.
template <int SEL> __device__ __forceinline__ uint32_t decode2_e2m1(uint32_t u, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(u, scale, SEL));
}
__device__ __forceinline__ u32x4_t decode8_e2m1(uint32_t u, float scale) {
  return u32x4_t{decode2_e2m1<0>(u, scale), decode2_e2m1<1>(u, scale), decode2_e2m1<2>(u, scale), decode2_e2m1<3>(u, scale)};
}

template <int QT> __device__ __forceinline__ u32x2_t decode4_bf16(uint32_t u, float scale = 1.f) {
  return u32x2_t{decode2_bf16<QT, 0>(u, scale), decode2_bf16<QT, 1>(u, scale)};
}

}  // namespace kv

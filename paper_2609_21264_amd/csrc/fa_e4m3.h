// Tiles of 8-bit floats (OCP e4m3) in LDS: their swizzles, and widening fragments to 16 bits. Internal; included by the
// kernel sources only.
#pragma once

#include "fa_device.h"

namespace fa {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// XOR swizzles of the 16-byte chunks of an 8-bit row, so that lanes served together hit different 16-byte
// bank slots: K rows are read whole chunks at a time by 16 rows at once; V by 8 keys x two chunks.
template <int CH>
__device__ __forceinline__ int k8_swizzle(int row) { return CH % 8 == 0 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int CH>
__device__ __forceinline__ int v8_swizzle(int row) { return CH % 8 == 0 ? 2 * ((row >> 1) & 3) : 2 * ((row >> 2) & 1); }

// Probabilities over e4m3 tiles are held times 2^7 (row sums too), by a reference maximum that much lower: fp16 has steps of
// 2^-24 below 2^-14, and keys that lie 2^-25 and more under a row's largest would be lost however many they are (131 072 of
// them at 2^-25.5: O 0 instead of 0.0028 max|V|); so they count down to 2^-32. At the top, 2^8 over the reference
// becomes 2^15, within fp16.
constexpr float kE4m3PLog2 = 7.f;

// Eight e4m3 (two registers) as bf16 or fp16, exactly.
__device__ __forceinline__ bf16x8 widen_bf16(uint32_t a, uint32_t b) {
  return bit_cast<bf16x8>(u32x4{bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false)),
                                bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true)),
                                bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false)),
                                bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true))});
}
__device__ __forceinline__ f16x8 widen_f16(uint32_t a, uint32_t b) {
  return bit_cast<f16x8>(u32x4{bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false)),
                               bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true)),
                               bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false)),
                               bit_cast<uint32_t>(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true))});
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  f32x2 f = {lo, hi};
  return bit_cast<uint32_t>(__builtin_convertvector(f, f16x2));  // RNE
}

}  // namespace
}  // namespace fa

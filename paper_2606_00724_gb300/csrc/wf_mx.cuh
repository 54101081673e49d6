// Codes of a quantised cache: blocks of 32 channels that share a power of two,
// elements in E4M3 or E2M1 (see wf_cache_quantize).
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "wf_internal.cuh"

namespace wf {

constexpr int kMxBlock = 32;

// The scale byte of a block whose largest magnitude has the fp32 bits `top`:
// with top = (1 + f) 2^E the least e with top <= 448 2^e is E - 8 for
// 1 + f <= 1.75 and E - 7 above it (6 2^e: E - 2 for 1 + f <= 1.5, E - 1 above);
// 255 for a NaN or an infinity, whose bits are above those of every number.
template <bool FP4>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const int e = FP4 ? (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u)
                    : (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u);
  return (uint32_t)max(e, 0);
}
// 2^-e of a scale byte below 255 (at most 253 - 1, so never subnormal).
__device__ __forceinline__ float mx_inv_scale(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// 2^e of a scale byte: byte 0 is the subnormal 2^-127, byte 255 NaN.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
  return __uint_as_float(byte == 0 ? 0x400000u : byte == 255 ? 0x7fffffffu : byte << 23);
}

// Two codes from two fp32 values (round to nearest even; nothing saturates).
template <bool FP4>
__device__ __forceinline__ uint32_t mx_encode2(float a, float b) {
  if (FP4) return __nv_cvt_float2_to_fp4x2(make_float2(a, b), __NV_E2M1, cudaRoundNearest);
  return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
}
// Two fp32 values from two codes (in the low bits of c).
template <bool FP4>
__device__ __forceinline__ float2 mx_decode2(uint32_t c) {
  const __half2_raw h = FP4 ? __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)c, __NV_E2M1)
                            : __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)c, __NV_E4M3);
  return __half22float2(__half2(h));
}

// Codes widened to pairs of bf16, exactly.  A code's exponent and mantissa bits
// placed in those of a bf16 number, whose bias is larger by 120 (E4M3) or 126
// (E2M1), stand for code x 2^-120 (2^-126), subnormal codes for subnormal
// numbers, so one product with 2^(120 + e) is the value.  That factor is a
// number for scale bytes up to kMxOne; for larger ones the rest of the scale is
// a second product.
template <bool FP4> constexpr uint32_t kMxOne = FP4 ? 128 : 134;
template <bool FP4>
__device__ __forceinline__ uint32_t mx_factor(uint32_t byte) {
  return ((min(byte, kMxOne<FP4>) + (FP4 ? 126u : 120u)) << 7) * 0x10001u;
}
template <bool FP4>
__device__ __forceinline__ uint32_t mx_second_factor(uint32_t byte) {
  return byte == 255 ? 0x7fff7fffu : ((max(byte, kMxOne<FP4>) - kMxOne<FP4> + 127u) << 7) * 0x10001u;
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// Pair i (channels 2 i, 2 i + 1) of a word of codes, before the factor: 2 pairs
// of E4M3 or 4 of E2M1.
template <bool FP4>
__device__ __forceinline__ uint32_t mx_pair(uint32_t w, int i) {
  if (FP4) {
    const uint32_t b = __byte_perm(w, 0, 0x4440 + i);
    return ((b * 0x00040040u) & 0x01c001c0u) | ((b * 0x01001000u) & 0x80008000u);
  }
  const uint32_t b = __byte_perm(w, 0, i ? 0x4342 : 0x4140);
  return ((b * 16u) & 0x07f007f0u) | ((b * 256u) & 0x80008000u);
}

}  // namespace wf

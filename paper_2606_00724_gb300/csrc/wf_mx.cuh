// Codes of a quantised cache: blocks of 32 channels that share a power of two,
// elements in E4M3 or E2M1 (see wf_cache_quantize).
#pragma once

#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "wf_internal.cuh"

namespace wf {

constexpr int kMxBlock = 32;

// See wf_cache_quantize, wf_cache_dequantize (Vn, Vo null: keys alone).
cudaError_t launch_quantize(const void* Kn, const void* Vn, const wf_tensor& nt, void* Kc, void* Ks, void* Vc,
                            void* Vs, const wf_tensor& kv, int64_t pos, cudaStream_t s);
cudaError_t launch_dequantize(const void* Kc, const void* Ks, const void* Vc, const void* Vs, const wf_tensor& kv,
                              const int32_t* idx, int64_t pos, void* Ko, void* Vo, const wf_tensor& out,
                              cudaStream_t s);

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
// 2^-e of a scale byte up to 253, the largest of a finite block: 2^-126, the
// least normal number.
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
// Bits of the largest magnitude of a thread's channels, as an fp32 number (a NaN
// wins over every number).
__device__ __forceinline__ uint32_t top_bits(const float*, const uint4& v) {
  return max(max(v.x & 0x7fffffffu, v.y & 0x7fffffffu), max(v.z & 0x7fffffffu, v.w & 0x7fffffffu));
}
__device__ __forceinline__ uint32_t top_bits(const bf16*, const uint4& v) {
  const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu));
  return max(m & 0xffff0000u, m << 16);
}

template <int BYTES> struct Word;
template <> struct Word<8> { typedef uint2 type; };
template <> struct Word<4> { typedef uint32_t type; };
template <> struct Word<2> { typedef uint16_t type; };

// Codes of the N channels of one thread from their values in units of the scale.
template <bool FP4, int N>
__device__ __forceinline__ typename Word<FP4 ? N / 2 : N>::type pack_codes(const float* y) {
  constexpr int BITS = FP4 ? 8 : 16;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i * BITS / 32] |= mx_encode2<FP4>(y[2 * i], y[2 * i + 1]) << (i * BITS % 32);
  if constexpr (!FP4 && N == 8) return make_uint2(w[0], w[1]);
  else return (typename Word<FP4 ? N / 2 : N>::type)w[0];
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
// A word of codes before the factor: 4 E4M3 codes to 2 pairs, 8 E2M1 codes to 4.
// The bytes of the results are formed for all codes of the word at once (the
// upper one: sign and upper exponent bits, the lower one: the rest) and then
// put in their places.
template <bool FP4>
__device__ __forceinline__ void mx_pairs(uint32_t w, uint32_t* y) {
  if (FP4) {
    const uint32_t he = ((w << 4) & 0x80808080u) | ((w >> 2) & 0x01010101u), le = (w << 6) & 0xc0c0c0c0u;
    const uint32_t ho = (w & 0x80808080u) | ((w >> 6) & 0x01010101u), lo = (w << 2) & 0xc0c0c0c0u;
    const uint32_t e0 = __byte_perm(le, he, 0x5140), e1 = __byte_perm(le, he, 0x7362);  // channels 0, 2 and 4, 6
    const uint32_t o0 = __byte_perm(lo, ho, 0x5140), o1 = __byte_perm(lo, ho, 0x7362);  // 1, 3 and 5, 7
    y[0] = __byte_perm(e0, o0, 0x5410);
    y[1] = __byte_perm(e0, o0, 0x7632);
    y[2] = __byte_perm(e1, o1, 0x5410);
    y[3] = __byte_perm(e1, o1, 0x7632);
  } else {
    const uint32_t h = (w & 0x80808080u) | ((w >> 4) & 0x07070707u), l = (w << 4) & 0xf0f0f0f0u;
    y[0] = __byte_perm(l, h, 0x5140);
    y[1] = __byte_perm(l, h, 0x7362);
  }
}

}  // namespace wf

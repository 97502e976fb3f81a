// Pages of the 8-bit key/value cache (include/fastcoder.h, "8-bit paged cache").
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastcoder.h"

namespace fc {

constexpr int kPage8 = FC_PAGE_TOKENS;                 // 64 tokens of one key head
constexpr int kDim8 = FC_TREE_ATTN_HEAD_DIM;           // 128
constexpr int kBlock8 = FC_PAGE8_BLOCK;                // 32 tokens that share a scale
constexpr int kQuarter8 = 16;                          // tokens whose values lie dim by dim
constexpr int kPage8V = kPage8 * kDim8;                // byte offsets inside a page
constexpr int kPage8Scales = 2 * kPage8V;              // the keys' two blocks, the values' two
constexpr int kPage8Bytes = kPage8Scales + 128;        // whole lines, so that every page starts one
static_assert(kPage8Bytes == FC_PAGE8_HEAD_BYTES, "page layout");
static_assert(kPage8 == 64 && kDim8 == 128 && kBlock8 == 32, "lane layouts");

// A key code lies where its token and dim say.  Value codes of 16 tokens lie dim by
// dim, so that 16 bytes are what one lane takes into a value product (whose sum runs
// over tokens): neither keys nor values are turned around when they are read.
__host__ __device__ __forceinline__ int k8_at(int t, int d) { return t * kDim8 + d; }
__host__ __device__ __forceinline__ int v8_at(int t, int d) {
  return kPage8V + t / kQuarter8 * (kQuarter8 * kDim8) + d * kQuarter8 + t % kQuarter8;
}

// A block's scale is 2^e, e the least in [-117, 119] with every finite magnitude at
// most 448 * 2^e, the largest code.  From -117 on the smallest code times the scale is
// a normal bfloat16, up to 119 the largest is a finite one.
constexpr int kLeastExp8 = -117, kMostExp8 = 119;
__device__ __forceinline__ int exponent8(uint32_t amax_bits) {
  // 448 * 2^e = 1.75 * 2^(e + 8): the next exponent from the first mantissa above 1.75
  const int e = (int)((amax_bits + 0x1FFFFFu) >> 23) - 127 - 8;
  return e < kLeastExp8 ? kLeastExp8 : e > kMostExp8 ? kMostExp8 : e;
}
__device__ __forceinline__ int clamp_exp8(int e) { return e < kLeastExp8 ? kLeastExp8 : e > kMostExp8 ? kMostExp8 : e; }
__device__ __forceinline__ float power8(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// The scale that a byte stands for, and 2^-e.
__device__ __forceinline__ float scale8(uint32_t byte) { return __uint_as_float(byte << 23); }

// Magnitude bits of what is finite, else 0: what a block's scale has to reach.
__device__ __forceinline__ uint32_t reach8(float x) {
  const uint32_t m = __float_as_uint(x) & 0x7FFFFFFFu;
  return m < 0x7F800000u ? m : 0u;
}

// x times the power `inv`, as far as a code goes: larger magnitudes (which only the
// largest scale leaves) become 448, what is not finite a NaN.
__device__ __forceinline__ float to_code8(float x, float inv) {
  const float y = __builtin_amdgcn_fmed3f(x * inv, -448.0f, 448.0f);
  return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u ? __builtin_nanf("") : y;
}
// Four codes: the nearest ones, ties to the even one.
__device__ __forceinline__ uint32_t codes8(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}
typedef float floatx2_8 __attribute__((ext_vector_type(2)));
// What four codes stand for times `inv`, as codes again (a NaN stays one).
__device__ __forceinline__ uint32_t recode8(uint32_t w, float inv) {
  const floatx2_8 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return codes8(lo[0] * inv, lo[1] * inv, hi[0] * inv, hi[1] * inv);
}

// Most calls need less: with only finite numbers and a scale between the ends, no
// quotient passes 448, and the conversion of two bfloat16 numbers at a time is the same
// codes.  (Its quotient by a power of two is exact before it rounds.)
typedef unsigned short ushort2_8 __attribute__((ext_vector_type(2)));
typedef short short2_8 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_8 __attribute__((ext_vector_type(2)));
// The larger magnitudes of two pairs of bfloat16 bits, infinities and NaN above all.
__device__ __forceinline__ uint32_t tops8(uint32_t top, uint32_t pair) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(ushort2_8, top),
                                                                __builtin_bit_cast(ushort2_8, pair & 0x7FFF7FFFu)));
}
__device__ __forceinline__ uint32_t codes8(uint32_t pair0, uint32_t pair1, float scale) {
  const short2_8 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(short2_8{0, 0}, __builtin_bit_cast(bf16x2_8, pair0), scale, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2_8, pair1), scale, true));
}
// Four codes of two pairs by the longer way.
__device__ __forceinline__ uint32_t codes8_any(uint32_t pair0, uint32_t pair1, float inv) {
  return codes8(to_code8(__uint_as_float(pair0 << 16), inv), to_code8(__uint_as_float(pair0 & 0xFFFF0000u), inv),
                to_code8(__uint_as_float(pair1 << 16), inv), to_code8(__uint_as_float(pair1 & 0xFFFF0000u), inv));
}

}  // namespace fc

// Pages of the 4-bit key/value cache (include/fastcoder.h, "Paged cache").
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastcoder.h"

namespace fc {

constexpr int kPage = FC_PAGE_TOKENS;              // 64 tokens of one key head
constexpr int kHeadDim = FC_TREE_ATTN_HEAD_DIM;    // 128
constexpr int kScaleGroup = 32;                    // dims of a token that share a scale
constexpr int kCodeRow = kHeadDim / 2;             // 64 bytes: a token's codes
constexpr int kPageCodes = kPage * kCodeRow;       // 4 KB: a page's key (or value) codes
constexpr int kPageScales = kPage * kHeadDim / kScaleGroup;
constexpr int kPageV = kPageCodes;                 // byte offsets inside a page
constexpr int kPageKScale = 2 * kPageCodes;
constexpr int kPageVScale = kPageKScale + kPageScales;
constexpr int kPageBytes = kPageVScale + kPageScales;
static_assert(kPageBytes == FC_PAGE_HEAD_BYTES, "page layout");
static_assert(kPage == 64 && kHeadDim == 128, "lane layouts");

// Workgroups of a launch.  It takes fewer than 2^32 threads in a dimension, so a
// longer call is several launches; this many keep the card busy for so long that
// one launch more does not show.
constexpr int64_t kMostGroups = 1 << 20;

// Byte of a page that holds the scale of group g of token t.  Keys: lane 16 g +
// t % 16 of a wave finds its four 16-token tiles' scales in one word, which is
// how the score product's lanes hold them.  Values: lane 4 (t % 16) + g does,
// which is how a wave walks a page's value codes 16 bytes at a time.
__host__ __device__ __forceinline__ int k_scale_at(int t, int g) { return kPageKScale + (g * 16 + t % 16) * 4 + t / 16; }
__host__ __device__ __forceinline__ int v_scale_at(int t, int g) { return kPageVScale + (t % 16 * 4 + g) * 4 + t / 16; }

// Scale byte of a group whose largest magnitude has these bits (sign cleared):
// the smallest power of two 2^e with amax <= 7 * 2^e, e in [-125, 125], so that
// every value but a saturated one is a normal bfloat16 and 7 rounds to 6 by no
// more than 5 does.  255 where something is not finite.
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7F800000u) return 255u;
  // 7 * 2^e = 1.75 * 2^(e + 2): the next exponent from the first mantissa above 1.75
  const int e = (int)((amax_bits + 0x1FFFFFu) >> 23) - 127 - 2;
  return (uint32_t)((e < -125 ? -125 : e > 125 ? 125 : e) + 127);
}
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

}  // namespace fc

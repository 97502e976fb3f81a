// Tree attention over the paged 4-bit cache on gfx950 matrix cores
// (fc_paged_attention).
//
// The rows of a tree that share a key head - its R rows times the H / Hkv query
// heads of the group - are one matrix of queries, cut into tiles of 16 rows.  A
// workgroup of four waves takes up to five of a (tree, key head)'s tiles and a
// part of its pages.
//
// Per page of 64 keys a wave computes the transposed scores S^T = K Q^T and
// O^T += V^T P^T, which keeps a lane's scores where the second product wants
// its weights.  The key codes go into the matrix cores as they lie in the page:
// a 16x16x128 product takes 4-bit keys with a scale for each 32 dims, which are
// the cache's own format, so no key is ever unpacked.  Its other operand has at
// most 6 bits at the full rate, so a query is the sum of three 6-bit parts, each
// with the scale of what the last one left over: three products of 16 cycles
// where bf16 would take four and the unpacking.  The tree's own keys, which are
// not cached yet, are three such parts too.  The value codes are unpacked to bf16
// in LDS (their scales vary along the sum, which the matrix cores do not take),
// a quarter of a page by each wave, and read back transposed.
//
// How the work is split:
// - one tile (a decoded token, a short chain): the waves go through every fourth
//   page alone, out of registers, without a barrier until the end.  One row over
//   131,000 tokens, 8 key heads: 29 us and 5 for the join, where a copy of its bytes
//   takes 29; bound by memory.  64 rows over up to 8,192: 60 us in place of 41, as
//   long as the longest take.
// - more: two pairs of waves, each wave with two tiles and half of a page's keys,
//   and a fifth tile (a tree's 65th row) split over all four waves.  64 trees over
//   2,048 tokens, 32 key heads: 271 us of 65 rows, 224 of 64.  Tried when these took
//   330 and 254 (every step of the softmax had its maximum then): one tile a wave
//   and twice the waves a SIMD 225 for 64 rows, but 406 for 65, as it reads every
//   page again for the fifth tile, and a tree's root and its 64 drafted rows make
//   that the usual case; a workgroup of five waves 458, as one SIMD has two of them.
// - up to two tiles: the four waves take 16 keys each.
// Prefixes are cut into parts where there are too few workgroups to fill the card,
// and joined by k_paged_merge.  So are trees of more than 96 rows, whose further rows
// are parts of their own: 96 rows 426 us, 97 486, 101 602, 128 701, 256 1,699 (the same
// 64 trees); the fp32 results of all rows that they leave are 215 MB at 101 rows,
// written and read again.
//
// What bounds the second form, at 64 trees of 65 rows, 32 heads, 2,048 tokens (271
// us; a copy of its bytes takes 143, its products 128): a page takes a pair of
// workgroups about 2,900 cycles, of which a SIMD's vector unit is at work for 46 %
// and its matrix unit for 26 %.  The two do not overlap within a wave - scores,
// weights, values follow one another - and 254 registers leave two waves a SIMD to
// fill the gaps.  A third of the time is what comes before and after the pages
// (without any, the call takes 89 us): queries and tree rows to 6-bit parts, the
// tree's own scores, and the hand-over.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fastcoder.h"
#include "fc_device.h"
#include "fc_host.h"
#include "fc_page.h"

namespace {

using fc::kHeadDim;
using fc::kPage;
using fc::kPageBytes;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef float floatx32 __attribute__((ext_vector_type(32)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef int int32x2 __attribute__((ext_vector_type(2)));
typedef int int32x6 __attribute__((ext_vector_type(6)));
typedef int int32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kTile = 16;                       // query rows of a tile
constexpr int kWaves = 4;                       // of a workgroup: one for each SIMD
constexpr int kThreads = kWaves * fc::kWave;
constexpr int kParts = 3;                       // 6-bit parts of a query
constexpr int kDTiles = kHeadDim / 16;          // output tiles of 16 dims
constexpr int kRowBytes = kHeadDim * 2 + 32;    // a bf16 row in LDS
constexpr int kValues = kPage * kRowBytes;      // a page's values in LDS: 18 KB
constexpr int kSlot = 9 * 1024;                 // a page as it lies in memory, in LDS
constexpr int kTreeTiles = 6;                   // tree rows of a workgroup: 96
constexpr int kTreeRows = 16 * kTreeTiles;
constexpr int kSixRow = 304;                    // a row of 6-bit parts in LDS: 4 groups x 3 parts x 24 bytes, 4 scale words
constexpr int kSlots = 4;                       // pages on their way or in use
constexpr int kSlot0 = 2 * kValues;             // behind two pages' values
constexpr int kLds = kSlot0 + kSlots * kSlot;   // 72 KB: two workgroups of a CU
constexpr int kMostParts = 124;                 // of a prefix; with those of a tree's rows a merging wave takes 128
constexpr int kXcds = 8;
constexpr int kCus = 256;
static_assert((kWaves + 1) * kTile * kSixRow <= kSlot0 && kTreeRows * kSixRow <= kSlot0 && kTreeRows * kRowBytes <= kSlot0,
              "query and tree rows where the values go");

struct Args {
  const uint16_t *q, *k_tree, *v_tree;
  int64_t q_stride, k_stride, v_stride;
  const uint8_t* pool;
  const int32_t *table, *prefix_len, *num_nodes, *mask, *pos_ids;
  int n_pages, max_pages, B, R, H, Hkv, max_len, chunks, part_pages, parts;
  double log2_base;  // 0: no rotation
  uint16_t* out;
  float2* part_ml;
  float* part_o;
};

// Sets what is not finite among 8 bf16 to zero; whether there was any.
__device__ __forceinline__ bool keep_finite(uint4& x) {
  bool any = false;
  uint32_t* w = (uint32_t*)&x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (w[i] & 0x7F80u) == 0x7F80u, hi = (w[i] & 0x7F800000u) == 0x7F800000u;
    any |= lo | hi;
    w[i] &= (lo ? 0xFFFF0000u : 0xFFFFFFFFu) & (hi ? 0x0000FFFFu : 0xFFFFFFFFu);
  }
  return any;
}

__device__ __forceinline__ int clamp_len(int len, int most) { return len < 0 ? 0 : (len > most ? most : len); }

// Byte offset of 16-byte chunk c of row r of a bf16 tile in LDS.  Rows are 32
// bytes longer than their values: the transposing reads take 32 bytes of 16 rows
// at a time, eight rows of which then fill the 64 banks once, and every read of
// a page is one address and a constant.
__device__ __forceinline__ constexpr uint32_t chunk_at(int r, int c) { return (uint32_t)(r * kRowBytes + c * 16); }

// 32 floats, the even ones and the odd ones, as 6-bit values of scale f, and
// back.  Both instructions take several passes over their registers, so the
// result must not share any with the operands; the compiler's own forms let it
// (rows came out 2^-7 off where it did), hence the early clobber.
__device__ __forceinline__ int32x6 to_six(const floatx16& even, const floatx16& odd, float f) {
  int32x6 r;
  asm("v_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(r) : "v"(even), "v"(odd), "v"(f));
  return r;
}
__device__ __forceinline__ floatx32 from_six(const int32x6& c, float f) {
  floatx32 r;
  asm("v_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1" : "=&v"(r) : "v"(c), "v"(f));
  return r;
}

// 32 dims of a row as three 6-bit parts and their scale bytes.  The first
// part's scale 2^e is the smallest with which the largest magnitude is at most
// 7.5; it leaves at most 2^-2 * 2^e, the second (scale 2^(e - 4)) at most 2^-7,
// the third (2^(e - 9)) at most 2^-12.  e is -110 at least, which keeps the scales of
// the products above the least that a byte holds.  Scale byte 255: something is not finite.
__device__ __forceinline__ void write_six(const float (&v)[32], uint8_t* row, int g) {
  uint32_t top = 0;
#pragma unroll
  for (int u = 0; u < 32; ++u) {
    const uint32_t bits = __float_as_uint(v[u]) & 0x7FFFFFFFu;
    top = bits > top ? bits : top;
  }
  int e = (int)((top + 0x0FFFFFu) >> 23) - 127 - 2;  // 7.5 = 1.875 * 2^2
  e = e < -110 ? -110 : e;
  floatx16 even, odd;
#pragma unroll
  for (int u = 0; u < 16; ++u) even[u] = v[2 * u], odd[u] = v[2 * u + 1];
  uint32_t word = 0;
#pragma unroll
  for (int s = 0; s < kParts; ++s) {
    const int es = e - (s == 0 ? 0 : s == 1 ? 4 : 9);
    const float f = __uint_as_float((uint32_t)(es + 127) << 23);
    const int32x6 c = to_six(even, odd, f);
#pragma unroll
    for (int u = 0; u < 3; ++u) *(int32x2*)(row + (g * kParts + s) * 24 + 8 * u) = int32x2{c[2 * u], c[2 * u + 1]};
    if (s + 1 < kParts) {
      const floatx32 r = from_six(c, f);
#pragma unroll
      for (int u = 0; u < 16; ++u) even[u] -= r[2 * u], odd[u] -= r[2 * u + 1];
    }
    word |= (uint32_t)(top >= 0x7F800000u ? 255 : es + 127) << (8 * s);
  }
  *(uint32_t*)(row + 288 + 4 * g) = word;
}

// Groups of 32 dims of rows of 128 bf16 on their way to LDS in 6-bit parts, rotated
// and scaled.  The lane beside this one (lane ^ 1) has the group 64 dims away, so
// the two share the angles, in double precision: turn(d) gives the sine and cosine
// of this lane's d-th angle, of the 16 from first_angle on.
__device__ __forceinline__ int first_angle(int g) { return 32 * (g & 1) + (g >= 2 ? 16 : 0); }
struct Group {
  uint4 own[4], other[4];
};
__device__ __forceinline__ void load_group(const uint16_t* src, int g, Group& x) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    x.own[u] = *(const uint4*)(src + 32 * g + 8 * u);
    x.other[u] = *(const uint4*)(src + 32 * (g ^ 2) + 8 * u);
  }
}
template <typename Turn>
__device__ __forceinline__ void stage_six(const Group& in, int g, float scale, bool rotate, Turn turn, uint8_t* row) {
  float v[32];
  const uint4(&other)[4] = in.other;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float x[8];
    fc::unpack8(in.own[u], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[8 * u + e] = x[e] * scale;
  }
  if (rotate) {
    const bool upper = g >= 2;
    const float sign = upper ? scale : -scale;
    const uint32_t* y = (const uint32_t*)other;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (u % 4 == 0) asm volatile("" ::: "memory");  // eight of the angles in registers at a time
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int d = 2 * u + e;
        const float2 t = turn(d);
        const float s = __uint_as_float(fc::dpp_mov<0xB1>(__float_as_uint(t.x)));
        const float c = __uint_as_float(fc::dpp_mov<0xB1>(__float_as_uint(t.y)));
        const float y0 = __uint_as_float(e ? y[u] & 0xFFFF0000u : y[u] << 16);
        const float y1 = __uint_as_float(e ? y[8 + u] & 0xFFFF0000u : y[8 + u] << 16);
        v[d] = v[d] * (upper ? c : t.y) + y0 * sign * (upper ? s : t.x);
        v[16 + d] = v[16 + d] * (upper ? t.y : c) + y1 * sign * (upper ? t.x : s);
      }
    }
  }
  write_six(v, row, g);
}
// The group of the u-th of a row's four threads.
__device__ __forceinline__ int group_of(int u) { return (u >> 1) | ((u & 1) << 1); }

// A lane's operand of a row staged so: group lg of three parts, and their scales.
struct Six {
  int32x8 part[kParts];
  int scales;
};
__device__ __forceinline__ Six read_six(const uint8_t* row, int lg) {
  Six f;
#pragma unroll
  for (int s = 0; s < kParts; ++s) {
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      const int32x2 x = *(const int32x2*)(row + (lg * kParts + s) * 24 + 8 * u);
      f.part[s][2 * u] = x[0], f.part[s][2 * u + 1] = x[1];
    }
    f.part[s][6] = f.part[s][7] = 0;
  }
  f.scales = *(const int*)(row + 288 + 4 * lg);
  return f;
}

// Scores of 16 keys of a page (tile T) with 16 query rows, on top of `acc`.  The
// scale operands' byte selectors are immediates.
template <int T>
__device__ __forceinline__ floatx4 score(const uint4& k, uint32_t ks, const Six& q, floatx4 acc) {
  const int32x8 a = {(int)k.x, (int)k.y, (int)k.z, (int)k.w, 0, 0, 0, 0};
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.part[0], acc, 4, 2, T, (int)ks, 0, q.scales);
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.part[1], acc, 4, 2, T, (int)ks, 1, q.scales);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, q.part[2], acc, 4, 2, T, (int)ks, 2, q.scales);
}

// Scores are read by ordinary instructions some cycles after their product was
// issued, and nothing but such a wait keeps those apart.  The compiler puts it in,
// but counts it along one way only where a branch lies between (a page that needed
// no cutting off was read too early, and rows came out as zeros).  So the wait
// stands here, before any branch.
__device__ __forceinline__ void settle(floatx4& a) { asm volatile("s_nop 7\n\ts_nop 3" : "+v"(a)); }
__device__ __forceinline__ void settle(floatx4& a, floatx4& b) {
  asm volatile("s_nop 7\n\ts_nop 3" : "+v"(a), "+v"(b));
}
__device__ __forceinline__ void settle(floatx4& a, floatx4& b, floatx4& c, floatx4& d) {
  asm volatile("s_nop 7\n\ts_nop 3" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
}

// Of 16 tree rows with 16 query rows, both in 6-bit parts, six of the nine products.
// With the first parts' scales 2^e and 2^f, second parts are at most 2^-2 and third
// ones 2^-7 of theirs, so the three left out (second with third, third with both)
// add up to 2 * 2^-9 + 2^-14 of 2^(e + f) a dim, where the groups' largest are above
// 3.75 of theirs: 2^-11 of the product of those.
__device__ __forceinline__ floatx4 score_six(const Six& k, const Six& q, floatx4 acc) {
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[2], q.part[0], acc, 2, 2, 2, k.scales, 0, q.scales);
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[1], q.part[1], acc, 2, 2, 1, k.scales, 1, q.scales);
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[0], q.part[2], acc, 2, 2, 0, k.scales, 2, q.scales);
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[1], q.part[0], acc, 2, 2, 1, k.scales, 0, q.scales);
  acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[0], q.part[1], acc, 2, 2, 0, k.scales, 1, q.scales);
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(k.part[0], q.part[0], acc, 2, 2, 0, k.scales, 0, q.scales);
}

// parts that a prefix is cut into, each of part_pages pages, and those that more
// tree rows than one workgroup takes have to themselves
__device__ __forceinline__ int parts_of(int pages, int part_pages) {
  return pages <= part_pages ? 1 : (pages + part_pages - 1) / part_pages;
}
__host__ __device__ __forceinline__ int more_parts(int n) { return n <= kTreeRows ? 0 : (n - 1) / kTreeRows; }

// A query row's outputs (lane (lg, lc): dims 16 t + 4 lg + e of row lc), its
// running maximum as 0 - m (0 while there is none), the sum of its weights, and
// whether it is yet to see a key.
struct Row {
  floatx4 o[kDTiles];
  floatx4 minus_m;
  float l;
  bool first;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) o[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    minus_m = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    l = 0.0f;
    first = true;
  }
  __device__ __forceinline__ float m() const { return first ? -INFINITY : 0.0f - minus_m[0]; }
};

// The softmax's usual step is a power of two, a rounding and a share of a sum for
// each score, and no maximum.  s holds scores less m (the products start from
// minus_m), -inf where a key is not allowed.  m is the maximum of what the row saw
// when it was last scaled; a factor common to a row's weights costs no accuracy,
// bf16 and fp32 having the same exponents, as long as the sums do not overflow: each
// step adds less than 2^24 times the largest value, and the 2^31 tokens that a table
// may hold are 2^27 steps at most, so values below 2^76 stay in.  A step whose weights add up to 2^24 or more (or to a NaN) is taken again
// with m raised to its maximum, and so is a row's first: rare enough (scores of 24
// bits above what came before) to cost nothing.  Against a maximum in every step,
// with rows scaled anew from 2^8 on: 64 trees of 65 rows over 2,048 tokens 300 ->
// 286 us.
constexpr float kMostWeight = 16777216.0f;  // 2^24
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

template <int N>
__device__ __forceinline__ void raise(floatx4 (&s)[N], Row& r, bool need) {
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < N; ++t) {
    top = fmaxf(fmaxf(top, s[t][0]), s[t][1]);
    top = fmaxf(fmaxf(top, s[t][2]), s[t][3]);
  }
  float mx = fmaxf(top, __shfl_xor(top, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  int row_needs = need;
  row_needs |= __shfl_xor(row_needs, 16);
  row_needs |= __shfl_xor(row_needs, 32);
  // by how much m rises; a row that has no need keeps it, so that its result goes
  // by its own scores alone
  const bool rise = row_needs != 0 && mx != -INFINITY;
  const float by = rise ? mx : 0.0f;
  const float alpha = r.first ? 0.0f : __builtin_amdgcn_exp2f(-by);
#pragma unroll
  for (int t = 0; t < N; ++t) s[t] -= by;
  r.l *= alpha;
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) r.o[t] *= alpha;
  const float minus = r.minus_m[0] - by;
  r.first = r.first && !rise;
  r.minus_m = floatx4{minus, minus, minus, minus};
}
// Rounded weights of N tiles of 16 keys, and their sum (of what the value product
// sees).
template <int N>
__device__ __forceinline__ float weigh(const floatx4 (&s)[N], bf16x2 (&p)[2 * N]) {
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < N; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      p[2 * t + e] = bf16x2{(__bf16)__builtin_amdgcn_exp2f(s[t][2 * e]), (__bf16)__builtin_amdgcn_exp2f(s[t][2 * e + 1])};
      sum = __builtin_amdgcn_fdot2_f32_bf16(p[2 * t + e], one, sum, false);
    }
  return sum;
}
__device__ __forceinline__ bool too_much(float sum, const Row& r) {
  return !(sum < (r.first ? -1.0f : kMostWeight));
}
template <int N>
__device__ __forceinline__ void weights(floatx4 (&s)[N], Row& r, bf16x2 (&p)[2 * N]) {
  float sum = weigh(s, p);
  if (__any(too_much(sum, r))) {
    raise(s, r, too_much(sum, r));
    sum = weigh(s, p);
  }
  r.l += sum;
}
__device__ __forceinline__ bf16x8 join(const bf16x2& a, const bf16x2& b, const bf16x2& c, const bf16x2& d) {
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;

// V^T of 32 keys, output tiles t0 and t0 + 1: a transposing read gives lane (lg,
// lc) dims 16 t + lc of keys 4 lg + e, the second one of keys 16 + 4 lg + e, as the
// weights lie.  `at` is this lane's place in the first of the 32 rows.  The fence
// keeps reads ahead of what comes after them in the source.
struct Frag {
  bf16x4 lo[2], hi[2];
};
__device__ __forceinline__ void read_values(lds_u8* at, int t0, Frag& f) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    f.lo[t] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + chunk_at(0, 2 * (t0 + t))));
    f.hi[t] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + chunk_at(16, 2 * (t0 + t))));
  }
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void add_values(const Frag& f, int t0, const bf16x8& pb, Row& r) {
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const bf16x8 a = {f.lo[t][0], f.lo[t][1], f.lo[t][2], f.lo[t][3], f.hi[t][0], f.hi[t][1], f.hi[t][2], f.hi[t][3]};
    r.o[t0 + t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb, r.o[t0 + t], 0, 0, 0);
  }
}
__device__ __forceinline__ void all_values(lds_u8* at, const bf16x8& pb, Row& r) {
  Frag f[4];
#pragma unroll
  for (int u = 0; u < 4; ++u) read_values(at, 2 * u, f[u]);
#pragma unroll
  for (int u = 0; u < 4; ++u) add_values(f[u], 2 * u, pb, r);
}

// 32 dims (16 bytes of codes, the scale in byte i4 of `scales`) of key i4 * 16 +
// lane / 4 of a page's values, to bf16 in LDS.  A key past the prefix has weight 0,
// and so that whatever its bytes hold does not matter its values are 0 too.
__device__ __forceinline__ void unpack(const uint4& raw, uint32_t scales, int i4, int lane, int left, uint8_t* to) {
  const int key = i4 * 16 + (lane >> 2), g = lane & 3;
  uint32_t sb = (scales >> (8 * i4)) & 255u;
  uint32_t c4[4] = {raw.x, raw.y, raw.z, raw.w};
  if (left < kPage) {
    asm volatile("");  // a branch: few pages end early
    const bool live = key < left;
    sb = live ? sb : 127u;
#pragma unroll
    for (int c = 0; c < 4; ++c) c4[c] = live ? c4[c] : 0u;
  }
  const float sc = fc::scale_of(sb);
  uint8_t* dst = to + chunk_at(key, 4 * g);
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    uint4 d;
    d.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c4[c], sc, 0));
    d.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c4[c], sc, 1));
    d.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c4[c], sc, 2));
    d.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c4[c], sc, 3));
    *(uint4*)(dst + 16 * c) = d;
  }
}

// keys of a page's tile t that lie past the prefix do not count
__device__ __forceinline__ void cut(floatx4& s, int t, int lg, int left) {
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = 16 * t + 4 * lg + e < left ? s[e] : -INFINITY;
}

// A pair's angle in revolutions a position, and its sine and cosine: reduced to
// [0, 1) in double precision, so far positions keep full accuracy.
__device__ __forceinline__ double angle_of(int d, double log2_base) {
  return exp2(-2.0 * d / (double)kHeadDim * log2_base) * 0.15915494309189533577;
}
__device__ __forceinline__ float2 turn_of(double revolutions) {
  const float f = (float)__builtin_amdgcn_fract(revolutions);
  return make_float2(__builtin_amdgcn_sinf(f), __builtin_amdgcn_cosf(f));
}
__device__ __forceinline__ float score_scale() { return 1.44269504088896340736f / sqrtf((float)kHeadDim); }

// What a workgroup works on.
struct Work {
  int bk, b, kv, G, M, P, n, part, parts, pg0, pg1, tree0;
  bool tree;
  __device__ __forceinline__ bool init(const Args& A, int bk_, int part_) {
    bk = bk_, part = part_;
    b = bk / A.Hkv, kv = bk - b * A.Hkv;
    G = A.H / A.Hkv, M = A.R * G;
    P = clamp_len(A.prefix_len[b], A.max_len);
    n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
    const int pages = (P + kPage - 1) / kPage, cached = parts_of(pages, A.part_pages);
    parts = cached + more_parts(n);
    if (part >= parts) return false;
    // the last part of the prefix has the tree's first rows, the others their own parts
    pg0 = part < cached ? part * A.part_pages : pages;
    pg1 = part < cached - 1 ? pg0 + A.part_pages : pages;
    tree0 = part < cached ? 0 : (part - cached + 1) * kTreeRows;
    tree = part >= cached - 1 && n > 0;
    return true;
  }
  // a tree row's position behind the prefix; their sum may pass 32 bits
  __device__ __forceinline__ int behind(const Args& A, int r) const {
    return A.pos_ids ? A.pos_ids[(int64_t)b * A.R + r] : r;
  }
  __device__ __forceinline__ double position(int behind) const { return (double)P + (double)behind; }
  // rows past the last one: the last one, whose results nobody takes
  __device__ __forceinline__ int row_at(int r) const { return r < M ? r : M - 1; }
  __device__ __forceinline__ const uint16_t* q_row(const Args& A, int r) const {
    const int tr = r / G;
    return A.q + ((int64_t)b * A.R + tr) * A.q_stride + ((int64_t)kv * G + (r - tr * G)) * kHeadDim;
  }
  __device__ __forceinline__ const uint16_t* k_row(const Args& A, int j) const {
    return A.k_tree + ((int64_t)b * A.R + j) * A.k_stride + (int64_t)kv * kHeadDim;
  }
  __device__ __forceinline__ const uint16_t* v_row(const Args& A, int j) const {
    return A.v_tree + ((int64_t)b * A.R + j) * A.v_stride + (int64_t)kv * kHeadDim;
  }
  // bit e: query row tr may see tree row 4 lg + e, of at most 16
  __device__ __forceinline__ uint32_t allowed(const Args& A, int tr, bool in, int lg) const {
    uint32_t bits = 0;
    const int j = 4 * lg;
    int m[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) m[e] = j + e <= tr;
    if (A.mask) {
      const int32_t* mrow = A.mask + ((int64_t)b * A.R + tr) * A.R;
#pragma unroll
      for (int e = 0; e < 4; ++e) m[e] = mrow[j + e < n ? j + e : 0];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) bits |= (uint32_t)(in && j + e < n && m[e] == 1) << e;
    return bits;
  }
  // Values of 32 tree rows that are not finite are 0 in LDS: a product with weight
  // 0 would be NaN, so the rows that do not see such a value must not meet it.  This
  // adds them for the rows that do: bit j of `bad` marks row j0 + j, `see` holds
  // the block's eight bits.
  __device__ __forceinline__ void add_marked(const Args& A, uint32_t bad, int j0, const bf16x8& pb, uint32_t see,
                                             int lg, int lc, Row& r) const {
    for (; bad; bad &= bad - 1) {
      const int j = __builtin_ctz(bad);
      const int u = j / 16 * 4 + j % 4, from = j % 16 / 4 * 16 + lc;  // whose weights for row j these are
      const uint16_t* vp = v_row(A, j0 + j) + 4 * lg;
      float weight = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) weight = e == u ? (float)pb[e] : weight;
      weight = __shfl(weight, from);
      const bool sees = (__shfl(see, from) >> u) & 1u;
#pragma unroll
      for (int t = 0; t < kDTiles; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const uint32_t x = (uint32_t)vp[16 * t + e] << 16;
          r.o[t][e] += sees && (x & 0x7F800000u) == 0x7F800000u ? weight * __uint_as_float(x) : 0.0f;
        }
    }
  }
};

// Which of `left` (at most 96) tree rows, from tree0 on, the query rows tr0 .. tr1
// may see.  load() asks for the mask's rows, four of a wave at a time, all on their
// way together; store() leaves them as bits: to[3 i + k], bit j: row tr0 + i may
// see tree row tree0 + 32 k + j.
struct See {
  static constexpr int kTimes = (kWaves + 1) * kTile / (4 * kWaves);
  int m[kTimes][4][2];
  template <typename F>
  __device__ __forceinline__ static void each(int tr0, int tr1, int w, F f) {
#pragma unroll
    for (int k = 0; k < kTimes; ++k)
      if (4 * (kWaves * k + w) <= tr1 - tr0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) f(k, i, 4 * (kWaves * k + w) + i);
      }
  }
  __device__ __forceinline__ void load(const Args& A, const Work& W, int tr0, int tr1, int left, int w) {
    const int lane = fc::lane_id();
    if (!A.mask) return;
    each(tr0, tr1, w, [&](int k, int i, int at) {
      const int32_t* row = A.mask + ((int64_t)W.b * A.R + (tr0 + at < tr1 ? tr0 + at : tr1)) * A.R + W.tree0;
      m[k][i][0] = row[lane < left ? lane : 0];
      m[k][i][1] = row[lane + 64 < left ? lane + 64 : 0];
    });
  }
  __device__ __forceinline__ void store(const Args& A, const Work& W, int tr0, int tr1, int left, int w,
                                        uint32_t* to) const {
    const int lane = fc::lane_id();
    each(tr0, tr1, w, [&](int k, int i, int at) {
      const bool a = A.mask ? m[k][i][0] == 1 : W.tree0 + lane <= tr0 + at;
      const bool b = A.mask ? m[k][i][1] == 1 : W.tree0 + lane + 64 <= tr0 + at;
      const uint64_t lo = fc::ballot(lane < left && a), hi = fc::ballot(lane + 64 < left && b);
      if (lane == 0 && tr0 + at <= tr1) {
        to[3 * at] = (uint32_t)lo;
        to[3 * at + 1] = (uint32_t)(lo >> 32);
        to[3 * at + 2] = (uint32_t)hi;
      }
    });
  }
};

// ---- waves that shared a tile's keys hand over to one of them, through LDS
constexpr int kRec = kTile * kHeadDim + 2 * kTile;  // floats of a tile: outputs, maxima, weights
__device__ __forceinline__ void whole(Row& r) {
  r.l += __shfl_xor(r.l, 16);
  r.l += __shfl_xor(r.l, 32);
}
__device__ __forceinline__ void give(const Row& r, float* rec) {
  const int lane = fc::lane_id();
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) *(floatx4*)(rec + (t * 64 + lane) * 4) = r.o[t];
  if (lane < 16) rec[kTile * kHeadDim + lane] = r.m(), rec[kTile * kHeadDim + kTile + lane] = r.l;
}
__device__ __forceinline__ void take(Row& r, float& m, const float* rec) {
  const int lane = fc::lane_id(), lc = lane & 15;
  const float m2 = rec[kTile * kHeadDim + lc], l2 = rec[kTile * kHeadDim + kTile + lc];
  const float both = fmaxf(m, m2);
  const float a1 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - both);
  const float a2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - both);
  m = both;
  r.l = r.l * a1 + l2 * a2;
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) r.o[t] = r.o[t] * a1 + *(const floatx4*)(rec + (t * 64 + lane) * 4) * a2;
}
__device__ __forceinline__ void finish(const Args& A, const Work& W, const Row& r, float m, int row) {
  const int lg = fc::lane_id() >> 4;
  if (W.parts > 1) {
    const int64_t at = ((int64_t)W.bk * A.parts + W.part) * W.M + row;
    if (lg == 0) A.part_ml[at] = make_float2(m, r.l);
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) *(floatx4*)(A.part_o + at * kHeadDim + 16 * t + 4 * lg) = r.o[t];
  } else {
    // a row without a key has weight 0; a NaN stays one
    const int tr = row / W.G;
    const float inv = tr < W.n && r.l != 0.0f ? 1.0f / r.l : 0.0f;
    uint16_t* dst = A.out + (((int64_t)W.b * A.R + tr) * A.H + W.kv * W.G + (row - tr * W.G)) * kHeadDim;
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) {
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(r.o[t][e] * inv);
      *(bf16x4*)(dst + 16 * t + 4 * lg) = x;
    }
  }
}

// Up to five tiles of query rows.  A wave has two tiles and a part of each page's
// keys: with KS 2 a pair of tiles for each two waves and 32 keys for each wave,
// with KS 4 one pair of tiles and 16 keys.  (Two tiles share what they read of a
// page's values, which is most of what goes through LDS.)  kFive: a fifth tile
// besides, 16 keys for each wave.
template <int KS, bool kFive>
__device__ __forceinline__ void attend(const Args& A, const Work& W, uint8_t* s_v, double* s_freq, uint32_t* s_bad,
                                       uint32_t* s_see, int tile0, int tiles) {
  static_assert(!kFive || KS == 2, "the fifth tile goes with two pairs");
  constexpr int NB = KS == 2 ? 2 : 1;  // blocks of 32 tree rows of a wave, at most
  const int tid = (int)threadIdx.x, lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane(tid / fc::kWave);
  const int pair = KS == 2 ? w & 1 : 0, ks = KS == 2 ? w >> 1 : w;
  const int lg = lane >> 4, lc = lane & 15;
  const bool rotate = A.log2_base > 0.0;
  int row[2];
  bool in[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    row[i] = (tile0 + 2 * pair + i) * kTile + lc;
    in[i] = 2 * pair + i < tiles && row[i] < W.M;
  }
  const bool five = kFive && tiles > kWaves;
  const int row5 = (tile0 + kWaves) * kTile + lc;
  const bool in5 = five && row5 < W.M;

  // ---- pages on their way: straight from memory into LDS as they lie (16 bytes
  // a lane, no registers), two while a third is used.  The keys' four chunks of 16
  // bytes change places by the row, so that a wave reads 16 rows without two lanes
  // in a bank.
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_v;
  const int32_t* table = A.table + (int64_t)W.b * A.max_pages;
  const auto slot_of = [&](int pg) { return kSlot0 + ((pg - W.pg0) & (kSlots - 1)) * kSlot; };
  // page numbers, 64 at a time in a register's lanes: read one by one they would
  // be loads to wait for among the loads that are meant to stay in flight
  int ids = 0;
  constexpr int kLoads = 3;  // of a wave and page
  const auto issue = [&](int pg) {
    const int i = (pg - W.pg0) & 63;
    if (i == 0) ids = pg + lane < W.pg1 ? table[pg + lane] : -1;
    const int id = __builtin_amdgcn_readlane(ids, i);
    const bool there = id >= 0 && id < A.n_pages;  // an absent page's loads give zeros, and none of its keys counts
    const fc::int32x4 rsrc = fc::buffer_rsrc(A.pool + ((int64_t)(there ? id : 0) * A.Hkv + W.kv) * kPageBytes,
                                             there ? (uint32_t)kPageBytes : 0u);
    const uint32_t to = lds0 + (uint32_t)slot_of(pg);
    fc::lds_load16(to + (uint32_t)w * 1024u, (uint32_t)(w * 1024 + (lane ^ (lane >> 4)) * 16), rsrc);
    fc::lds_load16(to + (uint32_t)(w + 4) * 1024u, (uint32_t)((w + 4) * 1024 + lane * 16), rsrc);
    fc::lds_load16(to + 8u * 1024u, (uint32_t)(8 * 1024 + lane * 16), rsrc);  // the scales: every wave the same
    return there;
  };
  bool here0 = false, here1 = false, here2 = false;  // whether page pg, pg + 1, pg + 2 is
  if (W.pg0 < W.pg1) here0 = issue(W.pg0);
  if (!W.tree && W.pg0 + 1 < W.pg1) here1 = issue(W.pg0 + 1);

  // ---- queries and the tree's keys, in 6-bit parts through LDS: a thread for each
  // group of a row, the next one's loads on their way; queries where the second
  // page will lie, or where values will if there is no tree
  static_assert(kTreeRows * kSixRow <= kSlot0 && (kWaves + 1) * kTile * kSixRow <= (kSlots - 1) * kSlot, "rows fit");
  uint8_t* const six_q = s_v + (W.tree ? kSlot0 + kSlot : 0);
  const int row0 = tile0 * kTile, rows = W.M - row0 < kTile * tiles ? W.M - row0 : kTile * tiles;
  const int left = !W.tree ? 0 : W.n - W.tree0 < kTreeRows ? W.n - W.tree0 : kTreeRows;  // tree rows
  const int tr0 = row0 / W.G, tr1 = (row0 + rows - 1) / W.G;
  See mask;
  if (rotate && tid < kHeadDim / 2) s_freq[tid] = angle_of(tid, A.log2_base);
  if (W.tree) {
    if (tid < kTreeTiles / 2) s_bad[tid] = 0;
    mask.load(A, W, tr0, tr1, left, w);
  }
  __syncthreads();
  {
    const int units = 4 * (rows + left);
    const auto load = [&](int u, Group& x, int& at) {
      const int r = (u < units ? u : units - 1) >> 2, qr = row0 + r, kr = W.tree0 + r - rows;
      load_group(r < rows ? W.q_row(A, qr) : W.k_row(A, kr), group_of(u & 3), x);
      if (rotate) at = W.behind(A, r < rows ? qr / W.G : kr);
    };
    double freq[16];  // of the lane's angles, in every row the same ones
    if (rotate) {
#pragma unroll
      for (int d = 0; d < 16; ++d) freq[d] = s_freq[first_angle(group_of(tid & 3)) + d];
    }
    Group x;
    int at = 0;
    load(tid, x, at);
    for (int u = tid; u < units; u += kThreads) {
      Group next;
      int next_at = 0;
      load(u + kThreads, next, next_at);
      const int r = u >> 2, g = group_of(u & 3);
      const double pos = W.position(at);
      stage_six(x, g, r < rows ? score_scale() : 1.0f, rotate,
                [&](int d) { return turn_of(pos * freq[d]); },
                r < rows ? six_q + r * kSixRow : s_v + (r - rows) * kSixRow);
      x = next;
      at = next_at;
    }
  }
  if (W.tree) mask.store(A, W, tr0, tr1, left, w, s_see);
  __syncthreads();
  // rows past the last one: the last one, whose results nobody takes
  const auto query = [&](int tile) {
    const int r = kTile * tile + lc;
    return read_six(six_q + (r < rows ? r : rows - 1) * kSixRow, lg);
  };
  Six q[2], q5;
#pragma unroll
  for (int i = 0; i < 2; ++i) q[i] = query(2 * pair + i);
  if (kFive) q5 = query(kWaves);

  lds_u8* const v_lane = (lds_u8*)(uintptr_t)(lds0 + chunk_at(4 * lg + (lc >> 2), 0) + (uint32_t)(lc & 3) * 8u);
  Row me[2], extra;
  me[0].clear();
  me[1].clear();
  if (kFive) extra.clear();

  // ---- the tree's own rows: keys in 6-bit parts as the queries, values in bf16.
  // Block k of 32 of them is for the waves with ks = k % KS; the second pair of
  // waves has the fifth tile.
  if (W.tree) {
    constexpr int kLoaded = kTreeRows * kHeadDim * 2 / 16 / kThreads;
    uint4 v[kLoaded];  // a thread's values: row tid / 16 of each 16
#pragma unroll
    for (int i = 0; i < kLoaded; ++i) {
      const int r = 16 * i + tid / 16;
      v[i] = *(const uint4*)(W.v_row(A, W.tree0 + (r < left ? r : left - 1)) + 8 * (tid % 16));
    }
    const bool also = five && pair == 1;
    uint32_t bits[3] = {0, 0, 0};  // eight for each block
    floatx4 s[3][2 * NB];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int block = ks + KS * k;
      const auto see = [&](int r) {  // bit 4 t + e: the block's row 16 t + 4 lg + e
        const uint32_t word = s_see[(r / W.G - tr0) * (kTreeTiles / 2) + block];
        return (((word >> (4 * lg)) & 0xFu) | ((word >> (12 + 4 * lg)) & 0xF0u)) << (8 * k);
      };
      if (32 * block < left) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (in[i]) bits[i] |= see(row[i]);
        if (also && in5) bits[2] |= see(row5);
      }
#pragma unroll
      for (int t = 2 * k; t < 2 * k + 2; ++t) {
        const int j = 32 * block + 16 * (t % 2);
        s[0][t] = s[1][t] = s[2][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
        if (j < left) {
          const Six key = read_six(s_v + (j + lc < left ? j + lc : left - 1) * kSixRow, lg);
          s[0][t] = score_six(key, q[0], s[0][t]);
          s[1][t] = score_six(key, q[1], s[1][t]);
          if (also) s[2][t] = score_six(key, q5, s[2][t]);
        }
      }
    }
    __syncthreads();  // queries and keys are read
#pragma unroll
    for (int i = 0; i < kLoaded; ++i) {
      const int r = 16 * i + tid / 16;
      if (16 * i >= (left + 31) / 32 * 32) break;
      if (r >= left) v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (keep_finite(v[i])) atomicOr(&s_bad[r / 32], 1u << (r % 32));
      *(uint4*)(s_v + chunk_at(r, tid % 16)) = v[i];
    }
    if (W.pg0 + 1 < W.pg1) here1 = issue(W.pg0 + 1);
    bf16x8 pb[3][NB];
    const auto tree_weights = [&](floatx4 (&s)[2 * NB], uint32_t see, Row& r, bf16x8 (&p)[NB]) {
#pragma unroll
      for (int k = 0; k < NB; ++k) settle(s[2 * k], s[2 * k + 1]);
#pragma unroll
      for (int u = 0; u < 8 * NB; ++u) s[u / 4][u % 4] = (see >> u) & 1u ? s[u / 4][u % 4] : -INFINITY;
      bf16x2 x[4 * NB];
      weights(s, r, x);
#pragma unroll
      for (int k = 0; k < NB; ++k) p[k] = join(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
    };
    tree_weights(s[0], bits[0], me[0], pb[0]);
    tree_weights(s[1], bits[1], me[1], pb[1]);
    if (also) tree_weights(s[2], bits[2], extra, pb[2]);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int at = 32 * (ks + KS * k);
      if (at >= left) break;
      const uint32_t bad = __builtin_amdgcn_readfirstlane(s_bad[at / 32]);
      Frag f[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) read_values(v_lane + chunk_at(1, 0) * at, 2 * u, f[u]);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        add_values(f[u], 2 * u, pb[0][k], me[0]);
        add_values(f[u], 2 * u, pb[1][k], me[1]);
        if (also) add_values(f[u], 2 * u, pb[2][k], extra);
      }
      if (bad) {
        W.add_marked(A, bad, W.tree0 + at, pb[0][k], bits[0] >> (8 * k), lg, lc, me[0]);
        W.add_marked(A, bad, W.tree0 + at, pb[1][k], bits[1] >> (8 * k), lg, lc, me[1]);
        if (also) W.add_marked(A, bad, W.tree0 + at, pb[2][k], bits[2] >> (8 * k), lg, lc, extra);
      }
    }
  }

  // ---- the prefix.  Between two barriers the waves have a page's scores, add its
  // values, and unpack the next one's, a quarter each.
  const auto unpack_page = [&](int pg, bool here) {
    const uint8_t* raw = s_v + slot_of(pg);
    unpack(*(const uint4*)(raw + fc::kPageV + (w * 64 + lane) * 16), *(const uint32_t*)(raw + fc::kPageVScale + 4 * lane),
           w, lane, here ? W.P - pg * kPage : 0, s_v + ((pg - W.pg0) & 1) * kValues);
  };
  lds_u8* const v_mine = v_lane + chunk_at(KS == 2 ? 32 : 16, 0) * ks;
  const uint32_t k_lane = (uint32_t)(lc * fc::kCodeRow + ((lg ^ (lc >> 2)) << 4));
  if (W.pg0 < W.pg1) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // the first pages are there, the place of their values is free
    unpack_page(W.pg0, here0);
  }
  for (int pg = W.pg0; pg < W.pg1; ++pg) {
    // the page after this one is there: only what was asked for last may be on its way
    if (pg + 2 < W.pg1) here2 = issue(pg + 2);
    if (pg + 2 < W.pg1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // and its values, for all; the values before them and their slot are free
    const int left = here0 ? W.P - pg * kPage : 0;  // keys that exist, if below 64
    const uint8_t* raw = s_v + slot_of(pg);
    lds_u8* const values = v_mine + ((pg - W.pg0) & 1) * kValues;
    const uint32_t kscales = *(const uint32_t*)(raw + fc::kPageKScale + 4 * lane);
    const auto key = [&](int t) { return *(const uint4*)(raw + t * 1024 + k_lane); };
    if constexpr (KS == 2) {
      const uint32_t mine = kscales >> (16 * ks);
      const uint4 k0 = key(2 * ks), k1 = key(2 * ks + 1);
      floatx4 s[2][2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i][0] = score<0>(k0, mine, q[i], me[i].minus_m);
        s[i][1] = score<1>(k1, mine, q[i], me[i].minus_m);
      }
      floatx4 s5[1] = {floatx4{0.0f, 0.0f, 0.0f, 0.0f}};
      if (kFive && five) s5[0] = pair ? score<1>(k1, mine, q5, extra.minus_m) : score<0>(k0, mine, q5, extra.minus_m);
      if (pg + 1 < W.pg1) unpack_page(pg + 1, here1);
      settle(s[0][0], s[0][1], s[1][0], s[1][1]);
      if (kFive) settle(s5[0]);
      if (left < kPage) {
#pragma unroll
        for (int i = 0; i < 2; ++i) cut(s[i][0], 2 * ks, lg, left), cut(s[i][1], 2 * ks + 1, lg, left);
        if (kFive && five) cut(s5[0], 2 * ks + pair, lg, left);
      }
      Frag f0, f1, f2;
      read_values(values, 0, f0);
      read_values(values, 2, f1);
      bf16x2 x0[4], x1[4], x5[2];
      float sum0 = weigh(s[0], x0), sum1 = weigh(s[1], x1);
      if (__any(too_much(sum0, me[0]) || too_much(sum1, me[1]))) {
        raise(s[0], me[0], too_much(sum0, me[0]));
        raise(s[1], me[1], too_much(sum1, me[1]));
        sum0 = weigh(s[0], x0), sum1 = weigh(s[1], x1);
      }
      me[0].l += sum0;
      me[1].l += sum1;
      const bf16x8 p0 = join(x0[0], x0[1], x0[2], x0[3]), p1 = join(x1[0], x1[1], x1[2], x1[3]);
      bf16x8 pb5;
      if (kFive) {
        if (five) weights(s5, extra, x5);
        else x5[0] = x5[1] = bf16x2{(__bf16)0.0f, (__bf16)0.0f};
        const bf16x2 none = {(__bf16)0.0f, (__bf16)0.0f};
        pb5 = pair ? join(none, none, x5[0], x5[1]) : join(x5[0], x5[1], none, none);
      }
      const auto add = [&](const Frag& f, int t0) {
        add_values(f, t0, p0, me[0]);
        add_values(f, t0, p1, me[1]);
        if (kFive && five) add_values(f, t0, pb5, extra);
      };
      read_values(values, 4, f2);
      add(f0, 0);
      read_values(values, 6, f0);
      add(f1, 2);
      add(f2, 4);
      add(f0, 6);
    } else {
      const uint4 k0 = key(ks);
      floatx4 s[2][1];
#pragma unroll
      for (int i = 0; i < 2; ++i) s[i][0] = score<0>(k0, kscales >> (8 * ks), q[i], me[i].minus_m);
      if (pg + 1 < W.pg1) unpack_page(pg + 1, here1);
      settle(s[0][0], s[1][0]);
      if (left < kPage) cut(s[0][0], ks, lg, left), cut(s[1][0], ks, lg, left);
      bf16x4 lo[kDTiles], p[2];
#pragma unroll
      for (int t = 0; t < kDTiles; ++t)
        lo[t] = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(values + chunk_at(0, 2 * t)));
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        bf16x2 x[2];
        weights(s[i], me[i], x);
        p[i] = bf16x4{x[0][0], x[0][1], x[1][0], x[1][1]};
      }
#pragma unroll
      for (int t = 0; t < kDTiles; ++t)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          me[i].o[t] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(shortx4, lo[t]),
                                                                 __builtin_bit_cast(shortx4, p[i]), me[i].o[t], 0, 0, 0);
    }
    here0 = here1;
    here1 = here2;
  }

  // ---- waves that share a tile: the one with ks = i takes tile i from the others,
  // the last wave the fifth tile
  float* rec = (float*)s_v;
  constexpr int kOthers = (kWaves / KS) * 2 * (KS - 1);
  static_assert((kOthers + (kFive ? kWaves - 1 : 0)) * kRec * 4 <= kLds, "hand-over fits");
  const auto rec_of = [&](int i, int from) {
    return rec + ((pair * 2 + i) * (KS - 1) + (from < i ? from : from - 1)) * kRec;
  };
#pragma unroll
  for (int i = 0; i < 2; ++i) whole(me[i]);
  if (kFive) whole(extra);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ks != i) give(me[i], rec_of(i, ks));
  if (kFive && five && w < kWaves - 1) give(extra, rec + (kOthers + w) * kRec);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 2; ++i)
    if (ks == i) {
      float m = me[i].m();
#pragma unroll
      for (int g = 0; g < KS; ++g)
        if (g != i) take(me[i], m, rec_of(i, g));
      if (in[i]) finish(A, W, me[i], m, row[i]);
    }
  if (kFive && five && w == kWaves - 1) {
    float m = extra.m();
#pragma unroll
    for (int g = 0; g < kWaves - 1; ++g) take(extra, m, rec + (kOthers + g) * kRec);
    if (in5) finish(A, W, extra, m, row5);
  }
}

template <bool kFive>
__global__ void __launch_bounds__(kThreads, 2) k_paged_attn(Args A) {
  __shared__ __align__(16) uint8_t s_v[kLds];
  __shared__ double s_freq[kHeadDim / 2];
  __shared__ uint32_t s_bad[kTreeTiles / 2];  // tree rows whose values are not all finite
  __shared__ uint32_t s_see[(kWaves + 1) * kTile * (kTreeTiles / 2)];  // and those that each row may see
  // consecutive workgroups of one XCD share a key head's pages in its L2
  const int total = (int)gridDim.x, x = (int)blockIdx.x;
  const int lin = total % kXcds == 0 ? (x % kXcds) * (total / kXcds) + x / kXcds : x;
  const int chunk = lin % A.chunks;
  Work W;
  if (!W.init(A, lin / A.chunks, (int)blockIdx.y)) return;
  const int tile0 = chunk * kWaves, all = (W.M + kTile - 1) / kTile;
  const int tiles = chunk == A.chunks - 1 ? all - tile0 : kWaves;  // up to five with kFive
  if (kFive || tiles > 2) attend<2, kFive>(A, W, s_v, s_freq, s_bad, s_see, tile0, tiles);
  else attend<4, false>(A, W, s_v, s_freq, s_bad, s_see, tile0, tiles);
}

// One tile of query rows: the four waves go through every fourth page alone, two
// pages on their way in a wave's registers, and wait for nobody until the end.  One
// row over 3,000 tokens, 8 key heads: 13 us, of which the start - queries, tree rows,
// the first pages' latency - is 9; one over 131,000: 29 us (4.9 TB/s).
__global__ void __launch_bounds__(kThreads, 2) k_paged_attn_alone(Args A) {
  __shared__ __align__(16) uint8_t s_v[kWaves * kValues];
  __shared__ uint32_t s_bad[1];
  const int tid = (int)threadIdx.x, lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane(tid / fc::kWave);
  const int lg = lane >> 4, lc = lane & 15;
  const int total = (int)gridDim.x, x = (int)blockIdx.x;
  Work W;
  if (!W.init(A, total % kXcds == 0 ? (x % kXcds) * (total / kXcds) + x / kXcds : x, (int)blockIdx.y)) return;
  const bool rotate = A.log2_base > 0.0, in = lc < W.M;

  // The few query and tree rows (16 at most) are asked for ahead of the pages, which
  // would be waited for with them otherwise: a lane for a quarter of each row in
  // waves 0 (queries) and 1 (tree keys), one chunk of values a thread.
  const int six_r = lane >> 2, six_g = group_of(lane & 3), tree_r = six_r < W.n ? six_r : W.n - 1;
  const bool has_six = w == 0 || (w == 1 && W.tree && six_r < W.n);
  Group six;
  if (w == 0) load_group(W.q_row(A, W.row_at(six_r)), six_g, six);
  if (w == 1 && W.tree) load_group(W.k_row(A, tree_r), six_g, six);
  uint4 tree_values = make_uint4(0u, 0u, 0u, 0u);  // of row tid / 16; the rows from 16 on are zeros
  if (W.tree) tree_values = *(const uint4*)(W.v_row(A, tid / 16 < W.n ? tid / 16 : W.n - 1) + 8 * (tid % 16));

  struct Page {
    uint4 kf[4], vf[4];
    uint32_t ks, vs;
    bool have;
  };
  const int32_t* table = A.table + (int64_t)W.b * A.max_pages;
  int pg_next = W.pg0 + w, ids = 0;
  const auto load = [&](Page& p) {
    // page numbers of 64 steps at a time, in a register's lanes
    const int i = ((pg_next - W.pg0) / kWaves) & 63;
    if (i == 0) ids = pg_next + kWaves * lane < W.pg1 ? table[pg_next + kWaves * lane] : -1;
    const int id = __builtin_amdgcn_readlane(ids, i);
    pg_next += kWaves;
    p.have = id >= 0 && id < A.n_pages;
    if (!p.have) return;
    const uint8_t* page = A.pool + ((int64_t)id * A.Hkv + W.kv) * kPageBytes;
#pragma unroll
    for (int t = 0; t < 4; ++t) p.kf[t] = *(const uint4*)(page + (16 * t + lc) * fc::kCodeRow + 16 * lg);
    p.ks = *(const uint32_t*)(page + fc::kPageKScale + 4 * lane);
#pragma unroll
    for (int t = 0; t < 4; ++t) p.vf[t] = *(const uint4*)(page + fc::kPageV + (t * 64 + lane) * 16);
    p.vs = *(const uint32_t*)(page + fc::kPageVScale + 4 * lane);
  };
  Page even, odd;
  load(even);
  load(odd);

  // Meanwhile those rows go to LDS: sines and cosines of every position once, then
  // 6-bit parts.  Wave 0 has the tree's rows in its buffer, the others' hold the
  // rest until their pages come.
  uint8_t *six_k = s_v, *tree_v = s_v + kTile * kSixRow, *six_q = s_v + kValues;
  float2* turns = (float2*)(s_v + 2 * kValues);
  if (tid == 0) s_bad[0] = 0;
  if (rotate) {
    const double f = angle_of(lane, A.log2_base);
    for (int r = w; r < A.R; r += kWaves) turns[r * 64 + lane] = turn_of(W.position(W.behind(A, r)) * f);
  }
  __syncthreads();
  if (W.tree) {
    const int r = tid / 16, c = tid % 16;
    if (r >= W.n) tree_values = make_uint4(0u, 0u, 0u, 0u);
    if (keep_finite(tree_values)) atomicOr(&s_bad[0], 1u << r);
    *(uint4*)(tree_v + chunk_at(r, c)) = tree_values;
    *(uint4*)(tree_v + chunk_at(kTile + r, c)) = make_uint4(0u, 0u, 0u, 0u);
  }
  if (has_six) {
    const int tr = w == 0 ? W.row_at(six_r) / W.G : six_r;
    stage_six(six, six_g, w == 0 ? score_scale() : 1.0f, rotate,
              [&](int d) { return turns[tr * 64 + first_angle(six_g) + d]; }, (w == 0 ? six_q : six_k) + six_r * kSixRow);
  }
  __syncthreads();
  const Six q = read_six(six_q + lc * kSixRow, lg);
  __syncthreads();

  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_v;
  lds_u8* const v_lane = (lds_u8*)(uintptr_t)(lds0 + chunk_at(4 * lg + (lc >> 2), 0) + (uint32_t)(lc & 3) * 8u);
  Row me;
  me.clear();
  if (W.tree && w == 0) {
    const uint32_t see = W.allowed(A, in ? lc / W.G : 0, in, lg);
    floatx4 s[2];
    s[0] = score_six(read_six(six_k + lc * kSixRow, lg), q, me.minus_m);
    settle(s[0]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      s[0][e] = (see >> e) & 1u ? s[0][e] : -INFINITY;
      s[1][e] = -INFINITY;
    }
    bf16x2 x[4];
    weights(s, me, x);
    const bf16x8 pb = join(x[0], x[1], x[2], x[3]);
    all_values(v_lane + kTile * kSixRow, pb, me);
    const uint32_t bad = __builtin_amdgcn_readfirstlane(s_bad[0]);
    if (bad) W.add_marked(A, bad, 0, pb, see, lg, lc, me);
  }
  uint8_t* mine = s_v + w * kValues;
  lds_u8* const v_mine = v_lane + w * kValues;
  const auto step = [&](Page& p, int pg) {
    const int left = W.P - pg * kPage;
    if (!p.have) {
      load(p);
      return;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t) unpack(p.vf[t], p.vs, t, lane, left, mine);
    floatx4 s[4];
    s[0] = score<0>(p.kf[0], p.ks, q, me.minus_m);
    s[1] = score<1>(p.kf[1], p.ks, q, me.minus_m);
    s[2] = score<2>(p.kf[2], p.ks, q, me.minus_m);
    s[3] = score<3>(p.kf[3], p.ks, q, me.minus_m);
    load(p);
    settle(s[0], s[1], s[2], s[3]);
    if (left < kPage) {
#pragma unroll
      for (int t = 0; t < 4; ++t) cut(s[t], t, lg, left);
    }
    bf16x2 x[8];
    weights(s, me, x);
    all_values(v_mine, join(x[0], x[1], x[2], x[3]), me);
    all_values(v_mine + chunk_at(32, 0), join(x[4], x[5], x[6], x[7]), me);
  };
  for (int pg = W.pg0 + w; pg < W.pg1; pg += 2 * kWaves) {
    step(even, pg);
    step(odd, pg + kWaves);
  }

  whole(me);
  float m = me.m();
  float* rec = (float*)s_v;
  __syncthreads();
  if (w > 0) give(me, rec + (w - 1) * kRec);
  __syncthreads();
  if (w > 0) return;
#pragma unroll
  for (int g = 0; g < kWaves - 1; ++g) take(me, m, rec + g * kRec);
  if (in) finish(A, W, me, m, lc);
}

// The parts of a row put together: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m)
// l_s with m the largest m_s.  A wave per row: a lane has the weight of one or two
// parts, then each 16 lanes add up every fourth part, eight dims a lane.  A prefix
// in one part is in place already.  4 us for 32 rows of 3 parts, 5 for 2,080 of 12 or
// 32 of 64: a launch and three round trips to memory.
constexpr int kMergeWaves = 4;
__global__ void __launch_bounds__(kMergeWaves* fc::kWave) k_paged_merge(Args A) {
  const int G = A.H / A.Hkv, M = A.R * G;
  const int lane = fc::lane_id();
  const int64_t at = (int64_t)blockIdx.x * kMergeWaves + (int)(threadIdx.x / fc::kWave);  // (tree, key head, row)
  if (at >= (int64_t)A.B * A.Hkv * M) return;
  const int64_t bk = at / M;
  const int r = (int)(at - bk * M), b = (int)(bk / A.Hkv), kv = (int)(bk - (int64_t)b * A.Hkv);
  const int P = clamp_len(A.prefix_len[b], A.max_len);
  const int n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
  const int parts = parts_of((P + kPage - 1) / kPage, A.part_pages) + more_parts(n);
  if (parts == 1) return;
  const int64_t at0 = bk * A.parts * M + r;
  const bool has_x = lane < parts, has_y = lane + 64 < parts;
  float2 x = A.part_ml[at0 + (int64_t)(has_x ? lane : 0) * M], y = A.part_ml[at0 + (int64_t)(has_y ? lane + 64 : 0) * M];
  if (!has_x) x = make_float2(-INFINITY, 0.0f);
  if (!has_y) y = make_float2(-INFINITY, 0.0f);
  float m = fmaxf(x.x, y.x);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float wx = x.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.x - m);  // 0: a part without a key
  const float wy = y.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(y.x - m);
  float l = wx * x.y + wy * y.y;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
  const int d = 8 * (lane & 15);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  for (int s0 = 0; s0 < parts; s0 += 16) {
    floatx4 lo[4], hi[4];
    float w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + 4 * u + (lane >> 4), i = s < parts ? s : parts - 1;
      const float* po = A.part_o + (at0 + (int64_t)i * M) * kHeadDim + d;
      lo[u] = *(const floatx4*)po;
      hi[u] = *(const floatx4*)(po + 4);
      const float ww = __shfl(wx, i & 63);
      const float w2 = __shfl(wy, i & 63);
      w[u] = s < parts ? (i < 64 ? ww : w2) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += w[u] * lo[u][e];
        acc[4 + e] += w[u] * hi[u][e];
      }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    acc[e] += __shfl_xor(acc[e], 16);
    acc[e] += __shfl_xor(acc[e], 32);
  }
  if (lane >= 16) return;
  const int i = r / G;
  const float inv = i < n && l != 0.0f ? 1.0f / l : 0.0f;
  bf16x8 res;
#pragma unroll
  for (int e = 0; e < 8; ++e) res[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(acc[e] * inv);
  *(bf16x8*)(A.out + (((int64_t)b * A.R + i) * A.H + kv * G + (r - i * G)) * kHeadDim + d) = res;
}

struct Shape {
  int chunks, part_pages, parts;
  bool alone, five;
};

// How a call is laid out: a workgroup for every four tiles of query rows of a key
// head (or five: 65 rows are four tiles and one row), parts of the pages where
// that leaves the chip idle.
Shape shape_of(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  const int tiles = (R * (H / Hkv) + kTile - 1) / kTile;
  Shape s;
  s.alone = tiles == 1;
  s.five = tiles % kWaves == 1 && tiles > 1;
  s.chunks = s.five ? tiles / kWaves : (tiles + kWaves - 1) / kWaves;
  const int64_t wgs = (int64_t)B * Hkv * s.chunks;
  const int64_t pages = ((int64_t)max_len + kPage - 1) / kPage;
  // As many parts as the card takes at once.  From 64 pages on, one more where they
  // do not come out even, so that up to twice as many workgroups start: sequences
  // that are shorter than the longest then leave room that these take (40 trees of
  // 65 rows, 8 key heads, up to 8,192 tokens: 125 us, 174 without; 33 single tokens
  // 40 and 50; but equal lengths lose a little, 63 single tokens 110 and 102).
  // Shorter prefixes only pay the second round and the join for it (63 single tokens
  // over 2,048: 37 us, 29 without; 15 trees, 32 key heads: 106 and 76).  Parts have 4
  // pages at least, or 16 where each wave takes every fourth: 16 single tokens over
  // 2,048 17.9 us, with 4 19.0; a single one over 1,000 12.3 and 16.8, and from 3,000
  // on no difference.
  const int64_t slots = 2 * kCus;  // workgroups at once
  int64_t each = s.alone ? 16 : 4;
  int64_t parts = (slots + (pages < 64 ? 0 : wgs - 1)) / wgs;
  if (parts > kMostParts) parts = kMostParts;
  const int64_t fit = (pages + each - 1) / each;
  if (parts > fit) parts = fit;
  if (parts < 1) parts = 1;
  each = (pages + parts - 1) / parts;
  if (s.alone) each = (each + kWaves - 1) / kWaves * kWaves;
  s.part_pages = each < 1 ? 1 : (int)each;
  s.parts = (pages <= s.part_pages ? 1 : (int)((pages + s.part_pages - 1) / s.part_pages)) + more_parts(R);
  return s;
}

// Trees of a launch (and of the join after it): at least two at the largest sizes.
// Those behind them are a launch of their own, which uses the workspace again.
int32_t trees_at_once(int32_t B, int32_t R, int32_t H, int32_t Hkv, const Shape& s) {
  const int64_t wgs = (int64_t)Hkv * s.chunks, joins = ((int64_t)H * R + kMergeWaves - 1) / kMergeWaves;
  const int64_t most = fc::kMostGroups / (wgs > joins ? wgs : joins);
  return B < most ? B : (int32_t)most;
}

size_t carve(void* p, int64_t rows, float2** ml, float** o) {
  fc::Carver c(p);
  *ml = c.take<float2>((size_t)rows);
  *o = c.take<float>((size_t)rows * kHeadDim);
  return c.used + 256;
}

bool sizes_ok(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  return B >= 0 && B <= 65536 && R >= 1 && R <= FC_MAX_TREE_ROWS && Hkv >= 1 && Hkv <= 1024 && H >= Hkv && H <= 8192 &&
         H % Hkv == 0 && max_len >= 0 && max_len <= 0x7FFFFFFF - kPage;
}

}  // namespace

extern "C" size_t fc_paged_attention_workspace_bytes(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  if (!sizes_ok(B, R, H, Hkv, max_len) || B == 0) return 0;
  const Shape s = shape_of(B, R, H, Hkv, max_len);
  float2* ml;
  float* o;
  return s.parts > 1 ? carve(nullptr, (int64_t)trees_at_once(B, R, H, Hkv, s) * H * R * s.parts, &ml, &o) : 0;
}

extern "C" fc_status fc_paged_attention(const uint16_t* q, int64_t q_stride, const uint16_t* k_tree, int64_t k_stride,
                                        const uint16_t* v_tree, int64_t v_stride, const uint8_t* pool,
                                        int32_t n_pages, const int32_t* table, int32_t max_pages,
                                        const int32_t* prefix_len, const int32_t* num_nodes, const int32_t* mask,
                                        const int32_t* pos_ids, int32_t B, int32_t R, int32_t H, int32_t Hkv,
                                        int32_t D, int32_t max_len, float rope_base, uint16_t* out, void* ws,
                                        size_t ws_bytes, hipStream_t stream) {
  if (!sizes_ok(B, R, H, Hkv, max_len) || n_pages < 1 || n_pages > (1 << 25) - 1 || max_pages < 1 ||
      (int64_t)max_len > (int64_t)max_pages * kPage)
    return FC_ERR_INVALID;
  if (!(rope_base == 0.0f || (rope_base > 1.0f && rope_base < __builtin_inff()))) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D ||
      ((q_stride | k_stride | v_stride) & 7))
    return FC_ERR_INVALID;
  if (B == 0) return FC_OK;
  if (!q || !k_tree || !v_tree || !pool || !table || !prefix_len || !out) return FC_ERR_INVALID;
  if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)pool | (uintptr_t)out) & 15)
    return FC_ERR_INVALID;
  // sizes whose queries alone would pass 2^39 bytes
  if ((int64_t)B * Hkv * (((int64_t)R * (H / Hkv) + kTile - 1) / kTile) > 0x7FFFFFFF) return FC_ERR_UNSUPPORTED;
  const Shape s = shape_of(B, R, H, Hkv, max_len);
  const int32_t at_once = trees_at_once(B, R, H, Hkv, s);
  float2* part_ml = nullptr;
  float* part_o = nullptr;
  if (s.parts > 1) {
    if (!ws || ws_bytes < fc_paged_attention_workspace_bytes(B, R, H, Hkv, max_len)) return FC_ERR_WORKSPACE;
    if ((uintptr_t)ws & 15) return FC_ERR_INVALID;
    carve(ws, (int64_t)at_once * H * R * s.parts, &part_ml, &part_o);
  }
  // A workgroup reads its query rows before it writes the same rows of the result, so
  // out may be q itself; what other workgroups read has to lie elsewhere.
  const int64_t all = (int64_t)B * R;
  const bool in_place = out == q && q_stride == (int64_t)H * D;
  if (!fc::apart({fc::rows_span(out, all, (int64_t)H * D, (int64_t)H * D),
                  {s.parts > 1 ? ws : nullptr, fc_paged_attention_workspace_bytes(B, R, H, Hkv, max_len)}},
                 {fc::rows_span(in_place ? nullptr : q, all, q_stride, (int64_t)H * D),
                  fc::rows_span(k_tree, all, k_stride, (int64_t)Hkv * D),
                  fc::rows_span(v_tree, all, v_stride, (int64_t)Hkv * D),
                  {pool, fc_paged_pool_bytes(n_pages, Hkv)},
                  {table, 4 * (uint64_t)B * max_pages},
                  {prefix_len, 4 * (uint64_t)B},
                  {num_nodes, 4 * (uint64_t)B},
                  {mask, 4 * (uint64_t)all * R},
                  {pos_ids, 4 * (uint64_t)all}}))
    return FC_ERR_INVALID;
  (void)hipGetLastError();
  for (int32_t b = 0; b < B; b += at_once) {
    const int32_t now = B - b < at_once ? B - b : at_once;
    const int64_t row = (int64_t)b * R;
    const Args a = {q + row * q_stride, k_tree + row * k_stride, v_tree + row * v_stride, q_stride, k_stride, v_stride,
                    pool, table + (int64_t)b * max_pages, prefix_len + b, num_nodes ? num_nodes + b : nullptr,
                    mask ? mask + row * R : nullptr, pos_ids ? pos_ids + row : nullptr, n_pages, max_pages, now, R, H,
                    Hkv, max_len, s.chunks, s.part_pages, s.parts, rope_base != 0.0f ? log2((double)rope_base) : 0.0,
                    out + row * H * kHeadDim, part_ml, part_o};
    const dim3 grid((uint32_t)now * (uint32_t)Hkv * (uint32_t)s.chunks, (uint32_t)s.parts);
    if (s.alone)
      hipLaunchKernelGGL(k_paged_attn_alone, grid, dim3(kThreads), 0, stream, a);
    else if (s.five)
      hipLaunchKernelGGL(k_paged_attn<true>, grid, dim3(kThreads), 0, stream, a);
    else
      hipLaunchKernelGGL(k_paged_attn<false>, grid, dim3(kThreads), 0, stream, a);
    FC_CHECK_LAUNCH();
    if (s.parts > 1) {
      const uint64_t rows = (uint64_t)now * H * R;
      hipLaunchKernelGGL(k_paged_merge, dim3(fc::div_up(rows, kMergeWaves)), dim3(kMergeWaves * fc::kWave), 0, stream, a);
      FC_CHECK_LAUNCH();
    }
  }
  return FC_OK;
}

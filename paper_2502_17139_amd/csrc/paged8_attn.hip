// Tree attention over the 8-bit paged cache on gfx950 matrix cores
// (fc_paged_byte_attention).
//
// The rows of a tree that share a key head - its R rows times the H / Hkv query
// heads of the group - are one matrix of queries, cut into tiles of 16 rows.  Per
// page of 64 keys a wave computes the transposed scores S^T = K Q^T and O^T += V^T
// P^T, which keeps a lane's scores where the second product wants its weights.
// Codes become bf16 in registers, right before their product: keys and queries are
// exact there (a code has four significant bits), and products of bf16 are summed in
// fp32.  (The 8-bit products, which would take the codes as they lie, drop what is
// below 2^-13 of a sum's largest term: scores would be off by as much.)
//
// Which key a lane has is free as long as both products agree, and is chosen so that
// every load is 16 bytes a lane and none is turned around: row 4 a + b of score tile
// t is key 16 a + 4 t + b, so that after four tiles lane (lg, lc) has the scores of
// query row lc with keys 16 lg .. 16 lg + 15, and of each dim the value codes of those
// 16 tokens are one piece of a page.  A key block's scale multiplies the lane's
// scores, a value block's goes into the conversion.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastcoder.h"
#include "fc_device.h"
#include "fc_host.h"
#include "fc_page8.h"

namespace {

using fc::kDim8;
using fc::kPage8;
using fc::kPage8Bytes;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;
typedef __attribute__((address_space(3))) uint8_t lds_u8;

constexpr int kTile = 16;                     // query rows of a tile
constexpr int kWaves = 4;                     // of a workgroup: one for each SIMD
constexpr int kThreads = kWaves * fc::kWave;
constexpr int kDTiles = kDim8 / 16;           // output tiles of 16 dims
constexpr int kKTiles = kPage8 / 16;          // score tiles of a page
constexpr int kWaveTiles = 2;                 // query tiles of a wave, at most
constexpr int kGroupTiles = kWaves * kWaveTiles;
constexpr int kRowBytes = kDim8 * 2 + 32;     // a tree's value row in LDS
constexpr int kSlots = 4;                     // pages on their way or in use
constexpr int kSlot = 2 * fc::kPage8V;        // a page's codes in LDS: 16 KB
constexpr int kMostParts = 128;               // of a prefix: a merging lane has two
constexpr int kXcds = 8;
constexpr int kCus = 256;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

struct Args {
  const uint16_t *q, *k_tree, *v_tree;
  int64_t q_stride, k_stride, v_stride;
  const uint8_t* pool;
  const int32_t *table, *prefix_len, *num_nodes, *mask;
  int n_pages, max_pages, B, R, H, Hkv, max_len, tiles, chunks, part_pages, parts, ordered;
  uint16_t* out;
  float* lse;
  float4* part_ml;
  float* part_o;
};

__device__ __forceinline__ int clamp_len(int len, int most) { return len < 0 ? 0 : (len > most ? most : len); }
__device__ __forceinline__ float score_scale() { return kLog2e / sqrtf((float)kDim8); }

// Eight codes as bf16, times a power of two.
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b, float s) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, s, true);
  const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, s, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}
__device__ __forceinline__ floatx4 product(const bf16x8& a, const bf16x8& b, const floatx4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// A product's result is read by ordinary instructions only some cycles after it was
// issued.  The compiler counts them along one way where a branch lies between, so the
// wait stands here, before any branch.
__device__ __forceinline__ void settle(floatx4 (&s)[kKTiles]) {
  asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1]), "+v"(s[2]), "+v"(s[3]));
}

// Parts that a prefix is cut into.
__device__ __forceinline__ int parts_of(int pages, int part_pages) {
  return pages <= part_pages ? 1 : (pages + part_pages - 1) / part_pages;
}

// Which of n (tree, key head) pairs, in `chunks` workgroups each, workgroup x has: an
// XCD gets every eighth workgroup, so a pair's workgroups lie eight apart, to share its
// pages in one L2, and pairs that follow each other, which have one tree's length, are
// spread over all XCDs.
struct Place {
  int pair, chunk;
};
__device__ __forceinline__ Place place_of(int x, int n, int chunks) {
  const int whole = n / kXcds * kXcds;  // pairs in rounds of eight
  if (x < whole * chunks) return Place{x / (kXcds * chunks) * kXcds + x % kXcds, x / kXcds % chunks};
  return Place{x / chunks, x % chunks};
}

// The tree with the r-th longest prefix, in pages; of equal ones the first is longer.  A
// wave holds the lengths, four a lane, and finds the r-th largest bit by bit, by counting.
constexpr int kOrdered = 4 * fc::kWave;  // trees of a launch, at most
__device__ __forceinline__ int longest(const Args& A, int r) {
  const int lane = fc::lane_id();
  int pages[kOrdered / fc::kWave];
#pragma unroll
  for (int i = 0; i < kOrdered / fc::kWave; ++i) {
    const int b = fc::kWave * i + lane;
    pages[i] = b < A.B ? (clamp_len(A.prefix_len[b], A.max_len) + kPage8 - 1) / kPage8 : -1;
  }
  const auto count = [&](int least) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kOrdered / fc::kWave; ++i) n += (int)__popcll(fc::ballot(pages[i] >= least));
    return n;
  };
  int v = 0;
  for (int bit = 31 - __builtin_clz((A.max_len + kPage8 - 1) / kPage8 | 1); bit >= 0; --bit)
    if (count(v | 1 << bit) > r) v |= 1 << bit;
  r -= count(v + 1);
#pragma unroll
  for (int i = 0; i < kOrdered / fc::kWave; ++i) {
    uint64_t same = fc::ballot(pages[i] == v);
    const int n = (int)__popcll(same);
    if (r < n) {
      for (; r > 0; --r) same &= same - 1;
      return fc::kWave * i + (int)__builtin_ctzll(same);
    }
    r -= n;
  }
  return 0;
}

// What a workgroup works on.
struct Work {
  int bk, b, kv, G, M, P, n, part, parts, pg0, pg1;
  bool tree;
  __device__ __forceinline__ bool init(const Args& A, int pair, int part_) {
    part = part_;
    b = pair / A.Hkv, kv = pair - b * A.Hkv;
    if (A.ordered) b = __builtin_amdgcn_readfirstlane(longest(A, b));
    bk = b * A.Hkv + kv;
    G = A.H / A.Hkv, M = A.R * G;
    P = clamp_len(A.prefix_len[b], A.max_len);
    n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
    const int pages = (P + kPage8 - 1) / kPage8;
    parts = parts_of(pages, A.part_pages);
    if (part >= parts) return false;
    pg0 = part * A.part_pages;
    pg1 = part < parts - 1 ? pg0 + A.part_pages : pages;
    tree = part == parts - 1 && n > 0;  // the last part has the tree's rows
    return true;
  }
  // rows past the last one: the last one, whose results nobody takes
  __device__ __forceinline__ const uint16_t* q_row(const Args& A, int r) const {
    r = r < M ? r : M - 1;
    const int tr = r / G;
    return A.q + ((int64_t)b * A.R + tr) * A.q_stride + ((int64_t)kv * G + (r - tr * G)) * kDim8;
  }
  __device__ __forceinline__ const uint16_t* k_row(const Args& A, int j) const {
    return A.k_tree + ((int64_t)b * A.R + j) * A.k_stride + (int64_t)kv * kDim8;
  }
  __device__ __forceinline__ const uint16_t* v_row(const Args& A, int j) const {
    return A.v_tree + ((int64_t)b * A.R + j) * A.v_stride + (int64_t)kv * kDim8;
  }
  // Bit 4 t + e: query row r may see tree row j0 + 16 t + 4 lg + e, of T tiles.
  template <int T>
  __device__ __forceinline__ uint32_t allowed(const Args& A, int r, int j0, int lg) const {
    uint32_t bits = 0;
    if (r >= M) return 0;
    const int tr = r / G;
    const int32_t* row = A.mask + ((int64_t)b * A.R + tr) * A.R;
    int m[4 * T];
#pragma unroll
    for (int u = 0; u < 4 * T; ++u) {
      const int j = j0 + 16 * (u / 4) + 4 * lg + u % 4;
      m[u] = A.mask ? row[j < n ? j : 0] : (j <= tr);
    }
#pragma unroll
    for (int u = 0; u < 4 * T; ++u) bits |= (uint32_t)(m[u] == 1 && j0 + 16 * (u / 4) + 4 * lg + u % 4 < n) << u;
    return bits;
  }
  // Whether query row r, of the wave's 16, may see any key of this part.
  __device__ __forceinline__ bool sees(const Args& A, int r) const {
    const int lane = fc::lane_id();
    const int32_t* of = A.table + (int64_t)b * A.max_pages;
    bool page = false;
    for (int pg = pg0; pg < pg1 && !page; pg += fc::kWave) {
      const int id = pg + lane < pg1 ? of[pg + lane] : -1;
      page = fc::ballot(id >= 0 && id < A.n_pages) != 0;
    }
    int rows = 0;
    if (tree)
      for (int j0 = 0; j0 < n; j0 += 16) rows |= (int)allowed<1>(A, r, j0, lane >> 4);
    rows |= __shfl_xor(rows, 16);
    rows |= __shfl_xor(rows, 32);
    return page || rows != 0;
  }
};

// A query row's outputs (lane (lg, lc): dims 16 t + 4 lg + e of row lc), its running
// maximum as 0 - m (0 while there is none), the sum of its weights as the value
// product sees them, the same before they are rounded (for the row's logarithm), and
// whether it is yet to see a key.
struct Row {
  floatx4 o[kDTiles];
  float minus_m, l, x;
  bool first;
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) o[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    minus_m = l = x = 0.0f;
    first = true;
  }
  __device__ __forceinline__ float m() const { return first ? -INFINITY : 0.0f - minus_m; }
};

// A tile of query rows: lane (lg, lc) has dims 64 u + 16 lg + 8 h .. + 7 of row lc in
// q[2 u + h], as the key codes lie.
struct Tile {
  bf16x8 q[4];
  Row row;
  __device__ __forceinline__ void load(const uint16_t* p, int lg) {
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = *(const bf16x8*)(p + 64 * (u / 2) + 16 * lg + 8 * (u % 2));
    row.clear();
  }
};

// The softmax's usual step is a multiplication and a power of two for each score, a
// rounding and a share of a sum for two, and no maximum: m is the maximum of what the
// row saw when it was last scaled.  A factor common to a row's weights costs no
// accuracy, bf16 and fp32 having the same exponents, as long as sums do not overflow:
// each of the four lanes that share a row and a page adds less than 2^22 times the
// largest value, and 2^31 tokens are 2^25 pages: 2^49 in all, so values below 2^78 stay
// in.  A step in which a lane's weights add up to 2^22 or more (or to a NaN) is taken
// again with m raised to its maximum, and so is a row's first.
constexpr float kMostWeight = 4194304.0f;  // 2^22

template <bool kLse, int T>
__device__ __forceinline__ float weigh(const floatx4 (&s)[T], float scale, float minus_m, bf16x2 (&p)[2 * T], float& x) {
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
  float sum = 0.0f;
  x = 0.0f;
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * e], scale, minus_m));
      const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][2 * e + 1], scale, minus_m));
      p[2 * t + e] = bf16x2{(__bf16)a, (__bf16)b};
      sum = __builtin_amdgcn_fdot2_f32_bf16(p[2 * t + e], one, sum, false);
      if (kLse) x += a, x += b;
    }
  return sum;
}
__device__ __forceinline__ bool too_much(float sum, const Row& r) {
  return !(sum < (r.first ? -1.0f : kMostWeight));
}
template <int T>
__device__ __forceinline__ void raise(const floatx4 (&s)[T], float scale, Row& r, bool need) {
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < T; ++t) {
    top = fmaxf(fmaxf(top, s[t][0]), s[t][1]);
    top = fmaxf(fmaxf(top, s[t][2]), s[t][3]);
  }
  // lanes of a row have blocks of different scales
  float mx = top == -INFINITY ? top : __builtin_fmaf(top, scale, r.minus_m);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  int row_needs = need;
  row_needs |= __shfl_xor(row_needs, 16);
  row_needs |= __shfl_xor(row_needs, 32);
  // by how much m rises; a row that has no need keeps it, so that its result goes by
  // its own scores alone
  const bool rise = row_needs != 0 && mx != -INFINITY;
  const float by = rise ? mx : 0.0f;
  const float alpha = r.first ? 0.0f : __builtin_amdgcn_exp2f(-by);
  r.l *= alpha;
  r.x *= alpha;
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) r.o[t] *= alpha;
  r.minus_m -= by;
  r.first = r.first && !rise;
}
template <bool kLse, int NT, int T>
__device__ __forceinline__ void weights(const floatx4 (&s)[NT][T], float scale, Tile (&tile)[kWaveTiles],
                                        bf16x2 (&p)[NT][2 * T]) {
  float sum[NT], x[NT];
  bool again = false;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    sum[i] = weigh<kLse>(s[i], scale, tile[i].row.minus_m, p[i], x[i]);
    again |= too_much(sum[i], tile[i].row);
  }
  if (__any(again)) {
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      raise(s[i], scale, tile[i].row, too_much(sum[i], tile[i].row));
      sum[i] = weigh<kLse>(s[i], scale, tile[i].row.minus_m, p[i], x[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    tile[i].row.l += sum[i];
    tile[i].row.x += x[i];
  }
}
__device__ __forceinline__ bf16x8 join(const bf16x2& a, const bf16x2& b, const bf16x2& c, const bf16x2& d) {
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// A page's scores with NT tiles: key(t, u) gives the codes of a lane's key of score
// tile t, dims 64 u + 16 lg .. + 15.
template <int NT, typename Key>
__device__ __forceinline__ void page_scores(Key key, const Tile (&tile)[kWaveTiles], floatx4 (&s)[NT][kKTiles]) {
#pragma unroll
  for (int t = 0; t < kKTiles; ++t)
#pragma unroll
    for (int i = 0; i < NT; ++i) s[i][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < 2; ++u) {  // no product waits for the one before
    uint4 c[kKTiles];
#pragma unroll
    for (int t = 0; t < kKTiles; ++t) c[t] = key(t, u);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int t = 0; t < kKTiles; ++t) {
        const bf16x8 a = h ? widen(c[t].z, c[t].w, 1.0f) : widen(c[t].x, c[t].y, 1.0f);
#pragma unroll
        for (int i = 0; i < NT; ++i) s[i][t] = product(a, tile[i].q[2 * u + h], s[i][t]);
      }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i) settle(s[i]);
}
// Keys 16 lg + 4 t + e from `left` on do not count.
template <int NT>
__device__ __forceinline__ void cut(floatx4 (&s)[NT][kKTiles], int lg, int left) {
  const int live = left - 16 * lg;  // of the lane's keys
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int t = 0; t < kKTiles; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) s[i][t][e] = 4 * t + e < live ? s[i][t][e] : -INFINITY;
}
// And that what their bytes hold does not matter, a weight of 0 times a NaN being
// one, their values are 0.
__device__ __forceinline__ uint4 cut_values(uint4 c, int lg, int left) {
  const int live = left - 16 * lg;  // of 16 codes
  uint32_t* w = (uint32_t*)&c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int n = live - 4 * i;
    w[i] = n >= 4 ? w[i] : n <= 0 ? 0u : w[i] & (0xFFFFFFFFu >> (32 - 8 * n));
  }
  return c;
}
// The scales of a lane's 16 keys and their values; `left`: as above.  A block without
// a key that counts may never have been written.
__device__ __forceinline__ float key_scale(uint32_t word, int lg, int left) {
  const float s = fc::scale8((word >> (8 * (lg >> 1))) & 255u);
  return 32 * (lg >> 1) < left ? s : 1.0f;
}
__device__ __forceinline__ float value_scale(uint32_t word, int lg, int left) { return key_scale(word >> 16, lg, left); }

// A page's values, with the weights of NT tiles: value(t) gives the codes of a lane's 16
// tokens at dim 16 t + lc.
template <int NT, typename Value>
__device__ __forceinline__ void page_values(Value value, float scale, const bf16x2 (&p)[NT][2 * kKTiles],
                                            Tile (&tile)[kWaveTiles]) {
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) {
    const uint4 c = value(t);
    const bf16x8 a = widen(c.x, c.y, scale), b = widen(c.z, c.w, scale);
#pragma unroll
    for (int i = 0; i < NT; ++i) tile[i].row.o[t] = product(a, join(p[i][0], p[i][1], p[i][2], p[i][3]), tile[i].row.o[t]);
#pragma unroll
    for (int i = 0; i < NT; ++i) tile[i].row.o[t] = product(b, join(p[i][4], p[i][5], p[i][6], p[i][7]), tile[i].row.o[t]);
  }
}

// The value rows of up to 64 of a tree's tokens lie in LDS, kRowBytes apart (32 bytes
// more than their values, so that a transposing read meets every bank once).  Such a
// read gives lane (lg, lc) dims 16 t + lc of rows 4 lg + e; `at` is the lane's place.
template <int NT, int T>
__device__ __forceinline__ void tree_values(lds_u8* at, const bf16x2 (&p)[NT][2 * T], Tile (&tile)[kWaveTiles]) {
#pragma unroll
  for (int t = 0; t < kDTiles; ++t)
#pragma unroll
    for (int u = 0; u < T / 2; ++u) {
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + 32 * u * kRowBytes + 32 * t));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + (32 * u + 16) * kRowBytes + 32 * t));
      const bf16x8 a = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
      for (int i = 0; i < NT; ++i)
        tile[i].row.o[t] = product(a, join(p[i][4 * u], p[i][4 * u + 1], p[i][4 * u + 2], p[i][4 * u + 3]), tile[i].row.o[t]);
    }
}
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
// Values that are not finite are 0 in LDS, as rows that do not see them must not meet
// them; this adds them for the rows that do.  Bit j of `bad` marks tree row j0 + j.
template <int T>
__device__ __forceinline__ void add_marked(const Args& A, const Work& W, uint64_t bad, int j0, const bf16x2 (&p)[2 * T],
                                           uint32_t see, Row& r) {
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  for (; bad; bad &= bad - 1) {
    const int j = __builtin_ctzll(bad);
    const int u = j / 16 * 4 + j % 4, from = j % 16 / 4 * 16 + lc;  // whose weight for row j it is, and where
    float weight = 0.0f;
#pragma unroll
    for (int e = 0; e < 4 * T; ++e) weight = e == u ? (float)p[e / 2][e % 2] : weight;
    weight = __shfl(weight, from);
    const bool sees = (__shfl((int)see, from) >> u) & 1;
    const uint16_t* v = W.v_row(A, j0 + j) + 4 * lg;
#pragma unroll
    for (int t = 0; t < kDTiles; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t x = (uint32_t)v[16 * t + e] << 16;
        r.o[t][e] += sees && (x & 0x7F800000u) == 0x7F800000u ? weight * __uint_as_float(x) : 0.0f;
      }
  }
}
// Scores of up to 16 T tree rows from j0 on, whose keys are read where they are.
template <int NT, int T>
__device__ __forceinline__ void tree_scores(const Args& A, const Work& W, int j0, const Tile (&tile)[kWaveTiles],
                                            floatx4 (&s)[NT][T]) {
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int i = 0; i < NT; ++i) s[i][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    if (j0 + 16 * t >= W.n) continue;
    const int j = j0 + 16 * t + lc;
    const uint16_t* p = W.k_row(A, j < W.n ? j : W.n - 1) + 16 * lg;
    bf16x8 k[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) k[u] = *(const bf16x8*)(p + 64 * (u / 2) + 8 * (u % 2));
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int i = 0; i < NT; ++i) s[i][t] = product(k[u], tile[i].q[u], s[i][t]);
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int t = 0; t < T; ++t) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[i][t]));
}
template <int NT, int T>
__device__ __forceinline__ void hide(floatx4 (&s)[NT][T], const uint32_t (&see)[NT]) {
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int u = 0; u < 4 * T; ++u) s[i][u / 4][u % 4] = (see[i] >> u) & 1u ? s[i][u / 4][u % 4] : -INFINITY;
}

// ---- results

__device__ __forceinline__ void whole(Row& r) {
  r.l += __shfl_xor(r.l, 16);
  r.l += __shfl_xor(r.l, 32);
  r.x += __shfl_xor(r.x, 16);
  r.x += __shfl_xor(r.x, 32);
}
// Waves that shared a tile's keys hand over to one of them, through LDS.
constexpr int kRec = kTile * kDim8 + 3 * kTile;  // floats of a tile: outputs, maxima, both sums
__device__ __forceinline__ void give(const Row& r, float m, float* rec) {
  const int lane = fc::lane_id();
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) *(floatx4*)(rec + (t * 64 + lane) * 4) = r.o[t];
  if (lane < 16) {
    float* s = rec + kTile * kDim8 + lane;
    s[0] = m, s[kTile] = r.l, s[2 * kTile] = r.x;
  }
}
__device__ __forceinline__ void take(Row& r, float& m, const float* rec) {
  const int lane = fc::lane_id();
  const float* s = rec + kTile * kDim8 + (lane & 15);
  const float m2 = s[0], both = fmaxf(m, m2);
  const float a1 = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m - both);
  const float a2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - both);
  m = both;
  r.l = r.l * a1 + s[kTile] * a2;
  r.x = r.x * a1 + s[2 * kTile] * a2;
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) r.o[t] = r.o[t] * a1 + *(const floatx4*)(rec + (t * 64 + lane) * 4) * a2;
}
// A row whose weights add up to nothing saw no key, or none but of scores of -infinity
// (an infinity in its query, a product past fp32).  Those are no keys beside others, but
// alone their softmax is a NaN: such a row's maximum is the lowest number, which any
// other key's weights leave without effect when rows are put together.  Whether it saw
// one is looked for here, where that is rare: kept from the loops over keys, it would
// take registers there (48 trees of 65 rows: 2 us).
constexpr float kLowest = -3.402823466e38f;
__device__ __forceinline__ float maximum_of(const Args& A, const Work& W, const Row& r, float m, int row) {
  const bool nothing = row < W.M && r.l == 0.0f;
  if (!__any(nothing)) return m;
  const bool sees = W.sees(A, row);
  return nothing && sees ? kLowest : m;
}
// 1 over a row's sum: 0 for a row without a key; infinite, so that its outputs of 0
// become NaN, for one of scores of -infinity alone.
__device__ __forceinline__ float inverse(float m, float l) { return l == 0.0f && m == -INFINITY ? 0.0f : 1.0f / l; }
__device__ __forceinline__ float log_sum(float m, float x) {
  if (x == 0.0f) return m == -INFINITY ? m : __builtin_nanf("");
  return (m + __builtin_amdgcn_logf(x)) * kLn2;  // base 2; a row of NaN alone has no m
}
__device__ __forceinline__ void finish(const Args& A, const Work& W, const Row& r, float m, int row) {
  const int lg = fc::lane_id() >> 4;
  if (W.parts > 1) {
    const int64_t at = ((int64_t)W.bk * A.parts + W.part) * W.M + row;
    if (lg == 0) A.part_ml[at] = make_float4(m, r.l, r.x, 0.0f);
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) *(floatx4*)(A.part_o + at * kDim8 + 16 * t + 4 * lg) = r.o[t];
    return;
  }
  // a row without a key has weight 0; a NaN stays one
  const int tr = row / W.G;
  const float inv = tr < W.n ? inverse(m, r.l) : 0.0f;
  const int64_t at = ((int64_t)W.b * A.R + tr) * A.H + W.kv * W.G + (row - tr * W.G);
#pragma unroll
  for (int t = 0; t < kDTiles; ++t) {
    bf16x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(r.o[t][e] * inv);
    *(bf16x4*)(A.out + at * kDim8 + 16 * t + 4 * lg) = x;
  }
  if (A.lse && lg == 0) A.lse[at] = tr < W.n ? log_sum(m, r.x) : -INFINITY;
}

// One or two tiles of query rows (a decoded token, a short chain): a workgroup's waves
// go through every fourth (or eighth) page alone, out of registers, and wait for
// nobody until the end.  A page's keys are asked for while the one before has its
// weights, its values while the next scores are made.  Bound by memory, 16.5 KB a page
// and head: 131,000 tokens of 8 key heads 43 us and 5 for the join, 5.7 TB/s; 64 sequences
// of up to 8,192 tokens 77 us, 4.7 TB/s; 3,000 tokens 10 and 4 us, a chain of round trips.
// 208 registers for one tile, no scratch; 256 for two, and 84 bytes of scratch a lane (8
// without logarithms).
template <int NT, int kAloneWaves, bool kLse>
__global__ void __launch_bounds__(kAloneWaves* fc::kWave, 2) k_paged8_attn_alone(Args A) {
  constexpr int T = 2;  // tiles of tree rows: at most 32
  constexpr int kTree = 16 * T * kRowBytes, kGiven = kAloneWaves / 2 * NT * kRec * 4;
  __shared__ __align__(16) uint8_t s_x[kTree > kGiven ? kTree : kGiven];
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave);
  Work W;
  if (!W.init(A, place_of((int)blockIdx.x, (int)gridDim.x, 1).pair, (int)blockIdx.y)) return;

  uint4 k[kKTiles][2], v[kDTiles];
  uint32_t k_word = 0, v_word = 0;
  const int32_t* table = A.table + (int64_t)W.b * A.max_pages;
  // page numbers, 64 steps at a time in a register's lanes
  int ids = 0;
  const auto id_of = [&](int pg) {
    const int i = ((pg - W.pg0) / kAloneWaves) & 63;
    if (i == 0) ids = pg + kAloneWaves * lane < W.pg1 ? table[pg + kAloneWaves * lane] : -1;
    return __builtin_amdgcn_readlane(ids, i);
  };
  const auto there = [&](int id) { return id >= 0 && id < A.n_pages; };
  const auto page_of = [&](int id) { return A.pool + ((int64_t)id * A.Hkv + W.kv) * kPage8Bytes; };
  // a lane's places in a page: 32 bits behind an address that all lanes share
  const uint32_t k_at = (uint32_t)((16 * (lc >> 2) + (lc & 3)) * kDim8 + 16 * lg);
  const uint32_t v_at = (uint32_t)(fc::kPage8V + lg * 2048 + lc * 16);
  const auto load_k = [&](int id) {
    const uint8_t* p = page_of(id);
#pragma unroll
    for (int t = 0; t < kKTiles; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) k[t][u] = *(const uint4*)(p + k_at + (4 * t * kDim8 + 64 * u));
    k_word = *(const uint32_t*)(p + fc::kPage8Scales);
  };
  const auto load_v = [&](int id) {
    const uint8_t* p = page_of(id);
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) v[t] = *(const uint4*)(p + v_at + 256 * t);
    v_word = *(const uint32_t*)(p + fc::kPage8Scales);
  };
  int pg = W.pg0 + w, id = pg < W.pg1 ? id_of(pg) : -1;
  Tile tile[kWaveTiles];
#pragma unroll
  for (int i = 0; i < NT; ++i) tile[i].load(W.q_row(A, kTile * i + lc), lg);
  if (there(id)) load_k(id), load_v(id);

  // The tree's own rows are the last wave's, whose pages may be fewer: one tile's while
  // the first page is on its way, two tiles' after the last one, for want of registers.
  const auto attend_tree = [&]() {
    uint64_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4 * T; ++i) {
      const int r = 4 * i + lg;
      uint4 val = make_uint4(0u, 0u, 0u, 0u);
      if (r < W.n) val = *(const uint4*)(W.v_row(A, r) + 8 * lc);
      uint64_t any = fc::ballot(keep_finite(val));
#pragma unroll
      for (int g = 0; g < 4; ++g) bad |= (uint64_t)(((any >> (16 * g)) & 0xFFFFu) != 0) << (4 * i + g);
      *(uint4*)(s_x + r * kRowBytes + 16 * lc) = val;
    }
    floatx4 s[NT][T];
    tree_scores<NT, T>(A, W, 0, tile, s);
    uint32_t see[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) see[i] = W.allowed<T>(A, kTile * i + lc, 0, lg);
    hide<NT, T>(s, see);
    bf16x2 p[NT][2 * T];
    weights<kLse, NT, T>(s, score_scale(), tile, p);
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)s_x;
    lds_u8* const at = (lds_u8*)(uintptr_t)(lds0 + (uint32_t)((4 * lg + (lc >> 2)) * kRowBytes + (lc & 3) * 8));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    tree_values<NT, T>(at, p, tile);
    if (bad) {
#pragma unroll
      for (int i = 0; i < NT; ++i) add_marked<T>(A, W, bad, 0, p[i], see[i], tile[i].row);
    }
  };
  if (NT == 1 && W.tree && w == kAloneWaves - 1) attend_tree();

  for (; pg < W.pg1; pg += kAloneWaves) {
    const int next = pg + kAloneWaves < W.pg1 ? id_of(pg + kAloneWaves) : -1;
    if (!there(id)) {
      id = next;
      if (there(id)) load_k(id), load_v(id);
      continue;
    }
    const int left = W.P - pg * kPage8;
    floatx4 s[NT][kKTiles];
    page_scores<NT>([&](int t, int u) { return k[t][u]; }, tile, s);
    const float ks = key_scale(k_word, lg, left) * score_scale(), vs = value_scale(v_word, lg, left);
    if (NT == 1 && there(next)) load_k(next);
    if (left < kPage8) {
      cut<NT>(s, lg, left);
#pragma unroll
      for (int t = 0; t < kDTiles; ++t) v[t] = cut_values(v[t], lg, left);
    }
    bf16x2 p[NT][2 * kKTiles];
    weights<kLse, NT, kKTiles>(s, ks, tile, p);
    if (NT == 2 && there(next)) load_k(next);  // the scores' registers are free
    page_values<NT>([&](int t) { return v[t]; }, vs, p, tile);
    if (there(next)) load_v(next);
    id = next;
  }

  if (NT == 2 && W.tree && w == kAloneWaves - 1) attend_tree();

  // half of the waves hand over to the others, until one has all
  float* rec = (float*)s_x;
  float m[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    whole(tile[i].row);
    m[i] = tile[i].row.m();
  }
#pragma unroll
  for (int half = kAloneWaves / 2; half >= 1; half /= 2) {
    __syncthreads();
    if (w >= half && w < 2 * half) {
#pragma unroll
      for (int i = 0; i < NT; ++i) give(tile[i].row, m[i], rec + ((w - half) * NT + i) * kRec);
    }
    __syncthreads();
    if (w < half) {
#pragma unroll
      for (int i = 0; i < NT; ++i) take(tile[i].row, m[i], rec + (w * NT + i) * kRec);
    }
  }
  if (w > 0) return;
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int row = kTile * i + lc;
    m[i] = maximum_of(A, W, tile[i].row, m[i], row);
    if (row < W.M) finish(A, W, tile[i].row, m[i], row);
  }
}

// More tiles: a workgroup's four waves take up to eight of them through the same pages,
// which go straight from memory into LDS as they lie (16 bytes a lane, no registers),
// two on their way while a third is used.  The keys' pieces of 16 bytes change places
// by the row, so that a wave reads its 16 rows without two lanes in a bank.
__device__ __forceinline__ int swap_of(int row) { return ((row >> 3) & 6) | ((row >> 1) & 1); }

// Pages on their way into LDS: a wave issues a quarter of each.
struct Pages {
  const Args& A;
  const Work& W;
  const int32_t* table;
  uint32_t lds0;
  int w;
  // page numbers and scales, 64 at a time in a register's lanes: read one by one they
  // would be loads to wait for among the loads that are meant to stay in flight
  int ids, words;
  static constexpr int kLoads = kSlot / (16 * fc::kWave) / kWaves;  // of a wave and page
  __device__ __forceinline__ Pages(const Args& a, const Work& work, uint8_t* lds, int wave)
      : A(a), W(work), table(a.table + (int64_t)work.b * a.max_pages), lds0((uint32_t)(uintptr_t)(lds_u8*)lds), w(wave),
        ids(0), words(0) {}
  __device__ __forceinline__ int slot_of(int pg) const { return ((pg - W.pg0) & (kSlots - 1)) * kSlot; }
  // Whether page pg is there, and its scales.
  __device__ __forceinline__ bool issue(int pg, int& word) {
    const int lane = fc::lane_id(), i = (pg - W.pg0) & 63;
    if (i == 0) {
      ids = pg + lane < W.pg1 ? table[pg + lane] : -1;
      const bool there = ids >= 0 && ids < A.n_pages;
      if (!there) ids = -1;
      words = there ? *(const int*)(A.pool + ((int64_t)ids * A.Hkv + W.kv) * kPage8Bytes + fc::kPage8Scales) : 0;
      asm volatile("" : "+v"(words));  // waited for here, as the queries are
    }
    const int id = __builtin_amdgcn_readlane(ids, i);
    word = __builtin_amdgcn_readlane(words, i);
    const bool there = id >= 0;  // an absent page's loads give zeros, and none of its keys counts
    const uint8_t* page = A.pool + ((int64_t)(there ? id : 0) * A.Hkv + W.kv) * kPage8Bytes;
#pragma unroll
    for (int l = 0; l < kLoads; ++l) {
      const int at = (w * kLoads + l) * 1024;  // the first half of them are keys: eight rows a load
      const int from = at < fc::kPage8V ? 16 * (lane ^ swap_of(at / kDim8 + (lane >> 3))) : 16 * lane;
      fc::lds_load16(lds0 + (uint32_t)(slot_of(pg) + at), (uint32_t)from, fc::buffer_rsrc(page + at, there ? 1024u : 0u));
    }
    return there;
  }
};

template <int NT, bool kLse>
__device__ __forceinline__ void group_page(const uint8_t* raw, uint32_t word, int left, Tile (&tile)[kWaveTiles]) {
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  const int key_row = 16 * (lc >> 2) + (lc & 3);
  const uint8_t* keys = raw + key_row * kDim8;
  const int places[2] = {16 * (lg ^ swap_of(key_row)), 16 * ((4 + lg) ^ swap_of(key_row))};
  floatx4 s[NT][kKTiles];
  page_scores<NT>([&](int t, int u) { return *(const uint4*)(keys + 4 * t * kDim8 + places[u]); }, tile, s);
  if (left < kPage8) cut<NT>(s, lg, left);
  bf16x2 p[NT][2 * kKTiles];
  weights<kLse, NT, kKTiles>(s, key_scale(word, lg, left) * score_scale(), tile, p);
  const float vs = value_scale(word, lg, left);
  const uint8_t* values = raw + fc::kPage8V + lg * 2048 + lc * 16;
  const auto value = [&](int t) { return *(const uint4*)(values + t * 256); };
  if (left >= kPage8) page_values<NT>(value, vs, p, tile);
  else page_values<NT>([&](int t) { return cut_values(value(t), lg, left); }, vs, p, tile);
}

// A part's pages, with NT tiles of this wave (0: it loads for the others alone).
template <int NT, bool kLse>
__device__ __forceinline__ void group_pages(Pages& pages, const uint8_t* lds, bool here0, bool here1, int word0, int word1,
                                            Tile (&tile)[kWaveTiles]) {
  const Work& W = pages.W;
  bool here2 = false;  // whether page pg, pg + 1, pg + 2 is
  int word2 = 0;
  for (int pg = W.pg0; pg < W.pg1; ++pg) {
    // this page is there: only the next may be on its way
    if (pg + 1 < W.pg1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(Pages::kLoads) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();  // for all; and the slot of the page before it is free
    if (pg + 2 < W.pg1) here2 = pages.issue(pg + 2, word2);
    const int left = here0 ? W.P - pg * kPage8 : 0;  // keys that exist, if below 64
    if constexpr (NT > 0) group_page<NT, kLse>(lds + pages.slot_of(pg), (uint32_t)word0, left, tile);
    here0 = here1, here1 = here2;
    word0 = word1, word1 = word2;
  }
}

// 64 tree rows on their way through a thread's registers to LDS: row 16 i + tid / 16,
// eight dims of its keys and values.
struct TreeRows {
  uint4 k[4], v[4];
  __device__ __forceinline__ void load(const Args& A, const Work& W, int j0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = j0 + 16 * i + (int)threadIdx.x / 16, c = 8 * ((int)threadIdx.x % 16);
      k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (r < W.n) {
        k[i] = *(const uint4*)(W.k_row(A, r) + c);
        v[i] = *(const uint4*)(W.v_row(A, r) + c);
      }
    }
  }
  __device__ __forceinline__ void store(uint8_t* keys, uint8_t* values, uint32_t* bad) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + (int)threadIdx.x / 16, c = 16 * ((int)threadIdx.x % 16);
      if (keep_finite(v[i])) atomicOr(&bad[r / 32], 1u << (r % 32));
      *(uint4*)(keys + r * kRowBytes + c) = k[i];
      *(uint4*)(values + r * kRowBytes + c) = v[i];
    }
  }
};

// 16 T tree rows from j0 on, which lie in LDS; `see`: which of them the lane's rows may.
template <int NT, int T, bool kLse>
__device__ __forceinline__ void group_tree(const Args& A, const Work& W, int j0, const uint32_t (&see)[kWaveTiles],
                                           const uint8_t* keys, uint8_t* values, uint64_t bad, Tile (&tile)[kWaveTiles]) {
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  floatx4 s[NT][T];
#pragma unroll
  for (int t = 0; t < T; ++t) {
#pragma unroll
    for (int i = 0; i < NT; ++i) s[i][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const bf16x8 k = *(const bf16x8*)(keys + (16 * t + lc) * kRowBytes + 128 * (u / 2) + 32 * lg + 16 * (u % 2));
#pragma unroll
      for (int i = 0; i < NT; ++i) s[i][t] = product(k, tile[i].q[u], s[i][t]);
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int t = 0; t < T; ++t) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[i][t]));
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int u = 0; u < 4 * T; ++u) s[i][u / 4][u % 4] = (see[i] >> u) & 1u ? s[i][u / 4][u % 4] : -INFINITY;
  bf16x2 p[NT][2 * T];
  weights<kLse, NT, T>(s, score_scale(), tile, p);
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_u8*)values;
  lds_u8* const at = (lds_u8*)(uintptr_t)(lds0 + (uint32_t)((4 * lg + (lc >> 2)) * kRowBytes + (lc & 3) * 8));
  tree_values<NT, T>(at, p, tile);
  if (bad) {
#pragma unroll
    for (int i = 0; i < NT; ++i) add_marked<T>(A, W, bad, j0, p[i], see[i], tile[i].row);
  }
}

// More tiles: a workgroup's waves share pages, four of them on their way through LDS, and
// have one or two tiles each.  Bound by what a wave does in turn - scores, weights, values
// - with two waves a SIMD, whose 256 registers are not enough: 42 more lie in scratch, 172
// bytes a lane, and come back in the loop over the tree's rows, each with a wait for all
// loads.  48 trees of 65 rows over up to 4,096 tokens, 32 heads on 8, 146 us (160 under a
// trace, where each launch begins on an idle card) where the products' rate allows 64; of
// 4,096 tokens each 388; without a prefix 71, as chains without a mask 52.
template <bool kLse>
__global__ void __launch_bounds__(kThreads, 2) k_paged8_attn(Args A) {
  static_assert(2 * kPage8 * kRowBytes <= kSlots * kSlot, "tree rows where the pages were");
  __shared__ __align__(16) uint8_t s_x[kSlots * kSlot];
  __shared__ uint32_t s_bad[2];
  const int tid = (int)threadIdx.x, lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid / fc::kWave);
  const Place place = place_of((int)blockIdx.x, A.B * A.Hkv, A.chunks);
  const int chunk = place.chunk;
  Work W;
  if (!W.init(A, place.pair, (int)blockIdx.y)) return;
  // a chunk's tiles, evenly; its waves have one or two, and which have two changes
  // from workgroup to workgroup, as a SIMD has one wave of each
  const int tile0 = (int)((int64_t)A.tiles * chunk / A.chunks), tile1 = (int)((int64_t)A.tiles * (chunk + 1) / A.chunks);
  const int turn = (w + 2 * (W.kv + chunk)) % kWaves;
  int row[kWaveTiles], mine = 0;
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) {
    const int t = tile0 + turn + kWaves * i;
    mine += t < tile1;
    row[i] = t < tile1 ? t * kTile + lc : W.M;
  }

  Pages pages(A, W, s_x, w);
  bool here0 = false, here1 = false;
  int word0 = 0, word1 = 0;
  if (W.pg0 < W.pg1) here0 = pages.issue(W.pg0, word0);
  if (W.pg0 + 1 < W.pg1) here1 = pages.issue(W.pg0 + 1, word1);

  Tile tile[kWaveTiles];
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) tile[i].load(W.q_row(A, row[i]), lg);
  // Queries are waited for here: in the loop below the compiler would wait for them in
  // every turn, and with them for the pages that are meant to stay on their way.
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i)
#pragma unroll
    for (int u = 0; u < 4; ++u) asm volatile("" : "+v"(tile[i].q[u]));

  if (mine == 2) group_pages<2, kLse>(pages, s_x, here0, here1, word0, word1, tile);
  else if (mine == 1) group_pages<1, kLse>(pages, s_x, here0, here1, word0, word1, tile);
  else group_pages<0, kLse>(pages, s_x, here0, here1, word0, word1, tile);

  if (W.tree) {
    // 64 of its rows at a time: what is read of them, and which of them each query row
    // may see, is asked for together, the next ones' before these are used
    uint8_t *const keys = s_x, *const values = s_x + kPage8 * kRowBytes;
    TreeRows rows;
    rows.load(A, W, 0);
    uint32_t see[kWaveTiles];
    __syncthreads();  // the last page is used
    for (int j0 = 0; j0 < W.n; j0 += kPage8) {
#pragma unroll
      for (int i = 0; i < kWaveTiles; ++i) {
        see[i] = W.allowed<kKTiles>(A, row[i], j0, lg);
      }
      if (tid < 2) s_bad[tid] = 0;
      __syncthreads();
      rows.store(keys, values, s_bad);
      __syncthreads();
      if (j0 + kPage8 < W.n) rows.load(A, W, j0 + kPage8);
      const uint64_t bad = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)s_bad[0]) |
                           (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)s_bad[1]) << 32;
      const bool few = W.n - j0 <= 32;  // a tree's 65th row
      if (mine == 2 && few) group_tree<2, 2, kLse>(A, W, j0, see, keys, values, bad, tile);
      else if (mine == 2) group_tree<2, kKTiles, kLse>(A, W, j0, see, keys, values, bad, tile);
      else if (mine == 1 && few) group_tree<1, 2, kLse>(A, W, j0, see, keys, values, bad, tile);
      else if (mine == 1) group_tree<1, kKTiles, kLse>(A, W, j0, see, keys, values, bad, tile);
      __syncthreads();
    }
  }
#pragma unroll
  for (int i = 0; i < kWaveTiles; ++i) {
    whole(tile[i].row);
    const float m = maximum_of(A, W, tile[i].row, tile[i].row.m(), row[i]);
    if (row[i] < W.M) finish(A, W, tile[i].row, m, row[i]);
  }
}

// The parts of a row put together: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s with m
// the largest m_s.  A wave per row: a lane has the weight of one or two parts, then
// each 16 lanes add up every fourth part, eight dims a lane.  A prefix in one part is
// in place already.
constexpr int kMergeWaves = 4;
__global__ void __launch_bounds__(kMergeWaves* fc::kWave) k_paged8_merge(Args A) {
  const int G = A.H / A.Hkv, M = A.R * G;
  const int lane = fc::lane_id();
  const int64_t at = (int64_t)blockIdx.x * kMergeWaves + (int)(threadIdx.x / fc::kWave);  // (tree, key head, row)
  if (at >= (int64_t)A.B * A.Hkv * M) return;
  const int64_t bk = at / M;
  const int r = (int)(at - bk * M), b = (int)(bk / A.Hkv), kv = (int)(bk - (int64_t)b * A.Hkv);
  const int P = clamp_len(A.prefix_len[b], A.max_len);
  const int n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
  const int parts = parts_of((P + kPage8 - 1) / kPage8, A.part_pages);
  if (parts == 1) return;
  const int64_t at0 = bk * A.parts * M + r;
  float4 ml[2];
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int s = lane + 64 * i;
    ml[i] = A.part_ml[at0 + (int64_t)(s < parts ? s : 0) * M];
    if (s >= parts) ml[i] = make_float4(-INFINITY, 0.0f, 0.0f, 0.0f);
    m = fmaxf(m, ml[i].x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  float w[2], l = 0.0f, x = 0.0f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    w[i] = ml[i].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml[i].x - m);  // 0: a part without a key
    l += w[i] * ml[i].y;
    x += w[i] * ml[i].z;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o), x += __shfl_xor(x, o);
  const int d = 8 * (lane & 15);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  for (int s0 = 0; s0 < parts; s0 += 16) {
    floatx4 lo[4], hi[4];
    float ww[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int s = s0 + 4 * u + (lane >> 4), i = s < parts ? s : parts - 1;
      const float* po = A.part_o + (at0 + (int64_t)i * M) * kDim8 + d;
      lo[u] = *(const floatx4*)po;
      hi[u] = *(const floatx4*)(po + 4);
      const float a = __shfl(w[0], i & 63), c = __shfl(w[1], i & 63);
      ww[u] = s < parts ? (i < 64 ? a : c) : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (s0 + 4 * u + (lane >> 4) >= parts) continue;  // nothing of it, not even a NaN
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[e] += ww[u] * lo[u][e];
        acc[4 + e] += ww[u] * hi[u][e];
      }
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    acc[e] += __shfl_xor(acc[e], 16);
    acc[e] += __shfl_xor(acc[e], 32);
  }
  if (lane >= 16) return;
  const int i = r / G;
  const int64_t to = ((int64_t)b * A.R + i) * A.H + kv * G + (r - i * G);
  const float inv = i < n ? inverse(m, l) : 0.0f;
  bf16x8 res;
#pragma unroll
  for (int e = 0; e < 8; ++e) res[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(acc[e] * inv);
  *(bf16x8*)(A.out + to * kDim8 + d) = res;
  if (A.lse && lane == 0) A.lse[to] = i < n ? log_sum(m, x) : -INFINITY;
}

struct Shape {
  int tiles, chunks, part_pages, parts;
  int alone;     // waves of a workgroup whose waves take pages alone; 0: they share them
  bool ordered;  // the longest prefixes first
};

// How a call is laid out: a workgroup for every eight tiles of query rows of a key
// head, parts of the pages where that leaves the chip idle (131,000 tokens, one query row:
// in 1 part 612 us, 8 91, 16 53, 32 48; a tree of 65 rows over 3,000 tokens: 83, 30, 33).
Shape shape_of(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  Shape s;
  s.tiles = (R * (H / Hkv) + kTile - 1) / kTile;
  s.chunks = s.tiles <= kWaveTiles ? 1 : (s.tiles + kGroupTiles - 1) / kGroupTiles;
  const int64_t wgs = (int64_t)B * Hkv * s.chunks;
  const int64_t pages = ((int64_t)max_len + kPage8 - 1) / kPage8;
  // Eight waves where prefixes are long or workgroups few, one workgroup to a CU (32 heads
  // on 8, single tokens: 64 sequences of up to 8,192 tokens 77 us, with four waves 107;
  // 128 of up to 1,000 tokens 42 with eight, 27 with four; 64 of up to 2,048 28 and 27).
  s.alone = s.tiles > kWaveTiles ? 0 : pages >= 64 || wgs <= kCus ? 8 : 4;
  const int64_t slots = s.alone == 8 ? kCus : 2 * kCus;  // workgroups at once
  int64_t each = s.alone ? s.alone : 4;
  // As many parts as fill the card once, below 64 pages rounded down, as beginning a part
  // and joining it cost as much as it takes over there, from 64 on up, so that the longest
  // of different lengths are cut (32 heads on 8, lengths from an eighth of the given one:
  // 20 trees of 65 rows over 1,000 tokens 50 us rounded down, 74 up, 20 over 2,048 87 and
  // 99; over 8,192 244 and 232, 14 over 8,192 208 and 168; 48 single tokens over 2,048 26
  // and 32, 25 over 8,192 54 and 55; all of one length, 20 trees over 8,192 297 and 319).
  int64_t parts = (slots + (pages < 64 ? 0 : wgs - 1)) / wgs;
  if (parts > kMostParts) parts = kMostParts;
  const int64_t fit = (pages + each - 1) / each;
  if (parts > fit) parts = fit;
  if (parts < 1) parts = 1;
  each = (pages + parts - 1) / parts;
  if (s.alone) each = (each + s.alone - 1) / s.alone * s.alone;
  s.part_pages = each < 1 ? 1 : (int)each;
  s.parts = pages <= s.part_pages ? 1 : (int)((pages + s.part_pages - 1) / s.part_pages);
  // Where not all workgroups run at once, a long one that began last would be waited
  // for alone (64 sequences of up to 8,192 tokens: 77 us, as they come 93; 48 trees of 65
  // rows over up to 4,096: 146 and 213; of equal lengths no difference).
  s.ordered = B > 1 && wgs * s.parts > slots;
  return s;
}

// Trees of a launch (and of the join after it).  Those behind them are a launch of
// their own, which uses the workspace again.
constexpr int64_t kMostGroups = 1 << 20;
int32_t trees_at_once(int32_t B, int32_t R, int32_t H, int32_t Hkv, const Shape& s) {
  const int64_t wgs = (int64_t)Hkv * s.chunks, joins = ((int64_t)H * R + kMergeWaves - 1) / kMergeWaves;
  const int64_t most = kMostGroups / (wgs > joins ? wgs : joins);
  return B < most ? B : most < 1 ? 1 : (int32_t)most;
}

size_t carve(void* p, int64_t rows, float4** ml, float** o) {
  fc::Carver c(p);
  *ml = c.take<float4>((size_t)rows);
  *o = c.take<float>((size_t)rows * kDim8);
  return c.used + 256;
}

bool sizes_ok(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  return B >= 0 && B <= 65536 && R >= 1 && R <= FC_MAX_TREE_ROWS && Hkv >= 1 && Hkv <= 1024 && H >= Hkv && H <= 8192 &&
         H % Hkv == 0 && max_len >= 0 && max_len <= 0x7FFFFFFF - kPage8;
}

template <int NT, bool kLse>
void launch_alone(const Args& a, const Shape& s, dim3 grid, hipStream_t stream) {
  if (s.alone == 8)
    hipLaunchKernelGGL((k_paged8_attn_alone<NT, 8, kLse>), grid, dim3(8 * fc::kWave), 0, stream, a);
  else
    hipLaunchKernelGGL((k_paged8_attn_alone<NT, 4, kLse>), grid, dim3(4 * fc::kWave), 0, stream, a);
}
template <bool kLse>
void launch(const Args& a, const Shape& s, hipStream_t stream) {
  const dim3 grid((uint32_t)a.B * (uint32_t)a.Hkv * (uint32_t)s.chunks, (uint32_t)s.parts);
  if (!s.alone) hipLaunchKernelGGL((k_paged8_attn<kLse>), grid, dim3(kThreads), 0, stream, a);
  else if (s.tiles == 1) launch_alone<1, kLse>(a, s, grid, stream);
  else launch_alone<2, kLse>(a, s, grid, stream);
}

}  // namespace

extern "C" size_t fc_paged_byte_attention_workspace_bytes(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  if (!sizes_ok(B, R, H, Hkv, max_len) || B == 0) return 0;
  const Shape s = shape_of(B, R, H, Hkv, max_len);
  float4* ml;
  float* o;
  return s.parts > 1 ? carve(nullptr, (int64_t)trees_at_once(B, R, H, Hkv, s) * H * R * s.parts, &ml, &o) : 0;
}

extern "C" fc_status fc_paged_byte_attention(const uint16_t* q, int64_t q_stride, const uint16_t* k_tree,
                                             int64_t k_stride, const uint16_t* v_tree, int64_t v_stride,
                                             const uint8_t* pool, int32_t n_pages, const int32_t* table,
                                             int32_t max_pages, const int32_t* prefix_len, const int32_t* num_nodes,
                                             const int32_t* mask, int32_t B, int32_t R, int32_t H, int32_t Hkv,
                                             int32_t D, int32_t max_len, uint16_t* out, float* lse, void* ws,
                                             size_t ws_bytes, hipStream_t stream) {
  if (!sizes_ok(B, R, H, Hkv, max_len) || n_pages < 1 || n_pages > (1 << 25) - 1 || max_pages < 1 ||
      (int64_t)max_len > (int64_t)max_pages * kPage8)
    return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (q_stride < (int64_t)H * D || k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D ||
      ((q_stride | k_stride | v_stride) & 7))
    return FC_ERR_INVALID;
  if (B == 0) return FC_OK;
  if (!q || !k_tree || !v_tree || !pool || !table || !prefix_len || !out) return FC_ERR_INVALID;
  if (((uintptr_t)q | (uintptr_t)k_tree | (uintptr_t)v_tree | (uintptr_t)pool | (uintptr_t)out) & 15)
    return FC_ERR_INVALID;
  if ((uintptr_t)lse & 3) return FC_ERR_INVALID;
  const Shape s = shape_of(B, R, H, Hkv, max_len);
  const int32_t at_once = trees_at_once(B, R, H, Hkv, s);
  float4* part_ml = nullptr;
  float* part_o = nullptr;
  const size_t need = fc_paged_byte_attention_workspace_bytes(B, R, H, Hkv, max_len);
  if (s.parts > 1) {
    if (!ws || ws_bytes < need) return FC_ERR_WORKSPACE;
    if ((uintptr_t)ws & 15) return FC_ERR_INVALID;
    carve(ws, (int64_t)at_once * H * R * s.parts, &part_ml, &part_o);
  }
  // A workgroup reads its query rows before it writes the same rows of the result, so
  // out may be q itself; what other workgroups read has to lie elsewhere.
  const int64_t all = (int64_t)B * R;
  const bool in_place = out == q && q_stride == (int64_t)H * D;
  if (!fc::apart({fc::rows_span(out, all, (int64_t)H * D, (int64_t)H * D),
                  {lse, 4 * (uint64_t)all * H},
                  {s.parts > 1 ? ws : nullptr, need}},
                 {fc::rows_span(in_place ? nullptr : q, all, q_stride, (int64_t)H * D),
                  fc::rows_span(k_tree, all, k_stride, (int64_t)Hkv * D),
                  fc::rows_span(v_tree, all, v_stride, (int64_t)Hkv * D),
                  {pool, fc_paged_byte_pool_bytes(n_pages, Hkv)},
                  {table, 4 * (uint64_t)B * max_pages},
                  {prefix_len, 4 * (uint64_t)B},
                  {num_nodes, 4 * (uint64_t)B},
                  {mask, 4 * (uint64_t)all * R}}))
    return FC_ERR_INVALID;
  (void)hipGetLastError();
  for (int32_t b = 0; b < B; b += at_once) {
    const int32_t now = B - b < at_once ? B - b : at_once;
    const int64_t row = (int64_t)b * R;
    const Args a = {q + row * q_stride, k_tree + row * k_stride, v_tree + row * v_stride, q_stride, k_stride, v_stride,
                    pool, table + (int64_t)b * max_pages, prefix_len + b, num_nodes ? num_nodes + b : nullptr,
                    mask ? mask + row * R : nullptr, n_pages, max_pages, now, R, H, Hkv, max_len, s.tiles, s.chunks,
                    s.part_pages, s.parts, s.ordered && now <= kOrdered, out + row * H * kDim8, lse ? lse + row * H : nullptr, part_ml, part_o};
    if (lse) launch<true>(a, s, stream);
    else launch<false>(a, s, stream);
    FC_CHECK_LAUNCH();
    if (s.parts > 1) {
      const uint64_t rows = (uint64_t)now * H * R;
      hipLaunchKernelGGL(k_paged8_merge, dim3(fc::div_up(rows, kMergeWaves)), dim3(kMergeWaves * fc::kWave), 0, stream, a);
      FC_CHECK_LAUNCH();
    }
  }
  return FC_OK;
}

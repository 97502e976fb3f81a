// Tree attention over the paged 4-bit cache on gfx950 matrix cores
// (fc_paged_attention).
//
// The rows of a tree that share a key head - its R rows times the H / Hkv query
// heads of the group - are one matrix of queries, cut into tiles of 16 rows.  A
// workgroup takes some of a (tree, key head)'s tiles and some of its pages; its
// waves are split over the tiles first and over the pages with what is left.
//
// Per page of 64 keys a wave computes the transposed scores S^T = K Q^T and
// O^T += V^T P^T, which keeps a lane's scores where the second product wants
// its weights.  The key codes go into the matrix cores as they lie in the page:
// a 16x16x128 product takes 4-bit keys with a scale for each 32 dims, which are
// the cache's own format, so no key is ever unpacked.  Its other operand has at
// most 6 bits at the full rate, so a query is the sum of three 6-bit parts, each
// with the scale of what the last one left over: three products of 16 cycles
// where bf16 would take four and the unpacking.  The value codes are unpacked to
// bf16 in LDS (their scales vary along the sum, which the matrix cores do not
// take) by the waves that share them, and read back transposed.
#include <hip/hip_runtime.h>
#include <stdint.h>

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
typedef int int32x6 __attribute__((ext_vector_type(6)));
typedef int int32x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kTile = 16;                       // query rows of a tile
constexpr int kParts = 3;                       // 6-bit parts of a query
constexpr int kDTiles = kHeadDim / 16;          // output tiles of 16 dims
constexpr int kRowBytes = kHeadDim * 2 + 32;    // a bf16 row in LDS
constexpr int kValues = kPage * kRowBytes;      // a page's values in LDS: 18 KB
constexpr int kTreeBlock = 32;                  // tree rows at a time: keys and values fill one such buffer
constexpr int kXcds = 8;
constexpr int kCus = 256;

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

// parts that a prefix is cut into: each takes part_pages pages
__device__ __forceinline__ int parts_of(int pages, int part_pages) {
  return pages <= part_pages ? 1 : (pages + part_pages - 1) / part_pages;
}

// Rows of a (tree, key head): row r is tree row r / G, head r % G of the group.
// A workgroup has WK groups of WR waves; a wave has NT tiles, wave w of a group
// tiles w, w + WR.
template <int NT, int WR, int WK>
__global__ void __launch_bounds__(WR* WK* fc::kWave, 2) k_paged_attn(Args A) {
  constexpr int kThreads = WR * WK * fc::kWave;
  constexpr int kBufs = WR > 1 ? 2 : 1;  // waves that share values write one page's while they read another's
  __shared__ __align__(16) uint8_t s_v[WK * kBufs * kValues];
  __shared__ double s_freq[kHeadDim / 2];
  __shared__ uint32_t s_bad[2][WK];  // tree rows of a block whose values are not all finite

  const int tid = (int)threadIdx.x, lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane(tid / fc::kWave);
  const int grp = w / WR, wr = w - grp * WR;
  const int lg = lane >> 4, lc = lane & 15;

  // consecutive workgroups of one XCD share a key head's pages in its L2
  const int total = (int)gridDim.x, x = (int)blockIdx.x;
  const int lin = total % kXcds == 0 ? (x % kXcds) * (total / kXcds) + x / kXcds : x;
  const int chunk = lin % A.chunks, bk = lin / A.chunks;
  const int b = bk / A.Hkv, kv = bk - b * A.Hkv;
  const int G = A.H / A.Hkv, M = A.R * G;
  const int tiles = (M + kTile - 1) / kTile;
  const int tile0 = (int)((int64_t)tiles * chunk / A.chunks), tile1 = (int)((int64_t)tiles * (chunk + 1) / A.chunks);

  const int P = clamp_len(A.prefix_len[b], A.max_len);
  const int n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
  const int pages = (P + kPage - 1) / kPage;
  const int parts = parts_of(pages, A.part_pages), part = (int)blockIdx.y;
  if (part >= parts) return;
  const int pg0 = part * A.part_pages;
  const int pg1 = parts == 1 ? pages : (pg0 + A.part_pages < pages ? pg0 + A.part_pages : pages);

  if (tid < 2 * WK) s_bad[tid / WK][tid % WK] = 0;
  if (A.log2_base > 0.0)
    for (int d = tid; d < kHeadDim / 2; d += kThreads) s_freq[d] = exp2(-2.0 * d / (double)kHeadDim * A.log2_base);
  __syncthreads();

  // this wave's rows: tile, row of the matrix, tree row
  int row[NT], tree_row[NT];
  bool in[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int t = tile0 + wr + WR * i;
    row[i] = t * kTile + lc;
    in[i] = t < tile1 && row[i] < M;
    tree_row[i] = in[i] ? row[i] / G : 0;
  }
  const auto q_row = [&](int i) {
    return A.q + ((int64_t)b * A.R + tree_row[i]) * A.q_stride + ((int64_t)kv * G + (row[i] - tree_row[i] * G)) * kHeadDim;
  };
  const auto position = [&](int r) { return P + (A.pos_ids ? A.pos_ids[(int64_t)b * A.R + r] : r); };
  // scores are in units of log2: softmax weights are powers of two
  const float scale = 1.44269504088896340736f / sqrtf((float)kHeadDim);

  // Queries as three 6-bit parts: lane (lg, lc) holds dims 32 lg .. 32 lg + 31
  // of row lc.  The first part's scale 2^e is the smallest with which the
  // largest magnitude is at most 7.5; it leaves at most 2^-2 * 2^e, the second
  // (scale 2^(e - 4)) at most 2^-7, the third (2^(e - 9)) at most 2^-12.
  int32x8 qf[NT][kParts];
  int qs[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    float v[32];
#pragma unroll
    for (int u = 0; u < 32; ++u) v[u] = 0.0f;
    if (in[i]) {
      const uint16_t* p = q_row(i);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float own[8];
        fc::unpack8(*(const uint4*)(p + 32 * lg + 8 * u), own);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * u + e] = own[e];
      }
      if (A.log2_base > 0.0) {
        const int pos = position(tree_row[i]);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float other[8];
          fc::unpack8(*(const uint4*)(p + ((32 * lg + 64) & 127) + 8 * u), other);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float s, c;
            fc::rope_sincos(pos, s_freq[(32 * lg & 63) + 8 * u + e], s, c);
            v[8 * u + e] = v[8 * u + e] * c + (lg < 2 ? -other[e] : other[e]) * s;
          }
        }
      }
    }
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < 32; ++u) {
      v[u] *= scale;
      const uint32_t bits = __float_as_uint(v[u]) & 0x7FFFFFFFu;
      top = bits > top ? bits : top;
    }
    int e = (int)((top + 0x0FFFFFu) >> 23) - 127 - 2;  // 7.5 = 1.875 * 2^2
    e = e < -110 ? -110 : e;
    floatx16 even, odd;
#pragma unroll
    for (int u = 0; u < 16; ++u) even[u] = v[2 * u], odd[u] = v[2 * u + 1];
    int word = 0;
#pragma unroll
    for (int s = 0; s < kParts; ++s) {
      const int es = e - (s == 0 ? 0 : s == 1 ? 4 : 9);
      const float f = __uint_as_float((uint32_t)(es + 127) << 23);
      const int32x6 c = to_six(even, odd, f);
#pragma unroll
      for (int u = 0; u < 6; ++u) qf[i][s][u] = c[u];
      qf[i][s][6] = qf[i][s][7] = 0;
      if (s + 1 < kParts) {
        const floatx32 r = from_six(c, f);
#pragma unroll
        for (int u = 0; u < 16; ++u) even[u] -= r[2 * u], odd[u] -= r[2 * u + 1];
      }
      word |= (top >= 0x7F800000u ? 255 : es + 127) << (8 * s);  // something not finite: NaN
    }
    qs[i] = word;
  }

  floatx4 o[NT][kDTiles];
  // a row's running maximum m, 0 - m (0 while there is none) four times, and by
  // how much a score may pass m before the row is scaled anew
  float m_run[NT], l_run[NT], slack[NT];
  floatx4 minus_m[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    m_run[i] = slack[i] = -INFINITY;
    l_run[i] = 0.0f;
    minus_m[i] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) o[i][t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // One step of the softmax.  s holds scores less m (the products start from
  // minus_m), -inf where a key is not allowed.  m is the maximum of what a row
  // saw when it was last scaled: while no score passes it by more than 8, weights
  // stay below 2^8 and neither sums nor outputs are touched (with bf16 weights a
  // common factor costs no accuracy), so the usual step is a power of two, a sum
  // and a rounding for each score.
  const auto softmax = [&](auto& s, auto& pb) {
    constexpr int KT = sizeof(s[0]) / sizeof(s[0][0]);
    bool up = false;
    float top[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      top[i] = -INFINITY;
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        top[i] = fmaxf(fmaxf(top[i], s[i][t][0]), s[i][t][1]);
        top[i] = fmaxf(fmaxf(top[i], s[i][t][2]), s[i][t][3]);
      }
      up |= top[i] > slack[i];
    }
    if (__any(up)) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        float mx = fmaxf(top[i], __shfl_xor(top[i], 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float was = 0.0f - minus_m[i][0];
        const float m_new = fmaxf(m_run[i], was + mx);
        const float by = m_new == -INFINITY ? 0.0f : m_new - was;
        const float alpha = m_run[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[i] - m_new);
#pragma unroll
        for (int t = 0; t < KT; ++t) s[i][t] -= by;
        l_run[i] *= alpha;
#pragma unroll
        for (int t = 0; t < kDTiles; ++t) o[i][t] *= alpha;
        m_run[i] = m_new;
        const float minus = m_new == -INFINITY ? 0.0f : -m_new;
        minus_m[i] = floatx4{minus, minus, minus, minus};
        slack[i] = m_new == -INFINITY ? -INFINITY : 8.0f;
      }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
#pragma unroll
      for (int t = 0; t < KT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f(s[i][t][e]);
          l_run[i] += p;
          pb[t / 2][i][4 * (t % 2) + e] = (__bf16)p;
        }
    }
  };
  // O^T += V^T P^T over 32 keys at byte `base` of the buffers: a transposing read
  // gives lane (lg, lc) dims 16 t + lc of keys 4 lg + e, the second one keys 16 +
  // 4 lg + e, as the weights lie
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)s_v;
  const uint32_t v_lane = lds0 + chunk_at(4 * lg + (lc >> 2), 0) + (uint32_t)(lc & 3) * 8u;
  const auto values = [&](uint32_t base, const bf16x8 (&pb)[NT]) {
    typedef __attribute__((address_space(3))) uint8_t lds_u8;
    lds_u8* at = (lds_u8*)(uintptr_t)(v_lane + base);
#pragma unroll
    for (int t = 0; t < kDTiles; ++t) {
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + chunk_at(0, 2 * t)));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(at + chunk_at(16, 2 * t)));
      const bf16x8 a = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
#pragma unroll
      for (int i = 0; i < NT; ++i) o[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[i], o[i][t], 0, 0, 0);
    }
  };

  // a page on its way: every wave of a group loads the key codes it multiplies,
  // and its share of the value codes (16 bytes a lane: 32 dims of a key)
  constexpr int kVUnits = (4 + WR - 1) / WR;
  uint4 kf[4], vf[kVUnits];
  uint32_t ks, vs;
  bool have;
  const int32_t* table = A.table + (int64_t)b * A.max_pages;
  const auto load = [&](int pg) {
    const int id = pg < pg1 ? __builtin_amdgcn_readfirstlane(table[pg]) : -1;
    have = id >= 0 && id < A.n_pages;
    if (!have) return;
    const uint8_t* page = A.pool + ((int64_t)id * A.Hkv + kv) * kPageBytes;
#pragma unroll
    for (int t = 0; t < 4; ++t) kf[t] = *(const uint4*)(page + (16 * t + lc) * fc::kCodeRow + 16 * lg);
    ks = *(const uint32_t*)(page + fc::kPageKScale + 4 * lane);
#pragma unroll
    for (int u = 0; u < kVUnits; ++u)
      if (wr + WR * u < 4) vf[u] = *(const uint4*)(page + fc::kPageV + ((wr + WR * u) * 64 + lane) * 16);
    vs = *(const uint32_t*)(page + fc::kPageVScale + 4 * lane);
  };
  const int steps = (pg1 - pg0 + WK - 1) / WK;
  load(pg0 + grp);
  for (int it = 0; it < steps; ++it) {
    const int pg = pg0 + it * WK + grp;
    const int left = P - pg * kPage;  // keys of this page that exist, if below 64
    const uint32_t buf = (uint32_t)(grp * kBufs + (kBufs > 1 ? it % kBufs : 0)) * kValues;
    const bool use = have;
    if (use) {
      // values to bf16; a key past the prefix has weight 0, and so that
      // whatever its bytes hold does not matter its values are 0 too
#pragma unroll
      for (int u = 0; u < kVUnits; ++u) {
        const int i4 = wr + WR * u;
        if (i4 < 4) {
          const int key = i4 * 16 + (lane >> 2), g = lane & 3;
          uint32_t sb = (vs >> (8 * i4)) & 255u;
          uint32_t c4[4] = {vf[u].x, vf[u].y, vf[u].z, vf[u].w};
          if (left < kPage) {
            const bool live = key < left;
            sb = live ? sb : 127u;
#pragma unroll
            for (int c = 0; c < 4; ++c) c4[c] = live ? c4[c] : 0u;
          }
          const float sc = fc::scale_of(sb);
          uint8_t* dst = s_v + buf + chunk_at(key, 4 * g);
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
      }
    }
    if (WR > 1) __syncthreads();
    floatx4 s[NT][4];
    if (use) {
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const int32x8 a = {(int)kf[t].x, (int)kf[t].y, (int)kf[t].z, (int)kf[t].w, 0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          floatx4 acc = minus_m[i];
          // the scale operands' byte selectors are immediates
#define FC_PART(S, T) acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, qf[i][S], acc, 4, 2, T, (int)ks, S, qs[i])
          if (t == 0) { FC_PART(0, 0); FC_PART(1, 0); FC_PART(2, 0); }
          if (t == 1) { FC_PART(0, 1); FC_PART(1, 1); FC_PART(2, 1); }
          if (t == 2) { FC_PART(0, 2); FC_PART(1, 2); FC_PART(2, 2); }
          if (t == 3) { FC_PART(0, 3); FC_PART(1, 3); FC_PART(2, 3); }
#undef FC_PART
          s[i][t] = acc;
        }
      }
    }
    load(pg + WK);
    if (use) {
      bf16x8 pb[2][NT];
      if (left < kPage) {
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[i][t][e] = 16 * t + 4 * lg + e < left ? s[i][t][e] : -INFINITY;
      }
      softmax(s, pb);
      values(buf, pb[0]);
      values(buf + chunk_at(32, 0), pb[1]);
    }
  }

  // the tree's own rows, in bf16, 32 at a time
  if (part == parts - 1 && n > 0) {
    bf16x8 qb[NT][4], ql[NT][4];  // rounded, and what that left over: only the key's rounding remains
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float v[4][8];
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[c][e] = 0.0f;
      if (in[i]) {
        const uint16_t* p = q_row(i);
#pragma unroll
        for (int c = 0; c < 4; ++c) fc::unpack8(*(const uint4*)(p + 32 * c + 8 * lg), v[c]);
        if (A.log2_base > 0.0) {
          const int pos = position(tree_row[i]);
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float sn, cs;
              fc::rope_sincos(pos, s_freq[32 * c + 8 * lg + e], sn, cs);
              const float x0 = v[c][e], x1 = v[c + 2][e];
              v[c][e] = x0 * cs - x1 * sn;
              v[c + 2][e] = x1 * cs + x0 * sn;
            }
        }
      }
#pragma unroll
      for (int c = 0; c < 4; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = v[c][e] * scale;
          qb[i][c][e] = (__bf16)x;
          ql[i][c][e] = (__bf16)(x - (float)qb[i][c][e]);
        }
    }
    const int blocks = (n + kTreeBlock - 1) / kTreeBlock;
    uint8_t* sk = s_v + grp * kBufs * kValues;
    uint8_t* sv = sk + kTreeBlock * kRowBytes;
    for (int it = 0; it < (blocks + WK - 1) / WK; ++it) {
      const int j0 = (it * WK + grp) * kTreeBlock;
      __syncthreads();  // what was in the buffer has been read
      for (int u = wr * fc::kWave + lane; u < kTreeBlock * 8; u += WR * fc::kWave) {
        const int r = u / 8, c = u % 8, j = j0 + r;  // chunks c and c + 8 hold the pairs of a rotation
        bf16x8 ka, kb;
        uint4 v0 = make_uint4(0u, 0u, 0u, 0u), v1 = v0;
        float x0[8], x1[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x0[e] = x1[e] = 0.0f;
        if (j < n) {
          const uint16_t* kp = A.k_tree + ((int64_t)b * A.R + j) * A.k_stride + (int64_t)kv * kHeadDim + 8 * c;
          const uint16_t* vp = A.v_tree + ((int64_t)b * A.R + j) * A.v_stride + (int64_t)kv * kHeadDim + 8 * c;
          fc::unpack8(*(const uint4*)kp, x0);
          fc::unpack8(*(const uint4*)(kp + kHeadDim / 2), x1);
          v0 = *(const uint4*)vp;
          v1 = *(const uint4*)(vp + kHeadDim / 2);
          const bool bad0 = keep_finite(v0), bad1 = keep_finite(v1);
          if (bad0 || bad1) atomicOr(&s_bad[it & 1][grp], 1u << r);
          if (A.log2_base > 0.0) {
            const int pos = position(j);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              float sn, cs;
              fc::rope_sincos(pos, s_freq[8 * c + e], sn, cs);
              const float a0 = x0[e], a1 = x1[e];
              x0[e] = a0 * cs - a1 * sn;
              x1[e] = a1 * cs + a0 * sn;
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) ka[e] = (__bf16)x0[e], kb[e] = (__bf16)x1[e];
        *(bf16x8*)(sk + chunk_at(r, c)) = ka;
        *(bf16x8*)(sk + chunk_at(r, c + 8)) = kb;
        *(uint4*)(sv + chunk_at(r, c)) = v0;
        *(uint4*)(sv + chunk_at(r, c + 8)) = v1;
      }
      __syncthreads();
      if (j0 < n) {
        floatx4 s[NT][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int i = 0; i < NT; ++i) s[i][t] = minus_m[i];
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            const bf16x8 a = *(const bf16x8*)(sk + chunk_at(16 * t + lc, 4 * c + lg));
#pragma unroll
            for (int i = 0; i < NT; ++i) {
              s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, ql[i][c], s[i][t], 0, 0, 0);
              s[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qb[i][c], s[i][t], 0, 0, 0);
            }
          }
        }
        bf16x8 pb[1][NT];
        uint32_t allowed[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          // bit 4 t + e: this lane's e-th key of tile t is allowed
          uint32_t allow = 0;
          if (in[i]) {
            const int32_t* mrow = A.mask ? A.mask + ((int64_t)b * A.R + tree_row[i]) * A.R : nullptr;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
              const int j = j0 + 16 * (u / 4) + 4 * lg + u % 4;
              if (j < n && (mrow ? mrow[j] == 1 : j <= tree_row[i])) allow |= 1u << u;
            }
          }
#pragma unroll
          for (int u = 0; u < 8; ++u) s[i][u / 4][u % 4] = (allow >> u) & 1u ? s[i][u / 4][u % 4] : -INFINITY;
          allowed[i] = allow;
        }
        softmax(s, pb);
        values((uint32_t)(grp * kBufs * kValues + kTreeBlock * kRowBytes), pb[0]);
        // A product with weight 0 is NaN where the value is not finite, so the
        // rows that do not see such a value must not meet it: it is 0 in LDS, and
        // the rows that do see it add it here.
        for (uint32_t bad = __builtin_amdgcn_readfirstlane(s_bad[it & 1][grp]); bad; bad &= bad - 1) {
          const int r = __builtin_ctz(bad);
          const int u = r / 16 * 4 + r % 4, from = r % 16 / 4 * 16 + lc;  // whose weights for key r these are
          const uint16_t* vp = A.v_tree + ((int64_t)b * A.R + j0 + r) * A.v_stride + (int64_t)kv * kHeadDim + 4 * lg;
#pragma unroll
          for (int i = 0; i < NT; ++i) {
            float weight = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if (e == u) weight = (float)pb[0][i][e];
            weight = __shfl(weight, from);
            const bool sees = (__shfl(allowed[i], from) >> u) & 1u;
#pragma unroll
            for (int t = 0; t < kDTiles; ++t)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const uint32_t bits = (uint32_t)vp[16 * t + e] << 16;
                if (sees && (bits & 0x7F800000u) == 0x7F800000u) o[i][t][e] += weight * __uint_as_float(bits);
              }
          }
        }
      }
      if (wr == 0 && lane == 0) s_bad[(it & 1) ^ 1][grp] = 0;  // of the block before, whose readers are past the barrier
    }
  }

  // the row's whole weight
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    l_run[i] += __shfl_xor(l_run[i], 16);
    l_run[i] += __shfl_xor(l_run[i], 32);
  }

  // groups that took other pages hand over to group 0, through LDS
  if constexpr (WK > 1) {
    constexpr int kRec = kTile * kHeadDim + 2 * kTile;  // floats of a tile: outputs, maxima, weights
    static_assert((WK - 1) * WR * NT * kRec * 4 <= WK * kBufs * kValues, "hand-over fits the value buffers");
    float* rec = (float*)s_v;
    __syncthreads();
    if (grp > 0) {
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        float* r = rec + (((grp - 1) * WR + wr) * NT + i) * kRec;
#pragma unroll
        for (int t = 0; t < kDTiles; ++t) *(floatx4*)(r + (t * 64 + lane) * 4) = o[i][t];
        if (lg == 0) r[kTile * kHeadDim + lc] = m_run[i], r[kTile * kHeadDim + kTile + lc] = l_run[i];
      }
    }
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int g = 1; g < WK; ++g)
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const float* r = rec + (((g - 1) * WR + wr) * NT + i) * kRec;
        const float m2 = r[kTile * kHeadDim + lc], l2 = r[kTile * kHeadDim + kTile + lc];
        const float m = fmaxf(m_run[i], m2);
        const float a1 = m_run[i] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m_run[i] - m);
        const float a2 = m2 == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(m2 - m);
        m_run[i] = m;
        l_run[i] = l_run[i] * a1 + l2 * a2;
#pragma unroll
        for (int t = 0; t < kDTiles; ++t) o[i][t] = o[i][t] * a1 + *(const floatx4*)(r + (t * 64 + lane) * 4) * a2;
      }
  }

#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if (!in[i]) continue;
    if (parts > 1) {
      const int64_t at = ((int64_t)bk * A.parts + part) * M + row[i];
      if (lg == 0) A.part_ml[at] = make_float2(m_run[i], l_run[i]);
#pragma unroll
      for (int t = 0; t < kDTiles; ++t) *(floatx4*)(A.part_o + at * kHeadDim + 16 * t + 4 * lg) = o[i][t];
    } else {
      // a row without a key has weight 0; a NaN stays one
      const float inv = tree_row[i] < n && l_run[i] != 0.0f ? 1.0f / l_run[i] : 0.0f;
      uint16_t* dst = A.out + (((int64_t)b * A.R + tree_row[i]) * A.H + kv * G + (row[i] - tree_row[i] * G)) * kHeadDim;
#pragma unroll
      for (int t = 0; t < kDTiles; ++t) {
        bf16x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(o[i][t][e] * inv);
        *(bf16x4*)(dst + 16 * t + 4 * lg) = r;
      }
    }
  }
}

// The parts of a row put together: sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m)
// l_s with m the largest m_s.  16 lanes per row, eight dims each.  A prefix in
// one part is in place already.
__global__ void __launch_bounds__(256) k_paged_merge(Args A) {
  const int G = A.H / A.Hkv, M = A.R * G;
  const int blocks = (M + 15) / 16, bk = (int)blockIdx.x / blocks, b = bk / A.Hkv, kv = bk - b * A.Hkv;
  const int r = ((int)blockIdx.x - bk * blocks) * 16 + (int)(threadIdx.x / 16), d = 8 * (int)(threadIdx.x % 16);
  if (r >= M) return;
  const int P = clamp_len(A.prefix_len[b], A.max_len);
  const int parts = parts_of((P + kPage - 1) / kPage, A.part_pages);
  if (parts == 1) return;
  const int n = A.num_nodes ? clamp_len(A.num_nodes[b], A.R) : A.R;
  const int64_t at = (int64_t)bk * A.parts * M + r;
  float m = -INFINITY, l = 0.0f;
  for (int s = 0; s < parts; ++s) m = fmaxf(m, A.part_ml[at + (int64_t)s * M].x);
  float acc[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) acc[e] = 0.0f;
  for (int s = 0; s < parts; ++s) {
    const float2 ml = A.part_ml[at + (int64_t)s * M];
    const float* po = A.part_o + (at + (int64_t)s * M) * kHeadDim + d;
    const float w = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - m);
    l += w * ml.y;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += w * po[e];
  }
  const int i = r / G;
  const float inv = i < n && l != 0.0f ? 1.0f / l : 0.0f;
  bf16x8 res;
#pragma unroll
  for (int e = 0; e < 8; ++e) res[e] = inv == 0.0f ? (__bf16)0.0f : (__bf16)(acc[e] * inv);
  *(bf16x8*)(A.out + (((int64_t)b * A.R + i) * A.H + kv * G + (r - i * G)) * kHeadDim + d) = res;
}

struct Shape {
  int nt, wr, wk, chunks, part_pages, parts;
};

// How a call is laid out.  Up to 128 query rows of a key head stay in one
// workgroup, which then reads its pages once; waves that the rows do not need
// are split over the pages.
Shape shape_of(int32_t B, int32_t R, int32_t H, int32_t Hkv, int32_t max_len) {
  const int tiles = (R * (H / Hkv) + kTile - 1) / kTile;
  const int chunks = (tiles + 7) / 8, most = (tiles + chunks - 1) / chunks;  // tiles of the largest chunk
  Shape s;
  s.chunks = chunks;
  s.nt = most > 1 ? 2 : 1;
  s.wr = (most + 1) / 2;
  s.wk = s.wr == 1 ? 4 : s.wr == 2 ? 2 : 1;
  const int64_t wgs = (int64_t)B * Hkv * chunks;
  const int64_t pages = ((int64_t)max_len + kPage - 1) / kPage;
  int64_t parts = (2 * kCus + wgs - 1) / wgs;
  const int64_t fit = (pages + 2 * s.wk - 1) / (2 * s.wk);  // two pages or more a wave
  if (parts > fit) parts = fit;
  if (parts > 64) parts = 64;
  if (parts < 1) parts = 1;
  int64_t each = (pages + parts - 1) / parts;
  each = (each + s.wk - 1) / s.wk * s.wk;
  s.part_pages = each < 1 ? 1 : (int)each;
  s.parts = pages <= s.part_pages ? 1 : (int)((pages + s.part_pages - 1) / s.part_pages);
  return s;
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
  return s.parts > 1 ? carve(nullptr, (int64_t)B * Hkv * s.parts * R * (H / Hkv), &ml, &o) : 0;
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
  // workgroups are numbered with 31 bits
  if ((int64_t)B * Hkv * (((int64_t)R * (H / Hkv) + kTile - 1) / kTile) > 0x7FFFFFFF) return FC_ERR_UNSUPPORTED;
  const Shape s = shape_of(B, R, H, Hkv, max_len);
  Args a = {q, k_tree, v_tree, q_stride, k_stride, v_stride, pool, table, prefix_len, num_nodes, mask, pos_ids,
            n_pages, max_pages, B, R, H, Hkv, max_len, s.chunks, s.part_pages, s.parts,
            rope_base != 0.0f ? log2((double)rope_base) : 0.0, out, nullptr, nullptr};
  if (s.parts > 1) {
    if (!ws || ws_bytes < fc_paged_attention_workspace_bytes(B, R, H, Hkv, max_len)) return FC_ERR_WORKSPACE;
    if ((uintptr_t)ws & 15) return FC_ERR_INVALID;
    carve(ws, (int64_t)B * Hkv * s.parts * R * (H / Hkv), &a.part_ml, &a.part_o);
  }
  const dim3 grid((uint32_t)B * (uint32_t)Hkv * (uint32_t)s.chunks, (uint32_t)s.parts);
  (void)hipGetLastError();
#define FC_ATTN(NT, WR, WK) \
  hipLaunchKernelGGL((k_paged_attn<NT, WR, WK>), grid, dim3(WR * WK * fc::kWave), 0, stream, a)
  if (s.nt == 1) FC_ATTN(1, 1, 4);
  else if (s.wr == 1) FC_ATTN(2, 1, 4);
  else if (s.wr == 2) FC_ATTN(2, 2, 2);
  else if (s.wr == 3) FC_ATTN(2, 3, 1);
  else FC_ATTN(2, 4, 1);
#undef FC_ATTN
  FC_CHECK_LAUNCH();
  if (s.parts > 1) {
    hipLaunchKernelGGL(k_paged_merge, dim3(fc::div_up((uint64_t)R * (H / Hkv), 16) * (uint32_t)B * (uint32_t)Hkv),
                       dim3(256), 0, stream, a);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

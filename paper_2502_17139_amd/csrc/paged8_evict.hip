// What cached tokens are worth on gfx950: the attention that they get
// (fc_paged_byte_weights), and the eviction of those that got least (fc_paged_byte_evict).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fastcoder.h"
#include "fc_device.h"
#include "fc_host.h"
#include "fc_page8.h"

namespace {

typedef __attribute__((address_space(3))) uint8_t lds_u8;

using fc::kBlock8;
using fc::kDim8;
using fc::kPage8;
using fc::kPage8Bytes;

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int clamp_len(int len, int most) { return len < 0 ? 0 : (len > most ? most : len); }

// ---------------------------------------------------------------- weights --

constexpr int kTile = 16;
constexpr int kWaves = 4;
constexpr int kThreads = kWaves * fc::kWave;
constexpr int kKTiles = kPage8 / 16;
constexpr float kLog2e = 1.44269504088896340736f;

struct Weights {
  float* weights;
  const uint16_t* q;
  int64_t q_stride;
  const float* lse;
  const uint8_t* pool;
  const int32_t *table, *len, *new_len, *cu, *src;
  int n_rows, n_pages, max_pages, n, H, Hkv, max_len;
  int y0;  // parts before this launch's
};

__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b) {
  const bf16x2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
  const bf16x2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
  return bf16x8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// 16 values a lane to their sums over the 16 lanes of a row: lane lc gets the sum of
// value lc.  Lanes that differ in one bit (and in all below it, as the row's mirrors
// have them) exchange the halves that the other keeps.
template <int HALF, int CTRL>
__device__ __forceinline__ void fold(float (&v)[16], int lc) {
  const bool up = lc & HALF;
#pragma unroll
  for (int i = 0; i < HALF; ++i) {
    const float keep = up ? v[HALF + i] : v[i], send = up ? v[i] : v[HALF + i];
    v[i] = keep + __uint_as_float(fc::dpp_mov<CTRL>(__float_as_uint(send)));
  }
}
__device__ __forceinline__ float sum_of_own(float (&v)[16], int lc) {
  fold<8, 0x140>(v, lc);  // row_mirror
  fold<4, 0x141>(v, lc);  // row_half_mirror
  fold<2, 0x1B>(v, lc);   // quad_perm 3 2 1 0
  fold<1, 0xB1>(v, lc);   // quad_perm 1 0 3 2
  return v[0];
}

// What a wave knows of its sequence and head.
struct Step {
  int len, end, G, kv, cu, n;  // n: new tokens, each with the group's G query heads as rows
  float inv;                   // 1 / G
  __device__ __forceinline__ Step(const Weights& A, int b, int kv_) {
    kv = kv_, G = A.H / A.Hkv;
    len = clamp_len(A.len[b], A.max_len), end = clamp_len(A.new_len[b], A.max_len);
    cu = A.cu[b], n = end - len;
    inv = 1.0f / (float)G;
  }
};
// A place among a sequence's rows: a token and a head of its group, to go on from.
struct Cursor {
  int t, h;
  __device__ __forceinline__ Cursor(const Step& S, int64_t row) : t((int)(row / S.G)), h((int)(row % S.G)) {}
  __device__ __forceinline__ void operator+=(const Cursor& d) { t += d.t, h += d.h; }
  __device__ __forceinline__ void carry(const Step& S) {
    if (h >= S.G) h -= S.G, ++t;
  }
  // The row `on` (below 2^13) rows further: quotients of such numbers are exact in fp32.
  __device__ __forceinline__ void at(const Step& S, int on, int& token, int& head) const {
    const int x = h + on, q = (int)(((float)x + 0.5f) * S.inv);
    token = t + q, head = x - q * S.G;
  }
};
// New token t's row among the call's: what src says, whatever that is, so that nobody
// waits for it before it is used.  A token or a place that is not there has none.
template <bool kSrc>
__device__ __forceinline__ int number_of(const Weights& A, const Step& S, int t) {
  const int64_t at = (int64_t)S.cu + t;
  const bool there = t < S.n && at >= 0 && at < A.n;
  const int row = kSrc ? A.src[there ? at : 0] : (int)at;
  return there ? row : -1;
}
// 16 rows of queries: lane (lg, lc) has dims 64 u + 16 lg + 8 h .. + 7 of row lc in
// q[2 u + h], as 16 key codes lie.
struct Rows {
  bf16x8 q[4];
  float lse;
  int last;  // the last key that the row sees; -1: there is no such row
  __device__ __forceinline__ void load(const Weights& A, const Step& S, int token, int head, int number) {
    const bool there = number >= 0 && number < A.n_rows;
    const int row = there ? number : 0;
    const int64_t h = S.kv * S.G + head;
    const uint16_t* p = A.q + row * A.q_stride + h * kDim8 + 16 * (fc::lane_id() >> 4);
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = *(const bf16x8*)(p + 64 * (u / 2) + 8 * (u % 2));
    lse = A.lse[(int64_t)row * A.H + h];
    last = there ? S.len + token : -1;
  }
};
// What 16 rows pay to a lane's 4 T keys, on top of `got`.  keys(t, u): the u-th quarter
// of the dims of key tile t, whose row 4 a + b is key 4 T a + 4 t + b.  minus: the row's
// logarithm, base 2, turned around; seen: the last of the lane's keys that the row sees.
template <int T, typename Keys>
__device__ __forceinline__ void pay(Keys keys, const bf16x8 (&q)[4], float scale, float minus, int seen, float (&got)[4 * T]) {
  floatx4 s[T];
#pragma unroll
  for (int t = 0; t < T; ++t) s[t] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int u = 0; u < 4; ++u)  // no product waits for the one before
#pragma unroll
    for (int t = 0; t < T; ++t) s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(keys(t, u), q[u], s[t], 0, 0, 0);
  // a product's result is read only some cycles after it was issued
  static_assert(T == 4 || T == 2, "the wait below");
  if constexpr (T == 4) asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1]), "+v"(s[2]), "+v"(s[3]));
  else asm volatile("s_nop 7\n\ts_nop 3" : "+v"(s[0]), "+v"(s[1]));
  const auto add = [&](bool all) {
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][e], scale, minus));
        got[4 * t + e] += all || 4 * t + e <= seen ? p : 0.0f;
      }
  };
  if (T == 2 && fc::ballot(seen < 4 * T - 1) == 0) add(true);
  else add(false);
}
__device__ __forceinline__ float key_scale(uint32_t byte) {
  return fc::scale8(byte) * (kLog2e / sqrtf((float)kDim8));
}
// A token's sum into its place: new tokens' weights become it.
__device__ __forceinline__ void settle_weight(const Weights& A, const Step& S, int id, int j, float sum, bool again) {
  float* to = A.weights + ((int64_t)id * A.Hkv + S.kv) * kPage8 + j % kPage8;
  if (j < S.end) *to = j < S.len || again ? *to + sum : sum;
}

// One wave loads 64 x 16 (or 64 x 4) bytes into LDS, lane L's behind lane L - 1's.
// Counted by vmcnt like any load; the compiler does not know of it.
__device__ __forceinline__ void to_lds16(uint32_t lds, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(from)
               : "memory");
}
__device__ __forceinline__ void to_lds4(uint32_t lds, const void* from) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(__builtin_amdgcn_readfirstlane((int)lds)), "v"(from)
               : "memory");
}

// Many rows (prompts): a workgroup's waves hold half a page's keys as bf16 and go through
// the sequence's rows, every eighth 16 of them each; the waves' sums are joined.  Nothing
// is added by two workgroups, so sums have one order.  Rows come through LDS, whole ones
// at a time: as a product takes them, 16 lanes would ask for 16 lines at once, and a CU
// gets one in a cycle (2,011 tokens, 32 heads on 8: 86 us like that, 46 so).  Whole pages
// with rows as a product takes them were 72, the first page's CU twice as long at work as
// the average.  Nothing is full now: vector unit busy 39 % of the time, matrix unit 14 %, LDS
// 27 %, and 9 us pass before the first product.
constexpr int kManyWaves = 8, kManyTiles = 2, kHalf = 16 * kManyTiles;
constexpr int kRing = 2, kRoundTiles = 4;  // tiles on their way, tiles whose rows lanes look after
constexpr int kTileBytes = kTile * kDim8 * 2;
constexpr int kCus = 256, kXcds = 8;
struct ManyShared {
  alignas(16) uint8_t rows[kManyWaves][kRing][kTileBytes];
  float lse[kManyWaves][fc::kWave];
  int number[kManyWaves][fc::kWave];
  float sum[kManyWaves - 1][fc::kWave];
};
template <bool kSrc>
__global__ void __launch_bounds__(kManyWaves* fc::kWave, 4) k_weights_many(Weights A, int pairs, int pieces) {
  constexpr int T = kManyTiles;
  __shared__ ManyShared sh;
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave);
  // A sequence's and head's workgroups follow one another, on one XCD if heads can be
  // dealt out like that: its L2 has the rows then.  The first keys are seen by most rows:
  // every other card full goes backwards, so that a CU which gets one workgroup of each
  // has no more to do than the others.
  const bool dealt = pairs % kXcds == 0;
  const int full = dealt ? kCus / kXcds : kCus, all = dealt ? pairs / kXcds * pieces : pairs * pieces;
  int at_pair = dealt ? (int)blockIdx.x % kXcds : 0, k = dealt ? (int)blockIdx.x / kXcds : (int)blockIdx.x;
  const int k0 = k / full * full;
  if (k / full % 2) k = k0 + (all - k0 < full ? all - k0 : full) - 1 - (k - k0);
  at_pair += k / pieces * (dealt ? kXcds : 1);
  const int piece = k % pieces, b = at_pair / A.Hkv, key0 = piece * kHalf;
  const Step S(A, b, at_pair % A.Hkv);
  if (S.n <= 0 || key0 >= S.end) return;  // all waves of the workgroup
  // rows that come before the first key see nothing
  const int64_t skip = (int64_t)key0 - S.len;
  const int64_t tiles = ((int64_t)S.n * S.G + kTile - 1) / kTile;
  int64_t tile = (skip > 0 ? skip * S.G / kTile : 0) + w;
  static_assert(kRoundTiles * kTile == fc::kWave, "a lane for each of a wave's rows");
  const Cursor round(S, kManyWaves * kRoundTiles * kTile);
  Cursor at(S, tile * kTile);
  // Each lane looks after one of a round's rows: its number is asked for first, from that
  // follow its place and its logarithm.
  const uint32_t lds_rows = (uint32_t)(uintptr_t)(lds_u8*)sh.rows[w], lds_lse = (uint32_t)(uintptr_t)(lds_u8*)sh.lse[w],
                 lds_number = (uint32_t)(uintptr_t)(lds_u8*)sh.number[w];
  int token, head, number;  // of the row after the one looked at
  bool there;
  const auto ask = [&] {
    at.at(S, kManyWaves * kTile * lg + lc, token, head);
    const int64_t i = (int64_t)S.cu + token;
    there = token < S.n && i >= 0 && i < A.n, number = (int)i;
    if (kSrc) to_lds4(lds_number, A.src + (there ? i : 0));
    at += round;
    at.carry(S);
  };
  int64_t place;
  int last;  // the last key that the row sees; -1: there is no such row
  const auto look = [&] {
    if (kSrc) number = sh.number[w][lane];
    const bool is = there && number >= 0 && number < A.n_rows;
    const int row = is ? number : 0, h = S.kv * S.G + head;
    place = row * A.q_stride + (int64_t)h * kDim8;
    last = is ? S.len + token : -1;
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(last) : : "memory");  // the number is read
    to_lds4(lds_lse, A.lse + (int64_t)row * A.H + h);
  };
  // Four rows at a time, 16 lanes each; a row's r-th 16 bytes lie at r ^ row, so that 16
  // rows' are read from all banks at once.
  const auto load = [&](int i) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int r = 4 * u + lg;
      const int64_t from = (int64_t)(uint32_t)__shfl((int)(uint32_t)place, kTile * i + r) |
                           (int64_t)__shfl((int)(place >> 32), kTile * i + r) << 32;
      to_lds16(lds_rows + (uint32_t)(i % kRing * kTileBytes + u * 1024), A.q + from + 8 * (lc ^ r));
    }
  };
  ask();
  const int id = A.table[(int64_t)b * A.max_pages + piece / 2];
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (id < 0 || id >= A.n_pages) return;
  look();
  ask();
  load(0);
  load(1);
  const uint8_t* page = A.pool + ((int64_t)id * A.Hkv + S.kv) * kPage8Bytes;
  const int key_row = piece % 2 * kHalf + 4 * T * (lc >> 2) + (lc & 3);
  bf16x8 key[T][4];
#pragma unroll
  for (int t = 0; t < T; ++t)
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint2 c = *(const uint2*)(page + (key_row + 4 * t) * kDim8 + 32 * u + 8 * lg);
      key[t][u] = widen(c.x, c.y);
    }
  static_assert(kHalf == fc::kBlock8, "one scale");
  const float scale = key_scale(page[fc::kPage8Scales + piece % 2]);
  float got[4 * T];
#pragma unroll
  for (int i = 0; i < 4 * T; ++i) got[i] = 0.0f;
  const int own0 = key0 + 4 * T * lg;
  int next_last = last;
  for (; tile < tiles; tile += kManyWaves * kRoundTiles) {
    float minus = 0.0f;
    int sees = -1;
#pragma unroll
    for (int i = 0; i < kRoundTiles; ++i) {
      // Behind tile i's loads: the next tile's, and what `look` and `ask` loaded.
      if (i == kRoundTiles - 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kSrc ? 6 : 5) : "memory");
      else asm volatile("s_waitcnt vmcnt(4)" ::: "memory");
      if (i == 0) {
        const float lse = sh.lse[w][lane];
        minus = 0.0f - lse * kLog2e;
        sees = lse == -INFINITY ? -1 : next_last;  // a row that saw nothing pays nothing
      }
      bf16x8 x[4];
#pragma unroll
      for (int u = 0; u < 4; ++u)
        x[u] = *(const bf16x8*)(sh.rows[w][i % kRing] + lc * (kDim8 * 2) + (((4 * u + lg) ^ lc) * 16));
      asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]) : : "memory");
      if (i == kRoundTiles - kRing) {
        look();
        ask();
        next_last = last;
      }
      load((i + kRing) % kRoundTiles);
      pay<T>([&](int t, int u) { return key[t][u]; }, x, scale, __shfl(minus, kTile * i + lc),
             __shfl(sees, kTile * i + lc) - own0, got);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing on its way into LDS that others may get
  float v[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = i < 4 * T ? got[i] : 0.0f;
  float sum = sum_of_own(v, lc);  // of key 8 lg + lc, lc < 8
  if (w > 0) sh.sum[w - 1][lane] = sum;
  __syncthreads();
  if (w > 0 || lc >= 4 * T) return;
#pragma unroll
  for (int g = 0; g < kManyWaves - 1; ++g) sum += sh.sum[g][lane];
  settle_weight(A, S, id, own0 + lc, sum, false);
}

// Few rows (a token, an accepted path): a wave holds up to 64 of them and goes through
// every fourth of its part's pages, the next one's keys on their way.  More rows are
// more rounds of the same pages.  Keys alone are read, 8 KB a page and head: 48 sequences
// of up to 4,096 tokens, 11 accepted at most, 8 key heads 31 us, 2.4 TB/s; what is left
// to memory's 15 us are the pages' exponentials and the longest sequences' parts.
constexpr int kFewTiles = 4;
template <bool kSrc>
__global__ void __launch_bounds__(kThreads, 2) k_weights_few(Weights A, int part_pages) {
  const int lane = fc::lane_id(), lg = lane >> 4, lc = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave);
  const int b = (int)blockIdx.x / A.Hkv;
  const Step S(A, b, (int)blockIdx.x % A.Hkv);
  const int pages = (S.end + kPage8 - 1) / kPage8;
  const int part = A.y0 + (int)blockIdx.y;
  const int pg0 = part * part_pages + w;
  const int pg1 = (part + 1) * part_pages < pages ? (part + 1) * part_pages : pages;
  if (S.n <= 0 || pg0 >= pg1) return;
  const int32_t* table = A.table + (int64_t)b * A.max_pages;
  const uint32_t k_at = (uint32_t)((16 * (lc >> 2) + (lc & 3)) * kDim8 + 16 * lg);
  uint4 k[kKTiles][2];
  uint32_t word = 0;
  const auto load_page = [&](int id) {
    if (id < 0 || id >= A.n_pages) return;
    const uint8_t* p = A.pool + ((int64_t)id * A.Hkv + S.kv) * kPage8Bytes;
#pragma unroll
    for (int t = 0; t < kKTiles; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u) k[t][u] = *(const uint4*)(p + k_at + (4 * t * kDim8 + 64 * u));
    word = *(const uint32_t*)(p + fc::kPage8Scales);
  };
  constexpr int kRound = kFewTiles * kTile;
  const int64_t rows = (int64_t)S.n * S.G;
  const Cursor round(S, kRound);
  Cursor c(S, 0);
  for (int64_t r0 = 0; r0 < rows; r0 += kRound) {
    int id = table[pg0], token, head;
    c.at(S, lane, token, head);
    const int mine = number_of<kSrc>(A, S, token);  // a row a lane
    load_page(id);
    Rows x[kFewTiles];
    const int n = rows - r0 < kRound ? (int)((rows - r0 + kTile - 1) / kTile) : kFewTiles;
#pragma unroll
    for (int i = 0; i < kFewTiles; ++i)
      if (i < n) {
        c.at(S, kTile * i + lc, token, head);
        x[i].load(A, S, token, head, __shfl(mine, kTile * i + lc));
      }
    c += round;
    c.carry(S);
    for (int pg = pg0; pg < pg1; pg += kWaves) {
      const int next = pg + kWaves < pg1 ? table[pg + kWaves] : -1;
      if (id >= 0 && id < A.n_pages) {
        bf16x8 key[kKTiles][4];
#pragma unroll
        for (int t = 0; t < kKTiles; ++t)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            key[t][2 * u] = widen(k[t][u].x, k[t][u].y);
            key[t][2 * u + 1] = widen(k[t][u].z, k[t][u].w);
          }
        const float scale = key_scale((word >> (8 * (lg >> 1))) & 255u);
        load_page(next);
        float got[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) got[i] = 0.0f;
#pragma unroll
        for (int i = 0; i < kFewTiles; ++i)
          if (i < n)
            pay<kKTiles>([&](int t, int u) { return key[t][u]; }, x[i].q, scale, 0.0f - x[i].lse * kLog2e,
                         // a row that saw nothing pays nothing
                         x[i].lse == -INFINITY ? -1 : x[i].last - (pg * kPage8 + 16 * lg), got);
        settle_weight(A, S, id, pg * kPage8 + lane, sum_of_own(got, lc), r0 > 0);  // key 16 lg + lc
      } else {
        load_page(next);
      }
      id = next;
    }
  }
}

// ------------------------------------------------------------------ evict --

constexpr int kSelThreads = 1024;
constexpr int kSelWaves = kSelThreads / fc::kWave;
constexpr int kBins = 2048;

struct Evict {
  uint8_t* pool;
  float* weights;
  const int32_t *table, *len, *budget;
  int32_t* add;
  int32_t* from;    // [B][Hkv][max_len] token that moves to each place
  int32_t* before;  // [B][Hkv][pages + 1] tokens that stay, ahead of each page
  int32_t* flags;   // [B][Hkv][pages + 1] pages whose tokens are read; the last: pages begun
  uint32_t* bins;   // [B][Hkv][3][kBins] and [B][Hkv][parts][2], where there are parts:
  uint32_t* kinds;  // how many tokens of each part stay, and how many do if there is room
  int n_pages, Hkv, max_pages, max_len, pages, parts, first, recent;
  int y0;  // parts before this launch's
};

// How a sequence is cut: its length, how many stay, the tokens that do by their place
// (before lo, from late on), and those of which the `heavy` heaviest do (lo .. hi - 1):
// what lies between, or the first ones where the budget does not take all of them.
struct Cut {
  int n, keep, lo, hi, late, heavy;
  __device__ __forceinline__ Cut(const Evict& A, int b) {
    n = clamp_len(A.len[b], A.max_len);
    keep = clamp_len(A.budget[b], n);
    const int recent = A.recent < keep ? A.recent : keep, rest = keep - recent;
    late = n - recent;
    const bool all = A.first <= rest;
    lo = all ? A.first : 0;
    hi = all || A.first > late ? late : A.first;
    heavy = rest - lo;
  }
};

// A weight as a number that sorts as it does: 0 for what is not above 0.
__device__ __forceinline__ uint32_t rank_of(float w) { return w > 0.0f ? __float_as_uint(w) : 0u; }

// What one head of one sequence keeps: the weight of the last one to stay is found 11
// bits at a time from the top, by counting; then, in order, which tokens are above it,
// and of those that equal it the first ones.  A wave's lanes are a page's tokens, a wave's
// pages follow one another, 16 of them in registers.  One workgroup has up to 256 pages
// and does it all; longer sequences are parts of as many, counted together in memory by
// one launch for each turn (the 131,000 tokens of 8 heads that eight workgroups alone
// read five times over: 186 us, in turns 56; 48 sequences of up to 4,096 tokens, one
// workgroup each, 14).
constexpr int kTogether = 16;
constexpr int kPartPages = kSelWaves * kTogether;

struct Select {
  const Evict& A;
  const Cut& c;
  const int32_t* table;
  int kv, lane, w, p0, p1;
  uint32_t found, left;  // the bits of the last one to stay, and how many of those that share them do
  uint32_t rank[kTogether];
  __device__ __forceinline__ Select(const Evict& a, const Cut& cut, int b, int kv_, int part)
      : A(a), c(cut), table(a.table + (int64_t)b * a.max_pages), kv(kv_), lane(fc::lane_id()),
        w(__builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave)), found(0), left((uint32_t)cut.heavy) {
    const int pages = (c.n + kPage8 - 1) / kPage8, q0 = part * kPartPages;
    const int n = pages - q0 < kPartPages ? pages - q0 : kPartPages;
    p0 = q0 + n * w / kSelWaves, p1 = q0 + n * (w + 1) / kSelWaves;
    // a page number a lane; what is not there has weight 0
    int id = lane < kTogether && p0 + lane < p1 ? table[p0 + lane] : -1;
    if (id >= A.n_pages) id = -1;
    float x[kTogether];
#pragma unroll
    for (int i = 0; i < kTogether; ++i) {
      const int page = __builtin_amdgcn_readlane(id, i);
      x[i] = A.weights[((int64_t)(page < 0 ? 0 : page) * A.Hkv + kv) * kPage8 + lane];
    }
#pragma unroll
    for (int i = 0; i < kTogether; ++i) rank[i] = __builtin_amdgcn_readlane(id, i) < 0 ? 0u : rank_of(x[i]);
  }
  // f(page, the lane's token's rank) for the wave's pages in their order
  template <typename F>
  __device__ __forceinline__ void each_page(F f) {
#pragma unroll
    for (int i = 0; i < kTogether; ++i)
      if (p0 + i < p1) f(p0 + i, rank[i]);
  }
  __device__ __forceinline__ static int shift(int level) { return level == 0 ? 20 : level == 1 ? 9 : 0; }
  __device__ __forceinline__ static int bits(int level) { return level == 2 ? 9 : 11; }
  // The tokens that share the bits found so far, by their next bits.
  __device__ __forceinline__ void count(int level, uint32_t* bins) {
    for (int i = (int)threadIdx.x; i < kBins; i += kSelThreads) bins[i] = 0;
    __syncthreads();
    each_page([&](int p, uint32_t r) {
      const int t = p * kPage8 + lane;
      if (t >= c.lo && t < c.hi && (level == 0 || (r >> (shift(level) + bits(level))) == found))
        atomicAdd(&bins[(r >> shift(level)) & ((1u << bits(level)) - 1u)], 1u);
    });
    __syncthreads();
  }
  // From such counts (x and y: this thread's two, from the largest down), the next bits.
  __device__ __forceinline__ void narrow(int level, uint32_t x, uint32_t y, uint32_t* sum, uint32_t* found_left) {
    const uint32_t top = kBins - 1 - 2 * threadIdx.x;
    const uint32_t ahead = fc::block_excl_sum<uint32_t>(x + y, sum, nullptr);
    if (ahead < left && left <= ahead + x) found_left[0] = top, found_left[1] = left - ahead;
    else if (ahead + x < left && left <= ahead + x + y) found_left[0] = top - 1, found_left[1] = left - ahead - x;
    __syncthreads();
    found = found << bits(level) | found_left[0];
    left = found_left[1];
    __syncthreads();
  }
  // Tokens of a page that stay, and that do if there is room.
  __device__ __forceinline__ void kinds(int p, uint32_t r, uint64_t& stays, uint64_t& equal) const {
    const int t = p * kPage8 + lane;
    const bool by_weight = c.heavy > 0 && t >= c.lo && t < c.hi;
    stays = fc::ballot(t < c.lo || (t >= c.late && t < c.n) || (by_weight && r > found));
    equal = fc::ballot(by_weight && r == found);
  }
  // How many each wave has of either kind, into s_wave; with those before the workgroup's,
  // how many come before this wave's.
  __device__ __forceinline__ void count_kinds(uint32_t (*s_wave)[kSelWaves], uint32_t& sure, uint32_t& maybe) {
    uint32_t a = 0, e = 0;
    each_page([&](int p, uint32_t r) {
      uint64_t stays, equal;
      kinds(p, r, stays, equal);
      a += (uint32_t)__popcll(stays);
      e += (uint32_t)__popcll(equal);
    });
    if (lane == 0) s_wave[0][w] = a, s_wave[1][w] = e;
    __syncthreads();
    for (int i = 0; i < w; ++i) sure += s_wave[0][i], maybe += s_wave[1][i];
  }
  __device__ __forceinline__ void write(int32_t* before, int32_t* from, uint32_t sure, uint32_t maybe) {
    each_page([&](int p, uint32_t r) {
      uint64_t stays, equal;
      kinds(p, r, stays, equal);
      const uint32_t at = sure + (maybe < left ? maybe : left);
      const uint64_t below = fc::lanemask_lt();
      const bool taken = ((equal >> lane) & 1u) && maybe + (uint32_t)__popcll(equal & below) < left;
      const uint64_t all = stays | fc::ballot(taken);
      if (lane == 0) before[p] = (int32_t)at;
      if ((all >> lane) & 1u) from[at + (uint32_t)__popcll(all & below)] = p * kPage8 + lane;
      sure += (uint32_t)__popcll(stays);
      maybe += (uint32_t)__popcll(equal);
    });
  }
};

__global__ void __launch_bounds__(kSelThreads) k_evict_select(Evict A) {
  __shared__ uint32_t s_bins[kBins];
  __shared__ uint32_t s_sum[kSelWaves + 1], s_found[2], s_wave[2][kSelWaves];
  const int tid = (int)threadIdx.x, kv = (int)blockIdx.x % A.Hkv, b = (int)blockIdx.x / A.Hkv;
  const Cut c(A, b);
  if (kv == 0 && tid == 0) A.add[b] = c.keep - c.n;
  if (c.keep >= c.n || c.keep == 0) return;
  const int64_t bk = (int64_t)b * A.Hkv + kv;
  int32_t* flags = A.flags + bk * (A.pages + 1);
  for (int p = tid; p <= A.pages; p += kSelThreads) flags[p] = 0;
  Select s(A, c, b, kv, 0);
  if (c.heavy > 0)
    for (int level = 0; level < 3; ++level) {
      s.count(level, s_bins);
      const int top = kBins - 1 - 2 * tid;
      s.narrow(level, s_bins[top], s_bins[top - 1], s_sum, s_found);
    }
  uint32_t sure = 0, maybe = 0;
  s.count_kinds(s_wave, sure, maybe);
  int32_t* before = A.before + bk * (A.pages + 1);
  s.write(before, A.from + bk * A.max_len, sure, maybe);
  if (tid == 0) before[(c.n + kPage8 - 1) / kPage8] = c.keep;
}

// The same in turns, a workgroup for each part: 0 clears what is counted in memory, 1 to
// 3 count bits, 4 counts what stays, 5 writes it down.  Sums of whole numbers, so the
// order of the atomic additions does not matter.
template <int TURN>
__global__ void __launch_bounds__(kSelThreads) k_evict_turn(Evict A) {
  __shared__ uint32_t s_bins[kBins];
  __shared__ uint32_t s_sum[kSelWaves + 1], s_found[2], s_wave[2][kSelWaves];
  const int tid = (int)threadIdx.x, kv = (int)blockIdx.x % A.Hkv, b = (int)blockIdx.x / A.Hkv;
  const int part = A.y0 + (int)blockIdx.y;
  const Cut c(A, b);
  if (TURN == 0 && kv == 0 && part == 0 && tid == 0) A.add[b] = c.keep - c.n;
  const int pages = (c.n + kPage8 - 1) / kPage8;
  if (c.keep >= c.n || c.keep == 0 || part * kPartPages >= pages) return;
  const int64_t bk = (int64_t)b * A.Hkv + kv;
  uint32_t* bins = A.bins + bk * 3 * kBins;
  uint32_t* of_part = A.kinds + bk * A.parts * 2;
  if (TURN == 0) {
    int32_t* flags = A.flags + bk * (A.pages + 1);
    for (int p = part * kPartPages + tid; p <= A.pages && p < (part + 1) * kPartPages; p += kSelThreads) flags[p] = 0;
    if (part == 0) {
      for (int i = tid; i < 3 * kBins; i += kSelThreads) bins[i] = 0;
      if (tid == 0) flags[A.pages] = 0;
    }
    return;
  }
  if (TURN <= 3 && c.heavy == 0) return;
  Select s(A, c, b, kv, part);
  if (c.heavy > 0)
    for (int level = 0; level < TURN - 1 && level < 3; ++level) {
      const uint32_t* now = bins + level * kBins + kBins - 1 - 2 * tid;
      s.narrow(level, now[0], now[-1], s_sum, s_found);
    }
  if (TURN <= 3) {
    s.count(TURN - 1, s_bins);
    for (int i = tid; i < kBins; i += kSelThreads)
      if (s_bins[i]) atomicAdd(&bins[(TURN - 1) * kBins + i], s_bins[i]);
    return;
  }
  uint32_t sure = 0, maybe = 0;
  if (TURN == 4) {
    s.count_kinds(s_wave, sure, maybe);
    if (tid == kSelThreads - 1) {
      of_part[2 * part] = sure + s_wave[0][kSelWaves - 1];
      of_part[2 * part + 1] = maybe + s_wave[1][kSelWaves - 1];
    }
    return;
  }
  for (int i = 0; i < part; ++i) sure += of_part[2 * i], maybe += of_part[2 * i + 1];
  s.count_kinds(s_wave, sure, maybe);
  int32_t* before = A.before + bk * (A.pages + 1);
  s.write(before, A.from + bk * A.max_len, sure, maybe);
  if (part == 0 && tid == 0) before[pages] = c.keep;
}

constexpr int kMoveThreads = 256;
// Workgroups of a launch: each goes on with the next page of its sequence and head.  48
// sequences cut from up to 4,096 tokens to 1,000, choice and reading back too: 1,024 93 us,
// 2,048 77, 4,096 and more 75; one of 131,000 cut to 60,000: the same with all.
constexpr uint32_t kMoveAtOnce = 4096;
constexpr int kMoveWaves = kMoveThreads / fc::kWave;

// Codes as numbers that sort as their magnitudes do, 0 for a NaN.  Eight times an
// exponent on top is a code's magnitude at that scale, as long as the code is a normal
// number (8 or more): an exponent is three bits above the mantissa's last.
__device__ __forceinline__ uint32_t magnitude7(uint32_t code) {
  const uint32_t m = code & 127u;
  return m == 127u ? 0u : m;
}
// What makes a token's codes those of another scale: 2^(was - now), as far as it matters
// (below, codes become 0; above, there are none but zeros and NaN).
__device__ __forceinline__ float ratio8(int was, int now) {
  const int e = was - now;
  return e < -126 ? 0.0f : fc::power8(e > 127 ? 127 : e);
}

// A workgroup brings 64 tokens to one page of their new places at a time.  They come
// from this page and later ones; it reads them into registers, says so, waits until the
// pages ahead of it that read from this one have said so too (two at most), and writes.
// Pages are taken in the order of a counter, so that whoever is waited for has begun,
// and nobody waits before it has read: the wait ends.  Two waves a block of 32: keys 16
// bytes a lane, values a dim a lane, whose bytes lie 16 apart.
__global__ void __launch_bounds__(kMoveThreads, 4) k_evict_move(Evict A) {
  __shared__ int s_page;
  __shared__ int s_top[2][kMoveWaves];
  const int tid = (int)threadIdx.x, lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane(tid / fc::kWave);
  const int kv = (int)blockIdx.x % A.Hkv, b = (int)blockIdx.x / A.Hkv;
  const Cut c(A, b);
  if (c.keep >= c.n || c.keep == 0) return;
  const int64_t bk = (int64_t)b * A.Hkv + kv;
  const int32_t* table = A.table + (int64_t)b * A.max_pages;
  const int32_t* before = A.before + bk * (A.pages + 1);
  int32_t* flags = A.flags + bk * (A.pages + 1);
  const int pages = (c.keep + kPage8 - 1) / kPage8;
  const int half = w >> 1, t0 = half * kBlock8;  // the wave's block
  const uint32_t d = (uint32_t)(64 * (w & 1) + lane);
  const auto take_page = [&]() {
    if (tid == 0) s_page = __hip_atomic_fetch_add(&flags[A.pages], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  take_page();
  for (;;) {
    __syncthreads();
    const int pg = __builtin_amdgcn_readfirstlane(s_page);
    if (pg >= pages) return;
    const int here = c.keep - pg * kPage8 < kPage8 ? c.keep - pg * kPage8 : kPage8;  // tokens of the page
    // lane i (and i + 32) has token t0 + i: its place, its scales, its weight
    const int mine = t0 + (lane & 31);
    const int t = mine < here ? A.from[bk * A.max_len + (int64_t)pg * kPage8 + mine] : -1;
    const int q0 = before[pg], q1 = before[pg + 1];
    const int to = table[pg];
    int id = t >= 0 ? table[t / kPage8] : -1;
    if (id >= A.n_pages) id = -1;
    const int64_t base = (int64_t)(id < 0 ? 0 : id) * A.Hkv + kv;  // what is not there reads page 0, for nothing
    const int row = id < 0 ? 0 : t % kPage8;
    const uint8_t* scales = A.pool + base * kPage8Bytes + fc::kPage8Scales + row / kBlock8;
    const int k_byte = scales[0], v_byte = scales[2];
    const float weight = A.weights[base * kPage8 + row];
    // keys: 16 rows a wave, eight lanes each
    const int64_t at = base * kPage8Bytes + row * kDim8;  // of the token's keys
    uint4 k[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const int64_t key = __shfl(at, 16 * (w & 1) + 8 * p + (lane >> 3));
      k[p] = *(const uint4*)(A.pool + key + 16 * (lane & 7));
    }
    // values: every token of the block, one dim a lane
    const int64_t v_at = base * kPage8Bytes + fc::v8_at(row, 0);
    uint32_t v[kBlock8];
#pragma unroll
    for (int i = 0; i < kBlock8; ++i) {
      const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v_at, i);
      const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)((uint64_t)v_at >> 32), i);
      v[i] = (A.pool + (((uint64_t)hi << 32) | lo))[d * fc::kQuarter8];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // all of it is here
    __syncthreads();
    if (tid == 0) __hip_atomic_store(&flags[pg], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    take_page();  // the next one

    // The largest magnitude of each block, as magnitude7 plus eight times the exponent
    // (-1024: none).  Codes below 8 count as nothing where one above them is as large at
    // the block's largest scale; where none is, their exact magnitudes decide.
    constexpr int kNone = -1024;
    const int k_exp = id < 0 ? kNone : fc::clamp_exp8(k_byte - 127), v_exp = id < 0 ? kNone : fc::clamp_exp8(v_byte - 127);
    int k_from[2], top[2] = {0, 0}, least[2];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      k_from[p] = __shfl(k_exp, 16 * (w & 1) + 8 * p + (lane >> 3));
      if (k_from[p] == kNone) k[p] = make_uint4(0u, 0u, 0u, 0u);
    }
    const auto code_of = [](const uint4& x, int i) { return ((i < 4 ? x.x : i < 8 ? x.y : i < 12 ? x.z : x.w) >> (8 * (i & 3))) & 255u; };
    const auto all_lanes = [](int x, auto join) {
#pragma unroll
      for (int o = 1; o < fc::kWave; o <<= 1) x = join(x, __shfl_xor(x, o));
      return x;
    };
    const auto larger = [](int x, int y) { return x > y ? x : y; };
    top[0] = top[1] = 8 * kNone;
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint32_t m = magnitude7(code_of(k[p], i));
        most = m > most ? m : most;
      }
      if (most > 0) top[0] = larger(top[0], (int)most + 8 * k_from[p]);
    }
#pragma unroll
    for (int i = 0; i < kBlock8; ++i) {
      const int e = __builtin_amdgcn_readlane(v_exp, i);
      if (e == kNone) v[i] = 0;
      const uint32_t m = magnitude7(v[i]);
      top[1] = larger(top[1], m > 0 ? (int)m + 8 * e : 8 * kNone);
    }
    // the block's largest exponents: those of its tokens, which every wave has
    least[0] = all_lanes(k_exp, larger);
    least[1] = all_lanes(v_exp, larger);
    top[0] = all_lanes(top[0], larger);
    top[1] = all_lanes(top[1], larger);
    if (lane == 0) s_top[0][w] = top[0], s_top[1][w] = top[1];
    __syncthreads();
    int e[2];
    bool exact = false;  // whether a small code's own magnitude may decide
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int x = larger(s_top[i][w & ~1], s_top[i][w | 1]);
      // 448 is code 126
      e[i] = x <= 8 * kNone ? fc::kLeastExp8 : fc::clamp_exp8((x - 126 + 7) >> 3);
      exact |= x > 8 * kNone && x < 8 + 8 * least[i];
    }
    if (__any(exact)) {  // both waves of a block alike
      uint32_t bits[2] = {0, 0};
      const auto reach = [](uint32_t code, int e) { return fc::reach8(__builtin_amdgcn_cvt_f32_fp8((int)code, 0) * fc::power8(e)); };
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t m = k_from[p] == kNone ? 0u : reach(code_of(k[p], i), k_from[p]);
          bits[0] = m > bits[0] ? m : bits[0];
        }
#pragma unroll
      for (int i = 0; i < kBlock8; ++i) {
        const int from = __builtin_amdgcn_readlane(v_exp, i);
        const uint32_t m = from == kNone ? 0u : reach(v[i], from);
        bits[1] = m > bits[1] ? m : bits[1];
      }
      top[0] = all_lanes((int)bits[0], larger);
      top[1] = all_lanes((int)bits[1], larger);
    }
    __syncthreads();
    if (lane == 0) s_top[0][w] = top[0], s_top[1][w] = top[1];
    __syncthreads();
    if (__any(exact)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) e[i] = fc::exponent8((uint32_t)larger(s_top[i][w & ~1], s_top[i][w | 1]));
    }
    // codes at another scale are rounded anew
#pragma unroll
    for (int p = 0; p < 2; ++p)
      if (__any(k_from[p] != kNone && k_from[p] != e[0])) {
        const float f = k_from[p] == kNone ? 0.0f : ratio8(k_from[p], e[0]);
        k[p] = make_uint4(fc::recode8(k[p].x, f), fc::recode8(k[p].y, f), fc::recode8(k[p].z, f), fc::recode8(k[p].w, f));
      }
    uint32_t codes[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) codes[i] = v[4 * i] | v[4 * i + 1] << 8 | v[4 * i + 2] << 16 | v[4 * i + 3] << 24;
    if (__any(v_exp != kNone && v_exp != e[1])) {
      const float f = v_exp == kNone ? 0.0f : ratio8(v_exp, e[1]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          x[u] = __builtin_amdgcn_cvt_f32_fp8((int)v[4 * i + u], 0) *
                 __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(f), 4 * i + u));
        codes[i] = fc::codes8(x[0], x[1], x[2], x[3]);
      }
    }

    // tokens of this page stay for pages ahead: those have to be read
    if (tid == 0 && q0 < q1) {
      for (int q = q0 / kPage8; q <= (q1 - 1) / kPage8 && q < pg; ++q)
        while (__hip_atomic_load(&flags[q], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == 0) __builtin_amdgcn_s_sleep(1);
    }
    __syncthreads();
    if (to < 0 || to >= A.n_pages || t0 >= here) continue;  // a block behind the last token stays as it was
    const int64_t dest = (int64_t)to * A.Hkv + kv;
    uint8_t* page = A.pool + dest * kPage8Bytes;
    if ((w & 1) == 0 && lane < kBlock8 && mine < here) A.weights[dest * kPage8 + mine] = id < 0 ? 0.0f : weight;
#pragma unroll
    for (int p = 0; p < 2; ++p)
      *(uint4*)(page + (t0 + 16 * (w & 1) + 8 * p + (lane >> 3)) * kDim8 + 16 * (lane & 7)) = k[p];
#pragma unroll
    for (int q = 0; q < 2; ++q)
      *(uint4*)(page + fc::v8_at(t0 + 16 * q, (int)d)) = make_uint4(codes[4 * q], codes[4 * q + 1], codes[4 * q + 2], codes[4 * q + 3]);
    if ((w & 1) == 0 && lane < 2) page[fc::kPage8Scales + 2 * lane + half] = (uint8_t)(e[lane] + 127);
  }
}

// A launch takes fewer than 2^32 threads in a dimension, and 65,536 workgroups in the
// second: longer calls are several.
constexpr uint32_t kMostY = 1 << 15;
constexpr int64_t kMostMany = 1 << 22;  // workgroups of 512 threads
template <int TURN>
void in_turn(Evict a, uint32_t pairs, hipStream_t stream) {
  for (uint32_t y = 0; y < (uint32_t)a.parts; y += kMostY) {
    a.y0 = (int)y;
    const uint32_t parts = (uint32_t)a.parts - y;
    hipLaunchKernelGGL(k_evict_turn<TURN>, dim3(pairs, parts < kMostY ? parts : kMostY), dim3(kSelThreads), 0, stream, a);
  }
}

size_t carve(void* p, int32_t B, int32_t Hkv, int32_t max_len, Evict& a) {
  fc::Carver c(p);
  const size_t rows = (size_t)B * Hkv;
  a.pages = (max_len + kPage8 - 1) / kPage8;
  a.from = c.take<int32_t>(rows * (size_t)max_len);
  a.before = c.take<int32_t>(rows * ((size_t)a.pages + 1));
  a.flags = c.take<int32_t>(rows * ((size_t)a.pages + 1));
  a.parts = (a.pages + kPartPages - 1) / kPartPages;
  a.bins = a.parts > 1 ? c.take<uint32_t>(rows * 3 * kBins) : nullptr;
  a.kinds = a.parts > 1 ? c.take<uint32_t>(rows * 2 * (size_t)a.parts) : nullptr;
  return c.used + 256;
}

int32_t sequences_at_once(int32_t B, int32_t Hkv) {
  const int32_t most = (1 << 20) / Hkv;  // Hkv is 1,024 at most
  return B < most ? B : most;
}

bool sizes_ok(int32_t B, int32_t Hkv, int32_t max_len) {
  return B >= 0 && B <= 65536 && Hkv >= 1 && Hkv <= 1024 && max_len >= 0 && max_len <= 0x7FFFFFFF - kPage8;
}

}  // namespace

extern "C" fc_status fc_paged_byte_weights(float* weights, const uint16_t* q, int64_t q_stride, const float* lse,
                                           int32_t n_rows, const uint8_t* pool, int32_t n_pages, const int32_t* table,
                                           int32_t max_pages, const int32_t* len, const int32_t* new_len,
                                           const int32_t* cu, const int32_t* src, int32_t n, int32_t B, int32_t H,
                                           int32_t Hkv, int32_t D, int32_t max_len, hipStream_t stream) {
  if (!sizes_ok(B, Hkv, max_len) || n_rows < 0 || n < 0 || H < Hkv || H > 8192 || H % Hkv || n_pages < 1 ||
      n_pages > (1 << 25) - 1 || max_pages < 1 || (int64_t)max_len > (int64_t)max_pages * kPage8)
    return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (q_stride < (int64_t)H * D || (q_stride & 7)) return FC_ERR_INVALID;
  if (B == 0 || n_rows == 0 || n == 0 || max_len == 0) return FC_OK;
  if (!weights || !q || !lse || !pool || !table || !len || !new_len || !cu) return FC_ERR_INVALID;
  if (((uintptr_t)q | (uintptr_t)pool) & 15 || ((uintptr_t)weights | (uintptr_t)lse) & 3) return FC_ERR_INVALID;
  const uint64_t seqs = 4 * (uint64_t)B;
  if (!fc::apart({{weights, 4 * (uint64_t)n_pages * Hkv * kPage8}},
                 {fc::rows_span(q, n_rows, q_stride, (int64_t)H * D),
                  {lse, 4 * (uint64_t)n_rows * H},
                  {pool, fc_paged_byte_pool_bytes(n_pages, Hkv)},
                  {table, seqs * max_pages},
                  {len, seqs},
                  {new_len, seqs},
                  {cu, seqs + 4},
                  {src, 4 * (uint64_t)n}}))
    return FC_ERR_INVALID;
  const uint32_t pages = fc::div_up((uint64_t)max_len, kPage8);
  // Held rows go through the pages in rounds of 64, P pages of all heads together at
  // 5.5 + 0.002 P us a round.  Held pages cost 9 + 0.034 P us to begin with (a workgroup
  // waits three times before its first product), and rows past the first 500 0.0018 P us
  // for each 64.  Both measured: 32 heads on 8, 1 sequence of 2,000 tokens, 264 pages: 256
  // rows 23 and 18 us, 2,048 rows 118 and 37; 8 sequences, 2,112 pages: 256 rows 43 and
  // 81, 512 rows 85 and 82, 1,024 rows 183 and 117; 48 sequences, 12,700 pages: 512 rows
  // 235 and 436, 1,024 rows 482 and 617.  A call goes one way whole, by its average and by
  // max_len: a prompt of 2,000 tokens beside 63 single tokens over up to 4,000 is 1,334 us,
  // as two calls 43 and 38.
  const int64_t all_pages = (int64_t)B * Hkv * pages;
  const bool many = all_pages * (kPage8 / kHalf) <= kMostMany &&
                    25 * (int64_t)n * (H / Hkv) >= 4 * (int64_t)B * (all_pages + 700);
  // Four pages a wave, or fewer where that leaves the card idle (48 sequences: 4 31 us, 2
  // 31, 1 40; one of 3,000 tokens: no difference).
  int each = 4;
  while (each > 1 && (int64_t)B * Hkv * fc::div_up(pages, each * kWaves) < 1024) each /= 2;
  (void)hipGetLastError();
  const auto now = [&](int32_t b, int y0) {
    return Weights{weights, q, q_stride, lse, pool, table + (int64_t)b * max_pages, len + b, new_len + b, cu + b, src,
                   n_rows, n_pages, max_pages, n, H, Hkv, max_len, y0};
  };
  if (many) {
    const uint32_t pieces = pages * (kPage8 / kHalf), pairs = (uint32_t)B * (uint32_t)Hkv;
    const auto kernel = src ? k_weights_many<true> : k_weights_many<false>;
    hipLaunchKernelGGL(kernel, dim3(pairs * pieces), dim3(kManyWaves * fc::kWave), 0, stream, now(0, 0), (int)pairs, (int)pieces);
    FC_CHECK_LAUNCH();
    return FC_OK;
  }
  const uint32_t parts = fc::div_up(pages, each * kWaves);
  const int32_t at_once = sequences_at_once(B, Hkv);
  for (int32_t b = 0; b < B; b += at_once) {
    const uint32_t pairs = (uint32_t)(B - b < at_once ? B - b : at_once) * (uint32_t)Hkv;
    for (uint32_t y = 0; y < parts; y += kMostY) {
      const auto kernel = src ? k_weights_few<true> : k_weights_few<false>;
      hipLaunchKernelGGL(kernel, dim3(pairs, parts - y < kMostY ? parts - y : kMostY), dim3(kThreads), 0, stream,
                         now(b, (int)y), each * kWaves);
      FC_CHECK_LAUNCH();
    }
  }
  return FC_OK;
}

extern "C" size_t fc_paged_byte_evict_workspace_bytes(int32_t B, int32_t Hkv, int32_t max_len) {
  if (!sizes_ok(B, Hkv, max_len) || B == 0) return 0;
  Evict a;
  return carve(nullptr, B, Hkv, max_len, a);
}

extern "C" fc_status fc_paged_byte_evict(uint8_t* pool, float* weights, int32_t n_pages, int32_t Hkv, int32_t D,
                                         const int32_t* table, int32_t max_pages, const int32_t* len,
                                         const int32_t* budget, int32_t B, int32_t max_len, int32_t first,
                                         int32_t recent, int32_t* add, void* ws, size_t ws_bytes, hipStream_t stream) {
  if (!sizes_ok(B, Hkv, max_len) || n_pages < 1 || n_pages > (1 << 25) - 1 || max_pages < 1 ||
      (int64_t)max_len > (int64_t)max_pages * kPage8 || first < 0 || recent < 0)
    return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (B == 0) return FC_OK;
  if (!pool || !weights || !table || !len || !budget || !add) return FC_ERR_INVALID;
  if ((uintptr_t)pool & 15 || (uintptr_t)weights & 3) return FC_ERR_INVALID;
  const size_t need = fc_paged_byte_evict_workspace_bytes(B, Hkv, max_len);
  if (!ws || ws_bytes < need) return FC_ERR_WORKSPACE;
  if ((uintptr_t)ws & 15) return FC_ERR_INVALID;
  const uint64_t seqs = 4 * (uint64_t)B;
  if (!fc::apart({{pool, fc_paged_byte_pool_bytes(n_pages, Hkv)},
                  {weights, 4 * (uint64_t)n_pages * Hkv * kPage8},
                  {add, seqs},
                  {ws, need}},
                 {{table, seqs * max_pages}, {len, seqs}, {budget, seqs}}))
    return FC_ERR_INVALID;
  Evict a = {pool, weights, table, len, budget, add, nullptr, nullptr, nullptr, nullptr, nullptr, n_pages, Hkv, max_pages,
             max_len, 0, 0, first, recent, 0};
  carve(ws, B, Hkv, max_len, a);
  (void)hipGetLastError();
  const int32_t at_once = sequences_at_once(B, Hkv);
  for (int32_t b = 0; b < B; b += at_once) {
    const uint32_t pairs = (uint32_t)(B - b < at_once ? B - b : at_once) * (uint32_t)Hkv;
    const int64_t before = (int64_t)b * Hkv;
    Evict now = a;
    now.table += (int64_t)b * max_pages, now.len += b, now.budget += b, now.add += b;
    now.from += before * max_len, now.before += before * (a.pages + 1), now.flags += before * (a.pages + 1);
    if (a.parts <= 1) {
      hipLaunchKernelGGL(k_evict_select, dim3(pairs), dim3(kSelThreads), 0, stream, now);
    } else {
      now.bins += before * 3 * kBins, now.kinds += before * 2 * a.parts;
      in_turn<0>(now, pairs, stream);
      in_turn<1>(now, pairs, stream);
      in_turn<2>(now, pairs, stream);
      in_turn<3>(now, pairs, stream);
      in_turn<4>(now, pairs, stream);
      in_turn<5>(now, pairs, stream);
    }
    FC_CHECK_LAUNCH();
    if (a.pages == 0) continue;
    const uint32_t each = fc::div_up(kMoveAtOnce, pairs);
    hipLaunchKernelGGL(k_evict_move, dim3(pairs, each < (uint32_t)a.pages ? each : (uint32_t)a.pages), dim3(kMoveThreads), 0,
                       stream, now);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

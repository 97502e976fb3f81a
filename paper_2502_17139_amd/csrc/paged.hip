// The paged 4-bit cache on gfx950: its plan, writes and reads (fc_paged_plan,
// fc_paged_write, fc_paged_read).
//
// All three move little arithmetic and are bound by launches (a decoding
// step's few hundred tokens) or by memory (prompts).
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

// ------------------------------------------------------------------- plan --

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / fc::kWave;
constexpr int kPlanEach = 4;                           // tokens of a thread
constexpr int kPlanTokens = kPlanThreads * kPlanEach;  // tokens of the slot map that a workgroup writes

// Exclusive prefix sums of three values over the first `waves` waves of the
// workgroup (no other holds one), and their totals, with one pass through LDS.
struct Sums {
  uint64_t x[3];
};
__device__ __forceinline__ Sums block_sums(const Sums& v, int waves, Sums* scratch, Sums& total) {
  const int w = (int)threadIdx.x / fc::kWave;
  Sums before = {{0, 0, 0}};
  total = before;
  if (w < waves) {
    Sums inc;
#pragma unroll
    for (int i = 0; i < 3; ++i) inc.x[i] = fc::wave_incl_sum_any(v.x[i]);
    if (fc::lane_id() == fc::kWave - 1) scratch[w] = inc;
#pragma unroll
    for (int i = 0; i < 3; ++i) before.x[i] = inc.x[i] - v.x[i];
  }
  __syncthreads();
#pragma unroll 4
  for (int k = 0; k < waves; ++k) {
    const Sums s = scratch[k];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      before.x[i] += k < w ? s.x[i] : 0;
      total.x[i] += s.x[i];
    }
  }
  __syncthreads();
  return before;
}

// Every workgroup scans all sequences (three prefix sums: tokens, new pages,
// pages given back) and keeps, in LDS, those whose tokens fall into its own
// window of the slot map; so no workgroup waits for another and one launch does
// it all.  A window position that starts a sequence carries that sequence's
// data; a running maximum over the positions takes each token to its start.
// What it costs is latency: a load of the lengths, the sums, and for a tree's
// step a load of each sequence's mask row; hence sixteen waves, four sequences' rows
// at a time each, and 4,096 tokens a workgroup, so that few workgroups scan.  64
// accepted paths 8.7 us (18 with four waves and a row at a time), 512 prompts of a
// million slots 21 (39; 64 with 1,024 tokens a workgroup; a copy of its bytes
// takes 2.4): a window's 24 bytes a position make 148 KB of LDS, so a CU has one
// workgroup, and 385 of them are two rounds.  The scan is 8 bytes a sequence from L2:
// at the 65,536 sequences allowed it is what costs, at the thousands of a serving
// batch it is not.
__global__ void __launch_bounds__(kPlanThreads) k_paged_plan(
    const int32_t* __restrict__ len, const int32_t* __restrict__ add, const int32_t* __restrict__ mask,
    const int32_t* __restrict__ last_node, int B, int R, int n_slots, int32_t* table, int max_pages, int32_t* queue,
    int n_pages, const int64_t* __restrict__ ends, int32_t* __restrict__ len_out, int32_t* __restrict__ cu,
    int32_t* __restrict__ slot, int32_t* __restrict__ pos, int32_t* __restrict__ src,
    int64_t* __restrict__ ends_out) {
  struct Seq {  // of a window position that starts a sequence
    int32_t pos0;    // position of the token at window position 0, were it this sequence's
    int32_t b;
    uint32_t page0;  // new pages taken before its own
    uint32_t count;  // tokens
    uint32_t first;  // its token number at this window position
    int32_t last;    // its accepted row, -2 if the sequence does not fit
  };
  struct Back {  // pages that a sequence gives back
    uint32_t to;
    int32_t b, from, count;
  };
  __shared__ Sums s_scan[kPlanWaves];
  __shared__ int s_scan_max[kPlanWaves + 1];
  __shared__ Seq s_seq[kPlanTokens];
  __shared__ uint16_t s_start[kPlanTokens];  // window position + 1 where a sequence starts, else 0
  __shared__ uint16_t s_list[kPlanTokens];   // those positions, in any order
  __shared__ int32_t s_src[kPlanTokens];
  __shared__ Back s_back[kPlanThreads];
  __shared__ int s_listed, s_backs;
  __shared__ unsigned long long s_given;

  const int tid = (int)threadIdx.x, wave = tid / fc::kWave, lane = fc::lane_id();
  const int64_t w0 = (int64_t)blockIdx.x * kPlanTokens;
  const int64_t head = ends[0], tail = ends[1];
  const uint64_t held_free = tail > head ? (uint64_t)(tail - head) : 0;
  const uint64_t avail = held_free < (uint64_t)n_pages ? held_free : (uint64_t)n_pages;
  // the first chunk's inputs, on their way while LDS is cleared
  const int32_t len0 = tid < B ? len[tid] : 0, add0 = tid < B ? add[tid] : 0;
  const int32_t last0 = tid < B && mask ? last_node[tid] : -1;
  for (int x = tid; x < kPlanTokens; x += kPlanThreads) s_start[x] = 0, s_src[x] = -1;
  if (tid == 0) s_listed = 0, s_given = 0, s_backs = 0;
  __syncthreads();

  uint64_t tokens = 0, taken = 0, given_back = 0;  // of the sequences before this chunk
  for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const bool in = b < B;
    const int64_t cap = (int64_t)max_pages * kPage;
    int64_t n = b0 == 0 ? len0 : in ? len[b] : 0;
    n = n < 0 ? 0 : n > cap ? cap : n;
    const int64_t a = b0 == 0 ? add0 : in ? add[b] : 0;
    const uint64_t want = a > 0 ? (uint64_t)a : 0;
    int64_t now = n + a < 0 ? 0 : n + a;
    const int64_t held = (n + kPage - 1) / kPage, pages = (now + kPage - 1) / kPage;
    const uint64_t back = a < 0 ? (uint64_t)(held - pages) : 0;
    const bool short_enough = a <= 0 || pages <= max_pages;
    uint64_t need = short_enough && a > 0 ? (uint64_t)(pages - held) : 0;
    int32_t last = b0 == 0 ? last0 : in && mask ? last_node[b] : -1;
    if (last >= R || last < 0) last = -1;
    const int waves = B - b0 < kPlanThreads ? (int)fc::div_up((uint64_t)(B - b0), fc::kWave) : kPlanWaves;
    Sums sum;
    const Sums before = block_sums(Sums{{want, back, need}}, waves, s_scan, sum);
    const uint64_t first = tokens + before.x[0], to = given_back + before.x[1];
    uint64_t page0 = taken + before.x[2];
    tokens += sum.x[0];
    given_back += sum.x[1];
    const bool fits = short_enough && (a <= 0 || first + want <= (uint64_t)n_slots);
    if (tokens > (uint64_t)n_slots) {  // the same for all threads: some do not fit, and take no pages
      need = fits ? need : 0;
      page0 = taken + block_sums(Sums{{need, 0, 0}}, waves, s_scan, sum).x[0];
      sum.x[2] = sum.x[0];
    }
    taken += sum.x[2];
    const bool ok = fits && (need == 0 || page0 + need <= avail);
    // the sums only grow: of a wave's sequences that take pages the last one has the most
    const uint64_t takes = fc::ballot(ok && need > 0);
    if (takes && lane == 63 - __builtin_clzll(takes)) atomicMax(&s_given, (unsigned long long)(page0 + need));
    if (!ok) now = n;
    if (in && blockIdx.x == 0) {
      len_out[b] = (int32_t)now;
      const uint64_t end = first + want;
      cu[b + 1] = (int32_t)(end < 0x7FFFFFFFu ? end : 0x7FFFFFFFu);
    }
    if (back > 0 && (uint32_t)b % gridDim.x == blockIdx.x)
      s_back[atomicAdd(&s_backs, 1)] = Back{(uint32_t)(((uint64_t)tail + to) % (uint32_t)n_pages), b, (int32_t)pages, (int32_t)back};
    const bool here = want > 0 && (int64_t)first < w0 + kPlanTokens && (int64_t)(first + want) > w0;
    const uint64_t in_wave = fc::ballot(here);
    int at = 0;
    if (in_wave && lane == 0) at = atomicAdd(&s_listed, (int)__builtin_popcountll(in_wave));
    at = __shfl(at, 0) + (int)__builtin_popcountll(in_wave & fc::lanemask_lt());
    if (here) {
      const int x = (int64_t)first > w0 ? (int)((int64_t)first - w0) : 0;
      s_seq[x] = Seq{(int32_t)(n - ((int64_t)first - w0)), b, (uint32_t)page0, (uint32_t)want,
                     (uint32_t)(w0 + x - (int64_t)first), ok ? last : -2};
      s_start[x] = (uint16_t)(x + 1);
      s_list[at] = (uint16_t)x;
    }
    __syncthreads();
    const int backs = s_backs;
    for (int i = wave; i < backs; i += kPlanWaves) {
      const Back r = s_back[i];
      for (int j = lane; j < r.count; j += fc::kWave)
        queue[(r.to + (uint32_t)j) % (uint32_t)n_pages] = table[(int64_t)r.b * max_pages + r.from + j];
    }
    __syncthreads();
    if (tid == 0) s_backs = 0;
  }
  if (tid == 0 && blockIdx.x == 0) {
    cu[0] = 0;
    ends_out[0] = head + (int64_t)s_given;
    ends_out[1] = tail + (int64_t)given_back;
  }

  // a tree step's source rows: a wave per sequence takes the rows that the
  // accepted row may see, in order
  if (mask) {
    constexpr int kAtOnce = 4;  // sequences of a wave whose rows are on their way together
    const int listed = s_listed;
    for (int i0 = wave; i0 < listed; i0 += kAtOnce * kPlanWaves) {
      int x[kAtOnce], before[kAtOnce];
      Seq q[kAtOnce];
      const int32_t* row[kAtOnce];
#pragma unroll
      for (int u = 0; u < kAtOnce; ++u) {
        const int i = i0 + u * kPlanWaves;
        x[u] = s_list[i < listed ? i : i0];
        q[u] = s_seq[x[u]];
        if (i >= listed) q[u].last = -1;
        row[u] = mask + ((int64_t)q[u].b * R + (q[u].last < 0 ? 0 : q[u].last)) * R;
        before[u] = 0;
      }
      for (int j0 = 0; j0 < R; j0 += fc::kWave) {
        const int j = j0 + lane;
        int32_t m[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) m[u] = row[u][j < R ? j : 0];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
          const bool on = j < R && m[u] == 1 && q[u].last >= 0;
          const uint64_t all = fc::ballot(on);
          const uint32_t t = (uint32_t)(before[u] + (int)__builtin_popcountll(all & fc::lanemask_lt()));
          const uint32_t to = x[u] + t - q[u].first;
          if (on && t >= q[u].first && t < q[u].count && to < kPlanTokens) s_src[to] = q[u].b * R + j;
          before[u] += (int)__builtin_popcountll(all);
        }
      }
    }
    __syncthreads();
  }

  const uint32_t head_at = (uint32_t)((uint64_t)head % (uint32_t)n_pages);
  int start[kPlanEach], run = 0;
#pragma unroll
  for (int e = 0; e < kPlanEach; ++e) {
    const int x = s_start[tid * kPlanEach + e];
    run = x > run ? x : run;
    start[e] = run;
  }
  const int before = fc::block_excl_max<int>(run, 0, s_scan_max);
  int32_t sl[kPlanEach], po[kPlanEach], sr[kPlanEach];
#pragma unroll
  for (int e = 0; e < kPlanEach; ++e) {
    const int x = tid * kPlanEach + e;
    const int64_t at = w0 + x;
    const int from = start[e] > before ? start[e] : before;
    sl[e] = po[e] = sr[e] = -1;
    if (from == 0 || (uint64_t)at >= tokens || at >= n_slots) continue;
    const Seq q = s_seq[from - 1];
    if (q.last == -2) continue;
    const int32_t p = q.pos0 + x;
    const int32_t n = q.pos0 + (from - 1) - (int32_t)q.first;  // tokens it had
    const int idx = p / kPage, held = (n + kPage - 1) / kPage;
    int32_t page;
    if (idx < held) {
      page = table[(int64_t)q.b * max_pages + idx];
    } else {
      const uint32_t i = head_at + q.page0 + (uint32_t)(idx - held);  // less than 2 n_pages
      page = queue[i < (uint32_t)n_pages ? i : i - (uint32_t)n_pages];
      if (p % kPage == 0) table[(int64_t)q.b * max_pages + idx] = page;  // every new page starts with a token
    }
    sl[e] = page >= 0 && page < n_pages ? page * kPage + p % kPage : -1;
    po[e] = p;
    sr[e] = mask ? s_src[x] : (int32_t)at;
  }
#pragma unroll
  for (int e = 0; e < kPlanEach; ++e) {
    const int64_t at = w0 + tid * kPlanEach + e;
    if (at >= n_slots) return;
    slot[at] = sl[e];
    pos[at] = po[e];
    src[at] = sr[e];
  }
}

// ------------------------------------------------------------------ write --

constexpr int kWriteThreads = 256;
constexpr int kWriteWaves = kWriteThreads / fc::kWave;
static_assert(kHeadDim / 2 == fc::kWave, "a lane per angle");
constexpr int kUnitLanes = 8;                              // lanes of one token's key (or value) head
constexpr int kUnits = kWriteThreads / kUnitLanes;         // units at work in a workgroup
constexpr int kMaxTokens = 16;                             // tokens of a workgroup at most: 16 KB of LDS, eight of a CU
constexpr double kInvPi = 0.31830988618379067154;

// Sine (x) and cosine of an angle in half turns.
__device__ __forceinline__ double2 turn(double half_turns) {
  double s, c;
  sincospi(half_turns - 2.0 * floor(half_turns * 0.5), &s, &c);
  return make_double2(s, c);
}

// A unit is one token's keys or values of one head.  Lane j of its eight holds
// dims 8 j .. 8 j + 7 and the same 64 further on: the two halves of each
// rotation, and quarters of two scale groups.  12 prompts of up to 4,096 tokens, 32
// key heads: 132 us, 70 % of the rate of a large copy.  113 MiB reach memory for the
// 91 written (rows of 64 bytes, scales byte by byte), 5 us of the 40 that are missing;
// the others may be the angles, which a workgroup of one token waits for.  One
// accepted path of each of 64 sequences: 4.4 us, a launch and the latency of a load.
__global__ void __launch_bounds__(kWriteThreads) k_paged_write(
    uint8_t* __restrict__ pool, int n_pages, int Hkv, const uint16_t* __restrict__ k, int64_t k_stride,
    const uint16_t* __restrict__ v, int64_t v_stride, int n_src, const int32_t* __restrict__ slot,
    const int32_t* __restrict__ pos, const int32_t* __restrict__ src, int n, int tokens, double log2_base) {
  __shared__ double2 s_turn[kMaxTokens * kHeadDim / 2];
  const int tid = (int)threadIdx.x;
  const int64_t i0 = (int64_t)blockIdx.x * tokens;
  if (log2_base > 0.0) {
    // a lane per angle, a wave per run of tokens: where one sits behind the other
    // its angles follow from the last ones by a turn of one position
    const int d = tid % fc::kWave, each = (tokens + kWriteWaves - 1) / kWriteWaves;
    const double freq = exp2(-2.0 * d / (double)kHeadDim * log2_base) * kInvPi;
    const double2 one = each > 1 ? turn(freq) : make_double2(0.0, 1.0);
    double2 t = one;
    int at = 0;
    for (int e = 0; e < each; ++e) {
      const int x = tid / fc::kWave * each + e;
      if (x >= tokens || i0 + x >= n) break;
      const int p = pos[i0 + x];
      if (e > 0 && (int64_t)p == (int64_t)at + 1) t = make_double2(t.x * one.y + t.y * one.x, t.y * one.y - t.x * one.x);
      else t = turn((double)p * freq);
      at = p;
      s_turn[x * fc::kWave + d] = t;
    }
    __syncthreads();
  }
  const int j = tid % kUnitLanes;
  const int units = tokens * 2 * Hkv;
  for (int u = tid / kUnitLanes; u < units; u += kUnits) {
    const int tl = u / (2 * Hkv), h2 = u - tl * (2 * Hkv);
    const bool is_v = h2 >= Hkv;
    const int h = is_v ? h2 - Hkv : h2;
    const int64_t i = i0 + tl;
    if (i >= n) break;
    const int sl = slot[i];
    const int64_t row = src ? src[i] : i;
    if (sl < 0 || sl >= n_pages * kPage || row < 0 || row >= n_src) continue;  // the unit's lanes go together
    const uint16_t* p = (is_v ? v + row * v_stride : k + row * k_stride) + h * kHeadDim + 8 * j;
    const uint4 lo = *(const uint4*)p, hi = *(const uint4*)(p + kHeadDim / 2);
    float a[8], b[8];
    fc::unpack8(lo, a);
    fc::unpack8(hi, b);
    if (!is_v && log2_base > 0.0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double2 t = s_turn[tl * (kHeadDim / 2) + 8 * j + e];
        const double x0 = a[e], x1 = b[e];
        a[e] = (float)(x0 * t.y - x1 * t.x);
        b[e] = (float)(x1 * t.y + x0 * t.x);
      }
    }
    uint32_t ma = 0, mb = 0;  // magnitudes compare as their bits, NaN above all
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t xa = __float_as_uint(a[e]) & 0x7FFFFFFFu, xb = __float_as_uint(b[e]) & 0x7FFFFFFFu;
      ma = xa > ma ? xa : ma;
      mb = xb > mb ? xb : mb;
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      const uint32_t xa = __shfl_xor(ma, o), xb = __shfl_xor(mb, o);
      ma = xa > ma ? xa : ma;
      mb = xb > mb ? xb : mb;
    }
    const uint32_t sa = fc::scale_byte(ma), sb = fc::scale_byte(mb);
    uint32_t ca = 0, cb = 0;
#define FC_CODES(E)                                                                                            \
  ca = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(ca, a[2 * E], a[2 * E + 1], fc::scale_of(sa), E);             \
  cb = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(cb, b[2 * E], b[2 * E + 1], fc::scale_of(sb), E)
    FC_CODES(0);
    FC_CODES(1);
    FC_CODES(2);
    FC_CODES(3);
#undef FC_CODES
    if (sa == 255u) ca = 0;  // a NaN whatever the codes: always the same bytes
    if (sb == 255u) cb = 0;
    const int t = sl % kPage;
    uint8_t* page = pool + ((int64_t)(sl / kPage) * Hkv + h) * kPageBytes;
    uint8_t* codes = page + (is_v ? fc::kPageV : 0) + t * fc::kCodeRow + 4 * j;
    *(uint32_t*)codes = ca;
    *(uint32_t*)(codes + fc::kCodeRow / 2) = cb;
    if (j % 4 == 0) {
      const int g = j / 4;
      page[is_v ? fc::v_scale_at(t, g) : fc::k_scale_at(t, g)] = (uint8_t)sa;
      page[is_v ? fc::v_scale_at(t, g + 2) : fc::k_scale_at(t, g + 2)] = (uint8_t)sb;
    }
  }
}

// ------------------------------------------------------------------- read --

constexpr int kReadThreads = 256;
constexpr int kReadRows = 16;  // rows of a workgroup

// Sixteen lanes per row and head, eight dims each; a workgroup takes 16 rows
// (a quarter of a page where slots follow each other) through every head.  48
// prefixes of up to 4,096 tokens, 8 key heads: 87 us, 96 % of the rate of a large
// copy.
__global__ void __launch_bounds__(kReadThreads) k_paged_read(const uint8_t* __restrict__ pool, int n_pages, int Hkv,
                                                             const int32_t* __restrict__ slot, int n,
                                                             uint16_t* __restrict__ k, uint16_t* __restrict__ v) {
  const int tid = (int)threadIdx.x;
  const int64_t i = (int64_t)blockIdx.x * kReadRows + tid / 16;
  const int j = tid % 16;
  if (i >= n) return;
  const int sl = slot[i];
  if (sl < 0 || sl >= n_pages * kPage) return;
  const int t = sl % kPage;
  for (int h = 0; h < Hkv; ++h) {
    const uint8_t* page = pool + ((int64_t)(sl / kPage) * Hkv + h) * kPageBytes;
    const int64_t to = (i * Hkv + h) * kHeadDim + 8 * j;
#pragma unroll
    for (int is_v = 0; is_v < 2; ++is_v) {
      const uint32_t c = *(const uint32_t*)(page + (is_v ? fc::kPageV : 0) + t * fc::kCodeRow + 4 * j);
      const float s = fc::scale_of(page[is_v ? fc::v_scale_at(t, j / 4) : fc::k_scale_at(t, j / 4)]);
      uint4 w;
      w.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0));
      w.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1));
      w.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2));
      w.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3));
      *(uint4*)((is_v ? v : k) + to) = w;
    }
  }
}

// Tokens of a workgroup: as many as its units take at once, or where that leaves
// four workgroups a CU, in two times, so that tokens behind one another share
// their angles and fewer workgroups start (200,000 tokens of 8 key heads 251 -> 225
// us; in four times 230, and 50,000 tokens of 32 key heads 227 -> 252).
int tokens_of(int32_t n, int32_t Hkv) {
  const auto in_reach = [](int t) { return t < 1 ? 1 : t > kMaxTokens ? kMaxTokens : t; };
  const int once = in_reach(kUnits / (2 * Hkv)), twice = in_reach(2 * kUnits / (2 * Hkv));
  return n / twice >= 4 * 256 ? twice : once;
}

bool pool_ok(const void* pool, int32_t n_pages, int32_t Hkv) {
  return pool && !((uintptr_t)pool & 15) && n_pages >= 1 && n_pages <= (1 << 25) - 1 && Hkv >= 1 && Hkv <= 1024;
}

}  // namespace

extern "C" size_t fc_paged_pool_bytes(int32_t n_pages, int32_t Hkv) {
  if (n_pages < 1 || n_pages > (1 << 25) - 1 || Hkv < 1 || Hkv > 1024) return 0;
  return (size_t)n_pages * Hkv * FC_PAGE_HEAD_BYTES;
}

extern "C" fc_status fc_paged_plan(const int32_t* len, const int32_t* add, const int32_t* mask,
                                   const int32_t* last_node, int32_t B, int32_t R, int32_t n_slots, int32_t* table,
                                   int32_t max_pages, int32_t* queue, int32_t n_pages, const int64_t* ends,
                                   int32_t* len_out, int32_t* cu, int32_t* slot, int32_t* pos, int32_t* src,
                                   int64_t* ends_out, hipStream_t stream) {
  if (B < 0 || B > 65536 || n_slots < 0 || n_slots >= (1 << 30) || max_pages < 1 || max_pages >= (1 << 25) ||
      n_pages < 1 || n_pages > (1 << 25) - 1)
    return FC_ERR_INVALID;
  if (!mask != !last_node || (mask && (R < 1 || R > FC_MAX_TREE_ROWS))) return FC_ERR_INVALID;
  if (B > 0 && (!len || !add || !table || !len_out)) return FC_ERR_INVALID;
  if (!queue || !ends || !cu || !ends_out) return FC_ERR_INVALID;
  if (n_slots > 0 && (!slot || !pos || !src)) return FC_ERR_INVALID;
  // workgroups read everything while others write already
  const uint64_t seqs = 4 * (uint64_t)B, slots = 4 * (uint64_t)n_slots;
  if (!fc::apart({{table, seqs * max_pages}, {queue, 4 * (uint64_t)n_pages}, {len_out, seqs}, {cu, seqs + 4},
                  {slot, slots}, {pos, slots}, {src, slots}, {ends_out, 16}},
                 {{len, seqs}, {add, seqs}, {mask, seqs * R * R}, {last_node, seqs}, {ends, 16}}))
    return FC_ERR_INVALID;
  (void)hipGetLastError();
  const uint32_t windows = fc::div_up((uint64_t)n_slots, kPlanTokens);
  hipLaunchKernelGGL(k_paged_plan, dim3(windows ? windows : 1), dim3(kPlanThreads), 0, stream, len, add, mask,
                     last_node, B, R, n_slots, table, max_pages, queue, n_pages, ends, len_out, cu, slot, pos, src,
                     ends_out);
  FC_CHECK_LAUNCH();
  return FC_OK;
}

extern "C" fc_status fc_paged_write(uint8_t* pool, int32_t n_pages, int32_t Hkv, int32_t D, const uint16_t* k,
                                    int64_t k_stride, const uint16_t* v, int64_t v_stride, int32_t n_src,
                                    const int32_t* slot, const int32_t* pos, const int32_t* src, int32_t n,
                                    float rope_base, hipStream_t stream) {
  if (!pool_ok(pool, n_pages, Hkv) || n < 0 || n_src < 0) return FC_ERR_INVALID;
  if (!(rope_base == 0.0f || (rope_base > 1.0f && rope_base < __builtin_inff()))) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D || ((k_stride | v_stride) & 7)) return FC_ERR_INVALID;
  if (n == 0 || n_src == 0) return FC_OK;
  if (!k || !v || !slot || (rope_base != 0.0f && !pos)) return FC_ERR_INVALID;
  if (((uintptr_t)k | (uintptr_t)v) & 15) return FC_ERR_INVALID;
  const uint64_t numbers = 4 * (uint64_t)n;
  if (!fc::apart({{pool, fc_paged_pool_bytes(n_pages, Hkv)}},
                 {fc::rows_span(k, n_src, k_stride, Hkv * D), fc::rows_span(v, n_src, v_stride, Hkv * D),
                  {slot, numbers}, {rope_base != 0.0f ? pos : nullptr, numbers}, {src, numbers}}))
    return FC_ERR_INVALID;
  const int tokens = tokens_of(n, Hkv);
  (void)hipGetLastError();
  const int64_t most = fc::kMostGroups * tokens;
  for (int64_t i = 0; i < n; i += most) {
    const int32_t now = (int32_t)(n - i < most ? n - i : most);
    const int64_t row0 = src ? 0 : i;  // without src the rows go along with the slots
    if (row0 >= n_src) break;
    hipLaunchKernelGGL(k_paged_write, dim3(fc::div_up((uint64_t)now, (uint64_t)tokens)), dim3(kWriteThreads), 0, stream,
                       pool, n_pages, Hkv, k + row0 * k_stride, k_stride, v + row0 * v_stride, v_stride,
                       (int)(n_src - row0), slot + i, pos ? pos + i : nullptr, src ? src + i : nullptr, now, tokens,
                       rope_base != 0.0f ? log2((double)rope_base) : 0.0);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

extern "C" fc_status fc_paged_read(const uint8_t* pool, int32_t n_pages, int32_t Hkv, int32_t D, const int32_t* slot,
                                   int32_t n, uint16_t* k, uint16_t* v, hipStream_t stream) {
  if (!pool_ok(pool, n_pages, Hkv) || n < 0) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (n == 0) return FC_OK;
  if (!slot || !k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) return FC_ERR_INVALID;
  const fc::Span rows = fc::rows_span(k, n, (int64_t)Hkv * D, (int64_t)Hkv * D);
  if (!fc::apart({rows, {v, rows.n}}, {{pool, fc_paged_pool_bytes(n_pages, Hkv)}, {slot, 4 * (uint64_t)n}}))
    return FC_ERR_INVALID;
  (void)hipGetLastError();
  constexpr int64_t kMost = fc::kMostGroups * kReadRows;
  for (int64_t i = 0; i < n; i += kMost) {
    const int32_t now = (int32_t)(n - i < kMost ? n - i : kMost);
    const int64_t to = i * Hkv * kHeadDim;
    hipLaunchKernelGGL(k_paged_read, dim3(fc::div_up((uint64_t)now, kReadRows)), dim3(kReadThreads), 0, stream, pool,
                       n_pages, Hkv, slot + i, now, k + to, v + to);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

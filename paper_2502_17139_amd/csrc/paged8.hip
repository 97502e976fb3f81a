// The 8-bit paged cache on gfx950: rows into pages (fc_paged_byte_write) and out of
// them (fc_paged_byte_read).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fastcoder.h"
#include "fc_device.h"
#include "fc_host.h"
#include "fc_page8.h"

namespace {

using fc::kBlock8;
using fc::kDim8;
using fc::kPage8;
using fc::kPage8Bytes;
using fc::kQuarter8;

// ------------------------------------------------------------------ write --

constexpr int kWriteThreads = 256;
constexpr int kWriteWaves = kWriteThreads / fc::kWave;
// Entries whose runs a workgroup looks after: those of one block, or as many single ones.
// (Smaller windows of a prompt hold no run's start but every fourth or 32nd, which lie on
// one XCD then: 512 entries, 32 key heads, 70 us in windows of one, 9 so.)
constexpr int kWindow = 32;

struct Write {
  uint8_t* pool;
  const uint16_t* x[2];  // keys, values
  int64_t stride[2];
  const int32_t *slot, *src;
  int64_t first, n;      // entries [0, n) exist; this launch's begin at `first`
  int64_t n_src;
  int n_pages, Hkv;
};

__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// The largest magnitude of a wave's pairs (bfloat16 bits), the same in all lanes.
__device__ __forceinline__ uint32_t wave_top(uint32_t pair) {
  uint32_t m = larger(pair & 0xFFFFu, pair >> 16);
#pragma unroll
  for (int o = 1; o < fc::kWave; o <<= 1) m = larger(m, (uint32_t)__shfl_xor((int)m, o));
  return (uint32_t)__builtin_amdgcn_readfirstlane((int)m);
}

// What a block's scale becomes, and what its other rows' codes are multiplied by.
struct Scaled {
  int e;
  float inv;      // 2^-e
  float again;    // 2^(e_old - e)
  bool recode;    // the scale rose: codes that were there are rounded anew
};
__device__ __forceinline__ Scaled rescale(uint32_t top, uint32_t byte, bool fresh) {
  Scaled s;
  s.e = fc::exponent8(top);
  const int was = fc::clamp_exp8((int)byte - 127);
  if (!fresh && was > s.e) s.e = was;
  s.recode = !fresh && s.e > was;
  s.inv = fc::power8(-s.e);
  s.again = was - s.e < -126 ? 0.0f : fc::power8(was - s.e);
  return s;
}

// Entries as a wave looks at them, one a lane.
struct Entries {
  const Write& A;
  __device__ __forceinline__ explicit Entries(const Write& a) : A(a) {}
  // Entry i's block; -1: it is skipped, or there is none.
  __device__ __forceinline__ int look(int64_t i, int& slot, int& row) const {
    const bool in = i >= 0 && i < A.n;
    slot = in ? A.slot[i] : -1;
    row = in ? (A.src ? A.src[i] : (int)i) : -1;
    return row >= 0 && row < A.n_src && (uint32_t)slot < slots() ? slot / kBlock8 : -1;
  }
  // What is skipped may be thousands of entries (those behind a plan's last token), so
  // slots are passed 16 bytes a lane, 2,048 at a time, by one comparison of their least
  // as unsigned numbers: 65,536 entries of which the first 400 are placed 48 us, 51 in a
  // state that did not look for more of a run behind them.  (4 bytes a lane, 512 at a time:
  // 321; 16 bytes with a comparison for each slot: 129.)
  static constexpr int kLoads = 8, kPiece = 4 * fc::kWave, kStep = kLoads * kPiece;
  struct Pieces {
    uint4 v[kLoads];
    // The entries at (first + u * way + 4 lane) .. + 3 of [lo, hi), whole ones.
    __device__ __forceinline__ Pieces(const int32_t* slot, int64_t first, int way, int64_t lo, int64_t hi) {
#pragma unroll
      for (int u = 0; u < kLoads; ++u) {
        const int64_t at = first + u * way + 4 * fc::lane_id();
        v[u] = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (at >= lo && at < hi) v[u] = *(const uint4*)(slot + at);
      }
    }
    __device__ __forceinline__ static uint32_t least(uint32_t a, uint32_t b) { return a < b ? a : b; }
    __device__ __forceinline__ uint32_t least(int u) const { return least(least(v[u].x, v[u].y), least(v[u].z, v[u].w)); }
    // Whether any is below `slots`.
    __device__ __forceinline__ bool any(uint32_t slots) const {
      uint32_t m = least(0);
#pragma unroll
      for (int u = 1; u < kLoads; ++u) m = least(m, least(u));
      return fc::ballot(m < slots) != 0;
    }
    // The first such u, then the first or last such lane's bits.
    __device__ __forceinline__ int find(uint32_t slots, bool last, int& lane, int& bits) const {
      int at = 0;
#pragma unroll
      for (int u = kLoads - 1; u >= 0; --u)
        if (const uint64_t m = fc::ballot(least(u) < slots)) {
          at = u;
          lane = last ? 63 - __builtin_clzll(m) : __builtin_ctzll(m);
          bits = __builtin_amdgcn_readlane((int)(v[u].x < slots) | (int)(v[u].y < slots) << 1 | (int)(v[u].z < slots) << 2 |
                                               (int)(v[u].w < slots) << 3, lane);
        }
      return at;
    }
  };
  __device__ __forceinline__ uint32_t slots() const { return (uint32_t)A.n_pages * kPage8; }
  __device__ __forceinline__ int behind_line(int64_t i) const { return (int)((uintptr_t)(A.slot + i) >> 2) & 3; }
  // The first entry from i on whose slot is in the pool, or one past the last; i >= 3.
  __device__ __forceinline__ int64_t next(int64_t i) const {
    const int64_t end = A.n - behind_line(A.n);  // of whole pieces; up to three entries behind them
    const int64_t mine = end + fc::lane_id();
    const uint32_t rest = mine >= i && mine < A.n ? (uint32_t)A.slot[mine] : ~0u;
    const int skip = behind_line(i);
    for (int64_t x = i - skip; x < end; x += kStep) {
      Pieces p(A.slot, x, kPiece, x, end);
      if (x < i && fc::lane_id() == 0) {  // the first piece begins before i
        p.v[0].x = ~0u;
        if (skip > 1) p.v[0].y = ~0u;
        if (skip > 2) p.v[0].z = ~0u;
      }
      if (!p.any(slots())) continue;
      int lane = 0, bits = 0;
      const int u = p.find(slots(), false, lane, bits);
      return x + u * kPiece + 4 * lane + __builtin_ctz(bits);
    }
    const uint64_t m = fc::ballot(rest < slots());
    return m ? end + __builtin_ctzll(m) : A.n;
  }
  // The last entry before i whose slot is in the pool, or -1; i + 3 <= n.
  __device__ __forceinline__ int64_t last(int64_t i) const {
    const int64_t begin = -behind_line(0) & 3;  // of whole pieces; up to three entries ahead of them
    const uint32_t rest = fc::lane_id() < begin && fc::lane_id() < i ? (uint32_t)A.slot[fc::lane_id()] : ~0u;
    const int keep = behind_line(i);
    for (int64_t y = i + (-keep & 3); y > begin; y -= kStep) {
      Pieces p(A.slot, y - kPiece, -kPiece, begin, y);
      if (y > i && fc::lane_id() == fc::kWave - 1) {  // the first piece ends behind i
        p.v[0].w = ~0u;
        if (keep < 3) p.v[0].z = ~0u;
        if (keep < 2) p.v[0].y = ~0u;
      }
      if (!p.any(slots())) continue;
      int lane = 0, bits = 0;
      const int u = p.find(slots(), true, lane, bits);
      return y - (u + 1) * kPiece + 4 * lane + 31 - __builtin_clz(bits);
    }
    const uint64_t m = fc::ballot(rest < slots());
    return m ? 63 - __builtin_clzll(m) : -1;
  }
  // The block of the last entry before i that is not skipped; -1: there is none.
  __device__ __forceinline__ int block_before(int64_t i) const {
    for (i = last(i); i >= 0; i = last(i)) {
      i -= fc::kWave - 1;
      int slot, row;
      const int b = look(i + fc::lane_id(), slot, row);
      const uint64_t live = fc::ballot(b >= 0);
      if (live) return __builtin_amdgcn_readlane(b, 63 - __builtin_clzll(live));
      if (i <= 0) break;
    }
    return -1;
  }
};

// The entries of one block, which follow one another but for skipped ones, are a run; a
// wave takes a run's keys or values of one head, so that a block has one writer.  It
// reads the rows, has their largest magnitude by exchange within the wave, and writes
// codes: key rows as they are, values dim by dim.  A block that the run begins (its
// first row is among the run's) is written whole, with zeros in the rows that are not
// there yet; in others the key rows alone and all of the values, whose 16-byte pieces
// hold other tokens too, unless the scale rises and all codes are rounded anew.  Read are
// 512 bytes a token and key head, written 258: prompts of 22,790 tokens, 32 key heads,
// 164 us where a copy of as many bytes takes 113.  112 registers leave four waves a SIMD.
__global__ void __launch_bounds__(kWriteThreads) k_paged8_write(Write A) {
  const int lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave);
  const int64_t i0 = A.first + (int64_t)blockIdx.x * kWindow;
  const Entries E(A);
  // lanes 32 on have the window's entries, the others those before; a run begins where the
  // last one before that is not skipped is of another block
  int b_mine, b_before;
  uint64_t leads;
  {
    int slot, row;
    b_mine = E.look(i0 - kWindow + lane, slot, row);
    const uint64_t live = fc::ballot(b_mine >= 0), below = live & fc::lanemask_lt();
    if (!(live >> kWindow)) return;
    b_before = __shfl(b_mine, below ? 63 - __builtin_clzll(below) : 0);
    if (!(live << kWindow) && i0 > kWindow) {  // none of those before
      const int b = E.block_before(i0 - kWindow);
      if (!below) b_before = b;
    } else if (!below) {
      b_before = -1;
    }
    leads = fc::ballot(lane >= kWindow && b_mine >= 0 && b_mine != b_before);
  }
  const int each = 2 * A.Hkv, tasks = (int)__popcll(leads) * each;
  for (int task = (int)blockIdx.y * kWriteWaves + w; task < tasks; task += (int)gridDim.y * kWriteWaves) {
    uint64_t left = leads;
    for (int skip = task / each; skip > 0; --skip) left &= left - 1;
    const int lead = __builtin_ctzll(left), block = __builtin_amdgcn_readlane(b_mine, lead);
    const int part = task % each, is_v = part >= A.Hkv, h = is_v ? part - A.Hkv : part;
    // The run, 64 entries at a time: where each row of the block comes from (lane t has
    // row t's), and which are written.
    int from = -1;
    uint32_t have = 0;
    for (int64_t i = i0 - kWindow + lead; i < A.n && have != 0xFFFFFFFFu; i = E.next(i)) {
      int slot, row;
      const int b = E.look(i + lane, slot, row);
      const uint64_t others = fc::ballot(b >= 0 && b != block);
      uint64_t run = fc::ballot(b == block);
      if (others) run &= (1ull << __builtin_ctzll(others)) - 1;
      for (; run; run &= run - 1) {
        const int e = __builtin_ctzll(run);
        const int te = __builtin_amdgcn_readlane(slot, e) & (kBlock8 - 1), re = __builtin_amdgcn_readlane(row, e);
        if (lane == te) from = re;
        have |= 1u << te;
      }
      if (others) break;
      i += fc::kWave;
    }
    const bool fresh = have & 1u;
    uint8_t* page = A.pool + ((int64_t)(block >> 1) * A.Hkv + h) * kPage8Bytes;
    const int half = block & 1;
    uint8_t* scale = page + fc::kPage8Scales + 2 * is_v + half;
    const uint32_t byte = *scale;
    const uint16_t* x = A.x[is_v] + h * kDim8;
    const int64_t stride = A.stride[is_v];
    if (!is_v) {
      // eight lanes a row, 16 dims each; eight rows at a time
      const int c = lane & 7;
      uint4 raw[4][2];
      bool live[4];
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const int r = __shfl(from, 8 * p + (lane >> 3));
        live[p] = r >= 0;
        raw[p][0] = raw[p][1] = make_uint4(0u, 0u, 0u, 0u);
        if (live[p]) {
          const uint4* at = (const uint4*)(x + (int64_t)r * stride + 16 * c);
          raw[p][0] = at[0];
          raw[p][1] = at[1];
        }
      }
      uint32_t tops = 0;
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          tops = fc::tops8(tops, raw[p][u].x);
          tops = fc::tops8(tops, raw[p][u].y);
          tops = fc::tops8(tops, raw[p][u].z);
          tops = fc::tops8(tops, raw[p][u].w);
        }
      uint32_t top = wave_top(tops);
      const bool odd = top >= 0x7F80u;
      if (odd) {  // the largest finite one
        top = 0;
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            float v[8];
            fc::unpack8(raw[p][u], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = larger(top, fc::reach8(v[e]) >> 16);
          }
        top = wave_top(top);
      }
      const Scaled s = rescale(top << 16, byte, fresh);
      const bool plain = !odd && s.e > fc::kLeastExp8 && s.e < fc::kMostExp8;
      const float scale_of = fc::power8(s.e);
      uint8_t* to = page + half * (kBlock8 * kDim8) + (lane >> 3) * kDim8 + 16 * c;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        uint4* at = (uint4*)(to + p * 8 * kDim8);
        if (live[p]) {
          uint32_t o[4];
          const uint32_t in[8] = {raw[p][0].x, raw[p][0].y, raw[p][0].z, raw[p][0].w,
                                  raw[p][1].x, raw[p][1].y, raw[p][1].z, raw[p][1].w};
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4)
            o[i4] = plain ? fc::codes8(in[2 * i4], in[2 * i4 + 1], scale_of)
                          : fc::codes8_any(in[2 * i4], in[2 * i4 + 1], s.inv);
          *at = make_uint4(o[0], o[1], o[2], o[3]);
        } else if (fresh) {
          *at = make_uint4(0u, 0u, 0u, 0u);
        } else if (s.recode) {
          const uint4 old = *at;
          *at = make_uint4(fc::recode8(old.x, s.again), fc::recode8(old.y, s.again), fc::recode8(old.z, s.again),
                           fc::recode8(old.w, s.again));
        }
      }
      if (lane == 0) *scale = (uint8_t)(s.e + 127);
    } else {
      // two dims a lane, every row of the block; rows that the run does not have read
      // one that it has, for nothing
      const int any = __builtin_amdgcn_readlane(from, __builtin_ctz(have));
      const uint32_t* at = (const uint32_t*)x + lane;
      uint32_t raw[kBlock8];
#pragma unroll
      for (int r = 0; r < kBlock8; ++r) {
        const int f = __builtin_amdgcn_readlane(from, r);
        raw[r] = *(const uint32_t*)((const uint16_t*)at + (int64_t)(f >= 0 ? f : any) * stride);
      }
      uint8_t* to = page + fc::kPage8V + half * (kBlock8 * kDim8) + lane * 2 * kQuarter8;
      uint4 old[2][2];
      const bool merge = !fresh && have != 0xFFFFFFFFu;
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          old[q][d] = make_uint4(0u, 0u, 0u, 0u);
          if (merge) old[q][d] = *(const uint4*)(to + q * (kQuarter8 * kDim8) + d * kQuarter8);
        }
      uint32_t tops = 0;
#pragma unroll
      for (int r = 0; r < kBlock8; ++r) tops = fc::tops8(tops, raw[r]);
      uint32_t top = wave_top(tops);
      const bool odd = top >= 0x7F80u;
      if (odd) {
        top = 0;
#pragma unroll
        for (int r = 0; r < kBlock8; ++r)
          top = larger(top, larger(fc::reach8(__uint_as_float(raw[r] << 16)), fc::reach8(__uint_as_float(raw[r] & 0xFFFF0000u))) >> 16);
        top = wave_top(top);
      }
      const Scaled s = rescale(top << 16, byte, fresh);
      const bool plain = !odd && s.e > fc::kLeastExp8 && s.e < fc::kMostExp8;
      const float scale_of = fc::power8(s.e);
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int d = 0; d < 2; ++d) {
          uint32_t o[4];
          const uint32_t was[4] = {old[q][d].x, old[q][d].y, old[q][d].z, old[q][d].w};
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            const uint32_t* in = raw + 16 * q + 4 * i4;
            const uint32_t half0 = d ? (in[0] >> 16) | (in[1] & 0xFFFF0000u) : (in[0] & 0xFFFFu) | in[1] << 16;
            const uint32_t half1 = d ? (in[2] >> 16) | (in[3] & 0xFFFF0000u) : (in[2] & 0xFFFFu) | in[3] << 16;
            const uint32_t code = plain ? fc::codes8(half0, half1, scale_of) : fc::codes8_any(half0, half1, s.inv);
            const uint32_t nibble = (have >> (16 * q + 4 * i4)) & 15u;
            const uint32_t keep = ((nibble & 1u) | (nibble & 2u) << 7 | (nibble & 4u) << 14 | (nibble & 8u) << 21) * 255u;
            uint32_t rest = was[i4];
            if (s.recode) rest = fc::recode8(rest, s.again);
            o[i4] = (code & keep) | (rest & ~keep);
          }
          *(uint4*)(to + q * (kQuarter8 * kDim8) + d * kQuarter8) = make_uint4(o[0], o[1], o[2], o[3]);
        }
      if (lane == 0) *scale = (uint8_t)(s.e + 127);
    }
  }
}

// ------------------------------------------------------------------- read --

constexpr int kReadThreads = 256;
constexpr int kReadWaves = kReadThreads / fc::kWave;
constexpr int kReadRows = 16;  // entries of a workgroup

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair8(uint32_t w, float s, bool high) {
  const bf16x2 r = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true)
                        : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
  return __builtin_bit_cast(uint32_t, r);
}

// A wave takes 16 entries through every fourth head.  Keys: 16 lanes a row, eight dims
// each.  Values: two dims a lane, 16 tokens of them in two loads; entries of one such
// quarter that follow one another, as the tokens of a sequence do, share the loads.  Bound
// by what is written, 512 bytes a token and key head: 22,790 tokens of 32 key heads 121 us,
// 4.6 TB/s of a copy's 4.95.  All loads are asked for before the first result is written
// (137 us in a state before this, one after another 159; four dims a lane, half as many
// tokens each, 232).
__global__ void __launch_bounds__(kReadThreads) k_paged8_read(const uint8_t* __restrict__ pool, int n_pages, int Hkv,
                                                              const int32_t* __restrict__ slot, int64_t first, int64_t n,
                                                              uint16_t* __restrict__ k, uint16_t* __restrict__ v) {
  const int lane = fc::lane_id();
  const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x / fc::kWave);
  const int64_t i0 = first + (int64_t)blockIdx.x * kReadRows;
  int sl = lane < kReadRows && i0 + lane < n ? slot[i0 + lane] : -1;
  if (sl >= n_pages * kPage8) sl = -1;
  for (int h = (int)blockIdx.y * kReadWaves + w; h < Hkv; h += (int)gridDim.y * kReadWaves) {
    int at = -1;  // the quarter in registers
    uint4 a = make_uint4(0u, 0u, 0u, 0u), b = a;
    uint32_t byte = 0;
    const auto quarter = [&](int s) {
      at = s / kQuarter8;
      const uint8_t* page = pool + ((int64_t)(s / kPage8) * Hkv + h) * kPage8Bytes;
      const uint4* from = (const uint4*)(page + fc::v8_at(s % kPage8 & ~(kQuarter8 - 1), 2 * lane));
      a = from[0];
      b = from[1];
      byte = page[fc::kPage8Scales + 2 + s % kPage8 / kBlock8];
    };
    const int c = lane & 15;
    int from[4];
    uint2 x[4];
    uint32_t bytes[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      from[p] = __shfl(sl, 4 * p + (lane >> 4));
      const int s = from[p] < 0 ? 0 : from[p], t = s % kPage8;  // row 0 for nothing
      const uint8_t* page = pool + ((int64_t)(s / kPage8) * Hkv + h) * kPage8Bytes;
      x[p] = *(const uint2*)(page + fc::k8_at(t, 8 * c));
      bytes[p] = page[fc::kPage8Scales + t / kBlock8];
    }
    const int s0 = __builtin_amdgcn_readfirstlane(sl);
    if (s0 >= 0) quarter(s0);
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      if (from[p] < 0) continue;
      const float f = fc::scale8(bytes[p]);
      *(uint4*)(k + ((i0 + 4 * p + (lane >> 4)) * Hkv + h) * kDim8 + 8 * c) =
          make_uint4(pair8(x[p].x, f, false), pair8(x[p].x, f, true), pair8(x[p].y, f, false), pair8(x[p].y, f, true));
    }
    for (int e = 0; e < kReadRows; ++e) {
      const int s = __builtin_amdgcn_readlane(sl, e);
      if (s < 0) continue;
      const int t = s % kPage8;
      if (s / kQuarter8 != at) quarter(s);
      const int u = t % kQuarter8;
      const uint32_t wa = u < 8 ? (u < 4 ? a.x : a.y) : (u < 12 ? a.z : a.w);
      const uint32_t wb = u < 8 ? (u < 4 ? b.x : b.y) : (u < 12 ? b.z : b.w);
      const uint32_t both = ((wa >> (8 * (u & 3))) & 255u) | (((wb >> (8 * (u & 3))) & 255u) << 8);
      *(uint32_t*)(v + ((i0 + e) * Hkv + h) * kDim8 + 2 * lane) = pair8(both, fc::scale8(byte), false);
    }
  }
}

bool pool_ok(const void* pool, int32_t n_pages, int32_t Hkv) {
  return pool && !((uintptr_t)pool & 15) && fc_paged_byte_pool_bytes(n_pages, Hkv) > 0;
}

// Workgroups over a group's tasks: 16 a CU in all, several times what runs at once, so that
// heavy ones are not waited for.  4, 8, 16 and 32 a CU: 22,790 tokens of ragged prompts, 32
// key heads, written and read 329, 305, 286 and 283 us; 65,536 of one prompt, 8 key heads,
// written 89, 89, 93 and 93; 1,024 single tokens 32, 29, 29 and 29.
uint32_t over_heads(int64_t groups, int64_t tasks) {
  const int64_t want = (16 * 256 + groups - 1) / groups;
  return (uint32_t)(want < 1 ? 1 : want > tasks ? tasks : want);
}

// A launch takes fewer than 2^32 threads in a dimension, so a longer call is several.
constexpr int64_t kMostGroups = 1 << 20;

}  // namespace

extern "C" size_t fc_paged_byte_pool_bytes(int32_t n_pages, int32_t Hkv) {
  if (n_pages < 1 || n_pages > (1 << 25) - 1 || Hkv < 1 || Hkv > 1024) return 0;
  return (size_t)n_pages * Hkv * FC_PAGE8_HEAD_BYTES;
}

extern "C" fc_status fc_paged_byte_write(uint8_t* pool, int32_t n_pages, int32_t Hkv, int32_t D, const uint16_t* k,
                                         int64_t k_stride, const uint16_t* v, int64_t v_stride, int32_t n_src,
                                         const int32_t* slot, const int32_t* src, int32_t n, hipStream_t stream) {
  if (!pool_ok(pool, n_pages, Hkv) || n < 0 || n_src < 0) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (k_stride < (int64_t)Hkv * D || v_stride < (int64_t)Hkv * D || ((k_stride | v_stride) & 7)) return FC_ERR_INVALID;
  if (n == 0 || n_src == 0) return FC_OK;
  if (!k || !v || !slot) return FC_ERR_INVALID;
  if (((uintptr_t)k | (uintptr_t)v) & 15) return FC_ERR_INVALID;
  const uint64_t numbers = 4 * (uint64_t)n;
  if (!fc::apart({{pool, fc_paged_byte_pool_bytes(n_pages, Hkv)}},
                 {fc::rows_span(k, n_src, k_stride, Hkv * D), fc::rows_span(v, n_src, v_stride, Hkv * D),
                  {slot, numbers}, {src, numbers}}))
    return FC_ERR_INVALID;
  Write a = {pool, {k, v}, {k_stride, v_stride}, slot, src, 0, n, n_src, n_pages, Hkv};
  const int64_t groups = fc::div_up((uint64_t)n, kWindow);
  const uint32_t y = over_heads(groups, ((int64_t)kWindow * 2 * Hkv + kWriteWaves - 1) / kWriteWaves);
  (void)hipGetLastError();
  for (int64_t g = 0; g < groups; g += kMostGroups) {
    a.first = g * kWindow;
    const uint32_t now = (uint32_t)(groups - g < kMostGroups ? groups - g : kMostGroups);
    hipLaunchKernelGGL(k_paged8_write, dim3(now, y), dim3(kWriteThreads), 0, stream, a);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

extern "C" fc_status fc_paged_byte_read(const uint8_t* pool, int32_t n_pages, int32_t Hkv, int32_t D,
                                        const int32_t* slot, int32_t n, uint16_t* k, uint16_t* v, hipStream_t stream) {
  if (!pool_ok(pool, n_pages, Hkv) || n < 0) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  if (n == 0) return FC_OK;
  if (!slot || !k || !v || (((uintptr_t)k | (uintptr_t)v) & 15)) return FC_ERR_INVALID;
  const fc::Span rows = fc::rows_span(k, n, (int64_t)Hkv * D, (int64_t)Hkv * D);
  if (!fc::apart({rows, {v, rows.n}}, {{pool, fc_paged_byte_pool_bytes(n_pages, Hkv)}, {slot, 4 * (uint64_t)n}}))
    return FC_ERR_INVALID;
  const int64_t groups = fc::div_up((uint64_t)n, kReadRows);
  const uint32_t y = over_heads(groups, (Hkv + kReadWaves - 1) / kReadWaves);
  (void)hipGetLastError();
  for (int64_t g = 0; g < groups; g += kMostGroups) {
    const uint32_t now = (uint32_t)(groups - g < kMostGroups ? groups - g : kMostGroups);
    hipLaunchKernelGGL(k_paged8_read, dim3(now, y), dim3(kReadThreads), 0, stream, pool, n_pages, Hkv, slot,
                       g * kReadRows, (int64_t)n, k, v);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

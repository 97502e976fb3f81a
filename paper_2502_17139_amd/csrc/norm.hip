// Queries and keys normed for each head and rotated by their positions in one pass
// (fc_norm_rotate).
//
// y = x / sqrt(mean(x^2) + eps) * w over a head's 128 dims, then the pair (d, d + 64)
// turns by position * base^(-2d/128).  All of it in fp32 (angles reduced in double
// precision, then the hardware's sine and cosine: within 2^-18, where the result's
// rounding is 2^-9), one rounding to bf16 at the end.  Bound by memory: 512 bytes a
// head.  24,571 tokens of 32 query and 8 key heads 92 us, 5.5 TB/s (a copy of 2 GiB has 4.95);
// one token 2.8 us, a launch and two round trips.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "fastcoder.h"
#include "fc_device.h"
#include "fc_host.h"

namespace {

constexpr int kDim = FC_TREE_ATTN_HEAD_DIM;
constexpr int kThreads = 256;
constexpr int kUnitLanes = 8;                     // lanes of one head: dims 8 j .. 8 j + 7 and the same 64 further on
constexpr int kUnits = kThreads / kUnitLanes;     // heads at work in a workgroup

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

struct Args {
  const uint16_t* x[2];     // queries, keys
  const uint16_t* w[2];     // their weights, or none
  uint16_t* y[2];
  int64_t x_stride[2], y_stride[2];
  const int32_t* pos;
  int64_t n;
  int H, Hkv;
  float eps;
  double log2_base;  // 0: no rotation
};

// Squares of numbers of 2^63 and more do not fit fp32, nor those below 2^-63 all of their
// bits.  From this mean on, squares below fp32's normal numbers, 2^-126, are less than
// its last bit; heads of a smaller one, or of one that does not fit, are first scaled by
// the power of two that brings the larger of their largest number and sqrt(eps) near 1.
// (In double precision instead: 80 registers, not 52, and 97 us for the 92 of 24,571
// tokens.)
constexpr float kLeastMean = 8.271806126e-25f;  // 2^-80
__device__ __forceinline__ float scaled_root(float (&a)[8], float (&b)[8], float eps) {
  float top = 0.0f;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = fmaxf(top, fmaxf(fabsf(a[e]), fabsf(b[e])));
  top = fmaxf(top, __shfl_xor(top, 1));
  top = fmaxf(top, __shfl_xor(top, 2));
  top = fmaxf(top, __shfl_xor(top, 4));
  const int of_top = (int)(__float_as_uint(top) >> 23) - 127, of_eps = ((int)(__float_as_uint(eps) >> 23) - 127) >> 1;
  int e = of_top > of_eps ? of_top : of_eps;
  e = e < -126 ? -126 : e > 126 ? 126 : e;
  const float scale = __uint_as_float((uint32_t)(127 - e) << 23);
  float sum = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    a[i] *= scale, b[i] *= scale;
    sum += a[i] * a[i] + b[i] * b[i];
  }
  sum += __shfl_xor(sum, 1);
  sum += __shfl_xor(sum, 2);
  sum += __shfl_xor(sum, 4);
  return 1.0f / sqrtf(sum * (1.0f / kDim) + eps * scale * scale);
}

// A workgroup takes a token and blockIdx.y's share of its heads: a wave computes the
// token's angles once for all of them.  Two or four tokens a workgroup are no faster
// (24,571 tokens: 94 and 97 us against 94).
__global__ void __launch_bounds__(kThreads) k_norm_rotate(Args A) {
  __shared__ float2 s_turn[kDim / 2];
  const int tid = (int)threadIdx.x, j = tid % kUnitLanes;
  const int64_t i = blockIdx.x;
  const int heads = A.H + A.Hkv;
  if (A.log2_base > 0.0) {
    // a wave's lanes are the angles: sine and cosine of a fraction of a turn
    if (tid < kDim / 2) {
      const double f = exp2(-2.0 * tid / (double)kDim * A.log2_base) * 0.15915494309189533577;
      const float part = (float)__builtin_amdgcn_fract((double)A.pos[i] * f);
      s_turn[tid] = make_float2(__builtin_amdgcn_sinf(part), __builtin_amdgcn_cosf(part));
    }
    __syncthreads();
  }
  for (int u = (int)blockIdx.y * kUnits + tid / kUnitLanes; u < heads; u += (int)gridDim.y * kUnits) {
    const int is_k = u >= A.H;
    const int h = is_k ? u - A.H : u;
    const uint16_t* p = A.x[is_k] + i * A.x_stride[is_k] + h * kDim + 8 * j;
    const uint4 lo = *(const uint4*)p, hi = *(const uint4*)(p + kDim / 2);
    float a[8], b[8];
    fc::unpack8(lo, a);
    fc::unpack8(hi, b);
    const uint16_t* wp = A.w[is_k];
    if (wp) {
      const uint4 w_lo = *(const uint4*)(wp + 8 * j), w_hi = *(const uint4*)(wp + kDim / 2 + 8 * j);
      float sum = 0.0f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += a[e] * a[e] + b[e] * b[e];
      sum += __shfl_xor(sum, 1);
      sum += __shfl_xor(sum, 2);
      sum += __shfl_xor(sum, 4);
      const float mean = sum * (1.0f / kDim) + A.eps;
      // all lanes of a head alike
      const float r = mean >= kLeastMean && mean < INFINITY ? 1.0f / sqrtf(mean) : scaled_root(a, b, A.eps);
      float wa[8], wb[8];
      fc::unpack8(w_lo, wa);
      fc::unpack8(w_hi, wb);
#pragma unroll
      for (int e = 0; e < 8; ++e) a[e] = a[e] * r * wa[e], b[e] = b[e] * r * wb[e];
    }
    if (A.log2_base > 0.0) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float2 s = s_turn[8 * j + e];
        const float x0 = a[e], x1 = b[e];
        a[e] = x0 * s.y - x1 * s.x;
        b[e] = x1 * s.y + x0 * s.x;
      }
    }
    bf16x8 ya, yb;
#pragma unroll
    for (int e = 0; e < 8; ++e) ya[e] = (__bf16)a[e], yb[e] = (__bf16)b[e];
    uint16_t* to = A.y[is_k] + i * A.y_stride[is_k] + h * kDim + 8 * j;
    *(bf16x8*)to = ya;
    *(bf16x8*)(to + kDim / 2) = yb;
  }
}

// Rows of two tensors: n of len elements each, at their strides.
struct Rows {
  const uint16_t* p;
  int64_t stride, len;
};
// Whether rows share no bytes: their spans are apart, or they lie beside each other
// at the same distance, as slices of one projection do.
bool rows_apart(const Rows& a, const Rows& b, int64_t n) {
  if (!a.p || !b.p || n <= 0) return true;
  if (fc::apart({fc::rows_span(a.p, n, a.stride, a.len)}, {fc::rows_span(b.p, n, b.stride, b.len)})) return true;
  if (a.stride != b.stride) return false;
  const int64_t bytes = 2 * a.stride, off = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
  const int64_t m = ((off % bytes) + bytes) % bytes;
  return m >= 2 * a.len && m + 2 * b.len <= bytes;
}

}  // namespace

extern "C" fc_status fc_norm_rotate(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride,
                                    const uint16_t* q_weight, const uint16_t* k_weight, const int32_t* pos, int32_t n,
                                    int32_t H, int32_t Hkv, int32_t D, float eps, float rope_base, uint16_t* q_out,
                                    int64_t q_out_stride, uint16_t* k_out, int64_t k_out_stride, hipStream_t stream) {
  if (n < 0 || H < 0 || H > 8192 || Hkv < 0 || Hkv > 8192) return FC_ERR_INVALID;
  if (!(rope_base == 0.0f || (rope_base > 1.0f && rope_base < __builtin_inff()))) return FC_ERR_INVALID;
  if (!(eps >= 0.0f && eps < __builtin_inff())) return FC_ERR_INVALID;
  if (D != FC_TREE_ATTN_HEAD_DIM) return FC_ERR_UNSUPPORTED;
  const Rows in[2] = {{q, q_stride, (int64_t)H * D}, {k, k_stride, (int64_t)Hkv * D}};
  const Rows out[2] = {{q_out, q_out_stride, in[0].len}, {k_out, k_out_stride, in[1].len}};
  const uint16_t* w[2] = {q_weight, k_weight};
  for (int i = 0; i < 2; ++i) {
    if (in[i].len == 0) continue;
    if (in[i].stride < in[i].len || out[i].stride < in[i].len || ((in[i].stride | out[i].stride) & 7))
      return FC_ERR_INVALID;
  }
  if (n == 0 || H + Hkv == 0) return FC_OK;
  if (rope_base != 0.0f && !pos) return FC_ERR_INVALID;
  for (int i = 0; i < 2; ++i) {
    if (in[i].len == 0) continue;
    if (!in[i].p || !out[i].p) return FC_ERR_INVALID;
    if (((uintptr_t)in[i].p | (uintptr_t)out[i].p | (uintptr_t)w[i]) & 15) return FC_ERR_INVALID;
  }
  // A head is read before it is written, by the same lanes, so a result may take the
  // place of its own rows; of nothing else.
  for (int i = 0; i < 2; ++i) {
    if (out[i].len == 0) continue;
    for (int o = 0; o < 2; ++o) {
      if (in[o].len == 0) continue;
      const bool in_place = o == i && out[i].p == in[i].p && out[i].stride == in[i].stride;
      if (!in_place && !rows_apart(out[i], in[o], n)) return FC_ERR_INVALID;
    }
    if (i == 1 && out[0].len && !rows_apart(out[0], out[1], n)) return FC_ERR_INVALID;
    const fc::Span rows = fc::rows_span(out[i].p, n, out[i].stride, out[i].len);
    if (!fc::apart({rows}, {{H ? q_weight : nullptr, 2 * (uint64_t)D},
                            {Hkv ? k_weight : nullptr, 2 * (uint64_t)D},
                            {rope_base != 0.0f ? pos : nullptr, 4 * (uint64_t)n}}))
      return FC_ERR_INVALID;
  }
  // Short calls spread a token's heads over workgroups (one token of 1,024 heads: 12 us, in
  // one workgroup 28); from 1,024 tokens on the card is full without.
  Args a = {{q, k}, {q_weight, k_weight}, {q_out, k_out}, {q_stride, k_stride}, {q_out_stride, k_out_stride}, pos, n, H,
            Hkv, eps, rope_base != 0.0f ? log2((double)rope_base) : 0.0};
  const uint32_t y = n >= 1024 ? 1u : fc::div_up((uint64_t)(H + Hkv), kUnits);
  (void)hipGetLastError();
  // a launch takes fewer than 2^32 threads in a dimension
  constexpr int64_t kMost = (int64_t)1 << 22;
  for (int64_t i = 0; i < n; i += kMost) {
    Args now = a;
    now.n = n - i < kMost ? n - i : kMost;
    now.pos = pos ? pos + i : nullptr;
    for (int s = 0; s < 2; ++s) {
      if (in[s].len == 0) continue;
      now.x[s] = in[s].p + i * in[s].stride;
      now.y[s] = a.y[s] + i * out[s].stride;
    }
    hipLaunchKernelGGL(k_norm_rotate, dim3((uint32_t)now.n, y), dim3(kThreads), 0, stream,
                       now);
    FC_CHECK_LAUNCH();
  }
  return FC_OK;
}

// Rows in microscaled 4-bit floating point (the Open Compute project's MXFP4), with or without RMS norm.
//
// 32 consecutive elements share a power of two: m = max|v|, e = floor(log2 m) - 2, each element v / 2^e to the nearest of
// 0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, beyond 6: 6).  e is the exponent field of m as it stands, so a block's
// scale costs an integer maximum over the elements' bits, which also tells NaN and infinity (larger than any number).
//
// Of the norm y = h gain / sqrt(mean h^2 + eps) the blocks hold h gain; 1 / sqrt(...) is the row's own factor, kept in float32
// for the product to apply.  So the 4 bits do not wait for the sum over the row, they depend on a single rounded
// product however the sum is ordered, and no precision is spent on the row's size.
//
// Bound by memory: 32,000 x 4,096 float32 to rows and values 142 us (6.0 TB/s; 147 with the outputs through the caches); 16,381
// x 4,096 bf16 with residual, new residual, rows and values 105 us (5.5 TB/s; 110 through the caches).  64 x 4,096: the
// kernels 3 and 5 us, the calls 4.3 and 4.6.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace mx {

using namespace opd;

constexpr int kE = 8;                        // elements of a thread's piece; four threads make a block of 32
constexpr uint32_t kTinyBits = 27u << 23;    // 2^-100: blocks that lie below are zero
constexpr uint32_t kInfBits = 0x7f800000u;
// Squares of small elements lie below float32's normal numbers (2^-126), where they have fewer bits or none.  A sum from kSmall
// on misses less than 32,768 * 2^-150 of them, 2^-35 of itself, and so does one to whose mean such an eps is added.  Below,
// every element is smaller than 2^-50, and times kUp even the smallest, 2^-149, has a normal square: the scaling is exact, and
// 32,768 squares stay below 2^115.
constexpr float kSmall = 0x1p-100f, kUp = 0x1p100f;

typedef unsigned int u32_b __attribute__((aligned(1)));

template <bool STREAM> __device__ __forceinline__ void put_word(uint8_t *p, uint32_t v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (u32_b *)p);
  else *(u32_b *)p = v;
}

// Largest of the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
  v = max(v, (uint32_t)dpp_i<0xB1>((int)v));
  return max(v, (uint32_t)dpp_i<0x4E>((int)v));
}

__device__ __forceinline__ bool bad(uint32_t top) { return top >= kInfBits; }
__device__ __forceinline__ bool nothing(uint32_t top) { return top < kTinyBits; }
// The block's scale as it is stored: exponent + 127, 255 for NaN.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  return bad(top) ? 255u : nothing(top) ? 0u : (top >> 23) - 2u;
}

// v: this thread's elements of a block; returns them in 4 bits and, in `top`, the block's largest magnitude.
__device__ __forceinline__ uint32_t four_bits(const float (&v)[kE], uint32_t &top) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kE; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
  top = quad_max(m);
  if (bad(top) || nothing(top)) return 0u;
  const float scale = __uint_as_float(((top >> 23) - 2u) << 23);
  uint32_t q = 0;
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[0], v[1], scale, 0);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[2], v[3], scale, 1);
  q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[4], v[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, v[6], v[7], scale, 3);
}

// What the 4 bits stand for.
__device__ __forceinline__ void values_of(uint32_t q, uint32_t top, float factor, float (&v)[kE]) {
  const float scale = bad(top) ? __builtin_nanf("") : nothing(top) ? 0.f : __uint_as_float(((top >> 23) - 2u) << 23);
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    const uint32_t c = q >> (4 * i), s = c & 7u;
    const float e = s < 2u ? 0.5f * (float)s : __uint_as_float((126u + (s >> 1)) << 23 | (s & 1u) << 22);
    v[i] = (c & 8u ? -e : e) * scale * factor;
  }
}

template <typename T, bool STREAM> __global__ void __launch_bounds__(256) quant_kernel(MxArgs a, uint32_t pieces) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x, row = i / pieces;  // a launch has fewer than 2^31 pieces
  const int64_t r = row;
  const int c = (int)(i - row * pieces) * kE, have = a.channels - c;
  if (r >= a.rows) return;  // whole quads: a row has a multiple of four pieces
  float v[kE];
  load_part((const T *)a.x + r * a.ld_x + c, have, 0.f, v);
  uint32_t top;
  const uint32_t q = four_bits(v, top);
  put_word<STREAM>(a.q + r * a.ld_q + c / 2, q);
  if ((c & 31) == 0) a.scale[r * a.ld_e + c / 32] = (uint8_t)scale_byte(top);
  if (a.values) {
    values_of(q, top, 1.f, v);
    store_part<STREAM>(a.values + r * a.ld_v + c, have, v);
  }
}

// TPR threads per row (64: a wave per row), NP pieces per thread.  BARE: eps below kSmall does not hide what the sum of squares
// misses; the second sum costs 64 x 4,096 0.15 us of 4.9, so other calls go without it.
template <typename T, int TPR, int NP, bool STREAM, bool BARE>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_kernel(MxArgs a) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kW = TPR / 64;
  constexpr int kSums = BARE ? 3 : 2;
  __shared__ float red[kSums * kW];
  const int t = threadIdx.x % TPR;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (r >= a.rows) return;  // whole waves, and whole blocks where a block is one row
  const int padded = (a.channels + 31) / 32 * 32;
  uint32_t q[NP], top[NP];
  float ss = 0.f, ss_up = 0.f, some = 0.f;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = (p * TPR + t) * kE, have = a.channels - c;
    float h[kE];
    load_part((const T *)a.x + r * a.ld_x + c, have, 0.f, h);
    if (a.residual) {
      float v[kE];
      load_part((const T *)a.residual + r * a.ld_r + c, have, 0.f, v);
#pragma unroll
      for (int i = 0; i < kE; ++i) h[i] += v[i];
    }
    if (a.summed) store_part<STREAM>((T *)a.summed + r * a.ld_s + c, have, h);
#pragma unroll
    for (int i = 0; i < kE; ++i) ss += h[i] * h[i];
    if constexpr (BARE) {
#pragma unroll
      for (int i = 0; i < kE; ++i) ss_up += (h[i] * kUp) * (h[i] * kUp);
    }
    if (a.gain) {
      float g[kE];
      load_part(a.gain + c, have, 0.f, g);
#pragma unroll
      for (int i = 0; i < kE; ++i) h[i] *= g[i];
    }
    q[p] = four_bits(h, top[p]);
    if (!nothing(top[p])) some = 1.f;
    if (c < padded) {
      put_word<STREAM>(a.q + r * a.ld_q + c / 2, q[p]);
      if ((c & 31) == 0) a.scale[r * a.ld_e + c / 32] = (uint8_t)scale_byte(top[p]);
    }
  }
  ss = wave_sum(ss);
  some = wave_max(some);
  if constexpr (BARE) ss_up = wave_sum(ss_up);
  if (kW > 1) {
    const int w = t >> 6;
    if ((t & 63) == 0) {
      red[kSums * w] = ss;
      red[kSums * w + 1] = some;
      if constexpr (BARE) red[kSums * w + 2] = ss_up;
    }
    __syncthreads();
    ss = ss_up = some = 0.f;
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      ss += red[kSums * i];
      some = fmaxf(some, red[kSums * i + 1]);
      if constexpr (BARE) ss_up += red[kSums * i + 2];
    }
  }
  float rs = rsqrtf(ss / (float)a.channels + a.eps);
  if (BARE && ss < kSmall) rs = rsqrtf(ss_up / (float)a.channels + a.eps * kUp * kUp) * kUp;
  // a row of nothing is zero whatever its size (a gain of zero); a NaN or an infinity makes its block something
  const float factor = some == 0.f ? 0.f : ss < kInf && rs < kInf ? rs : __builtin_nanf("");
  if (t == 0) a.row_scale[r] = factor;
  if (!a.values) return;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = (p * TPR + t) * kE;
    float v[kE];
    values_of(q[p], top[p], factor, v);
    store_part<STREAM>(a.values + r * a.ld_v + c, a.channels - c, v);
  }
}

// Bytes that a launch writes.
template <typename T> int64_t written(const MxArgs &a) {
  return a.rows * a.channels * ((a.summed ? (int64_t)sizeof(T) : 0) + (a.values ? 2 : 0)) + a.rows * (a.channels / 2);
}

template <typename T, int TPR, int NP, bool STREAM> hipError_t go_as(const MxArgs &a, hipStream_t s) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
  const dim3 grid((unsigned)((a.rows + kRows - 1) / kRows)), block(TPR < 256 ? 256 : TPR);
  if (a.eps < kSmall) hipLaunchKernelGGL((norm_kernel<T, TPR, NP, STREAM, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_kernel<T, TPR, NP, STREAM, false>), grid, block, 0, s, a);
  return hipGetLastError();
}
template <typename T, int TPR, int NP> hipError_t go(const MxArgs &a, hipStream_t s) {
  return written<T>(a) < kStreamBytes ? go_as<T, TPR, NP, false>(a, s) : go_as<T, TPR, NP, true>(a, s);
}

template <typename T> hipError_t run_norm(const MxArgs &a, hipStream_t s) {
  const int d = a.channels;
  if (d <= 64 * kE) return go<T, 64, 1>(a, s);
  if (d <= 2 * 64 * kE) return go<T, 64, 2>(a, s);
  if (d <= 256 * kE) return go<T, 256, 1>(a, s);
  if (d <= 2 * 256 * kE) return go<T, 256, 2>(a, s);
  if (d <= 1024 * kE) return go<T, 1024, 1>(a, s);
  if (d <= 2 * 1024 * kE) return go<T, 1024, 2>(a, s);
  return go<T, 1024, 4>(a, s);
}

template <typename T> hipError_t run_quant(const MxArgs &a, hipStream_t s) {
  const uint32_t pieces = (a.channels + 31) / 32 * 4;
  const dim3 grid((unsigned)((a.rows * pieces + 255) / 256));
  if (written<T>(a) < kStreamBytes) hipLaunchKernelGGL((quant_kernel<T, false>), grid, dim3(256), 0, s, a, pieces);
  else hipLaunchKernelGGL((quant_kernel<T, true>), grid, dim3(256), 0, s, a, pieces);
  return hipGetLastError();
}

}  // namespace mx

hipError_t launch_quant_mx(const MxArgs &a, int dtype, hipStream_t s) {
  return dtype == FWG_BF16 ? mx::run_quant<uint16_t>(a, s) : mx::run_quant<float>(a, s);
}
hipError_t launch_norm_mx(const MxArgs &a, int dtype, hipStream_t s) {
  return dtype == FWG_BF16 ? mx::run_norm<uint16_t>(a, s) : mx::run_norm<float>(a, s);
}

}  // namespace fwg

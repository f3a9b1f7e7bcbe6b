// RMS norm with the residual's addition and 8-bit rows with a scale each.
//
// Per row: h = x + r, y = h / sqrt(mean h^2 + eps) * gain, scale = max|y| / 127, q = y / scale to the nearest
// whole number (ties to even).  The factor 1 / sqrt(...) is common to a row, so q = h gain * (127 / max|h gain|)
// needs only max|h gain| beside the sum of squares: both are reduced together, and the row, held in registers
// between, is read once and written once.  All of it is float32; h is rounded once where x's type is bf16.
//
// Bound by memory: 16,381 rows of 4,096 bf16 with residual, new residual, 8-bit rows and values (9 bytes an element, 604 MB)
// in 103 to 105 us (5.8 TB/s).  64 rows take the kernel 4.6 us and the call 8.2.  A row is one wave's up to 1,024 elements,
// else four waves' (sixteen's beyond 4,096): as few threads as hold it in 16 registers each, or 32 at the widest rows.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace nrm {

using namespace opd;

constexpr int kE = 8;  // elements of a thread's piece: 8 bytes of q, 16 of bf16
constexpr float kTiny = 7.888609052210118e-31f;   // 2^-100: rows whose result lies below it are zero
constexpr float kTinyIn = 7.52316384526264e-37f;  // 2^-120: 127 / max stays finite above it

// Largest value, NaN if one is NaN.
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

// TPR threads per row (64: a wave per row), NP pieces per thread.
template <typename T, int TPR, int NP, bool STREAM>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_quant_kernel(NormArgs a) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1, kW = TPR / 64;
  __shared__ float red[2 * kW];
  const int t = threadIdx.x % TPR;
  const int64_t r = (int64_t)blockIdx.x * kRows + threadIdx.x / TPR;
  if (r >= a.rows) return;  // whole waves, and whole blocks where a block is one row
  const T *x = (const T *)a.x + r * a.ld_x;
  float h[NP][kE], hg[NP][kE];
#pragma unroll
  for (int p = 0; p < NP; ++p) load_part(x + (p * TPR + t) * kE, a.channels - (p * TPR + t) * kE, 0.f, h[p]);
  if (a.residual) {
    const T *res = (const T *)a.residual + r * a.ld_r;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      float v[kE];
      load_part(res + (p * TPR + t) * kE, a.channels - (p * TPR + t) * kE, 0.f, v);
#pragma unroll
      for (int i = 0; i < kE; ++i) h[p][i] += v[i];
    }
  }
  float ss = 0.f, top = 0.f;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = (p * TPR + t) * kE;
    float g[kE];
    if (a.gain) load_part(a.gain + c, a.channels - c, 0.f, g);
#pragma unroll
    for (int i = 0; i < kE; ++i) {
      hg[p][i] = a.gain ? h[p][i] * g[i] : h[p][i];
      if (a.norm) ss += h[p][i] * h[p][i];
      top = max_nan(fabsf(hg[p][i]), top);
    }
    if (a.summed) store_part<STREAM>((T *)a.summed + r * a.ld_s + c, a.channels - c, h[p]);
  }
  // a NaN or an infinity anywhere goes on in the sum
  const float poison = top < kInf ? 0.f : __builtin_nanf("");
  top = wave_max(top);
  ss = wave_sum(ss + poison);
  if (kW > 1) {
    const int w = t >> 6;
    if ((t & 63) == 0) {
      red[2 * w] = ss;
      red[2 * w + 1] = top;
    }
    __syncthreads();
    ss = 0.f;
    top = 0.f;
#pragma unroll
    for (int i = 0; i < kW; ++i) {
      ss += red[2 * i];
      top = fmaxf(top, red[2 * i + 1]);
    }
  }
  const float rs = a.norm ? rsqrtf(ss / (float)a.channels + a.eps) : 1.f;
  const float amax = top * rs;
  // a row of (nearly) nothing is zero whatever 1 / rms is: it may be infinite where eps is 0
  const bool nothing = !(top >= kTinyIn);
  const bool bad = !(ss < kInf) || (!nothing && !(amax < kInf));
  const bool zero = bad || nothing || !(amax >= kTiny);
  const float inv = zero ? 0.f : 127.f / top;
  const float scale = bad ? __builtin_nanf("") : zero ? 0.f : amax / 127.f;
  if (t == 0) a.scale[r] = scale;
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = (p * TPR + t) * kE, have = a.channels - c;
    if (have <= 0) continue;
    float v[kE];
#pragma unroll
    for (int i = 0; i < kE; ++i) v[i] = zero ? 0.f : rintf(hg[p][i] * inv);
    int8_t *q = a.q + r * a.ld_q + c;
    if (have >= kE) {
      uint32_t w[2] = {0, 0};
#pragma unroll
      for (int i = 0; i < kE; ++i) w[i / 4] |= ((uint32_t)(int)v[i] & 0xffu) << (8 * (i % 4));
      store_bytes<STREAM>(q, w[0], w[1]);
    } else {
      for (int i = 0; i < kE; ++i)
        if (i < have) q[i] = (int8_t)(int)v[i];
    }
    if (a.values) {
#pragma unroll
      for (int i = 0; i < kE; ++i) v[i] *= scale;
      store_part<STREAM>(a.values + r * a.ld_v + c, have, v);
    }
  }
}

template <typename T, int TPR, int NP> hipError_t go(const NormArgs &a, hipStream_t s) {
  constexpr int kRows = TPR < 256 ? 256 / TPR : 1;
  const dim3 grid((unsigned)((a.rows + kRows - 1) / kRows)), block(TPR < 256 ? 256 : TPR);
  const int64_t bytes = a.rows * a.channels * (1 + (a.summed ? (int64_t)sizeof(T) : 0) + (a.values ? 2 : 0));
  if (bytes < kStreamBytes) hipLaunchKernelGGL((norm_quant_kernel<T, TPR, NP, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((norm_quant_kernel<T, TPR, NP, true>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename T> hipError_t run(const NormArgs &a, hipStream_t s) {
  const int d = a.channels;
  if (d <= 64 * kE) return go<T, 64, 1>(a, s);
  if (d <= 2 * 64 * kE) return go<T, 64, 2>(a, s);
  if (d <= 256 * kE) return go<T, 256, 1>(a, s);
  if (d <= 2 * 256 * kE) return go<T, 256, 2>(a, s);
  if (d <= 1024 * kE) return go<T, 1024, 1>(a, s);
  if (d <= 2 * 1024 * kE) return go<T, 1024, 2>(a, s);
  return go<T, 1024, 4>(a, s);
}

}  // namespace nrm

hipError_t launch_norm_quant(const NormArgs &a, int dtype, hipStream_t s) {
  return dtype == FWG_BF16 ? nrm::run<uint16_t>(a, s) : nrm::run<float>(a, s);
}

}  // namespace fwg

// Product of rows in microscaled 4-bit floating point with weights in the same form:
//   out[m][n] = row_scale[m] * sum over blocks b of 2^(ex[m][b] + ew[n][b]) * (sum over the block of x[m][k] w[n][k]) + bias[n].
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes both operands as they lie in memory: a lane holds one block of 32 consecutive
// elements of one row (16 bytes) and that block's scale byte.  Products and sums are float32.  The product is taken as
// D[n][m] = W X^T: a lane then holds four consecutive outputs of one row and stores them together.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace mmx {

using namespace opd;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4_b __attribute__((ext_vector_type(4), aligned(1)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// One product of 32 outputs x 32 rows x 64 elements; byte A of sa and byte B of sb are the scales of the lane's blocks.
template <int A, int B>
__device__ __forceinline__ f32x16 mma(const i32x4 &w, const i32x4 &x, const f32x16 &c, int sa, int sb) {
  const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, A, sa, B, sb);
}

// A wave per 32 outputs x 32 rows, operands straight from memory.
template <typename TO> __global__ void __launch_bounds__(256) plain_kernel(MatmulMxArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 31, half = lane >> 5;
  const int64_t m0 = (int64_t)blockIdx.x * 32;
  const int n0 = (blockIdx.y * 4 + wave) * 32;
  if (n0 >= a.N) return;
  const int64_t m = m0 + row;
  const int n = min(n0 + row, a.N - 1);
  const int64_t mc = m < a.M ? m : a.M - 1;
  const uint8_t *w = a.w + (int64_t)n * a.ld_w, *x = a.x + mc * a.ld_x;
  const uint8_t *ew = a.w_scale + (int64_t)n * a.ld_ew, *ex = a.x_scale + mc * a.ld_ex;
  f32x16 acc = {};
  for (int b = 0; b < a.blocks; b += 2) {
    i32x4 vw = {0, 0, 0, 0}, vx = {0, 0, 0, 0};
    int sw = 127, sx = 127;
    if (b + half < a.blocks) {
      vw = *(const i32x4_b *)(w + (b + half) * 16);
      vx = *(const i32x4_b *)(x + (b + half) * 16);
      sw = ew[b + half];
      sx = ex[b + half];
    }
    acc = mma<0, 0>(vw, vx, acc, sw, sx);
  }
  if (m >= a.M) return;
  const float f = a.row_scale ? a.row_scale[m] : 1.f;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const int at = n0 + 8 * g + 4 * half;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (at + e >= a.N) break;
      float v = acc[4 * g + e] * f;
      if (a.bias) v += a.bias[at + e];
      put((TO *)a.out + m * a.ld_o + at + e, v);
    }
  }
}

template <typename TO> hipError_t run(const MatmulMxArgs &a, hipStream_t s) {
  constexpr int64_t kRows = (int64_t)1 << 20;  // rows of a launch
  constexpr int kCols = 128 * 128;             // outputs of a launch
  for (int64_t m = 0; m < a.M; m += kRows)
    for (int64_t n = 0; n < a.N; n += kCols) {
      MatmulMxArgs b = a;
      b.M = a.M - m < kRows ? a.M - m : kRows;
      b.N = (int)(a.N - n < kCols ? a.N - n : kCols);
      b.x = a.x + m * a.ld_x;
      b.x_scale = a.x_scale + m * a.ld_ex;
      b.w = a.w + n * a.ld_w;
      b.w_scale = a.w_scale + n * a.ld_ew;
      if (a.row_scale) b.row_scale = a.row_scale + m;
      if (a.bias) b.bias = a.bias + n;
      b.out = (TO *)a.out + m * a.ld_o + n;
      hipLaunchKernelGGL((plain_kernel<TO>), dim3((unsigned)((b.M + 31) / 32), (unsigned)((b.N + 127) / 128)), dim3(256), 0, s,
                         b);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace mmx

size_t matmul_mx_bytes(int64_t, int, int) { return 0; }

hipError_t launch_matmul_mx(const MatmulMxArgs &a, int out_dtype, hipStream_t s) {
  return out_dtype == FWG_BF16 ? mmx::run<uint16_t>(a, s) : mmx::run<float>(a, s);
}

}  // namespace fwg

// Product of 8-bit rows with 8-bit weights: out[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n] + bias[n].
//
// The sum is exact: 8-bit integer products accumulated in 32 bits on the matrix cores
// (v_mfma_i32_16x16x64_i8), the scales and the bias in float32, one rounding where the output is bf16.  Both
// operands lie with k along their rows, which is what a lane of the instruction holds (16 consecutive k of one
// row), so no operand is transposed.  The product is taken as D[n][m] = W X^T: a lane then holds four
// consecutive outputs of one row and stores them together.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace mmq {

using namespace opd;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4_b __attribute__((ext_vector_type(4), aligned(1)));

__device__ __forceinline__ i32x4 mma(const i32x4 &a, const i32x4 &b, const i32x4 &c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// 16 bytes of a row from byte k on; bytes from K on and absent rows are 0.
__device__ __forceinline__ i32x4 load16(const int8_t *row, int k, int K, bool exists) {
  i32x4 v = {0, 0, 0, 0};
  if (!exists) return v;
  if (k + 16 <= K) return *(const i32x4_b *)(row + k);
  for (int i = 0; i < 16; ++i)
    if (k + i < K) v[i / 4] |= ((int)(uint8_t)row[k + i]) << (8 * (i % 4));
  return v;
}

// Four outputs n .. n + 3 of row m.
template <typename TO>
__device__ __forceinline__ void epilogue(const MatmulArgs &a, int64_t m, int n, const i32x4 &c) {
  if (m >= a.M || n >= a.N) return;
  const float sx = a.x_scale[m];
  const int have = a.N - n;
  float v[4], ws[4], b[4];
  load_part(a.w_scale + n, have, 0.f, ws);
  if (a.bias) load_part(a.bias + n, have, 0.f, b);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = (float)c[i] * sx * ws[i];
    if (a.bias) v[i] += b[i];
  }
  store_part((TO *)a.out + m * a.ld_o + n, have, v);
}

// 128 outputs x 128 rows per block of four waves, 64 bytes of k at a time through LDS.
constexpr int BM = 128, BN = 128, BK = 64, PAD = 16;
template <typename TO> __global__ void __launch_bounds__(256) tile_kernel(MatmulArgs a) {
  __shared__ __align__(16) int8_t sw[BN][BK + PAD], sx[BM][BK + PAD];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int n0 = blockIdx.x * BN;
  const int64_t m0 = (int64_t)blockIdx.y * BM;
  const int wn = (wave & 1) * 64, wm = (wave >> 1) * 64;
  i32x4 acc[4][4] = {};
  for (int k0 = 0; k0 < a.K; k0 += BK) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int p = i * 256 + t, r = p >> 2, k = (p & 3) * 16;
      *(i32x4 *)&sw[r][k] = load16(a.w + (int64_t)(n0 + r) * a.ld_w, k0 + k, a.K, n0 + r < a.N);
      *(i32x4 *)&sx[r][k] = load16(a.x + (m0 + r) * a.ld_x, k0 + k, a.K, m0 + r < a.M);
    }
    __syncthreads();
    i32x4 fw[4], fx[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      fw[i] = *(const i32x4 *)&sw[wn + 16 * i + (lane & 15)][(lane >> 4) * 16];
      fx[i] = *(const i32x4 *)&sx[wm + 16 * i + (lane & 15)][(lane >> 4) * 16];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = mma(fw[i], fx[j], acc[i][j]);
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      epilogue<TO>(a, m0 + wm + 16 * j + (lane & 15), n0 + wn + 16 * i + (lane >> 4) * 4, acc[i][j]);
}

template <typename TO> hipError_t run(const MatmulArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((tile_kernel<TO>), dim3((a.N + BN - 1) / BN, (unsigned)((a.M + BM - 1) / BM)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace mmq

size_t matmul_quant_bytes(int64_t, int, int) { return 0; }

hipError_t launch_matmul_quant(const MatmulArgs &a, int out_dtype, hipStream_t s) {
  return out_dtype == FWG_BF16 ? mmq::run<uint16_t>(a, s) : mmq::run<float>(a, s);
}

}  // namespace fwg

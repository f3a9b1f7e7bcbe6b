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

// A wave's LDS accesses are in order; this keeps the compiler to the order of the source.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

__device__ __forceinline__ i32x4 mma(const i32x4 &a, const i32x4 &b, const i32x4 &c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

// 16 bytes of a row from byte k on; bytes from K on and absent rows are 0.
__device__ __forceinline__ i32x4 load16(const int8_t *row, int k, int K, bool exists) {
  i32x4 v = {0, 0, 0, 0};
  if (!exists || k >= K) return v;
  if (k + 16 <= K) return *(const i32x4_b *)(row + k);
  if (K >= 16) {  // the row's last 16 bytes, shifted down
    const unsigned __int128 last = __builtin_bit_cast(unsigned __int128, (i32x4)*(const i32x4_b *)(row + K - 16));
    return __builtin_bit_cast(i32x4, last >> (8 * (k + 16 - K)));
  }
  unsigned __int128 part = 0;
#pragma unroll 1
  for (int i = K - 1; i >= k; --i) part = part << 8 | (uint8_t)row[i];
  return __builtin_bit_cast(i32x4, part);
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

// 256 outputs x 256 rows per block of eight waves, 128 bytes of k per stage, two stages in LDS (128 KB): one is filled
// while the other is multiplied.  A wave multiplies 64 outputs x 128 rows (v_mfma_i32_32x32x32_i8).  A stage's rows are
// 128 bytes; the 16-byte pieces of row r lie permuted by (r >> 1) & 7, so that the 32 rows that an instruction reads
// at one k spread over the banks.  ALIGNED: rows start at multiples of 16 bytes and are copied to LDS without passing
// through registers; else they pass through registers, which takes them at any address.
constexpr int HT = 256, HK = 128, kHugeThreads = 512;
constexpr int kStageBytes = 2 * HT * HK;
constexpr int kHugeLds = 2 * kStageBytes + 3 * HT * (int)sizeof(float);
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ int piece_of(int row, int piece) { return piece ^ ((row >> 1) & 7); }

template <typename TO, bool ALIGNED>
__global__ void __launch_bounds__(kHugeThreads) huge_kernel(MatmulArgs a, int tiles_m, int tiles_n) {
  extern __shared__ __align__(1024) int8_t smem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // each XCD (blocks go to the eight in turn) takes a contiguous share of the tiles, eight rows of tiles at a time
  const int tiles = tiles_m * tiles_n, share = (tiles + 7) / 8;
  const int tile = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  if (tile >= tiles || (int)(blockIdx.x >> 3) >= share) return;
  constexpr int G = 8;
  const int band = tile / (G * tiles_n), in_band = tile - band * G * tiles_n;
  const int high = min(G, tiles_m - band * G);
  const int n0 = in_band / high * HT;
  const int64_t m0 = (int64_t)(band * G + in_band % high) * HT;
  const int wn = (wave >> 1) * 64, wm = (wave & 1) * 128;

  // a wave copies 32 rows of each operand, 8 rows of 8 pieces at a time; rows past the end are the last one again
  auto from_w = [&](int r) { return a.w + (int64_t)min(n0 + r, a.N - 1) * a.ld_w; };
  auto from_x = [&](int r) { return a.x + (m0 + r < a.M ? m0 + r : a.M - 1) * a.ld_x; };
  const int8_t *gw[4], *gx[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = wave * 32 + i * 8 + (lane >> 3), p = piece_of(r, lane & 7) * 16;
    gw[i] = from_w(r) + p;
    gx[i] = from_x(r) + p;
  }
  auto copy = [&](int k0, int buf) {
    int8_t *w = smem + buf * kStageBytes + wave * 32 * HK, *x = w + HT * HK;
    if (k0 + HK <= a.K) {
      if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gw[i] + k0),
                                           (__attribute__((address_space(3))) void *)(w + i * 8 * HK), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(gx[i] + k0),
                                           (__attribute__((address_space(3))) void *)(x + i * 8 * HK), 16, 0, 0);
        }
      } else {
        i32x4 vw[4], vx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vw[i] = *(const i32x4_b *)(gw[i] + k0);
          vx[i] = *(const i32x4_b *)(gx[i] + k0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          *(i32x4 *)(w + i * 8 * HK + lane * 16) = vw[i];
          *(i32x4 *)(x + i * 8 * HK + lane * 16) = vx[i];
        }
      }
    } else {  // the last stage, where K ends inside it
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        const int r = wave * 32 + i * 8 + (lane >> 3), k = k0 + piece_of(r, lane & 7) * 16;
        *(i32x4 *)(w + i * 8 * HK + lane * 16) = load16(from_w(r), k, a.K, true);
        *(i32x4 *)(x + i * 8 * HK + lane * 16) = load16(from_x(r), k, a.K, true);
      }
    }
  };
  i32x16 acc[2][4] = {};
  const int row = lane & 31, half = lane >> 5;
  // the operands of one k-step (32 bytes), read while the step before is multiplied
  i32x4 fw[2][2], fx[2][4];
  auto read = [&](int buf, int k, int slot) {
    const int8_t *w = smem + buf * kStageBytes + (wn + row) * HK, *x = smem + buf * kStageBytes + HT * HK + (wm + row) * HK;
    const int p = piece_of(row, 2 * k + half) * 16;  // wn, wm and 32 leave (r >> 1) & 7 as it is
#pragma unroll
    for (int i = 0; i < 2; ++i) fw[slot][i] = *(const i32x4 *)(w + i * 32 * HK + p);
#pragma unroll
    for (int j = 0; j < 4; ++j) fx[slot][j] = *(const i32x4 *)(x + j * 32 * HK + p);
  };
  auto multiply = [&](int slot) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[slot][i], fx[slot][j], acc[i][j], 0, 0, 0);
  };
  // one read between two products
  auto interleave = [] {
#pragma unroll
    for (int i = 0; i < 6; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);
  };
  copy(0, 0);
  // the tile's scales and biases: w_scale, bias, x_scale
  float *scales = (float *)(smem + 2 * kStageBytes);
  if (threadIdx.x < HT) {
    const int n = min(n0 + (int)threadIdx.x, a.N - 1);
    scales[threadIdx.x] = a.w_scale[n];
    scales[HT + threadIdx.x] = a.bias ? a.bias[n] : 0.f;
  } else {
    const int64_t m = m0 + threadIdx.x - HT;
    scales[HT + threadIdx.x] = a.x_scale[m < a.M ? m : a.M - 1];
  }
  __syncthreads();
  read(0, 0, 0);
  int buf = 0;
  for (int k0 = 0; k0 < a.K; k0 += HK) {
    if (k0 + HK < a.K) copy(k0 + HK, buf ^ 1);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      read(buf, k + 1, (k + 1) & 1);
      multiply(k & 1);
      interleave();
    }
    __syncthreads();
    buf ^= 1;
    read(buf, 0, 0);  // after the last stage: unused
    multiply(1);
    interleave();
  }
  __syncthreads();
  // The results of a wave pass through its eighth of the LDS, so that rows go out in whole 128-byte lines: as rows of
  // 128 bytes (64 bf16, or 32 float32 at a time), pieces of 16 bytes permuted by the row.
  constexpr int kTiles = sizeof(TO) == 2 ? 2 : 1;  // 32-output tiles of a line
  int8_t *mine = smem + wave * (2 * kStageBytes / 8);
#pragma unroll
  for (int i0 = 0; i0 < 2; i0 += kTiles) {
    if (i0) in_order();
#pragma unroll
    for (int ii = 0; ii < kTiles; ++ii) {
      const int i = i0 + ii;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = wn + i * 32 + g * 8 + half * 4;
        const f32x4 ws = *(const f32x4 *)(scales + n), b = *(const f32x4 *)(scales + HT + n);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float sx = scales[2 * HT + wm + j * 32 + row];
          float v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[e] = (float)acc[i][j][4 * g + e] * sx * ws[e];
            if (a.bias) v[e] += b[e];
          }
          const int at = (ii * 32 + g * 8 + half * 4) * (int)sizeof(TO), r = j * 32 + row;
          store((TO *)(mine + r * 128 + (((at >> 4) ^ (r & 7)) << 4) + (at & 15)), v);
        }
      }
    }
    in_order();
    constexpr int E = 16 / sizeof(TO);
    const int n = n0 + wn + i0 * 32 + (lane & 7) * E;
#pragma unroll
    for (int q = 0; q < 16; ++q) {
      const int r = q * 8 + (lane >> 3);
      const int64_t m = m0 + wm + r;
      const u32x4 v = *(const u32x4 *)(mine + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
      if (m >= a.M) continue;
      TO *out = (TO *)a.out + m * a.ld_o + n;
      if (n + E <= a.N) {
        *(u32x4_el *)out = v;
      } else {
        const TO *e = (const TO *)(mine + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
        for (int k = 0; k < E; ++k)
          if (n + k < a.N) out[k] = e[k];
      }
    }
  }
}

template <typename TO, bool ALIGNED> hipError_t run_huge(const MatmulArgs &a, hipStream_t s) {
  static const hipError_t set = hipFuncSetAttribute((const void *)huge_kernel<TO, ALIGNED>,
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, kHugeLds);
  if (set != hipSuccess) return set;
  const int tm = (int)((a.M + HT - 1) / HT), tn = (a.N + HT - 1) / HT;
  const unsigned grid = (unsigned)(((int64_t)tm * tn + 7) / 8 * 8);
  hipLaunchKernelGGL((huge_kernel<TO, ALIGNED>), dim3(grid), dim3(kHugeThreads), kHugeLds, s, a, tm, tn);
  return hipGetLastError();
}

template <typename TO> hipError_t run(const MatmulArgs &a, hipStream_t s) {
  const bool aligned = (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & 15) == 0;
  if ((a.M + HT - 1) / HT * ((a.N + HT - 1) / HT) >= 128)
    return aligned ? run_huge<TO, true>(a, s) : run_huge<TO, false>(a, s);
  hipLaunchKernelGGL((tile_kernel<TO>), dim3((a.N + BN - 1) / BN, (unsigned)((a.M + BM - 1) / BM)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace mmq

size_t matmul_quant_bytes(int64_t, int, int) { return 0; }

hipError_t launch_matmul_quant(const MatmulArgs &a, int out_dtype, hipStream_t s) {
  return out_dtype == FWG_BF16 ? mmq::run<uint16_t>(a, s) : mmq::run<float>(a, s);
}

}  // namespace fwg

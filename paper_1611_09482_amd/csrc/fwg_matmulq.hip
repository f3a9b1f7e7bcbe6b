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
constexpr int kHugeLds = 2 * kStageBytes + 2 * 3 * HT * (int)sizeof(float);
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ int piece_of(int row, int piece) { return piece ^ ((row >> 1) & 7); }

// From memory to LDS without registers: lane l's bytes land at the (uniform) address + 16 l, or 4 l.
__device__ __forceinline__ void copy_16(const int8_t *g, int8_t *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 16, 0, 0);
}
__device__ __forceinline__ void copy_4(const float *g, float *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 4, 0, 0);
}

template <typename TO, bool ALIGNED>
__global__ void __launch_bounds__(kHugeThreads) huge_kernel(MatmulArgs a, int tiles_m, int tiles_n) {
  extern __shared__ __align__(1024) int8_t smem[];
  float *const scales = (float *)(smem + 2 * kStageBytes);  // [2]: w_scale, bias, x_scale of the tile
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = (wave >> 1) * 64, wm = (wave & 1) * 128, row = lane & 31, half = lane >> 5;
  // Each XCD (blocks go to the eight in turn) takes a contiguous share of the tiles, eight rows of tiles at a time;
  // its blocks go through the share together.
  const int tiles = tiles_m * tiles_n, share = (tiles + 7) / 8, stride = gridDim.x >> 3;
  int tile = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  const int end = min(tiles, (int)(blockIdx.x & 7) * share + share);
  if (tile >= end) return;

  // Copies: a wave brings 32 rows of each operand, 8 rows of 8 pieces at a time; rows past the end are the last one.
  int n0;
  int64_t m0;
  const int8_t *bw, *bx;  // the tile's first rows
  unsigned ow[4], ox[4];  // this lane's pieces from there (rows_fit: below 2^31)
  auto go_to = [&](int t) {
    constexpr int G = 8;
    const int band = t / (G * tiles_n), in_band = t - band * G * tiles_n, high = min(G, tiles_m - band * G);
    n0 = in_band / high * HT;
    m0 = (int64_t)(band * G + in_band % high) * HT;
    bw = a.w + n0 * a.ld_w;
    bx = a.x + m0 * a.ld_x;
    const int rows_w = min(HT, a.N - n0), rows_x = (int)min((int64_t)HT, a.M - m0);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = wave * 32 + i * 8 + (lane >> 3), p = piece_of(r, lane & 7) * 16;
      ow[i] = (unsigned)min(r, rows_w - 1) * (unsigned)a.ld_w + p;
      ox[i] = (unsigned)min(r, rows_x - 1) * (unsigned)a.ld_x + p;
    }
  };
  auto copy = [&](int k0, int buf) {
    int8_t *w = smem + buf * kStageBytes + wave * 32 * HK, *x = w + HT * HK;
    if (k0 + HK <= a.K) {
      if constexpr (ALIGNED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          copy_16(bw + k0 + ow[i], w + i * 8 * HK);
          copy_16(bx + k0 + ox[i], x + i * 8 * HK);
        }
      } else {
        i32x4 vw[4], vx[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          vw[i] = *(const i32x4_b *)(bw + k0 + ow[i]);
          vx[i] = *(const i32x4_b *)(bx + k0 + ox[i]);
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
        const int rw = min(r, a.N - 1 - n0), rx = (int)min((int64_t)r, a.M - 1 - m0);
        *(i32x4 *)(w + i * 8 * HK + lane * 16) = load16(bw + rw * a.ld_w, k, a.K, true);
        *(i32x4 *)(x + i * 8 * HK + lane * 16) = load16(bx + rx * a.ld_x, k, a.K, true);
      }
    }
  };
  auto copy_scales = [&](int which) {  // waves 0 .. 3: 64 channels each, 4 .. 7: 64 rows each
    float *to = scales + which * 3 * HT;
    const int o = (wave & 3) * 64, n = min(n0 + o + lane, a.N - 1);
    const int64_t m = m0 + o + lane;
    if (wave < 4) {
      copy_4(a.w_scale + n, to + o);
      if (a.bias) copy_4(a.bias + n, to + HT + o);
    } else {
      copy_4(a.x_scale + (m < a.M ? m : a.M - 1), to + 2 * HT + o);
    }
  };

  // the operands of one k-step (32 bytes), read while the step before is multiplied
  i32x16 acc[2][4] = {};
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

  // Results: a wave's 64 outputs x 128 rows pass through 8 KB of LDS (of the stage that was multiplied last), so that
  // they go out in whole 128-byte lines: 64 rows of 128 bytes at a time (64 bf16, or 32 float32), pieces of 16 bytes
  // permuted by the row.
  auto write = [&](int8_t *mine, const float *sc, int n_at, int64_t m_at) {
    constexpr int kTiles = sizeof(TO) == 2 ? 2 : 1;  // 32-output tiles of a line
    constexpr int E = 16 / sizeof(TO);
#pragma unroll
    for (int i0 = 0; i0 < 2; i0 += kTiles) {
#pragma unroll
      for (int j0 = 0; j0 < 4; j0 += 2) {
        in_order();
#pragma unroll
        for (int ii = 0; ii < kTiles; ++ii) {
          const int i = i0 + ii;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int n = wn + i * 32 + g * 8 + half * 4;
            const f32x4 ws = *(const f32x4 *)(sc + n), b = *(const f32x4 *)(sc + HT + n);
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const float sx = sc[2 * HT + wm + (j0 + jj) * 32 + row];
              float v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                v[e] = (float)acc[i][j0 + jj][4 * g + e] * sx * ws[e];
                if (a.bias) v[e] += b[e];
              }
              const int at = (ii * 32 + g * 8 + half * 4) * (int)sizeof(TO), r = jj * 32 + row;
              store((TO *)(mine + r * 128 + (((at >> 4) ^ (r & 7)) << 4) + (at & 15)), v);
            }
          }
        }
        in_order();
        const int n = n_at + wn + i0 * 32 + (lane & 7) * E;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int r = q * 8 + (lane >> 3);
          const int64_t m = m_at + wm + j0 * 32 + r;
          const int8_t *line = mine + r * 128 + (((lane & 7) ^ (r & 7)) << 4);
          if (m >= a.M) continue;
          TO *out = (TO *)a.out + m * a.ld_o + n;
          if (n + E <= a.N) {
            *(u32x4_el *)out = *(const u32x4 *)line;
          } else {
            for (int k = 0; k < E; ++k)
              if (n + k < a.N) out[k] = ((const TO *)line)[k];
          }
        }
      }
    }
  };

  go_to(tile);
  copy(0, 0);
  copy_scales(0);
  __syncthreads();
  int buf = 0, which = 0;
  while (true) {
    const int n_at = n0, next = tile + stride;
    const int64_t m_at = m0;
    read(buf, 0, 0);
    auto three_steps = [&] {
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        read(buf, k + 1, (k + 1) & 1);
        multiply(k & 1);
        interleave();
      }
      __syncthreads();  // the next stage has arrived, and this one has been read
    };
    int k0 = 0;
    for (; k0 + HK < a.K; k0 += HK) {
      copy(k0 + HK, buf ^ 1);
      three_steps();
      buf ^= 1;
      read(buf, 0, 0);
      multiply(1);
      interleave();
    }
    // the stages of all tiles are one stream: while a tile's last one is multiplied, the next tile's first is copied
    if (next < end) {
      go_to(next);
      copy(0, buf ^ 1);
      copy_scales(which ^ 1);
    }
    three_steps();
    multiply(1);
    write(smem + buf * kStageBytes + wave * (kStageBytes / 8), scales + which * 3 * HT, n_at, m_at);
    if (next >= end) break;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = i32x16{};
    tile = next;
    buf ^= 1;
    which ^= 1;
    // the LDS just used may be copied over now; the results on their way out are not waited for
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  }
}

template <typename TO, bool ALIGNED> hipError_t run_huge(const MatmulArgs &a, hipStream_t s) {
  static const hipError_t set = hipFuncSetAttribute((const void *)huge_kernel<TO, ALIGNED>,
                                                    hipFuncAttributeMaxDynamicSharedMemorySize, kHugeLds);
  if (set != hipSuccess) return set;
  const int tm = (int)((a.M + HT - 1) / HT), tn = (a.N + HT - 1) / HT;
  const int64_t blocks = ((int64_t)tm * tn + 7) / 8 * 8;
  const unsigned grid = blocks < 256 ? (unsigned)blocks : 256;  // one per compute unit: they fill its LDS
  hipLaunchKernelGGL((huge_kernel<TO, ALIGNED>), dim3(grid), dim3(kHugeThreads), kHugeLds, s, a, tm, tn);
  return hipGetLastError();
}

template <typename TO> hipError_t run(const MatmulArgs &a, hipStream_t s) {
  const bool aligned = (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & 15) == 0;
  const bool rows_fit = a.ld_x < (1 << 22) && a.ld_w < (1 << 22);  // a tile's rows lie within 2^30 bytes
  if (rows_fit && (a.M + HT - 1) / HT * ((a.N + HT - 1) / HT) >= 128)
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

// Product of 8-bit rows with 8-bit weights: out[m][n] = (sum_k x[m][k] w[n][k]) * x_scale[m] * w_scale[n] + bias[n].
//
// The sum is exact: 8-bit integer products accumulated in 32 bits on the matrix cores (v_mfma_i32_32x32x32_i8 in
// tiles, v_mfma_i32_16x16x64_i8 for few rows), the scales and the bias in float32, one rounding where the output is bf16.  Both
// operands lie with k along their rows, which is what a lane of the instruction holds (16 consecutive k of one
// row), so no operand is transposed.  The product is taken as D[n][m] = W X^T: a lane then holds four
// consecutive outputs of one row and stores them together.
//
// Measured (steady clocks): 4,093 x 32,000 x 4,096 to bf16 512 us (2,095 TOP/s), 8,192^3 442 us (2,486 TOP/s): the rates of
// the largest library product here (2,050 and 2,490).  The matrix cores are busy 54 to 59% of the cycles at the 1.5 to 2.1
// GHz that the card keeps up under this load; LDS conflicts take 2%.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

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

// 16 bytes at any address.  Where they are no aligned words the hardware takes 2.3 times as long (16 x 7,637 x 4,343: 22.7
// us, x 4,352: 9.8), so with SHIFT the five words that hold the bytes are loaded and shifted: 14.2 us.  (For the tiles
// below it costs more than it saves: 4,000 x 8,000 x 1,001 takes 71 us with it, 60 without.)
template <bool SHIFT> __device__ __forceinline__ i32x4 load_any(const int8_t *p) {
  if constexpr (!SHIFT) return *(const i32x4_b *)p;
  typedef unsigned int u32x4_w __attribute__((ext_vector_type(4), aligned(4)));
  const unsigned s = (unsigned)(uintptr_t)p & 3u;
  const int8_t *q = p - s;
  const u32x4_w a = *(const u32x4_w *)q;
  const unsigned e = *(const unsigned *)(q + (s ? 16 : 12));  // not past the words that hold the bytes
  return i32x4{(int)__builtin_amdgcn_alignbyte(a[1], a[0], s), (int)__builtin_amdgcn_alignbyte(a[2], a[1], s),
               (int)__builtin_amdgcn_alignbyte(a[3], a[2], s), (int)__builtin_amdgcn_alignbyte(e, a[3], s)};
}

// 16 bytes of a row from byte k on; bytes from K on are 0.
__device__ __forceinline__ i32x4 load16(const int8_t *row, int k, int K) {
  i32x4 v = {0, 0, 0, 0};
  if (k >= K) return v;
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

// Tiles of T outputs x T rows (256: eight waves; 128: four), 128 bytes of k per stage, two stages in LDS: one is filled
// while the other is multiplied.  A wave multiplies 64 outputs x T / 2 rows (v_mfma_i32_32x32x32_i8).  A stage's rows
// are 128 bytes; the 16-byte pieces of row r lie permuted by (r >> 1) & 7, so that the 32 rows that an instruction
// reads at one k spread over the banks.  ALIGNED: rows start at multiples of 16 bytes and are copied to LDS without
// passing through registers; else they pass through registers, which takes them at any address but waits for a stage's
// memory before the products of the stage at hand (4,000 x 8,000 x 1,001 in 60 us, the products alone 31).  TO = int:
// sums of a part of k go to the workspace as they are.
constexpr int HK = 128;
template <int T> struct Tile {
  static constexpr int kWaves = T / 32, kThreads = 64 * kWaves, kWM = T / 2, kJ = kWM / 32;
  static constexpr int kStage = 2 * T * HK;                               // bytes of a stage: weights, then rows
  static constexpr int kLds = 2 * kStage + 2 * 3 * T * (int)sizeof(float);  // two stages, two tiles' scales
};
typedef int i32x16 __attribute__((ext_vector_type(16)));

__device__ __forceinline__ int piece_of(int row, int piece) { return piece ^ ((row >> 1) & 7); }

struct Cut {
  int tiles_m, tiles_n, splits, per;  // k is cut into `splits` parts of `per` bytes (a multiple of HK)
};

// From memory to LDS without registers: lane l's bytes land at the (uniform) address + 16 l, or 4 l.
__device__ __forceinline__ void copy_16(const int8_t *g, int8_t *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 16, 0, 0);
}
__device__ __forceinline__ void copy_4(const float *g, float *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 4, 0, 0);
}

template <typename TO, bool ALIGNED, int T>
__global__ void __launch_bounds__(Tile<T>::kThreads, 2) tile_kernel(MatmulArgs a, Cut cut) {
  constexpr int J = Tile<T>::kJ, kStage = Tile<T>::kStage;
  constexpr bool kSums = std::is_same<TO, int>::value;
  extern __shared__ __align__(1024) int8_t smem[];
  float *const scales = (float *)(smem + 2 * kStage);  // [2]: w_scale, bias, x_scale of the tile
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = (wave >> 1) * 64, wm = (wave & 1) * Tile<T>::kWM, row = lane & 31, half = lane >> 5;
  const int tiles_m = cut.tiles_m, tiles_n = cut.tiles_n;
  const int k_at = (int)blockIdx.y * cut.per, k_end = min(a.K, k_at + cut.per);
  TO *const result = (TO *)a.out + (kSums ? (int64_t)blockIdx.y * a.M * a.ld_o : 0);
  // Each XCD (blocks go to the eight in turn) takes a contiguous share of the tiles, eight rows of tiles at a time;
  // its blocks go through the share together.
  const int tiles = tiles_m * tiles_n, share = (tiles + 7) / 8, stride = gridDim.x >> 3;
  int tile = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  const int end = min(tiles, (int)(blockIdx.x & 7) * share + share);
  if (tile >= end) return;

  // Copies: a wave brings 32 rows of each operand, 8 rows of 8 pieces at a time; rows past the end are the last one.
  int n0;
  int64_t m0;
  const int8_t *bw, *bx;                    // the tile's first rows
  int rows_w, rows_x;
  unsigned ow[4], ox[4];                    // ALIGNED: this lane's pieces from there (below 2^31)
  const int cr = wave * 32 + (lane >> 3);   // the first of the lane's rows; the others follow 8 apart
  auto go_to = [&](int t) {
    constexpr int G = 8;
    const int band = t / (G * tiles_n), in_band = t - band * G * tiles_n, high = min(G, tiles_m - band * G);
    n0 = in_band / high * T;
    m0 = (int64_t)(band * G + in_band % high) * T;
    bw = a.w + n0 * a.ld_w;
    bx = a.x + m0 * a.ld_x;
    rows_w = min(T, a.N - n0);
    rows_x = (int)min((int64_t)T, a.M - m0);
    if constexpr (ALIGNED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = cr + i * 8, p = piece_of(r, lane & 7) * 16;
        ow[i] = (unsigned)min(r, rows_w - 1) * (unsigned)a.ld_w + p;
        ox[i] = (unsigned)min(r, rows_x - 1) * (unsigned)a.ld_x + p;
      }
    }
  };
  auto copy = [&](int k0, int buf) {
    int8_t *w = smem + buf * kStage + wave * 32 * HK, *x = w + T * HK;
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
          const int r = cr + i * 8, p = k0 + piece_of(r, lane & 7) * 16;
          vw[i] = *(const i32x4_b *)(bw + min(r, rows_w - 1) * a.ld_w + p);
          vx[i] = *(const i32x4_b *)(bx + min(r, rows_x - 1) * a.ld_x + p);
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
        const int r = cr + i * 8, p = k0 + piece_of(r, lane & 7) * 16;
        *(i32x4 *)(w + i * 8 * HK + lane * 16) = load16(bw + min(r, rows_w - 1) * a.ld_w, p, a.K);
        *(i32x4 *)(x + i * 8 * HK + lane * 16) = load16(bx + min(r, rows_x - 1) * a.ld_x, p, a.K);
      }
    }
  };
  auto copy_scales = [&](int which) {  // the first half of the waves: 64 channels each, the others: 64 rows each
    if constexpr (kSums) return;
    constexpr int kHalf = Tile<T>::kWaves / 2;
    float *to = scales + which * 3 * T;
    const int o = (wave % kHalf) * 64, n = min(n0 + o + lane, a.N - 1);
    const int64_t m = m0 + o + lane;
    if (wave < kHalf) {
      copy_4(a.w_scale + n, to + o);
      if (a.bias) copy_4(a.bias + n, to + T + o);
    } else {
      copy_4(a.x_scale + (m < a.M ? m : a.M - 1), to + 2 * T + o);
    }
  };

  // the operands of one k-step (32 bytes), read while the step before is multiplied
  i32x16 acc[2][J] = {};
  i32x4 fw[2][2], fx[2][J];
  auto read = [&](int buf, int k, int slot) {
    const int8_t *w = smem + buf * kStage + (wn + row) * HK, *x = smem + buf * kStage + T * HK + (wm + row) * HK;
    const int p = piece_of(row, 2 * k + half) * 16;  // wn, wm and 32 leave (r >> 1) & 7 as it is
#pragma unroll
    for (int i = 0; i < 2; ++i) fw[slot][i] = *(const i32x4 *)(w + i * 32 * HK + p);
#pragma unroll
    for (int j = 0; j < J; ++j) fx[slot][j] = *(const i32x4 *)(x + j * 32 * HK + p);
  };
  auto multiply = [&](int slot) {
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fw[slot][i], fx[slot][j], acc[i][j], 0, 0, 0);
  };
  // one read between two products
  auto interleave = [] {
#pragma unroll
    for (int i = 0; i < min(2 + J, 2 * J); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if constexpr (J > 2) __builtin_amdgcn_sched_group_barrier(0x008, J - 2, 0);
  };

  // Results: a wave's 64 outputs x T / 2 rows pass through 8 KB of LDS (of the stage that was multiplied last), so that
  // they go out in whole 128-byte lines: 64 rows of 128 bytes at a time (64 bf16, or 32 float32), pieces of 16 bytes
  // permuted by the row.
  auto write = [&](int8_t *mine, const float *sc, int n_at, int64_t m_at) {
    constexpr int kTiles = sizeof(TO) == 2 ? 2 : 1;  // 32-output tiles of a line
    constexpr int E = 16 / sizeof(TO);
#pragma unroll
    for (int i0 = 0; i0 < 2; i0 += kTiles) {
#pragma unroll
      for (int j0 = 0; j0 < J; j0 += 2) {
        in_order();
#pragma unroll
        for (int ii = 0; ii < kTiles; ++ii) {
          const int i = i0 + ii;
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int n = wn + i * 32 + g * 8 + half * 4;
            const f32x4 ws = *(const f32x4 *)(sc + n), b = *(const f32x4 *)(sc + T + n);
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
              const float sx = sc[2 * T + wm + (j0 + jj) * 32 + row];
              const int at = (ii * 32 + g * 8 + half * 4) * (int)sizeof(TO), r = jj * 32 + row;
              int8_t *to = mine + r * 128 + (((at >> 4) ^ (r & 7)) << 4) + (at & 15);
              if constexpr (kSums) {
                *(i32x4 *)to = i32x4{acc[i][j0 + jj][4 * g], acc[i][j0 + jj][4 * g + 1], acc[i][j0 + jj][4 * g + 2],
                                     acc[i][j0 + jj][4 * g + 3]};
              } else {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  v[e] = (float)acc[i][j0 + jj][4 * g + e] * sx * ws[e];
                  if (a.bias) v[e] += b[e];
                }
                store_aligned((TO *)to, v);
              }
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
          TO *out = result + m * a.ld_o + n;
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
  copy(k_at, 0);
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
    for (int k0 = k_at; k0 + HK < k_end; k0 += HK) {
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
      copy(k_at, buf ^ 1);
      copy_scales(which ^ 1);
    }
    three_steps();
    multiply(1);
    write(smem + buf * kStage + wave * 8192, scales + which * 3 * T, n_at, m_at);
    if (next >= end) break;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) acc[i][j] = i32x16{};
    tile = next;
    buf ^= 1;
    which ^= 1;
    // the LDS just used may be copied over now; the results on their way out are not waited for
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  }
}

// Few rows (M <= 16 MT): the weights are read once, straight into registers, by one block per 16 NT outputs; the rows
// come from the caches.  The W waves of a block take 128 bytes of k in turn, kUnits turns in flight, and their sums
// meet in LDS.  Bound by memory: 16 x 32,000 x 4,096 in 31 us (4.3 TB/s; 22 us where the weights are in the last-level
// cache), one row in 25 us (5.2 TB/s).  W: with 4 waves 16 x 1,000 x 8,000 takes 17 us instead of 10, 16 x 4,096 x
// 8,192 15.9 instead of 10.8.  NT: two tiles of outputs share the rows' reads (16 x 32,000 x 4,096 31 us, 38 with one) but
// leave compute units idle below 8,192 outputs (16 x 4,096 x 8,192 15.1 us, 10.8 with one).
template <typename TO, int MT, int NT, int kUnits, bool SHIFT>
__global__ void __launch_bounds__(1024) rows_kernel(MatmulArgs a) {
  constexpr int W = 16;
  __shared__ int sums[W][MT * 16][NT * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, p = (lane >> 4) * 16;
  const int n0 = blockIdx.x * (16 * NT);
  const int8_t *w[NT], *x[MT];
#pragma unroll
  for (int i = 0; i < NT; ++i) w[i] = a.w + (int64_t)min(n0 + i * 16 + r, a.N - 1) * a.ld_w;
#pragma unroll
  for (int j = 0; j < MT; ++j) x[j] = a.x + (int64_t)min(j * 16 + r, (int)a.M - 1) * a.ld_x;
  i32x4 acc[NT][MT] = {};
  int k = wave * 128;
  for (; k + (kUnits - 1) * (128 * W) + 128 <= a.K; k += kUnits * (128 * W)) {
    i32x4 vw[kUnits][2][NT], vx[kUnits][2][MT];
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < NT; ++i) vw[u][h][i] = load_any<SHIFT>(w[i] + k + u * (128 * W) + h * 64 + p);
#pragma unroll
        for (int j = 0; j < MT; ++j) vx[u][h][j] = load_any<SHIFT>(x[j] + k + u * (128 * W) + h * 64 + p);
      }
#pragma unroll
    for (int u = 0; u < kUnits; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
          for (int j = 0; j < MT; ++j) acc[i][j] = mma(vw[u][h][i], vx[u][h][j], acc[i][j]);
  }
#pragma unroll 1
  for (; k < a.K; k += 128 * W) {
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
      i32x4 vw[NT], vx[MT];
#pragma unroll
      for (int i = 0; i < NT; ++i) vw[i] = load16(w[i], k + h * 64 + p, a.K);
#pragma unroll
      for (int j = 0; j < MT; ++j) vx[j] = load16(x[j], k + h * 64 + p, a.K);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = mma(vw[i], vx[j], acc[i][j]);
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) *(i32x4 *)&sums[wave][j * 16 + r][i * 16 + (lane >> 4) * 4] = acc[i][j];
  __syncthreads();
  for (int t = threadIdx.x; t < MT * NT * 256; t += 64 * W) {
    const int m = t / (16 * NT), c = t % (16 * NT), n = n0 + c;
    if (m >= a.M || n >= a.N) continue;
    int sum = 0;
#pragma unroll
    for (int v = 0; v < W; ++v) sum += sums[v][m][c];
    float v = (float)sum * a.x_scale[m] * a.w_scale[n];
    if (a.bias) v += a.bias[n];
    put((TO *)a.out + m * a.ld_o + n, v);
  }
}

// (Latency: 300 x 515 x 4,096 takes 15.4 us in 240 blocks and this launch, 57 us without parts.)
//
// Adds the parts of k up: whole numbers, so their order does not matter.
template <typename TO> __global__ void __launch_bounds__(256) add_kernel(MatmulArgs a, int splits) {
  const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4, all = a.M * a.N;
  if (i >= all) return;
  const int *sums = (const int *)a.ws;
  if (i + 4 <= all && a.N % 4 == 0) {
    i32x4 c = {0, 0, 0, 0};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) c += *(const i32x4 *)(sums + s * all + i);
    const int64_t m = i / a.N;
    const int n = (int)(i - m * a.N);
    const float sx = a.x_scale[m];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[e] = (float)c[e] * sx * a.w_scale[n + e];
      if (a.bias) v[e] += a.bias[n + e];
    }
    store((TO *)a.out + m * a.ld_o + n, v);
    return;
  }
  for (int64_t e = i; e < i + 4 && e < all; ++e) {
    int c = 0;
    for (int s = 0; s < splits; ++s) c += sums[s * all + e];
    const int64_t m = e / a.N;
    const int n = (int)(e - m * a.N);
    float v = (float)c * a.x_scale[m] * a.w_scale[n];
    if (a.bias) v += a.bias[n];
    put((TO *)a.out + m * a.ld_o + n, v);
  }
}

// rows_kernel or tiles (us at k = 4096): 32 rows x 32,000 outputs 28.3 or 26.9, x 4,096 7.3 or 10.7; 64 rows x 32,000
// 36.3 or 27.9, x 4,096 12.0 or 12.5, x 8,192 (k = 8192) 38.1 or 21.1.
bool rows_form(int64_t M, int N) { return M <= 16 || (M <= 32 && N <= 8192) || (M <= 64 && N <= 4096); }
// How a product of more rows is cut: the tile's side, and parts of k where the tiles alone leave compute units idle.
int cut_of(int64_t M, int N, int K, Cut *c) {
  const int64_t big = (M + 255) / 256 * ((N + 255) / 256);
  const int side = big >= 192 ? 256 : 128;
  c->tiles_m = (int)((M + side - 1) / side);
  c->tiles_n = (N + side - 1) / side;
  const int64_t tiles = (int64_t)c->tiles_m * c->tiles_n;
  const int stages = (K + HK - 1) / HK;
  // one part per compute unit: two measured 25.1 -> 27.3 us at 300 x 8,000 x 4,096, 27.9 -> 30.0 at 64 x 32,000 x 4,096
  int64_t splits = side == 256 ? 1 : 256 / tiles;
  if (splits > stages / 4) splits = stages / 4;  // a part shorter than four stages costs more than it saves
  if (splits < 1) splits = 1;
  c->per = (int)((stages + splits - 1) / splits) * HK;
  c->splits = (K + c->per - 1) / c->per;
  return side;
}

// Whether all rows of both operands start at multiples of so many bytes.
bool aligned_to(const MatmulArgs &a, int bytes) {
  return (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & (bytes - 1)) == 0;
}

// Lets a kernel have its LDS, once per device (`done`: one bit each; a device past the 64th is told every time).
hipError_t allow_lds(const void *kernel, int bytes, std::atomic<uint64_t> &done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  const uint64_t bit = dev < 64 ? 1ull << dev : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

template <typename TO, bool ALIGNED, int T> hipError_t run_tiles(const MatmulArgs &a, const Cut &c, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void *)tile_kernel<TO, ALIGNED, T>, Tile<T>::kLds, done);
  if (e != hipSuccess) return e;
  // a block goes through several tiles where there are more than the device holds (one of 256, or two of 128 per
  // compute unit)
  const int64_t blocks = ((int64_t)c.tiles_m * c.tiles_n + 7) / 8 * 8, most = T == 256 ? 256 : 512;
  hipLaunchKernelGGL((tile_kernel<TO, ALIGNED, T>), dim3((unsigned)(blocks < most ? blocks : most), (unsigned)c.splits),
                     dim3(Tile<T>::kThreads), Tile<T>::kLds, s, a, c);
  return hipGetLastError();
}

template <typename TO, int T> hipError_t run_cut(const MatmulArgs &a, const Cut &c, hipStream_t s) {
  const bool near = a.ld_x < (1 << 22) && a.ld_w < (1 << 22);  // a tile's rows lie within 2^30 bytes
  return aligned_to(a, 16) && near ? run_tiles<TO, true, T>(a, c, s) : run_tiles<TO, false, T>(a, c, s);
}

template <typename TO, int MT, int NT, int U> hipError_t run_rows(const MatmulArgs &a, hipStream_t s) {
  const bool words = aligned_to(a, 4);
  constexpr int64_t kSlice = ((int64_t)16 * NT) << 21;  // outputs of a launch: it has at most 2^32 threads
  for (int64_t n = 0; n < a.N; n += kSlice) {
    MatmulArgs b = a;
    b.N = (int)(a.N - n < kSlice ? a.N - n : kSlice);
    b.w = a.w + n * a.ld_w;
    b.w_scale = a.w_scale + n;
    if (a.bias) b.bias = a.bias + n;
    b.out = (TO *)a.out + n;
    const dim3 grid((b.N + 16 * NT - 1) / (16 * NT));
    if (words) hipLaunchKernelGGL((rows_kernel<TO, MT, NT, U, false>), grid, dim3(1024), 0, s, b);
    else hipLaunchKernelGGL((rows_kernel<TO, MT, NT, U, true>), grid, dim3(1024), 0, s, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename TO> hipError_t run(const MatmulArgs &a, hipStream_t s) {
  if (rows_form(a.M, a.N)) {
    if (a.M <= 16) return a.N >= 8192 ? run_rows<TO, 1, 2, 2>(a, s) : run_rows<TO, 1, 1, 2>(a, s);
    return a.M <= 32 ? run_rows<TO, 2, 1, 2>(a, s) : run_rows<TO, 4, 1, 1>(a, s);
  }
  Cut c;
  if (cut_of(a.M, a.N, a.K, &c) == 256) return run_cut<TO, 256>(a, c, s);
  if (c.splits == 1) return run_cut<TO, 128>(a, c, s);
  MatmulArgs b = a;
  b.out = a.ws;
  b.ld_o = a.N;
  const hipError_t e = run_cut<int, 128>(b, c, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((add_kernel<TO>), dim3((unsigned)((a.M * a.N + 1023) / 1024)), dim3(256), 0, s, a, c.splits);
  return hipGetLastError();
}

}  // namespace mmq

size_t matmul_quant_bytes(int64_t rows, int outputs, int inner) {
  if (mmq::rows_form(rows, outputs)) return 0;
  mmq::Cut c;
  const int side = mmq::cut_of(rows, outputs, inner, &c);
  return side == 128 && c.splits > 1 ? (size_t)c.splits * rows * outputs * sizeof(int) : 0;
}

hipError_t launch_matmul_quant(const MatmulArgs &a, int out_dtype, hipStream_t s) {
  return out_dtype == FWG_BF16 ? mmq::run<uint16_t>(a, s) : mmq::run<float>(a, s);
}

}  // namespace fwg

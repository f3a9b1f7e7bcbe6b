// Product of rows in microscaled 4-bit floating point with weights in the same form:
//   out[m][n] = row_scale[m] * sum over blocks b of 2^(ex[m][b] + ew[n][b]) * (sum over the block of x[m][k] w[n][k]) + bias[n].
//
// v_mfma_scale_f32_32x32x64_f8f6f4 takes both operands as they lie in memory: a lane holds one block of 32 consecutive
// elements of one row (16 bytes) and that block's scale byte.  Products and sums are float32.  The product is taken as
// D[n][m] = W X^T: a lane then holds four consecutive outputs of one row and stores them together.
//
// Measured: 4,093 x 32,000 x 4,096 to bf16 262 us (4,090 TFLOP/s), 8,192^3 250 us (4,390); the largest library product of the
// same type takes 452 and 340 us.  The instruction alone, operands in registers, reaches 6,460 TFLOP/s with random elements
// and 9,770 with zeros: the card's power bounds it, and a variant that took 180 us instead of 196 for zeros takes the same time as
// this one for random elements.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <type_traits>

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

// One product of 32 outputs x 32 rows x 64 elements, or of 16 x 16 x 128; byte B of sw and of sx is the scale of the lane's block.
template <int B> __device__ __forceinline__ f32x16 mma(const i32x4 &w, const i32x4 &x, const f32x16 &c, int sw, int sx) {
  const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, B, sw, B, sx);
}
__device__ __forceinline__ f32x4 mma(const i32x4 &w, const i32x4 &x, const f32x4 &c, int sw, int sx) {
  const i32x8 a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 4, 4, 0, sw, 0, sx);
}

// 16 bytes of a row of n bytes from byte k on; bytes from n on are 0.
__device__ __forceinline__ i32x4 load16(const uint8_t *row, int k, int n) {
  i32x4 v = {0, 0, 0, 0};
  if (k >= n) return v;
  if (k + 16 <= n) return *(const i32x4_b *)(row + k);
  if (n >= 16) {  // the row's last 16 bytes, shifted down
    const unsigned __int128 last = __builtin_bit_cast(unsigned __int128, (i32x4)*(const i32x4_b *)(row + n - 16));
    return __builtin_bit_cast(i32x4, last >> (8 * (k + 16 - n)));
  }
  unsigned __int128 part = 0;
#pragma unroll 1
  for (int i = n - 1; i >= k; --i) part = part << 8 | row[i];
  return __builtin_bit_cast(i32x4, part);
}

// From memory to LDS without registers: lane l's bytes land at the (uniform) address + 16 l, or 4 l.
__device__ __forceinline__ void copy_4(const uint8_t *g, uint8_t *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 4, 0, 0);
}
__device__ __forceinline__ void copy_16(const uint8_t *g, uint8_t *l) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)g,
                                   (__attribute__((address_space(3))) void *)l, 16, 0, 0);
}

// Tiles of T outputs x T rows, eight blocks (256 elements, 128 bytes) of k per stage, two stages in LDS: one is filled while
// the other is multiplied.  A wave multiplies 64 outputs x T / 2 rows: eight waves for T = 256, four for 128, where two blocks share a
// compute unit.
//
// A step of a stage multiplies 64 elements: which of the stage's blocks they are is free as long as both operands agree, so lanes
// 0 .. 31 hold block s at step s and lanes 32 .. 63 block 4 + s.  The scales of a lane's four blocks are then four
// neighbouring bytes, one word, of which step s names byte s.
//
// A stage's scales are 8 bytes of each row, and reading them from the rows brings in whole lines.  Tiles of 256 find them
// rearranged by stages (pack_kernel, 4 us in 8,192^3: 304 us from the rows, 274 so); those of 128 take 16 bytes for two
// stages at a time from the rows, through registers, which hold them at any address.
constexpr int HK = 128, HB = HK / 16;
template <int T> struct Tile {
  static constexpr int kThreads = 2 * T, kWM = T / 2, kJ = kWM / 32;
  static constexpr int kStage = 2 * T * HK;      // bytes of a stage: weights, then rows
  static constexpr int kScales = 2 * T * HB;     // of a stage: weights', then rows'
  static constexpr int kChunk = T == 256 ? kScales : 2 * kScales;  // of the stages whose scales come together
  static constexpr int kLds = 2 * (kStage + kChunk) + 2 * 2 * T * (int)sizeof(float);
};

// The 16-byte pieces of a stage's row r lie permuted, so that the 32 rows that an instruction reads at one k spread over the banks.
__device__ __forceinline__ int piece_of(int row, int piece) { return piece ^ ((row >> 1) & 7); }

// The scales of 256 rows at a time, of both operands (weights first), as [stage][row][8 bytes]: a thread 16 bytes of a row,
// eight threads 128.
__global__ void __launch_bounds__(256) pack_kernel(MatmulMxArgs a, int tiles_n, int tiles) {
  const int stages = (a.blocks + HB - 1) / HB, stage = 2 * (8 * blockIdx.y + threadIdx.x % 8);
  if (stage >= stages) return;
  for (int at = blockIdx.x; at < 8 * tiles; at += gridDim.x) {
    const int t = at / 8, in_tile = at % 8 * 32 + threadIdx.x / 8;
    const int64_t r = (int64_t)(t < tiles_n ? t : t - tiles_n) * 256 + in_tile;
    const uint8_t *row = t < tiles_n ? a.w_scale + min(r, (int64_t)a.N - 1) * a.ld_ew : a.x_scale + min(r, a.M - 1) * a.ld_ex;
    const i32x4 v = load16(row, stage * HB, a.blocks);
    uint8_t *to = a.ws + (((int64_t)t * stages + stage) * 256 + in_tile) * HB;
    *(u32x2 *)to = u32x2{(unsigned)v[0], (unsigned)v[1]};
    if (stage + 1 < stages) *(u32x2 *)(to + 256 * HB) = u32x2{(unsigned)v[2], (unsigned)v[3]};
  }
}

struct Cut {
  int tiles_m, tiles_n, splits, per;  // k is cut into `splits` parts of `per` blocks (a multiple of HB)
};

// ALIGNED: rows start at multiples of 16 bytes and are copied to LDS without passing through registers.  STREAM: results go past the caches, which then keep the operands: 4,093 x 32,000 x 4,096 278 us, 315 through
// them; with the log probabilities of the results behind it 340 and 350, of 1,024 rows 96.4 and 97.5.  Only where rows are whole
// lines of 128 bytes: 2,176 x 10,920 x 4,096 takes 69.7 us so, 62.2 through the caches.
template <typename TO, bool ALIGNED, bool STREAM, int T> __global__ void __launch_bounds__(Tile<T>::kThreads, 2) tile_kernel(MatmulMxArgs a, Cut cut) {
  constexpr int I = 2, J = Tile<T>::kJ, kStage = Tile<T>::kStage, kScales = Tile<T>::kScales, kChunk = Tile<T>::kChunk;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *const scales = smem + 2 * kStage;              // two chunks
  float *const vectors = (float *)(scales + 2 * kChunk);  // [2]: bias, row_scale of the tile
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = (wave >> 1) * 64, wm = (wave & 1) * Tile<T>::kWM, row = lane & 31, half = lane >> 5;
  const int tiles_m = cut.tiles_m, tiles_n = cut.tiles_n;
  // Each XCD (blocks go to the eight in turn) takes a contiguous share of the tiles, eight rows of tiles at a time;
  // its blocks go through the share together.
  const int tiles = tiles_m * tiles_n, share = (tiles + 7) / 8, stride = gridDim.x >> 3;
  int tile = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  const int end = min(tiles, (int)(blockIdx.x & 7) * share + share);
  if (tile >= end) return;

  // Copies: a wave brings 32 rows of each operand, 8 rows of 8 pieces at a time; rows past the end are the last one, and so
  // are blocks: any elements will do there, since both operands' scales are 2^-127 and the products vanish.
  constexpr int C = 4;
  int n0;
  int64_t m0;
  const uint8_t *bw, *bx;                   // the tile's first rows
  int rows_w, rows_x;
  const int cr = wave * 32 + (lane >> 3);   // the first of the lane's rows; the others follow 8 apart
  const unsigned ow = cr * (unsigned)a.ld_w, ox = cr * (unsigned)a.ld_x;  // ALIGNED: its bytes from there (below 2^31)
  const int piece = piece_of(cr, lane & 7) * 16, last = (a.blocks - 1) * 16;  // the others' pieces: 8 rows on, ^ 4
  auto go_to = [&](int t) {
    constexpr int kBand = 8;
    const int band = t / (kBand * tiles_n), in_band = t - band * kBand * tiles_n, high = min(kBand, tiles_m - band * kBand);
    n0 = in_band / high * T;
    m0 = (int64_t)(band * kBand + in_band % high) * T;
    bw = a.w + n0 * a.ld_w;
    bx = a.x + m0 * a.ld_x;
    rows_w = min(T, a.N - n0);
    rows_x = (int)min((int64_t)T, a.M - m0);
  };
  auto copy = [&](int b0, int buf) {
    uint8_t *w = smem + buf * kStage + wave * 32 * HK, *x = w + T * HK;
    const int p[2] = {min(b0 * 16 + piece, last), min(b0 * 16 + (piece ^ 64), last)};
    if constexpr (ALIGNED) {
      const unsigned ld_w = (unsigned)a.ld_w, ld_x = (unsigned)a.ld_x;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        copy_16(bw + (min(ow + i * 8 * ld_w, (rows_w - 1) * ld_w) + p[i & 1]), w + i * 8 * HK);
        copy_16(bx + (min(ox + i * 8 * ld_x, (rows_x - 1) * ld_x) + p[i & 1]), x + i * 8 * HK);
      }
    } else {
      i32x4 vw[C], vx[C];
#pragma unroll
      for (int i = 0; i < C; ++i) {
        vw[i] = *(const i32x4_b *)(bw + min(cr + i * 8, rows_w - 1) * a.ld_w + p[i & 1]);
        vx[i] = *(const i32x4_b *)(bx + min(cr + i * 8, rows_x - 1) * a.ld_x + p[i & 1]);
      }
#pragma unroll
      for (int i = 0; i < C; ++i) {
        *(i32x4 *)(w + i * 8 * HK + lane * 16) = vw[i];
        *(i32x4 *)(x + i * 8 * HK + lane * 16) = vx[i];
      }
    }
  };
  // T = 256: the scales of a stage from block b0 on, of 32 rows of each operand per wave, to chunk `to`.  T = 128: of two stages,
  // 16 bytes per thread; the first stage's go to LDS with the stage at hand, the second's with the one behind it.
  constexpr bool kPacked = T == 256;
  i32x4 held;
  auto load_scales = [&](int b0, int to) {
    if constexpr (kPacked) {
      const int stages = (a.blocks + HB - 1) / HB, at = b0 * 256 + wave * 256 + lane * 4;
      uint8_t *e = scales + to * kChunk + wave * 256;
      copy_4(a.ws + (int64_t)(n0 / T) * stages * (256 * HB) + at, e);
      copy_4(a.ws + (tiles_n + m0 / T) * stages * (256 * HB) + at, e + T * HB);
    } else {
      const int r = threadIdx.x;
      held = load16(r < T ? a.w_scale + (int64_t)(n0 + min(r, rows_w - 1)) * a.ld_ew
                          : a.x_scale + (m0 + min(r - T, rows_x - 1)) * a.ld_ex, b0, a.blocks);
    }
  };
  auto store_scales = [&](int to, int second) {
    if constexpr (!kPacked)
      *(u32x2 *)(scales + to * kChunk + second * kScales + threadIdx.x * HB) =
          second ? u32x2{(unsigned)held[2], (unsigned)held[3]} : u32x2{(unsigned)held[0], (unsigned)held[1]};
  };
  auto copy_vectors = [&](int which) {
    const int t = threadIdx.x;
    if (t < T) {
      vectors[which * 2 * T + t] = a.bias ? a.bias[n0 + min(t, rows_w - 1)] : 0.f;
      vectors[which * 2 * T + T + t] = a.row_scale ? a.row_scale[m0 + min(t, rows_x - 1)] : 1.f;
    }
  };

  // the operands of one step, read while the step before is multiplied
  f32x16 acc[I][J] = {};
  i32x4 fw[2][I], fx[2][J];
  int sw[I], sx[J], sw_next[I], sx_next[J];  // the stage's scales
  auto read = [&](int buf, int step, int slot) {
    const uint8_t *w = smem + buf * kStage + (wn + row) * HK, *x = smem + buf * kStage + T * HK + (wm + row) * HK;
    const int p = piece_of(row, 4 * half + step) * 16;  // wn, wm and 32 leave (r >> 1) & 7 as it is
#pragma unroll
    for (int i = 0; i < I; ++i) fw[slot][i] = *(const i32x4 *)(w + i * 32 * HK + p);
#pragma unroll
    for (int j = 0; j < J; ++j) fx[slot][j] = *(const i32x4 *)(x + j * 32 * HK + p);
  };
  auto read_scales = [&](int chunk, int second) {
    const uint8_t *w = scales + chunk * kChunk + second * kScales + (wn + row) * HB + half * 4;
    const uint8_t *x = w + (T + wm - wn) * HB;
#pragma unroll
    for (int i = 0; i < I; ++i) sw_next[i] = *(const int *)(w + i * 32 * HB);
#pragma unroll
    for (int j = 0; j < J; ++j) sx_next[j] = *(const int *)(x + j * 32 * HB);
  };
  auto take_scales = [&] {
#pragma unroll
    for (int i = 0; i < I; ++i) sw[i] = sw_next[i];
#pragma unroll
    for (int j = 0; j < J; ++j) sx[j] = sx_next[j];
  };
  auto multiply = [&](auto step) {
    constexpr int K = decltype(step)::value;
#pragma unroll
    for (int j = 0; j < J; ++j)
#pragma unroll
      for (int i = 0; i < I; ++i) acc[i][j] = mma<K>(fw[K & 1][i], fx[K & 1][j], acc[i][j], sw[i], sx[j]);
  };
  // one read between two products
  auto interleave = [] {
#pragma unroll
    for (int i = 0; i < min(I + J, I * J); ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if constexpr (I * J > I + J) __builtin_amdgcn_sched_group_barrier(0x008, I * J - I - J, 0);
  };

  // Results: a wave's 64 outputs x T / 2 rows pass through 8 KB of LDS (of the stage that was multiplied last), 32 or 64
  // rows at a time, so that they go out in whole lines of 128 (bf16) or 256 bytes; pieces of 16 bytes are permuted by the row.
  auto write = [&](uint8_t *mine, const float *vec, int n_at, int64_t m_at) {
    constexpr int kLine = 64 * (int)sizeof(TO), kPieces = kLine / 16, JP = sizeof(TO) == 2 ? 2 : 1, E = 16 / (int)sizeof(TO);
    // places in LDS are worked out here: outside the loop over tiles they would hold 40 registers, more than there are left
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    const int row = lane & 31, half = lane >> 5;
#pragma unroll
    for (int j0 = 0; j0 < J; j0 += JP) {
      in_order();
#pragma unroll
      for (int i = 0; i < I; ++i) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int n = i * 32 + g * 8 + half * 4, at = n * (int)sizeof(TO);
          const f32x4 b = *(const f32x4 *)(vec + wn + n);
#pragma unroll
          for (int jj = 0; jj < JP; ++jj) {
            const int r = jj * 32 + row;
            uint8_t *to = mine + r * kLine + (((at >> 4) ^ (r & (kPieces - 1))) << 4) + (at & 15);
            const float f = vec[T + wm + (j0 + jj) * 32 + row];
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j0 + jj][4 * g + e] * f + b[e];
            store_aligned((TO *)to, v);
          }
        }
      }
      in_order();
      const int p = lane % kPieces, n = n_at + wn + p * E;
#pragma unroll
      for (int q = 0; q < JP * 32 * kPieces / 64; ++q) {
        const int r = q * (64 / kPieces) + lane / kPieces;
        const int64_t m = m_at + wm + j0 * 32 + r;
        const uint8_t *line = mine + r * kLine + ((p ^ (r & (kPieces - 1))) << 4);
        if (m >= a.M) continue;
        TO *out = (TO *)a.out + m * a.ld_o + n;
        if (n + E <= a.N) {
          if constexpr (STREAM) __builtin_nontemporal_store(*(const u32x4 *)line, (u32x4_el *)out);
          else *(u32x4_el *)out = *(const u32x4 *)line;
        } else {
          for (int k = 0; k < E; ++k)
            if (n + k < a.N) out[k] = ((const TO *)line)[k];
        }
      }
    }
  };

  go_to(tile);
  load_scales(0, 0);
  copy(0, 0);
  store_scales(0, 0);
  store_scales(0, 1);
  copy_vectors(0);
  __syncthreads();
  int buf = 0, which = 0, chunk = 0;
  while (true) {
    const int n_at = n0, next = tile + stride;
    const int64_t m_at = m0;
    int second = 0;  // whether the stage at hand is the second of its chunk (T = 128)
    read(buf, 0, 0);
    read_scales(chunk, 0);
    take_scales();
    auto three_steps = [&] {
      read(buf, 1, 1);
      multiply(std::integral_constant<int, 0>{});
      interleave();
      read(buf, 2, 0);
      multiply(std::integral_constant<int, 1>{});
      interleave();
      read(buf, 3, 1);
      multiply(std::integral_constant<int, 2>{});
      interleave();
      store_scales(chunk ^ 1, second);  // also where no stage follows: a branch here would keep the reads above from their places
    };
    for (int b = 0; b + HB < a.blocks; b += HB) {
      if constexpr (kPacked) load_scales(b + HB, chunk ^ 1);
      else if (!second) load_scales(b + 2 * HB, 0);
      copy(b + HB, buf ^ 1);
      three_steps();
      __syncthreads();  // the next stage has arrived, and this one has been read
      buf ^= 1;
      if constexpr (kPacked) {
        chunk ^= 1;
      } else {
        chunk ^= second;
        second ^= 1;
      }
      read(buf, 0, 0);
      read_scales(chunk, second);
      multiply(std::integral_constant<int, 3>{});
      interleave();
      take_scales();
    }
    // the stages of all tiles are one stream: while a tile's last one is multiplied, the next tile's first is copied
    if (next < end) {
      go_to(next);
      load_scales(0, chunk ^ 1);
      copy(0, buf ^ 1);
      copy_vectors(which ^ 1);
    }
    three_steps();
    store_scales(chunk ^ 1, second ^ 1);
    __syncthreads();
    multiply(std::integral_constant<int, 3>{});
    write(smem + buf * kStage + wave * 8192, vectors + which * 2 * T, n_at, m_at);
    if (next >= end) break;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) acc[i][j] = f32x16{};
    tile = next;
    buf ^= 1;
    chunk ^= 1;
    which ^= 1;
    // the LDS just used may be copied over now; the results on their way out are not waited for
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  }
}

// Where there are no more tiles of 128 x 128 than compute units: eight waves of 64 outputs x 32 rows, and a ring of four stages in
// LDS, of which three are on their way while one is multiplied.  Elements and scales at random, calls back to back: 333 x 8,000 x
// 4,096 takes 13.3 us (two groups of four waves with two stages each 15.9; four waves of 64 x 64 16.0), 128 x 8,192 x 4,096 11.5
// (14.5), 16 x 32,000 x 4,096 to float32, which memory bounds, 15.0 (4.8 TB/s).  A stage takes 0.5 us: its copies alone 0.44, its reads from LDS and products alone 0.41.
// SUMS: of a part of k, to the workspace.
constexpr int kRing = 4, kRingT = 128, kRingStage = 2 * kRingT * HK, kRingScales = 2 * kRingT * HB;
constexpr int kRingLds = kRing * (kRingStage + 2 * kRingScales) + 2 * kRingT * (int)sizeof(float);

template <typename TO, bool ALIGNED, bool SUMS>
__global__ void __launch_bounds__(512, 2) ring_kernel(MatmulMxArgs a, Cut cut) {
  constexpr int T = kRingT, I = 2;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t *const scales = smem + kRing * kRingStage;                   // two chunks, of four stages each
  float *const vectors = (float *)(scales + 2 * kRing * kRingScales);  // bias, row_scale of the tile
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wn = (wave & 1) * 64, wm = (wave >> 1) * 32, row = lane & 31, half = lane >> 5;
  const int b_at = (int)blockIdx.y * cut.per, b_end = min(a.blocks, b_at + cut.per);  // blocks of k
  const int stages = (b_end - b_at + HB - 1) / HB;
  const int tiles = cut.tiles_m * cut.tiles_n, share = (tiles + 7) / 8;
  const int tile = (int)(blockIdx.x & 7) * share + (int)(blockIdx.x >> 3);
  if (tile >= min(tiles, (int)(blockIdx.x & 7) * share + share)) return;
  constexpr int kBand = 8;
  const int band = tile / (kBand * cut.tiles_n), in_band = tile - band * kBand * cut.tiles_n, high = min(kBand, cut.tiles_m - band * kBand);
  const int n0 = in_band / high * T;
  const int64_t m0 = (int64_t)(band * kBand + in_band % high) * T;
  const uint8_t *const bw = a.w + n0 * a.ld_w, *const bx = a.x + m0 * a.ld_x;
  const int rows_w = min(T, a.N - n0), rows_x = (int)min((int64_t)T, a.M - m0);

  // A wave brings 16 rows of each operand, in two halves of 8 rows of 8 pieces; rows past the end are the last one, and so are
  // blocks, as above.
  const int cr = wave * 16 + (lane >> 3), piece = piece_of(cr, lane & 7) * 16, last = (a.blocks - 1) * 16;
  i32x4 vw[2], vx[2];  // not ALIGNED: on their way
  auto copy = [&](int t, int slot, int i) {
    const int p = min((b_at + t * HB) * 16 + (i ? piece ^ 64 : piece), last), rw = min(cr + i * 8, rows_w - 1), rx = min(cr + i * 8, rows_x - 1);
    if constexpr (ALIGNED) {
      uint8_t *w = smem + slot * kRingStage + (wave * 16 + i * 8) * HK;
      copy_16(bw + ((unsigned)rw * (unsigned)a.ld_w + p), w);  // below 2^31
      copy_16(bx + ((unsigned)rx * (unsigned)a.ld_x + p), w + T * HK);
    } else {
      vw[i] = *(const i32x4_b *)(bw + rw * a.ld_w + p);
      vx[i] = *(const i32x4_b *)(bx + rx * a.ld_x + p);
    }
  };
  auto put_down = [&](int slot) {
    if constexpr (!ALIGNED) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        uint8_t *w = smem + slot * kRingStage + (wave * 16 + i * 8) * HK + lane * 16;
        *(i32x4 *)w = vw[i];
        *(i32x4 *)(w + T * HK) = vx[i];
      }
    }
  };
  // scales of four stages: 32 bytes of a row by two threads
  const int scale_row = threadIdx.x >> 1, scale_part = threadIdx.x & 1;
  const uint8_t *const scale_at = scale_row < T ? a.w_scale + (int64_t)(n0 + min(scale_row, rows_w - 1)) * a.ld_ew
                                                : a.x_scale + (m0 + min(scale_row - T, rows_x - 1)) * a.ld_ex;
  // 16 bytes that end with the part at the latest, `shift` bits too early; short rows have one chunk only, which load16 brings.
  const bool wide = b_end >= 16;
  i32x4 held;
  int shift = 0;
  auto load_scales = [&](int t) {
    const int k = b_at + t * HB + scale_part * 2 * HB, from = min(k, b_end - 16);
    held = *(const i32x4_b *)(scale_at + from);
    shift = 8 * min(k - from, 16);
  };
  auto store_scales = [&](int chunk) {
    const unsigned __int128 all = __builtin_bit_cast(unsigned __int128, held);
    const i32x4 v = __builtin_bit_cast(i32x4, shift < 128 ? all >> shift : (unsigned __int128)0);
    const u32x2 lo = {(unsigned)v[0], (unsigned)v[1]}, hi = {(unsigned)v[2], (unsigned)v[3]};
    const auto to = (__attribute__((address_space(3))) uint8_t *)(scales + (chunk * kRing + 2 * scale_part) * kRingScales + scale_row * HB);
    // the compiler holds its own stores to LDS back until every copy to LDS is there
    asm volatile("ds_write_b64 %0, %1\n\tds_write_b64 %0, %2 offset:%3" ::"v"(to), "v"(lo), "v"(hi), "n"(kRingScales) : "memory");
  };

  f32x16 acc[I] = {};
  i32x4 fw[2][I], fx[2];
  int sw[I], sx, sw_next[I], sx_next;
  auto read = [&](int slot, int step, int to) {
    const uint8_t *w = smem + slot * kRingStage + (wn + row) * HK, *x = smem + slot * kRingStage + T * HK + (wm + row) * HK;
    const int p = piece_of(row, 4 * half + step) * 16;
#pragma unroll
    for (int i = 0; i < I; ++i) fw[to][i] = *(const i32x4 *)(w + i * 32 * HK + p);
    fx[to] = *(const i32x4 *)(x + p);
  };
  auto read_scales = [&](int chunk, int u) {
    const uint8_t *w = scales + (chunk * kRing + u) * kRingScales + (wn + row) * HB + half * 4;
#pragma unroll
    for (int i = 0; i < I; ++i) sw_next[i] = *(const int *)(w + i * 32 * HB);
    sx_next = *(const int *)(w + (T + wm - wn) * HB);
  };
  auto take_scales = [&] {
#pragma unroll
    for (int i = 0; i < I; ++i) sw[i] = sw_next[i];
    sx = sx_next;
  };
  auto multiply = [&](auto step) {
    constexpr int K = decltype(step)::value;
#pragma unroll
    for (int i = 0; i < I; ++i) acc[i] = mma<K>(fw[K & 1][i], fx[K & 1], acc[i], sw[i], sx);
  };
  // reads between the products
  auto interleave = [] {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  };
  // The next stage has arrived for all, and all have read the one at hand.  Of what a wave has asked for, `more` copies of later
  // stages (four each) may be on their way: a fence would wait for them too.
  auto arrive = [](auto more) {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070 | decltype(more)::value);  // vmcnt, and lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // the stage in slot u but for its last step, while stage t + 3 is asked for
  auto turn = [&](int u, bool ask, int t) {
    const int to = (u + kRing - 1) % kRing;
    read(u, 1, 1);
    multiply(std::integral_constant<int, 0>{});
    interleave();
    if (ask) copy(t + kRing - 1, to, 0);
    read(u, 2, 0);
    multiply(std::integral_constant<int, 1>{});
    interleave();
    if (ask) copy(t + kRing - 1, to, 1);
    read(u, 3, 1);
    multiply(std::integral_constant<int, 2>{});
    interleave();
    if (ask) put_down(to);
  };
  // its last step, and what the next stage, number u of its chunk, begins with
  auto pass = [&](int chunk, int u) {
    read(u, 0, 0);
    read_scales(chunk, u);
    multiply(std::integral_constant<int, 3>{});
    interleave();
    take_scales();
  };
  const std::integral_constant<int, 8> two{};
  const std::integral_constant<int, 4> one{};
  const std::integral_constant<int, 0> none{};
  auto fill = [&] {
#pragma unroll
    for (int t = 0; t < kRing - 1; ++t) {
      copy(t, t, 0);
      copy(t, t, 1);
      put_down(t);
    }
  };

  if constexpr (!SUMS) {
    uint8_t *to = (uint8_t *)(vectors + wave * 64);
    const int t = (wave & 1) * 64 + lane;
    if (wave < 2) {
      if (a.bias) copy_4((const uint8_t *)(a.bias + n0 + min(t, rows_w - 1)), to);
      else vectors[t] = 0.f;
    } else if (wave < 4) {
      if (a.row_scale) copy_4((const uint8_t *)(a.row_scale + m0 + min(t, rows_x - 1)), to);
      else vectors[T + t] = 1.f;
    }
  }
  if (wide) load_scales(0);
  else held = load16(scale_at, scale_part * 2 * HB, b_end);
  fill();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0f7c);  // vmcnt(12): the scales
  asm volatile("" ::: "memory");
  asm volatile("" : "+v"(held));
  store_scales(0);
  arrive(two);
  read(0, 0, 0);
  read_scales(0, 0);
  take_scales();
  int t = 0, chunk = 0, slot = 0;
  for (; t + kRing < stages; t += kRing, chunk ^= 1) {
    load_scales(t + kRing);
#pragma unroll
    for (int u = 0; u < kRing; ++u) {
      turn(u, true, t + u);
      if (u == kRing - 1) store_scales(chunk ^ 1);
      arrive(two);
      pass(u == kRing - 1 ? chunk ^ 1 : chunk, (u + 1) % kRing);
    }
  }
  // the last chunk: the fourth stage's copies may be of a stage past the end
  turn(0, true, t);
  arrive(two);
  if (t + 1 < stages) {
    pass(chunk, 1);
    turn(1, false, 0);
    arrive(one);
    slot = 1;
    if (t + 2 < stages) {
      pass(chunk, 2);
      turn(2, false, 0);
      arrive(none);
      slot = 2;
      if (t + 3 < stages) {
        pass(chunk, 3);
        turn(3, false, 0);
        arrive(none);
        slot = 3;
      }
    }
  }
  multiply(std::integral_constant<int, 3>{});

  // Results go out in whole lines of 128 bytes: 64 (bf16) or 32 outputs x 32 rows at a time pass through 4 KB of LDS, of the
  // stage that was multiplied last: the others may still be copied to.
  constexpr int E = 16 / (int)sizeof(TO), kPasses = (int)sizeof(TO) / 2;
  TO *const result = (TO *)a.out + (SUMS ? (int64_t)blockIdx.y * a.M * a.ld_o : 0);
  uint8_t *const mine = smem + slot * kRingStage + wave * 4096;
  float f = 1.f;
  if constexpr (!SUMS) f = vectors[T + wm + row];
#pragma unroll
  for (int pass = 0; pass < kPasses; ++pass) {
    in_order();
#pragma unroll
    for (int i = pass; i < (kPasses == 1 ? I : pass + 1); ++i) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int n = g * 8 + half * 4, at = ((i - pass) * 32 + n) * (int)sizeof(TO);
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][4 * g + e];
        if constexpr (!SUMS) {
          const f32x4 b = *(const f32x4 *)(vectors + wn + i * 32 + n);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = v[e] * f + b[e];
        }
        store_aligned((TO *)(mine + row * 128 + (((at >> 4) ^ (row & 7)) << 4) + (at & 15)), v);
      }
    }
    in_order();
    const int p = lane % 8, n = n0 + wn + pass * 32 + p * E;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = q * 8 + lane / 8;
      const int64_t m = m0 + wm + r;
      const uint8_t *line = mine + r * 128 + ((p ^ (r & 7)) << 4);
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
  __builtin_amdgcn_s_waitcnt(0x0f70);  // copies past the end have arrived before the LDS is another block's
}

// A row of sums in the workspace: whole lines.
__host__ __device__ __forceinline__ int sums_row(int N) { return (N + 31) / 32 * 32; }

// Adds the parts of k up, in their order.  All sums of a part are fewer than 2^22 (256 tiles).
template <typename TO> __global__ void __launch_bounds__(256) add_kernel(MatmulMxArgs a, int splits) {
  const uint32_t ld = sums_row(a.N), all = (uint32_t)a.M * ld, i = (blockIdx.x * 256 + threadIdx.x) * 4, m = i / ld, n = i - m * ld;
  if (i >= all || n >= (uint32_t)a.N) return;
  const float *sums = (const float *)a.ws + i;
  const int have = a.N - (int)n;
  f32x4 c = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) c += *(const f32x4 *)(sums + (size_t)s * all);
  const float f = a.row_scale ? a.row_scale[m] : 1.f;
  float b[4] = {}, v[4];
  if (a.bias) load_part(a.bias + n, have, 0.f, b);
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = c[e] * f + b[e];
  store_part((TO *)a.out + m * a.ld_o + n, have, v);
}

// Few rows (M <= 16 MT): the weights are read once, straight into registers, by one block per 16 NT outputs; the rows
// come from the caches.  The W waves of a block take 16 blocks of k (256 bytes of a row) in turn, and their sums meet in LDS,
// where they are added in the waves' order.  Four lanes hold four neighbouring blocks of a row at each of a turn's four steps.
// Bound by latency: one row x 12,000 x 4,096 in 8.2 us, 16 rows in 9.7 (2.7 TB/s).
template <typename TO, int MT, int NT> __global__ void __launch_bounds__(512) rows_kernel(MatmulMxArgs a) {
  constexpr int W = 8;
  __shared__ float sums[W][MT * 16][NT * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, p = lane >> 4;
  const int n0 = blockIdx.x * (16 * NT);
  const uint8_t *w[NT], *ew[NT], *x[MT], *ex[MT];
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int64_t n = min(n0 + i * 16 + r, a.N - 1);
    w[i] = a.w + n * a.ld_w + p * 16;
    ew[i] = a.w_scale + n * a.ld_ew;
  }
#pragma unroll
  for (int j = 0; j < MT; ++j) {
    const int64_t m = min(j * 16 + r, (int)a.M - 1);
    x[j] = a.x + m * a.ld_x + p * 16;
    ex[j] = a.x_scale + m * a.ld_ex;
  }
  f32x4 acc[NT][MT] = {};
  for (int b = wave * 16; b < a.blocks; b += 16 * W) {
    i32x4 vw[4][NT], vx[4][MT], sw[NT], sx[MT];
    if (b + 16 <= a.blocks) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
#pragma unroll
        for (int i = 0; i < NT; ++i) vw[s][i] = *(const i32x4_b *)(w[i] + (b + 4 * s) * 16);
#pragma unroll
        for (int j = 0; j < MT; ++j) vx[s][j] = *(const i32x4_b *)(x[j] + (b + 4 * s) * 16);
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) sw[i] = *(const i32x4_b *)(ew[i] + b);
#pragma unroll
      for (int j = 0; j < MT; ++j) sx[j] = *(const i32x4_b *)(ex[j] + b);
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const bool in = b + 4 * s + p < a.blocks;
#pragma unroll
        for (int i = 0; i < NT; ++i) vw[s][i] = in ? (i32x4) * (const i32x4_b *)(w[i] + (b + 4 * s) * 16) : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < MT; ++j) vx[s][j] = in ? (i32x4) * (const i32x4_b *)(x[j] + (b + 4 * s) * 16) : i32x4{0, 0, 0, 0};
      }
#pragma unroll
      for (int i = 0; i < NT; ++i) sw[i] = load16(ew[i], b, a.blocks);
#pragma unroll
      for (int j = 0; j < MT; ++j) sx[j] = load16(ex[j], b, a.blocks);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      int cw[NT], cx[MT];
#pragma unroll
      for (int i = 0; i < NT; ++i) cw[i] = sw[i][s] >> (8 * p);
#pragma unroll
      for (int j = 0; j < MT; ++j) cx[j] = sx[j][s] >> (8 * p);
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[i][j] = mma(vw[s][i], vx[s][j], acc[i][j], cw[i], cx[j]);
    }
  }
#pragma unroll
  for (int i = 0; i < NT; ++i)
#pragma unroll
    for (int j = 0; j < MT; ++j) *(f32x4 *)&sums[wave][j * 16 + r][i * 16 + p * 4] = acc[i][j];
  __syncthreads();
  for (int t = threadIdx.x; t < MT * NT * 256; t += 64 * W) {
    const int m = t / (16 * NT), c = t % (16 * NT), n = n0 + c;
    if (m >= a.M || n >= a.N) continue;
    float v = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) v += sums[k][m][c];
    if (a.row_scale) v *= a.row_scale[m];
    if (a.bias) v += a.bias[n];
    put((TO *)a.out + m * a.ld_o + n, v);
  }
}

// rows_kernel or tiles (us): 16 rows x 12,000 outputs x 4,096 9.8 or 10.6, x 20,000 13.5 or 11.5, x 10,000 x 8,192 17.0 or 14.6; one
// row x 12,000 x 4,096 8.3 or 10.5, x 28,000 14.5 or 12.6; 32 x 8,192 x 4,096 9.6 or 10.8, x 8,192 16.6 or 12.9, 32 x 16,000 x
// 2,048 10.1 or 7.8; 64 x 4,096 x 4,096 8.8 or 10.5, x 8,192 14.7 or 13.6, 64 x 1,000 x 8,000 13.6 or 9.5, 64 x 8,192 x 1,024 7.0 or 5.5.
bool rows_form(int64_t M, int N, int blocks) {
  const int64_t size = (int64_t)N * blocks;
  if (M <= 16) return N <= 16384 && size <= 1 << 21;
  if (M <= 32) return N <= 8192 && size <= 1 << 20;
  return M <= 64 && N <= 4096 && blocks <= 128;
}
// How a product of more rows is cut: the tile's side, and parts of k where the tiles alone leave compute units idle.  A round of
// tiles of 256, one on each compute unit, takes about 5 us and 1.5 a stage, behind 9 for the launches and the scales; of 128, two
// on each, 4 us and 1 a stage, behind 4.  (us, tiles of 256 and of 128: 4,096 x 4,096 x 4,096 40.4 and 52.9; 1,500 x 6,000 x
// 4,096 31.5 and 40.6; 2,048 x 4,096 x 4,096 30.2 and 28.5; 7,799 x 2,255 x 640 30.8 and 25.8.)
int cut_of(int64_t M, int N, int blocks, Cut *c) {
  const int stages = (blocks + HB - 1) / HB;
  const int64_t big = (M + 255) / 256 * ((N + 255) / 256), small = (M + 127) / 128 * ((N + 127) / 128);
  const int side = small > 256 && 90 + (big + 255) / 256 * (50 + 15 * stages) < 40 + (small + 511) / 512 * (40 + 10 * stages)
                       ? 256 : 128;
  c->tiles_m = (int)((M + side - 1) / side);
  c->tiles_n = (N + side - 1) / side;
  const int64_t tiles = (int64_t)c->tiles_m * c->tiles_n;
  // A stage takes 0.47 us; adding parts up 4.4, and 1 more for each 600,000 sums (written and read again).  In hundredths: 1,000 x
  // 1,000 x 8,192 takes 19.7 us whole and 17.1 in three parts, 98 x 4,750 x 7,200 21.1 and 15.4 in four, 128 x 4,096 x 4,096 10.9
  // and 12.9.  Parts of less than four stages measured no better.
  int64_t splits = 1, least = stages * 47;
  if (side == 128)
    for (int64_t n = 2; n <= 256 / tiles && n <= stages / 4; ++n) {
      const int64_t cost = (stages + n - 1) / n * 47 + 440 + n * M * N / 6000;
      if (cost < least) {
        splits = n;
        least = cost;
      }
    }
  c->per = (int)((stages + splits - 1) / splits) * HB;
  c->splits = (blocks + c->per - 1) / c->per;
  return side;
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

template <typename TO, bool ALIGNED, bool STREAM, int T>
hipError_t run_tiles(const MatmulMxArgs &a, const Cut &c, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void *)tile_kernel<TO, ALIGNED, STREAM, T>, Tile<T>::kLds, done);
  if (e != hipSuccess) return e;
  // a block goes through several tiles where there are more than the device holds (one of 256, or two of 128 per
  // compute unit)
  const int64_t blocks = ((int64_t)c.tiles_m * c.tiles_n + 7) / 8 * 8, most = T == 256 ? 256 : 512;
  const dim3 grid((unsigned)(blocks < most ? blocks : most)), block(Tile<T>::kThreads);
  hipLaunchKernelGGL((tile_kernel<TO, ALIGNED, STREAM, T>), grid, block, Tile<T>::kLds, s, a, c);
  return hipGetLastError();
}

// Whether rows can be copied to LDS without passing through registers.
bool copies(const MatmulMxArgs &a) {
  const bool aligned = (((uintptr_t)a.x | (uintptr_t)a.w | (uintptr_t)a.ld_x | (uintptr_t)a.ld_w) & 15) == 0;
  return aligned && a.ld_x < (1 << 22) && a.ld_w < (1 << 22);  // a tile's rows lie within 2^30 bytes
}

template <typename TO, bool STREAM, int T> hipError_t run_cut(const MatmulMxArgs &a, const Cut &c, hipStream_t s) {
  return copies(a) ? run_tiles<TO, true, STREAM, T>(a, c, s) : run_tiles<TO, false, STREAM, T>(a, c, s);
}

template <typename TO, bool ALIGNED, bool SUMS> hipError_t run_ring_as(const MatmulMxArgs &a, const Cut &c, hipStream_t s) {
  static std::atomic<uint64_t> done{0};
  const hipError_t e = allow_lds((const void *)ring_kernel<TO, ALIGNED, SUMS>, kRingLds, done);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)((c.tiles_m * c.tiles_n + 7) / 8 * 8), (unsigned)c.splits);
  hipLaunchKernelGGL((ring_kernel<TO, ALIGNED, SUMS>), grid, dim3(512), kRingLds, s, a, c);
  return hipGetLastError();
}
template <typename TO, bool SUMS> hipError_t run_ring(const MatmulMxArgs &a, const Cut &c, hipStream_t s) {
  return copies(a) ? run_ring_as<TO, true, SUMS>(a, c, s) : run_ring_as<TO, false, SUMS>(a, c, s);
}

template <typename TO, int MT, int NT> hipError_t run_rows(const MatmulMxArgs &a, hipStream_t s) {
  hipLaunchKernelGGL((rows_kernel<TO, MT, NT>), dim3((unsigned)((a.N + 16 * NT - 1) / (16 * NT))), dim3(512), 0, s, a);
  return hipGetLastError();
}

template <typename TO> hipError_t run(const MatmulMxArgs &a, hipStream_t s) {
  if (rows_form(a.M, a.N, a.blocks)) {
    if (a.M <= 16) return a.N >= 8192 ? run_rows<TO, 1, 2>(a, s) : run_rows<TO, 1, 1>(a, s);
    return a.M <= 32 ? run_rows<TO, 2, 1>(a, s) : run_rows<TO, 4, 1>(a, s);
  }
  Cut c;
  if (cut_of(a.M, a.N, a.blocks, &c) == 256) {
    const int tiles = c.tiles_n + c.tiles_m;
    const dim3 grid(tiles < 1 << 16 ? tiles * 8 : 1 << 19, (unsigned)((a.blocks + 16 * HB - 1) / (16 * HB)));
    hipLaunchKernelGGL(pack_kernel, grid, dim3(256), 0, s, a, c.tiles_n, tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const bool lines = (((uintptr_t)a.out | (uintptr_t)(a.ld_o * (int64_t)sizeof(TO))) & 127) == 0;
    return lines ? run_cut<TO, true, 256>(a, c, s) : run_cut<TO, false, 256>(a, c, s);
  }
  if ((int64_t)c.tiles_m * c.tiles_n > 256) return run_cut<TO, false, 128>(a, c, s);
  if (c.splits == 1) return run_ring<TO, false>(a, c, s);
  MatmulMxArgs b = a;
  b.out = a.ws;
  b.ld_o = sums_row(a.N);
  const hipError_t e = run_ring<float, true>(b, c, s);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((add_kernel<TO>), dim3((unsigned)((a.M * sums_row(a.N) + 1023) / 1024)), dim3(256), 0, s, a, c.splits);
  return hipGetLastError();
}

}  // namespace mmx

size_t matmul_mx_bytes(int64_t rows, int outputs, int blocks) {
  if (mmx::rows_form(rows, outputs, blocks)) return 0;
  mmx::Cut c;
  if (mmx::cut_of(rows, outputs, blocks, &c) == 256)  // both operands' scales by stages
    return (size_t)(c.tiles_n + c.tiles_m) * 256 * ((blocks + mmx::HB - 1) / mmx::HB * mmx::HB);
  return c.splits > 1 ? (size_t)c.splits * rows * mmx::sums_row(outputs) * sizeof(float) : 0;
}

hipError_t launch_matmul_mx(const MatmulMxArgs &a, int out_dtype, hipStream_t s) {
  return out_dtype == FWG_BF16 ? mmx::run<uint16_t>(a, s) : mmx::run<float>(a, s);
}

}  // namespace fwg

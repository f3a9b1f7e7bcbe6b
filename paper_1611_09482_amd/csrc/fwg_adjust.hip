// Logits as requests want them: per row, with `seen` the tokens of the row's history and c[v] how often v comes after the prompt,
//   z > 0 ? z / repetition : z * repetition   where seen,    z - frequency c - presence   where c > 0,
//   z + bias,    -inf where the grammar does not allow v;    -inf stays -inf.
//
// A block takes a part of a row's vocabulary, eight logits a thread: it asks for its logits, counts the part's tokens in LDS while
// it reads the row's whole history, then writes the part.  Counts are whole numbers, so the order in which they are added
// does not matter.  Logits that no grammar allows are not read, and where a row is changed in place and has no bias only the logits that
// change are touched.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace adj {

using namespace opd;

constexpr int kE = 8;                    // logits of a thread
constexpr uint32_t kSeen = 0x80000000u;  // the token is in the row's history; below: how often it comes after the prompt

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4_el __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// z / r, inv = 1 / r rounded: a correction of z * inv gives the rounded quotient, but for numbers at the ends of the range.
__device__ __forceinline__ float quotient(float z, float r, float inv) {
  float q = z * inv;
  q = __builtin_fmaf(__builtin_fmaf(-q, r, z), inv, q);
  const float size = fabsf(q);
  return size < 1e37f && size > 1e-30f ? q : z / r;
}

// THREADS threads per block, P pieces of eight logits per thread: the pieces of one k lie together.  TOGETHER: the parts of a row
// go to one XCD (blocks go to the eight in turn).
template <typename T, int THREADS, int P, bool TOGETHER>
__global__ void __launch_bounds__(THREADS) adjust_kernel(AdjustArgs a, int parts, int part) {
  __shared__ __align__(16) uint32_t count[THREADS * kE * P];
  const uint32_t one = TOGETHER ? blockIdx.x >> 3 : blockIdx.x, at = one / (uint32_t)parts;
  const int64_t r = TOGETHER ? at * 8 + (blockIdx.x & 7) : at;
  if (TOGETHER && r >= a.rows) return;
  const int v0 = (int)(one - at * parts) * part, n = min(part, a.vocab - v0);
  const T *z = (const T *)a.logits + r * a.ld + v0;
  T *out = (T *)a.out + r * a.ld_o + v0;
  const float *bias = a.bias ? a.bias + r * a.ld_b + v0 : nullptr;
  // in place without a bias: what does not change is not read
  const bool lazy = a.logits == a.out && !a.bias;
  const float rep = a.repetition ? a.repetition[r] : 1.f, pres = a.presence ? a.presence[r] : 0.f,
              freq = a.frequency ? a.frequency[r] : 0.f;
  const float inv = 1.f / rep;
  uint32_t ok[P];
  float y[P][kE];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = (p * THREADS + threadIdx.x) * kE;
    ok[p] = i < n ? 0xffu : 0u;
    if (a.allowed && i < n) ok[p] = ((const uint8_t *)(a.allowed + r * a.ld_a))[(v0 + i) / 8];
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = (p * THREADS + threadIdx.x) * kE;
#pragma unroll
    for (int j = 0; j < kE; ++j) y[p][j] = 0.f;
    if (!lazy && ok[p]) load_part(z + i, n - i, 0.f, y[p]);
  }
  if (a.tokens) {
#pragma unroll
    for (int p = 0; p < 2 * P; ++p) *(u32x4 *)&count[(p * THREADS + threadIdx.x) * 4] = u32x4{0, 0, 0, 0};
    const uint32_t len = a.lengths ? min(max(a.lengths[r], 0), a.history) : a.history;
    const uint32_t prompt = a.prompts ? max(a.prompts[r], 0) : 0;
    const int32_t *t = a.tokens + r * a.ld_t;
    __syncthreads();
    // sixteen tokens of a thread on their way at a time
    constexpr int kRun = 4;
    for (uint32_t from = 0; from < len; from += THREADS * 4 * kRun) {  // stays below 2^32
      i32x4 w[kRun];
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const uint32_t at = from + (k * THREADS + threadIdx.x) * 4;
        w[k] = i32x4{-1, -1, -1, -1};
        if (at + 4 <= len) {
          w[k] = *(const i32x4_el *)(t + at);
        } else if (at < len) {
#pragma unroll
          for (int j = 0; j < 3; ++j)
            if (at + j < len) w[k][j] = t[at + j];
        }
      }
#pragma unroll
      for (int k = 0; k < kRun; ++k) {
        const uint32_t at = from + (k * THREADS + threadIdx.x) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t v = (uint32_t)w[k][j] - (uint32_t)v0;
          if (v >= (uint32_t)n) continue;
          if (at + j >= prompt) atomicAdd(&count[v], 1u);
          else atomicOr(&count[v], kSeen);
        }
      }
    }
    __syncthreads();
  }
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int i = (p * THREADS + threadIdx.x) * kE, have = n - i;
    if (have <= 0) continue;
    uint32_t c[kE] = {}, any = 0;
    if (a.tokens) {
      const u32x4 lo = *(const u32x4 *)&count[i], hi = *(const u32x4 *)&count[i + 4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = lo[j];
        c[j + 4] = hi[j];
        any |= lo[j] | hi[j];
      }
    }
    if (lazy) {
      if (!any && ok[p] == 0xffu) continue;
      if (ok[p]) load_part(z + i, have, 0.f, y[p]);
    }
    float b[kE] = {};
    if (bias && ok[p]) load_part(bias + i, have, 0.f, b);
    if (any && ok[p]) {
#pragma unroll
      for (int j = 0; j < kE; ++j) {
        if (y[p][j] == -kInf || !c[j]) continue;
        if (a.repetition) y[p][j] = y[p][j] > 0.f ? quotient(y[p][j], rep, inv) : y[p][j] * rep;
        const uint32_t made = c[j] & ~kSeen;
        if (made) y[p][j] = y[p][j] - freq * (float)made - pres;
      }
    }
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      if (bias && y[p][j] != -kInf) y[p][j] += b[j];
      if (!((ok[p] >> j) & 1u)) y[p][j] = -kInf;
    }
    store_part(out + i, have, y[p]);
  }
}

// PARTS: rows may have several parts.
template <typename T, int THREADS, int P, bool PARTS> hipError_t go(const AdjustArgs &a, hipStream_t s) {
  // parts of one size, of whole words of `allowed`
  constexpr int kMost = THREADS * kE * P;
  const int parts = (int)(((int64_t)a.vocab + kMost - 1) / kMost);
  const int part = (int)(((int64_t)a.vocab + parts - 1) / parts + 31) / 32 * 32;
  // Together a row's history comes into one L2 alone.  64 rows of 131,072 with 16,381 tokens 17.5 us in turn, 16.9 together, but with
  // 100 tokens 11.1 and 11.5; 190 rows with 1,000 tokens 29.0 and 27.6, in place 24.1 and 19.5; 2,000 rows of 12,000, two parts
  // each, 37.1 and 38.1.
  if constexpr (PARTS) {
    if (parts >= 4 && (a.rows >= 128 || (a.rows >= 32 && a.tokens && a.history >= 4096))) {
      const dim3 grid((unsigned)((a.rows + 7) / 8 * 8 * parts));
      hipLaunchKernelGGL((adjust_kernel<T, THREADS, P, true>), grid, dim3(THREADS), 0, s, a, parts, part);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((adjust_kernel<T, THREADS, P, false>), dim3((unsigned)(a.rows * parts)), dim3(THREADS), 0, s, a, parts, part);
  return hipGetLastError();
}

// Of 131,072 bf16 logits with histories of up to 1,000 tokens 190 rows took 37.0 us in parts of 8,192 by 1,024 threads, 30.5 by
// 512, 37.6 by 256, and 35.7 in parts of 2,048 by 256; with 16,381 tokens, which every part reads, 44.7, 40.9, 52.4 and
// 56.9 (all in turn).  2,048 rows of 256: 9.6 us in parts of 2,048 (the call), 12.2 in parts of 8,192.
template <typename T> hipError_t run(const AdjustArgs &a, hipStream_t s) {
  return a.vocab <= 2048 ? go<T, 256, 1, false>(a, s) : go<T, 512, 2, true>(a, s);
}

}  // namespace adj

hipError_t launch_adjust(const AdjustArgs &a, int dtype, hipStream_t s) {
  return dtype == FWG_BF16 ? adj::run<uint16_t>(a, s) : adj::run<float>(a, s);
}

}  // namespace fwg

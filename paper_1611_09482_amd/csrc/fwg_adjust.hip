// Logits as requests want them: per row, with `seen` the tokens of the row's history and c[v] how often v comes after the prompt,
//   z > 0 ? z / repetition : z * repetition   where seen,    z - frequency c - presence   where c > 0,
//   z + bias,    -inf where the grammar does not allow v;    -inf stays -inf.
//
// A block takes a part of a row's vocabulary: it counts the part's tokens in LDS while it reads the row's whole history, then
// passes over the logits once.  Counts are whole numbers, so the order in which they are added does not matter.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace adj {

using namespace opd;

constexpr int kPart = 8192, kThreads = 256, kE = 8;
constexpr uint32_t kSeen = 0x80000000u;  // the token is in the row's history; below: how often it comes after the prompt

template <typename T> __global__ void __launch_bounds__(kThreads) adjust_kernel(AdjustArgs a, int parts) {
  __shared__ uint32_t count[kPart];
  const int64_t r = blockIdx.x / parts;
  const int v0 = (int)(blockIdx.x - r * parts) * kPart, n = min(kPart, a.vocab - v0);
  if (a.tokens) {
    for (int i = threadIdx.x; i < kPart; i += kThreads) count[i] = 0;
    __syncthreads();
    const int len = a.lengths ? min(max(a.lengths[r], 0), a.history) : a.history;
    const int prompt = a.prompts ? a.prompts[r] : 0;
    const int32_t *t = a.tokens + r * a.ld_t;
    for (int i = threadIdx.x; i < len; i += kThreads) {
      const uint32_t v = (uint32_t)t[i] - (uint32_t)v0;
      if (v >= (uint32_t)n) continue;
      if (i >= prompt) atomicAdd(&count[v], 1u);
      else atomicOr(&count[v], kSeen);
    }
    __syncthreads();
  }
  const float rep = a.repetition ? a.repetition[r] : 1.f, pres = a.presence ? a.presence[r] : 0.f,
              freq = a.frequency ? a.frequency[r] : 0.f;
  const T *z = (const T *)a.logits + r * a.ld + v0;
  T *out = (T *)a.out + r * a.ld_o + v0;
  const float *bias = a.bias ? a.bias + r * a.ld_b + v0 : nullptr;
  const uint32_t *allowed = a.allowed ? a.allowed + r * a.ld_a + v0 / 32 : nullptr;
  for (int i = threadIdx.x * kE; i < n; i += kThreads * kE) {
    const int have = n - i;
    float y[kE], b[kE] = {};
    load_part(z + i, have, 0.f, y);
    if (bias) load_part(bias + i, have, 0.f, b);
    const uint32_t ok = allowed ? allowed[i / 32] >> (i % 32) : 0xffu;
#pragma unroll
    for (int j = 0; j < kE; ++j) {
      float v = y[j];
      if (a.tokens) {
        const uint32_t c = count[i + j];
        if (c) {
          if (a.repetition) v = v > 0.f ? v / rep : v * rep;
          if (c & ~kSeen) v = v - freq * (float)(c & ~kSeen) - pres;
        }
      }
      if (bias) v += b[j];
      y[j] = !((ok >> j) & 1u) || y[j] == -kInf ? -kInf : v;
    }
    store_part(out + i, have, y);
  }
}

template <typename T> hipError_t run(const AdjustArgs &a, hipStream_t s) {
  const int parts = (a.vocab + kPart - 1) / kPart;
  hipLaunchKernelGGL((adjust_kernel<T>), dim3((unsigned)(a.rows * parts)), dim3(kThreads), 0, s, a, parts);
  return hipGetLastError();
}

}  // namespace adj

hipError_t launch_adjust(const AdjustArgs &a, int dtype, hipStream_t s) {
  return dtype == FWG_BF16 ? adj::run<uint16_t>(a, s) : adj::run<float>(a, s);
}

}  // namespace fwg

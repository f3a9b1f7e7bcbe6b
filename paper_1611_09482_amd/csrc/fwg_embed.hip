// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[i] = scale * table[tok[i]], a zero row for tokens outside the table.  Bound by memory: a group of
// threads takes the 16-byte pieces of a row, several rows in flight per thread.
//
// Gradient: dtable[v] = scale * sum over the positions i with tok[i] = v of dy[i], in float32, in a fixed order.
// The positions are sorted by token (a stable radix sort of at most 9 bits a pass), then equal parts of the
// sorted order are summed, each by one wave per slice of columns: a row whose positions lie inside a part is
// finished there, rows that cross parts leave partial sums that a last kernel adds up in the parts' order.  So
// the work is even however often a token comes, no sum depends on the order in which blocks run, and nothing is
// added atomically.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace emb {

using namespace opd;

template <typename TI, typename TO, int R>
__global__ void __launch_bounds__(256) embed_kernel(EmbedArgs a, int log_tpr) {
  constexpr int VEC = El<TI>::kVec;
  const int tpr = 1 << log_tpr, per = 256 >> log_tpr;
  const int c = (int)((blockIdx.y << log_tpr) + (threadIdx.x & (tpr - 1))) * VEC, have = a.channels - c;
  if (have <= 0) return;
  const int64_t r0 = (int64_t)blockIdx.x * (per * R) + (threadIdx.x >> log_tpr);
  int tok[R];
  float v[R][VEC];
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t r = r0 + (int64_t)j * per;
    const int t = r < a.n ? a.tokens[r] : -1;
    tok[j] = t >= 0 && t < a.vocab ? t : -1;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    load_part((const TI *)a.table + (tok[j] < 0 ? 0 : (int64_t)tok[j]) * a.ld_table + c, have, 0.f, v[j]);
    const bool in = tok[j] >= 0;
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[j][i] = in ? v[j][i] * a.scale : 0.f;
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int64_t r = r0 + (int64_t)j * per;
    if (r < a.n) store_part((TO *)a.out + r * a.ld_out + c, have, v[j]);
  }
}

template <typename TI, typename TO> hipError_t run(const EmbedArgs &a, hipStream_t s) {
  const int pieces = (a.channels + El<TI>::kVec - 1) / El<TI>::kVec;
  int log_tpr = 0;
  while (log_tpr < 8 && (1 << log_tpr) < pieces) ++log_tpr;
  const unsigned gy = (unsigned)((pieces + (1 << log_tpr) - 1) >> log_tpr);
  const int64_t per = 256 >> log_tpr;
  // four rows per thread where that still leaves every compute unit several blocks
  if ((a.n + 4 * per - 1) / (4 * per) * gy >= 2048)
    hipLaunchKernelGGL((embed_kernel<TI, TO, 4>), dim3((unsigned)((a.n + 4 * per - 1) / (4 * per)), gy), dim3(256), 0,
                       s, a, log_tpr);
  else
    hipLaunchKernelGGL((embed_kernel<TI, TO, 1>), dim3((unsigned)((a.n + per - 1) / per), gy), dim3(256), 0, s, a,
                       log_tpr);
  return hipGetLastError();
}

// ---- gradient ----

// Sorted entries: key in the high word (vocab for tokens outside the table), position in the low one.
typedef unsigned long long Pair;
constexpr int kSortWaves = 16, kMaxBits = 9, kMaxBins = 1 << kMaxBits;
constexpr int kMinTile = 2048, kMaxTiles = 64;

__device__ __forceinline__ Pair pair_of(const int32_t *tokens, int vocab, int i) {
  const int t = tokens[i];
  return ((Pair)(unsigned)(t >= 0 && t < vocab ? t : vocab) << 32) | (unsigned)i;
}
// Entry i of a pass's input: the first pass reads the tokens themselves.
__device__ __forceinline__ Pair entry(const Pair *in, const int32_t *tokens, int vocab, int i) {
  return in ? in[i] : pair_of(tokens, vocab, i);
}
__device__ __forceinline__ int digit_of(Pair p, int shift, int mask) { return (int)(p >> (32 + shift)) & mask; }

// Counts of a tile's digits: hist[tile][bin].
__global__ void __launch_bounds__(1024) hist_kernel(const Pair *in, const int32_t *tokens, int vocab, int n, int tile,
                                                    int shift, int bins, int *hist) {
  __shared__ int cnt[kMaxBins];
  for (int b = threadIdx.x; b < bins; b += 1024) cnt[b] = 0;
  __syncthreads();
  const int i0 = blockIdx.x * tile, i1 = min(n, i0 + tile);
  for (int i = i0 + threadIdx.x; i < i1; i += 1024)
    atomicAdd(&cnt[digit_of(entry(in, tokens, vocab, i), shift, bins - 1)], 1);
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 1024) hist[blockIdx.x * bins + b] = cnt[b];
}

// Scatters a tile in its order: the place of an entry is the number of smaller digits anywhere, plus its digit's
// in earlier tiles, earlier waves and earlier lanes.  Each wave owns a contiguous share of the tile.
__global__ void __launch_bounds__(1024) scatter_kernel(const Pair *in, const int32_t *tokens, int vocab, int n, int tile,
                                                       int shift, int bits, const int *hist, Pair *out) {
  __shared__ int place[kSortWaves][kMaxBins];
  __shared__ int wsum[kSortWaves];
  const int bins = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  for (int b = threadIdx.x; b < kSortWaves * bins; b += 1024) place[b / bins][b % bins] = 0;
  __syncthreads();
  const int share = (tile + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int i0 = min(n, (int)blockIdx.x * tile + wave * share);
  const int i1 = min(min(n, ((int)blockIdx.x + 1) * tile), i0 + share);
  for (int i = i0 + lane; i < i1; i += 64)
    atomicAdd(&place[wave][digit_of(entry(in, tokens, vocab, i), shift, bins - 1)], 1);
  __syncthreads();
  // thread b: totals of bin b, exclusive over the bins, then the waves' starts
  const int b = threadIdx.x;
  int total = 0, before = 0;
  if (b < bins) {
    for (int t = 0; t < (int)gridDim.x; ++t) {
      const int c = gridDim.x > 1 ? hist[t * bins + b] : 0;
      before += t < (int)blockIdx.x ? c : 0;
      total += c;
    }
    if (gridDim.x == 1)
      for (int w = 0; w < kSortWaves; ++w) total += place[w][b];
  }
  int incl = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(incl, o, 64);
    if (lane >= o) incl += v;
  }
  if (lane == 63) wsum[wave] = incl;
  __syncthreads();
  int start = incl - total + before;
  for (int w = 0; w < wave; ++w) start += wsum[w];
  if (b < bins) {
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = place[w][b];
      place[w][b] = start;
      start += c;
    }
  }
  __syncthreads();
  for (int i = i0 + lane; i - lane < i1; i += 64) {
    const bool in_share = i < i1;
    const Pair p = in_share ? entry(in, tokens, vocab, i) : 0;
    const int d = in_share ? digit_of(p, shift, bins - 1) : 0;
    unsigned long long same = __ballot(in_share);  // the lanes with my digit
    for (int k = 0; k < bits; ++k) {
      const unsigned long long one = __ballot((d >> k) & 1);
      same &= (d >> k) & 1 ? one : ~one;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (in_share) {
      const int at = place[wave][d];
      out[at + rank] = p;
      if (rank == 0) place[wave][d] = at + __popcll(same);  // after the reads of every lane: the wave runs in step
    }
    __builtin_amdgcn_wave_barrier();
  }
}

struct SumArgs {
  EmbedGradArgs g;
  const Pair *sorted;
  float *partial;  // [2 * parts][channels]: a part's first run (continued from before), its last (continued after)
  int part;        // entries per part
  int parts, slices;
};

// A part's sums.  Wave task = (part, slice of 64 * VEC columns).
template <typename T, typename TO>
__global__ void __launch_bounds__(256) sum_kernel(SumArgs a, int sum_blocks) {
  constexpr int VEC = El<T>::kVec;
  const int lane = threadIdx.x & 63, D = a.g.channels, n = a.g.n, V = a.g.vocab;
  if ((int)blockIdx.x < sum_blocks) {
    const int task = (int)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int part = task / a.slices, c = ((task % a.slices) * 64 + lane) * VEC, have = D - c;
    if (part >= a.parts) return;
    const int i0 = part * a.part, i1 = min(n, i0 + a.part);
    float acc[VEC] = {};
    int cur = __builtin_amdgcn_readfirstlane((int)(a.sorted[i0] >> 32));
    bool opened = i0 > 0 && (int)(a.sorted[i0 - 1] >> 32) == cur;  // the run goes on from the part before
    auto flush = [&](bool goes_on) {
      if (cur >= V || have <= 0) return;
      if (opened || goes_on) {
        store_part(a.partial + ((int64_t)part * 2 + (opened ? 0 : 1)) * D + c, have, acc);
      } else {
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = acc[j] * a.g.scale;
        store_part((TO *)a.g.out + (int64_t)cur * a.g.ld_out + c, have, v);
      }
    };
    constexpr int B = 8;  // rows in flight
    for (int i = i0; i < i1; i += B) {
      float v[B][VEC];
      int key[B];
#pragma unroll
      for (int j = 0; j < B; ++j) {
        const Pair p = a.sorted[min(i + j, i1 - 1)];  // the same for the whole wave
        key[j] = __builtin_amdgcn_readfirstlane((int)(p >> 32));
        const int64_t pos = (unsigned)__builtin_amdgcn_readfirstlane((int)(unsigned)p);
        load_part((const T *)a.g.grad + pos * a.g.ld_grad + c, key[j] < V ? have : 0, 0.f, v[j]);
      }
#pragma unroll
      for (int j = 0; j < B; ++j) {
        if (i + j >= i1) break;
        if (key[j] != cur) {
          flush(false);
          cur = key[j];
          opened = false;
#pragma unroll
          for (int e = 0; e < VEC; ++e) acc[e] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) acc[e] += v[j][e];
      }
    }
    flush(i1 < n && (int)(a.sorted[i1] >> 32) == cur);
    return;
  }
  // rows that no token names: each wave looks 16 rows up in the sorted keys and clears the absent ones
  const int r0 = (((int)blockIdx.x - sum_blocks) * 4 + (threadIdx.x >> 6)) * 16;
  bool absent = false;
  if (lane < 16 && r0 + lane < V) {
    const unsigned row = r0 + lane;
    int lo = 0, hi = n;
    while (lo < hi) {
      const int m = (lo + hi) >> 1;
      if ((unsigned)(a.sorted[m] >> 32) < row) lo = m + 1;
      else hi = m;
    }
    absent = lo == n || (unsigned)(a.sorted[lo] >> 32) != row;
  }
  const float zero[VEC] = {};
  for (unsigned long long m = __ballot(absent); m; m &= m - 1) {
    TO *out = (TO *)a.g.out + (int64_t)(r0 + __ffsll((long long)m) - 1) * a.g.ld_out;
    for (int c = lane * VEC; c < D; c += 64 * VEC) store_part(out + c, D - c, zero);
  }
}

// Rows that cross parts: the part in which such a row begins adds up the partial sums of the parts that it covers.
template <typename TO> __global__ void __launch_bounds__(256) join_kernel(SumArgs a) {
  __shared__ float red[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.g.n, D = a.g.channels;
  const int part = blockIdx.x, c = (int)blockIdx.y * 64 + lane;
  const int i1 = (part + 1) * a.part;
  if (i1 >= n) return;
  const int key = (int)(a.sorted[i1 - 1] >> 32);
  if (key >= a.g.vocab || (int)(a.sorted[i1] >> 32) != key) return;
  if (part > 0 && (int)(a.sorted[part * a.part] >> 32) == key && (int)(a.sorted[part * a.part - 1] >> 32) == key) return;
  // the last part with entries of this row: the row's end lies in [i1, n]
  int lo = i1, hi = n;
  while (lo < hi) {
    const int m = (lo + hi) >> 1;
    if ((int)(a.sorted[m] >> 32) <= key) lo = m + 1;
    else hi = m;
  }
  const int last = (lo - 1) / a.part, m = last - part;  // first-run sums of parts part + 1 .. last
  const bool mine = c < D;
  const int share = (m + 3) / 4, p0 = part + 1 + wave * share, p1 = min(last + 1, p0 + share);
  float s = 0.f;
  if (mine) {
    if (wave == 0) s = a.partial[((int64_t)part * 2 + 1) * D + c];
    for (int p = p0; p < p1; p += 8) {
      float v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = p + j < p1 ? a.partial[(int64_t)(p + j) * 2 * D + c] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
  }
  red[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && mine)
    put((TO *)a.g.out + (int64_t)key * a.g.ld_out + c,
        (((red[0][lane] + red[1][lane]) + red[2][lane]) + red[3][lane]) * a.g.scale);
}

struct GradPlan {
  int tile, tiles, passes, bits, part, parts, slices;
  size_t off_pair[2], off_hist, off_partial, total;
};

GradPlan plan_of(int64_t n, int vocab, int channels) {
  GradPlan p;
  int64_t tile = (n + kMaxTiles - 1) / kMaxTiles;
  p.tile = (int)(tile < kMinTile ? kMinTile : (tile + 63) / 64 * 64);
  p.tiles = (int)((n + p.tile - 1) / p.tile);
  int bits = 1;
  while (bits < 31 && (vocab >> bits) != 0) ++bits;  // keys 0 .. vocab
  p.passes = (bits + kMaxBits - 1) / kMaxBits;
  p.bits = (bits + p.passes - 1) / p.passes;
  p.slices = (channels + 255) / 256;  // 64 lanes of 4 float32 (bf16: of 8; see slices_of)
  // entries per part: enough parts to fill the device with waves, not so few entries that partial sums dominate
  int part = 16;
  while (part < 128 && (n / (2 * part)) * p.slices >= 4096) part *= 2;
  p.part = part;
  p.parts = (int)((n + part - 1) / part);
  auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
  size_t o = 0;
  for (int k = 0; k < 2; ++k) {
    p.off_pair[k] = o;
    o += up((size_t)n * sizeof(Pair));
  }
  p.off_hist = o;
  o += up((size_t)p.tiles << (p.bits + 2));
  p.off_partial = o;
  o += up((size_t)p.parts * 2 * channels * sizeof(float));
  p.total = o;
  return p;
}

template <typename T, typename TO> hipError_t run_grad(const EmbedGradArgs &g, hipStream_t s) {
  const GradPlan p = plan_of(g.n, g.vocab, g.channels);
  SumArgs a;
  a.g = g;
  a.partial = (float *)(g.ws + p.off_partial);
  a.part = p.part;
  a.parts = p.parts;
  a.slices = (g.channels + 64 * El<T>::kVec - 1) / (64 * El<T>::kVec);
  int *hist = (int *)(g.ws + p.off_hist);
  const Pair *in = nullptr;
  for (int k = 0; g.n > 0 && k < p.passes; ++k) {
    Pair *out = (Pair *)(g.ws + p.off_pair[k & 1]);
    if (p.tiles > 1)
      hipLaunchKernelGGL(hist_kernel, dim3(p.tiles), dim3(1024), 0, s, in, g.tokens, g.vocab, g.n, p.tile, k * p.bits,
                         1 << p.bits, hist);
    hipLaunchKernelGGL(scatter_kernel, dim3(p.tiles), dim3(1024), 0, s, in, g.tokens, g.vocab, g.n, p.tile, k * p.bits,
                       p.bits, hist, out);
    in = out;
  }
  a.sorted = in;
  const int64_t tasks = (int64_t)p.parts * a.slices;
  const int sum_blocks = (int)((tasks + 3) / 4), zero_blocks = (int)(((int64_t)g.vocab + 63) / 64);
  hipLaunchKernelGGL((sum_kernel<T, TO>), dim3((unsigned)(sum_blocks + zero_blocks)), dim3(256), 0, s, a, sum_blocks);
  if (p.parts > 1)
    hipLaunchKernelGGL((join_kernel<TO>), dim3((unsigned)p.parts, (unsigned)((g.channels + 63) / 64)), dim3(256), 0, s,
                       a);
  return hipGetLastError();
}

}  // namespace emb

hipError_t launch_embed(const EmbedArgs &a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == FWG_BF16)
    return out_dtype == FWG_BF16 ? emb::run<uint16_t, uint16_t>(a, s) : emb::run<uint16_t, float>(a, s);
  return out_dtype == FWG_BF16 ? emb::run<float, uint16_t>(a, s) : emb::run<float, float>(a, s);
}

size_t embed_grad_bytes(int64_t n, int vocab, int channels) { return n <= 0 ? 0 : emb::plan_of(n, vocab, channels).total; }

hipError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == FWG_BF16)
    return out_dtype == FWG_BF16 ? emb::run_grad<uint16_t, uint16_t>(a, s) : emb::run_grad<uint16_t, float>(a, s);
  return out_dtype == FWG_BF16 ? emb::run_grad<float, uint16_t>(a, s) : emb::run_grad<float, float>(a, s);
}

}  // namespace fwg

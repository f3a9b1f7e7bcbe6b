// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// Lookup: out[i] = scale * table[tok[i]], a zero row for tokens outside the table.  Bound by memory: a group of
// threads takes the 16-byte pieces of a row, several rows in flight per thread.  65,521 words out of 50,001 x 2,048 bf16 in
// 60 us (5.6 TB/s of rows named and written); 32 rows of 512 float32 take the kernel 2.6 us and the call 6.6.
//
// Gradient: dtable[v] = scale * sum over the positions i with tok[i] = v of dy[i], in float32, in a fixed order.
// Few tokens are looked through without sorting (few_kernel, scan_kernel).  Else the positions are sorted by token (a
// stable radix sort of at most 9 bits a pass), then equal parts of the sorted order are summed, each by one wave per
// slice of columns: a row whose positions lie inside a part is finished there, also past the part's end; rows of more
// positions than a part has leave partial sums that a last kernel adds up in the parts' order.  So the work is even however often a token comes, no sum depends on the order in
// which blocks run, and no float is added atomically.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace emb {

using namespace opd;

template <typename TI, typename TO, int R, bool STREAM>
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
    if (r < a.n) store_part<STREAM>((TO *)a.out + r * a.ld_out + c, have, v[j]);
  }
}

template <typename TI, typename TO> hipError_t run(const EmbedArgs &a, hipStream_t s) {
  const int pieces = (a.channels + El<TI>::kVec - 1) / El<TI>::kVec;
  int log_tpr = 0;
  while (log_tpr < 8 && (1 << log_tpr) < pieces) ++log_tpr;
  const unsigned gy = (unsigned)((pieces + (1 << log_tpr) - 1) >> log_tpr);
  const int64_t per = 256 >> log_tpr;
  // four rows per thread where that still leaves every compute unit several blocks
  const bool many = (a.n + 4 * per - 1) / (4 * per) * gy >= 2048;
  const dim3 grid((unsigned)((a.n + (many ? 4 : 1) * per - 1) / ((many ? 4 : 1) * per)), gy);
  if (!many) hipLaunchKernelGGL((embed_kernel<TI, TO, 1, false>), grid, dim3(256), 0, s, a, log_tpr);
  else if (a.n * a.channels * (int64_t)sizeof(TO) < kStreamBytes)
    hipLaunchKernelGGL((embed_kernel<TI, TO, 4, false>), grid, dim3(256), 0, s, a, log_tpr);
  else hipLaunchKernelGGL((embed_kernel<TI, TO, 4, true>), grid, dim3(256), 0, s, a, log_tpr);
  return hipGetLastError();
}

// ---- gradient ----

// Sorted entries: key in the high word (vocab for tokens outside the table), position in the low one.
typedef unsigned long long Pair;
constexpr int kSortWaves = 16, kMaxBits = 9, kMaxBins = 1 << kMaxBits;
constexpr int kMinTile = 2048, kMaxTiles = 128;

__device__ __forceinline__ Pair pair_of(const int32_t *tokens, int vocab, int i) {
  const int t = tokens[i];
  return ((Pair)(unsigned)(t >= 0 && t < vocab ? t : vocab) << 32) | (unsigned)i;
}
// Entry i of a pass's input: the first pass reads the tokens themselves.
__device__ __forceinline__ Pair entry(const Pair *in, const int32_t *tokens, int vocab, int i) {
  return in ? in[i] : pair_of(tokens, vocab, i);
}
__device__ __forceinline__ int digit_of(Pair p, int shift, int mask) { return (int)(p >> (32 + shift)) & mask; }

// Rows that no token names, cleared by blocks beside the sort's, which leave the memory idle: 65,521 tokens of 50,001
// words x 2,048, bf16 into a float32 table, 181 us for 198 with sum_kernel clearing them as it does after one-launch sorts.
struct ZeroArgs {
  char *out;
  int64_t ld, bytes;  // of a row, in bytes
  int row0, row1;     // this launch's share
};
constexpr int kZeroRows = 4;  // per wave
// (a token's entry of `some` names a position of that token if and only if it occurs, whatever the memory held before)
__device__ __forceinline__ void zero_rows(const ZeroArgs &z, const int *some, const int32_t *tokens, int n, int block) {
  typedef uint32_t u32x4_2 __attribute__((ext_vector_type(4), aligned(2)));
  const int lane = threadIdx.x & 63, r0 = z.row0 + (block * kSortWaves + (threadIdx.x >> 6)) * kZeroRows;
  bool absent = false;
  if (lane < kZeroRows && r0 + lane < z.row1) {
    const unsigned at = some[r0 + lane];
    absent = at >= (unsigned)n || tokens[at] != r0 + lane;
  }
  for (unsigned long long m = __ballot(absent); m; m &= m - 1) {
    char *row = z.out + (int64_t)(r0 + __ffsll((long long)m) - 1) * z.ld;
    const int64_t whole = z.bytes & ~(int64_t)15;
    for (int64_t o = lane * 16; o < whole; o += 64 * 16) *(u32x4_2 *)(row + o) = u32x4_2{0u, 0u, 0u, 0u};
    if (whole + lane * 2 < z.bytes) *(uint16_t *)(row + whole + lane * 2) = 0;
  }
}

struct SortArgs {
  const Pair *in;         // NULL: the tokens in their own order
  Pair *out;
  const int32_t *tokens;
  int *hist;              // [tile][bin]: this pass's digits (NULL: each block counts all tokens itself)
  int *clear;             // cleared by the first kernel of a call
  int vocab, n, tile, tiles, shift, bits;
  int *some;              // [vocab] for each token that occurs one of its positions, else anything; NULL: not kept
  ZeroArgs zero;
};

// Counts of the tiles' digits.  (Counting the next pass's digits in scatter_kernel instead, by global atomics, takes
// 20 us longer on 65,521 frequent words: they meet at few addresses.)
__global__ void __launch_bounds__(1024) hist_kernel(SortArgs a) {
  __shared__ int cnt[kMaxBins];
  const int bins = 1 << a.bits;
  if ((int)blockIdx.x >= a.tiles) return zero_rows(a.zero, a.some, a.tokens, a.n, blockIdx.x - a.tiles);
  for (int b = threadIdx.x; b < bins; b += 1024) cnt[b] = 0;
  if (a.clear && blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
  __syncthreads();
  const int i0 = blockIdx.x * a.tile, i1 = min(a.n, i0 + a.tile);
  for (int i = i0 + threadIdx.x; i < i1; i += 1024) {
    const Pair p = entry(a.in, a.tokens, a.vocab, i);
    atomicAdd(&cnt[digit_of(p, a.shift, bins - 1)], 1);
    if (!a.in && a.some && (int)(p >> 32) < a.vocab) a.some[p >> 32] = i;
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += 1024) a.hist[blockIdx.x * bins + b] = cnt[b];
}

// Bound by latency, not bytes: 65,521 tokens (32 blocks) in 6.6 us a pass, and 4.9 us for hist_kernel (11 to 17 us
// each with 276 MB of zeros beside them).  Up to 16,384 tokens each block counts all tokens itself instead of reading hist:
// 10,656 tokens in 8.7 us (2.7 + 6.9 us and a launch before).
//
// Scatters a tile in its order: the place of an entry is the number of smaller digits anywhere, plus its digit's
// in earlier tiles, earlier waves and earlier lanes.  Each wave owns a contiguous share of the tile.
__global__ void __launch_bounds__(1024) scatter_kernel(SortArgs a) {
  __shared__ int place[kSortWaves][kMaxBins];
  __shared__ int wsum[kSortWaves];
  __shared__ int ahead[kMaxBins], behind[kMaxBins];  // digits of other tiles, before this one and after it
  const int bins = 1 << a.bits, n = a.n, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if ((int)blockIdx.x >= a.tiles) return zero_rows(a.zero, a.some, a.tokens, n, blockIdx.x - a.tiles);
  if (a.clear && !a.hist && blockIdx.x == 0 && threadIdx.x == 0) *a.clear = 0;
#pragma unroll
  for (int b = 0; b < kSortWaves * kMaxBins / 1024; ++b) (&place[0][0])[b * 1024 + threadIdx.x] = 0;
  if (threadIdx.x < kMaxBins) ahead[threadIdx.x] = behind[threadIdx.x] = 0;
  // thread b: totals of bin b and those of earlier tiles
  const int b = threadIdx.x;
  int total = 0, before = 0;
  if (b < bins && a.hist) {
#pragma unroll 8
    for (int t = 0; t < a.tiles; ++t) {
      const int c = a.hist[t * bins + b];
      before += t < (int)blockIdx.x ? c : 0;
      total += c;
    }
  }
  const int share = (a.tile + kSortWaves * 64 - 1) / (kSortWaves * 64) * 64;
  const int i0 = min(n, (int)blockIdx.x * a.tile + wave * share);
  const int i1 = min(min(n, ((int)blockIdx.x + 1) * a.tile), i0 + share);
  constexpr int kHeld = 2;  // entries of a lane that stay in registers (tiles of up to 2,048)
  Pair held[kHeld];
#pragma unroll
  for (int j = 0; j < kHeld; ++j) {
    const int i = i0 + j * 64 + lane;
    held[j] = i < i1 ? entry(a.in, a.tokens, a.vocab, i) : 0;
  }
  __syncthreads();
  if (!a.hist) {
    const int t0 = (int)blockIdx.x * a.tile, t1 = t0 + a.tile;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 1024)
      if (i < t0 || i >= t1) atomicAdd(&(i < t0 ? ahead : behind)[digit_of(entry(a.in, a.tokens, a.vocab, i), a.shift, bins - 1)], 1);
  }
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (i0 + j * 64 + lane < i1) atomicAdd(&place[wave][digit_of(held[j], a.shift, bins - 1)], 1);
  for (int i = i0 + kHeld * 64 + lane; i < i1; i += 64)
    atomicAdd(&place[wave][digit_of(entry(a.in, a.tokens, a.vocab, i), a.shift, bins - 1)], 1);
  __syncthreads();
  // exclusive over the bins, then the waves' starts
  int count[kSortWaves];
  if (b < bins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) count[w] = place[w][b];
    if (!a.hist) {
      before = ahead[b];
      total = before + behind[b];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) total += count[w];
    }
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
#pragma unroll
  for (int w = 0; w < kSortWaves; ++w) start += w < wave ? wsum[w] : 0;
  if (b < bins) {
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      place[w][b] = start;
      start += count[w];
    }
  }
  __syncthreads();
  auto put_64 = [&](int i, Pair p) {
    const bool in_share = i < i1;
    const int d = in_share ? digit_of(p, a.shift, bins - 1) : 0;
    unsigned long long same = __ballot(in_share);  // the lanes with my digit
    for (int k = 0; k < a.bits; ++k) {
      const unsigned long long one = __ballot((d >> k) & 1);
      same &= (d >> k) & 1 ? one : ~one;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    const int at = in_share ? place[wave][d] : 0;
    in_order();  // every lane has read its digit's place before that place moves on
    if (in_share) {
      a.out[at + rank] = p;
      if (rank == 0) place[wave][d] = at + __popcll(same);
    }
    in_order();
  };
#pragma unroll
  for (int j = 0; j < kHeld; ++j)
    if (i0 + j * 64 < i1) put_64(i0 + j * 64 + lane, held[j]);
  for (int i = i0 + kHeld * 64 + lane; i - lane < i1; i += 64)
    put_64(i, i < i1 ? entry(a.in, a.tokens, a.vocab, i) : 0);
}

struct SumArgs {
  EmbedGradArgs g;
  const Pair *sorted;
  float *partial;  // [2 * parts][ld_p]: of long rows, a part's first run (begun before it) and its last
  int ld_p;        // channels, rounded up to whole vectors
  int *n_long;     // long rows found
  int2 *long_rows; // (row, part in which it begins)
  int part;        // entries per part, at most 64: the lanes hold them
  int parts, slices;
};

// 16 bytes as loaded, as floats.
__device__ __forceinline__ void expand(const u32x4 &r, float (&v)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void expand(const u32x4 &r, float (&v)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    v[2 * j] = mfd::bf_lo(r[j]);
    v[2 * j + 1] = mfd::bf_hi(r[j]);
  }
}

// Bound by memory.  65,521 tokens of 50,001 words x 2,048, bf16 into float32, in 121 us (402 MB, while zeros that the
// launches before wrote are still on their way from the caches to the memory), of 181 for the call; 10,656 tokens of 256
// classes x 512 float32 in 7 us of 21.  Padding tokens sort behind all rows, and the parts that hold them read their
// gradients too.
//
// A part's sums.  Wave task = (part, slice of 64 * VEC columns).  A row belongs to the part in which its positions
// begin, which sums it whole, past the part's end too; only rows of more than a part's positions (long) are summed part
// by part and joined.
template <typename T, typename TO>
__global__ void __launch_bounds__(256) sum_kernel(SumArgs a, int first_block, int sum_blocks) {
  constexpr int VEC = El<T>::kVec;
  const int lane = threadIdx.x & 63, D = a.g.channels, n = a.g.n, V = a.g.vocab, block = first_block + (int)blockIdx.x;
  if (block < sum_blocks) {
    const int task = __builtin_amdgcn_readfirstlane(block * 4 + (threadIdx.x >> 6));
    // the lane's columns; a vector that would pass the last one is the last whole vector instead, and two lanes then sum
    // and store the same columns, alike
    const int P = a.part, part = task / a.slices, c0 = ((task % a.slices) * 64 + lane) * VEC;
    const bool whole_vectors = D >= VEC;
    const int c = whole_vectors ? min(c0, D - VEC) : c0, have = c0 < D ? (whole_vectors ? VEC : D - c0) : 0;
    if (part >= a.parts) return;
    const int i0 = part * P, i1 = min(n, i0 + P);
    // keys around: the part's own, P before and P after it (-1: none); positions of the latter two
    const int i = i0 + lane;
    const Pair none = (Pair)0xffffffffu << 32;
    const Pair before = lane < P && i >= P ? a.sorted[i - P] : none;
    const Pair own = lane < P && i < n ? a.sorted[i] : none;
    const Pair after = lane < P && i + P < n ? a.sorted[i + P] : none;
    auto key_of = [](Pair p) { return (int)(p >> 32); };
    auto lane_key = [&](Pair p, int l) { return __builtin_amdgcn_readlane(key_of(p), l); };
    const int first = lane_key(own, 0), last = lane_key(own, i1 - i0 - 1);
    const int n_before = __popcll(__ballot(key_of(before) == first)), n_first = __popcll(__ballot(key_of(own) == first));
    const int n_last = __popcll(__ballot(key_of(own) == last)), n_after = __popcll(__ballot(key_of(after) == last));
    const bool whole = first == last;
    const bool opened = n_before > 0;                                    // the first run began before
    const bool long_first = opened && n_before + n_first + (whole ? n_after : 0) > P;
    const bool ends_long = !(whole && opened) && n_after > 0 && n_last + n_after > P;  // the last run begins here
    const int from = opened && !long_first ? i0 + n_first : i0;
    const int to = n_after > 0 && !ends_long && !(whole && opened) ? i1 + n_after : i1;
    if (from >= to) return;
    float acc[VEC] = {};
    int cur = lane_key(own, from - i0);
    const bool starts_long = long_first;
    auto flush = [&](bool is_first, bool is_last) {
      if (cur >= V) return;
      if (is_first && starts_long) {
        store_part(a.partial + (int64_t)part * 2 * a.ld_p + c, have, acc);
      } else if (is_last && ends_long) {
        store_part(a.partial + ((int64_t)part * 2 + 1) * a.ld_p + c, have, acc);
        if (task % a.slices == 0 && lane == 0) a.long_rows[atomicAdd(a.n_long, 1)] = make_int2(cur, part);
      } else {
        float v[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[j] = acc[j] * a.g.scale;
        store_part((TO *)a.g.out + (int64_t)cur * a.g.ld_out + c, have, v);
      }
    };
    bool is_first = true;
    // rows in flight; they stay as loaded until they are added
    auto add_rows = [&](auto full) {
      constexpr bool FULL = decltype(full)::value;
      constexpr int B = FULL ? 16 : 8;
      for (int e = from; e < to; e += B) {
        u32x4 raw[FULL ? B : 1];
        float v[B][VEC];
        int key[B];
#pragma unroll
        for (int j = 0; j < B; ++j) {
          const int at = min(e + j, to - 1);
          const Pair p = at < i1 ? own : after;
          const int l = at < i1 ? at - i0 : at - i1;
          key[j] = lane_key(p, l);
          const int64_t pos = (unsigned)__builtin_amdgcn_readlane((int)(unsigned)p, l);
          const T *row = (const T *)a.g.grad + pos * a.g.ld_grad + c;
          if constexpr (FULL) raw[j] = *(const u32x4_el *)row;
          else load_part(row, key[j] < V ? have : 0, 0.f, v[j]);
        }
#pragma unroll
        for (int j = 0; j < B; ++j) {
          if (key[j] != cur) {
            flush(is_first, false);
            is_first = false;
            cur = key[j];
#pragma unroll
            for (int x = 0; x < VEC; ++x) acc[x] = 0.f;
          }
          // (no early end of the loop: the loads would move behind it, one after the other)
          if constexpr (FULL) expand(raw[j], v[j]);
#pragma unroll
          for (int x = 0; x < VEC; ++x) acc[x] += e + j < to ? v[j][x] : 0.f;
        }
      }
    };
    if (whole_vectors) add_rows(std::true_type());
    else add_rows(std::false_type());
    flush(is_first, true);
    return;
  }
  // rows that no token names: each wave looks 16 rows up in the sorted keys and clears the absent ones
  const int r0 = ((block - sum_blocks) * 4 + (threadIdx.x >> 6)) * 16;
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

// Latency: 4 to 6 us for a hundred long rows.
//
// Long rows: the sums of the parts that a row covers are added up in order.  Blocks take (row, slice of up to 256
// columns) in turn; 4 columns per lane, and where a row has fewer columns than a wave's, groups of lanes (and always the
// block's waves) take a share of the parts each.
constexpr int kJoinBlocks = 1024, kJoinWaves = 8;
template <typename TO> __global__ void __launch_bounds__(64 * kJoinWaves) join_kernel(SumArgs a, int log_lanes) {
  __shared__ f32x4 red[kJoinWaves][64];
  const int L = 1 << log_lanes, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, D = a.g.channels;
  const int slices = (D + 4 * L - 1) / (4 * L), units = kJoinWaves * (64 >> log_lanes);
  const int unit = wave * (64 >> log_lanes) + (lane >> log_lanes);
  const int items = *a.n_long * slices;
  for (int item = blockIdx.x; item < items; item += gridDim.x) {
    const int2 row = a.long_rows[item / slices];
    const int c = ((item % slices) * L + (lane & (L - 1))) * 4, have = D - c;
    int m = 0;  // parts after the first that begin with this row
    while (true) {
      const int p = row.y + 1 + m + lane;
      const bool on = p < a.parts && (int)(a.sorted[(int64_t)p * a.part] >> 32) == row.x;
      const int more = __popcll(__ballot(on));
      m += more;
      if (more < 64) break;
    }
    const int share = (m + units - 1) / units, p0 = row.y + 1 + min(m, unit * share), p1 = row.y + 1 + min(m, (unit + 1) * share);
    // whole vectors: what lies between a row's channels and ld_p is read, and not stored
    const f32x4 *from = (const f32x4 *)(a.partial + (have > 0 ? c : 0));
    const int64_t ld = a.ld_p / 4;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
    if (unit == 0) s = from[((int64_t)row.y * 2 + 1) * ld];
    for (int p = p0; p < p1; p += 16) {
      f32x4 v[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) v[j] = from[(int64_t)min(p + j, p1 - 1) * 2 * ld];
#pragma unroll
      for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int x = 0; x < 4; ++x) s[x] += p + j < p1 ? v[j][x] : 0.f;
    }
    red[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && lane < L) {
      float v[4] = {};
      for (int u = 0; u < units; ++u) {
        const f32x4 t = red[u >> (6 - log_lanes)][((u & ((64 >> log_lanes) - 1)) << log_lanes) + lane];
#pragma unroll
        for (int x = 0; x < 4; ++x) v[x] += t[x];
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) v[x] *= a.g.scale;
      store_part((TO *)a.g.out + (int64_t)row.x * a.g.ld_out + c, have, v);
    }
    __syncthreads();
  }
}

// Few tokens and a table too large for scan_kernel: one launch without sorting.  A wave takes a position and a slice of
// 64 * VEC columns; the wave of a token's first position adds up all of its positions, in order.  The remaining waves
// clear the rows that no token names, 16 each.  Every block holds the tokens in LDS.  512 tokens of 4,000 words x 256 bf16:
// 6.4 us (the host's time for a call), sorted 20; 460 of them alike: 46 us, since one wave per slice then adds them all,
// and sorted 20.  The rule goes by the number of tokens alone: how often each comes is not known before the launch.
constexpr int kFew = 512;
template <typename T, typename TO>
__global__ void __launch_bounds__(256) few_kernel(EmbedGradArgs a, int slices, int sum_blocks) {
  constexpr int VEC = El<T>::kVec, B = 8;
  __shared__ int tok[kFew];
  __shared__ unsigned named[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = a.n, V = a.vocab, D = a.channels;
  for (int i = threadIdx.x; i < (n + 63) / 64 * 64; i += 256) {
    const int t = i < n ? a.tokens[i] : -1;
    tok[i] = t >= 0 && t < V ? t : -1;  // -1 for all padding: differences below stay inside 32 bits
  }
  if (threadIdx.x < 4) named[threadIdx.x] = 0u;
  __syncthreads();
  if ((int)blockIdx.x < sum_blocks) {
    const int task = __builtin_amdgcn_readfirstlane((int)blockIdx.x * 4 + wave);
    const int i = task / slices, c0 = ((task % slices) * 64 + lane) * VEC;
    const bool full = D >= VEC;  // columns as in sum_kernel
    const int c = full ? min(c0, D - VEC) : c0, have = c0 < D ? (full ? VEC : D - c0) : 0;
    if (i >= n) return;
    const int t = __builtin_amdgcn_readfirstlane(tok[i]);
    if (t < 0) return;
    for (int j = 0; j < i; j += 64)
      if (__ballot(tok[j + lane] == t && j + lane < i)) return;
    float acc[VEC] = {};
    for (int j = i / 64 * 64; j < n; j += 64)
      for (unsigned long long m = __ballot(tok[j + lane] == t); m;) {
        int pos[B];
        int k = 0;
#pragma unroll
        for (int b = 0; b < B; ++b) {
          pos[b] = j + (m ? __ffsll((long long)m) - 1 : 0);
          k += m ? 1 : 0;
          m &= m - 1;
        }
        float v[B][VEC];
        if (full) {
          u32x4 raw[B];
#pragma unroll
          for (int b = 0; b < B; ++b) raw[b] = *(const u32x4_el *)((const T *)a.grad + (int64_t)pos[b] * a.ld_grad + c);
#pragma unroll
          for (int b = 0; b < B; ++b) expand(raw[b], v[b]);
        } else {
#pragma unroll
          for (int b = 0; b < B; ++b)
            load_part((const T *)a.grad + (int64_t)pos[b] * a.ld_grad + c, b < k ? have : 0, 0.f, v[b]);
        }
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
          for (int x = 0; x < VEC; ++x) acc[x] += b < k ? v[b][x] : 0.f;
      }
#pragma unroll
    for (int x = 0; x < VEC; ++x) acc[x] *= a.scale;
    store_part((TO *)a.out + (int64_t)t * a.ld_out + c, have, acc);
    return;
  }
  const int r0 = (((int)blockIdx.x - sum_blocks) * 4 + wave) * 16;
  for (int j = 0; j < n; j += 64) {
    const int d = tok[j + lane] - r0;
    if (d >= 0 && d < 16) atomicOr(&named[wave], 1u << d);
  }
  __syncthreads();
  const float zero[VEC] = {};
  for (int d = 0; d < 16 && r0 + d < V; ++d) {
    if (named[wave] >> d & 1) continue;
    TO *out = (TO *)a.out + (int64_t)(r0 + d) * a.ld_out;
    for (int c = lane * VEC; c < D; c += 64 * VEC) store_part(out + c, D - c, zero);
  }
}

// Up to 1,024 tokens and a small table: a block takes a row of the table and a slice of 64 * VEC columns; each of its 16
// waves looks through 64 of the tokens and adds up the row's positions among them, in order, and the waves' sums meet in
// LDS.  Bound by latency: 1,024 tokens of 256 classes x 512 float32 in 7.5 us (the host's time for a call), sorted 15; if
// 9 in 10 are of one class 20 us, sorted 16, and of 512 tokens 12 us, by few_kernel 36.
constexpr int kScanWaves = 16, kScan = 64 * kScanWaves;
template <typename T, typename TO>
__global__ void __launch_bounds__(64 * kScanWaves) scan_kernel(EmbedGradArgs a) {
  constexpr int VEC = El<T>::kVec, B = 8;
  __shared__ __align__(16) float red[kScanWaves][64 * VEC];
  __shared__ int some[kScanWaves];  // waves that found positions
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), D = a.channels;
  const int row = blockIdx.x, c0 = ((int)blockIdx.y * 64 + lane) * VEC, i0 = wave * 64;
  const bool full = D >= VEC;  // columns as in sum_kernel
  const int c = full ? min(c0, D - VEC) : c0, have = c0 < D ? (full ? VEC : D - c0) : 0;
  float acc[VEC] = {};
  unsigned long long m = __ballot(i0 + lane < a.n && a.tokens[min(i0 + lane, a.n - 1)] == row);
  const bool mine = m != 0;
  if (lane == 0) some[wave] = mine;
  while (m) {
    int pos[B];
    int k = 0;
#pragma unroll
    for (int b = 0; b < B; ++b) {
      pos[b] = i0 + (m ? __ffsll((long long)m) - 1 : 0);
      k += m ? 1 : 0;
      m &= m - 1;
    }
    float v[B][VEC];
    if (full) {
      u32x4 raw[B];
#pragma unroll
      for (int b = 0; b < B; ++b) raw[b] = *(const u32x4_el *)((const T *)a.grad + (int64_t)pos[b] * a.ld_grad + c);
#pragma unroll
      for (int b = 0; b < B; ++b) expand(raw[b], v[b]);
    } else {
#pragma unroll
      for (int b = 0; b < B; ++b)
        load_part((const T *)a.grad + (int64_t)pos[b] * a.ld_grad + c, b < k ? have : 0, 0.f, v[b]);
    }
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int x = 0; x < VEC; ++x) acc[x] += b < k ? v[b][x] : 0.f;
  }
  if (mine) store_aligned(&red[wave][lane * VEC], acc);
  __syncthreads();
  if (wave != 0) return;
  for (unsigned long long w = __ballot(lane > 0 && lane < kScanWaves && some[lane & (kScanWaves - 1)]); w; w &= w - 1)
#pragma unroll
    for (int x = 0; x < VEC; ++x) acc[x] += red[__ffsll((long long)w) - 1][lane * VEC + x];
#pragma unroll
  for (int x = 0; x < VEC; ++x) acc[x] *= a.scale;
  store_part((TO *)a.out + (int64_t)row * a.ld_out + c, have, acc);
}
// Blocks look for tokens in vain where a table has many rows: 4,096 rows take 512 tokens 8.6 to 11 us and few_kernel 6.4,
// 1,024 tokens 10 to 13 us and the sort 20.
bool scan_form(int n, int vocab, int slices) {
  return n > 0 && n <= kScan && (int64_t)vocab * slices <= (n <= kFew ? 2048 : 4096);
}

struct GradPlan {
  int tile, tiles, passes, bits, part, parts;
  bool counted, zero_early;
  size_t off_pair[2], off_hist, off_some, off_long, off_rows, off_partial, total;
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
  // entries per part: enough parts to fill the device with waves of 256 columns, not so few entries that their search
  // and partial sums dominate
  const int slices = (channels + 255) / 256;
  int part = 16;
  while (part < 64 && (n / (2 * part)) * slices >= 4096) part *= 2;
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
  // up to 16,384 tokens every block counts all of them itself, which takes less than a launch
  p.counted = p.tiles > 1 && n > 16384;
  // (narrower tables are cleared in no time, and `some` would be more than a few hundredths of them: 300,000 words x 64
  // bf16 take 20,000 tokens 48 us with it and 65 without)
  p.zero_early = p.counted && channels >= 64;
  p.off_some = o;
  o += p.zero_early ? up((size_t)vocab * sizeof(int)) : 0;
  p.off_long = o;
  o += 256;
  p.off_rows = o;
  o += up((size_t)p.parts * sizeof(int2));
  p.off_partial = o;
  o += up((size_t)p.parts * 2 * ((channels + 3) / 4 * 4) * sizeof(float));
  p.total = o;
  return p;
}

template <typename T, typename TO> hipError_t run_grad(const EmbedGradArgs &g, hipStream_t s) {
  const int slices = (g.channels + 64 * El<T>::kVec - 1) / (64 * El<T>::kVec);
  if (scan_form(g.n, g.vocab, slices)) {
    hipLaunchKernelGGL((scan_kernel<T, TO>), dim3(g.vocab, slices), dim3(64 * kScanWaves), 0, s, g);
    return hipGetLastError();
  }
  if (g.n <= kFew) {
    const int sum_blocks = (int)(((int64_t)g.n * slices + 3) / 4), zero_blocks = (int)(((int64_t)g.vocab + 63) / 64);
    hipLaunchKernelGGL((few_kernel<T, TO>), dim3((unsigned)(sum_blocks + zero_blocks)), dim3(256), 0, s, g, slices,
                       sum_blocks);
    return hipGetLastError();
  }
  const GradPlan p = plan_of(g.n, g.vocab, g.channels);
  SumArgs a;
  a.g = g;
  a.partial = (float *)(g.ws + p.off_partial);
  a.ld_p = (g.channels + 3) / 4 * 4;
  a.n_long = (int *)(g.ws + p.off_long);
  a.long_rows = (int2 *)(g.ws + p.off_rows);
  a.part = p.part;
  a.parts = p.parts;
  a.slices = slices;
  a.sorted = nullptr;
  int *hist = (int *)(g.ws + p.off_hist);
  const int shares = p.zero_early ? 2 * p.passes - 1 : 0;  // the launches after the first
  const int per_share = shares ? (g.vocab + shares - 1) / shares : 0;
  int share = 0;
  SortArgs q;
  q.tokens = g.tokens;
  q.hist = p.counted ? hist : nullptr;
  q.vocab = g.vocab;
  q.n = g.n;
  q.tile = p.tile;
  q.tiles = p.tiles;
  q.bits = p.bits;
  q.some = p.zero_early ? (int *)(g.ws + p.off_some) : nullptr;
  q.zero = {(char *)g.out, g.ld_out * (int64_t)sizeof(TO), g.channels * (int64_t)sizeof(TO), 0, 0};
  auto grid = [&](bool clears) {
    if (!clears || !shares) return dim3(p.tiles);
    q.zero.row0 = (int)((int64_t)share * per_share < g.vocab ? (int64_t)share * per_share : g.vocab);
    q.zero.row1 = g.vocab - q.zero.row0 < per_share ? g.vocab : q.zero.row0 + per_share;
    ++share;
    return dim3(p.tiles + (q.zero.row1 - q.zero.row0 + kSortWaves * kZeroRows - 1) / (kSortWaves * kZeroRows));
  };
  for (int k = 0; k < p.passes; ++k) {
    q.in = a.sorted;
    q.out = (Pair *)(g.ws + p.off_pair[k & 1]);
    q.clear = k == 0 ? a.n_long : nullptr;
    q.shift = k * p.bits;
    if (p.counted) {
      const dim3 blocks = grid(k > 0);
      hipLaunchKernelGGL(hist_kernel, blocks, dim3(1024), 0, s, q);
    }
    const dim3 blocks = grid(true);
    hipLaunchKernelGGL(scatter_kernel, blocks, dim3(1024), 0, s, q);
    a.sorted = q.out;
  }
  const int64_t tasks = (int64_t)p.parts * a.slices;
  const int sum_blocks = (int)((tasks + 3) / 4), zero_blocks = p.zero_early ? 0 : (int)(((int64_t)g.vocab + 63) / 64);
  // at most 2^32 threads in a launch: repeated rows may make more tasks than that of 2^28 tokens and more
  constexpr int kBlocks = 1 << 23;
  for (int b = 0; b < sum_blocks + zero_blocks; b += kBlocks) {
    const int blocks = sum_blocks + zero_blocks - b < kBlocks ? sum_blocks + zero_blocks - b : kBlocks;
    hipLaunchKernelGGL((sum_kernel<T, TO>), dim3((unsigned)blocks), dim3(256), 0, s, a, b, sum_blocks);
  }
  if (p.parts > 1) {
    const int64_t most = (int64_t)p.parts * ((g.channels + 255) / 256);
    int log_lanes = 0;
    while (log_lanes < 6 && (4 << log_lanes) < g.channels) ++log_lanes;
    hipLaunchKernelGGL((join_kernel<TO>), dim3((unsigned)(most < kJoinBlocks ? most : kJoinBlocks)),
                       dim3(64 * kJoinWaves), 0, s, a, log_lanes);
  }
  return hipGetLastError();
}

}  // namespace emb

hipError_t launch_embed(const EmbedArgs &a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == FWG_BF16)
    return out_dtype == FWG_BF16 ? emb::run<uint16_t, uint16_t>(a, s) : emb::run<uint16_t, float>(a, s);
  return out_dtype == FWG_BF16 ? emb::run<float, uint16_t>(a, s) : emb::run<float, float>(a, s);
}

size_t embed_grad_bytes(int64_t n, int vocab, int channels) {
  return n <= emb::kFew ? 0 : emb::plan_of(n, vocab, channels).total;
}

hipError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, int out_dtype, hipStream_t s) {
  if (dtype == FWG_BF16)
    return out_dtype == FWG_BF16 ? emb::run_grad<uint16_t, uint16_t>(a, s) : emb::run_grad<uint16_t, float>(a, s);
  return out_dtype == FWG_BF16 ? emb::run_grad<float, uint16_t>(a, s) : emb::run_grad<float, float>(a, s);
}

}  // namespace fwg

// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
//
// Per row z[0..V): m = max z, S = sum e^(z-m), U = sum e^(z-m) (z-m); then lse = m + ln S,
// logp = (z[t] - m) - ln S, H = ln S - U / S.  One pass: every lane carries its own (m, S, U) and
// rescales it when a batch raises its m; partial statistics are joined over the lanes, the waves of a
// block and the parts of a row in a fixed order.  Differences are taken before the scaling by log2(e), so
// logits near the type's limits (masks of the lowest value) neither overflow nor lose their place.
//
// The k alternatives are a list of (logit, index), one entry per lane in order (logit descending, index
// ascending).  A batch whose largest logit does not pass the list's last entry costs one comparison per
// lane; otherwise the batch's best elements are inserted one at a time, k at most.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace lpr {

using namespace opd;

constexpr int kNoIndex = 0x7fffffff;
constexpr int kWaves = 4, kThreadsLp = 64 * kWaves;
constexpr float kFloor = -200.f;  // 2^-200 is zero in float32: products with it stay zero and finite

struct Acc {
  float m, s, u;  // running max; sum of e = 2^d and of e d, d = (z - m) log2(e)
};

// m as the reference of differences: a lane that has seen -inf only refers to 0 (every e is 0).
__device__ __forceinline__ float ref_of(float m) { return m == -kInf ? 0.f : m; }

__device__ __forceinline__ void rescale(Acc &a, float ref) {
  const float d = (a.m - ref) * kLog2e, f = __builtin_amdgcn_exp2f(d);
  a.u = f * (a.u + a.s * fmaxf(d, kFloor));
  a.s *= f;
}

template <int N> __device__ __forceinline__ void add(Acc &a, const float (&z)[N], float batch_max) {
  const float m = fmaxf(a.m, batch_max), ref = ref_of(m);
  rescale(a, ref);
  a.m = m;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float d = (z[i] - ref) * kLog2e, e = __builtin_amdgcn_exp2f(d);  // NaN stays NaN in s and u
    a.s += e;
    a.u += e * fmaxf(d, kFloor);
  }
}

// Statistics of the whole wavefront, the same in every lane.
__device__ __forceinline__ Acc wave_join(Acc a) {
  const float m = wave_max(a.m);
  rescale(a, ref_of(m));
  return Acc{m, wave_sum(a.s), wave_sum(a.u)};
}

struct Entry {
  float v;
  int i;
};
// (v descending, index ascending)
__device__ __forceinline__ bool before(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

// Puts the lanes' candidates z[j] with index idx(j) (kNoIndex: none; NaN ranks as -inf) that come before
// the list's entry k - 1 into the list.
template <int N, typename Index>
__device__ __forceinline__ void insert_batch(Entry &list, int k, const float (&z)[N], Index idx) {
  const int lane = threadIdx.x & 63;
  float lv = -kInf;  // the last one taken; first none
  int li = -1;
  bool mine = true;  // my best has to be found anew
  Entry best{-kInf, kNoIndex};
  bool first = true;
  for (int n = 0; n < k; ++n) {
    if (mine) {
      best = Entry{-kInf, kNoIndex};
#pragma unroll
      for (int j = 0; j < N; ++j) {
        const float v = z[j] == z[j] ? z[j] : -kInf;
        const int i = idx(j);
        if (i != kNoIndex && (first || before(lv, li, v, i)) && before(v, i, best.v, best.i)) best = Entry{v, i};
      }
    }
    const float v = wave_max(best.v);
    const unsigned long long at = __ballot(best.v == v);
    int i;
    if (__popcll(at) == 1) i = __builtin_amdgcn_readlane(best.i, __ffsll((long long)at) - 1);
    else i = wave_min(best.v == v ? best.i : kNoIndex);
    const float tv = mfd::lane_f(list.v, k - 1);
    const int ti = __builtin_amdgcn_readlane(list.i, k - 1);
    if (i == kNoIndex || !before(v, i, tv, ti)) break;
    const int pos = __popcll(__ballot(before(list.v, list.i, v, i)));
    const float pv = __shfl_up(list.v, 1, 64);
    const int pi = __shfl_up(list.i, 1, 64);
    if (lane == pos) list = Entry{v, i};
    else if (lane > pos) list = Entry{pv, pi};
    lv = v;
    li = i;
    first = false;
    mine = best.i == i;
  }
}

// One wave's share of a row: batches of 64 * U vectors, `step` batches apart, from element `at` up to `end`.
template <typename T, bool TOP, int U>
__device__ __forceinline__ void scan(const T *row, int at, int end, int step, int k, Acc &acc, Entry &list) {
  constexpr int VEC = El<T>::kVec, N = U * VEC;
  const int lane = threadIdx.x & 63;
  for (; at < end; at += step) {
    float z[N];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int c = at + (j * 64 + lane) * VEC;
      float v[VEC];
      load_part(row + c, end - c, -kInf, v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) z[j * VEC + i] = v[i];
    }
    float bm = z[0];
#pragma unroll
    for (int i = 1; i < N; ++i) bm = fmaxf(bm, z[i]);
    bm = fmaxf(bm, -kInf);
    add(acc, z, bm);
    if (TOP) {
      const float tv = mfd::lane_f(list.v, k - 1);
      const int ti = __builtin_amdgcn_readlane(list.i, k - 1);
      // an equal logit of a later batch may have a lower index only where waves interleave: never within one wave
      if (__ballot(bm > tv) != 0ull || ti == kNoIndex)
        insert_batch(list, k, z, [&](int j) {
          const int c = at + ((j / VEC) * 64 + lane) * VEC + j % VEC;
          return c < end ? c : kNoIndex;
        });
    }
  }
}

// What a row's statistics say, written by one wave.
__device__ __forceinline__ void finish(const LogProbArgs &a, int64_t r, const Acc &t, const Entry &list, int token,
                                       float z) {
  const int lane = threadIdx.x & 63;
  const bool none = t.m == -kInf && t.s == 0.f;  // nothing left in this row (a NaN makes s NaN)
  const float ls = logf(t.s), ref = ref_of(t.m);
  if (lane == 0) {
    a.lse[r] = none ? -kInf : ref + ls;
    a.entropy[r] = none ? 0.f : ls - kLn2 * (t.u / t.s);
    a.logp[r] = token < 0 ? 0.f : none ? -kInf : (z - ref) - ls;
  }
  if (lane < a.top) {
    a.top_ids[r * a.top + lane] = list.i;
    a.top_logp[r * a.top + lane] = none ? -kInf : (list.v - ref) - ls;
  }
}

// The row's token (or -1) and its logit.
template <typename T> __device__ __forceinline__ int token_of(const LogProbArgs &a, int64_t r, const T *row, float *z) {
  const int t = a.tokens[r];
  const bool in = t >= 0 && t < a.vocab;
  *z = to_f(row[in ? t : 0]);
  return in ? t : -1;
}

// One wave per row.
template <typename T, bool TOP, int U>
__global__ void __launch_bounds__(kThreadsLp) rows_kernel(LogProbArgs a) {
  const int64_t r = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (r >= a.rows) return;
  const T *row = (const T *)a.logits + r * a.ld;
  float z;
  const int token = token_of(a, r, row, &z);
  Acc acc{-kInf, 0.f, 0.f};
  Entry list{-kInf, kNoIndex};
  scan<T, TOP, U>(row, 0, a.vocab, 64 * U * El<T>::kVec, a.top, acc, list);
  finish(a, r, wave_join(acc), list, token, z);
}

// A part of a row as the workspace holds it: statistics, then the list.
__host__ __device__ inline size_t part_floats(int top) { return 4 + 2 * (size_t)top; }

// One block per (row, part): its waves take the part's batches in turn.  One part: the row's results, else the
// part's statistics and list go to the workspace.
template <typename T, bool TOP, int U>
__global__ void __launch_bounds__(kThreadsLp) parts_kernel(LogProbArgs a, int parts, int per) {
  __shared__ Acc accs[kWaves];
  __shared__ Entry lists[kWaves][kMaxTop];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t r = blockIdx.x / (unsigned)parts;
  const int p = blockIdx.x % (unsigned)parts;
  const T *row = (const T *)a.logits + r * a.ld;
  float z;
  const int token = token_of(a, r, row, &z);
  Acc acc{-kInf, 0.f, 0.f};
  Entry list{-kInf, kNoIndex};
  constexpr int kBatch = 64 * U * El<T>::kVec;
  scan<T, TOP, U>(row, p * per + wave * kBatch, min(a.vocab, (p + 1) * per), kWaves * kBatch, a.top, acc, list);
  acc = wave_join(acc);
  if (lane == 0) accs[wave] = acc;
  if (TOP) lists[wave][lane] = list;
  __syncthreads();
  if (wave != 0) return;
  acc = wave_join(lane < kWaves ? accs[lane] : Acc{-kInf, 0.f, 0.f});
  if (TOP) {
    for (int w = 1; w < kWaves; ++w) {
      const Entry e = lists[w][lane];
      const float v[1] = {e.v};
      insert_batch(list, a.top, v, [&](int) { return lane < a.top ? e.i : kNoIndex; });
    }
  }
  if (parts == 1) {
    finish(a, r, acc, list, token, z);
    return;
  }
  float *out = (float *)a.ws + (size_t)blockIdx.x * part_floats(a.top);
  if (lane == 0) {
    out[0] = acc.m;
    out[1] = acc.s;
    out[2] = acc.u;
  }
  if (lane < a.top) {
    out[4 + lane] = list.v;
    ((int *)out)[4 + a.top + lane] = list.i;
  }
}

// Joins the parts of a row: one wave per row.
template <typename T, bool TOP> __global__ void __launch_bounds__(64) join_kernel(LogProbArgs a, int parts) {
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  float z;
  const int token = token_of(a, r, (const T *)a.logits + r * a.ld, &z);
  const size_t stride = part_floats(a.top);
  const float *in = (const float *)a.ws + (size_t)r * parts * stride;
  Acc acc{-kInf, 0.f, 0.f};
  for (int p = lane; p < parts; p += 64) {
    const Acc b{in[p * stride], in[p * stride + 1], in[p * stride + 2]};
    const float m = fmaxf(acc.m, b.m), ref = ref_of(m);
    Acc c = b;
    rescale(acc, ref);
    rescale(c, ref);
    acc = Acc{m, acc.s + c.s, acc.u + c.u};
  }
  acc = wave_join(acc);
  Entry list{-kInf, kNoIndex};
  if (TOP) {
    for (int c = lane; c - lane < parts * a.top; c += 64) {
      const bool in_list = c < parts * a.top;
      const int p = in_list ? c / a.top : 0, e = in_list ? c % a.top : 0;
      const float v[1] = {in_list ? in[p * stride + 4 + e] : -kInf};
      const int i = in_list ? ((const int *)in)[p * stride + 4 + a.top + e] : kNoIndex;
      insert_batch(list, a.top, v, [&](int) { return i; });
    }
  }
  finish(a, r, acc, list, token, z);
}

// Elements of a batch of one wave (U = 4), and the parts a row is cut into.
template <typename T> constexpr int batch_of(int U) { return 64 * U * El<T>::kVec; }
constexpr int kMaxParts = 256;
int parts_of(int64_t rows, int vocab, int batch) {
  // a part is at least one batch for each of a block's waves; parts are made only where the rows alone do not
  // fill the device (256 compute units with four blocks each)
  const int64_t most = (vocab + (int64_t)kWaves * batch - 1) / ((int64_t)kWaves * batch);
  const int64_t want = (1024 + rows - 1) / rows;
  int64_t p = want < most ? want : most;
  return (int)(p < 1 ? 1 : p > kMaxParts ? kMaxParts : p);
}

template <typename T, bool TOP> hipError_t run(const LogProbArgs &a, bool in_parts, hipStream_t s) {
  const int batch = batch_of<T>(4);
  if (a.vocab <= batch) {
    const dim3 grid((unsigned)((a.rows + kWaves - 1) / kWaves));
    if (a.vocab <= batch_of<T>(1)) hipLaunchKernelGGL((rows_kernel<T, TOP, 1>), grid, dim3(kThreadsLp), 0, s, a);
    else hipLaunchKernelGGL((rows_kernel<T, TOP, 4>), grid, dim3(kThreadsLp), 0, s, a);
    return hipGetLastError();
  }
  const int parts = in_parts ? parts_of(a.rows, a.vocab, batch) : 1;
  const int per = (int)(((int64_t)a.vocab + parts - 1) / parts);
  hipLaunchKernelGGL((parts_kernel<T, TOP, 4>), dim3((unsigned)(a.rows * parts)), dim3(kThreadsLp), 0, s, a, parts, per);
  if (parts > 1) hipLaunchKernelGGL((join_kernel<T, TOP>), dim3((unsigned)a.rows), dim3(64), 0, s, a, parts);
  return hipGetLastError();
}

// The gradient: dz[j] = g (1[j = t] - p_j) - gH p_j (log p_j + H), p_j = e^(z_j - lse).  Every element is read once
// and written once by the thread that read it (the output may be the logits' own array).
template <typename T, bool ENT, int U>
__global__ void __launch_bounds__(kThreadsLp) grad_kernel(LogProbGradArgs a, int chunks) {
  constexpr int VEC = El<T>::kVec;
  const int64_t task = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const int64_t r = task / chunks;
  if (r >= a.rows) return;
  const int c0 = (int)(task - r * chunks) * (64 * U * VEC) + lane * VEC;
  const T *row = (const T *)a.logits + r * a.ld;
  T *out = (T *)a.out + r * a.ld_o;
  const float lse = a.lse[r];
  const bool none = lse == -kInf;
  const int t = a.tokens[r];
  const bool in = t >= 0 && t < a.vocab && !none;
  const float g = in ? a.g_logp[r] : 0.f, ge = ENT && !none ? a.g_entropy[r] : 0.f, h = ENT ? a.entropy[r] : 0.f;
  float z[U][VEC];
#pragma unroll
  for (int j = 0; j < U; ++j) load_part(row + c0 + j * 64 * VEC, a.vocab - (c0 + j * 64 * VEC), -kInf, z[j]);
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int c = c0 + j * 64 * VEC;
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      const float lp = z[j][i] - lse, p = __builtin_amdgcn_exp2f(lp * kLog2e);
      const float w = ENT ? g + ge * (fmaxf(lp, kFloor) + h) : g;
      z[j][i] = none ? 0.f : -p * w;
    }
    if (in && t - c >= 0 && t - c < VEC) {
#pragma unroll
      for (int i = 0; i < VEC; ++i)
        if (t - c == i) z[j][i] += g;
    }
    store_part(out + c, a.vocab - c, z[j]);
  }
}

template <typename T, bool ENT> hipError_t run_grad(const LogProbGradArgs &a, hipStream_t s) {
  const int one = batch_of<T>(1), four = batch_of<T>(4);
  const bool small = a.vocab <= one;
  const int chunks = small ? 1 : (a.vocab + four - 1) / four;
  const int64_t tasks = a.rows * chunks;
  const dim3 grid((unsigned)((tasks + kWaves - 1) / kWaves));
  if (small) hipLaunchKernelGGL((grad_kernel<T, ENT, 1>), grid, dim3(kThreadsLp), 0, s, a, chunks);
  else hipLaunchKernelGGL((grad_kernel<T, ENT, 4>), grid, dim3(kThreadsLp), 0, s, a, chunks);
  return hipGetLastError();
}

}  // namespace lpr

size_t log_probs_bytes(int64_t rows, int vocab, int top, int dtype) {
  const int batch = dtype == FWG_BF16 ? lpr::batch_of<uint16_t>(4) : lpr::batch_of<float>(4);
  if (rows <= 0 || vocab <= batch) return 0;
  const int parts = lpr::parts_of(rows, vocab, batch);
  return parts == 1 ? 0 : (size_t)rows * parts * lpr::part_floats(top) * sizeof(float);
}

hipError_t launch_log_probs(const LogProbArgs &a, int dtype, bool in_parts, hipStream_t s) {
  if (dtype == FWG_BF16)
    return a.top ? lpr::run<uint16_t, true>(a, in_parts, s) : lpr::run<uint16_t, false>(a, in_parts, s);
  return a.top ? lpr::run<float, true>(a, in_parts, s) : lpr::run<float, false>(a, in_parts, s);
}

hipError_t launch_log_probs_grad(const LogProbGradArgs &a, int dtype, hipStream_t s) {
  if (dtype == FWG_BF16) return a.g_entropy ? lpr::run_grad<uint16_t, true>(a, s) : lpr::run_grad<uint16_t, false>(a, s);
  return a.g_entropy ? lpr::run_grad<float, true>(a, s) : lpr::run_grad<float, false>(a, s);
}

}  // namespace fwg

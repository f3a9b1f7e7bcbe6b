// Log probabilities of given tokens with entropy and top alternatives, and their gradient.
//
// Per row z[0..V): m = max z, S = sum e^(z-m), U = sum e^(z-m) (z-m); then lse = m + ln S,
// logp = (z[t] - m) - ln S, H = ln S - U / S.  One pass: every lane carries its own (m, S, U) and
// rescales it when a batch raises its m; partial statistics are joined over the lanes, the waves of a
// block and the parts of a row in a fixed order.  Differences are taken before the scaling by log2(e), so
// logits near the type's limits (masks of the lowest value) neither overflow nor lose their place.
//
// The k alternatives are a list with one entry per lane in order (logit descending, index ascending).  A batch
// whose largest logit does not pass the list's last entry costs one comparison per lane; otherwise the elements
// that pass it are joined with the list.
//
// Measured: 4,093 rows of 50,001 float32 with 8 alternatives 150 us (5.4 TB/s), bound by memory; 192,064 rows of 256 float32
// with 4 alternatives 50 us (4.1 TB/s; 29 us and 6.8 TB/s without alternatives), bound by instructions; 16 rows of 131,072
// bf16 with 20 alternatives 13 us in two launches (5 us without alternatives), bound by latency.  The gradient of 8,190
// rows of 50,001 bf16 takes 280 to 286 us (5.7 to 5.9 TB/s), bound by memory.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg.h"
#include "fwg_ops.h"
#include "fwg_ops_dev.h"

namespace fwg {
namespace lpr {

using namespace opd;

constexpr int kWaves = 4, kThreadsLp = 64 * kWaves;
constexpr float kMax = 3.4028234663852886e38f;
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

// An alternative as one double: the logit's bits are the high word, its place the low one, so that doubles
// compare as (logit descending, index ascending).  Every float but NaN (which ranks as -inf), -inf included, makes a
// finite double; for negative numbers a larger low word is a smaller double, so the place is stored as it is there
// and inverted elsewhere.
__device__ __forceinline__ double key_of(float z, int i) {
  const int h = __float_as_int(fmaxf(z, -kInf) + 0.f);  // NaN out, one zero
  return __hiloint2double(h, i ^ ~(h >> 31));
}
__device__ __forceinline__ double below(float v) { return key_of(v, -1); }  // below every key of logit v
__device__ __forceinline__ float value_of(double key) { return __int_as_float(__double2hiint(key)); }
__device__ __forceinline__ int index_of(double key) { return __double2loint(key) ^ ~(__double2hiint(key) >> 31); }
__device__ __forceinline__ double lane_d(double v, int l) {
  return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), l), __builtin_amdgcn_readlane(__double2loint(v), l));
}
template <int CTRL> __device__ __forceinline__ double dpp_d(double v) {
  return __hiloint2double(dpp_i<CTRL>(__double2hiint(v)), dpp_i<CTRL>(__double2loint(v)));
}
// Largest key of each row of 16 lanes, in all of its lanes.
__device__ __forceinline__ double row16_max(double v) {
  v = fmax(v, dpp_d<0xB1>(v));
  v = fmax(v, dpp_d<0x4E>(v));
  v = fmax(v, dpp_d<0x141>(v));
  return fmax(v, dpp_d<0x140>(v));
}

// What a wave keeps in LDS to select: candidates (logit bits, index), and the two sides of a merge.
constexpr int kSlots = 256;
struct Select {
  int2 slot[kSlots];
  double cand[64], place[kMaxTop];
};
// Floats as whole numbers of the same order, and back (no NaN).
__device__ __forceinline__ int ordered(float v) {
  const int b = __float_as_int(v);
  return b ^ ((b >> 31) & 0x7fffffff);
}
__device__ __forceinline__ float from_ordered(int o) { return __int_as_float(o ^ ((o >> 31) & 0x7fffffff)); }

// A bound that at least k, and where values differ at most 2 k, of the lanes' 64 U values reach (k <= 64, and every
// lane has values: -inf at least).  Bisection over the values in order; a count takes a ballot per value.
template <int U> __device__ __forceinline__ float bound_of(const float (&v)[U], int k) {
  float most = v[0];
#pragma unroll
  for (int u = 1; u < U; ++u) most = fmaxf(most, v[u]);
  int lo = ordered(-wave_max(-most)), hi = ordered(wave_max(most));  // all 64 lanes reach lo
  while (lo < hi) {
    const int mid = (int)(((long long)lo + hi + 1) >> 1);
    const float t = from_ordered(mid);
    int n = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) n += __popcll(__ballot(v[u] >= t));
    if (n >= k) lo = mid;
    else hi = mid - 1;
    if (n >= k && n <= 2 * k) break;
  }
  return from_ordered(lo);
}

// The list: lane i < k holds the i-th best key so far (below(-inf): none).  Joins it with candidates, at most one
// per lane, in the first n lanes: everybody's place is the number of keys before it, counted over keys that all
// lanes read at once.
__device__ __forceinline__ void merge(double &list, int k, double cand, int n, Select &s) {
  const int lane = threadIdx.x & 63;
  const double none = below(-kInf);
  int pc = 0, pl = lane;
  s.cand[lane] = cand;
  s.place[lane] = list;
  in_order();
#pragma unroll 1
  for (int j = 0; j < n; j += 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const double c = s.cand[j + i];
      pc += c > cand;
      pl += c > list;
    }
  const int held = __popcll(__ballot(list > none));
#pragma unroll 1
  for (int j = 0; j < held; j += 8)
#pragma unroll
    for (int i = 0; i < 8; ++i) pc += s.place[j + i] > cand;
  in_order();
  s.place[lane] = none;
  in_order();
  if (cand > none && pc < k) s.place[pc] = cand;
  if (list > none && pl < k) s.place[pl] = list;
  in_order();
  list = s.place[lane];
  in_order();
}

// Joins the list with the n <= kSlots candidates of the slots.
__device__ __forceinline__ void merge_slots(double &list, int k, int n, Select &s) {
  const int lane = threadIdx.x & 63;
  in_order();
#pragma unroll 1
  for (int o = 0; o < n; o += 64) {
    double cand = below(-kInf);
    if (o + lane < n) {
      const int2 v = s.slot[o + lane];
      cand = key_of(__int_as_float(v.x), v.y);
    }
    merge(list, k, cand, min(64, n - o), s);
  }
}

// Appends an element of each lane that wants to; n counts them, also beyond the slots.
__device__ __forceinline__ void append(float z, int i, bool want, int &n, Select &s) {
  const unsigned long long m = __ballot(want);
  if (m == 0ull) return;
  const int at = n + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
  if (want && at < kSlots) s.slot[at] = make_int2(__float_as_int(z), i);
  n += __popcll(m);
}

// Puts the elements of a batch (U vectors per lane, at .. min(end, at + 64 U VEC) of the row) that come before the
// list's entry k - 1 into the list.  best: the largest of each vector.  Where many lanes have candidates (the first
// batch, above all), a bound that k vectors' best reach leaves out what cannot be among the k, and little more than
// those pass it.  Where more than the slots pass (many equal logits, rising rows) the elements are read again, 64 at
// a time.
template <typename T, int U>
__device__ __forceinline__ void take(double &list, int k, const float (&batch)[U * El<T>::kVec], const float (&best)[U],
                                     float most, const T *row, int at, int end, Select &s) {
  constexpr int VEC = El<T>::kVec, N = U * VEC;
  const int lane = threadIdx.x & 63;
  float least = value_of(lane_d(list, k - 1));
  if (__popcll(__ballot(most > least)) > 8) least = fmaxf(least, bound_of(best, k));
  least = fmaxf(least, -kMax);
  int n = 0, c = at + lane * VEC;
  float z[N];
#pragma unroll
  for (int i = 0; i < N; ++i) z[i] = batch[i];
#pragma unroll 1
  for (int u = 0; u < U; ++u) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) append(z[i], min(c, end - VEC) + i, z[i] >= least, n, s);
#pragma unroll
    for (int i = 0; i < N - VEC; ++i) z[i] = z[i + VEC];  // a loop over registers: move, not index
    c += 64 * VEC;
  }
  const bool fits = n <= kSlots;
  int c0 = at;
  const int c1 = min(end, at + 64 * N);
  do {
    if (!fits) {
      n = 0;
      const double key = c0 + lane < c1 ? key_of(to_f(row[c0 + lane]), c0 + lane) : below(-kInf);
      append(value_of(key), c0 + lane, key > lane_d(list, k - 1) && value_of(key) >= -kMax, n, s);
      c0 += 64;
    }
    merge_slots(list, k, n, s);
  } while (!fits && c0 < c1);
}

// Logits of -inf (and NaN, which ranks with them) are no candidates above: rows have them by the thousand.  Where
// fewer than k others were found, the lowest tokens of them fill the list; 2 k tokens of the row hold enough.
template <typename T> __device__ __forceinline__ void fill(double &list, int k, const T *row, int vocab, Select &s) {
  const int lane = threadIdx.x & 63;
  int n = __popcll(__ballot(lane < k && list > below(-kInf)));
  if (n >= k) return;
  in_order();
  s.place[lane] = list;
#pragma unroll 1
  for (int c0 = 0; n < k && c0 < vocab; c0 += 64) {
    const bool out = c0 + lane < vocab && !(to_f(row[c0 + lane]) > -kInf);
    const unsigned long long m = __ballot(out);
    const int at = n + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
    if (out && at < k) s.place[at] = key_of(-kInf, c0 + lane);
    n += __popcll(m);
  }
  in_order();
  list = s.place[lane];
}

// One wave's share of a row: batches of 64 * U vectors, `step` elements apart, from element `at` up to `end` (at least a
// vector from the row's start).
template <typename T, bool TOP, int U>
__device__ __forceinline__ void scan(const T *row, int at, int end, int step, int k, Acc &acc, double &list, Select *sel) {
  constexpr int VEC = El<T>::kVec, N = U * VEC;
  const int lane = threadIdx.x & 63;
  float last = -kInf;  // the logit of the list's last entry
  for (; at < end; at += step) {
    float z[N];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      // a vector that would pass the end is taken from the last VEC elements instead
      float v[VEC];
      load(row + min(at + (j * 64 + lane) * VEC, end - VEC), v);
#pragma unroll
      for (int i = 0; i < VEC; ++i) z[j * VEC + i] = v[i];
    }
    if (at + 64 * N > end) {  // and what it has from vectors before does not count again
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int over = at + (j * 64 + lane) * VEC - (end - VEC);
#pragma unroll
        for (int i = 0; i < VEC; ++i) z[j * VEC + i] = i < over ? -kInf : z[j * VEC + i];
      }
    }
    float best[U], bm = -kInf;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      best[j] = -kInf;
#pragma unroll
      for (int i = 0; i < VEC; ++i) best[j] = fmaxf(best[j], z[j * VEC + i]);
      bm = fmaxf(bm, best[j]);
    }
    add(acc, z, bm);
    // a later batch of the same wave has larger indexes throughout, so an equal logit does not come before
    if (TOP && __ballot(bm > last) != 0ull) {
      take<T, U>(list, k, z, best, bm, row, at, end, *sel);
      last = value_of(lane_d(list, k - 1));
    }
  }
}

// What a row's statistics say: written by the group of lanes `l` = 0 .. that hold them and the list.
struct Row {
  float ref, ls;  // the reference of its logits, and the logarithm of their sum
  bool none;      // nothing left in this row (a NaN makes the sum NaN)
};
__device__ __forceinline__ Row finish(const LogProbArgs &a, int64_t r, int l, const Acc &t, int token, float z) {
  const Row o{ref_of(t.m), kLn2 * __builtin_amdgcn_logf(t.s), t.m == -kInf && t.s == 0.f};  // t.s >= 1, or 0
  if (l == 0) {
    a.lse[r] = o.none ? -kInf : o.ref + o.ls;
    a.entropy[r] = o.none ? 0.f : o.ls - kLn2 * (t.u / t.s);
    a.logp[r] = token < 0 ? 0.f : o.none ? -kInf : (z - o.ref) - o.ls;
  }
  return o;
}
__device__ __forceinline__ void put_alternative(const LogProbArgs &a, int64_t r, int place, double key, const Row &o) {
  if (place >= a.top) return;
  a.top_ids[r * a.top + place] = index_of(key);
  a.top_logp[r * a.top + place] = o.none ? -kInf : (value_of(key) - o.ref) - o.ls;
}
__device__ __forceinline__ void finish(const LogProbArgs &a, int64_t r, int l, const Acc &t, double list, int token,
                                       float z) {
  const Row o = finish(a, r, l, t, token, z);
  put_alternative(a, r, l, list, o);
}

// The row's token (or -1) and its logit.
template <typename T> __device__ __forceinline__ int token_of(const LogProbArgs &a, int64_t r, const T *row, float *z) {
  const int t = a.tokens[r];
  const bool in = t >= 0 && t < a.vocab;
  *z = to_f(row[in ? t : 0]);
  return in ? t : -1;
}

__device__ __forceinline__ void exchange(double &a, double &b) {
  const double m = fmax(a, b);
  b = fmin(a, b);
  a = m;
}
// Descending order of N keys in registers (odd-even merge sort).
template <int N> __device__ __forceinline__ void sort_keys(double (&a)[N]) {
#pragma unroll
  for (int p = 1; p < N; p *= 2)
#pragma unroll
    for (int k = p; k >= 1; k /= 2)
#pragma unroll
      for (int j = k % p; j + k < N; j += 2 * k)
#pragma unroll
        for (int i = 0; i < k; ++i)
          if (i + j + k < N && (i + j) / (2 * p) == (i + j + k) / (2 * p)) exchange(a[i + j], a[i + j + k]);
}

// Rows of at most 256 logits: 16 lanes per row, 16 logits per lane, four rows per wave, so that the reductions
// (inside rows of 16 lanes, without lane reads) and what follows them are shared by four rows.
constexpr int kShort = 256, kE = 16, kL = 16;
template <typename T> __device__ __forceinline__ int place_of(int j, int l) {  // the index of a lane's j-th logit
  return (j / El<T>::kVec * kL + l) * El<T>::kVec + j % El<T>::kVec;
}
template <typename T> __device__ __forceinline__ Acc short_row(const T *row, int vocab, int l, float (&z)[kE]) {
  constexpr int VEC = El<T>::kVec;
#pragma unroll
  for (int j = 0; j < kE / VEC; ++j) {
    const int c = (j * kL + l) * VEC;
    float v[VEC];
    load_part(row + c, vocab - c, -kInf, v);
#pragma unroll
    for (int i = 0; i < VEC; ++i) z[j * VEC + i] = v[i];
  }
  float m = -kInf;
#pragma unroll
  for (int i = 0; i < kE; ++i) m = fmaxf(m, z[i]);
  m = fmaxf(m, dpp_f<0xB1>(m));
  m = fmaxf(m, dpp_f<0x4E>(m));
  m = fmaxf(m, dpp_f<0x141>(m));
  m = fmaxf(m, dpp_f<0x140>(m));
  const float ref = ref_of(m);
  Acc acc{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    const float d = (z[i] - ref) * kLog2e, e = __builtin_amdgcn_exp2f(d);
    acc.s += e;
    acc.u += e * fmaxf(d, kFloor);
  }
  auto row_sum = [](float v) {
    v += dpp_f<0xB1>(v);
    v += dpp_f<0x4E>(v);
    v += dpp_f<0x141>(v);
    return v + dpp_f<0x140>(v);
  };
  acc.s = row_sum(acc.s);
  acc.u = row_sum(acc.u);
  return acc;
}

// Up to TOP alternatives: the lanes sort the TOP best of their keys; the row's best are then taken off the lanes' heads
// one at a time.
template <typename T, int TOP>
__global__ void __launch_bounds__(kThreadsLp) short_kernel(LogProbArgs a) {
  const int l = threadIdx.x & (kL - 1);
  const int64_t r0 = ((int64_t)blockIdx.x * kThreadsLp + threadIdx.x) / kL, r = r0 < a.rows ? r0 : a.rows - 1;
  const T *row = (const T *)a.logits + r * a.ld;
  float zt, z[kE];
  const int token = token_of(a, r, row, &zt);
  const Acc acc = short_row(row, a.vocab, l, z);
  double mine = 0.0;
  if constexpr (TOP > 0) {
    double best[TOP];
#pragma unroll
    for (int g = 0; g < kE / TOP; ++g) {
      double k[TOP];
#pragma unroll
      for (int i = 0; i < TOP; ++i) {
        const int j = g * TOP + i;
        k[i] = key_of(z[j], place_of<T>(j, l));  // places past the vocabulary: -inf, after every token
      }
      sort_keys(k);
      if (g == 0) {
#pragma unroll
        for (int i = 0; i < TOP; ++i) best[i] = k[i];
      } else {  // the best of two sorted lists: pair them end to end, then merge
#pragma unroll
        for (int i = 0; i < TOP; ++i) best[i] = fmax(best[i], k[TOP - 1 - i]);
#pragma unroll
        for (int h = TOP / 2; h >= 1; h /= 2)
#pragma unroll
          for (int i = 0; i < TOP; ++i)
            if ((i & h) == 0) exchange(best[i], best[i + h]);
      }
    }
    for (int n = 0; n < a.top; ++n) {
      const double w = row16_max(best[0]);
      if (l == n) mine = w;
      const bool mine_goes = best[0] == w;
#pragma unroll
      for (int i = 0; i < TOP; ++i) best[i] = mine_goes ? (i + 1 < TOP ? best[i + 1] : below(-kInf)) : best[i];
    }
  }
  if (r0 < a.rows) finish(a, r, l, acc, mine, token, zt);
}

// A lane's key against its partner's: the larger stays in the lower lane.
__device__ __forceinline__ double keep(double mine, double other, bool low) { return (mine > other) == low ? mine : other; }
template <int CTRL> __device__ __forceinline__ void cross_lanes(double (&k)[kE], bool low) {
#pragma unroll
  for (int i = 0; i < kE; ++i) k[i] = keep(k[i], dpp_d<CTRL>(k[i]), low);
}
// Merges the sorted lists of two halves of a group of lanes: FLIP pairs them end to end, then lane distances DIST .. 1,
// then the lane's own keys.
template <int FLIP, int HALF> __device__ __forceinline__ void merge_lanes(double (&k)[kE], int l) {
  const bool low = (l & HALF) == 0;
#pragma unroll
  for (int i = 0; i < kE / 2; ++i) {
    const double a = dpp_d<FLIP>(k[kE - 1 - i]), b = dpp_d<FLIP>(k[i]);
    k[i] = keep(k[i], a, low);
    k[kE - 1 - i] = keep(k[kE - 1 - i], b, low);
  }
  if constexpr (HALF > 4) {  // lanes 4 apart: mirrored in eight, then in four
#pragma unroll
    for (int i = 0; i < kE; ++i) k[i] = keep(k[i], dpp_d<0x1B>(dpp_d<0x141>(k[i])), (l & 4) == 0);
  }
  if constexpr (HALF > 2) cross_lanes<0x4E>(k, (l & 2) == 0);
  if constexpr (HALF > 1) cross_lanes<0xB1>(k, (l & 1) == 0);
#pragma unroll
  for (int h = kE / 2; h >= 1; h /= 2)
#pragma unroll
    for (int i = 0; i < kE; ++i)
      if ((i & h) == 0) exchange(k[i], k[i + h]);
}

// More alternatives of such rows: the whole row is sorted, sixteen keys per lane in order.  40,872 rows of 256 bf16 with
// 64 alternatives: 33 us (127 with a wave per row and a list), with 8: 28 us (30 in short_kernel's way).
template <typename T> __global__ void __launch_bounds__(kThreadsLp) sorted_kernel(LogProbArgs a) {
  const int l = threadIdx.x & (kL - 1);
  const int64_t r0 = ((int64_t)blockIdx.x * kThreadsLp + threadIdx.x) / kL, r = r0 < a.rows ? r0 : a.rows - 1;
  const T *row = (const T *)a.logits + r * a.ld;
  float zt, z[kE];
  const int token = token_of(a, r, row, &zt);
  const Acc acc = short_row(row, a.vocab, l, z);
  double k[kE];
#pragma unroll
  for (int j = 0; j < kE; ++j) k[j] = key_of(z[j], place_of<T>(j, l));
  sort_keys(k);
  merge_lanes<0xB1, 1>(k, l);
  merge_lanes<0x1B, 2>(k, l);
  merge_lanes<0x141, 4>(k, l);
  merge_lanes<0x140, 8>(k, l);
  if (r0 >= a.rows) return;
  const Row o = finish(a, r, l, acc, token, zt);
#pragma unroll
  for (int j = 0; j < kE; ++j) put_alternative(a, r, l * kE + j, k[j], o);
}

// One wave per row.
template <typename T, bool TOP, int U>
__global__ void __launch_bounds__(kThreadsLp) rows_kernel(LogProbArgs a) {
  const int64_t r = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  __shared__ Select sel[TOP ? kWaves : 1];
  if (r >= a.rows) return;
  const T *row = (const T *)a.logits + r * a.ld;
  float z;
  const int token = token_of(a, r, row, &z);
  Acc acc{-kInf, 0.f, 0.f};
  double list = below(-kInf);
  scan<T, TOP, U>(row, 0, a.vocab, 64 * U * El<T>::kVec, a.top, acc, list, &sel[TOP ? threadIdx.x >> 6 : 0]);
  if (TOP) fill(list, a.top, row, a.vocab, sel[TOP ? threadIdx.x >> 6 : 0]);
  finish(a, r, threadIdx.x & 63, wave_join(acc), list, token, z);
}

// Rows in parts: the workspace holds the parts' statistics (m, s, u and a gap), then their lists.
struct Parts {
  float4 *stat;  // [rows][parts]
  double *keys;  // [rows][parts][top]
};
__host__ __device__ inline Parts parts_at(unsigned char *ws, int64_t rows, int parts) {
  return Parts{(float4 *)ws, (double *)(ws + (size_t)rows * parts * sizeof(float4))};
}

// One block per (row, part): its waves take the part's batches in turn and join what they found.  One part: the
// row's results, else the part's statistics and list go to the workspace.
template <typename T, bool TOP, int U>
__global__ void __launch_bounds__(kThreadsLp) parts_kernel(LogProbArgs a, int parts, int per) {
  __shared__ Acc accs[kWaves];
  __shared__ Select sel[TOP ? kWaves : 1];
  __shared__ double merged[kMaxTop];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t r = blockIdx.x / (unsigned)parts;
  const int p = blockIdx.x % (unsigned)parts;
  const T *row = (const T *)a.logits + r * a.ld;
  float z;
  const int token = token_of(a, r, row, &z);
  Acc acc{-kInf, 0.f, 0.f};
  double list = below(-kInf);
  constexpr int kBatch = 64 * U * El<T>::kVec;
  scan<T, TOP, U>(row, p * per + wave * kBatch, min(a.vocab, (p + 1) * per), kWaves * kBatch, a.top, acc, list,
                  &sel[TOP ? wave : 0]);
  acc = wave_join(acc);
  if (lane == 0) accs[wave] = acc;
  if (TOP) {
    sel[wave].place[lane] = list;
    if (wave == 0) merged[lane] = below(-kInf);
  }
  __syncthreads();
  if (TOP) {
    // an entry's place is its place in its own list plus the entries of the others before it
    int place[kWaves] = {};
    int h = 64;
    while (h > a.top) h >>= 1;
    for (; h; h >>= 1) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        if (place[w] + h <= a.top && sel[w].place[place[w] + h - 1] > list) place[w] += h;
    }
    int at = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) at += place[w];  // in its own list: the lane itself
    if (lane < a.top && list > below(-kInf) && at < a.top) merged[at] = list;
    __syncthreads();
  }
  if (wave != 0) return;
  acc = wave_join(lane < kWaves ? accs[lane] : Acc{-kInf, 0.f, 0.f});
  if (TOP) list = merged[lane];
  if (parts == 1) {
    if (TOP) fill(list, a.top, row, a.vocab, sel[0]);
    finish(a, r, lane, acc, list, token, z);
    return;
  }
  const Parts o = parts_at(a.ws, a.rows, parts);
  if (lane == 0) o.stat[blockIdx.x] = make_float4(acc.m, acc.s, acc.u, 0.f);
  if (lane < a.top) o.keys[(size_t)blockIdx.x * a.top + lane] = list;
}

// Joins the parts of a row (at most 64): one wave per row.
template <typename T, bool TOP> __global__ void __launch_bounds__(64) join_kernel(LogProbArgs a, int parts) {
  __shared__ Select sel;
  const int lane = threadIdx.x;
  const int64_t r = blockIdx.x;
  const Parts in = parts_at(a.ws, a.rows, parts);
  float z;
  const int token = token_of(a, r, (const T *)a.logits + r * a.ld, &z);
  Acc acc{-kInf, 0.f, 0.f};
  double list = below(-kInf);
  if (lane < parts) {
    const float4 v = in.stat[r * parts + lane];
    acc = Acc{v.x, v.y, v.z};
  }
  acc = wave_join(acc);
  if (TOP) {
    // a bound from the heads of the lists: one key per lane
    const int e = lane / parts;
    float head[1] = {-kInf};
    if (e < a.top && (e + 1) * parts <= 64) head[0] = value_of(in.keys[(r * parts + lane % parts) * a.top + e]);
    float least = bound_of(head, a.top);
    const double *keys = in.keys + r * parts * a.top;
    const int n = parts * a.top;
#pragma unroll 1
    for (int c0 = 0; c0 < n; c0 += kSlots) {
      double key[kSlots / 64];
#pragma unroll
      for (int j = 0; j < kSlots / 64; ++j) key[j] = c0 + j * 64 + lane < n ? keys[c0 + j * 64 + lane] : below(-kInf);
      int found = 0;
#pragma unroll
      for (int j = 0; j < kSlots / 64; ++j)
        append(value_of(key[j]), index_of(key[j]), value_of(key[j]) >= least && key[j] > below(-kInf), found, sel);
      merge_slots(list, a.top, found, sel);
      least = fmaxf(least, value_of(lane_d(list, a.top - 1)));
    }
    fill(list, a.top, (const T *)a.logits + r * a.ld, a.vocab, sel);
  }
  finish(a, r, lane, acc, list, token, z);
}

// Elements of a batch of one wave, and the parts a row is cut into.  16 rows of 131,072 bf16: 16 parts of four batches.
template <typename T> constexpr int batch_of(int U) { return 64 * U * El<T>::kVec; }
constexpr int kMaxParts = 64;  // the join holds one per lane
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
  const dim3 block(kThreadsLp);
  if (a.vocab <= kShort) {
    const dim3 grid((unsigned)((a.rows + kThreadsLp / kL - 1) / (kThreadsLp / kL)));
    if (a.top > 4) hipLaunchKernelGGL((sorted_kernel<T>), grid, block, 0, s, a);
    else if (!TOP) hipLaunchKernelGGL((short_kernel<T, 0>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((short_kernel<T, TOP ? 4 : 0>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  if (a.vocab <= batch) {
    const dim3 grid((unsigned)((a.rows + kWaves - 1) / kWaves));
    if constexpr (batch_of<T>(1) > kShort) {  // float32 rows of one batch are short rows
      if (a.vocab <= batch_of<T>(1)) {
        hipLaunchKernelGGL((rows_kernel<T, TOP, 1>), grid, block, 0, s, a);
        return hipGetLastError();
      }
    }
    hipLaunchKernelGGL((rows_kernel<T, TOP, 4>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  const int parts = in_parts ? parts_of(a.rows, a.vocab, batch) : 1;
  const int per = (int)(((int64_t)a.vocab + parts - 1) / parts + 63) / 64 * 64;
  hipLaunchKernelGGL((parts_kernel<T, TOP, 4>), dim3((unsigned)(a.rows * parts)), block, 0, s, a, parts, per);
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
  return parts == 1 ? 0 : (size_t)rows * parts * (sizeof(float4) + top * sizeof(double));
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

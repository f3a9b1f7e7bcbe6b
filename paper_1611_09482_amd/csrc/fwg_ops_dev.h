// Device helpers of the token operators (fwg_embed.hip, fwg_normq.hip, fwg_matmulq.hip,
// fwg_logprob.hip): vectors of float32 or bf16 elements at any element address, reductions over a
// wavefront.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fwg_mfma_dev.h"

namespace fwg {
namespace opd {

using mfd::f32x4;
using mfd::pack2;
using mfd::u32x4;

constexpr float kInf = __builtin_huge_valf();
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Rows may start at any element (odd row lengths, views), so wide accesses promise the element's
// alignment only; the hardware takes them in one instruction all the same.
typedef float f32x4_el __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned int u32x4_el __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned int u32x2_el __attribute__((ext_vector_type(2), aligned(2)));
typedef unsigned int u32x2_b __attribute__((ext_vector_type(2), aligned(1)));

// Elements of one 16-byte access.
template <typename T> struct El;
template <> struct El<float> { static constexpr int kVec = 4; };
template <> struct El<uint16_t> { static constexpr int kVec = 8; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t *p, float v) { *p = (uint16_t)pack2(v, 0.f); }

// N consecutive elements (N a multiple of 4) from or to an element address.
template <int N> __device__ __forceinline__ void load(const float *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const f32x4_el x = *(const f32x4_el *)(p + 4 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[4 * i + j] = x[j];
  }
}
template <int N> __device__ __forceinline__ void load(const uint16_t *p, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i) {
    const u32x4_el x = *(const u32x4_el *)(p + 8 * i);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[8 * i + 2 * j] = mfd::bf_lo(x[j]);
      v[8 * i + 2 * j + 1] = mfd::bf_hi(x[j]);
    }
  }
  if constexpr (N % 8 == 4) {
    const u32x2_el x = *(const u32x2_el *)(p + N - 4);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      v[N - 4 + 2 * j] = mfd::bf_lo(x[j]);
      v[N - 4 + 2 * j + 1] = mfd::bf_hi(x[j]);
    }
  }
}
// Vectors to an element's address.  STREAM: past the caches (outputs too large to be found there by whoever reads them
// next).  Each vector type is named at its store: as a template's argument a type loses its alignment attribute, and
// the store would promise the vector's own.
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
template <bool STREAM> __device__ __forceinline__ void put_vector(float *p, f32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (f32x4_el *)p);
  else *(f32x4_el *)p = v;
}
template <bool STREAM> __device__ __forceinline__ void put_vector(uint16_t *p, u32x4 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (u32x4_el *)p);
  else *(u32x4_el *)p = v;
}
template <bool STREAM> __device__ __forceinline__ void put_vector(uint16_t *p, u32x2 v) {
  if constexpr (STREAM) __builtin_nontemporal_store(v, (u32x2_el *)p);
  else *(u32x2_el *)p = v;
}
// Eight bytes, first to last in (lo, hi).
template <bool STREAM> __device__ __forceinline__ void store_bytes(int8_t *p, uint32_t lo, uint32_t hi) {
  if constexpr (STREAM) __builtin_nontemporal_store(u32x2{lo, hi}, (u32x2_b *)p);
  else *(u32x2_b *)p = u32x2{lo, hi};
}
template <bool STREAM = false, int N> __device__ __forceinline__ void store(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i)
    put_vector<STREAM>(p + 4 * i, f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]});
}
template <bool STREAM = false, int N> __device__ __forceinline__ void store(uint16_t *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 8; ++i)
    put_vector<STREAM>(p + 8 * i, u32x4{pack2(v[8 * i], v[8 * i + 1]), pack2(v[8 * i + 2], v[8 * i + 3]),
                                        pack2(v[8 * i + 4], v[8 * i + 5]), pack2(v[8 * i + 6], v[8 * i + 7])});
  if constexpr (N % 8 == 4) put_vector<STREAM>(p + N - 4, u32x2{pack2(v[N - 4], v[N - 3]), pack2(v[N - 2], v[N - 1])});
}
// To an address that is a multiple of the vector's size, as rows in LDS are.
template <int N> __device__ __forceinline__ void store_aligned(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N / 4; ++i) *(f32x4 *)(p + 4 * i) = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
__device__ __forceinline__ void store_aligned(uint16_t *p, const float (&v)[4]) {
  *(u32x2 *)p = u32x2{pack2(v[0], v[1]), pack2(v[2], v[3])};
}

// The same where only the first `have` elements exist (have may be <= 0 or >= N); absent ones read as `fill`.
template <typename T, int N>
__device__ __forceinline__ void load_part(const T *p, int have, float fill, float (&v)[N]) {
  if (have >= N) {
    load(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = i < have ? to_f(p[i]) : fill;
}
template <bool STREAM = false, typename T, int N>
__device__ __forceinline__ void store_part(T *p, int have, const float (&v)[N]) {
  if (have >= N) {
    store<STREAM>(p, v);
    return;
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (i < have) put(p + i, v[i]);
}

// A wave's LDS accesses are in order; this keeps the compiler to the order of the source.
__device__ __forceinline__ void in_order() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

// Reductions over the wavefront: inside rows of 16 lanes by DPP moves, the four rows by lane reads.
// The result is the same in every lane.
template <int CTRL> __device__ __forceinline__ float dpp_f(float v) { return mfd::dpp<CTRL>(v); }
template <int CTRL> __device__ __forceinline__ int dpp_i(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xF, 0xF, true);
}
__device__ __forceinline__ float wave_max(float m) {
  m = fmaxf(m, dpp_f<0xB1>(m));   // quad_perm [1,0,3,2]
  m = fmaxf(m, dpp_f<0x4E>(m));   // quad_perm [2,3,0,1]
  m = fmaxf(m, dpp_f<0x141>(m));  // row_half_mirror
  m = fmaxf(m, dpp_f<0x140>(m));  // row_mirror
  return fmaxf(fmaxf(mfd::lane_f(m, 0), mfd::lane_f(m, 16)), fmaxf(mfd::lane_f(m, 32), mfd::lane_f(m, 48)));
}
__device__ __forceinline__ float wave_sum(float s) {
  s += dpp_f<0xB1>(s);
  s += dpp_f<0x4E>(s);
  s += dpp_f<0x141>(s);
  s += dpp_f<0x140>(s);
  return (mfd::lane_f(s, 0) + mfd::lane_f(s, 16)) + (mfd::lane_f(s, 32) + mfd::lane_f(s, 48));
}

}  // namespace opd
}  // namespace fwg

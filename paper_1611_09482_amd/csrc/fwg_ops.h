// Launchers of the token operators (embedding, norms and products in 8 and 4 bits, adjusted logits, log
// probabilities), called by their C entries in fwg_ops.cpp, which check every argument first.  Element types: FWG_F32 or
// FWG_BF16; strides in elements.  Not part of the public ABI.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fwg {

// Sets the calling thread's fwg_last_error() message and returns `code` (fwg_host.cpp).
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));

// Outputs from this size on are stored past the caches.  Half of the 256 MB last-level cache and less is better left
// there for whoever reads it next: embed and a sum over its output take 73 us (84 past the caches) at 128 MB, but 126
// (121) at 192 MB and 174 (160) at 256 MB.  norm_quant alone: 89 us (66) at 240 MB, 114 (86) at 320 MB.
constexpr int64_t kStreamBytes = (int64_t)192 << 20;

struct EmbedArgs {
  const void *table;
  const int32_t *tokens;
  void *out;
  int64_t n, ld_table, ld_out;
  int vocab, channels;
  float scale;
};
hipError_t launch_embed(const EmbedArgs &a, int dtype, int out_dtype, hipStream_t s);

struct EmbedGradArgs {
  const void *grad;
  const int32_t *tokens;
  void *out;
  int64_t ld_grad, ld_out;
  int n, vocab, channels;
  float scale;
  unsigned char *ws;
};
size_t embed_grad_bytes(int64_t n, int vocab, int channels);
hipError_t launch_embed_grad(const EmbedGradArgs &a, int dtype, int out_dtype, hipStream_t s);

constexpr int kNormMaxChannels = 32768;
struct NormArgs {
  const void *x, *residual;  // residual may be NULL
  const float *gain;         // NULL: ones
  void *summed;              // may be NULL
  int8_t *q;
  float *scale;
  uint16_t *values;          // may be NULL
  int64_t rows, ld_x, ld_r, ld_s, ld_q, ld_v;
  int channels;
  float eps;
  bool norm;                 // false: x is quantised as it is
};
hipError_t launch_norm_quant(const NormArgs &a, int dtype, hipStream_t s);

constexpr int kQuantMaxInner = 131071;  // 128 * 128 * K stays below 2^31
struct MatmulArgs {
  const int8_t *x, *w;
  const float *x_scale, *w_scale, *bias;  // bias may be NULL
  void *out;
  int64_t M, ld_x, ld_w, ld_o;
  int N, K;
  unsigned char *ws;
};
size_t matmul_quant_bytes(int64_t rows, int outputs, int inner);
hipError_t launch_matmul_quant(const MatmulArgs &a, int out_dtype, hipStream_t s);

constexpr int kMxMaxBlocks = 32768;  // of a product's rows: 2^20 elements
struct MxArgs {
  const void *x, *residual;  // residual may be NULL
  const float *gain;         // NULL: ones
  void *summed;              // may be NULL
  uint8_t *q, *scale;
  float *row_scale;
  uint16_t *values;          // may be NULL
  int64_t rows, ld_x, ld_r, ld_s, ld_q, ld_e, ld_v;
  int channels;
  float eps;
};
hipError_t launch_quant_mx(const MxArgs &a, int dtype, hipStream_t s);  // x, q, scale and values only
hipError_t launch_norm_mx(const MxArgs &a, int dtype, hipStream_t s);

struct MatmulMxArgs {
  const uint8_t *x, *x_scale, *w, *w_scale;
  const float *row_scale, *bias;  // each may be NULL
  void *out;
  int64_t M, ld_x, ld_ex, ld_w, ld_ew, ld_o;
  int N, blocks;
  unsigned char *ws;
};
size_t matmul_mx_bytes(int64_t rows, int outputs, int blocks);
hipError_t launch_matmul_mx(const MatmulMxArgs &a, int out_dtype, hipStream_t s);

struct AdjustArgs {
  const void *logits;
  const int32_t *tokens, *lengths, *prompts;           // each may be NULL
  const float *repetition, *presence, *frequency, *bias;  // each may be NULL
  const uint32_t *allowed;                             // may be NULL
  void *out;
  int64_t rows, ld, ld_t, ld_b, ld_a, ld_o;
  int vocab, history;
};
hipError_t launch_adjust(const AdjustArgs &a, int dtype, hipStream_t s);

constexpr int kMaxTop = 64;  // alternatives are held one per lane
struct LogProbArgs {
  const void *logits;
  const int32_t *tokens;
  float *logp, *entropy, *lse, *top_logp;
  int32_t *top_ids;
  int64_t rows, ld;
  int vocab, top;
  unsigned char *ws;
};
size_t log_probs_bytes(int64_t rows, int vocab, int top, int dtype);
// in_parts: the rows are cut into parts as log_probs_bytes() planned (a.rows are all rows of the call).
hipError_t launch_log_probs(const LogProbArgs &a, int dtype, bool in_parts, hipStream_t s);

struct LogProbGradArgs {
  const void *logits;
  const int32_t *tokens;
  const float *lse, *entropy, *g_logp, *g_entropy;  // g_entropy (and entropy) may be NULL
  void *out;
  int64_t rows, ld, ld_o;
  int vocab;
};
hipError_t launch_log_probs_grad(const LogProbGradArgs &a, int dtype, hipStream_t s);

}  // namespace fwg

// C entries of the token operators: every argument is checked here, before anything is enqueued, then the
// launchers of fwg_ops.h run on the caller's stream.  Nothing is allocated and nothing waits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <cmath>

#include "fwg.h"
#include "fwg_ops.h"

using namespace fwg;

namespace {

constexpr int kMaxVocab = 1 << 29, kMaxChannels = 1 << 20;
constexpr int64_t kMaxRows = (int64_t)1 << 40, kMaxTokens = (int64_t)1 << 30;

int size_of(int dtype) { return dtype == FWG_BF16 ? 2 : 4; }

int check_type(const char *name, int dtype) {
  return dtype == FWG_F32 || dtype == FWG_BF16 ? FWG_OK : fail(FWG_EINVAL, "%s %d is neither FWG_F32 nor FWG_BF16", name, dtype);
}
int check_size(const char *name, int64_t v, int64_t least, int64_t most) {
  if (v < least) return fail(FWG_EINVAL, "%s is %lld: at least %lld is wanted", name, (long long)v, (long long)least);
  if (v > most) return fail(FWG_EUNSUPPORTED, "%s is %lld: at most %lld is supported", name, (long long)v, (long long)most);
  return FWG_OK;
}
int check_ptr(const char *name, const void *p, int align) {
  if (!p) return fail(FWG_EINVAL, "%s is NULL", name);
  if ((uintptr_t)p % align) return fail(FWG_EINVAL, "%s is not aligned to its elements (%d bytes)", name, align);
  return FWG_OK;
}
// Rows that are written must not overlap; rows that are read may (a stride of 0 repeats one row).
int check_stride(const char *name, int64_t stride, int64_t least) {
  if (stride < least) return fail(FWG_EINVAL, "%s is %lld: at least %lld is wanted", name, (long long)stride, (long long)least);
  if (stride > ((int64_t)1 << 40)) return fail(FWG_EUNSUPPORTED, "%s is %lld: at most 2^40 is supported", name, (long long)stride);
  return FWG_OK;
}
int check_workspace(size_t need, const void *ws, size_t bytes) {
  if (need == 0) return FWG_OK;
  if (!ws) return fail(FWG_EINVAL, "workspace is NULL: %zu bytes are needed", need);
  if (bytes < need) return fail(FWG_ENOSPACE, "workspace of %zu bytes: %zu are needed", bytes, need);
  if ((uintptr_t)ws % 256) return fail(FWG_ENOSPACE, "workspace is not aligned to 256 bytes");
  return FWG_OK;
}
int done(hipError_t e, const char *what) {
  return e == hipSuccess ? FWG_OK : fail(FWG_EHIP, "%s: %s", what, hipGetErrorString(e));
}

#define CHECK(expr)                \
  do {                             \
    const int rc_ = (expr);        \
    if (rc_ != FWG_OK) return rc_; \
  } while (0)

// Rows of one launch: a launch has at most 2^32 threads, and no operator gives a row more than 256 threads for
// each 256 of its elements.
int64_t rows_per_launch(int64_t width) {
  const int64_t n = ((int64_t)1 << 23) / ((width + 255) / 256);
  return n < 1 ? 1 : n;
}

template <typename T> T *at(T *p, int64_t elements, int dtype) {
  return p ? (T *)((uintptr_t)p + (uintptr_t)(elements * size_of(dtype))) : nullptr;
}

int log_probs_sizes(int dtype, int64_t rows, int32_t vocab, int32_t top) {
  CHECK(check_type("dtype", dtype));
  CHECK(check_size("rows", rows, 0, kMaxRows));
  CHECK(check_size("vocab", vocab, 1, kMaxVocab));
  CHECK(check_size("top", top, 0, kMaxTop));
  if (top > vocab) return fail(FWG_EINVAL, "top is %d: there are %d tokens", top, vocab);
  return FWG_OK;
}

int norm_impl(NormArgs a, int dtype, void *hip_stream) {
  CHECK(check_type("dtype", dtype));
  CHECK(check_size("rows", a.rows, 0, kMaxRows));
  CHECK(check_size("channels", a.channels, 1, kNormMaxChannels));
  CHECK(check_stride("x_stride", a.ld_x, 0));
  CHECK(check_stride("q_stride", a.ld_q, a.channels));
  if (a.residual) CHECK(check_stride("residual_stride", a.ld_r, 0));
  if (a.summed) CHECK(check_stride("summed_stride", a.ld_s, a.channels));
  if (a.values) CHECK(check_stride("values_stride", a.ld_v, a.channels));
  if (a.norm && !(a.eps >= 0.f && std::isfinite(a.eps))) return fail(FWG_EINVAL, "eps has to be finite and not negative");
  if (a.rows == 0) return FWG_OK;
  CHECK(check_ptr("x", a.x, size_of(dtype)));
  if (a.residual) CHECK(check_ptr("residual", a.residual, size_of(dtype)));
  if (a.gain) CHECK(check_ptr("gain", a.gain, 4));
  if (a.summed) CHECK(check_ptr("summed", a.summed, size_of(dtype)));
  CHECK(check_ptr("q", a.q, 1));
  CHECK(check_ptr("scale", a.scale, 4));
  if (a.values) CHECK(check_ptr("values", a.values, 2));
  const int64_t rows = a.rows, per = rows_per_launch(a.channels);
  for (int64_t r = 0; r < rows; r += per) {
    NormArgs b = a;
    b.rows = rows - r < per ? rows - r : per;
    b.x = at(a.x, r * a.ld_x, dtype);
    b.residual = at(a.residual, r * a.ld_r, dtype);
    b.summed = at(a.summed, r * a.ld_s, dtype);
    b.q = a.q + r * a.ld_q;
    b.scale = a.scale + r;
    if (a.values) b.values = a.values + r * a.ld_v;
    CHECK(done(launch_norm_quant(b, dtype, (hipStream_t)hip_stream), "norm_quant"));
  }
  return FWG_OK;
}

}  // namespace

extern "C" {

int fwg_embed(int32_t dtype, int32_t out_dtype, int64_t n, int32_t vocab, int32_t channels, const void *table,
              int64_t table_stride, const int32_t *tokens, float scale, void *out, int64_t out_stride, void *hip_stream) {
  CHECK(check_type("dtype", dtype));
  CHECK(check_type("out_dtype", out_dtype));
  CHECK(check_size("n", n, 0, kMaxRows));
  CHECK(check_size("vocab", vocab, 1, kMaxVocab));
  CHECK(check_size("channels", channels, 1, kMaxChannels));
  CHECK(check_stride("table_stride", table_stride, 0));
  CHECK(check_stride("out_stride", out_stride, channels));
  if (n == 0) return FWG_OK;
  CHECK(check_ptr("table", table, size_of(dtype)));
  CHECK(check_ptr("tokens", tokens, 4));
  CHECK(check_ptr("out", out, size_of(out_dtype)));
  const int64_t per = rows_per_launch(channels);
  for (int64_t r = 0; r < n; r += per) {
    EmbedArgs a{table,      tokens + r, at(out, r * out_stride, out_dtype), n - r < per ? n - r : per, table_stride,
                out_stride, vocab,      channels,                           scale};
    CHECK(done(launch_embed(a, dtype, out_dtype, (hipStream_t)hip_stream), "embed"));
  }
  return FWG_OK;
}

int fwg_embed_grad_workspace(int64_t n, int32_t vocab, int32_t channels, size_t *bytes) {
  if (!bytes) return fail(FWG_EINVAL, "bytes is NULL");
  CHECK(check_size("n", n, 0, kMaxTokens));
  CHECK(check_size("vocab", vocab, 1, kMaxVocab));
  CHECK(check_size("channels", channels, 1, kMaxChannels));
  *bytes = embed_grad_bytes(n, vocab, channels);
  return FWG_OK;
}

int fwg_embed_grad(int32_t dtype, int32_t out_dtype, int64_t n, int32_t vocab, int32_t channels, const void *grad,
                   int64_t grad_stride, const int32_t *tokens, float scale, void *out, int64_t out_stride,
                   void *workspace, size_t ws_bytes, void *hip_stream) {
  CHECK(check_type("dtype", dtype));
  CHECK(check_type("out_dtype", out_dtype));
  size_t need = 0;
  CHECK(fwg_embed_grad_workspace(n, vocab, channels, &need));
  CHECK(check_stride("grad_stride", grad_stride, 0));
  CHECK(check_stride("out_stride", out_stride, channels));
  CHECK(check_ptr("out", out, size_of(out_dtype)));
  if (n > 0) {
    CHECK(check_ptr("grad", grad, size_of(dtype)));
    CHECK(check_ptr("tokens", tokens, 4));
  }
  CHECK(check_workspace(need, workspace, ws_bytes));
  EmbedGradArgs a{grad, tokens, out, grad_stride, out_stride, (int)n, vocab, channels, scale, (unsigned char *)workspace};
  return done(launch_embed_grad(a, dtype, out_dtype, (hipStream_t)hip_stream), "embed_grad");
}

int fwg_quant_rows(int32_t dtype, int64_t rows, int32_t channels, const void *x, int64_t x_stride, int8_t *q,
                   int64_t q_stride, float *scale, void *hip_stream) {
  NormArgs a{};
  a.x = x;
  a.q = q;
  a.scale = scale;
  a.rows = rows;
  a.ld_x = x_stride;
  a.ld_q = q_stride;
  a.channels = channels;
  a.norm = false;
  return norm_impl(a, dtype, hip_stream);
}

int fwg_norm_quant(int32_t dtype, int64_t rows, int32_t channels, const void *x, int64_t x_stride, const void *residual,
                   int64_t residual_stride, const float *gain, float eps, void *summed, int64_t summed_stride, int8_t *q,
                   int64_t q_stride, float *scale, uint16_t *values, int64_t values_stride, void *hip_stream) {
  NormArgs a{x,        residual, gain,            summed,        q,        scale,         values,   rows,
             x_stride, residual_stride, summed_stride, q_stride, values_stride, channels, eps,      true};
  return norm_impl(a, dtype, hip_stream);
}

int fwg_matmul_quant_workspace(int64_t rows, int32_t outputs, int32_t inner, size_t *bytes) {
  if (!bytes) return fail(FWG_EINVAL, "bytes is NULL");
  CHECK(check_size("rows", rows, 0, kMaxTokens));
  CHECK(check_size("outputs", outputs, 1, kMaxVocab));
  CHECK(check_size("inner", inner, 1, kQuantMaxInner));
  *bytes = rows ? matmul_quant_bytes(rows, outputs, inner) : 0;
  return FWG_OK;
}

int fwg_matmul_quant(int32_t out_dtype, int64_t rows, int32_t outputs, int32_t inner, const int8_t *x, int64_t x_stride,
                     const float *x_scale, const int8_t *w, int64_t w_stride, const float *w_scale, const float *bias,
                     void *out, int64_t out_stride, void *workspace, size_t ws_bytes, void *hip_stream) {
  CHECK(check_type("out_dtype", out_dtype));
  size_t need = 0;
  CHECK(fwg_matmul_quant_workspace(rows, outputs, inner, &need));
  CHECK(check_stride("x_stride", x_stride, 0));
  CHECK(check_stride("w_stride", w_stride, 0));
  CHECK(check_stride("out_stride", out_stride, outputs));
  if (rows == 0) return FWG_OK;
  CHECK(check_ptr("x", x, 1));
  CHECK(check_ptr("x_scale", x_scale, 4));
  CHECK(check_ptr("w", w, 1));
  CHECK(check_ptr("w_scale", w_scale, 4));
  if (bias) CHECK(check_ptr("bias", bias, 4));
  CHECK(check_ptr("out", out, size_of(out_dtype)));
  CHECK(check_workspace(need, workspace, ws_bytes));
  MatmulArgs a{x, w, x_scale, w_scale, bias, out, rows, x_stride, w_stride, out_stride, outputs, inner, (unsigned char *)workspace};
  return done(launch_matmul_quant(a, out_dtype, (hipStream_t)hip_stream), "matmul_quant");
}

int fwg_log_probs_workspace(int32_t dtype, int64_t rows, int32_t vocab, int32_t top, size_t *bytes) {
  if (!bytes) return fail(FWG_EINVAL, "bytes is NULL");
  CHECK(log_probs_sizes(dtype, rows, vocab, top));
  *bytes = log_probs_bytes(rows, vocab, top, dtype);
  return FWG_OK;
}

int fwg_log_probs(int32_t dtype, int64_t rows, int32_t vocab, const void *logits, int64_t logits_stride,
                  const int32_t *tokens, int32_t top, float *logp, float *entropy, float *lse, int32_t *top_ids,
                  float *top_logp, void *workspace, size_t ws_bytes, void *hip_stream) {
  size_t need = 0;
  CHECK(fwg_log_probs_workspace(dtype, rows, vocab, top, &need));
  CHECK(check_stride("logits_stride", logits_stride, 0));
  if (rows == 0) return FWG_OK;
  CHECK(check_ptr("logits", logits, size_of(dtype)));
  CHECK(check_ptr("tokens", tokens, 4));
  CHECK(check_ptr("logp", logp, 4));
  CHECK(check_ptr("entropy", entropy, 4));
  CHECK(check_ptr("lse", lse, 4));
  if (top) {
    CHECK(check_ptr("top_ids", top_ids, 4));
    CHECK(check_ptr("top_logp", top_logp, 4));
  }
  CHECK(check_workspace(need, workspace, ws_bytes));
  // a launch of many rows takes them in slices; rows are cut into parts (and need workspace) only where they are few
  const int64_t per = need ? rows : rows_per_launch(vocab);
  for (int64_t r = 0; r < rows; r += per) {
    LogProbArgs a{at(logits, r * logits_stride, dtype), tokens + r, logp + r, entropy + r, lse + r,
                  top ? top_logp + r * top : nullptr, top ? top_ids + r * top : nullptr,
                  rows - r < per ? rows - r : per, logits_stride, vocab, top, (unsigned char *)workspace};
    CHECK(done(launch_log_probs(a, dtype, need != 0, (hipStream_t)hip_stream), "log_probs"));
  }
  return FWG_OK;
}

int fwg_log_probs_grad(int32_t dtype, int64_t rows, int32_t vocab, const void *logits, int64_t logits_stride,
                       const int32_t *tokens, const float *lse, const float *entropy, const float *grad_logp,
                       const float *grad_entropy, void *out, int64_t out_stride, void *hip_stream) {
  CHECK(log_probs_sizes(dtype, rows, vocab, 0));
  CHECK(check_stride("logits_stride", logits_stride, 0));
  CHECK(check_stride("out_stride", out_stride, vocab));
  if (rows == 0) return FWG_OK;
  CHECK(check_ptr("logits", logits, size_of(dtype)));
  CHECK(check_ptr("tokens", tokens, 4));
  CHECK(check_ptr("lse", lse, 4));
  CHECK(check_ptr("grad_logp", grad_logp, 4));
  if (grad_entropy) {
    CHECK(check_ptr("grad_entropy", grad_entropy, 4));
    CHECK(check_ptr("entropy", entropy, 4));
  }
  CHECK(check_ptr("out", out, size_of(dtype)));
  const int64_t per = rows_per_launch(vocab);
  for (int64_t r = 0; r < rows; r += per) {
    LogProbGradArgs a{at(logits, r * logits_stride, dtype), tokens + r, lse + r, entropy ? entropy + r : nullptr,
                      grad_logp + r, grad_entropy ? grad_entropy + r : nullptr, at(out, r * out_stride, dtype),
                      rows - r < per ? rows - r : per, logits_stride, out_stride, vocab};
    CHECK(done(launch_log_probs_grad(a, dtype, (hipStream_t)hip_stream), "log_probs_grad"));
  }
  return FWG_OK;
}

}  // extern "C"

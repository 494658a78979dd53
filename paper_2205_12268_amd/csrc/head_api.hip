// C ABI of the operators of a model's head: argument checks, then one launcher each.
#include <cmath>

#include "ctx.h"
#include "head.h"

namespace wcc {
namespace {

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1, kMostWidth = 1 << 20;

bool real_type(int t) { return t == WCC_F32 || t == WCC_BF16; }
bool off_grid(const void *p, int t) { return (reinterpret_cast<uintptr_t>(p) & (t == WCC_F32 ? 3 : 1)) != 0; }
bool off_word(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }
bool bad_stride(int64_t ld, int64_t width) { return ld < width || ld > kMostRows; }

wcc_status check(const wcc_adapter_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype)) return WCC_ERR_DTYPE;
  if (d->rows < 0 || d->rows > kMostRows) return WCC_ERR_SHAPE;
  if (d->C_in < 1 || d->C_in > kMostWidth || d->C_out < 1 || d->C_out > kMostWidth) return WCC_ERR_SHAPE;
  if (d->adapters < 0 || d->rank < 0 || (d->adapters > 0 && d->rank < 1)) return WCC_ERR_SHAPE;
  if (d->rank > WCC_MAX_RANK) return WCC_ERR_UNSUPPORTED;
  // (lines of all adapters are counted in 32 bits)
  if ((int64_t)d->adapters * d->rank > kMostRows) return WCC_ERR_SHAPE;
  if (bad_stride(d->ldx, d->C_in) || bad_stride(d->ldy, d->C_out)) return WCC_ERR_SHAPE;
  return WCC_OK;
}

wcc_status check(const wcc_scores_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype)) return WCC_ERR_DTYPE;
  if (d->rows < 0 || d->rows > kMostRows || d->V < 1 || bad_stride(d->ld, d->V)) return WCC_ERR_SHAPE;
  if (d->top < 0 || d->top > d->V) return WCC_ERR_SHAPE;
  if (d->top > WCC_MAX_TOP) return WCC_ERR_UNSUPPORTED;
  return WCC_OK;
}

wcc_status check(const wcc_distill_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype) || !real_type(d->t_dtype)) return WCC_ERR_DTYPE;
  if (d->rows < 0 || d->rows > kMostRows || d->V < 1 || d->K < 1) return WCC_ERR_SHAPE;
  if (bad_stride(d->ld, d->V) || bad_stride(d->ld_grad, d->V)) return WCC_ERR_SHAPE;
  // (exponents are made with log2(e) / temperature)
  if (!(d->temperature > 0.f) || !std::isfinite(d->temperature) || !std::isfinite(1.f / d->temperature * 1.44269504f)) return WCC_ERR_SHAPE;
  if (d->K > WCC_MAX_TEACHER) return WCC_ERR_UNSUPPORTED;
  return WCC_OK;
}

wcc_status need(const wcc_ctx *ctx, size_t bytes) {
  return bytes > 0 && (!ctx->ws || ctx->ws_bytes < bytes) ? WCC_ERR_WORKSPACE : WCC_OK;
}

}  // namespace
}  // namespace wcc

using namespace wcc;

extern "C" {

wcc_status wcc_adapter_workspace_bytes(const wcc_adapter_desc *desc, size_t *bytes) {
  if (!bytes) return WCC_ERR_NULL;
  const wcc_status st = check(desc);
  if (st == WCC_OK) *bytes = adapter_bytes(*desc);
  return st;
}

wcc_status wcc_adapter_forward(wcc_ctx *ctx, const wcc_adapter_desc *desc, const void *x, const void *w,
                               const int32_t *adapter_of_row, const void *a, const void *b, const int32_t *ranks,
                               const float *scale, void *y, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  const int t = desc->dtype;
  if (!x || !w || !y) return WCC_ERR_NULL;
  const bool low = desc->adapters > 0 && adapter_of_row;
  if (low && (!a || !b)) return WCC_ERR_NULL;
  if (off_grid(x, t) || off_grid(w, t) || off_grid(y, t)) return WCC_ERR_ALIGN;
  if (low && (off_grid(a, t) || off_grid(b, t) || off_word(adapter_of_row) || off_word(ranks) || off_word(scale)))
    return WCC_ERR_ALIGN;
  if ((st = need(ctx, adapter_bytes(*desc))) != WCC_OK) return st;
  const AdapterArgs g{x, w, low ? adapter_of_row : nullptr, a, b, ranks, scale, nullptr, y, nullptr, nullptr,
                      static_cast<char *>(ctx->ws)};
  WCC_TRY(launch_adapter_forward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_adapter_backward(wcc_ctx *ctx, const wcc_adapter_desc *desc, const void *x, const void *w,
                                const int32_t *adapter_of_row, const void *a, const void *b, const int32_t *ranks,
                                const float *scale, const void *dy, void *dx, float *da, float *db, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  const int t = desc->dtype;
  const bool some = desc->adapters > 0, low = some && adapter_of_row;
  float *const ga = some ? da : nullptr, *const gb = some ? db : nullptr;
  if (desc->rows > 0) {
    if (!dy || (dx && !w) || ((ga || gb) && !x)) return WCC_ERR_NULL;
    if (low && (!a || !b)) return WCC_ERR_NULL;
    if (off_grid(dy, t) || off_grid(dx, t) || off_grid(w, t) || off_grid(x, t)) return WCC_ERR_ALIGN;
    if (low && (off_grid(a, t) || off_grid(b, t) || off_word(adapter_of_row) || off_word(ranks) || off_word(scale)))
      return WCC_ERR_ALIGN;
  }
  if (off_word(ga) || off_word(gb)) return WCC_ERR_ALIGN;
  if (!ga && !gb && (!dx || desc->rows == 0)) return WCC_OK;
  if ((st = need(ctx, adapter_bytes(*desc))) != WCC_OK) return st;
  const AdapterArgs g{x, w, low && desc->rows > 0 ? adapter_of_row : nullptr, a, b, ranks, scale, dy,
                      desc->rows > 0 ? dx : nullptr, ga, gb, static_cast<char *>(ctx->ws)};
  WCC_TRY(launch_adapter_backward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_scores_workspace_bytes(const wcc_scores_desc *desc, size_t *bytes) {
  if (!bytes) return WCC_ERR_NULL;
  const wcc_status st = check(desc);
  if (st == WCC_OK) *bytes = scores_bytes(*desc);
  return st;
}

wcc_status wcc_token_scores(wcc_ctx *ctx, const wcc_scores_desc *desc, const void *logits, const int32_t *tokens,
                            float *logprob, float *entropy, int32_t *top_idx, float *top_logprob, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  if (!logits || (logprob && !tokens) || (desc->top > 0 && !top_idx)) return WCC_ERR_NULL;
  if (off_grid(logits, desc->dtype) || off_word(tokens) || off_word(logprob) || off_word(entropy) || off_word(top_idx) ||
      off_word(top_logprob))
    return WCC_ERR_ALIGN;
  if ((st = need(ctx, scores_bytes(*desc))) != WCC_OK) return st;
  const ScoresArgs g{logits, tokens, logprob, entropy, top_idx, top_logprob, static_cast<char *>(ctx->ws)};
  WCC_TRY(launch_scores(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_distill_workspace_bytes(const wcc_distill_desc *desc, size_t *bytes) {
  if (!bytes) return WCC_ERR_NULL;
  const wcc_status st = check(desc);
  if (st == WCC_OK) *bytes = distill_bytes(*desc);
  return st;
}

wcc_status wcc_distill_forward(wcc_ctx *ctx, const wcc_distill_desc *desc, const void *logits, const int32_t *t_idx,
                               const void *t_logit, float *loss, float *stats, const float *weight, void *dlogits,
                               void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  if (!logits || !t_idx || !t_logit || !loss) return WCC_ERR_NULL;
  if (dlogits == logits && desc->ld != desc->ld_grad) return WCC_ERR_SHAPE;
  if (off_grid(logits, desc->dtype) || off_grid(dlogits, desc->dtype) || off_grid(t_logit, desc->t_dtype) || off_word(t_idx) ||
      off_word(loss) || off_word(stats) || off_word(weight))
    return WCC_ERR_ALIGN;
  if ((st = need(ctx, distill_bytes(*desc))) != WCC_OK) return st;
  const DistillArgs g{logits, t_idx, t_logit, loss, stats, weight, dlogits, static_cast<char *>(ctx->ws)};
  WCC_TRY(launch_distill_forward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_distill_backward(wcc_ctx *ctx, const wcc_distill_desc *desc, const void *logits, const int32_t *t_idx,
                                const void *t_logit, const float *stats, const float *weight, void *dlogits, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  if (!logits || !t_idx || !t_logit || !stats || !dlogits) return WCC_ERR_NULL;
  if (dlogits == logits && desc->ld != desc->ld_grad) return WCC_ERR_SHAPE;
  if (off_grid(logits, desc->dtype) || off_grid(dlogits, desc->dtype) || off_grid(t_logit, desc->t_dtype) || off_word(t_idx) ||
      off_word(stats) || off_word(weight))
    return WCC_ERR_ALIGN;
  if ((st = need(ctx, distill_bytes(*desc))) != WCC_OK) return st;
  const DistillArgs g{logits, t_idx, t_logit, nullptr, const_cast<float *>(stats), weight, dlogits,
                      static_cast<char *>(ctx->ws)};
  WCC_TRY(launch_distill_backward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

}  // extern "C"

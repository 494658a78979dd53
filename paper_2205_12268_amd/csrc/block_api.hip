// C ABI of the operators of a block on rows: argument checks, then one launcher each.
#include <cmath>

#include "block.h"
#include "ctx.h"

namespace wcc {
namespace {

constexpr int64_t kMostRows = ((int64_t)1 << 31) - 1, kMostWidth = 1 << 20, kMostGroups = 1 << 23;

bool real_type(int t) { return t == WCC_F32 || t == WCC_BF16; }
bool off_grid(const void *p, int t) { return (reinterpret_cast<uintptr_t>(p) & (t == WCC_F32 ? 3 : 1)) != 0; }
bool off_word(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3) != 0; }
bool off_16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }
bool bad_stride(int64_t ld, int64_t width) { return ld < width || ld > kMostRows; }
bool bad_act(int a) { return a < WCC_ACT_NONE || a > WCC_ACT_GELU; }

wcc_status check(const wcc_rows_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype)) return WCC_ERR_DTYPE;
  if (d->rows < 0 || d->rows > kMostRows || d->width < 1 || d->width > kMostWidth || bad_stride(d->ld, d->width)) return WCC_ERR_SHAPE;
  return WCC_OK;
}

wcc_status check(const wcc_group_norm_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype) || bad_act(d->act)) return WCC_ERR_DTYPE;
  if (d->samples < 0 || d->pixels < 1 || d->pixels > kMostRows || d->C < 1 || d->C > kMostWidth) return WCC_ERR_SHAPE;
  if (d->groups < 1 || d->C % d->groups != 0 || !(d->eps > 0.f) || !std::isfinite(d->eps)) return WCC_ERR_SHAPE;
  if (d->samples * d->pixels > kMostRows || (int64_t)d->samples * d->groups > kMostGroups) return WCC_ERR_SHAPE;
  if (bad_stride(d->ldx, d->C) || bad_stride(d->ldy, d->C)) return WCC_ERR_SHAPE;
  return WCC_OK;
}

wcc_status check(const wcc_gated_desc *d) {
  if (!d) return WCC_ERR_NULL;
  if (!real_type(d->dtype) || bad_act(d->act)) return WCC_ERR_DTYPE;
  if (d->rows < 0 || d->rows > kMostRows || d->C_in < 1 || d->C_in > kMostWidth || d->C_out < 1 || d->C_out > kMostWidth) return WCC_ERR_SHAPE;
  if (bad_stride(d->ldx, d->C_in) || bad_stride(d->ldy, d->C_out)) return WCC_ERR_SHAPE;
  // (a launch has fewer than 2^24 workgroups of 256)
  const int64_t rows = (d->rows + 127) / 128, in = (d->C_in + 63) / 64, out = (d->C_out + 63) / 64;
  if (rows * out > kMostGroups || rows * in > kMostGroups || in * out > kMostGroups) return WCC_ERR_UNSUPPORTED;
  return WCC_OK;
}

wcc_status need(const wcc_ctx *ctx, size_t bytes) {
  return bytes > 0 && (!ctx->ws || ctx->ws_bytes < bytes) ? WCC_ERR_WORKSPACE : WCC_OK;
}

wcc_status check_codes(const int8_t *codes, const uint8_t *steps) {
  if (!codes || !steps) return WCC_ERR_NULL;
  return off_16(codes) ? WCC_ERR_ALIGN : WCC_OK;
}

}  // namespace
}  // namespace wcc

using namespace wcc;

extern "C" {

wcc_status wcc_rows_keep(wcc_ctx *ctx, const wcc_rows_desc *desc, const void *x, int8_t *codes, uint8_t *steps, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  if (!x) return WCC_ERR_NULL;
  if ((st = check_codes(codes, steps)) != WCC_OK) return st;
  if (off_grid(x, desc->dtype)) return WCC_ERR_ALIGN;
  WCC_TRY(launch_keep(*desc, KeepArgs{x, nullptr, codes, steps}, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_rows_restore(wcc_ctx *ctx, const wcc_rows_desc *desc, const int8_t *codes, const uint8_t *steps, void *x, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  if (!x) return WCC_ERR_NULL;
  if ((st = check_codes(codes, steps)) != WCC_OK) return st;
  if (off_grid(x, desc->dtype)) return WCC_ERR_ALIGN;
  WCC_TRY(launch_restore(*desc, KeepArgs{nullptr, x, const_cast<int8_t *>(codes), const_cast<uint8_t *>(steps)},
                         static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_group_norm_workspace_bytes(const wcc_group_norm_desc *desc, size_t *bytes) {
  if (!bytes) return WCC_ERR_NULL;
  const wcc_status st = check(desc);
  if (st == WCC_OK) *bytes = norm_bytes(*desc);
  return st;
}

wcc_status wcc_group_norm_forward(wcc_ctx *ctx, const wcc_group_norm_desc *desc, const void *x, const float *gamma, const float *beta,
                                  const int32_t *counts, void *y, float *stats, int8_t *codes, uint8_t *steps, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->samples == 0) return WCC_OK;
  const int t = desc->dtype;
  if (!x || !y) return WCC_ERR_NULL;
  if ((codes || steps) && (st = check_codes(codes, steps)) != WCC_OK) return st;
  if (y == x && desc->ldx != desc->ldy) return WCC_ERR_SHAPE;
  if (off_grid(x, t) || off_grid(y, t) || off_word(gamma) || off_word(beta) || off_word(counts) || off_word(stats)) return WCC_ERR_ALIGN;
  if ((st = need(ctx, norm_bytes(*desc))) != WCC_OK) return st;
  NormArgs g = {};
  g.x = x, g.codes = codes, g.steps = steps, g.gamma = gamma, g.beta = beta, g.counts = counts, g.y = y, g.stats = stats;
  g.ws = static_cast<char *>(ctx->ws);
  WCC_TRY(launch_norm_forward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_group_norm_backward(wcc_ctx *ctx, const wcc_group_norm_desc *desc, const void *x, const int8_t *codes, const uint8_t *steps,
                                   const float *gamma, const float *beta, const int32_t *counts, const float *stats, const void *dy,
                                   void *dx, float *dgamma, float *dbeta, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  const int t = desc->dtype;
  if (desc->samples > 0) {
    if (!dy || !stats) return WCC_ERR_NULL;
    if (!x && (st = check_codes(codes, steps)) != WCC_OK) return st;
    if (dx == dy && desc->ldx != desc->ldy) return WCC_ERR_SHAPE;
    if (off_grid(x, t) || off_grid(dy, t) || off_grid(dx, t) || off_word(gamma) || off_word(beta) || off_word(counts) || off_word(stats))
      return WCC_ERR_ALIGN;
  }
  if (off_word(dgamma) || off_word(dbeta)) return WCC_ERR_ALIGN;
  if (!dgamma && !dbeta && (!dx || desc->samples == 0)) return WCC_OK;
  if ((st = need(ctx, norm_bytes(*desc))) != WCC_OK) return st;
  NormArgs g = {};
  g.x = x, g.codes = const_cast<int8_t *>(codes), g.steps = const_cast<uint8_t *>(steps), g.gamma = gamma, g.beta = beta, g.counts = counts;
  g.stats = const_cast<float *>(stats), g.dy = dy, g.dx = dx, g.dgamma = dgamma, g.dbeta = dbeta, g.ws = static_cast<char *>(ctx->ws);
  WCC_TRY(launch_norm_backward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_gated_workspace_bytes(const wcc_gated_desc *desc, size_t *bytes) {
  if (!bytes) return WCC_ERR_NULL;
  const wcc_status st = check(desc);
  if (st == WCC_OK) *bytes = gated_bytes(*desc, desc->train != 0);
  return st;
}

wcc_status wcc_gated_forward(wcc_ctx *ctx, const wcc_gated_desc *desc, const void *x, const void *w_gate, const void *w_up, void *y,
                             int8_t *codes, uint8_t *steps, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  if (desc->rows == 0) return WCC_OK;
  const int t = desc->dtype;
  if (!x || !w_gate || !w_up || !y) return WCC_ERR_NULL;
  if ((codes || steps) && (st = check_codes(codes, steps)) != WCC_OK) return st;
  if (off_grid(x, t) || off_grid(w_gate, t) || off_grid(w_up, t) || off_grid(y, t)) return WCC_ERR_ALIGN;
  if ((st = need(ctx, gated_bytes(*desc, false))) != WCC_OK) return st;
  GatedArgs g = {};
  g.x = x, g.w_gate = w_gate, g.w_up = w_up, g.codes = codes, g.steps = steps, g.y = y, g.ws = static_cast<char *>(ctx->ws);
  WCC_TRY(launch_gated_forward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

wcc_status wcc_gated_backward(wcc_ctx *ctx, const wcc_gated_desc *desc, const void *x, const int8_t *x_codes, const uint8_t *x_steps,
                              const void *w_gate, const void *w_up, const int8_t *codes, const uint8_t *steps, const void *dy, void *dx,
                              void *dw_gate, void *dw_up, void *stream) {
  if (!ctx) return WCC_ERR_NULL;
  wcc_status st = check(desc);
  if (st != WCC_OK) return st;
  const int t = desc->dtype;
  const bool some = desc->rows > 0;
  if (some) {
    if (!dy) return WCC_ERR_NULL;
    if ((codes || steps) && (st = check_codes(codes, steps)) != WCC_OK) return st;
    const bool again = !codes;  // the projections are made again
    if ((dx || again) && (!w_gate || !w_up)) return WCC_ERR_NULL;
    if ((dw_gate || dw_up || again) && !x && (st = check_codes(x_codes, x_steps)) != WCC_OK) return st;
    if (off_grid(x, t) || off_grid(w_gate, t) || off_grid(w_up, t) || off_grid(dy, t) || off_grid(dx, t)) return WCC_ERR_ALIGN;
  }
  if (off_grid(dw_gate, t) || off_grid(dw_up, t)) return WCC_ERR_ALIGN;
  if (!dw_gate && !dw_up && (!dx || !some)) return WCC_OK;
  if (some && (st = need(ctx, gated_bytes(*desc, true))) != WCC_OK) return st;
  GatedArgs g = {};
  g.x = x, g.x_codes = x_codes, g.x_steps = x_steps, g.w_gate = w_gate, g.w_up = w_up;
  g.codes = const_cast<int8_t *>(codes), g.steps = const_cast<uint8_t *>(steps), g.dy = dy, g.dx = dx, g.dw_gate = dw_gate, g.dw_up = dw_up;
  g.ws = static_cast<char *>(ctx->ws);
  WCC_TRY(launch_gated_backward(*desc, g, static_cast<hipStream_t>(stream)));
  return WCC_OK;
}

}  // extern "C"

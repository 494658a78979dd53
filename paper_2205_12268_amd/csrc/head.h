// The operators of a model's head (rows of tokens): what their translation units share.
#pragma once

#include "wcc_internal.h"

namespace wcc {

struct AdapterArgs {
  const void *x, *w;
  const int32_t *of_row;  // nullable: no row has an adapter
  const void *a, *b;
  const int32_t *ranks;   // nullable: every adapter has all its lines
  const float *scale;     // nullable: 1
  const void *dy;         // backward only
  void *y;                // y, or dx (nullable then)
  float *da, *db;         // backward only, nullable
  char *ws;
};
size_t adapter_bytes(const wcc_adapter_desc &d);
hipError_t launch_adapter_forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s);
hipError_t launch_adapter_backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s);

struct ScoresArgs {
  const void *x;
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_idx;
  float *top_logprob;
  char *ws;
};
size_t scores_bytes(const wcc_scores_desc &d);
hipError_t launch_scores(const wcc_scores_desc &d, const ScoresArgs &g, hipStream_t s);

struct DistillArgs {
  const void *x;
  const int32_t *t_idx;
  const void *t_logit;
  float *loss, *stats;    // forward: written (stats nullable); backward: loss nullptr, stats read
  const float *weight;    // nullable: 1
  void *dx;               // nullable in the forward call
  char *ws;
};
size_t distill_bytes(const wcc_distill_desc &d);
hipError_t launch_distill_forward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s);
hipError_t launch_distill_backward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s);

// ---- elements of rows ----------------------------------------------------------------------------------
// (bf16_t is a bit pattern; the narrowing is the hardware's, to nearest even, NaN kept)
__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return __uint_as_float((uint32_t)v << 16); }
template <class T>
__device__ __forceinline__ T narrow(float v);
template <>
__device__ __forceinline__ float narrow<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t narrow<bf16_t>(float v) {
  return __builtin_bit_cast(bf16_t, (__bf16)v);
}

}  // namespace wcc

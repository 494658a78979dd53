// Distillation from a teacher's top logits: loss and gradient (wcc_distill_forward, wcc_distill_backward).
#include "head.h"

namespace wcc {
namespace {

template <class Op, class T>
__device__ __forceinline__ T block_all(T v, T *part, Op op) {
  for (int off = 32; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int i = 1; i < (int)(blockDim.x >> 6); ++i) v = op(v, part[i]);
  return v;
}

// One workgroup of 256 a row; thread k has the teacher's pair k.
template <class T>
__global__ __launch_bounds__(256) void distill_rows_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int V, int K,
                                                           const int32_t *__restrict__ t_idx, const void *__restrict__ t_logit,
                                                           int t_bf16, float inv_tau, float tau, float *loss, float *stats,
                                                           const float *__restrict__ weight, T *dx, int64_t ldg) {
  __shared__ float fpart[4];
  __shared__ int at_s[256];
  __shared__ float q_s[256];
  auto larger = [](float a, float b) { return fmaxf(a, b); };
  auto sum = [](float a, float b) { return a + b; };
  const int k = threadIdx.x;
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x) {
    const T *r = x + t * ld;
    // the teacher
    int at = k < K ? t_idx[t * K + k] : -1;
    float z = -INFINITY;
    if ((uint32_t)at < (uint32_t)V) z = t_bf16 ? widen(((const bf16_t *)t_logit)[t * K + k]) : ((const float *)t_logit)[t * K + k];
    z *= inv_tau;
    if (z == -INFINITY) at = -1;
    const float zm = block_all(at >= 0 ? z : -INFINITY, fpart, larger);
    const bool some = zm > -INFINITY || zm != zm;
    const float zt = block_all(at >= 0 ? expf(z - zm) : 0.f, fpart, sum);
    const float logq = (z - zm) - logf(zt), q = at >= 0 ? expf(logq) : 0.f;
    const float xk = at >= 0 ? widen(r[at]) * inv_tau : 0.f;
    at_s[k] = at;
    q_s[k] = q;
    // the student
    float m, log_total;
    if (loss) {
      m = -INFINITY;
      for (int v = threadIdx.x; v < V; v += 256) m = fmaxf(m, widen(r[v]) * inv_tau);
      m = block_all(m, fpart, larger);
      const float base = m == -INFINITY ? 0.f : m;
      float total = 0.f;
      for (int v = threadIdx.x; v < V; v += 256) total += expf(widen(r[v]) * inv_tau - base);
      log_total = logf(block_all(total, fpart, sum));
      const bool live = some && log_total != -INFINITY;
      const float l = block_all(live && q > 0.f ? q * (logq - ((xk - m) - log_total)) : 0.f, fpart, sum);
      if (threadIdx.x == 0) {
        loss[t] = tau * tau * l;
        if (stats) stats[2 * t] = m, stats[2 * t + 1] = log_total;
      }
    } else {
      m = stats[2 * t], log_total = stats[2 * t + 1];
    }
    if (!dx) continue;
    const bool live = some && log_total != -INFINITY;
    const float f = tau * (weight ? weight[t] : 1.f);
    float mine = 0.f;  // what the pairs of this index take off
    __syncthreads();
    if (at >= 0)
      for (int i = 0; i < K; ++i)
        if (at_s[i] == at) mine += q_s[i];
    __syncthreads();  // (x may be dx: every pair's logit has been read)
    T *o = dx + t * ldg;
    float keep = 0.f;
    if (at >= 0 && live) keep = f * (expf((xk - m) - log_total) - mine);
    for (int v = threadIdx.x; v < V; v += 256)
      o[v] = narrow<T>(live ? f * expf((widen(r[v]) * inv_tau - m) - log_total) : 0.f);
    __syncthreads();
    if (at >= 0 && live) o[at] = narrow<T>(keep);
    __syncthreads();
  }
}

template <class T>
void launch(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  const unsigned blocks = (unsigned)std::min<int64_t>(d.rows, 1 << 20);
  distill_rows_kernel<T><<<blocks, 256, 0, s>>>((const T *)g.x, d.ld, d.rows, d.V, d.K, g.t_idx, g.t_logit, d.t_dtype == WCC_BF16,
                                               1.f / d.temperature, d.temperature, g.loss, g.stats, g.weight, (T *)g.dx, d.ld_grad);
}

}  // namespace

size_t distill_bytes(const wcc_distill_desc &) { return 0; }

hipError_t launch_distill_forward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  if (d.dtype == WCC_BF16) launch<bf16_t>(d, g, s);
  else launch<float>(d, g, s);
  return hipGetLastError();
}

hipError_t launch_distill_backward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  return launch_distill_forward(d, g, s);
}

}  // namespace wcc

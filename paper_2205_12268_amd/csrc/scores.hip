// Log probabilities of given tokens, entropy and the top alternatives of rows of logits (wcc_token_scores).
#include "head.h"

namespace wcc {
namespace {

// A logit and its index as one number that orders as the answer does: larger logit first, then lower index.  NaN sorts
// above +inf, -0 is +0.
__device__ __forceinline__ uint64_t order_key(float v, int i) {
  const uint32_t u = __float_as_uint(v + 0.f);
  const uint32_t o = v != v ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (uint32_t)~i;
}

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

// One workgroup a row: the maximum, then the sums, then the alternatives one by one.
template <class T>
__global__ __launch_bounds__(256) void scores_rows_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int V, int top,
                                                          const int32_t *__restrict__ tokens, float *logprob, float *entropy,
                                                          int32_t *top_idx, float *top_logprob) {
  __shared__ float fpart[4];
  __shared__ uint64_t kpart[4];
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x) {
    const T *r = x + t * ld;
    auto larger = [](float a, float b) { return fmaxf(a, b); };
    auto sum = [](float a, float b) { return a + b; };
    float m = -INFINITY, total = 0.f, e = 0.f;
    for (int v = threadIdx.x; v < V; v += 256) m = fmaxf(m, widen(r[v]));
    m = block_all(m, fpart, larger);
    const float base = m == -INFINITY ? 0.f : m;
    for (int v = threadIdx.x; v < V; v += 256) {
      const float d = widen(r[v]) - base, p = expf(d);
      total += p;
      e += p == 0.f ? 0.f : p * d;
    }
    total = block_all(total, fpart, sum);
    e = block_all(e, fpart, sum);
    const float log_total = logf(total);  // -inf in a row that has nothing left
    if (threadIdx.x == 0) {
      if (logprob) {
        const int v = tokens[t];
        logprob[t] = (uint32_t)v >= (uint32_t)V ? NAN : total == 0.f ? -INFINITY : (widen(r[v]) - base) - log_total;
      }
      if (entropy) entropy[t] = total == 0.f ? 0.f : log_total - e / total;
    }
    uint64_t last = ~0ull;
    for (int j = 0; j < top; ++j) {
      uint64_t best = 0;
      for (int v = threadIdx.x; v < V; v += 256) {
        const uint64_t k = order_key(widen(r[v]), v);
        if ((j == 0 || k < last) && k > best) best = k;
      }
      last = block_all(best, kpart, [](uint64_t a, uint64_t b) { return a > b ? a : b; });
      if (threadIdx.x == 0) {
        const int v = (int)~(uint32_t)last;
        top_idx[t * top + j] = v;
        if (top_logprob) top_logprob[t * top + j] = total == 0.f ? -INFINITY : (widen(r[v]) - base) - log_total;
      }
    }
  }
}

}  // namespace

size_t scores_bytes(const wcc_scores_desc &) { return 0; }

hipError_t launch_scores(const wcc_scores_desc &d, const ScoresArgs &g, hipStream_t s) {
  const unsigned blocks = (unsigned)std::min<int64_t>(d.rows, 1 << 20);
  if (d.dtype == WCC_BF16)
    scores_rows_kernel<bf16_t><<<blocks, 256, 0, s>>>((const bf16_t *)g.x, d.ld, d.rows, d.V, d.top, g.tokens, g.logprob,
                                                     g.entropy, g.top_idx, g.top_logprob);
  else
    scores_rows_kernel<float><<<blocks, 256, 0, s>>>((const float *)g.x, d.ld, d.rows, d.V, d.top, g.tokens, g.logprob,
                                                    g.entropy, g.top_idx, g.top_logprob);
  return hipGetLastError();
}

}  // namespace wcc

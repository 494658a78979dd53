// Distillation from a teacher's top logits: loss and gradient (wcc_distill_forward, wcc_distill_backward).
//
// With c = log2(e) / temperature, mx a row's largest logit and S = sum 2^((x - mx) c):
//   p = 2^((x - mx) c) / S,   loss = tau^2 sum q (log q - log p),   gradient = w tau (p - q).
// The gradient of a row is p in all places but the teacher's few: a workgroup writes w tau p throughout, then, behind a
// barrier, the teacher's places once more.  Equal indices all write the one value, so no order matters.
//
// Memory is what bounds it: logits in, gradients out.  A workgroup holds a whole row in registers where it fits and there
// are rows enough, and reads it once for loss and gradient both.  Otherwise rows are cut into slices: a first launch leaves
// (mx, S) of every slice and the logits at the teacher's places (the second may overwrite them, dlogits being logits), the
// second joins them, in the order of the slices, in every workgroup that writes a slice's gradient.
// Loss and gradient of 4096 x 65536 bf16: 216 us, 5.0 TB/s, the rate of a large copy, the loss alone 107; with a first form that read rows three times 1062.
#include "rows.h"

namespace wcc {
namespace {

constexpr int kPairs = WCC_MAX_TEACHER;

struct Teacher {
  const int32_t *idx;
  const void *logit;
  int K, bf16;
};

// A row's pairs, pair k with thread k % NT: index (-1: none), q and log q.
template <int NT>
struct Pairs {
  static constexpr int P = NT >= kPairs ? 1 : kPairs / NT;
  int at[P];
  float q[P], log_q[P];
  bool some;
  __device__ __forceinline__ void read(const Teacher &te, int64_t t, int V, float inv_tau) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      const int k = p * NT + (int)threadIdx.x;
      at[p] = -1;
      log_q[p] = -INFINITY;  // (the logit, until solve())
      if (k < te.K) {
        const int i = te.idx[t * te.K + k];
        const float z = (te.bf16 ? widen(static_cast<const bf16_t *>(te.logit)[t * te.K + k])
                                 : static_cast<const float *>(te.logit)[t * te.K + k]) * inv_tau;
        if ((uint32_t)i < (uint32_t)V && z != -INFINITY) at[p] = i, log_q[p] = z;
      }
    }
  }
  __device__ __forceinline__ void solve(float (*part)[16]) {
    float top = -INFINITY;
    bool any = false;
#pragma unroll
    for (int p = 0; p < P; ++p) top = fmaxf(top, log_q[p]), any |= at[p] >= 0;
    top = block_all<NT>(top, part[0], Larger());
    some = __syncthreads_or(any);
    float sum = 0.f;
#pragma unroll
    for (int p = 0; p < P; ++p) sum += at[p] >= 0 ? expf(log_q[p] - top) : 0.f;
    const float log_sum = logf(block_all<NT>(sum, part[1], Sum()));
#pragma unroll
    for (int p = 0; p < P; ++p) {
      log_q[p] = (log_q[p] - top) - log_sum;
      q[p] = at[p] >= 0 ? expf(log_q[p]) : 0.f;
    }
  }
};

// What the pairs of each index take off together, in the order of k; at_s, q_s: LDS of this row's pairs.
template <int NT>
__device__ __forceinline__ void masses(const Pairs<NT> &pr, int K, int *at_s, float *q_s, float (&mass)[Pairs<NT>::P]) {
#pragma unroll
  for (int p = 0; p < Pairs<NT>::P; ++p) {
    const int k = p * NT + (int)threadIdx.x;
    if (k < kPairs) at_s[k] = pr.at[p], q_s[k] = pr.q[p];
    mass[p] = 0.f;
  }
  __syncthreads();
  for (int i = 0; i < K; ++i) {
    const int a = at_s[i];
    const float q = q_s[i];
#pragma unroll
    for (int p = 0; p < Pairs<NT>::P; ++p)
      if (a == pr.at[p]) mass[p] += q;
  }
}

// The exponent of p S to base 2, (a x - b) c.  From a row's own largest a = 1, b = mx, c = log2(e) / tau: the difference comes
// first, so that nothing overflows or is lost beside a large mx.  From the caller's stats a = 1 / tau, b = m, c = log2(e).
struct Exponent {
  float a, b, c;
  __device__ __forceinline__ float operator()(float x) const { return fmaf(x, a, -b) * c; }
};

// w tau p of the vectors of a slice of n elements, to o
template <class T, int NT, int NV>
__device__ __forceinline__ void write_p(T *o, int n, const u32x4 (&v)[NV], const Exponent &ex, float factor, bool live) {
  constexpr int VE = VecOf<T>::N;
  if (!live) {
    store_slice<T, NT, NV>(o, n, [](int) { return u32x4{0, 0, 0, 0}; });
    return;
  }
  store_slice<T, NT, NV>(o, n, [&](int i) {
    float f[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = factor * __builtin_amdgcn_exp2f(ex(elem<T>(v[i], j)));
    return pack<T>(f);
  });
}

// sum 2^((x - mx) c) over the workgroup's vectors, S
template <class T, int NT, int NV>
__device__ __forceinline__ float sum_p(const u32x4 (&v)[NV], float mx, float c, float *part) {
  constexpr int VE = VecOf<T>::N;
  float s[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < VE; ++j) s[j & 1] += __builtin_amdgcn_exp2f((elem<T>(v[i], j) - mx) * c);
  return block_all<NT>(s[0] + s[1], part, Sum());
}

template <class T, int NT, int NV>
__device__ __forceinline__ float largest(const u32x4 (&v)[NV], float *part) {
  constexpr int VE = VecOf<T>::N;
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int j = 0; j < VE; ++j) m = fmaxf(m, elem<T>(v[i], j));
  return block_all<NT>(m, part, Larger());
}

// m = largest / temperature from here on: its rounding to fp32 moves exponents by up to 32 and more, which the log of the sum cannot
// carry (at 1e38 it would leave nothing else of it).  The log of the sum is then relative to the largest logit itself, and from the
// stats a logit's exponent is the difference of quotients rounded alike: 0 at the largest, exact to fp32's steps (32 and more) at others.
constexpr float kFar = 268435456.f;  // 2^28

struct Row {
  float *loss, *stats;
  const float *weight;
  float inv_tau, tau;
  // what a row's logits are taken relative to: its largest, or 0 where nothing is left (then every exponential is 0)
  __device__ __forceinline__ float base(float mx) const { return mx * inv_tau == -INFINITY ? 0.f : mx; }
};

// The loss of a row from its pairs and the logits xk at them; thread 0 writes it.
template <int NT>
__device__ __forceinline__ void write_loss(const Row &o, int64_t t, const Pairs<NT> &pr, const float (&xk)[Pairs<NT>::P], float mx,
                                           float S, float (*part)[16]) {
  const float log_s = logf(S), base = o.base(mx);
  float l = 0.f;
  if (pr.some && S != 0.f) {
#pragma unroll
    for (int p = 0; p < Pairs<NT>::P; ++p)
      if (pr.at[p] >= 0 && !(pr.q[p] == 0.f)) l += pr.q[p] * (pr.log_q[p] - ((xk[p] - base) * o.inv_tau - log_s));
  }
  l = block_all<NT>(l, part[2], Sum());
  if (threadIdx.x == 0) {
    if (o.loss) o.loss[t] = o.tau * o.tau * l;
    if (o.stats) {
      // (m is rounded; what that takes off goes to the other one, whose sum is then relative to m as it is written)
      const float m = S == 0.f ? -INFINITY : mx / o.tau;
      o.stats[2 * t] = m;
      o.stats[2 * t + 1] = S == 0.f ? -INFINITY : fabsf(m) >= kFar ? log_s : log_s + fmaf(base, o.inv_tau, -m);
    }
  }
}

// Whole rows: loss, and with dx their gradients.
template <class T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_row_kernel(const T *x, int64_t ld, int64_t rows, int V, Teacher te, Row out, T *dx,
                                                            int64_t ldg) {
  __shared__ float part[5][16];
  __shared__ int at_s[kPairs];
  __shared__ float q_s[kPairs];
  using Pr = Pairs<NT>;
  const float c = out.inv_tau * kLog2e;
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x) {
    const T *r = x + t * ld;
    u32x4 v[NV];
    load_slice<T, NT, NV>(r, V, v);
    Pr pr;
    pr.read(te, t, V, out.inv_tau);
    float xk[Pr::P];
#pragma unroll
    for (int p = 0; p < Pr::P; ++p) xk[p] = pr.at[p] >= 0 ? widen(r[pr.at[p]]) : 0.f;
    pr.solve(part);
    const float mx = largest<T, NT, NV>(v, part[3]), base = out.base(mx);
    hold(v);
    const float S = sum_p<T, NT, NV>(v, base, c, part[4]);
    write_loss<NT>(out, t, pr, xk, mx, S, part);
    if (dx) {
      float mass[Pr::P];
      masses<NT>(pr, te.K, at_s, q_s, mass);  // (its barrier: every pair's logit has been read, x may be dx)
      hold(v);
      const bool live = pr.some && S != 0.f;
      const float f = out.tau * (out.weight ? out.weight[t] : 1.f);
      T *o = dx + t * ldg;
      const Exponent ex{1.f, base, c};
      write_p<T, NT, NV>(o, V, v, ex, f / S, live);
      __syncthreads();
#pragma unroll
      for (int p = 0; p < Pr::P; ++p)
        if (pr.at[p] >= 0 && live) o[pr.at[p]] = narrow<T>(f * (__builtin_amdgcn_exp2f(ex(xk[p])) / S - mass[p]));
    }
    __syncthreads();  // LDS is used again
  }
}

// (mx, S) of every slice, and of the first slice's workgroup the logits at the teacher's places
template <class T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_stats_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int V, int slices,
                                                              int length, Teacher te, Row out, float2 *__restrict__ parts,
                                                              float *__restrict__ picked) {
  __shared__ float part[2][16];
  const int64_t total = rows * slices;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int64_t t = w / slices;
    const int first = (int)(w - t * slices) * length, n = min(length, V - first);
    const T *r = x + t * ld;
    u32x4 v[NV];
    load_slice<T, NT, NV>(r + first, n, v);
    if (first == 0)
      for (int k = threadIdx.x; k < te.K; k += NT) {
        const int i = te.idx[t * te.K + k];
        picked[t * te.K + k] = (uint32_t)i < (uint32_t)V ? widen(r[i]) : 0.f;
      }
    const float mx = largest<T, NT, NV>(v, part[0]), base = out.base(mx);
    hold(v);
    const float S = sum_p<T, NT, NV>(v, base, out.inv_tau * kLog2e, part[1]);
    if (threadIdx.x == 0) parts[w] = make_float2(mx, S);
    __syncthreads();
  }
}

// The slices' (mx, S) of a row as one, in the order of the threads whatever NT's place in the grid.
template <int NT>
__device__ __forceinline__ float2 join(const float2 *p, int slices, const Row &o, float (*part)[16]) {
  float mx = -INFINITY, S = 0.f;
  for (int i = threadIdx.x; i < slices; i += NT) mx = fmaxf(mx, p[i].x);
  mx = block_all<NT>(mx, part[0], Larger());
  const float base = o.base(mx), c = o.inv_tau * kLog2e;
  for (int i = threadIdx.x; i < slices; i += NT) {
    const float2 q = p[i];
    if (q.y != 0.f) S = fmaf(q.y, __builtin_amdgcn_exp2f((q.x - base) * c), S);
  }
  S = block_all<NT>(S, part[1], Sum());
  return make_float2(mx, S);
}

// The gradient, a slice a workgroup; from the slices' parts (then the first slice's workgroup also writes the loss) or, with
// parts = nullptr, from what out.stats holds.
template <class T, int NT, int NV>
__global__ __launch_bounds__(NT, 4) void distill_grad_kernel(const T *x, int64_t ld, int64_t rows, int V, int slices, int length,
                                                             Teacher te, Row out, const float2 *__restrict__ parts,
                                                             const float *__restrict__ picked, T *dx, int64_t ldg) {
  __shared__ float part[7][16];
  __shared__ int at_s[kPairs];
  __shared__ float q_s[kPairs];
  using Pr = Pairs<NT>;
  const int64_t total = rows * slices;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int64_t t = w / slices;
    const int first = (int)(w - t * slices) * length, n = min(length, V - first);
    const T *r = x + t * ld + first;
    u32x4 v[NV];
    load_slice<T, NT, NV>(r, n, v);
    Pr pr;
    pr.read(te, t, V, out.inv_tau);
    float own[Pr::P];  // the logits at the places in this slice
#pragma unroll
    for (int p = 0; p < Pr::P; ++p) {
      const int i = pr.at[p] - first;
      own[p] = pr.at[p] >= 0 && i >= 0 && i < n ? widen(r[i]) : 0.f;
    }
    pr.solve(part);
    Exponent ex;
    float S;
    if (parts) {
      const float2 j = join<NT>(parts + t * slices, slices, out, part + 3);
      const float mx = j.x;
      S = j.y;
      ex = Exponent{1.f, out.base(mx), out.inv_tau * kLog2e};
      if (first == 0) {
        float xk[Pr::P];
#pragma unroll
        for (int p = 0; p < Pr::P; ++p) {
          const int k = p * NT + (int)threadIdx.x;
          xk[p] = k < te.K ? picked[t * te.K + k] : 0.f;
        }
        write_loss<NT>(out, t, pr, xk, mx, S, part);
      }
    } else {
      ex = Exponent{out.inv_tau, out.stats[2 * t], kLog2e};
      S = expf(out.stats[2 * t + 1]);
      if (fabsf(ex.b) >= kFar) {  // (the differences take the logits' places: bf16 ones are 0 or beyond -2^18, which rounding leaves so)
        auto apart = [&](float z) { return z / out.tau - ex.b; };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          float d[VecOf<T>::N];
#pragma unroll
          for (int j = 0; j < VecOf<T>::N; ++j) d[j] = apart(elem<T>(v[i], j));
          v[i] = pack<T>(d);
        }
#pragma unroll
        for (int p = 0; p < Pr::P; ++p) own[p] = apart(own[p]);
        ex = Exponent{1.f, 0.f, kLog2e};
      }
    }
    float mass[Pr::P];
    masses<NT>(pr, te.K, at_s, q_s, mass);
    const bool live = pr.some && S != 0.f;
    const float f = out.tau * (out.weight ? out.weight[t] : 1.f);
    T *o = dx + t * ldg + first;
    write_p<T, NT, NV>(o, n, v, ex, f / S, live);
    __syncthreads();
#pragma unroll
    for (int p = 0; p < Pr::P; ++p) {
      const int i = pr.at[p] - first;
      if (pr.at[p] >= 0 && i >= 0 && i < n && live)
        o[i] = narrow<T>(f * (__builtin_amdgcn_exp2f(ex(own[p])) / S - mass[p]));
    }
    __syncthreads();
  }
}

// The loss of rows in slices, without a gradient.
__global__ __launch_bounds__(256) void distill_loss_kernel(int64_t rows, int V, int slices, Teacher te, Row out,
                                                           const float2 *__restrict__ parts, const float *__restrict__ picked) {
  __shared__ float part[5][16];
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x) {
    Pairs<256> pr;
    pr.read(te, t, V, out.inv_tau);
    float xk[1] = {(int)threadIdx.x < te.K ? picked[t * te.K + threadIdx.x] : 0.f};
    pr.solve(part);
    const float2 j = join<256>(parts + t * slices, slices, out, part + 3);
    write_loss<256>(out, t, pr, xk, j.x, j.y, part);
    __syncthreads();
  }
}

constexpr int64_t kGridMost = 1 << 20;

// A whole row a workgroup where 1024 threads hold it and there are rows for most compute units, or rows are so short that
// slicing would not help; else slices of up to 256 x 8 vectors, two workgroups a compute unit at least.  (bf16, loss and gradient,
// whole and in slices: 200 rows of 32768 14.3 and 18.9 us, 64 of 32768 12.6 and 13.9, 100 of 120000 26.4 and 22.6.)
SlicePlan plan(const wcc_distill_desc &d, bool backward) {
  const int ve = d.dtype == WCC_BF16 ? 8 : 4;
  const int64_t vecs = ((int64_t)d.V + ve - 1) / ve;
  SlicePlan p{1, d.V, 0, 1};
  if (!backward && vecs <= 1024 * 16 && (d.rows >= 128 || vecs <= 512)) {
    p.nt = vecs <= 64 * 4 ? 64 : vecs <= 256 * 16 ? 256 : vecs <= 512 * 16 ? 512 : 1024;
    while ((int64_t)p.nt * p.nv < vecs) p.nv *= 2;
    return p;
  }
  const int64_t rows = std::max<int64_t>(d.rows, 1);
  int64_t want = (vecs + 256 * 8 - 1) / (256 * 8);
  if (rows * want < 512) want = std::max(want, std::min((512 + rows - 1) / rows, vecs / 256));
  want = std::max<int64_t>(want, 1);
  const int64_t each = (vecs + want - 1) / want;
  p.length = (int)std::min<int64_t>(each * ve, d.V);
  p.slices = (int)(((int64_t)d.V + p.length - 1) / p.length);
  p.nt = each <= 64 * 4 ? 64 : 256;
  while ((int64_t)p.nt * p.nv < each) p.nv *= 2;
  return p;
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

struct Call {
  const wcc_distill_desc &d;
  const DistillArgs &g;
  const SlicePlan &p;
  hipStream_t s;
  Teacher te;
  Row out;
  unsigned blocks;
};

template <class T, int NT, int NV>
void rows_of(const Call &c) {
  distill_row_kernel<T, NT, NV><<<c.blocks, NT, 0, c.s>>>((const T *)c.g.x, c.d.ld, c.d.rows, c.d.V, c.te, c.out, (T *)c.g.dx, c.d.ld_grad);
}

template <class T, int NT, int NV>
void slices_of(const Call &c) {
  const T *x = (const T *)c.g.x;
  T *dx = (T *)c.g.dx;
  if (!c.g.loss) {
    distill_grad_kernel<T, NT, NV><<<c.blocks, NT, 0, c.s>>>(x, c.d.ld, c.d.rows, c.d.V, c.p.slices, c.p.length, c.te, c.out, nullptr,
                                                             nullptr, dx, c.d.ld_grad);
    return;
  }
  float2 *parts = (float2 *)c.g.ws;
  float *picked = (float *)(c.g.ws + align256((size_t)c.d.rows * c.p.slices * 8));
  distill_stats_kernel<T, NT, NV><<<c.blocks, NT, 0, c.s>>>(x, c.d.ld, c.d.rows, c.d.V, c.p.slices, c.p.length, c.te, c.out,
                                                            parts, picked);
  if (dx)
    distill_grad_kernel<T, NT, NV><<<c.blocks, NT, 0, c.s>>>(x, c.d.ld, c.d.rows, c.d.V, c.p.slices, c.p.length, c.te, c.out, parts,
                                                             picked, dx, c.d.ld_grad);
  else
    distill_loss_kernel<<<(unsigned)std::min<int64_t>(c.d.rows, kGridMost), 256, 0, c.s>>>(c.d.rows, c.d.V, c.p.slices, c.te, c.out,
                                                                                          parts, picked);
}

template <class T>
void launch(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  const SlicePlan p = plan(d, !g.loss);
  const Call c{d, g, p, s, Teacher{g.t_idx, g.t_logit, d.K, d.t_dtype == WCC_BF16},
               Row{g.loss, g.stats, g.weight, 1.f / d.temperature, d.temperature},
               (unsigned)std::min<int64_t>(d.rows * p.slices, kGridMost)};
  if (g.loss && p.slices == 1) {
    switch (p.nt * 100 + p.nv) {
      case 6401: return rows_of<T, 64, 1>(c);
      case 6402: return rows_of<T, 64, 2>(c);
      case 6404: return rows_of<T, 64, 4>(c);
      case 25602: return rows_of<T, 256, 2>(c);
      case 25604: return rows_of<T, 256, 4>(c);
      case 25608: return rows_of<T, 256, 8>(c);
      case 25616: return rows_of<T, 256, 16>(c);
      case 51216: return rows_of<T, 512, 16>(c);
      default: return rows_of<T, 1024, 16>(c);
    }
  }
  switch (p.nt * 100 + p.nv) {
    case 6401: return slices_of<T, 64, 1>(c);
    case 6402: return slices_of<T, 64, 2>(c);
    case 6404: return slices_of<T, 64, 4>(c);
    case 25602: return slices_of<T, 256, 2>(c);
    case 25604: return slices_of<T, 256, 4>(c);
    default: return slices_of<T, 256, 8>(c);
  }
}

}  // namespace

size_t distill_bytes(const wcc_distill_desc &d) {
  const SlicePlan p = plan(d, false);
  if (p.slices == 1) return 0;
  return align256((size_t)d.rows * p.slices * 8) + align256((size_t)d.rows * d.K * 4);
}

hipError_t launch_distill_forward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  if (d.dtype == WCC_BF16) launch<bf16_t>(d, g, s);
  else launch<float>(d, g, s);
  return hipGetLastError();
}

hipError_t launch_distill_backward(const wcc_distill_desc &d, const DistillArgs &g, hipStream_t s) {
  return launch_distill_forward(d, g, s);
}

}  // namespace wcc

// Group norm with an activation on maps whose channels come last, forward and backward.
//
// With xh = (x - mean) rstd over the pixels of a sample and the channels of a group, z = gamma xh + beta, y = act(z):
//   dz = dy act'(z), dbeta = sum dz, dgamma = sum dz xh over samples and pixels,
//   dx = rstd (gamma dz - m1 - xh m2), m1 and m2 the means over the group of gamma dz and of gamma dz xh.
// x (backward) is the tensor, or the values that its codes stand for, with the statistics of the tensor.
//
// A thread owns a vector of 16 bytes of channels and walks over pixels, so that sums are by channel and groups may have any size.  The
// sums of x and x^2 are fp64: products of fp32 values are exact there, so that a mean far above the spread costs nothing that a
// shift would have to bring back.
//
// Three launches: sums of chunks of pixels by channel; a small one that joins them; a second pass that goes backwards over the chunks,
// so that it begins with what the caches hold.  Bound by memory: the second pass reads again what the first has read.
#include "block.h"

namespace wcc {
namespace {

struct Shape {
  int64_t pixels, ldx, ldy;
  int samples, C, groups, per;  // per: channels of a group
  float eps;
};

// What is kept in the workspace.
struct Sums {
  double2 *part;  // [samples][chunks][C]
  float4 *group;  // [samples][groups]: mean, rstd, m1, m2
  double2 *chan;  // [samples][C]: backward, sums over a sample
  int chunks;
  int64_t chunk;  // pixels of one
};

__device__ __forceinline__ int64_t pixels_of(const int32_t *counts, int64_t pixels, int sample) {
  return counts ? min((int64_t)max(counts[sample], 0), pixels) : pixels;
}

// The input of the backward pass: x itself, or what it is kept as.
template <class T, bool KEPT>
struct Input {
  const T *x;
  int64_t ld;
  const int8_t *codes;
  const uint8_t *steps;
  int blocks;
  struct Raw {
    u32x4 v;
    uint2 c;
    uint32_t step;
  };
  __device__ __forceinline__ Raw load(int64_t row, int e, int left) const {
    Raw r = {};
    if constexpr (KEPT) {
      const int8_t *p = codes + row * blocks * kKept + e;
      if constexpr (sizeof(T) == 4) r.c.x = *reinterpret_cast<const uint32_t *>(p);
      else r.c = *reinterpret_cast<const uint2 *>(p);
      r.step = steps[row * blocks + e / kKept];
    } else {
      r.v = load_part<T>(x + row * ld + e, left);
    }
    return r;
  }
  __device__ __forceinline__ static float at(const Raw &r, int j, float step) {
    if constexpr (KEPT) return kept_value(j < 4 ? r.c.x : r.c.y, j & 3, step);
    else return elem<T>(r.v, j);
  }
  __device__ __forceinline__ static float step(const Raw &r) { return KEPT ? step_value(r.step) : 0.f; }
};

// A thread's place: `lanes` threads side by side hold vectors of channels, the others of the workgroup further pixels; a workgroup has
// a chunk of a sample's pixels.
template <int VE>
struct Place {
  int sample, chunk, rows, col, ty, c0;
  int64_t begin, end;  // the thread's first pixel, the chunk's end
  __device__ __forceinline__ Place(int64_t b, const Shape &d, const Sums &s, const int32_t *counts, int lanes) {
    sample = (int)(b / s.chunks), chunk = (int)(b % s.chunks);
    rows = 256 / lanes;
    col = threadIdx.x % lanes, ty = threadIdx.x / lanes;
    c0 = (blockIdx.y * lanes + col) * VE;
    begin = chunk * s.chunk + ty;
    end = min(pixels_of(counts, d.pixels, sample), (chunk + 1) * s.chunk);
  }
};

// gamma and beta of a thread's channels; 1 and 0 where there are none
template <int VE>
__device__ __forceinline__ void affine(const float *gamma, const float *beta, int c0, int C, float (&g)[VE], float (&b)[VE]) {
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const int c = min(c0 + j, C - 1);
    g[j] = gamma ? gamma[c] : 1.f;
    b[j] = beta ? beta[c] : 0.f;
  }
}

// the threads' sums by channel added up over the pixels' threads, to the chunk's place in `part`
template <int VE>
__device__ __forceinline__ void leave_sums(const Shape &d, const Sums &s, const Place<VE> &at, int lanes, const double (&a)[VE],
                                           const double (&b)[VE], double2 *room) {
#pragma unroll
  for (int j = 0; j < VE; ++j) room[threadIdx.x * VE + j] = double2{a[j], b[j]};
  __syncthreads();
  const int width = lanes * VE, first = blockIdx.y * width;
  double2 *out = s.part + ((int64_t)at.sample * s.chunks + at.chunk) * d.C + first;
  for (int c = threadIdx.x; c < min(width, d.C - first); c += 256) {
    double2 v = room[c];
    for (int r = 1; r < at.rows; ++r) v.x += room[r * width + c].x, v.y += room[r * width + c].y;
    out[c] = v;
  }
}

// ---- forward: sums of a chunk ------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const T *__restrict__ x, const int32_t *__restrict__ counts, Shape d, Sums s,
                                                        int lanes) {
  constexpr int VE = VecOf<T>::N;
  __shared__ double2 room[256 * VE];
  const Place<VE> at(blockIdx.x, d, s, counts, lanes);
  double sum[VE] = {}, sq[VE] = {};
  if (at.ty < at.rows && at.c0 < d.C) {
    const T *p = x + (int64_t)at.sample * d.pixels * d.ldx + at.c0;
    for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
      u32x4 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = t + u * at.rows < at.end ? load_part<T>(p + (t + u * at.rows) * d.ldx, d.C - at.c0) : u32x4{};
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const double f = elem<T>(v[u], j);
          sum[j] += f, sq[j] = fma(f, f, sq[j]);
        }
    }
  }
  leave_sums<VE>(d, s, at, lanes, sum, sq, room);
}

// ---- the chunks joined: a workgroup for each group of a sample -------------------------------------------------
// `lanes` channels side by side, the other threads over the chunks.  BACK: chan is left too, and m1, m2 beside the statistics.
template <bool BACK>
__global__ __launch_bounds__(256) void norm_join_kernel(const int32_t *__restrict__ counts, Shape d, Sums s, const float *__restrict__ gamma,
                                                        float *__restrict__ stats, int lanes) {
  __shared__ double2 room[256];
  const int group = blockIdx.x % d.groups, sample = blockIdx.x / d.groups, rows = 256 / lanes, tid = threadIdx.x;
  const int col = tid % lanes, ty = tid / lanes;
  const int64_t n = pixels_of(counts, d.pixels, sample);
  const int chunks = (int)min((int64_t)s.chunks, (n + s.chunk - 1) / s.chunk);
  double2 all = {0.0, 0.0};
  for (int c0 = 0; c0 < d.per; c0 += lanes) {
    double2 a = {0.0, 0.0};
    const int c = c0 + col;
    if (ty < rows && c < d.per) {
      const double2 *p = s.part + (int64_t)sample * s.chunks * d.C + group * d.per + c;
#pragma unroll 4
      for (int k = ty; k < chunks; k += rows) {
        const double2 v = p[(int64_t)k * d.C];
        a.x += v.x, a.y += v.y;
      }
    }
    room[tid] = a;
    __syncthreads();
    if (tid < lanes && c < d.per) {
      for (int r = 1; r < rows; ++r) a.x += room[r * lanes + col].x, a.y += room[r * lanes + col].y;
      if constexpr (BACK) {
        s.chan[(int64_t)sample * d.C + group * d.per + c] = a;
        const double w = gamma ? gamma[group * d.per + c] : 1.f;
        a.x *= w, a.y *= w;
      }
      all.x += a.x, all.y += a.y;
    }
    __syncthreads();
  }
  room[tid] = all;  // (0 beyond `lanes`)
  __syncthreads();
  for (int h = 128; h > 0; h >>= 1) {
    if (tid < h) room[tid].x += room[tid + h].x, room[tid].y += room[tid + h].y;
    __syncthreads();
  }
  if (tid != 0) return;
  const double size = (double)max(n * d.per, (int64_t)1);
  const int64_t at = blockIdx.x;
  if constexpr (BACK) {
    s.group[at] = float4{stats[2 * at], stats[2 * at + 1], (float)(room[0].x / size), (float)(room[0].y / size)};
  } else {
    const double mean = room[0].x / size, left = room[0].y / size - mean * mean, var = left < 0.0 ? 0.0 : left;  // (NaN stays)
    const float rstd = (float)(1.0 / sqrt(var + (double)d.eps));
    s.group[at] = float4{(float)mean, rstd, 0.f, 0.f};
    if (stats) stats[2 * at] = (float)mean, stats[2 * at + 1] = rstd;
  }
}

// ---- forward: the second pass ------------------------------------------------------------------------------
template <class T, int ACT, bool KEEP>
__global__ __launch_bounds__(256) void norm_apply_kernel(const T *x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                         const int32_t *__restrict__ counts, Shape d, Sums s, int lanes, T *y,
                                                         int8_t *__restrict__ codes, uint8_t *__restrict__ steps) {
  constexpr int VE = VecOf<T>::N;
  const Place<VE> at(gridDim.x - 1 - blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0, blocks = (d.C + kKept - 1) / kKept;
  if (at.ty >= at.rows || c0 >= (KEEP ? blocks * kKept : d.C)) return;
  float g[VE], b[VE], mean[VE];
  affine<VE>(gamma, beta, c0, d.C, g, b);
#pragma unroll
  for (int j = 0; j < VE; ++j) {
    const float4 q = s.group[(int64_t)at.sample * d.groups + min(c0 + j, d.C - 1) / d.per];
    mean[j] = q.x, g[j] *= q.y;
  }
  const int64_t row0 = (int64_t)at.sample * d.pixels;
  for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
    u32x4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      v[u] = t + u * at.rows < at.end ? load_part<T>(x + (row0 + t + u * at.rows) * d.ldx + c0, d.C - c0) : u32x4{};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = row0 + t + u * at.rows;
      if (t + u * at.rows >= at.end) break;
      if constexpr (KEEP) {  // (the lanes of a block have the same pixels)
        const uint32_t step = step_of(top_of_block<T>(v[u]));
        store_codes<T>(codes + row * blocks * kKept + c0, v[u], per_step(step));
        if (c0 % kKept == 0) steps[row * blocks + c0 / kKept] = (uint8_t)step;
      }
      float f[VE];
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        float slope;
        act_of<T, ACT>(fmaf(elem<T>(v[u], j) - mean[j], g[j], b[j]), f[j], slope);
      }
      store_part<T>(y + row * d.ldy + c0, d.C - c0, pack<T>(f));
    }
  }
}

// ---- backward: sums of a chunk -----------------------------------------------------------------------------
template <class T, int ACT, bool KEPT>
__global__ __launch_bounds__(256) void norm_grad_sums_kernel(Input<T, KEPT> in, const T *__restrict__ dy, const float *__restrict__ gamma,
                                                             const float *__restrict__ beta, const float *__restrict__ stats,
                                                             const int32_t *__restrict__ counts, Shape d, Sums s, int lanes) {
  constexpr int VE = VecOf<T>::N;
  __shared__ double2 room[256 * VE];
  const Place<VE> at(blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0;
  double sum[VE] = {}, dot[VE] = {};
  if (at.ty < at.rows && c0 < d.C) {
    float g[VE], b[VE], mean[VE], rstd[VE];
    affine<VE>(gamma, beta, c0, d.C, g, b);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const int64_t q = 2 * ((int64_t)at.sample * d.groups + min(c0 + j, d.C - 1) / d.per);
      mean[j] = stats[q], rstd[j] = stats[q + 1];
    }
    const int64_t row0 = (int64_t)at.sample * d.pixels;
    for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
      u32x4 w[4];
      typename Input<T, KEPT>::Raw v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int64_t row = row0 + (t + u * at.rows < at.end ? t + u * at.rows : t);
        v[u] = in.load(row, c0, d.C - c0);
        w[u] = load_part<T>(dy + row * d.ldy + c0, d.C - c0);
      }
      float s4[VE] = {}, d4[VE] = {};  // (four at a time in fp32)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (t + u * at.rows >= at.end) break;
        const float step = in.step(v[u]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const float xh = (in.at(v[u], j, step) - mean[j]) * rstd[j];
          float value, slope;
          act_of<T, ACT>(fmaf(xh, g[j], b[j]), value, slope);
          const float dz = elem<T>(w[u], j) * slope;
          s4[j] += dz, d4[j] = fmaf(dz, xh, d4[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) sum[j] += s4[j], dot[j] += d4[j];
    }
  }
  leave_sums<VE>(d, s, at, lanes, sum, dot, room);
}

// ---- backward: the second pass -----------------------------------------------------------------------------
template <class T, int ACT, bool KEPT>
__global__ __launch_bounds__(256) void norm_grad_apply_kernel(Input<T, KEPT> in, const T *dy, const float *__restrict__ gamma,
                                                              const float *__restrict__ beta, const int32_t *__restrict__ counts, Shape d,
                                                              Sums s, int lanes, T *dx) {
  constexpr int VE = VecOf<T>::N;
  const Place<VE> at(gridDim.x - 1 - blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0;
  if (at.ty >= at.rows || c0 >= d.C) return;
  float g[VE], b[VE];
  float4 q[VE];
  affine<VE>(gamma, beta, c0, d.C, g, b);
#pragma unroll
  for (int j = 0; j < VE; ++j) q[j] = s.group[(int64_t)at.sample * d.groups + min(c0 + j, d.C - 1) / d.per];
  const int64_t row0 = (int64_t)at.sample * d.pixels;
  for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
    u32x4 w[4];
    typename Input<T, KEPT>::Raw v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = row0 + (t + u * at.rows < at.end ? t + u * at.rows : t);
      v[u] = in.load(row, c0, d.C - c0);
      w[u] = load_part<T>(dy + row * d.ldy + c0, d.C - c0);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (t + u * at.rows >= at.end) break;
      const float step = in.step(v[u]);
      float f[VE];
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float xh = (in.at(v[u], j, step) - q[j].x) * q[j].y;
        float value, slope;
        act_of<T, ACT>(fmaf(xh, g[j], b[j]), value, slope);
        f[j] = q[j].y * ((elem<T>(w[u], j) * slope) * g[j] - q[j].z - xh * q[j].w);
      }
      store_part<T>(dx + (row0 + t + u * at.rows) * d.ldx + c0, d.C - c0, pack<T>(f));
    }
  }
}

// dgamma and dbeta: a thread for each channel, over the samples in their order
__global__ __launch_bounds__(256) void norm_affine_grad_kernel(const double2 *__restrict__ chan, int samples, int C, float *__restrict__ dgamma,
                                                               float *__restrict__ dbeta) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= C) return;
  double2 a = {0.0, 0.0};
#pragma unroll 4
  for (int i = 0; i < samples; ++i) {
    const double2 v = chan[(int64_t)i * C + c];
    a.x += v.x, a.y += v.y;
  }
  if (dbeta) dbeta[c] = (float)a.x;
  if (dgamma) dgamma[c] = (float)a.y;
}

// ---- host ---------------------------------------------------------------------------------------------------
struct Plan {
  int lanes, cols;  // threads side by side, workgroups side by side
  int chunks;
  int64_t chunk;
  size_t part, group, chan, bytes;
};

size_t up(size_t v) { return (v + 255) / 256 * 256; }

Plan plan_of(const wcc_group_norm_desc &d) {
  const int VE = d.dtype == WCC_F32 ? 4 : 8;
  const int64_t vectors = kept_blocks(d.C) * (kKept / VE);  // (whole blocks: what keeps x needs all lanes of each)
  Plan p;
  p.lanes = (int)std::min<int64_t>(vectors, 256);
  p.cols = (int)((vectors + p.lanes - 1) / p.lanes);
  const int rows = 256 / p.lanes;
  // chunks: as many as give every compute unit eight workgroups, of four pixels a thread at least
  const int64_t most = std::max<int64_t>((d.pixels + 4 * rows - 1) / (4 * rows), 1);
  const int64_t want = std::max<int64_t>(2048 / std::max<int64_t>((int64_t)d.samples * p.cols, 1), 1);
  const int64_t n = std::min(most, want);
  p.chunk = std::max<int64_t>((d.pixels + n - 1) / n, 1);
  p.chunks = (int)std::max<int64_t>((d.pixels + p.chunk - 1) / p.chunk, 1);
  p.part = 0;
  p.group = up((size_t)d.samples * p.chunks * d.C * sizeof(double2));
  p.chan = p.group + up((size_t)d.samples * d.groups * sizeof(float4));
  p.bytes = p.chan + up((size_t)d.samples * d.C * sizeof(double2));
  return p;
}

Sums sums_of(const Plan &p, char *ws) {
  return Sums{reinterpret_cast<double2 *>(ws + p.part), reinterpret_cast<float4 *>(ws + p.group), reinterpret_cast<double2 *>(ws + p.chan),
              p.chunks, p.chunk};
}
Shape shape_of(const wcc_group_norm_desc &d) {
  return Shape{d.pixels, d.ldx, d.ldy, d.samples, d.C, d.groups, d.C / d.groups, d.eps};
}
int join_lanes(const wcc_group_norm_desc &d) { return std::min(d.C / d.groups, 256); }

template <class F>
void by_act(int act, F f) {
  switch (act) {
    case WCC_ACT_RELU: return f(std::integral_constant<int, WCC_ACT_RELU>());
    case WCC_ACT_SILU: return f(std::integral_constant<int, WCC_ACT_SILU>());
    case WCC_ACT_GELU: return f(std::integral_constant<int, WCC_ACT_GELU>());
    default: return f(std::integral_constant<int, WCC_ACT_NONE>());
  }
}

template <class T>
hipError_t forward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t st) {
  const Plan p = plan_of(d);
  const Sums s = sums_of(p, g.ws);
  const Shape sh = shape_of(d);
  const T *x = static_cast<const T *>(g.x);
  T *y = static_cast<T *>(g.y);
  const dim3 grid((unsigned)(p.chunks * d.samples), p.cols);
  norm_sums_kernel<T><<<grid, 256, 0, st>>>(x, g.counts, sh, s, p.lanes);
  norm_join_kernel<false><<<(unsigned)(d.groups * d.samples), 256, 0, st>>>(g.counts, sh, s, nullptr, g.stats, join_lanes(d));
  by_act(d.act, [&](auto act) {
    if (g.codes) norm_apply_kernel<T, act(), true><<<grid, 256, 0, st>>>(x, g.gamma, g.beta, g.counts, sh, s, p.lanes, y, g.codes, g.steps);
    else norm_apply_kernel<T, act(), false><<<grid, 256, 0, st>>>(x, g.gamma, g.beta, g.counts, sh, s, p.lanes, y, nullptr, nullptr);
  });
  return hipGetLastError();
}

template <class T, bool KEPT>
hipError_t backward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t st) {
  const Plan p = plan_of(d);
  const Sums s = sums_of(p, g.ws);
  const Shape sh = shape_of(d);
  const Input<T, KEPT> in{static_cast<const T *>(g.x), d.ldx, g.codes, g.steps, (int)kept_blocks(d.C)};
  const T *dy = static_cast<const T *>(g.dy);
  const dim3 grid((unsigned)(p.chunks * d.samples), p.cols);
  if (d.samples > 0)
    by_act(d.act, [&](auto act) {
      norm_grad_sums_kernel<T, act(), KEPT><<<grid, 256, 0, st>>>(in, dy, g.gamma, g.beta, g.stats, g.counts, sh, s, p.lanes);
      norm_join_kernel<true><<<(unsigned)(d.groups * d.samples), 256, 0, st>>>(g.counts, sh, s, g.gamma, g.stats, join_lanes(d));
      if (g.dx)
        norm_grad_apply_kernel<T, act(), KEPT>
            <<<grid, 256, 0, st>>>(in, dy, g.gamma, g.beta, g.counts, sh, s, p.lanes, static_cast<T *>(g.dx));
    });
  if (g.dgamma || g.dbeta)
    norm_affine_grad_kernel<<<(unsigned)((d.C + 255) / 256), 256, 0, st>>>(s.chan, d.samples, d.C, g.dgamma, g.dbeta);
  return hipGetLastError();
}

}  // namespace

size_t norm_bytes(const wcc_group_norm_desc &d) { return plan_of(d).bytes; }

hipError_t launch_norm_forward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t s) {
  return d.dtype == WCC_F32 ? forward<float>(d, g, s) : forward<bf16_t>(d, g, s);
}
hipError_t launch_norm_backward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t s) {
  if (d.dtype == WCC_F32) return g.x ? backward<float, false>(d, g, s) : backward<float, true>(d, g, s);
  return g.x ? backward<bf16_t, false>(d, g, s) : backward<bf16_t, true>(d, g, s);
}

}  // namespace wcc

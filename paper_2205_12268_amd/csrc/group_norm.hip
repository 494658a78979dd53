// Group norm with an activation on maps whose channels come last, forward and backward.
//
// With xh = (x - mean) rstd over the pixels of a sample and the channels of a group, z = gamma xh + beta, y = act(z):
//   dz = dy act'(z), dbeta = sum dz, dgamma = sum dz xh over samples and pixels,
//   dx = rstd (gamma dz - m1 - xh m2), m1 and m2 the means over the group of gamma dz and of gamma dz xh.
// x (backward) is the tensor, or the values that its codes stand for, with the statistics of the tensor.
//
// A thread owns a vector of 16 bytes of channels and walks over pixels, so that sums are by channel and groups may have any size.  The
// statistics come from fp64 sums of x - s and its square, s the first pixel's value of the group's first channel: the variance of n values
// is at least (s - mean)^2 / n, so what the mean takes from the squares leaves an error of about n 2^-53 at most (with s = 0 it is mean^2 /
// var 2^-53 and its growth over the sums: 10^-4 for a mean of 10^4 beside a spread of 0.05).  The mean is kept as a fp32 value and the rest
// that it rounds off, so y is as near for a mean far above the spread.  The backward pass has the rounded mean of `stats` alone: its xh are
// off by up to 2^-24 |mean| rstd.
//
// Maps that one workgroup's registers hold (a sample, some of its groups) take one launch.  Larger ones take three: sums of chunks of
// pixels by channel; a small one that joins them; a second pass that goes backwards over the chunks, so that it begins with what the caches
// hold; where the chunks are few, the second pass joins them and there are two.  Bound by memory: the second pass reads again what the
// first has read. 8 x 16384 x 256 bf16, 32 groups, silu: 47 to 49 us forward on inputs in turn (19.6 the first pass, 3.4 TB/s beside the y
// of the call before, which is still leaving the caches, and 13 without; 4.8 the join; 22.8 the second, 5.9 TB/s); x to codes beside y 31
// in place of 23; backward from codes 29, 5 and 32 (3.5 and 5.3 TB/s: in its first pass the slopes take as long as the loads).  One map of
// 256 pixels and 96 channels, by registers: 7, nearly all of it the way of one load, the statistics and one store.
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
  float4 *group;  // [samples][groups]: forward: mean, rstd, the mean's rest, s (from the first pass); backward: mean, rstd, m1, m2
  double2 *chan;  // [samples][C]: backward, sums over a sample
  int chunks;
  int64_t chunk;  // pixels of one
};

__device__ __forceinline__ int64_t pixels_of(const int32_t *counts, int64_t pixels, int sample) {
  return counts ? min((int64_t)max(counts[sample], 0), pixels) : pixels;
}

// mean, rstd and the mean's rest from the sums of values less s and of their squares, by 1 / their number.  The reciprocal root is the
// hardware's, two steps of Newton's behind it.
__device__ __forceinline__ float4 stat_of(const double2 &sum, double per, float s, float eps) {
  const double off = sum.x * per, rest = sum.y * per - off * off, v = (rest < 0.0 ? 0.0 : rest) + (double)eps;  // (NaN stays)
  double r = __builtin_amdgcn_rsq(v);
  r = r * fma(-0.5 * v * r, r, 1.5);
  r = r * fma(-0.5 * v * r, r, 1.5);
  const double mean = (double)s + off;
  const float near = (float)mean;
  return float4{near, (float)r, (float)(mean - (double)near), 0.f};
}

// The groups of neighbouring channels from c on, by one division.
struct GroupOf {
  int g, r, per;
  __device__ __forceinline__ GroupOf(int c, int per_) : g(c / per_), r(c - g * per_), per(per_) {}
  __device__ __forceinline__ int next() {  // of this channel; on to the next one
    const int now = g;
    if (++r == per) r = 0, ++g;
    return now;
  }
};

// A thread's vector of channels in a row: `left` of them from c0 on, the rest 0.  Loads have no branch between them, or they would wait for each
// other (7 us for one small map): all are whole, in the row's last vector from where it ends backwards, and are moved and cut where they are
// used.  Rows narrower than a vector are read in pieces.
template <class T>
struct Columns {
  static constexpr int VE = VecOf<T>::N;
  int off, back, left;
  uint32_t mask[4];
  bool cut, narrow;  // (the same for all threads)
  __device__ __forceinline__ Columns(int c0, int left_, int C, bool cut_) : left(max(left_, 0)), cut(cut_), narrow(C < VE) {
    off = narrow ? (left > 0 ? c0 : 0) : min(c0, C - VE);
    back = left > 0 ? c0 - off : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (sizeof(T) == 4) mask[i] = i < left ? ~0u : 0u;
      else mask[i] = 2 * i + 1 < left ? ~0u : 2 * i < left ? 0xffffu : 0u;
    }
  }
  // row(i): the row of vector i, which is there
  template <int N, class F>
  __device__ __forceinline__ void load(u32x4 (&v)[N], F row) const {
    if (!narrow) {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = *reinterpret_cast<const u32x4_any *>(row(i) + off);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) v[i] = load_part<T>(row(i) + off, left);
    }
  }
  __device__ __forceinline__ u32x4 fix(u32x4 v) const {
    if (!cut || narrow) return v;
    const int words = sizeof(T) == 4 ? back : back >> 1;
    if (words & 2) v = u32x4{v[2], v[3], 0, 0};
    if (words & 1) v = u32x4{v[1], v[2], v[3], 0};
    if constexpr (sizeof(T) == 2) {
      if (back & 1) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    }
    return u32x4{v[0] & mask[0], v[1] & mask[1], v[2] & mask[2], v[3] & mask[3]};
  }
};

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
  // vectors of rows row(i), which are there
  template <int N, class F>
  __device__ __forceinline__ void load(Raw (&r)[N], const Columns<T> &cols, int c0, F row) const {
    if constexpr (KEPT) {
      const int e = min(c0, blocks * kKept - VecOf<T>::N);  // (threads past the row's end)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int8_t *p = codes + row(i) * blocks * kKept + e;
        if constexpr (sizeof(T) == 4) r[i].c.x = *reinterpret_cast<const uint32_t *>(p);
        else r[i].c = *reinterpret_cast<const uint2 *>(p);
        r[i].step = steps[row(i) * blocks + e / kKept];
      }
    } else {
      u32x4 v[N];
      cols.load(v, [&](int i) { return x + row(i) * ld; });
#pragma unroll
      for (int i = 0; i < N; ++i) r[i].v = v[i];
    }
  }
  __device__ __forceinline__ static Raw fix(Raw r, const Columns<T> &cols) {
    if constexpr (!KEPT) r.v = cols.fix(r.v);
    return r;
  }
  // element j without the mean
  __device__ __forceinline__ static float at(const Raw &r, int j, float step, float mean) {
    if constexpr (KEPT) return fmaf((float)(int8_t)((j < 4 ? r.c.x : r.c.y) >> (8 * (j & 3))), step, -mean);
    else return elem<T>(r.v, j) - mean;
  }
  __device__ __forceinline__ static float step(const Raw &r) { return KEPT ? step_value(r.step) : 0.f; }
};

// A thread's place: `lanes` threads side by side hold vectors of channels, the others of the workgroup further pixels; a workgroup has
// a chunk of a sample's pixels.
template <int VE>
struct Place {
  int sample, chunk, rows, col, ty, c0;
  int64_t begin, end;  // the thread's first pixel, the chunk's end
  __device__ __forceinline__ Place(int b, const Shape &d, const Sums &s, const int32_t *counts, int lanes) {
    sample = b / s.chunks, chunk = b % s.chunks;
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
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
  const bool whole = c0 + VE <= C;
  auto take = [&](const float *p, float none, float(&v)[VE]) {
    if (!p) {
#pragma unroll
      for (int j = 0; j < VE; ++j) v[j] = none;
    } else if (whole) {
#pragma unroll
      for (int j = 0; j < VE; j += 4) {
        const f32x4_any q = *reinterpret_cast<const f32x4_any *>(p + c0 + j);
        v[j] = q[0], v[j + 1] = q[1], v[j + 2] = q[2], v[j + 3] = q[3];
      }
    } else {
#pragma unroll
      for (int j = 0; j < VE; ++j) v[j] = p[min(c0 + j, C - 1)];
    }
  };
  take(gamma, 1.f, g), take(beta, 0.f, b);
}
// use(j, load(group)) for the channels c + j of a thread, groups up to `last`: one load where they are all of one group
template <int VE, class L, class U>
__device__ __forceinline__ void by_groups(int c, int per, int last, L load, U use) {
  GroupOf of(c, per);
  if (per % VE == 0) {
    const auto q = load(min(of.g, last));
#pragma unroll
    for (int j = 0; j < VE; ++j) use(j, q);
  } else {
#pragma unroll
    for (int j = 0; j < VE; ++j) use(j, load(min(of.next(), last)));
  }
}

// Pairs of sums of NT threads' VE channels in LDS, one channel's after the other (a thread's own side by side would all be on one bank).
template <int NT, int VE>
struct Room {
  double2 v[VE][NT + 1];
  __device__ __forceinline__ void put(const double (&a)[VE], const double (&b)[VE]) {
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j][threadIdx.x] = double2{a[j], b[j]};
  }
  // channel c of the threads from `first` on
  __device__ __forceinline__ double2 at(int first, int c) const { return v[c % VE][first + c / VE]; }
};

// the threads' sums by channel added up over the pixels' threads, to the chunk's place in `part`
template <int VE>
__device__ __forceinline__ void leave_sums(const Shape &d, const Sums &s, const Place<VE> &at, int lanes, const double (&a)[VE],
                                           const double (&b)[VE], Room<256, VE> &room) {
  room.put(a, b);
  __syncthreads();
  const int width = lanes * VE, first = blockIdx.y * width;
  double2 *out = s.part + ((int64_t)at.sample * s.chunks + at.chunk) * d.C + first;
  for (int c = threadIdx.x; c < min(width, d.C - first); c += 256) {
    double2 v = {0.0, 0.0};
    for (int r = 0; r < at.rows; ++r) {
      const double2 q = room.at(r * lanes, c);
      v.x += q.x, v.y += q.y;
    }
    out[c] = v;
  }
}

// A pair of sums for each group from `entries` pairs each, entry(g, i), a power of two of threads for each group; to all[g].
template <int NT, class F>
__device__ __forceinline__ void by_group(int groups, int entries, double2 *all, F entry) {
  int lg = 0;
  while (lg < 6 && groups << (lg + 1) <= NT) ++lg;
  for (int g = threadIdx.x >> lg; g < groups; g += NT >> lg) {
    double2 v = {0.0, 0.0};
    for (int i = threadIdx.x & ((1 << lg) - 1); i < entries; i += 1 << lg) {
      const double2 q = entry(g, i);
      v.x += q.x, v.y += q.y;
    }
    for (int off = 1 << lg >> 1; off > 0; off >>= 1) v.x += __shfl_xor(v.x, off, 64), v.y += __shfl_xor(v.y, off, 64);
    if ((threadIdx.x & ((1 << lg) - 1)) == 0) all[g] = v;
  }
}

// ---- forward: sums of a chunk ------------------------------------------------------------------------------
template <class T>
__global__ __launch_bounds__(256) void norm_sums_kernel(const T *__restrict__ x, const int32_t *__restrict__ counts, Shape d, Sums s,
                                                        int lanes) {
  constexpr int VE = VecOf<T>::N;
  __shared__ Room<256, VE> room;
  const Place<VE> at(blockIdx.x, d, s, counts, lanes);
  const T *p = x + (int64_t)at.sample * d.pixels * d.ldx;
  if (at.chunk == 0) {  // (what joins the chunks may find x overwritten by y)
    const bool some = pixels_of(counts, d.pixels, at.sample) > 0;
    for (int g = blockIdx.y * 256 + threadIdx.x; g < d.groups; g += gridDim.y * 256)
      s.group[(int64_t)at.sample * d.groups + g].w = some ? widen(p[g * d.per]) : 0.f;
  }
  double sum[VE] = {}, sq[VE] = {};
  if (at.ty < at.rows && at.c0 < d.C && at.begin < at.end) {
    double first[VE];
    by_groups<VE>(at.c0, d.per, d.groups - 1, [&](int g) { return widen(p[g * d.per]); }, [&](int j, float q) { first[j] = q; });
    const Columns<T> cols(at.c0, d.C - at.c0, d.C, d.C % VE != 0);
    for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
      u32x4 v[4];
      cols.load(v, [&](int u) { return p + min(t + u * at.rows, at.end - 1) * d.ldx; });
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (t + u * at.rows >= at.end) break;
        v[u] = cols.fix(v[u]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const double f = elem<T>(v[u], j) - first[j];
          sum[j] += f, sq[j] = fma(f, f, sq[j]);
        }
      }
    }
  }
  leave_sums<VE>(d, s, at, lanes, sum, sq, room);
}

// ---- the chunks joined -----------------------------------------------------------------------------------------
// A workgroup for each group of a sample: a power of two (`lanes`, 64 at most) of channels side by side, the other threads over the
// chunks.  BACK: m1 and m2 beside the statistics, and chan is left.
template <bool BACK, int NT>
__global__ __launch_bounds__(NT) void norm_join_kernel(const int32_t *__restrict__ counts, Shape d, Sums s, const float *__restrict__ gamma,
                                                        float *__restrict__ stats, int lanes) {
  __shared__ double2 room[NT / 64][64];
  const int group = blockIdx.x % d.groups, sample = blockIdx.x / d.groups, tid = threadIdx.x, lane = tid & 63;
  const int rows = NT / lanes, col = tid % lanes, ty = tid / lanes;
  const int64_t n = pixels_of(counts, d.pixels, sample);
  const int chunks = (int)min((int64_t)s.chunks, (n + s.chunk - 1) / s.chunk);
  const double per = 1.0 / (double)max(n * d.per, (int64_t)1);
  const float first = BACK ? 0.f : s.group[blockIdx.x].w;
  double2 all = {0.0, 0.0};
  for (int c0 = 0; c0 < d.per; c0 += lanes) {
    const int c = c0 + col;
    double2 a = {0.0, 0.0};
    if (c < d.per) {
      const double2 *p = s.part + (int64_t)sample * s.chunks * d.C + group * d.per + c;
#pragma unroll 8
      for (int k = ty; k < chunks; k += rows) {
        const double2 v = p[(int64_t)k * d.C];
        a.x += v.x, a.y += v.y;
      }
    }
    for (int off = lanes; off < 64; off <<= 1) a.x += __shfl_xor(a.x, off, 64), a.y += __shfl_xor(a.y, off, 64);
    if (lane < lanes) room[tid >> 6][lane] = a;
    __syncthreads();
    if (tid < lanes && c < d.per) {
      a = {0.0, 0.0};
#pragma unroll
      for (int w = 0; w < NT / 64; ++w) a.x += room[w][lane].x, a.y += room[w][lane].y;
      if constexpr (BACK) {
        s.chan[(int64_t)sample * d.C + group * d.per + c] = a;
        const double w = gamma ? gamma[group * d.per + c] : 1.f;
        a.x *= w, a.y *= w;
      }
      all.x += a.x, all.y += a.y;
    }
    __syncthreads();
  }
  if (tid >= 64) return;
  for (int off = lanes >> 1; off > 0; off >>= 1) all.x += __shfl_xor(all.x, off, 64), all.y += __shfl_xor(all.y, off, 64);
  if (tid != 0) return;
  const int64_t at = blockIdx.x;
  if constexpr (BACK) {
    s.group[at] = float4{stats[2 * at], stats[2 * at + 1], (float)(all.x * per), (float)(all.y * per)};
  } else {
    const float4 q = stat_of(all, per, first, d.eps);
    s.group[at] = q;
    if (stats) stats[2 * at] = q.x, stats[2 * at + 1] = q.y;
  }
}

// The same by every workgroup of the second pass for its sample, where the chunks are few and the channels kShort at most: groups'
// values to `group` in LDS.  The sample's first workgroup leaves the statistics.
constexpr int kShort = 512;
struct ShortRoom {
  double2 chan[kShort], all[kShort];
  float4 group[kShort];
};
template <bool BACK>
__device__ __forceinline__ void join_short(int sample, bool first, int64_t n, const Shape &d, const Sums &s, const float *gamma, float *stats,
                                           ShortRoom &room) {
  const int chunks = (int)min((int64_t)s.chunks, (n + s.chunk - 1) / s.chunk);
  const double per = 1.0 / (double)max(n * d.per, (int64_t)1);
  const int parts = max(256 / d.C, 1);
  if constexpr (!BACK) {
    for (int g = threadIdx.x; g < d.groups; g += 256) room.group[g].w = s.group[(int64_t)sample * d.groups + g].w;
  }
  for (int i = threadIdx.x; i < parts * d.C; i += 256) {
    const int c = i % d.C;
    const double2 *p = s.part + (int64_t)sample * s.chunks * d.C + c;
    double2 a = {0.0, 0.0};
#pragma unroll 8
    for (int k = i / d.C; k < chunks; k += parts) {
      const double2 v = p[(int64_t)k * d.C];
      a.x += v.x, a.y += v.y;
    }
    const double w = BACK && gamma ? gamma[c] : 1.f;
    room.chan[i] = double2{a.x * w, a.y * w};
  }
  __syncthreads();
  by_group<256>(d.groups, parts * d.per, room.all, [&](int g, int i) { return room.chan[i / d.per * d.C + g * d.per + i % d.per]; });
  __syncthreads();
  for (int g = threadIdx.x; g < d.groups; g += 256) {
    const int64_t at = (int64_t)sample * d.groups + g;
    if constexpr (BACK) {
      room.group[g] = float4{stats[2 * at], stats[2 * at + 1], (float)(room.all[g].x * per), (float)(room.all[g].y * per)};
    } else {
      const float4 q = stat_of(room.all[g], per, room.group[g].w, d.eps);
      room.group[g] = q;
      if (stats && first) stats[2 * at] = q.x, stats[2 * at + 1] = q.y;
    }
  }
  __syncthreads();
}

// ---- forward: the second pass ------------------------------------------------------------------------------
template <class T, int ACT, bool KEEP, bool SHORT>
__global__ __launch_bounds__(256) void norm_apply_kernel(const T *x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                         const int32_t *__restrict__ counts, Shape d, Sums s, int lanes, T *y,
                                                         float *__restrict__ stats, int8_t *__restrict__ codes,
                                                         uint8_t *__restrict__ steps) {
  constexpr int VE = VecOf<T>::N;
  __shared__ std::conditional_t<SHORT, ShortRoom, char> room;
  const Place<VE> at(gridDim.x - 1 - blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0, blocks = (d.C + kKept - 1) / kKept;
  if constexpr (SHORT)
    join_short<false>(at.sample, at.chunk == 0 && blockIdx.y == 0, pixels_of(counts, d.pixels, at.sample), d, s, nullptr, stats, room);
  if (at.ty >= at.rows || c0 >= (KEEP ? blocks * kKept : d.C)) return;
  float g[VE], b[VE], mean[VE];
  affine<VE>(gamma, beta, c0, d.C, g, b);
  by_groups<VE>(
      c0, d.per, d.groups - 1,
      [&](int group) {
        if constexpr (SHORT) return room.group[group];
        else return s.group[(int64_t)at.sample * d.groups + group];
      },
      [&](int j, const float4 &q) { mean[j] = q.x, g[j] *= q.y, b[j] = fmaf(-q.z, g[j], b[j]); });
  const int64_t row0 = (int64_t)at.sample * d.pixels;
  const Columns<T> cols(c0, d.C - c0, d.C, d.C % (KEEP ? kKept : VE) != 0);
  for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
    u32x4 v[4];
    cols.load(v, [&](int u) { return x + (row0 + min(t + u * at.rows, at.end - 1)) * d.ldx; });
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t row = row0 + t + u * at.rows;
      if (t + u * at.rows >= at.end) break;
      v[u] = cols.fix(v[u]);
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
  __shared__ Room<256, VE> room;
  const Place<VE> at(blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0;
  double sum[VE] = {}, dot[VE] = {};
  if (at.ty < at.rows && c0 < d.C) {
    float g[VE], b[VE], mean[VE], rstd[VE];
    affine<VE>(gamma, beta, c0, d.C, g, b);
    const float *own = stats + 2 * (int64_t)at.sample * d.groups;
    by_groups<VE>(
        c0, d.per, d.groups - 1, [&](int group) { return float2{own[2 * group], own[2 * group + 1]}; },
        [&](int j, const float2 &q) { mean[j] = q.x, rstd[j] = q.y, g[j] *= q.y; });
    const int64_t row0 = (int64_t)at.sample * d.pixels;
    const Columns<T> cols(c0, d.C - c0, d.C, d.C % VE != 0);
    for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
      u32x4 w[4];
      typename Input<T, KEPT>::Raw v[4];
      auto row = [&](int u) { return row0 + min(t + u * at.rows, at.end - 1); };
      in.load(v, cols, c0, row);
      cols.load(w, [&](int u) { return dy + row(u) * d.ldy; });
      float s4[VE] = {}, d4[VE] = {};  // (four at a time in fp32)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        if (t + u * at.rows >= at.end) break;
        v[u] = in.fix(v[u], cols), w[u] = cols.fix(w[u]);
        const float step = in.step(v[u]);
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const float x = in.at(v[u], j, step, mean[j]);
          float value, slope;
          act_of<T, ACT>(fmaf(x, g[j], b[j]), value, slope);
          const float dz = elem<T>(w[u], j) * slope;
          s4[j] += dz, d4[j] = fmaf(dz, x, d4[j]);
        }
      }
#pragma unroll
      for (int j = 0; j < VE; ++j) sum[j] += s4[j], dot[j] += d4[j];
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) dot[j] *= rstd[j];
  }
  leave_sums<VE>(d, s, at, lanes, sum, dot, room);
}

// ---- backward: the second pass -----------------------------------------------------------------------------
// dgamma and dbeta of a channel: n pairs of sums of it, `stride` rows of C apart, in their order
__device__ __forceinline__ double2 sum_of(const double2 *p, int n, int64_t stride) {
  double2 a = {0.0, 0.0};
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const double2 v = p[i * stride];
    a.x += v.x, a.y += v.y;
  }
  return a;
}
__device__ __forceinline__ void affine_grad(int c, int C, const double2 *p, int n, int64_t stride, float *dgamma, float *dbeta) {
  if (c >= C) return;
  const double2 a = sum_of(p + c, n, stride);
  if (dbeta) dbeta[c] = (float)a.x;
  if (dgamma) dgamma[c] = (float)a.y;
}
__global__ __launch_bounds__(256) void norm_affine_grad_kernel(const double2 *__restrict__ p, int C, int n, int64_t stride,
                                                               float *__restrict__ dgamma, float *__restrict__ dbeta) {
  affine_grad(blockIdx.x * 256 + threadIdx.x, C, p, n, stride, dgamma, dbeta);
}
// Many samples: `each` of them joined in the place of their first.
constexpr int kFewSamples = 64;
__global__ __launch_bounds__(256) void norm_samples_kernel(double2 *chan, int C, int samples, int each) {
  const int c = blockIdx.x * 256 + threadIdx.x, first = blockIdx.y * each;
  if (c >= C) return;
  double2 *p = chan + (int64_t)first * C + c;
  *p = sum_of(p, min(each, samples - first), C);
}

// (workgroups past `tiles` do dgamma and dbeta)
template <class T, int ACT, bool KEPT, bool SHORT>
__global__ __launch_bounds__(256) void norm_grad_apply_kernel(Input<T, KEPT> in, const T *dy, const float *__restrict__ gamma,
                                                              const float *__restrict__ beta, const int32_t *__restrict__ counts, Shape d,
                                                              Sums s, int lanes, int tiles, T *dx, float *__restrict__ stats,
                                                              float *__restrict__ dgamma, float *__restrict__ dbeta) {
  constexpr int VE = VecOf<T>::N;
  __shared__ std::conditional_t<SHORT, ShortRoom, char> room;
  if ((int)blockIdx.x >= tiles) {
    if (blockIdx.y == 0)
      affine_grad((blockIdx.x - tiles) * 256 + threadIdx.x, d.C, SHORT ? s.part : s.chan, d.samples * (SHORT ? s.chunks : 1), d.C, dgamma, dbeta);
    return;
  }
  const Place<VE> at(tiles - 1 - blockIdx.x, d, s, counts, lanes);
  const int c0 = at.c0;
  if constexpr (SHORT) join_short<true>(at.sample, false, pixels_of(counts, d.pixels, at.sample), d, s, gamma, stats, room);
  if (at.ty >= at.rows || c0 >= d.C) return;
  float g[VE], b[VE];
  float4 q[VE];
  affine<VE>(gamma, beta, c0, d.C, g, b);
  by_groups<VE>(
      c0, d.per, d.groups - 1,
      [&](int group) {
        float4 v;
        if constexpr (SHORT) v = room.group[group];
        else v = s.group[(int64_t)at.sample * d.groups + group];
        v.z *= v.y, v.w *= v.y * v.y;  // dx = gamma rstd dz - rstd m1 - (x - mean) rstd^2 m2
        return v;
      },
      [&](int j, const float4 &v) { q[j] = v, g[j] *= v.y; });
  const int64_t row0 = (int64_t)at.sample * d.pixels;
  const Columns<T> cols(c0, d.C - c0, d.C, d.C % VE != 0);
  for (int64_t t = at.begin; t < at.end; t += 4 * at.rows) {
    u32x4 w[4];
    typename Input<T, KEPT>::Raw v[4];
    auto row = [&](int u) { return row0 + min(t + u * at.rows, at.end - 1); };
    in.load(v, cols, c0, row);
    cols.load(w, [&](int u) { return dy + row(u) * d.ldy; });
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (t + u * at.rows >= at.end) break;
      v[u] = in.fix(v[u], cols), w[u] = cols.fix(w[u]);
      const float step = in.step(v[u]);
      float f[VE];
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float x = in.at(v[u], j, step, q[j].x);
        float value, slope;
        act_of<T, ACT>(fmaf(x, g[j], b[j]), value, slope);
        f[j] = fmaf(elem<T>(w[u], j) * slope, g[j], -fmaf(x, q[j].w, q[j].z));
      }
      store_part<T>(dx + (row0 + t + u * at.rows) * d.ldx + c0, d.C - c0, pack<T>(f));
    }
  }
}

// ---- maps that a workgroup's registers hold: one launch --------------------------------------------------------
// A workgroup has a sample's pixels of `take` neighbouring groups; `lanes` threads side by side hold vectors of their channels (from the
// first group's on, at any element), kHeld vectors a thread at most.  NT: its threads, and the channels it has at most.
constexpr int kHeld = 8;  // (or 2, where they suffice: a quarter of the instructions to fetch)

template <class T, int NT>
struct HeldPlace {
  static constexpr int VE = VecOf<T>::N;
  int sample, first, groups, width, lanes, rows, col, ty, c0, left;  // first: group; c0: channel; left: channels of the workgroup from it on
  int64_t n, row0;
  __device__ __forceinline__ HeldPlace(const Shape &d, const int32_t *counts, int take, int lanes_) : lanes(lanes_) {
    const int tiles = (d.groups + take - 1) / take;
    sample = blockIdx.x / tiles, first = blockIdx.x % tiles * take;
    groups = min(take, d.groups - first), width = groups * d.per;
    rows = NT / lanes;
    col = threadIdx.x % lanes, ty = threadIdx.x / lanes;
    c0 = first * d.per + col * VE, left = ty < rows ? width - col * VE : 0;
    n = pixels_of(counts, d.pixels, sample);
    row0 = (int64_t)sample * d.pixels;
  }
  __device__ __forceinline__ bool there(int i) const { return left > 0 && ty + (int64_t)i * rows < n; }
  __device__ __forceinline__ int64_t row(int i) const { return row0 + ty + (int64_t)i * rows; }
  __device__ __forceinline__ int64_t some_row(int i) const { return row0 + min(ty + (int64_t)i * rows, n - 1); }  // (one that is there)
  __device__ __forceinline__ Columns<T> columns(const Shape &d) const { return Columns<T>(c0, left, d.C, width % (lanes * VE) != 0 || NT % lanes != 0); }
};

// The threads' pairs of sums by channel joined: the sum of each channel goes to f, the groups' to `all`; w(c): what a channel counts in
// its group.  Columns first, in as many parts as there are threads, then the groups.
template <class T, int NT, class F, class W>
__device__ __forceinline__ void join_held(const HeldPlace<T, NT> &at, int per, const double (&a)[VecOf<T>::N], const double (&b)[VecOf<T>::N],
                                          Room<NT, VecOf<T>::N> &room, double2 *col_room, double2 *all, F f, W w) {
  const int tid = threadIdx.x;
  room.put(a, b);
  __syncthreads();
  const int parts = max(min(NT / at.width, at.rows / 8), 1);  // (of eight rows and more: one thread adds up the parts of a channel)
  for (int i = tid; i < parts * at.width; i += NT) {
    const int c = i % at.width;
    double2 v = {0.0, 0.0};
#pragma unroll 8
    for (int r = i / at.width; r < at.rows; r += parts) {
      const double2 q = room.at(r * at.lanes, c);
      v.x += q.x, v.y += q.y;
    }
    col_room[i] = v;
  }
  __syncthreads();
  for (int c = tid; c < at.width; c += NT) {
    double2 v = col_room[c];
#pragma unroll 4
    for (int p = 1; p < parts; ++p) v.x += col_room[p * at.width + c].x, v.y += col_room[p * at.width + c].y;
    f(c, v);
  }
  by_group<NT>(at.groups, parts * per, all, [&](int g, int i) {
    const int c = g * per + i % per;
    const double2 q = col_room[i / per * at.width + c];
    const double weight = w(c);
    return double2{q.x * weight, q.y * weight};
  });
  __syncthreads();
}

template <class T, int NT, int HELD, int ACT, bool KEEP>
__global__ __launch_bounds__(NT) void norm_held_kernel(const T *x, const float *__restrict__ gamma, const float *__restrict__ beta,
                                                             const int32_t *__restrict__ counts, Shape d, int take, int lanes, T *y,
                                                             float *__restrict__ stats, int8_t *__restrict__ codes,
                                                             uint8_t *__restrict__ steps) {
  constexpr int VE = VecOf<T>::N;
  __shared__ Room<NT, VE> room;
  __shared__ double2 col_room[NT], all[NT];
  const HeldPlace<T, NT> at(d, counts, take, lanes);
  u32x4 v[HELD];
  const Columns<T> cols = at.columns(d);
  const T *top = x + at.row0 * d.ldx + at.first * d.per;
  float first[VE] = {};
  if (at.n > 0) {
    cols.load(v, [&](int i) { return x + at.some_row(i) * d.ldx; });
    by_groups<VE>(at.col * VE, d.per, at.groups - 1, [&](int g) { return widen(top[g * d.per]); }, [&](int j, float q) { first[j] = q; });
  }
  const float own_first = at.n > 0 ? widen(top[min((int)threadIdx.x, at.groups - 1) * d.per]) : 0.f;
#pragma unroll
  for (int i = 0; i < HELD; ++i) v[i] = at.there(i) ? cols.fix(v[i]) : u32x4{};
  float g[VE], b[VE], mean[VE];
  affine<VE>(gamma, beta, at.c0, d.C, g, b);
  const double per = 1.0 / (double)max(at.n * d.per, (int64_t)1);
  double sum[VE] = {}, sq[VE] = {};
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (!at.there(i)) break;
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const double f = (double)elem<T>(v[i], j) - (double)first[j];
      sum[j] += f, sq[j] = fma(f, f, sq[j]);
    }
  }
  join_held<T, NT>(at, d.per, sum, sq, room, col_room, all, [](int, double2) {}, [](int) { return 1.0; });
  float4 *stat_room = reinterpret_cast<float4 *>(col_room);  // (read by nobody any more)
  if (const int g = threadIdx.x; g < at.groups) {            // (a group for each thread at most)
    const float4 q = stat_of(all[g], per, own_first, d.eps);
    stat_room[g] = q;
    if (stats) {
      float *p = stats + 2 * ((int64_t)at.sample * d.groups + at.first + g);
      p[0] = q.x, p[1] = q.y;
    }
  }
  __syncthreads();
  const int blocks = (d.C + kKept - 1) / kKept;
  const bool mine = KEEP ? at.ty < at.rows && at.c0 < blocks * kKept : at.left > 0;
  if (!mine) return;
  by_groups<VE>(
      at.col * VE, d.per, at.groups - 1, [&](int group) { return stat_room[group]; },
      [&](int j, const float4 &q) { mean[j] = q.x, g[j] *= q.y, b[j] = fmaf(-q.z, g[j], b[j]); });
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (at.ty + (int64_t)i * at.rows >= at.n) break;
    const int64_t row = at.row(i);
    if constexpr (KEEP) {  // (the lanes of a block have the same pixels)
      const uint32_t step = step_of(top_of_block<T>(v[i]));
      store_codes<T>(codes + row * blocks * kKept + at.c0, v[i], per_step(step));
      if (at.c0 % kKept == 0) steps[row * blocks + at.c0 / kKept] = (uint8_t)step;
    }
    float f[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      float slope;
      act_of<T, ACT>(fmaf(elem<T>(v[i], j) - mean[j], g[j], b[j]), f[j], slope);
    }
    store_part<T>(y + row * d.ldy + at.c0, at.left, pack<T>(f));
  }
}

template <class T, int NT, int HELD, int ACT, bool KEPT>
__global__ __launch_bounds__(NT) void norm_grad_held_kernel(Input<T, KEPT> in, const T *dy, const float *__restrict__ gamma,
                                                                  const float *__restrict__ beta, const float *__restrict__ stats,
                                                                  const int32_t *__restrict__ counts, Shape d, double2 *__restrict__ chan,
                                                                  int take, int lanes, T *dx, float *__restrict__ dgamma,
                                                                  float *__restrict__ dbeta) {
  constexpr int VE = VecOf<T>::N;
  __shared__ Room<NT, VE> room;
  __shared__ double2 col_room[NT], all[NT];
  const HeldPlace<T, NT> at(d, counts, take, lanes);
  typename Input<T, KEPT>::Raw v[HELD];
  u32x4 w[HELD];
  const Columns<T> cols = at.columns(d);
  if (at.n > 0) {
    auto row = [&](int i) { return at.some_row(i); };
    in.load(v, cols, at.c0, row);
    cols.load(w, [&](int i) { return dy + row(i) * d.ldy; });
#pragma unroll
    for (int i = 0; i < HELD; ++i) v[i] = in.fix(v[i], cols), w[i] = cols.fix(w[i]);
  }
  float g[VE], b[VE], mean[VE], rstd[VE];
  affine<VE>(gamma, beta, at.c0, d.C, g, b);
  const float *own = stats + 2 * ((int64_t)at.sample * d.groups + at.first);
  by_groups<VE>(
      at.col * VE, d.per, at.groups - 1, [&](int group) { return float2{own[2 * group], own[2 * group + 1]}; },
      [&](int j, const float2 &q) { mean[j] = q.x, rstd[j] = q.y, g[j] *= q.y; });
  const double per = 1.0 / (double)max(at.n * d.per, (int64_t)1);
  double sum[VE] = {}, dot[VE] = {};
#pragma unroll
  for (int i0 = 0; i0 < HELD; i0 += 4) {
    float s4[VE] = {}, d4[VE] = {};  // (four at a time in fp32)
#pragma unroll
    for (int i = i0; i < min(i0 + 4, HELD); ++i) {
      if (!at.there(i)) break;
      const float step = in.step(v[i]);
#pragma unroll
      for (int j = 0; j < VE; ++j) {
        const float x = in.at(v[i], j, step, mean[j]);
        float value, slope;
        act_of<T, ACT>(fmaf(x, g[j], b[j]), value, slope);
        const float dz = elem<T>(w[i], j) * slope;
        s4[j] += dz, d4[j] = fmaf(dz, x, d4[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < VE; ++j) sum[j] += s4[j], dot[j] += d4[j];
  }
#pragma unroll
  for (int j = 0; j < VE; ++j) dot[j] *= rstd[j];
  const int first = at.first * d.per;
  join_held<T, NT>(
      at, d.per, sum, dot, room, col_room, all,
      [&](int c, double2 s) {
        if (d.samples > 1) {
          chan[(int64_t)at.sample * d.C + first + c] = s;
        } else {
          if (dbeta) dbeta[first + c] = (float)s.x;
          if (dgamma) dgamma[first + c] = (float)s.y;
        }
      },
      [&](int c) { return gamma ? (double)gamma[first + c] : 1.0; });
  if (!dx || at.left <= 0) return;
  float m1[VE], m2[VE];
  by_groups<VE>(
      at.col * VE, d.per, at.groups - 1, [&](int group) { return float2{(float)(all[group].x * per), (float)(all[group].y * per)}; },
      [&](int j, const float2 &q) { m1[j] = rstd[j] * q.x, m2[j] = rstd[j] * rstd[j] * q.y; });
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (!at.there(i)) break;
    const float step = in.step(v[i]);
    float f[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float x = in.at(v[i], j, step, mean[j]);
      float value, slope;
      act_of<T, ACT>(fmaf(x, g[j], b[j]), value, slope);
      f[j] = fmaf(elem<T>(w[i], j) * slope, g[j], -fmaf(x, m2[j], m1[j]));
    }
    store_part<T>(dx + at.row(i) * d.ldx + at.c0, at.left, pack<T>(f));
  }
}

// ---- host ---------------------------------------------------------------------------------------------------
// A launch has fewer than 2^32 threads.
bool launches(int64_t workgroups, int threads) { return workgroups * threads < (int64_t)1 << 32; }

// Groups of a workgroup whose registers hold their sample, and its threads.
struct Held {
  int take, threads, held;  // take 0: no workgroup's registers do; held: vectors of a thread, at most
};
struct Plan {
  Held held, held_kept;  // with codes
  int lanes, cols;  // threads side by side, workgroups side by side
  int chunks;
  int64_t chunk;
  bool few;  // the second pass joins the chunks by itself
  size_t part, group, chan, bytes;
};

int held_lanes(const wcc_group_norm_desc &d, int take, int VE, bool kept);

// Groups of a workgroup whose registers hold their sample (take), and its threads, 256 where they suffice: three workgroups a compute unit.
// As many groups as read 128 bytes of a pixel, a line of memory, where that leaves 512 workgroups, else 64 or 16 bytes: a small map is bound
// by what a compute unit computes (one map of 256 pixels and 96 channels in one workgroup 9.8 us).  With codes, whole blocks of channels.
Held held_of(const wcc_group_norm_desc &d, int VE, bool kept) {
  const int per = d.C / d.groups, size = 16 / VE;
  Held best = {0, 0, 0};
  if (d.pixels > kHeld * 512) return best;
  int whole = 1;  // groups whose channels are whole blocks
  if (kept)
    while ((int64_t)whole * per % kKept != 0) whole *= 2;
  for (const int least : {16, 64, 128}) {
    int take = std::max((least + per * size - 1) / (per * size), 1);
    take = std::min((take + whole - 1) / whole * whole, d.groups);
    const int64_t width = (int64_t)take * per;
    if (width > 512) break;
    const int lanes = held_lanes(d, take, VE, kept);
    for (const int threads : {256, 512}) {
      if (width > threads || lanes > threads || !launches((int64_t)d.samples * ((d.groups + take - 1) / take), threads)) continue;
      const int64_t most = (d.pixels + threads / lanes - 1) / (threads / lanes);
      if (most > kHeld) continue;
      best = Held{take, threads, most <= 2 ? 2 : kHeld};
      break;
    }
    if (best.take && (int64_t)d.samples * ((d.groups + best.take - 1) / best.take) <= 512) break;
  }
  return best;
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

Plan plan_of(const wcc_group_norm_desc &d) {
  const int VE = d.dtype == WCC_F32 ? 4 : 8;
  const int64_t vectors = kept_blocks(d.C) * (kKept / VE);  // (whole blocks: what keeps x needs all lanes of each)
  Plan p;
  p.held = held_of(d, VE, false), p.held_kept = held_of(d, VE, true);
  p.lanes = (int)std::min<int64_t>(vectors, 64);  // (1 KiB a pixel; with all of a wide map's a workgroup had one pixel at a time, and many chunks)
  p.cols = (int)((vectors + p.lanes - 1) / p.lanes);
  const int rows = 256 / p.lanes;
  // Chunks: as many as give every compute unit four workgroups (512 to 4096 of them take 40 to 42 us for 8 x 16384 x 256), two where the
  // join would have more than 32768 pairs of sums to read for a group (512 KB: 500 chunks of 120 channels take it 15 us), of eight pixels a
  // thread at least; four where there are few, as long as the second pass can join them by itself: up to 2048 pairs of sums, two workgroups a
  // compute unit.
  const int64_t fours = std::max<int64_t>((d.pixels + 4 * rows - 1) / (4 * rows), 1), eights = (fours + 1) / 2;
  const int64_t each = std::max<int64_t>((int64_t)d.samples * p.cols, 1);
  const int64_t want = std::max<int64_t>({std::min<int64_t>(1024 / each, 32768 / (d.C / d.groups)), 512 / each, 1});
  const int64_t joined = d.C <= kShort ? std::min<int64_t>(2048 / d.C, 512 / each) : 0;
  int64_t n = std::min(eights, want);
  if (n < joined) n = std::min({fours, want, joined});
  p.chunk = std::max<int64_t>((d.pixels + n - 1) / n, 1);
  p.chunks = (int)std::max<int64_t>((d.pixels + p.chunk - 1) / p.chunk, 1);
  p.few = p.chunks <= joined;
  p.part = 0;
  p.group = p.held.take && p.held_kept.take ? 0 : up((size_t)d.samples * p.chunks * d.C * sizeof(double2));
  p.chan = p.group + up((size_t)d.samples * d.groups * sizeof(float4));
  p.bytes = p.chan + up((size_t)d.samples * d.C * sizeof(double2));
  return p;
}

int held_lanes(const wcc_group_norm_desc &d, int take, int VE, bool kept) {
  const int64_t width = (int64_t)take * (d.C / d.groups);
  return (int)(kept ? kept_blocks(width) * (kKept / VE) : (width + VE - 1) / VE);
}

Sums sums_of(const Plan &p, char *ws) {
  return Sums{reinterpret_cast<double2 *>(ws + p.part), reinterpret_cast<float4 *>(ws + p.group), reinterpret_cast<double2 *>(ws + p.chan),
              p.chunks, p.chunk};
}
Shape shape_of(const wcc_group_norm_desc &d) {
  return Shape{d.pixels, d.ldx, d.ldy, d.samples, d.C, d.groups, d.C / d.groups, d.eps};
}
int join_lanes(const wcc_group_norm_desc &d) {
  int n = 1;
  while (n < 64 && n < d.C / d.groups) n *= 2;
  return n;
}

template <class F>
void by_act(int act, F f) {
  switch (act) {
    case WCC_ACT_RELU: return f(std::integral_constant<int, WCC_ACT_RELU>());
    case WCC_ACT_SILU: return f(std::integral_constant<int, WCC_ACT_SILU>());
    case WCC_ACT_GELU: return f(std::integral_constant<int, WCC_ACT_GELU>());
    default: return f(std::integral_constant<int, WCC_ACT_NONE>());
  }
}

template <class F>
void by_held(const Held &h, F f) {
  const std::integral_constant<int, 256> few;
  const std::integral_constant<int, 512> many;
  const std::integral_constant<int, 2> two;
  const std::integral_constant<int, kHeld> all;
  if (h.threads == 256) h.held == 2 ? f(few, two) : f(few, all);
  else h.held == 2 ? f(many, two) : f(many, all);
}

// The chunks joined: by 1024 threads a group where it has many pairs of sums, which a few workgroups would take long to read (and as many
// workgroups as a launch of these does not have are not few).
template <bool BACK>
void join(const wcc_group_norm_desc &d, const Plan &p, const NormArgs &g, const Shape &sh, const Sums &s, hipStream_t st) {
  const unsigned n = (unsigned)(d.groups * d.samples);
  const float *gamma = BACK ? g.gamma : nullptr;
  if ((int64_t)p.chunks * (d.C / d.groups) > 2048 && launches(n, 1024)) norm_join_kernel<BACK, 1024><<<n, 1024, 0, st>>>(g.counts, sh, s, gamma, g.stats, join_lanes(d));
  else norm_join_kernel<BACK, 256><<<n, 256, 0, st>>>(g.counts, sh, s, gamma, g.stats, join_lanes(d));
}

template <class T>
hipError_t forward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t st) {
  const Plan p = plan_of(d);
  const Sums s = sums_of(p, g.ws);
  const Shape sh = shape_of(d);
  const T *x = static_cast<const T *>(g.x);
  T *y = static_cast<T *>(g.y);
  const Held held = g.codes ? p.held_kept : p.held;
  if (const int take = held.take) {
    const unsigned n = (unsigned)(d.samples * ((d.groups + take - 1) / take));
    const int lanes = held_lanes(d, take, VecOf<T>::N, g.codes != nullptr);
    by_act(d.act, [&](auto act) {
      by_held(held, [&](auto threads, auto held) {
        auto go = [&](auto keep) {
          norm_held_kernel<T, threads(), held(), act(), keep()>
              <<<n, threads(), 0, st>>>(x, g.gamma, g.beta, g.counts, sh, take, lanes, y, g.stats, g.codes, g.steps);
        };
        g.codes ? go(std::true_type()) : go(std::false_type());
      });
    });
    return hipGetLastError();
  }
  const dim3 grid((unsigned)(p.chunks * d.samples), p.cols);
  norm_sums_kernel<T><<<grid, 256, 0, st>>>(x, g.counts, sh, s, p.lanes);
  if (!p.few) join<false>(d, p, g, sh, s, st);
  by_act(d.act, [&](auto act) {
    auto go = [&](auto keep, auto few) {
      norm_apply_kernel<T, act(), keep(), few()>
          <<<grid, 256, 0, st>>>(x, g.gamma, g.beta, g.counts, sh, s, p.lanes, y, g.stats, g.codes, g.steps);
    };
    const std::true_type yes;
    const std::false_type no;
    if (p.few) g.codes ? go(yes, yes) : go(no, yes);
    else g.codes ? go(yes, no) : go(no, no);
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
  const bool wide = g.dgamma || g.dbeta, fused = wide && (p.few || d.samples <= kFewSamples);  // (beside dx's tiles)
  const Held held = KEPT ? p.held_kept : p.held;
  const int take = held.take;
  if (take && d.samples > 0) {
    const unsigned n = (unsigned)(d.samples * ((d.groups + take - 1) / take));
    const int lanes = held_lanes(d, take, VecOf<T>::N, KEPT);
    by_act(d.act, [&](auto act) {
      by_held(held, [&](auto threads, auto held) {
        norm_grad_held_kernel<T, threads(), held(), act(), KEPT><<<n, threads(), 0, st>>>(
            in, dy, g.gamma, g.beta, g.stats, g.counts, sh, s.chan, take, lanes, static_cast<T *>(g.dx), g.dgamma, g.dbeta);
      });
    });
    if (d.samples == 1) return hipGetLastError();
  } else if (d.samples > 0) {
    const int n = p.chunks * d.samples, more = fused ? (d.C + 255) / 256 : 0;
    by_act(d.act, [&](auto act) {
      norm_grad_sums_kernel<T, act(), KEPT><<<grid, 256, 0, st>>>(in, dy, g.gamma, g.beta, g.stats, g.counts, sh, s, p.lanes);
      if (!p.few) join<true>(d, p, g, sh, s, st);
      if (!g.dx) return;
      const dim3 both((unsigned)(n + more), p.cols);
      T *dx = static_cast<T *>(g.dx);
      if (p.few)
        norm_grad_apply_kernel<T, act(), KEPT, true>
            <<<both, 256, 0, st>>>(in, dy, g.gamma, g.beta, g.counts, sh, s, p.lanes, n, dx, g.stats, g.dgamma, g.dbeta);
      else
        norm_grad_apply_kernel<T, act(), KEPT, false>
            <<<both, 256, 0, st>>>(in, dy, g.gamma, g.beta, g.counts, sh, s, p.lanes, n, dx, g.stats, g.dgamma, g.dbeta);
    });
    if (g.dx && (fused || !wide)) return hipGetLastError();
  }
  if (wide) {
    const unsigned n = (unsigned)((d.C + 255) / 256);
    if (p.few && !take) {
      norm_affine_grad_kernel<<<n, 256, 0, st>>>(s.part, d.C, d.samples * p.chunks, d.C, g.dgamma, g.dbeta);
    } else if (d.samples <= kFewSamples) {
      norm_affine_grad_kernel<<<n, 256, 0, st>>>(s.chan, d.C, d.samples, d.C, g.dgamma, g.dbeta);
    } else {
      const int each = std::max((d.samples + 255) / 256, 16), left = (d.samples + each - 1) / each;
      norm_samples_kernel<<<dim3(n, left), 256, 0, st>>>(s.chan, d.C, d.samples, each);
      norm_affine_grad_kernel<<<n, 256, 0, st>>>(s.chan, d.C, left, (int64_t)each * d.C, g.dgamma, g.dbeta);
    }
  }
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

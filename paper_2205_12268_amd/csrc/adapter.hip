// One projection with a low-rank adapter for each row (wcc_adapter_forward, wcc_adapter_backward).
//
// Both directions are a product with W beside two thin ones that go through the rank lines of the row's adapter:
//   forward   h[t,j] = s_a sum_c A_a[j,c] x[t,c],    y[t,o]  = sum_c W[o,c] x[t,c]   + sum_j B_a[o,j] h[t,j]
//   backward  g[t,j] = s_a sum_o B_a[o,j] dy[t,o],   dx[t,c] = sum_o W[o,c] dy[t,o]  + sum_j A_a[j,c] g[t,j]
//   gradients dA_a[j,c] = sum_t g[t,j] x[t,c],       dB_a[o,j] = sum_t h[t,j] dy[t,o]
//
// Few rows: what has to be read is W and the adapters, once, and what counts is how many loads are in flight.  The first
// launch has the product with W, cut along k over waves and workgroups, each wave's operands straight from memory into
// registers, and in further workgroups the rank lines (they are but more lines that x meets).  The second adds the partial
// sums, the thin product with h and rounds.  Many rows: the rank lines, then tiles through LDS with the thin product in
// their last step (adapter_tile.hip).
#include "adapter.h"

namespace wcc {
namespace {

// ---- the rank lines of rows -----------------------------------------------------------------------------------
// A wave takes 32 rows, a range of k and, of the distinct adapters among the rows, every groups-th.
template <class T>
struct ThinJob {
  const T *x;
  int64_t ldx, rows;
  int width;
  Thin<T> m;
  float *out;  // [splits][rows][rank]
  int splits, chunk, groups;
  int64_t units;
};

template <class T>
__device__ __forceinline__ void thin_unit(const ThinJob<T> &g, const Low &low, int64_t unit) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, U = 4;
  const int lane = threadIdx.x & 63, ln = lane & 31, half = lane >> 5;
  const int group = (int)(unit % g.groups), split = (int)(unit / g.groups % g.splits);
  const int64_t t0 = unit / g.groups / g.splits * 32, t = t0 + ln;
  const int id = t < g.rows ? low.of(t) : -1;
  const int k0 = split * g.chunk, k1 = min(g.width, k0 + g.chunk);
  const T *xr = g.x + min(t, g.rows - 1) * g.ldx + half * VE;
  float *out = g.out + ((int64_t)split * g.rows + t0) * low.rank;
  uint32_t rest = (uint32_t)__ballot(id >= 0);  // (the halves of the wave hold the same rows)
  for (int nth = 0; rest != 0; ++nth) {
    const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(rest));
    const uint32_t same = (uint32_t)__ballot(id == a);
    rest &= ~same;
    if (nth % g.groups != group) continue;
    const int lines = low.lines(a);
    const float f = low.factor(a);
    for (int j0 = 0; j0 < lines; j0 += 32) {
      const T *mr = g.m.p + a * g.m.major + (int64_t)min(j0 + ln, lines - 1) * g.m.sj + (int64_t)(half * VE) * g.m.sc;
      f32x16 acc = {};
      int k = k0;
      for (; k + KS * U <= k1; k += KS * U) {
        u32x4 xf[U], mf[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          xf[u] = *reinterpret_cast<const u32x4_any *>(xr + k + u * KS);
          mf[u] = g.m.sc == 1 ? *reinterpret_cast<const u32x4_any *>(mr + k + u * KS)
                              : load_k_strided(mr + (int64_t)(k + u * KS) * g.m.sc, g.m.sc, VE);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) acc = mma<T>(xf[u], mf[u], acc);
      }
      for (; k < k1; k += KS) {
        const int left = k1 - k - half * VE;
        const u32x4 xf = load_k(xr + k, left);
        const u32x4 mf = g.m.sc == 1 ? load_k(mr + k, left) : load_k_strided(mr + (int64_t)k * g.m.sc, g.m.sc, left);
        acc = mma<T>(xf, mf, acc);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = result_line(i, half);
        if ((same >> row & 1) && j0 + ln < lines) out[(int64_t)row * low.rank + j0 + ln] = acc[i] * f;
      }
    }
  }
}

// ---- the product with W for few rows ----------------------------------------------------------------------------
// 32 RT rows x 64 outputs x a range of k a workgroup; each of its four waves has a quarter of the range and all results.
// NN: W's outputs are contiguous, not its k.
template <class T>
struct StreamJob {
  const T *x;
  int64_t ldx, rows;
  int width, outs;
  const T *w;
  int64_t ldw;  // between outputs, or (NN) between k
  float *part;  // [splits][rows][outs]
  int splits, chunk, tiles_o;
  int64_t blocks;
};

template <class T, int RT, bool NN>
__device__ __forceinline__ void stream_block(const StreamJob<T> &g, int64_t block, float *red) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, U = 4, LD = 72;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  const int split = (int)(block % g.splits), o0 = (int)(block / g.splits % g.tiles_o) * 64;
  const int64_t t0 = block / g.splits / g.tiles_o * (32 * RT);
  const int quarter = g.chunk / 4, k0 = split * g.chunk + wv * quarter, k1 = min(g.width, k0 + quarter);
  const T *xr[RT], *wr[2];
#pragma unroll
  for (int r = 0; r < RT; ++r) xr[r] = g.x + min(t0 + r * 32 + ln, g.rows - 1) * g.ldx + half * VE;
  if (!NN) {
#pragma unroll
    for (int e = 0; e < 2; ++e) wr[e] = g.w + (int64_t)min(o0 + e * 32 + ln, g.outs - 1) * g.ldw + half * VE;
  } else {
    wr[0] = g.w + min(o0 + 2 * ln, g.outs - 1) + (int64_t)(half * VE) * g.ldw;
  }
  const bool both = o0 + 2 * ln + 1 < g.outs;
  f32x16 acc[RT][2] = {};
  int k = k0;
  for (; k + KS * U <= k1; k += KS * U) {
    u32x4 xf[U][RT], wf[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!NN) {
#pragma unroll
        for (int e = 0; e < 2; ++e) wf[u][e] = *reinterpret_cast<const u32x4_any *>(wr[e] + k + u * KS);
      } else {
        load_k_pair(wr[0] + (int64_t)(k + u * KS) * g.ldw, g.ldw, VE, both, wf[u][0], wf[u][1]);
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) xf[u][r] = *reinterpret_cast<const u32x4_any *>(xr[r] + k + u * KS);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) acc[r][e] = mma<T>(xf[u][r], wf[u][e], acc[r][e]);
  }
  for (; k < k1; k += KS) {
    const int left = k1 - k - half * VE;
    u32x4 wf[2];
    if (!NN) {
#pragma unroll
      for (int e = 0; e < 2; ++e) wf[e] = load_k(wr[e] + k, left);
    } else {
      load_k_pair(wr[0] + (int64_t)k * g.ldw, g.ldw, left, both, wf[0], wf[1]);
    }
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const u32x4 xf = load_k(xr[r] + k, left);
#pragma unroll
      for (int e = 0; e < 2; ++e) acc[r][e] = mma<T>(xf, wf[e], acc[r][e]);
    }
  }
  float *mine = red + wv * 32 * RT * LD;
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) mine[(r * 32 + result_line(i, half)) * LD + (NN ? 2 * ln + e : e * 32 + ln)] = acc[r][e][i];
  __syncthreads();
  const int o = o0 + lane;
  float *out = g.part + ((int64_t)split * g.rows + t0) * g.outs + o;
  if (o < g.outs)
    for (int r = wv; r < 32 * RT && t0 + r < g.rows; r += 4) {
      const float *p = red + r * LD + lane;
      constexpr int next = 32 * RT * LD;
      out[(int64_t)r * g.outs] = (p[0] + p[next]) + (p[2 * next] + p[3 * next]);
    }
}

// First launch: blocks of the product with W, then waves of one or two jobs of rank lines.
template <class T, int RT, bool NN>
__global__ __launch_bounds__(256) void adapter_products_kernel(StreamJob<T> g, ThinJob<T> thin, ThinJob<T> thin2, Low low) {
  __shared__ float red[4 * 32 * RT * 72];
  const int64_t block = blockIdx.x;
  if (block < g.blocks) return stream_block<T, RT, NN>(g, block, red);
  const int64_t unit = (block - g.blocks) * 4 + (threadIdx.x >> 6);
  if (unit < thin.units) return thin_unit<T>(thin, low, unit);
  if (unit - thin.units < thin2.units) thin_unit<T>(thin2, low, unit - thin.units);
}

// Second launch: y[t, o] = the sum of the parts + sum_j m(a, j, o) h[t, j].  256 outputs x RB rows a workgroup.
template <class T>
__global__ __launch_bounds__(256) void adapter_finish_kernel(const float *__restrict__ part, int splits, int64_t rows, int outs,
                                                             Low low, Thin<T> m, Lines h, T *__restrict__ y, int64_t ldy, int rb,
                                                             int tiles_o, int64_t blocks) {
  constexpr int VE = VecOf<T>::N;
  __shared__ float hs[WCC_MAX_RANK];
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int o = (int)(b % tiles_o) * 256 + (int)threadIdx.x;
    const int64_t t0 = b / tiles_o * rb;
    for (int64_t t = t0; t < min(t0 + rb, rows); ++t) {
      const int a = low.of(t), lines = a >= 0 ? low.lines(a) : 0;
      __syncthreads();
      if ((int)threadIdx.x < lines) hs[threadIdx.x] = h.at(t * low.rank + threadIdx.x);
      float v = 0.f;
      if (o < outs)
        for (int s = 0; s < splits; ++s) v += part[(s * rows + t) * outs + o];
      __syncthreads();
      if (o >= outs) continue;
      if (lines > 0) {
        const T *mr = m.p + a * m.major + (int64_t)o * m.sc;
        float low_v = 0.f;
        if (m.sj == 1) {
          for (int j = 0; j < lines; j += VE) {
            const u32x4 f = load_k(mr + j, lines - j);
#pragma unroll
            for (int i = 0; i < VE; ++i)
              if (j + i < lines) low_v = fmaf(elem<T>(f, i), hs[j + i], low_v);
          }
        } else {
          for (int j = 0; j < lines; ++j) low_v = fmaf(widen(mr[(int64_t)j * m.sj]), hs[j], low_v);
        }
        v += low_v;
      }
      y[t * ldy + o] = narrow<T>(v);
    }
  }
}

// ---- gradients of the adapters ------------------------------------------------------------------------------------
// grad(a, j, c) = sum over the rows t of adapter a of h[t, j] x[t, c], at a * major + j * sj + c * sc.
template <class T>
struct GradJob {
  const T *x;
  int64_t ldx;
  int width;
  Lines h;
  float *out;    // the gradient, or [splits] of them
  int64_t size;  // of one: n * rank * width
  int64_t major;
  int sj, sc;
  int32_t *found;  // [splits][n]: rows of the adapter in the range, with more than one split
  int tiles_c;
  int64_t blocks;
};

// A workgroup has an adapter, 256 columns, 32 lines and a range of rows; it lists the rows that are the adapter's, so that rows
// of many adapters in any order are read once in all.
template <class T>
__device__ __forceinline__ void grad_block(const GradJob<T> &g, const Low &low, int64_t rows, int splits, int64_t range, int64_t block,
                                           int *list, int *counts) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, P = PartsOf<T>::Grad;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5;
  const int tiles_j = (low.rank + 31) / 32;
  const int split = (int)(block % splits), j0 = (int)(block / splits % tiles_j) * 32;
  const int tile_c = (int)(block / splits / tiles_j % g.tiles_c), a = (int)(block / splits / tiles_j / g.tiles_c);
  const int lines = low.lines(a), c = tile_c * 256 + wv * 64 + 2 * ln, j = j0 + ln;
  const bool here = c < g.width, both = c + 1 < g.width;
  const T *xc = g.x + min(c, g.width - 1);
  const int64_t t_end = min(rows, (split + 1) * range);
  f32x16 acc[2] = {};
  int have = 0, total = 0;
  auto step = [&](int at, int n) {  // n (at most KS) listed rows from `at` on
    float hv[VE];
    u32x4 xf[2], hf[P];
    uint32_t v32[VE];
    uint64_t v64[VE];
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const int q = half * VE + i;
      hv[i] = 0.f;
      v32[i] = 0, v64[i] = 0;
      if (q < n) {
        const int64_t t = list[at + q];
        if (j < lines) hv[i] = g.h.at(t * low.rank + j);
        const T *p = xc + t * g.ldx;
        if constexpr (sizeof(T) == 4) v64[i] = both ? *reinterpret_cast<const u64_any *>(p) : here ? (uint64_t)__float_as_uint(*p) : 0;
        else v32[i] = both ? *reinterpret_cast<const u32_any *>(p) : here ? (uint32_t)*p : 0;
      }
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) xf[0][i] = (uint32_t)v64[i], xf[1][i] = (uint32_t)(v64[i] >> 32);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        xf[0][i] = __builtin_amdgcn_perm(v32[2 * i + 1], v32[2 * i], 0x05040100);
        xf[1][i] = __builtin_amdgcn_perm(v32[2 * i + 1], v32[2 * i], 0x07060302);
      }
    }
    split_to<T, P>(hv, hf);
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int p = P - 1; p >= 0; --p) acc[e] = mma<T>(hf[p], xf[e], acc[e]);
  };
  if (j0 < lines) {
    for (int64_t t0 = split * range; t0 < t_end; t0 += 256) {
      const int64_t t = t0 + tid;
      const bool mine = t < t_end && low.of(t) == a;
      const uint64_t vote = __ballot(mine);
      if (lane == 0) counts[wv] = __popcll(vote);
      __syncthreads();
      int before = have, all = have;
      for (int i = 0; i < 4; ++i) {
        const int n = counts[i];
        if (i < wv) before += n;
        all += n;
      }
      if (mine) list[before + __popcll(vote & ((1ull << lane) - 1))] = (int)t;
      __syncthreads();
      total += all - have;
      const int full = all / KS * KS;
      for (int at = 0; at < full; at += KS) step(at, KS);
      have = all - full;
      __syncthreads();
      if (tid < have) counts[4 + tid] = list[full + tid];
      __syncthreads();
      if (tid < have) list[tid] = counts[4 + tid];
      // (the next round's first barrier comes before the list is read)
    }
    __syncthreads();
    if (have > 0) step(0, have);
  }
  if (splits > 1) {
    if (g.found && tile_c == 0 && j0 == 0 && tid == 0) g.found[(int64_t)split * low.n + a] = total;
    if (total == 0) return;
  }
  float *out = g.out + (splits > 1 ? split * g.size : 0) + a * g.major;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int line = j0 + result_line(i, half);
    if (line >= low.rank) continue;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (c + e < g.width) out[(int64_t)line * g.sj + (int64_t)(c + e) * g.sc] = line < lines ? acc[e][i] : 0.f;
  }
}

template <class T>
__global__ __launch_bounds__(256) void adapter_grad_kernel(GradJob<T> ga, GradJob<T> gb, Low low, int64_t rows, int splits, int64_t range) {
  __shared__ int list[256 + 16], counts[4 + 16];
  for (int64_t b = blockIdx.x; b < ga.blocks + gb.blocks; b += gridDim.x) {
    if (b < ga.blocks) grad_block<T>(ga, low, rows, splits, range, b, list, counts);
    else grad_block<T>(gb, low, rows, splits, range, b - ga.blocks, list, counts);
    __syncthreads();
  }
}

// The ranges' sums as one, in their order; lines past an adapter's rank are 0.
struct JoinJob {
  const float *part;
  float *out;
  int64_t size, major;
  int sj, sc;
};
__global__ __launch_bounds__(256) void adapter_grad_join_kernel(JoinJob ja, JoinJob jb, Low low, int splits,
                                                                const int32_t *__restrict__ found) {
  const int64_t total = ja.size + jb.size, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const bool first = i < ja.size;
    const JoinJob &g = first ? ja : jb;
    const int64_t at = first ? i : i - ja.size;
    const int a = (int)(at / g.major);
    const int in = (int)(at - a * g.major), j = g.sj == 1 ? in % low.rank : in / g.sj;
    float v = 0.f;
    if (j < low.lines(a))
      for (int s = 0; s < splits; ++s)
        if (found[(int64_t)s * low.n + a] > 0) v += g.part[s * g.size + at];
    g.out[at] = v;
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// k of a range is a multiple of 64 bf16 / 32 fp32 elements (four waves' steps)
int step4(const wcc_adapter_desc &d) { return d.dtype == WCC_BF16 ? 64 : 32; }

// Ranges of k for the rank lines: about a thousand waves.
int thin_splits(const wcc_adapter_desc &d, int width) {
  const int64_t tiles = ceil_div(d.rows, 32);
  return (int)std::clamp<int64_t>(ceil_div(1024, std::max<int64_t>(tiles, 1)), 1, std::clamp<int64_t>(width / 256, 1, 16));
}
size_t lines_bytes(const wcc_adapter_desc &d, int width) {
  return align256((size_t)thin_splits(d, width) * d.rows * d.rank * 4);
}

// The product with W for few rows: whether, and ranges of k.
struct StreamPlan {
  bool taken;
  int rt, splits, chunk, tiles_o;
  int64_t blocks;
};
StreamPlan stream_plan(const wcc_adapter_desc &d, int width, int outs) {
  StreamPlan p{};
  p.rt = d.rows <= 32 ? 1 : 2;
  p.tiles_o = (int)ceil_div(outs, 64);
  const int64_t tiles = ceil_div(d.rows, 32 * p.rt) * p.tiles_o;
  p.taken = tiles <= 1024;
  const int unit = 4 * step4(d);
  const int64_t splits = std::clamp<int64_t>(ceil_div(512, std::max<int64_t>(tiles, 1)), 1, std::min<int64_t>(ceil_div(width, unit), 16));
  p.chunk = (int)(ceil_div(ceil_div(width, splits), unit) * unit);
  p.splits = (int)ceil_div(width, p.chunk);
  p.blocks = tiles * p.splits;
  return p;
}
size_t parts_bytes(const wcc_adapter_desc &d, const StreamPlan &p, int outs) {
  return p.taken ? align256((size_t)p.splits * d.rows * outs * 4) : 0;
}

// Ranges of rows for the gradients: enough workgroups even where a range has rows of one adapter only, 64 MB of sums at most.
struct GradPlan {
  int splits;
  int64_t range;
};
GradPlan grad_plan(const wcc_adapter_desc &d) {
  const int64_t tiles = ceil_div(std::min(d.C_in, d.C_out), 256);
  const int64_t bytes = (int64_t)d.adapters * d.rank * (d.C_in + d.C_out) * 4;
  int64_t splits = std::clamp<int64_t>(ceil_div(512, tiles), 1, std::max<int64_t>(ceil_div(d.rows, 256), 1));
  if (bytes > 0) splits = std::clamp<int64_t>(splits, 1, std::max<int64_t>(((int64_t)64 << 20) / bytes, 1));
  GradPlan p;
  p.range = std::max<int64_t>(ceil_div(ceil_div(d.rows, splits), 256) * 256, 256);
  p.splits = (int)std::max<int64_t>(ceil_div(d.rows, p.range), 1);
  return p;
}

Low low_of(const wcc_adapter_desc &d, const AdapterArgs &g) { return Low{g.of_row, g.ranks, g.scale, d.adapters, d.rank}; }

template <class T>
ThinJob<T> thin_job(const wcc_adapter_desc &d, const AdapterArgs &g, bool back, float *out) {
  ThinJob<T> j{};
  if (!g.of_row) return j;
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank;
  j.x = (const T *)(back ? g.dy : g.x);
  j.ldx = back ? d.ldy : d.ldx;
  j.rows = d.rows;
  j.width = back ? d.C_out : d.C_in;
  j.m = back ? Thin<T>{(const T *)g.b, co * r, 1, (int)r} : Thin<T>{(const T *)g.a, r * ci, (int)ci, 1};
  j.out = out;
  const int splits = thin_splits(d, j.width);
  j.chunk = (int)(ceil_div(ceil_div(j.width, splits), step4(d)) * step4(d));
  j.splits = (int)ceil_div(j.width, j.chunk);
  j.groups = (int)std::clamp<int64_t>(std::min<int64_t>(d.adapters, 32), 1, d.rows <= 512 ? 32 : 4);
  j.units = ceil_div(d.rows, 32) * j.splits * j.groups;
  return j;
}
template <class T>
Lines lines_of(const wcc_adapter_desc &d, const ThinJob<T> &j) {
  return Lines{j.out, std::max(j.splits, 1), d.rows * d.rank};
}

template <class T>
__global__ __launch_bounds__(256) void adapter_lines_kernel(ThinJob<T> thin, ThinJob<T> thin2, Low low) {
  const int64_t step = (int64_t)gridDim.x * 4;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); unit < thin.units + thin2.units; unit += step) {
    if (unit < thin.units) thin_unit<T>(thin, low, unit);
    else thin_unit<T>(thin2, low, unit - thin.units);
  }
}

// y = x W^T + h m (back: dx from dy), with another job of rank lines beside (the forward ones, for dB)
template <class T>
hipError_t project(const wcc_adapter_desc &d, const AdapterArgs &g, bool back, const ThinJob<T> &thin, const ThinJob<T> &other, float *part,
                   hipStream_t s) {
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank;
  Project<T> p{};
  p.x = (const T *)(back ? g.dy : g.x);
  p.ldx = back ? d.ldy : d.ldx;
  p.rows = d.rows;
  p.width = back ? d.C_out : d.C_in;
  p.outs = back ? d.C_in : d.C_out;
  p.w = (const T *)g.w;
  p.wo = back ? 1 : ci;
  p.wk = back ? ci : 1;
  p.low = low_of(d, g);
  p.m = back ? Thin<T>{(const T *)g.a, r * ci, (int)ci, 1} : Thin<T>{(const T *)g.b, co * r, 1, (int)r};
  p.h = lines_of(d, thin);
  p.y = (T *)g.y;
  p.ldy = back ? d.ldx : d.ldy;
  const StreamPlan sp = stream_plan(d, p.width, p.outs);
  const int64_t thin_blocks = ceil_div(thin.units + other.units, 4);
  if (!sp.taken) {
    if (thin_blocks > 0) adapter_lines_kernel<T><<<(unsigned)std::min<int64_t>(thin_blocks, 1 << 20), 256, 0, s>>>(thin, other, p.low);
    return launch_tiles(p, s);
  }
  const StreamJob<T> job{p.x, p.ldx, p.rows, p.width, p.outs, p.w, ci, part, sp.splits, sp.chunk, sp.tiles_o, sp.blocks};
  const unsigned blocks = (unsigned)(sp.blocks + thin_blocks);
  if (back) {
    if (sp.rt == 1) adapter_products_kernel<T, 1, true><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
    else adapter_products_kernel<T, 2, true><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
  } else {
    if (sp.rt == 1) adapter_products_kernel<T, 1, false><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
    else adapter_products_kernel<T, 2, false><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
  }
  const int tiles_o = (int)ceil_div(p.outs, 256);
  const int rb = (int)std::clamp<int64_t>(d.rows * tiles_o / 512, 1, 16);
  const int64_t fin = ceil_div(d.rows, rb) * tiles_o;
  adapter_finish_kernel<T><<<(unsigned)std::min<int64_t>(fin, 1 << 20), 256, 0, s>>>(part, sp.splits, d.rows, p.outs, p.low, p.m, p.h, p.y,
                                                                                    p.ldy, rb, tiles_o, fin);
  return hipGetLastError();
}

template <class T>
hipError_t forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  const ThinJob<T> thin = thin_job<T>(d, g, false, (float *)g.ws);
  return project<T>(d, g, false, thin, ThinJob<T>{}, (float *)(g.ws + lines_bytes(d, d.C_in)), s);
}

template <class T>
hipError_t backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  char *at = g.ws;
  auto take = [&](size_t bytes) { char *p = at; at += bytes; return p; };
  float *h = (float *)take(lines_bytes(d, d.C_in)), *gr = (float *)take(lines_bytes(d, d.C_out));
  float *part = (float *)take(parts_bytes(d, stream_plan(d, d.C_out, d.C_in), d.C_in));
  const ThinJob<T> back = g.y || g.da ? thin_job<T>(d, g, true, gr) : ThinJob<T>{};
  const ThinJob<T> fore = g.db ? thin_job<T>(d, g, false, h) : ThinJob<T>{};
  const Low low = low_of(d, g);
  if (g.y) {
    const hipError_t e = project<T>(d, g, true, back, fore, part, s);
    if (e != hipSuccess) return e;
  } else if (back.units + fore.units > 0) {
    adapter_lines_kernel<T><<<(unsigned)std::min<int64_t>(ceil_div(back.units + fore.units, 4), 1 << 20), 256, 0, s>>>(back, fore, low);
  }
  if (!g.da && !g.db) return hipGetLastError();
  const GradPlan gp = grad_plan(d);
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank, na = d.adapters * r * ci, nb = d.adapters * r * co;
  int32_t *found = (int32_t *)take(align256((size_t)gp.splits * d.adapters * 4));
  float *pa = (float *)take(gp.splits > 1 ? align256((size_t)gp.splits * na * 4) : 0);
  float *pb = (float *)take(gp.splits > 1 ? align256((size_t)gp.splits * nb * 4) : 0);
  const int tiles_j = (int)ceil_div(r, 32);
  GradJob<T> ja{}, jb{};
  if (g.da) {
    const int tiles = (int)ceil_div(ci, 256);
    ja = GradJob<T>{(const T *)g.x, d.ldx, d.C_in, lines_of(d, back), gp.splits > 1 ? pa : g.da, na, r * ci, (int)ci, 1, found, tiles,
                    (int64_t)tiles * tiles_j * d.adapters * gp.splits};
  }
  if (g.db) {
    const int tiles = (int)ceil_div(co, 256);
    jb = GradJob<T>{(const T *)g.dy, d.ldy, d.C_out, lines_of(d, fore), gp.splits > 1 ? pb : g.db, nb, co * r, 1, (int)r, found, tiles,
                    (int64_t)tiles * tiles_j * d.adapters * gp.splits};
  }
  adapter_grad_kernel<T><<<(unsigned)std::min<int64_t>(ja.blocks + jb.blocks, 1 << 20), 256, 0, s>>>(ja, jb, low, d.rows, gp.splits, gp.range);
  if (gp.splits > 1) {
    const JoinJob a{pa, g.da, g.da ? na : 0, r * ci, (int)ci, 1}, b{pb, g.db, g.db ? nb : 0, co * r, 1, (int)r};
    adapter_grad_join_kernel<<<(unsigned)std::min<int64_t>(ceil_div(a.size + b.size, 256), 1 << 20), 256, 0, s>>>(a, b, low, gp.splits, found);
  }
  return hipGetLastError();
}

}  // namespace

size_t adapter_bytes(const wcc_adapter_desc &d) {
  const StreamPlan f = stream_plan(d, d.C_in, d.C_out), b = stream_plan(d, d.C_out, d.C_in);
  const GradPlan gp = grad_plan(d);
  const size_t lines = lines_bytes(d, d.C_in), sums = (size_t)d.adapters * d.rank * 4;
  const size_t back = lines + lines_bytes(d, d.C_out) + parts_bytes(d, b, d.C_in) + align256((size_t)gp.splits * d.adapters * 4) +
                      (gp.splits > 1 ? align256(gp.splits * sums * d.C_in) + align256(gp.splits * sums * d.C_out) : 0);
  return std::max(lines + parts_bytes(d, f, d.C_out), back);
}

hipError_t launch_adapter_forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  return d.dtype == WCC_BF16 ? forward<bf16_t>(d, g, s) : forward<float>(d, g, s);
}

hipError_t launch_adapter_backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  return d.dtype == WCC_BF16 ? backward<bf16_t>(d, g, s) : backward<float>(d, g, s);
}

}  // namespace wcc

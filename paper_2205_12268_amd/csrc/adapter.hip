// One projection with a low-rank adapter for each row (wcc_adapter_forward, wcc_adapter_backward).
//
// Both directions are a product with W beside two thin ones that go through the rank lines of the row's adapter:
//   forward   h[t,j] = s_a sum_c A_a[j,c] x[t,c],    y[t,o]  = sum_c W[o,c] x[t,c]   + sum_j B_a[o,j] h[t,j]
//   backward  g[t,j] = s_a sum_o B_a[o,j] dy[t,o],   dx[t,c] = sum_o W[o,c] dy[t,o]  + sum_j A_a[j,c] g[t,j]
//   gradients dA_a[j,c] = sum_t g[t,j] x[t,c],       dB_a[o,j] = sum_t h[t,j] dy[t,o]
//
// What is left out of the product with W by the first launch, in ranges of k, a second one adds up, with the thin product, and rounds;
// whole tiles need one launch for the rank lines and one for all else.  Up to 64 rows what has to be read is W and the adapters, once,
// and what counts is how many loads are in flight; from some hundred rows on it is the matrix cores.  Which way a call goes: plan_of.
#include "adapter.h"

namespace wcc {
namespace {

// One or two jobs of rank lines by themselves, before whole tiles.
template <class T>
__global__ __launch_bounds__(256, 2) void adapter_lines_kernel(ThinJob<T> g1, ThinJob<T> g2, Low low) {
  __shared__ ThinLds lds;
  __shared__ __align__(1024) unsigned char room[4][kThinRoom];
  unsigned char *own = room[threadIdx.x >> 6];
  for (int64_t b = blockIdx.x; b < g1.blocks + g2.blocks; b += gridDim.x) {
    const bool second = b >= g1.blocks;
    thin_block<T>(second ? g2 : g1, low, second ? b - g1.blocks : b, lds, own);
    __syncthreads();
  }
}

// ---- the product with W for few rows: fp32, and bf16 that 16-byte loads cannot take ---------------------------------
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
      if constexpr (!NN) {
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
    if constexpr (!NN) {
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

// First launch: workgroups of one or two jobs of rank lines (they take longest), then of the product with W.
template <class T, int RT, bool NN>
__global__ __launch_bounds__(256, 2) void adapter_products_kernel(StreamJob<T> g, ThinJob<T> thin, ThinJob<T> thin2, Low low) {
  __shared__ float red[4 * 32 * RT * 72];
  const int64_t block = blockIdx.x;
  if (block < thin.blocks + thin2.blocks) {
    __shared__ ThinLds lds;
    unsigned char *own = nullptr;  // (few rows: not by ranges)
    if (block < thin.blocks) thin_block<T>(thin, low, block, lds, own);
    else thin_block<T>(thin2, low, block - thin.blocks, lds, own);
    return;
  }
  stream_block<T, RT, NN>(g, block - thin.blocks - thin2.blocks, red);
}

// The sum of the parts of one result, four loads at a time.
__device__ __forceinline__ float sum_parts(const float *__restrict__ p, int splits, int64_t stride) {
  float v = p[0];
  for (int s = 1; s < splits; s += 4) {
    float w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) w[u] = s + u < splits ? p[(s + u) * stride] : 0.f;
    v += (w[0] + w[1]) + (w[2] + w[3]);
  }
  return v;
}

template <class T>
struct FinishJob {
  const float *part;
  int splits, outs, tiles_o;
  int64_t rows;
  Thin<T> m;
  Lines h;
  T *y;
  int64_t ldy, blocks;
};

// Second launch: y[t, o] = the sum of the parts + sum_j m(a, j, o) h[t, j].
// Few rows, each likely with an adapter of its own: 256 outputs of a row a workgroup.
template <class T>
__global__ __launch_bounds__(256) void adapter_finish_row_kernel(FinishJob<T> g, Low low) {
  constexpr int VE = VecOf<T>::N, Q = 32 / VE;
  __shared__ float hs[WCC_MAX_RANK];
  for (int64_t b = blockIdx.x; b < g.blocks; b += gridDim.x) {
    const int o = (int)(b % g.tiles_o) * 256 + (int)threadIdx.x, oc = min(o, g.outs - 1);
    const int64_t t = b / g.tiles_o;
    const int a = low.of(t), lines = a >= 0 ? low.lines(a) : 0;
    u32x4 mf[Q] = {};
    if (low.of_row) {  // the first 32 lines' loads go out together with the others (without adapters there may be nothing at m.p)
#pragma unroll
      for (int q = 0; q < Q; ++q) mf[q] = thin_k(g.m, max(a, 0), oc, q * VE, lines);
    }
    float v = sum_parts(g.part + t * g.outs + oc, g.splits, g.rows * g.outs);
    if ((int)threadIdx.x < lines) hs[threadIdx.x] = g.h.at(t * g.h.ld + threadIdx.x);
    __syncthreads();
    float low_v = 0.f;
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (q * VE + i < lines) low_v = fmaf(elem<T>(mf[q], i), hs[q * VE + i], low_v);
    for (int j = 32; j < lines; j += VE) {
      const u32x4 f = thin_k(g.m, a, oc, j, lines);
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (j + i < lines) low_v = fmaf(elem<T>(f, i), hs[j + i], low_v);
    }
    if (o < g.outs) g.y[t * g.ldy + o] = narrow<T>(v + low_v);
    __syncthreads();
  }
}

// More rows: 32 rows x 64 outputs a workgroup.  Each wave has all of them and, of the distinct adapters among the rows, every
// fourth: the thin products of rows in any order are as many trips to memory one after the other as there are adapters, and those
// trips are what bounds it.  (One wave for all adapters of 32 outputs: 190 rows of mixed adapters, rank 64, 4072 outputs took 28 us,
// this 17.  Three workgroups a compute unit: 777 rows x 1537 outputs 11 us, with two 17.)
template <class T>
__global__ __launch_bounds__(256, 3) void adapter_finish_tile_kernel(FinishJob<T> g, Low low) {
  constexpr int LD = 68;
  __shared__ __align__(16) float sums[4][32][LD];
  __shared__ __align__(16) T h[32 * PartsOf<T>::Out * WCC_MAX_RANK];
  const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), ln = lane & 31, half = lane >> 5;
  for (int64_t b = blockIdx.x; b < g.blocks; b += gridDim.x) {
    const int o0 = (int)(b % g.tiles_o) * 64, r = tid >> 4, c = (tid & 15) * 4, oq = o0 + c;
    const int64_t t0 = b / g.tiles_o * 32, stride = g.rows * g.outs;
    f32x4_any v[2] = {};
    if (low.of_row) gather_lines<T, 32>(low, g.h, [&](int row) { return h + row * PartsOf<T>::Out * g.h.ld; }, t0, g.rows);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float *p = g.part + min(t0 + r + 16 * i, g.rows - 1) * g.outs + min(oq, g.outs - 1);
      if (oq + 4 <= g.outs) {
        int s = 0;
        for (; s + 4 <= g.splits; s += 4) {
          f32x4_any w[4];
#pragma unroll
          for (int u = 0; u < 4; ++u) w[u] = *reinterpret_cast<const f32x4_any *>(p + (s + u) * stride);
          v[i] += (w[0] + w[1]) + (w[2] + w[3]);
        }
        for (; s < g.splits; ++s) v[i] += *reinterpret_cast<const f32x4_any *>(p + s * stride);
      } else {
#pragma unroll
        for (int q = 0; q < 3; ++q)
          if (oq + q < g.outs) v[i][q] = sum_parts(p + q, g.splits, stride);
      }
    }
    if (low.of_row) {
      const int o[2] = {o0 + ln, o0 + 32 + ln};
      f32x16 acc[2][1] = {};
      __syncthreads();
      add_thin<T, 2, 1, true, 2>(low, g.m, g.h.ld, [&](int) { return h; }, g.rows, g.outs, t0, o, acc, wv, 4);
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) sums[wv][result_line(i, half)][e * 32 + ln] = acc[e][0][i];
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        f32x4_any w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = *reinterpret_cast<const f32x4_any *>(&sums[u][r + 16 * i][c]);
        v[i] += (w[0] + w[1]) + (w[2] + w[3]);  // (a row's is one of them, the others' are 0)
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t t = t0 + r + 16 * i;
      if (t >= g.rows) continue;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (oq + q < g.outs) g.y[t * g.ldy + oq + q] = narrow<T>(v[i][q]);
    }
    __syncthreads();
  }
}

// ---- gradients of the adapters ------------------------------------------------------------------------------------
// grad(a, j, c) = sum over the rows t of adapter a of h[t, j] x[t, c], at a * major + j * sj + c * sc.
// A workgroup has an adapter, 512 columns, 32 lines and a range of rows.  It lists the rows that are the adapter's, 256 of the
// range at a time, so that rows of many adapters in any order are read once in all.  The listed rows' h go to LDS as
// operands (bf16: in three parts, which keep all 24 bits), x from memory: a lane has four columns of the rows of a step.
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

constexpr int kListed = 256 + 16;  // rows of a round, and what is left of the last step of the one before

template <class T>
struct GradLds {
  static constexpr int P = PartsOf<T>::Grad;
  T h[P][32][kListed];
  int list[kListed], rest[16], counts[2][4], odd[2][4];
};

// four columns (some of them past the width) of a row
template <class T>
__device__ __forceinline__ void load_four(const T *p, int left, uint32_t (&v)[(int)sizeof(T)]) {
  if constexpr (sizeof(T) == 4) {
    if (left >= 4) {
      const u32x4 q = *reinterpret_cast<const u32x4_any *>(p);
      v[0] = q[0], v[1] = q[1], v[2] = q[2], v[3] = q[3];
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = i < left ? __float_as_uint(p[i]) : 0u;
    }
  } else {
    if (left >= 4) {
      typedef uint64_t u64_2 __attribute__((aligned(2)));
      const uint64_t q = *reinterpret_cast<const u64_2 *>(p);
      v[0] = (uint32_t)q, v[1] = (uint32_t)(q >> 32);
    } else {
      v[0] = left > 0 ? (uint32_t)p[0] | (left > 1 ? (uint32_t)p[1] << 16 : 0u) : 0u;
      v[1] = left > 2 ? (uint32_t)p[2] : 0u;
    }
  }
}

// AGAIN: an infinity of x meets no part of a line past the first, which is 0 where the first has all of it (infinity times 0 is NaN).
// Whether sums of the wave are not finite: then the workgroup has to do the block so (bf16).
template <class T, bool FLIP, bool AGAIN>
__device__ __forceinline__ bool grad_block(const GradJob<T> &g, const Low &low, int64_t rows, int splits, int64_t range, int64_t block,
                                           GradLds<T> &lds) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, P = GradLds<T>::P, D = (int)sizeof(T);
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5;
  const int tiles_j = (low.rank + 31) / 32;
  const int split = (int)(block % splits), j0 = (int)(block / splits % tiles_j) * 32;
  const int tile_c = (int)(block / splits / tiles_j % g.tiles_c), a = (int)(block / splits / tiles_j / g.tiles_c);
  const int lines = low.lines(a), cw = tile_c * 512 + wv * 128, c = cw + 4 * ln, left = g.width - c;
  const bool busy = cw < g.width;
  const T *xc = g.x + min(c, g.width - 1);
  const int64_t t_end = min(rows, (split + 1) * range);
  f32x16 acc[4] = {};
  int have = 0, total = 0, round = 0;
  // most ranges have rows of few adapters: a wave looks by itself whether there are any of this one
  if (range <= 256) {
    bool any = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t t = split * range + i * 64 + lane;
      any |= i * 64 + lane < range && t < rows && low.of(t) == a;
    }
    if (splits > 1 && __ballot(any) == 0) {
      if (tile_c == 0 && j0 == 0 && tid == 0) g.found[(int64_t)split * low.n + a] = 0;
      return false;
    }
  }

  // the columns of the listed rows of step s; of a single step of n < KS rows the others are zeros
  auto fetch = [&](int s, int n, uint32_t (&v)[VE][D]) {
    const int at = s * KS + half * VE;
#pragma unroll
    for (int i = 0; i < VE; ++i) {
#pragma unroll
      for (int d = 0; d < D; ++d) v[i][d] = 0u;
      if (n >= KS || half * VE + i < n) load_four<T>(xc + (int64_t)lds.list[at + i] * g.ldx, left, v[i]);
    }
  };
  auto multiply = [&](int s, const uint32_t (&v)[VE][D]) {
    u32x4 hf[P];
#pragma unroll
    for (int p = 0; p < P; ++p) hf[p] = *reinterpret_cast<const u32x4 *>(&lds.h[p][ln][s * KS + half * VE]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u32x4 xf;
      if constexpr (D == 4) {
#pragma unroll
        for (int i = 0; i < 4; ++i) xf[i] = v[i][e];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          xf[i] = __builtin_amdgcn_perm(v[2 * i + 1][e >> 1], v[2 * i][e >> 1], e & 1 ? 0x07060302 : 0x05040100);
      }
#pragma unroll
      for (int p = P - 1; p >= 0; --p) {
        const u32x4 xp = AGAIN && p > 0 ? finite_of(xf) : xf;
        acc[e] = FLIP ? mma<T>(xp, hf[p], acc[e]) : mma<T>(hf[p], xp, acc[e]);
      }
    }
  };
  // the operands of listed rows from..to of h; zeros to the end of their step
  auto stage = [&](int from, int to) {
    const int end = (to + KS - 1) / KS * KS;
    for (int i = from * 32 + tid; i < end * 32; i += 256) {
      const int q = i >> 5, line = i & 31;
      float v = 0.f;
      if (q < to && j0 + line < lines) v = g.h.at((int64_t)lds.list[q] * g.h.ld + j0 + line);
      if constexpr (D == 4) {
        lds.h[0][line][q] = v;
      } else {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const bf16_t b = narrow<bf16_t>(v);
          lds.h[p][line][q] = b;
          v = left_of(v, b);
        }
      }
    }
  };
  if (j0 < lines) {
    for (int64_t t0 = split * range; t0 < t_end; t0 += 256, round ^= 1) {
      const int64_t t = t0 + tid;
      const bool mine = t < t_end && low.of(t) == a;
      const uint64_t vote = __ballot(mine);
      if (lane == 0) lds.counts[round][wv] = __popcll(vote);
      __syncthreads();
      int before = have, all = have;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int n = lds.counts[round][i];
        if (i < wv) before += n;
        all += n;
      }
      if (all == have) continue;  // (the other counts are written next)
      if (mine) lds.list[before + __popcll(vote & ((1ull << lane) - 1))] = (int)t;
      __syncthreads();
      total += all - have;
      const int full = all / KS * KS;
      if (full > 0) {
        // (two steps' columns are on their way while h is staged, and while the two before are multiplied)
        uint32_t v0[VE][D], v1[VE][D];
        const int steps = full / KS;
        if (busy) {
          fetch(0, KS, v0);
          if (steps > 1) fetch(1, KS, v1);
        }
        stage(0, full);
        __syncthreads();
        if (busy)
          for (int s = 0; s < steps; s += 2) {
            multiply(s, v0);
            if (s + 2 < steps) fetch(s + 2, KS, v0);
            if (s + 1 < steps) multiply(s + 1, v1);
            if (s + 3 < steps) fetch(s + 3, KS, v1);
          }
        __syncthreads();
        have = all - full;
        if (tid < have) lds.rest[tid] = lds.list[full + tid];
        __syncthreads();
        if (tid < have) lds.list[tid] = lds.rest[tid];
      } else {
        have = all;
      }
    }
    __syncthreads();
    if (have > 0) {
      uint32_t v0[VE][D];
      if (busy) fetch(0, have, v0);
      stage(0, have);
      __syncthreads();
      if (busy) multiply(0, v0);
    }
  }
  if (splits > 1) {
    if (tile_c == 0 && j0 == 0 && tid == 0) g.found[(int64_t)split * low.n + a] = total;
    if (total == 0) return false;
  }
  if (!busy) return false;
  float *out = g.out + (splits > 1 ? split * g.size : 0) + a * g.major;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int q = result_line(i, half);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int line = j0 + (FLIP ? ln : q), col = cw + 4 * (FLIP ? q : ln) + e;
      if (line < low.rank && col < g.width) out[(int64_t)line * g.sj + (int64_t)col * g.sc] = line < lines ? acc[e][i] : 0.f;
    }
  }
  float none[4] = {};
  if constexpr (P > 1 && !AGAIN) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) none[e] = fmaf(acc[e][i], 0.f, none[e]);
  }
  return __ballot((none[0] + none[1]) + (none[2] + none[3]) != 0.f) != 0;
}

// dA's blocks, then dB's (whose lines are the contiguous ones: its results lie the other way round)
template <class T>
__global__ __launch_bounds__(256, 3) void adapter_grad_kernel(GradJob<T> ga, GradJob<T> gb, Low low, int64_t rows, int splits, int64_t range) {
  __shared__ __align__(16) GradLds<T> lds;
  int turn = 0;
  for (int64_t b = blockIdx.x; b < ga.blocks + gb.blocks; b += gridDim.x, turn ^= 1) {
    const bool odd = b < ga.blocks ? grad_block<T, false, false>(ga, low, rows, splits, range, b, lds)
                                   : grad_block<T, true, false>(gb, low, rows, splits, range, b - ga.blocks, lds);
    if constexpr (GradLds<T>::P > 1) {
      if ((threadIdx.x & 63) == 0) lds.odd[turn][threadIdx.x >> 6] = odd;
    }
    __syncthreads();
    if constexpr (GradLds<T>::P > 1) {
      const int *all = lds.odd[turn];
      if ((all[0] | all[1] | all[2] | all[3]) == 0) continue;
      if (b < ga.blocks) grad_block<T, false, true>(ga, low, rows, splits, range, b, lds);
      else grad_block<T, true, true>(gb, low, rows, splits, range, b - ga.blocks, lds);
      __syncthreads();
    }
  }
}

// The ranges' sums as one, in their order; lines past an adapter's rank are 0.  A workgroup has 1024 entries of an adapter and
// lists the ranges that have rows of it first.
struct JoinJob {
  const float *part;
  float *out;
  int64_t size, major;
  int sj, sc, tiles;
};
constexpr int kRanges = 1024;
__global__ __launch_bounds__(256) void adapter_grad_join_kernel(JoinJob ja, JoinJob jb, Low low, int splits,
                                                                const int32_t *__restrict__ found) {
  __shared__ int list[kRanges], counts[4];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int64_t blocks = (int64_t)(ja.tiles + jb.tiles) * low.n;
  for (int64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
    const int a = (int)(b / (ja.tiles + jb.tiles)), tile = (int)(b % (ja.tiles + jb.tiles));
    const bool first = tile < ja.tiles;
    const JoinJob &g = first ? ja : jb;
    int n = 0;
    for (int s0 = 0; s0 < splits; s0 += 256) {
      const int s = s0 + tid;
      const bool has = s < splits && found[(int64_t)s * low.n + a] > 0;
      const uint64_t vote = __ballot(has);
      if (lane == 0) counts[wv] = __popcll(vote);
      __syncthreads();
      int before = n;
      for (int i = 0; i < wv; ++i) before += counts[i];
      if (has) list[before + __popcll(vote & ((1ull << lane) - 1))] = s;
      n += counts[0] + counts[1] + counts[2] + counts[3];
      __syncthreads();
    }
    const int lines = low.lines(a);
    const int64_t at0 = (int64_t)(first ? tile : tile - ja.tiles) * 1024;
    const int64_t in = at0 + tid * 4;
    const float *p = g.part + a * g.major + in;
    float *out = g.out + a * g.major + in;
    if (in + 4 <= g.major) {
      f32x4_any v = {};
      int i = 0;
      for (; i + 4 <= n; i += 4) {
        f32x4_any w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = *reinterpret_cast<const f32x4_any *>(p + list[i + u] * g.size);
        v += (w[0] + w[1]) + (w[2] + w[3]);
      }
      for (; i < n; ++i) v += *reinterpret_cast<const f32x4_any *>(p + list[i] * g.size);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if ((g.sj == 1 ? (int)((in + q) % low.rank) : (int)((in + q) / g.sj)) >= lines) v[q] = 0.f;
      *reinterpret_cast<f32x4_any *>(out) = v;
    } else {
      for (int q = 0; in + q < g.major; ++q) {
        float v = 0.f;
        if ((g.sj == 1 ? (int)((in + q) % low.rank) : (int)((in + q) / g.sj)) < lines)
          for (int i = 0; i < n; ++i) v += p[list[i] * g.size + q];
        out[q] = v;
      }
    }
    __syncthreads();
  }
}

// ---- rows that 16-byte loads cannot take --------------------------------------------------------------------------
// A copy of a bf16 matrix, its rows `chunks` whole chunks of 8 long, what is past its width and its rows 0.
struct PackJob {
  const bf16_t *from;
  int64_t ld, rows, rows_to;
  int width, chunks;
  bf16_t *to;
};

__global__ __launch_bounds__(256) void adapter_pack_kernel(PackJob g1, PackJob g2) {
  const int64_t n1 = g1.rows_to * g1.chunks, n = n1 + g2.rows_to * g2.chunks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const bool second = i >= n1;
    const PackJob &g = second ? g2 : g1;
    const int64_t at = second ? i - n1 : i, row = at / g.chunks;
    const int c = (int)(at - row * g.chunks) * 8;
    reinterpret_cast<u32x4 *>(g.to)[at] = load_k(g.from + row * g.ld + c, row < g.rows ? g.width - c : 0);
  }
}

// ---- host ------------------------------------------------------------------------------------------------------------
size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// k of a range is a multiple of 64 bf16 / 32 fp32 elements (four waves' steps)
int step4(const wcc_adapter_desc &d) { return d.dtype == WCC_BF16 ? 64 : 32; }
int lines_ld(const wcc_adapter_desc &d) { return (d.rank + 7) / 8 * 8; }

// How y = x W^T is made: bf16 that 16-byte loads can take by adapter_gemm.hip, whatever else by the stream (up to 64 rows) or
// adapter_tile.hip; in ranges of k where the tiles alone would leave compute units without work.  (fp32, stream and tiles: 64 rows,
// 2048 -> 2048 25 and 30 us, 40 rows, 1024 -> 512 15 and 18; 1588 rows, 3520 -> 704 157 and 142.)
struct Plan {
  enum { kStream, kTiles, kGemm, kGemmSplit } route;
  int rt, splits, chunk, tiles_o;
  int64_t blocks;  // of the stream
  bool parts() const { return route == kStream || route == kGemmSplit || splits > 1; }
};
Plan plan_of(const wcc_adapter_desc &d, int width, int outs, bool aligned) {
  Plan p{};
  const int64_t rows = std::max<int64_t>(d.rows, 1);
  if (aligned) {
    p.splits = gemm_splits(rows, (width + 7) / 8 * 8, outs);
    p.route = p.splits > 1 || rows <= 64 ? Plan::kGemmSplit : Plan::kGemm;
  } else if (rows <= 64) {
    p.route = Plan::kStream;
    p.rt = rows <= 32 ? 1 : 2;
    p.tiles_o = (int)ceil_div(outs, 64);
    const int unit = 4 * step4(d);
    const int64_t splits = std::clamp<int64_t>(ceil_div(512, p.tiles_o), 1, std::min<int64_t>(ceil_div(width, unit), 16));
    p.chunk = (int)(ceil_div(ceil_div(width, splits), unit) * unit);
    p.splits = (int)ceil_div(width, p.chunk);
    p.blocks = (int64_t)p.tiles_o * p.splits;
  } else {
    p.route = Plan::kTiles;
    p.splits = tile_splits(rows, width, outs, d.dtype == WCC_BF16 ? 2 : 4);
  }
  return p;
}
// Ranges of k of the rank lines, of 256 (many rows: 128) at least: as many as give two workgroups (many rows: one) a compute unit, 16 at most; 8 where
// more than four adapters share many rows among groups of workgroups (512 rows, 4096 -> 4096, 24 adapters, with the product: 24 us
// with 8, 32 with 16; 190 rows, 5232 -> 4072, 4 adapters: 42 and 35).
int thin_splits(const wcc_adapter_desc &d, int width) {
  const int64_t rows = std::max<int64_t>(d.rows, 1), most = std::clamp<int64_t>(width / (rows <= 64 ? 256 : 128), 1, rows <= 64 || d.adapters <= 4 ? 16 : 8);
  return (int)std::clamp<int64_t>(ceil_div(rows <= 64 ? 512 : 256, ceil_div(rows, kRange)), 1, most);
}
size_t lines_bytes(const wcc_adapter_desc &d, int width) { return align256((size_t)thin_splits(d, width) * d.rows * lines_ld(d) * 4); }
size_t parts_bytes(const wcc_adapter_desc &d, const Plan &p, int outs) {
  return p.parts() ? align256((size_t)p.splits * d.rows * outs * 4) : 0;
}

// Copies of x (back: dy) and W that 16-byte loads can take, where the strides do not allow them: then the products go through
// adapter_gemm.hip.  From 2^32 of them on, and if W is copied from 512 rows on: the copies take 4 to 7 us, and W's the time of twice
// its bytes (rows 3 further apart: 1172 rows, 2816 -> 4224, 29 adapters, 121 us without and 100 with; 777 rows, 1000 -> 1537,
// 34 and 39).
struct Packs {
  bool x, w;
  int width, outs;  // of the copies
  size_t x_bytes, w_bytes;
};
Packs packs_of(const wcc_adapter_desc &d, bool back) {
  const int width = back ? d.C_out : d.C_in, outs = back ? d.C_in : d.C_out;
  const int64_t ld = back ? d.ldy : d.ldx;
  Packs k{};
  k.width = (width + 7) / 8 * 8, k.outs = back ? (outs + 7) / 8 * 8 : outs;
  k.x = ld % 8 != 0 || k.width != width;
  k.w = k.width != width || k.outs != outs;
  if (d.dtype != WCC_BF16 || d.rows <= 64 || (k.w && d.rows < 512) || d.rows * width < ((int64_t)1 << 32) / outs) k.x = k.w = false;
  if (k.x) k.x_bytes = align256((size_t)d.rows * k.width * 2);
  if (k.w) k.w_bytes = align256((size_t)k.width * k.outs * 2);
  return k;
}

// Ranges of rows for the gradients: the sums of the ranges no more than twice what x takes, 64 rows at least in a range.
struct GradPlan {
  int splits;
  int64_t range;
};
GradPlan grad_plan(const wcc_adapter_desc &d) {
  const int64_t size = d.dtype == WCC_BF16 ? 2 : 4, lines = std::max<int64_t>((int64_t)d.adapters * d.rank, 1);
  const int64_t tiles = ceil_div(d.C_in, 512) + ceil_div(d.C_out, 512);
  int64_t splits = std::min(ceil_div(d.rows, 64), d.rows * size / (2 * lines));
  splits = std::clamp<int64_t>(splits, 1, std::clamp<int64_t>(1024 / tiles, 1, kRanges));
  GradPlan p;
  p.range = std::max<int64_t>(ceil_div(ceil_div(d.rows, splits), 64) * 64, 64);
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
  j.chunk = (int)(ceil_div(ceil_div(j.width, thin_splits(d, j.width)), step4(d)) * step4(d));
  j.out = Lines{out, (int)ceil_div(j.width, j.chunk), lines_ld(d), d.rows * lines_ld(d)};
  j.by_range = d.rows > 64;
  const int64_t ranges = ceil_div(d.rows, kRange) * j.out.splits;
  // (up to 64 rows a wave an adapter, more: workgroups for two a compute unit, but not where few adapters leave them idle)
  j.groups = j.by_range ? (int)std::clamp<int64_t>(512 / ranges, 1, std::min<int64_t>(8, ceil_div(d.adapters, 4))) : std::clamp(d.adapters, 1, 32);
  j.units = ceil_div(d.rows, 32) * j.out.splits * j.groups;
  j.blocks = j.by_range ? ranges * j.groups : ceil_div(j.units, 4);
  return j;
}

template <class T>
void launch_lines(const ThinJob<T> &g1, const ThinJob<T> &g2, const Low &low, hipStream_t s) {
  if (g1.blocks + g2.blocks > 0)
    adapter_lines_kernel<T><<<(unsigned)std::min<int64_t>(g1.blocks + g2.blocks, 1 << 20), 256, 0, s>>>(g1, g2, low);
}

template <class T>
Project<T> project_of(const wcc_adapter_desc &d, const AdapterArgs &g, bool back) {
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
  p.y = (T *)g.y;
  p.ldy = back ? d.ldx : d.ldy;
  return p;
}
template <class T>
bool aligned(const Project<T> &p) {
  if constexpr (sizeof(T) == 2) return gemm_takes(p);
  return false;
}

// p on copies, where they let 16-byte loads take it; `at`: their place
void pack(Project<bf16_t> &p, const wcc_adapter_desc &d, bool back, char *at, hipStream_t s) {
  const Packs k = packs_of(d, back);
  if (!k.x && !k.w) return;
  Project<bf16_t> q = p;
  PackJob jx{}, jw{};
  if (k.x) {
    q.x = (const bf16_t *)at, q.ldx = k.width;
    jx = PackJob{p.x, p.ldx, p.rows, p.rows, p.width, k.width / 8, (bf16_t *)at};
    at += k.x_bytes;
  }
  if (k.w) {
    q.w = (const bf16_t *)at;
    (back ? q.wk : q.wo) = back ? k.outs : k.width;
    jw = back ? PackJob{p.w, p.wk, p.width, k.width, p.outs, k.outs / 8, (bf16_t *)at} : PackJob{p.w, p.wo, p.outs, p.outs, p.width, k.width / 8, (bf16_t *)at};
  }
  q.width = k.width;
  if (!gemm_takes(q)) return;  // (what is not copied begins between 16 bytes)
  p = q;
  const int64_t n = jx.rows_to * jx.chunks + jw.rows_to * jw.chunks;
  adapter_pack_kernel<<<(unsigned)std::min<int64_t>(ceil_div(n, 256), 1 << 14), 256, 0, s>>>(jx, jw);
}

// y = x W^T + h m (back: dx from dy), with another job of rank lines beside (the forward ones, for dB)
template <class T>
void project(Project<T> p, const Plan &pl, const ThinJob<T> &thin, const ThinJob<T> &other, float *part, hipStream_t s) {
  p.h = thin.out;
  if (!pl.parts()) {
    launch_lines(thin, other, p.low, s);
    if constexpr (sizeof(T) == 2) {
      if (pl.route == Plan::kGemm) return launch_gemm(p, s);
    }
    return launch_tiles(p, 1, nullptr, thin, other, s);
  }
  if (pl.route == Plan::kGemmSplit) {
    if constexpr (sizeof(T) == 2) launch_gemm_split(p, pl.splits, part, thin, other, s);
  } else if (pl.route == Plan::kTiles) {
    // The rank lines beside the tiles where all workgroups have a place at once; else they would keep tiles waiting for a second
    // turn (1588 rows, 3520 -> 704, fp32: 150 us beside, 133 us with a launch of their own).
    const bool beside = tiles_of(p.rows, p.outs) * pl.splits + thin.blocks + other.blocks <= kPlaces;
    if (!beside) launch_lines(thin, other, p.low, s);
    launch_tiles(p, pl.splits, part, beside ? thin : ThinJob<T>{}, beside ? other : ThinJob<T>{}, s);
  } else {
    const bool nn = p.wk != 1;
    const StreamJob<T> job{p.x, p.ldx, p.rows, p.width, p.outs, p.w, nn ? p.wk : p.wo, part, pl.splits, pl.chunk, pl.tiles_o, pl.blocks};
    const unsigned blocks = (unsigned)(pl.blocks + thin.blocks + other.blocks);
    if (nn) {
      if (pl.rt == 1) adapter_products_kernel<T, 1, true><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
      else adapter_products_kernel<T, 2, true><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
    } else {
      if (pl.rt == 1) adapter_products_kernel<T, 1, false><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
      else adapter_products_kernel<T, 2, false><<<blocks, 256, 0, s>>>(job, thin, other, p.low);
    }
  }
  const bool by_row = p.rows <= 64;  // (64 rows, 2048 -> 2048, 4 adapters, by row and by tiles: bf16 15.2 and 18.1 us, fp32 24.7 and 28.2)
  const int tiles_o = (int)ceil_div(p.outs, by_row ? 256 : 64);
  const FinishJob<T> f{part, pl.splits, p.outs, tiles_o, p.rows, p.m, p.h, p.y, p.ldy, ceil_div(p.rows, by_row ? 1 : 32) * tiles_o};
  if (by_row) adapter_finish_row_kernel<T><<<(unsigned)std::min<int64_t>(f.blocks, 1 << 20), 256, 0, s>>>(f, p.low);
  else adapter_finish_tile_kernel<T><<<(unsigned)std::min<int64_t>(f.blocks, 1 << 20), 256, 0, s>>>(f, p.low);
}

template <class T>
hipError_t forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  char *at = g.ws;
  auto take = [&](size_t bytes) { char *p = at; at += bytes; return p; };
  const Packs k = packs_of(d, false);
  float *h = (float *)take(lines_bytes(d, d.C_in));
  char *copies = take(k.x_bytes + k.w_bytes);
  Project<T> p = project_of<T>(d, g, false);
  if constexpr (sizeof(T) == 2) pack(p, d, false, copies, s);
  project<T>(p, plan_of(d, d.C_in, d.C_out, aligned(p)), thin_job<T>(d, g, false, h), ThinJob<T>{}, (float *)at, s);
  return hipGetLastError();
}

template <class T>
hipError_t backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  char *at = g.ws;
  auto take = [&](size_t bytes) { char *p = at; at += bytes; return p; };
  Project<T> p = project_of<T>(d, g, true);
  const Low low = p.low;
  float *gr = (float *)take(lines_bytes(d, d.C_out)), *h = (float *)take(lines_bytes(d, d.C_in));
  const Packs k = packs_of(d, true);
  char *copies = take(k.x_bytes + k.w_bytes);
  if constexpr (sizeof(T) == 2) {
    if (g.y) pack(p, d, true, copies, s);
  }
  const Plan pl = plan_of(d, d.C_out, d.C_in, aligned(p));
  float *part = (float *)take(g.y ? parts_bytes(d, pl, d.C_in) : 0);
  const ThinJob<T> back = g.y || g.da ? thin_job<T>(d, g, true, gr) : ThinJob<T>{};
  const ThinJob<T> fore = g.db ? thin_job<T>(d, g, false, h) : ThinJob<T>{};
  if (g.y) project<T>(p, pl, back, fore, part, s);
  else launch_lines(back, fore, low, s);
  if (!g.da && !g.db) return hipGetLastError();
  const GradPlan gp = grad_plan(d);
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank, na = d.adapters * r * ci, nb = d.adapters * r * co;
  int32_t *found = (int32_t *)take(align256((size_t)gp.splits * d.adapters * 4));
  float *pa = (float *)take(gp.splits > 1 ? align256((size_t)gp.splits * na * 4) : 0);
  float *pb = (float *)take(gp.splits > 1 ? align256((size_t)gp.splits * nb * 4) : 0);
  const int tiles_j = (int)ceil_div(r, 32);
  GradJob<T> ja{}, jb{};
  if (g.da) {
    const int tiles = (int)ceil_div(ci, 512);
    ja = GradJob<T>{(const T *)g.x, d.ldx, d.C_in, back.out, gp.splits > 1 ? pa : g.da, na, r * ci, (int)ci, 1, found, tiles,
                    (int64_t)tiles * tiles_j * d.adapters * gp.splits};
  }
  if (g.db) {
    const int tiles = (int)ceil_div(co, 512);
    jb = GradJob<T>{(const T *)g.dy, d.ldy, d.C_out, fore.out, gp.splits > 1 ? pb : g.db, nb, co * r, 1, (int)r, found, tiles,
                    (int64_t)tiles * tiles_j * d.adapters * gp.splits};
  }
  adapter_grad_kernel<T><<<(unsigned)std::min<int64_t>(ja.blocks + jb.blocks, 1 << 20), 256, 0, s>>>(ja, jb, low, d.rows, gp.splits, gp.range);
  if (gp.splits > 1) {
    const JoinJob a{pa, g.da, na, r * ci, (int)ci, 1, g.da ? (int)ceil_div(r * ci, 1024) : 0};
    const JoinJob b{pb, g.db, nb, co * r, 1, (int)r, g.db ? (int)ceil_div(co * r, 1024) : 0};
    adapter_grad_join_kernel<<<(unsigned)std::min<int64_t>((int64_t)(a.tiles + b.tiles) * d.adapters, 1 << 20), 256, 0, s>>>(a, b, low, gp.splits, found);
  }
  return hipGetLastError();
}

}  // namespace

size_t adapter_bytes(const wcc_adapter_desc &d) {
  const GradPlan gp = grad_plan(d);
  const size_t sums = (size_t)d.adapters * d.rank * 4;
  const size_t grads = align256((size_t)gp.splits * d.adapters * 4) +
                       (gp.splits > 1 ? align256(gp.splits * sums * d.C_in) + align256(gp.splits * sums * d.C_out) : 0);
  const Packs fore = packs_of(d, false), back = packs_of(d, true);
  size_t most = 0;
  for (const bool fits : {false, true}) {  // (alignment is known with the pointers)
    const bool al = fits && d.dtype == WCC_BF16;
    most = std::max(most, parts_bytes(d, plan_of(d, d.C_in, d.C_out, al), d.C_out) + fore.x_bytes + fore.w_bytes);
    most = std::max(most, parts_bytes(d, plan_of(d, d.C_out, d.C_in, al), d.C_in) + lines_bytes(d, d.C_out) + grads + back.x_bytes + back.w_bytes);
  }
  return lines_bytes(d, d.C_in) + most;
}

hipError_t launch_adapter_forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  return d.dtype == WCC_BF16 ? forward<bf16_t>(d, g, s) : forward<float>(d, g, s);
}

hipError_t launch_adapter_backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  return d.dtype == WCC_BF16 ? backward<bf16_t>(d, g, s) : backward<float>(d, g, s);
}

}  // namespace wcc

// The projection with adapters: what its translation units share.  (How its products meet on the matrix cores: tiles.h.)
#pragma once

#include <type_traits>

#include "tiles.h"

namespace wcc {

// ---- the adapters as the kernels see them ------------------------------------------------------------------
struct Low {
  const int32_t *of_row;  // nullptr: none
  const int32_t *ranks;
  const float *scale;
  int n, rank;
  __device__ __forceinline__ int of(int64_t t) const {
    const int a = of_row ? of_row[t] : -1;
    return (uint32_t)a < (uint32_t)n ? a : -1;
  }
  __device__ __forceinline__ int lines(int a) const { return ranks ? min(max(ranks[a], 0), rank) : rank; }
  __device__ __forceinline__ float factor(int a) const { return scale ? scale[a] : 1.f; }
};

// A or B of the adapters: element (a, line j, column c) at a * major + j * sj + c * sc
template <class T>
struct Thin {
  const T *p;
  int64_t major;
  int sj, sc;
};

// ---- fp32 values of k for one line, as operands, in P parts ----------------------------------------------------
template <class T, int P>
__device__ __forceinline__ void split_to(const float *v, u32x4 (&f)[P]) {
  if constexpr (sizeof(T) == 4) {
    f[0] = u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  } else {
    float rest[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) rest[j] = v[j];
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t lo = narrow<bf16_t>(rest[2 * j]), hi = narrow<bf16_t>(rest[2 * j + 1]);
        f[p][j] = lo | hi << 16;
        rest[2 * j] = left_of(rest[2 * j], lo);
        rest[2 * j + 1] = left_of(rest[2 * j + 1], hi);
      }
    }
  }
}
template <class T>
struct PartsOf {
  static constexpr int Out = sizeof(T) == 4 ? 1 : 2;   // into a result of type T
  static constexpr int Grad = sizeof(T) == 4 ? 1 : 3;  // into an fp32 gradient
};

// The rank lines of every row: [splits][rows][ld] fp32, ld a multiple of 8, summed over the splits (in their order) where they
// are used.  Lines past an adapter's rank are 0 up to the next multiple of 8; rows without an adapter hold anything.
struct Lines {
  float *p;
  int splits, ld;
  int64_t stride;  // rows * ld
  __device__ __forceinline__ float at(int64_t i) const {
    float v = p[i];
    for (int s = 1; s < splits; s += 4) {  // (four loads at a time: one by one each would wait for the last)
      float w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) w[u] = s + u < splits ? p[(s + u) * stride + i] : 0.f;
      v += (w[0] + w[1]) + (w[2] + w[3]);
    }
    return v;
  }
};

// VE rank lines of one column of the thin operand from line j on.  No branch, so that loads do not wait for each other: what is not
// there is loaded from where something is, and cut off where it is used.
template <class T>
__device__ __forceinline__ u32x4 thin_k(const Thin<T> &m, int a, int o, int j, int lines) {
  constexpr int VE = VecOf<T>::N;
  const T *p = m.p + a * m.major + (int64_t)o * m.sc;
  if (m.sj == 1 && m.sc % VE == 0) return *reinterpret_cast<const u32x4_any *>(p + min(j, m.sc - VE));  // (sc: the rank of all)
  uint32_t e[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) e[i] = bits_of(p[(int64_t)max(min(j + i, lines - 1), 0) * m.sj]);
  if constexpr (sizeof(T) == 4) return u32x4{e[0], e[1], e[2], e[3]};
  else return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}
// those past `lines` 0
template <class T>
__device__ __forceinline__ u32x4 cut_k(u32x4 v, int j, int lines) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) v[i] = j + i < lines ? v[i] : 0u;
    else v[i] = j + 2 * i + 1 < lines ? v[i] : j + 2 * i < lines ? v[i] & 0xffffu : 0u;
  }
  return v;
}

// One projection: y[t, o] = sum_k x[t, k] w(o, k) + sum_j m(a, j, o) h[t, j], w(o, k) at o * wo + k * wk (one of them is 1).
template <class T>
struct Project {
  const T *x;
  int64_t ldx, rows;
  int width, outs;
  const T *w;
  int64_t wo, wk;
  Low low;
  Thin<T> m;
  Lines h;
  T *y;
  int64_t ldy;
};

// The lines of N rows from t0 on to LDS by a workgroup, as operands: [N][P][ld], bf16 in P = 2 parts; room(row): where a row's are.
// Those past an adapter's rank, and of rows without an adapter, 0.
template <class T, int N, class F>
__device__ __forceinline__ void gather_lines(const Low &low, const Lines &h, F room, int64_t t0, int64_t rows) {
  const int pieces = h.ld / 4;
  const int64_t step = h.stride >> 2;
#pragma unroll 2
  for (int i = threadIdx.x; i < N * pieces; i += 256) {
    const int row = i / pieces, c = i - row * pieces;
    const int64_t t = min(t0 + row, rows - 1);
    const int id = low.of(t);
    const float4 *q = reinterpret_cast<const float4 *>(h.p + t * h.ld) + c;
    float4 v = q[0];
    for (int s = 1; s < h.splits; s += 7) {
      float4 w[7];
#pragma unroll
      for (int u = 0; u < 7; ++u) w[u] = q[min(s + u, h.splits - 1) * step];
#pragma unroll
      for (int u = 0; u < 7; ++u)
        if (s + u < h.splits) v = make_float4(v.x + w[u].x, v.y + w[u].y, v.z + w[u].z, v.w + w[u].w);
    }
    const int left = (id >= 0 ? low.lines(id) : 0) - c * 4;
    v = make_float4(left > 0 ? v.x : 0.f, left > 1 ? v.y : 0.f, left > 2 ? v.z : 0.f, left > 3 ? v.w : 0.f);
    if constexpr (sizeof(T) == 4) {
      *reinterpret_cast<float4 *>(room(row) + c * 4) = v;
    } else {
      const float e[8] = {v.x, v.y, v.z, v.w};
      u32x4 f[2];
      split_to<T, 2>(e, f);
#pragma unroll
      for (int part = 0; part < 2; ++part) *reinterpret_cast<uint2 *>(room(row) + part * h.ld + c * 4) = make_uint2(f[part][0], f[part][1]);
    }
  }
}

// acc += the rank lines' product for 32 R rows from t0 on and 32 E outputs, o of each lane; lines_of(r): the lines of the r-th 32 rows
// in LDS (gather_lines).  ROWS: rows are the first operand (the lines of a result), outputs the second; else the other way round.
// Of each adapter among the rows J steps of lines at a time, the next ones' operands on their way meanwhile; of the distinct adapters
// every turn-th from the first-th on.  The lines of rows with other adapters are replaced by zeros, except where an adapter holds
// infinities or NaN (a product of its operands with zeros tells): its sums are made apart then, and rows take none but their own.
// (With all sums apart, and the lines of each 32 rows by themselves: 8192 rows, 4096 -> 4096, 8 adapters of rank 32 in runs took a
// tenth longer.  With the additions for operands that are not finite in the one loop, whose results then moved between the
// registers of the vector unit and of the matrix cores: 4096 rows, 4096 -> 4096, 24 adapters in mixed order 244 us instead of 195.
// In that loop 256 x 256 tiles run out of registers and spill; the others do not.)
template <class T, int E, int R, bool ROWS, int J, class F>
__device__ __forceinline__ void add_thin(const Low &low, const Thin<T> &m, int ld, F lines_of, int64_t rows, int outs, int64_t t0,
                                         const int (&o)[E], f32x16 (&acc)[E][R], int first = 0, int turn = 1) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, P = PartsOf<T>::Out;
  const int ln = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
  int id[R];
  uint32_t rest[R];
#pragma unroll
  for (int r = 0; r < R; ++r) id[r] = low.of(min(t0 + r * 32 + ln, rows - 1));
#pragma unroll
  for (int r = 0; r < R; ++r) {
    if (t0 + r * 32 + ln >= rows) id[r] = -1;
    rest[r] = (uint32_t)__ballot(id[r] >= 0);
  }
  auto front = [&] {
    int a = -1;
#pragma unroll
    for (int r = R - 1; r >= 0; --r)
      if (rest[r] != 0) a = __builtin_amdgcn_readlane(id[r], __builtin_ctz(rest[r]));
    return a;
  };
  auto pass = [&](int n) {
    for (; n > 0; --n) {
      const int a = front();
#pragma unroll
      for (int r = 0; r < R; ++r) rest[r] &= ~(uint32_t)__ballot(id[r] == a);
    }
  };
  const u32x4 zeros = {0, 0, 0, 0};
  // (one e at a time, all of a row's steps)
  auto product = [&](auto apart, const T *h, int j, const u32x4 &mf, bool mine, f32x16 c) {
    u32x4 hf[P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
      const u32x4 v = *reinterpret_cast<const u32x4 *>(h + (ln * P + q) * ld + min(j, ld - VE));
      hf[q] = mine && j < ld ? v : zeros;
    }
#pragma unroll
    for (int q = P - 1; q >= 0; --q) {
      u32x4 m = mf;
      if constexpr (apart && P > 1) {
        if (q > 0) {
          asm volatile("" : "+v"(m));  // (made where it is used: kept for all rows' products, it would cost registers of the loop above)
          m = finite_of(m);
        }
      }
      c = ROWS ? mma<T>(hf[q], m, c) : mma<T>(m, hf[q], c);
    }
    return c;
  };
  u32x4 mf[J][E];
#pragma unroll
  for (int s = 0; s < J; ++s)
#pragma unroll
    for (int e = 0; e < E; ++e) mf[s][e] = zeros;
  // NaN if any of J steps' operands are not finite
  auto checked = [&](const u32x4 (&f)[J][E]) {
    f32x16 none = {};
#pragma unroll
    for (int s = 0; s < J; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) {  // (four instructions of the vector unit, not four of the matrix cores)
#pragma unroll
          for (int i = 0; i < 4; ++i) none[0] = fmaf(__uint_as_float(f[s][e][i]), 0.f, none[0]);
        } else if (s == 0 || s * KS < low.rank) {
          none = mma<T>(zeros, f[s][e], none);
        }
      }
    return __ballot(none[0] != 0.f) != 0;
  };
  pass(first);
  int a = -2, lines = 0, j0 = 0;  // (none yet: the first round only loads)
  bool apart = false, some_apart = false;
  while (a != -1) {
    int next = a, next_lines = lines, next_j = j0 + J * KS;
    if (next_j >= lines) {
      next = front(), next_lines = next >= 0 ? low.lines(next) : 0, next_j = 0;
      pass(turn);
    }
    u32x4 nf[J][E];
#pragma unroll
    for (int s = 0; s < J; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e)
        nf[s][e] = s == 0 || s * KS < low.rank ? thin_k(m, max(next, 0), min(o[e], outs - 1), next_j + s * KS + half * VE, next_lines) : zeros;
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (a < 0) break;
      const bool mine = id[r] == a && !apart;  // (a line may be infinite, and its product with the zeros NaN)
      const T *h = lines_of(r);
#pragma unroll
      for (int s = 0; s < J; ++s)
        if (s == 0 || s * KS < low.rank)
#pragma unroll
          for (int e = 0; e < E; ++e) acc[e][r] = product(std::false_type{}, h, j0 + s * KS + half * VE, mf[s][e], mine, acc[e][r]);
    }
    a = next, lines = next_lines, j0 = next_j;
#pragma unroll
    for (int s = 0; s < J; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e) mf[s][e] = cut_k<T>(nf[s][e], j0 + s * KS + half * VE, lines);
    apart = checked(mf);
    if (apart) {
      some_apart = true;
#pragma unroll
      for (int s = 0; s < J; ++s)
#pragma unroll
        for (int e = 0; e < E; ++e) mf[s][e] = zeros;
    }
  }
  if (!some_apart) return;
  // (a loop of its own: the vector unit's additions in the loop above would keep the results out of the matrix cores' registers)
#pragma unroll
  for (int r = 0; r < R; ++r) rest[r] = (uint32_t)__ballot(id[r] >= 0);
  pass(first);
#pragma unroll 1
  for (a = front(); a != -1; a = front()) {
    lines = low.lines(a);
#pragma unroll 1
    for (j0 = 0; j0 < lines; j0 += J * KS) {
#pragma unroll
      for (int s = 0; s < J; ++s)
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const int j = j0 + s * KS + half * VE;
          mf[s][e] = cut_k<T>(thin_k(m, a, min(o[e], outs - 1), j, lines), j, lines);
        }
      if (!checked(mf)) continue;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const bool mine = id[r] == a;
        const uint32_t same = (uint32_t)__ballot(mine);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          f32x16 d = {};
#pragma unroll
          for (int s = 0; s < J; ++s) d = product(std::true_type{}, lines_of(r), j0 + s * KS + half * VE, mf[s][e], true, d);
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[e][r][i] += (ROWS ? (same >> result_line(i, half) & 1) != 0 : mine) ? d[i] : 0.f;
        }
      }
    }
    pass(turn);
  }
}

// ---- making the rank lines --------------------------------------------------------------------------------------
// h[t, j] = s_a sum_c m(a, j, c) x[t, c] for the rows of every adapter, in ranges of k.
// Up to 64 rows: a wave takes 32 of them, a range of k and, of the distinct adapters among the rows, every groups-th.
// More: a workgroup takes 128 rows and a range of k and brings the rows in the order of their adapters; its waves, and those of the
// `groups` workgroups that share the rows and the range, take 32 rows of one adapter at a time, so that rows in any order meet
// each adapter's lines once.
template <class T>
struct ThinJob {
  const T *x;
  int64_t ldx, rows;
  int width;
  Thin<T> m;
  Lines out;
  int chunk, groups;
  bool by_range;
  int64_t units, blocks;  // blocks of four waves; units: of waves, not by_range
};

constexpr int kRange = 128;
struct ThinLds {
  int4 key[kRange / 4];
  int row[kRange], of[kRange], head[kRange];
};
constexpr int kThinRoom = 8192;  // bytes of LDS of a wave: 32 rows and 32 lines by 128 bytes of k

// the sums over k0 .. k1 of 32 rows (of the lane: xr, at its half's chunk) with 32 lines (mr); CONT: sc = 1.  Eight steps' loads go
// out together.
template <class T, bool CONT>
__device__ __forceinline__ f32x16 thin_sums(const T *xr, const T *mr, int sc, int k0, int k1, int half) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, U = CONT ? 8 : 4;
  f32x16 acc = {};
  int k = k0;
  for (; k + KS * U <= k1; k += KS * U) {
    u32x4 xf[U], mf[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      xf[u] = *reinterpret_cast<const u32x4_any *>(xr + k + u * KS);
      if constexpr (CONT) mf[u] = *reinterpret_cast<const u32x4_any *>(mr + k + u * KS);
      else mf[u] = load_k_strided(mr + (int64_t)(k + u * KS) * sc, sc, VE);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) acc = mma<T>(xf[u], mf[u], acc);
  }
  for (; k < k1; k += KS) {
    const int left = k1 - k - half * VE;
    const u32x4 xf = load_k(xr + k, left);
    u32x4 mf;
    if constexpr (CONT) mf = load_k(mr + k, left);
    else mf = load_k_strided(mr + (int64_t)k * sc, sc, left);
    acc = mma<T>(xf, mf, acc);
  }
  return acc;
}

template <class T>
__device__ __forceinline__ void thin_unit(const ThinJob<T> &g, const Low &low, int64_t unit) {
  constexpr int VE = VecOf<T>::N;
  const int lane = threadIdx.x & 63, ln = lane & 31, half = lane >> 5;
  const int group = (int)(unit % g.groups), split = (int)(unit / g.groups % g.out.splits);
  const int64_t t0 = unit / g.groups / g.out.splits * 32, t = t0 + ln;
  const int id = t < g.rows ? low.of(t) : -1;
  const int k0 = split * g.chunk, k1 = min(g.width, k0 + g.chunk);
  const T *xr = g.x + min(t, g.rows - 1) * g.ldx + half * VE;
  float *out = g.out.p + split * g.out.stride + t0 * g.out.ld;
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
      const f32x16 acc = g.m.sc == 1 ? thin_sums<T, true>(xr, mr, 1, k0, k1, half) : thin_sums<T, false>(xr, mr, g.m.sc, k0, k1, half);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int row = result_line(i, half);
        if ((same >> row & 1) && j0 + ln < g.out.ld) out[(int64_t)row * g.out.ld + j0 + ln] = j0 + ln < lines ? acc[i] * f : 0.f;
      }
    }
  }
}

// The sums over k0 .. k1 of the 32 rows at xr (a lane's for each load: row 8 i + lane / 8) with 32 lines from j0 on, in stages of 128
// bytes of k through the wave's own LDS, the next stage's loads in flight meanwhile.  A load asks for whole lines of 128 bytes of
// eight rows; straight into operands, 32 bytes of 32 rows, 190 rows, 5232 -> 4072, rank 64 took 54 us (with the product) instead
// of 42.  Two stages ahead: no gain (45 us).
template <class T>
__device__ __forceinline__ f32x16 thin_stages(const ThinJob<T> &g, int a, int lines, int j0, const T *const (&xr)[4], int k0, int k1,
                                              unsigned char *own) {
  constexpr int VE = VecOf<T>::N, KB = kLine / (int)sizeof(T), PerK = 32 / VE;  // PerK: lanes of a line of k
  const int lane = thread_here() & 63, ln = lane & 31, half = lane >> 5;
  const int chunk = lane % kChunks, line = lane / kChunks;
  const bool cont = g.m.sc == 1, even = g.m.sc % VE == 0;  // even: (not cont) 16 bytes of lines from any of them on are there
  const T *mr = g.m.p + a * g.m.major;
  const T *ml[4];  // the lane's place of the loads of m
#pragma unroll
  for (int i = 0; i < 4; ++i)
    ml[i] = cont ? mr + (int64_t)min(j0 + i * 8 + line, lines - 1) * g.m.sj + chunk * VE
                 : mr + (int64_t)(i * (64 / PerK) + lane / PerK) * g.m.sc + (even ? min(j0 + lane % PerK * VE, g.m.sc - VE) : j0 + lane % PerK * VE);
  u32x4 st[8];
  auto load = [&](int k) {
    if (k + KB <= k1 && (cont || even)) {  // (nothing to check: no branch between the loads; lines past the adapter's are not used)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st[i] = *reinterpret_cast<const u32x4_any *>(xr[i] + k + chunk * VE);
        st[4 + i] = *reinterpret_cast<const u32x4_any *>(ml[i] + (int64_t)k * g.m.sc);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int left = k1 - k - chunk * VE;
      st[i] = load_k(xr[i] + k + chunk * VE, left);
      if (cont) st[4 + i] = load_k(ml[i] + k, left);
      else st[4 + i] = load_k(ml[i] + (int64_t)k * g.m.sc, k + i * (64 / PerK) + lane / PerK < k1 ? even ? VE : lines - j0 - lane % PerK * VE : 0);
    }
  };
  f32x16 acc = {};
  load(k0);
  for (int k = k0; k < k1; k += KB) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + line, at = row * kLine + ((chunk ^ chunk_key(row)) << 4);
      *reinterpret_cast<u32x4 *>(own + at) = st[i];
      *reinterpret_cast<u32x4 *>(own + 4096 + (cont ? at : i * 1024 + lane * 16)) = st[4 + i];
    }
    if (k + KB < k1) load(k + KB);
    // (LDS serves a wave in order; the compiler shall not turn it round)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    const unsigned char *ms = own + 4096;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 xf = chunk_of(own, ln, s * 2 + half);
      u32x4 mf;
      if (cont) {
        mf = chunk_of(ms, ln, s * 2 + half);
      } else if constexpr (sizeof(T) == 2) {
        const unsigned char *at = ms + (s * 16 + half * 8 + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
        const uint2 u = turned(at), v = turned(at + 4 * 64);
        mf = u32x4{u.x, u.y, v.x, v.y};
      } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) mf[q] = *reinterpret_cast<const uint32_t *>(ms + (s * 8 + half * 4 + q) * 128 + ln * 4);
      }
      acc = mma<T>(xf, mf, acc);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  return acc;
}

template <class T>
__device__ __forceinline__ void thin_range(const ThinJob<T> &g, const Low &low, int64_t block, ThinLds &lds, unsigned char *own) {
  constexpr int none = 0x7fffffff;
  const int tid = thread_here(), lane = tid & 63, ln = lane & 31, half = lane >> 5;
  const int split = (int)(block % g.out.splits), share = (int)(block / g.out.splits % g.groups);
  const int64_t base = block / g.out.splits / g.groups * kRange;
  if (tid < kRange) {
    const int id = base + tid < g.rows ? low.of(base + tid) : -1;
    reinterpret_cast<int *>(lds.key)[tid] = id < 0 ? none : id;
  }
  __syncthreads();
  if (tid < kRange) {
    const int key = reinterpret_cast<const int *>(lds.key)[tid];
    int less = 0, before = 0, equal = 0;
#pragma unroll 8
    for (int i = 0; i < kRange / 4; ++i) {
      const int4 k = lds.key[i];
      less += (k.x < key) + (k.y < key) + (k.z < key) + (k.w < key);
      equal += (k.x == key) + (k.y == key) + (k.z == key) + (k.w == key);
      before += (k.x == key && 4 * i < tid) + (k.y == key && 4 * i + 1 < tid) + (k.z == key && 4 * i + 2 < tid) + (k.w == key && 4 * i + 3 < tid);
    }
    lds.row[less + before] = tid;
    lds.of[less + before] = key;
    lds.head[less + before] = key != none && before % 32 == 0 ? min(equal - before, 32) : 0;
  }
  __syncthreads();
  const int k0 = split * g.chunk, k1 = min(g.width, k0 + g.chunk);
  // (the heads, in the order of the rows, go round the waves of all workgroups that share the range)
  const int first = share * 4 + __builtin_amdgcn_readfirstlane(tid >> 6), turn = 4 * g.groups;
  int nth = 0;
  for (int pos = 0, n; pos < kRange; pos += n) {
    n = __builtin_amdgcn_readfirstlane(lds.head[pos]);
    if (n == 0) break;  // rows without an adapter come last
    if (nth++ % turn != first) continue;
    const int a = __builtin_amdgcn_readfirstlane(lds.of[pos]);
    const int lines = low.lines(a);
    const float f = low.factor(a);
    float *out = g.out.p + split * g.out.stride + base * g.out.ld;
    for (int j0 = 0; j0 < lines; j0 += 32) {
      const T *xr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) xr[i] = g.x + (base + lds.row[pos + min(i * 8 + lane / kChunks, n - 1)]) * g.ldx;
      const f32x16 acc = thin_stages<T>(g, a, lines, j0, xr, k0, k1, own);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int q = result_line(i, half);
        if (q < n && j0 + ln < g.out.ld) out[(int64_t)lds.row[pos + q] * g.out.ld + j0 + ln] = j0 + ln < lines ? acc[i] * f : 0.f;
      }
    }
  }
}

// a workgroup of four waves; `own`: the wave's LDS, of kThinRoom bytes (by_range)
template <class T>
__device__ __forceinline__ void thin_block(const ThinJob<T> &g, const Low &low, int64_t block, ThinLds &lds, unsigned char *own) {
  if (g.by_range) return thin_range<T>(g, low, block, lds, own);
  const int64_t unit = block * 4 + (threadIdx.x >> 6);
  if (unit < g.units) thin_unit<T>(g, low, unit);
}

// adapter_tile.hip: anything.  Ranges of k; with more than one, their sums go to part [splits][rows][outs], and the rank lines of one
// or two jobs are made beside.
constexpr int kPlaces = 512;  // workgroups of tiles that a card of 256 compute units holds at once
int64_t tiles_of(int64_t rows, int outs);
int tile_splits(int64_t rows, int width, int outs, int size);
template <class T>
void launch_tiles(const Project<T> &p, int splits, float *part, const ThinJob<T> &thin, const ThinJob<T> &other, hipStream_t s);
// adapter_gemm.hip: rows that 16-byte loads can take
bool gemm_takes(const Project<bf16_t> &p);
int gemm_splits(int64_t rows, int width, int outs);  // ranges of k; 1: whole tiles
void launch_gemm(const Project<bf16_t> &p, hipStream_t s);
// the ranges' sums to part [splits][rows][outs], and the rank lines of one or two jobs beside
void launch_gemm_split(const Project<bf16_t> &p, int splits, float *part, const ThinJob<bf16_t> &thin, const ThinJob<bf16_t> &other,
                       hipStream_t s);

}  // namespace wcc

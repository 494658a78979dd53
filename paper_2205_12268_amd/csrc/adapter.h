// The projection with adapters: what its translation units share.
//
// A product here has k running over the width of the rows it reads.  Its operands meet in 32 x 32 tiles of the matrix cores:
// lane l of a wave has line l % 32 of an operand and 16 bytes of k, the first half of the lanes the first 16 of 32 bytes.  For
// bf16 that is one v_mfma_f32_32x32x16_bf16, for fp32 four v_mfma_f32_32x32x2_f32 (both operands take k in the same order,
// which is all that matters).
#pragma once

#include "head.h"
#include "rows.h"

namespace wcc {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));

template <class T>
__device__ __forceinline__ f32x16 mma(const u32x4 &a, const u32x4 &b, f32x16 c);
template <>
__device__ __forceinline__ f32x16 mma<bf16_t>(const u32x4 &a, const u32x4 &b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ f32x16 mma<float>(const u32x4 &a, const u32x4 &b, f32x16 c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a[i]), __uint_as_float(b[i]), c, 0, 0, 0);
  return c;
}
// line of the first operand that register i of a result belongs to, for the lane's half (lane / 32); the second's is lane % 32
__device__ __forceinline__ int result_line(int i, int half) { return (i >> 2) * 8 + half * 4 + (i & 3); }

// k of one mma
template <class T>
struct StepOf {
  static constexpr int K = 32 / (int)sizeof(T);
};

// ---- straight from memory to LDS: 16 bytes a lane to 1 KiB in a row --------------------------------------------
__device__ const uint4 kZeros = {0, 0, 0, 0};  // where chunks come from that are not there

__device__ __forceinline__ void to_lds(const void *from, unsigned char *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}
// Lines of 64 k (128 bytes) without padding: chunk c of line `line` lies at chunk c ^ chunk_key(line), which spreads the 16 lines of a
// read over all banks.
constexpr int kK = 64, kLine = 2 * kK, kChunks = kK / 8;
__device__ __forceinline__ int chunk_key(int line) { return (line >> 1) & 7; }
__device__ __forceinline__ u32x4 chunk_of(const unsigned char *s, int line, int chunk) {
  return *reinterpret_cast<const u32x4 *>(s + line * kLine + ((chunk ^ chunk_key(line)) << 4));
}
// Four bf16 of k from LDS lines of k: within 16 lanes, lane 4j + q supplies four neighbours of line k + j, and lane 4q + e receives
// the e-th of them for j = 0..3.
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
__device__ __forceinline__ uint2 turned(const unsigned char *at) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                                       (__attribute__((address_space(3))) bf16x4 *)(__attribute__((address_space(3))) void *)at));
}

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

// ---- 16 bytes of k of one line -------------------------------------------------------------------------------
// `left` elements are there (any number; <= 0: none), the rest is 0; consecutive k are `sk` elements apart.
template <class T>
__device__ __forceinline__ u32x4 load_k_strided(const T *p, int64_t sk, int left) {
  constexpr int VE = VecOf<T>::N;
  uint32_t e[VE];
#pragma unroll
  for (int j = 0; j < VE; ++j) e[j] = j < left ? bits_of(p[j * sk]) : 0u;
  if constexpr (sizeof(T) == 4) return u32x4{e[0], e[1], e[2], e[3]};
  else return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
}
// the same where they are neighbours
template <class T>
__device__ __forceinline__ u32x4 load_k(const T *p, int left) {
  constexpr int VE = VecOf<T>::N;
  if (left >= VE) return *reinterpret_cast<const u32x4_any *>(p);
  return load_k_strided(p, 1, left);
}
// Two neighbouring lines at once where lines are contiguous and k is not: (line, line + 1) of each k is one load, the halves of
// which go to the two lines.  `both`: the second line is there (it may be the end of memory).
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef uint64_t u64_any __attribute__((aligned(4)));
template <class T>
__device__ __forceinline__ void load_k_pair(const T *p, int64_t sk, int left, bool both, u32x4 &f0, u32x4 &f1) {
  constexpr int VE = VecOf<T>::N;
  if constexpr (sizeof(T) == 4) {
    uint64_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j)
      v[j] = j < left ? both ? *reinterpret_cast<const u64_any *>(p + j * sk) : (uint64_t)__float_as_uint(p[j * sk]) : 0;
    f0 = u32x4{(uint32_t)v[0], (uint32_t)v[1], (uint32_t)v[2], (uint32_t)v[3]};
    f1 = u32x4{(uint32_t)(v[0] >> 32), (uint32_t)(v[1] >> 32), (uint32_t)(v[2] >> 32), (uint32_t)(v[3] >> 32)};
  } else {
    uint32_t v[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) v[j] = j < left ? both ? *reinterpret_cast<const u32_any *>(p + j * sk) : (uint32_t)p[j * sk] : 0u;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f0[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x05040100);
      f1[j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x07060302);
    }
  }
}

// ---- fp32 values of k for one line, as operands ---------------------------------------------------------------
// bf16 operands carry 8 bits each: P of them take P * 8 bits of the values, the rest of each going to the next.
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
        rest[2 * j] -= __uint_as_float(lo << 16);
        rest[2 * j + 1] -= __uint_as_float(hi << 16);
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
  // eight lines from j (a multiple of 8) on
  __device__ __forceinline__ void eight(int64_t t, int j, float (&v)[8]) const {
    const float4 *q = reinterpret_cast<const float4 *>(p + t * ld + j);
    float4 a = q[0], b = q[1];
    auto add = [](const float4 &u, const float4 &w) { return make_float4(u.x + w.x, u.y + w.y, u.z + w.z, u.w + w.w); };
    const int64_t step = stride >> 2;
    int s = 1;
    for (; s + 1 < splits; s += 2) {  // (the order of the splits; two at a time so that loads do not wait for each other)
      const float4 c0 = q[s * step], d0 = q[s * step + 1], c1 = q[(s + 1) * step], d1 = q[(s + 1) * step + 1];
      a = add(add(a, c0), c1), b = add(add(b, d0), d1);
    }
    if (s < splits) a = add(a, q[s * step]), b = add(b, q[s * step + 1]);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  }
};

// VE rank lines of one column of the thin operand from line j on, `left` > 0 of them there.  What is past them repeats the last one
// and meets zeros of h.
template <class T>
__device__ __forceinline__ u32x4 thin_k(const Thin<T> &m, int a, int o, int j, int left) {
  constexpr int VE = VecOf<T>::N;
  const T *p = m.p + a * m.major + (int64_t)o * m.sc + (int64_t)j * m.sj;
  if (m.sj == 1 && left >= VE) return *reinterpret_cast<const u32x4_any *>(p);
  uint32_t e[VE];
#pragma unroll
  for (int i = 0; i < VE; ++i) e[i] = bits_of(p[(int64_t)min(i, left - 1) * m.sj]);
  if constexpr (sizeof(T) == 4) return u32x4{e[0], e[1], e[2], e[3]};
  else return u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
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

// acc += the rank lines' product for the 32 rows from t0 on and 32 E outputs, o of each lane.  ROWS: rows are the first operand (the
// lines of a result), outputs the second; else the other way round.  The sums of each adapter among the rows apart: a row takes
// its own, whatever (infinities, NaN) other adapters hold.  A row's lines meet no adapter but its own, so they are loaded once; the
// next adapter's operands are on their way while one's are multiplied.
template <class T, int E, bool ROWS>
__device__ __forceinline__ void add_thin(const Low &low, const Thin<T> &m, const Lines &h, int64_t rows, int outs, int64_t t0,
                                         const int (&o)[E], f32x16 (&acc)[E]) {
  constexpr int VE = VecOf<T>::N, KS = StepOf<T>::K, P = PartsOf<T>::Out, J = 2;  // J steps of lines are held
  const int ln = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
  const int64_t t = min(t0 + ln, rows - 1);
  const int id = t0 + ln < rows ? low.of(t) : -1;
  const int mine = id >= 0 ? low.lines(id) : 0;
  auto own_lines = [&](int j0, u32x4 (&hf)[P]) {
    const int j = j0 + half * VE;
    float hv[8] = {};
    if (j < mine) h.eight(t, j & ~7, hv);
    if constexpr (VE == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) hv[i] = half ? hv[4 + i] : hv[i];
    }
    split_to<T, P>(hv, hf);
  };
  auto operands = [&](int a, int lines, int j0, u32x4 (&mf)[E]) {
    const int j = j0 + half * VE;
#pragma unroll
    for (int e = 0; e < E; ++e) mf[e] = j < lines ? thin_k(m, a, min(o[e], outs - 1), j, lines - j) : u32x4{0, 0, 0, 0};
  };
  auto product = [&](const u32x4 (&hf)[P], const u32x4 (&mf)[E], f32x16 (&d)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int q = P - 1; q >= 0; --q) d[e] = ROWS ? mma<T>(hf[q], mf[e], d[e]) : mma<T>(mf[e], hf[q], d[e]);
  };
  uint32_t rest = (uint32_t)__ballot(id >= 0);
  u32x4 hf[J][P], mf[J][E];
#pragma unroll
  for (int s = 0; s < J; ++s) {
    own_lines(s * KS, hf[s]);
#pragma unroll
    for (int e = 0; e < E; ++e) mf[s][e] = u32x4{0, 0, 0, 0};
  }
  int a = -2, lines = 0;  // (none yet: the first round only loads)
  while (a != -1) {
    const int next = rest != 0 ? __builtin_amdgcn_readlane(id, __builtin_ctz(rest)) : -1;
    const int next_lines = next >= 0 ? low.lines(next) : 0;
    u32x4 nf[J][E];
#pragma unroll
    for (int s = 0; s < J; ++s) operands(next, next_lines, s * KS, nf[s]);
    f32x16 d[E] = {};
#pragma unroll
    for (int s = 0; s < J; ++s) product(hf[s], mf[s], d);
    for (int j0 = J * KS; j0 < lines; j0 += KS) {
      u32x4 hj[P], mj[E];
      own_lines(j0, hj);
      operands(a, lines, j0, mj);
      product(hj, mj, d);
    }
    const uint32_t same = (uint32_t)__ballot(id == a);
#pragma unroll
    for (int e = 0; e < E; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[e][i] += (ROWS ? (same >> result_line(i, half) & 1) != 0 : id == a) ? d[e][i] : 0.f;
    a = next, lines = next_lines;
    rest &= ~(uint32_t)__ballot(id == a);
#pragma unroll
    for (int s = 0; s < J; ++s)
#pragma unroll
      for (int e = 0; e < E; ++e) mf[s][e] = nf[s][e];
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
  bool by_range, through_lds;  // through_lds: by_range, bf16, and all of x and m in whole chunks of 16 bytes
  int64_t units, blocks;  // blocks of four waves; units: of waves, not by_range
};

constexpr int kRange = 128;
struct ThinLds {
  int4 key[kRange / 4];
  int row[kRange], of[kRange], head[kRange];
};
// two stages of x and of m, 4 KiB a wave each
struct ThinStages {
  unsigned char *x0, *m0, *x1, *m1;
};

// the sums over k0 .. k1 of 32 rows (of the lane: xr, at its half's chunk) with 32 lines (mr); CONT: sc = 1.  Eight steps' loads go
// out together: with four, and the next four on their way meanwhile, 128 rows x 512 k a workgroup took 50 us where these take 38.
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

// The sums over k0 .. k1 of the 32 rows at xr (a lane's for each load: row 8 i + lane / 8) with 32 lines from j0 on, in stages of 64 k
// through the wave's own LDS.  Straight into registers, 32 rows x 32 bytes at a time, four loads in a row ask for the same lines
// of memory, and wait for each other's: 8192 rows x 4096 k took 38 us.
__device__ __forceinline__ f32x16 thin_stages(const ThinJob<bf16_t> &g, int a, int lines, int j0, const bf16_t *const (&xr)[4], int k0,
                                              int k1, const ThinStages &st) {
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, half = lane >> 5;
  const bool cont = g.m.sc == 1;
  const bf16_t *mr = g.m.p + a * g.m.major;
  auto load = [&](int k, unsigned char *xs, unsigned char *ms) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 8 + lane / kChunks, c = ((lane % kChunks) ^ chunk_key(row)) * 8;
      to_lds(k + c < k1 ? (const void *)(xr[i] + k + c) : &kZeros, xs + wv * 4096 + i * 1024);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const void *at = &kZeros;
      if (cont) {
        const int row = i * 8 + lane / kChunks, c = ((lane % kChunks) ^ chunk_key(row)) * 8;
        if (k + c < k1) at = mr + (int64_t)min(j0 + row, lines - 1) * g.m.sj + k + c;
      } else {  // lines of k of 32 neighbours
        const int kk = k + i * 16 + lane / 4, j = j0 + lane % 4 * 8;
        if (kk < k1 && j < lines) at = mr + (int64_t)kk * g.m.sc + j;
      }
      to_lds(at, ms + wv * 4096 + i * 1024);
    }
  };
  f32x16 acc = {};
  auto add = [&](const unsigned char *xs, const unsigned char *ms) {
    xs += wv * 4096, ms += wv * 4096;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const u32x4 xf = chunk_of(xs, ln, s * 2 + half);
      u32x4 mf;
      if (cont) {
        mf = chunk_of(ms, ln, s * 2 + half);
      } else {
        const unsigned char *at = ms + (s * 16 + half * 8 + ((lane & 15) >> 2)) * 64 + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
        const uint2 u = turned(at), v = turned(at + 4 * 64);
        mf = u32x4{u.x, u.y, v.x, v.y};
      }
      acc = mma<bf16_t>(xf, mf, acc);
    }
  };
  load(k0, st.x0, st.m0);
  for (int k = k0; k < k1; k += 2 * kK) {  // (stages past the end are zeros)
    load(k + kK, st.x1, st.m1);
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    add(st.x0, st.m0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load(k + 2 * kK, st.x0, st.m0);
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
    add(st.x1, st.m1);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  return acc;
}

template <class T>
__device__ __forceinline__ void thin_range(const ThinJob<T> &g, const Low &low, int64_t block, ThinLds &lds, const ThinStages &st) {
  constexpr int VE = VecOf<T>::N, none = 0x7fffffff;
  const int tid = threadIdx.x, lane = tid & 63, ln = lane & 31, half = lane >> 5;
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
      f32x16 acc;
      bool done = false;
      if constexpr (sizeof(T) == 2) {
        if (g.through_lds) {
          const bf16_t *xr[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) xr[i] = g.x + (base + lds.row[pos + min(i * 8 + lane / kChunks, n - 1)]) * g.ldx;
          acc = thin_stages(g, a, lines, j0, xr, k0, k1, st);
          done = true;
        }
      }
      if (!done) {
        const T *xr = g.x + (base + lds.row[pos + min(ln, n - 1)]) * g.ldx + half * VE;
        const T *mr = g.m.p + a * g.m.major + (int64_t)min(j0 + ln, lines - 1) * g.m.sj + (int64_t)(half * VE) * g.m.sc;
        acc = g.m.sc == 1 ? thin_sums<T, true>(xr, mr, 1, k0, k1, half) : thin_sums<T, false>(xr, mr, g.m.sc, k0, k1, half);
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int q = result_line(i, half);
        if (q < n && j0 + ln < g.out.ld) out[(int64_t)lds.row[pos + q] * g.out.ld + j0 + ln] = j0 + ln < lines ? acc[i] * f : 0.f;
      }
    }
  }
}

// a workgroup of four waves
template <class T>
__device__ __forceinline__ void thin_block(const ThinJob<T> &g, const Low &low, int64_t block, ThinLds &lds, const ThinStages &st) {
  if (g.by_range) return thin_range<T>(g, low, block, lds, st);
  const int64_t unit = block * 4 + (threadIdx.x >> 6);
  if (unit < g.units) thin_unit<T>(g, low, unit);
}

template <class T>
void launch_tiles(const Project<T> &p, hipStream_t s);  // adapter_tile.hip: anything
// adapter_gemm.hip: rows that 16-byte loads can take
bool gemm_takes(const Project<bf16_t> &p);
int gemm_splits(int64_t rows, int width, int outs);  // ranges of k; 1: whole tiles
void launch_gemm(const Project<bf16_t> &p, hipStream_t s);
// the ranges' sums to part [splits][rows][outs], and the rank lines of one or two jobs beside
void launch_gemm_split(const Project<bf16_t> &p, int splits, float *part, const ThinJob<bf16_t> &thin, const ThinJob<bf16_t> &other,
                       hipStream_t s);

}  // namespace wcc

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
// `left` elements are there (any number; <= 0: none), the rest is 0.
template <class T>
__device__ __forceinline__ u32x4 load_k(const T *p, int left) {
  constexpr int VE = VecOf<T>::N;
  if (left >= VE) return *reinterpret_cast<const u32x4_any *>(p);
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < VE - 1; ++j)
    if (j < left) {
      if constexpr (sizeof(T) == 4) v[j] = __float_as_uint(p[j]);
      else v[j >> 1] |= (uint32_t)p[j] << (16 * (j & 1));
    }
  return v;
}
// the same where consecutive k are `sk` elements apart
template <class T>
__device__ __forceinline__ u32x4 load_k_strided(const T *p, int64_t sk, int left) {
  constexpr int VE = VecOf<T>::N;
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < VE; ++j)
    if (j < left) {
      if constexpr (sizeof(T) == 4) v[j] = __float_as_uint(p[j * sk]);
      else v[j >> 1] |= (uint32_t)p[j * sk] << (16 * (j & 1));
    }
  return v;
}
// Two neighbouring lines at once where lines are contiguous and k is not: (line, line + 1) of each k is one load, the halves of
// which go to the two lines.  `both`: the second line is there (it may be the end of memory).
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef uint64_t u64_any __attribute__((aligned(4)));
template <class T>
__device__ __forceinline__ void load_k_pair(const T *p, int64_t sk, int left, bool both, u32x4 &f0, u32x4 &f1) {
  constexpr int VE = VecOf<T>::N;
  f0 = f1 = u32x4{0, 0, 0, 0};
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int j = 0; j < VE; ++j)
      if (j < left) {
        if (both) {
          const uint64_t v = *reinterpret_cast<const u64_any *>(p + j * sk);
          f0[j] = (uint32_t)v, f1[j] = (uint32_t)(v >> 32);
        } else {
          f0[j] = __float_as_uint(p[j * sk]);
        }
      }
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

// The rank lines of every row: [splits][rows][rank] fp32, summed over the splits (in their order) where they are used.
struct Lines {
  float *p;
  int splits;
  int64_t stride;  // rows * rank
  __device__ __forceinline__ float at(int64_t i) const {
    float v = p[i];
    for (int s = 1; s < splits; ++s) v += p[s * stride + i];
    return v;
  }
};

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

template <class T>
hipError_t launch_tiles(const Project<T> &p, hipStream_t s);

}  // namespace wcc

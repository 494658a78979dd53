// Rows of logits held in the registers of a workgroup: loading, storing, reductions.
//
// A slice of a row is NT threads times NV vectors of 16 bytes.  Vector i of thread t begins at element (i * NT + t) * VE of the
// slice, so that a wave reads 1 KiB in one instruction.  Rows begin at any element (odd widths and strides), which costs the
// vector loads no more than a cache line at each end; elements past the slice's end are -inf and are never stored.
#pragma once

#include "head.h"

namespace wcc {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // at any element of a row

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;

template <class T>
struct VecOf {
  static constexpr int N = 16 / (int)sizeof(T);
};

__device__ __forceinline__ uint32_t bits_of(bf16_t v) { return v; }
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }

// element j of a vector, as fp32
template <class T>
__device__ __forceinline__ float elem(const u32x4 &v, int j);
template <>
__device__ __forceinline__ float elem<float>(const u32x4 &v, int j) { return __uint_as_float(v[j]); }
template <>
__device__ __forceinline__ float elem<bf16_t>(const u32x4 &v, int j) {
  return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
}

template <class T>
__device__ __forceinline__ u32x4 pack(const float *f);
template <>
__device__ __forceinline__ u32x4 pack<float>(const float *f) {
  return u32x4{__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])};
}
template <>
__device__ __forceinline__ u32x4 pack<bf16_t>(const float *f) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (uint32_t)narrow<bf16_t>(f[2 * i]) | (uint32_t)narrow<bf16_t>(f[2 * i + 1]) << 16;
  return v;
}

// The thread's number, computed anew where it is called: without, the offsets of all vectors are made before the loop over the
// rows and take more registers than the row.
__device__ __forceinline__ int thread_here() {
  int t = (int)threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// n elements from p on into the registers, the rest -inf
template <class T, int NT, int NV>
__device__ __forceinline__ void load_slice(const T *p, int n, u32x4 (&v)[NV]) {
  constexpr int VE = VecOf<T>::N;
  constexpr uint32_t none = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  const int tid = thread_here();
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (i * NT + tid) * VE;
    if (e + VE <= n) v[i] = *reinterpret_cast<const u32x4_any *>(p + e);
    else v[i] = u32x4{none, none, none, none};
  }
  // the one vector that the end cuts
  const int last = n / VE;
  if (n % VE != 0 && last % NT == tid) {
    u32x4 c = {none, none, none, none};
#pragma unroll
    for (int j = 0; j < VE - 1; ++j)
      if (last * VE + j < n) {
        const uint32_t b = bits_of(p[last * VE + j]);
        if constexpr (sizeof(T) == 4) c[j] = b;
        else c[j >> 1] = j & 1 ? (c[j >> 1] & 0xffffu) | b << 16 : (c[j >> 1] & 0xffff0000u) | b;
      }
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (i == last / NT) v[i] = c;
  }
}

// The vectors as they are: what has been widened of them is not kept (it would take twice the registers of bf16 rows).
template <int NV>
__device__ __forceinline__ void hold(u32x4 (&v)[NV]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(v[i]));
}

// n elements of a slice to p: the vectors f(i) in order, i from 0 on.
template <class T, int NT, int NV, class F>
__device__ __forceinline__ void store_slice(T *p, int n, F f) {
  constexpr int VE = VecOf<T>::N;
  const int tid = thread_here();
  u32x4 cut = {};
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const u32x4 v = f(i);
    const int e = (i * NT + tid) * VE;
    if (e + VE <= n) *reinterpret_cast<u32x4_any *>(p + e) = v;
    if (i == n / VE / NT) cut = v;
    __builtin_amdgcn_sched_barrier(0);  // (interleaved, the results would not fit beside the row)
  }
  const int last = n / VE;
  if (n % VE != 0 && last % NT == tid) {
#pragma unroll
    for (int j = 0; j < VE - 1; ++j)
      if (last * VE + j < n) {
        if constexpr (sizeof(T) == 4) p[last * VE + j] = __uint_as_float(cut[j]);
        else p[last * VE + j] = (bf16_t)(cut[j >> 1] >> (16 * (j & 1)));
      }
  }
}

// ---- reductions over a workgroup; every thread gets the result ----------------------------------------------
struct Larger {
  __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
// (NaN if one of them is)
__device__ __forceinline__ float largest_of(float a, float b) { return __builtin_elementwise_maximum(a, b); }
struct Largest {
  __device__ __forceinline__ float operator()(float a, float b) const { return largest_of(a, b); }
};
struct Sum {
  __device__ __forceinline__ float operator()(float a, float b) const { return a + b; }
};
template <class Op>
__device__ __forceinline__ float wave_all(float v, Op op) {
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off, 64));
  return v;
}
// part: NT / 64 floats of LDS that nobody else uses until the next barrier but one
template <int NT, class Op>
__device__ __forceinline__ float block_all(float v, float *part, Op op) {
  v = wave_all(v, op);
  if constexpr (NT > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v = op(v, part[i]);
  }
  return v;
}

// How rows of V elements are cut: `slices` of `length` elements each (the last shorter), NT and NV of the kernels.
struct SlicePlan {
  int slices, length, nt, nv;
};

}  // namespace wcc

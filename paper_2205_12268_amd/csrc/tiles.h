// Products of rows on the matrix cores: what the translation units of the projection with adapters and of the gated block share.
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

// ---- fp32 values as operands of bf16 ---------------------------------------------------------------------------
// bf16 operands carry 8 bits each: P of them take P * 8 bits of the values, the rest of each going to the next.
__device__ __forceinline__ float left_of(float v, uint32_t part) {  // (nothing of an infinity, or it would be NaN)
  return (part & 0x7f80) == 0x7f80 ? 0.f : v - __uint_as_float(part << 16);
}
// bf16 operands with 0 in the place of infinities and NaN: what meets parts past the first, which are 0 where the first has all of a
// value, so that an infinity by a value is not made NaN by its parts
__device__ __forceinline__ u32x4 finite_of(u32x4 v) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
    if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
  }
  return v;
}
// An order of workgroups that leaves each of the eight XCDs (they go to them in turn) a run of neighbours, and of tiles within it in
// blocks of up to eight row tiles, so that what neighbours share is in their L2.
__device__ __forceinline__ int64_t in_runs(int64_t b, int64_t n) {
  const int64_t each = n / 8;
  return b < each * 8 ? b % 8 * each + b / 8 : b;
}
__device__ __forceinline__ void tile_of(int64_t b, int64_t tiles_t, int tiles_o, int64_t &tt, int &to) {
  const int64_t band = (int64_t)8 * tiles_o, first = b / band * 8, in = b % band;
  const int64_t high = min(tiles_t - first, (int64_t)8);
  tt = first + in % high;
  to = (int)(in / high);
}

}  // namespace wcc

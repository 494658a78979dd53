// The operators of a block on rows (rows in 8 bits, group norm, gated feed-forward): what their translation units share.
#pragma once

#include "head.h"
#include "rows.h"

namespace wcc {

constexpr int kKept = WCC_KEPT_BLOCK;  // neighbouring values of a row that share a step
inline int64_t kept_blocks(int64_t width) { return (width + kKept - 1) / kKept; }

struct KeepArgs {
  const void *x;
  void *back;  // restore: written
  int8_t *codes;
  uint8_t *steps;
};
hipError_t launch_keep(const wcc_rows_desc &d, const KeepArgs &g, hipStream_t s);
hipError_t launch_restore(const wcc_rows_desc &d, const KeepArgs &g, hipStream_t s);

struct NormArgs {
  const void *x;        // backward: nullptr where codes hold it
  int8_t *codes;        // forward: nullable, written; backward: read where x is nullptr
  uint8_t *steps;
  const float *gamma, *beta;  // nullable: 1 and 0
  const int32_t *counts;      // nullable: every sample has all its pixels
  void *y;                    // forward
  float *stats;               // forward: nullable, written; backward: read
  const void *dy;             // backward
  void *dx;                   // nullable
  float *dgamma, *dbeta;      // nullable
  char *ws;
};
size_t norm_bytes(const wcc_group_norm_desc &d);
hipError_t launch_norm_forward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t s);
hipError_t launch_norm_backward(const wcc_group_norm_desc &d, const NormArgs &g, hipStream_t s);

struct GatedArgs {
  const void *x;  // backward: nullptr where x_codes hold it
  const int8_t *x_codes;
  const uint8_t *x_steps;
  const void *w_gate, *w_up;
  int8_t *codes;  // of both projections, nullable; forward: written, backward: read
  uint8_t *steps;
  void *y;         // forward
  const void *dy;  // backward
  void *dx, *dw_gate, *dw_up;  // nullable
  char *ws;
};
size_t gated_bytes(const wcc_gated_desc &d, bool backward);
hipError_t launch_gated_forward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s);
hipError_t launch_gated_backward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s);

// ---- rows in 8 bits ------------------------------------------------------------------------------------
// A block's step is 2^e, e = floor(log2 top) - 6 (top: its largest magnitude), so codes reach 64 to 127; where top would round to
// 128 steps, e is one more (at the top of fp32's range, where there is no value for one more, codes end at 127).  e is -126 at
// least, so that no step and no value is subnormal.  A code times a step has 7 bits: exact in bf16 and fp32.
// The byte of a step is e + 127; 255 stands for a block that holds an infinity or NaN.

// The byte from the bits of top, sign cleared: whole numbers order as the magnitudes do, infinities and NaN above all.
__device__ __forceinline__ uint32_t step_of(uint32_t top) {
  const uint32_t E = top >> 23;
  if (E == 255) return 255;
  uint32_t b = E > 7 ? E - 6 : 1;
  if (E > 6 && E < 254 && (top & 0x7fffffu) >= 0x7f0000u) ++b;
  return b;
}
__device__ __forceinline__ float per_step(uint32_t b) { return b == 255 ? 0.f : __uint_as_float((254 - b) << 23); }
__device__ __forceinline__ float step_value(uint32_t b) { return __uint_as_float(b == 255 ? 0x7fc00000u : b << 23); }

// 4 codes; rounding to nearest even is that of the sum with 1.5 * 2^23, whose lowest byte the code is
__device__ __forceinline__ uint32_t codes_of(float a, float b, float c, float d, float per) {
  auto one = [&](float v) { return __float_as_uint(__builtin_amdgcn_fmed3f(v * per, -127.f, 127.f) + 12582912.f); };
  const uint32_t lo = __builtin_amdgcn_perm(one(b), one(a), 0x0c0c0400), hi = __builtin_amdgcn_perm(one(d), one(c), 0x0c0c0400);
  return lo | hi << 16;
}
__device__ __forceinline__ uint32_t code_byte(float v, float per) {
  return __float_as_uint(__builtin_amdgcn_fmed3f(v * per, -127.f, 127.f) + 12582912.f) & 255u;
}
// the value of code j of a word
__device__ __forceinline__ float kept_value(uint32_t codes, int j, float step) {
  return (float)(int8_t)(codes >> (8 * j)) * step;
}

// ---- activations ---------------------------------------------------------------------------------------
// 2^v and 1 / v of the hardware, off by 1 ulp each
__device__ __forceinline__ float exp2_fast(float v) { return __builtin_amdgcn_exp2f(v); }
__device__ __forceinline__ float rcp_fast(float v) { return __builtin_amdgcn_rcpf(v); }

// exp(-z).  Where results are fp32 the rest that z * log2(e) rounds off is put back; in bf16's 8 bits it is lost anyway.
template <class T>
__device__ __forceinline__ float exp_neg(float z) {
  const float t = -z * kLog2e, e = exp2_fast(t);
  if constexpr (sizeof(T) == 2) return e;
  const float rest = fmaf(-z, kLog2e, -t) + -z * 1.925963033500e-08f;  // (log2(e) - its fp32 value)
  return fabsf(t) < 126.f ? fmaf(e * kLn2, rest, e) : e;
}

// v = act(z) and s = act'(z); relu has slope 0 at 0
template <class T, int ACT>
__device__ __forceinline__ void act_of(float z, float &v, float &s) {
  if constexpr (ACT == WCC_ACT_NONE) {
    v = z, s = 1.f;
  } else if constexpr (ACT == WCC_ACT_RELU) {
    v = z > 0.f ? z : z != z ? z : 0.f, s = z > 0.f ? 1.f : 0.f;
  } else if constexpr (ACT == WCC_ACT_SILU) {
    const float e = exp_neg<T>(z), d = 1.f + e, p = sizeof(T) == 2 ? rcp_fast(d) : 1.f / d;
    v = z * p, s = p * fmaf(z, 1.f - p, 1.f);
  } else {
    // Phi(-|z|) = exp(-z^2 / 2) q(t) with t = 1 / (1 + c |z|), q a polynomial; the slope needs the exponential too.  bf16: q from formula
    // 7.1.26 of Abramowitz and Stegun for erf, off by 1.5e-7.  fp32: q fitted to scaled erfc on (0, 1], largest |z| times the error made
    // smallest, 8e-11; evaluated in fp32 Phi is off by 2.2e-7 at most.  (erfcf and expf by themselves: 1156 x 960 values three times
    // 13.3 us for the gradient's first pass.)
    const float bell = exp2_fast(z * z * (-0.5f * kLog2e));
    float q;
    if constexpr (sizeof(T) == 2) {
      const float t = rcp_fast(fmaf(fabsf(z), 0.3275911f * 0.70710678f, 1.f));
      q = 0.5f * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    } else {
      constexpr float c[8] = {0.10840163007532476f, 0.12539058690897514f, 0.020029725850715104f, 0.3222110849783336f, -0.35860964023713915f,
                              0.4851653549820245f, -0.24534892171368822f, 0.04276017923424634f};
      const float t = rcp_fast(fmaf(fabsf(z), 0.275f, 1.f));
      q = c[7];
#pragma unroll
      for (int i = 6; i >= 0; --i) q = fmaf(q, t, c[i]);
      q *= t;
    }
    const float tail = q * bell, below = z > 0.f ? 1.f - tail : tail;
    v = z * below, s = fmaf(z * 0.39894228040143268f, bell, below);
  }
}

// ---- rows by vectors -----------------------------------------------------------------------------------
// 16 bytes of a row of which `left` elements are there, the rest 0; cut ones in pieces of 8, 4 and 2 bytes
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32x1_any __attribute__((aligned(2)));
template <class T>
__device__ __forceinline__ u32x4 load_part(const T *p, int left) {
  constexpr int VE = VecOf<T>::N;
  if (left >= VE) return *reinterpret_cast<const u32x4_any *>(p);
  u32x4 v = {};
  if (left <= 0) return v;
  const char *at = reinterpret_cast<const char *>(p);
  const int bytes = left * (int)sizeof(T);
  uint32_t four = 0, two = 0;
  if (bytes & 8) {
    const u32x2_any q = *reinterpret_cast<const u32x2_any *>(at);
    v[0] = q[0], v[1] = q[1];
  }
  if (bytes & 4) four = *reinterpret_cast<const u32x1_any *>(at + (bytes & 8));
  if constexpr (sizeof(T) == 2) {
    if (bytes & 2) two = *reinterpret_cast<const uint16_t *>(at + (bytes & 12));
  }
  const uint32_t next = bytes & 4 ? four : two, last = bytes & 4 ? two : 0;
  if (bytes & 8) v[2] = next, v[3] = last;
  else v[0] = next, v[1] = last;
  return v;
}
template <class T>
__device__ __forceinline__ void store_part(T *p, int left, const u32x4 &v) {
  constexpr int VE = VecOf<T>::N;
  if (left >= VE) {
    *reinterpret_cast<u32x4_any *>(p) = v;
    return;
  }
  if (left <= 0) return;
  char *at = reinterpret_cast<char *>(p);
  const int bytes = left * (int)sizeof(T);
  if (bytes & 8) *reinterpret_cast<u32x2_any *>(at) = u32x2_any{v[0], v[1]};
  const uint32_t next = bytes & 8 ? v[2] : v[0], last = bytes & 8 ? v[3] : v[1];
  if (bytes & 4) *reinterpret_cast<u32x1_any *>(at + (bytes & 8)) = next;
  if constexpr (sizeof(T) == 2) {
    if (bytes & 2) *reinterpret_cast<uint16_t *>(at + (bytes & 12)) = (uint16_t)(bytes & 4 ? last : next);
  }
}
// the largest magnitude of a vector, as bits
template <class T>
__device__ __forceinline__ uint32_t top_of(const u32x4 &v) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < VecOf<T>::N; ++j) m = max(m, __float_as_uint(elem<T>(v, j)) & 0x7fffffffu);
  return m;
}
// the same over the lanes that share a block: 32 / VE neighbours
template <class T>
__device__ __forceinline__ uint32_t top_of_block(const u32x4 &v) {
  uint32_t m = top_of<T>(v);
#pragma unroll
  for (int off = 1; off < kKept / VecOf<T>::N; off <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, off, 64));
  return m;
}
// codes of a vector: 8 bytes (bf16) or 4
template <class T>
__device__ __forceinline__ void store_codes(int8_t *p, const u32x4 &v, float per) {
  if (per == 0.f) {  // (nothing finite to round)
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t *>(p) = 0;
    else *reinterpret_cast<uint2 *>(p) = uint2{0, 0};
    return;
  }
  const uint32_t lo = codes_of(elem<T>(v, 0), elem<T>(v, 1), elem<T>(v, 2), elem<T>(v, 3), per);
  if constexpr (sizeof(T) == 4) *reinterpret_cast<uint32_t *>(p) = lo;
  else *reinterpret_cast<uint2 *>(p) = uint2{lo, codes_of(elem<T>(v, 4), elem<T>(v, 5), elem<T>(v, 6), elem<T>(v, 7), per)};
}

}  // namespace wcc

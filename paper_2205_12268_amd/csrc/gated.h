// The gated feed-forward block: what its translation units share.
//
// With g = Wg x and u = Wu x of a row:  y = act(g) u,  dg = dy u act'(g),  du = dy act(g),
//   dx = Wg^T dg + Wu^T du,  dWg = sum_t dg x^T,  dWu = sum_t du x^T.
// dg and du of all rows are held in the workspace, [rows][2][room of C_out] in the type of x: rounded to bf16 once, which the products
// they go into need anyway.  That rounding is of the size of the results' own: together they are 1.41 times as far off as the second alone
// (0.0023 of a step of 4096 rows 2048 <-> 5632, and 0.0017).  Where dg and du are few values its share in a result may be well above the
// average's, so there, and where the caller asks for it (WCC_TRAIN_FINE), they are held in two parts of bf16, [rows][2 parts][2][room], 16 bits,
// and the products take the second parts too (with 0 for weights and rows that are not finite: 0 of a second part by infinity is NaN).
#pragma once

#include "block.h"
#include "tiles.h"

namespace wcc {

constexpr int kRoom = 64;  // lines of d are a multiple of this long, zeros behind C_out
inline int64_t room_of(int64_t width) { return (width + kRoom - 1) / kRoom * kRoom; }

// Where a pair of projections goes.
template <class T>
struct Gate {
  int64_t rows;
  int outs;
  // forward
  T *y;
  int64_t ldy;
  int8_t *codes;   // nullable: [2][rows][blocks * 32]
  uint8_t *steps;  // [2][rows][blocks]
  // backward
  const T *dy;     // stride ldy
  T *d;            // [rows][parts][2][room]
  int64_t room;
  int parts;
};
// values of dg or du that are held in two parts
constexpr int64_t kFew = 1 << 17;

// 4 neighbouring outputs from o on (o a multiple of 4) of row t.  Forward: step bytes of the blocks they lie in, where codes are kept.
// What lies behind the last output is 0 in codes and in d.
template <class T, int ACT, bool BACK>
__device__ __forceinline__ void finish(const Gate<T> &p, int64_t t, int o, float (&g)[4], float (&u)[4], uint32_t gb, uint32_t ub) {
  const int left = p.outs - o;
  T *out = BACK ? nullptr : p.y + t * p.ldy + o;
  if constexpr (!BACK) {
    if (p.codes) {
      const int64_t blocks = (p.outs + kKept - 1) / kKept, at = t * blocks * kKept + o, up = p.rows * blocks * kKept;
      if (o < blocks * kKept) {
        *reinterpret_cast<uint32_t *>(p.codes + at) = gb == 255 ? 0 : codes_of(g[0], g[1], g[2], g[3], per_step(gb));
        *reinterpret_cast<uint32_t *>(p.codes + up + at) = ub == 255 ? 0 : codes_of(u[0], u[1], u[2], u[3], per_step(ub));
        if (o % kKept == 0) {
          p.steps[t * blocks + o / kKept] = (uint8_t)gb;
          p.steps[p.rows * blocks + t * blocks + o / kKept] = (uint8_t)ub;
        }
      }
    }
    float f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v, s;
      act_of<T, ACT>(g[j], v, s);
      f[j] = v * u[j];
    }
    if (left >= 4) {
      if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<f32x4_any *>(out) = f32x4_any{f[0], f[1], f[2], f[3]};
      } else {
          *reinterpret_cast<u32x2_any *>(out) = u32x2_any{(uint32_t)narrow<bf16_t>(f[0]) | (uint32_t)narrow<bf16_t>(f[1]) << 16,
                                                        (uint32_t)narrow<bf16_t>(f[2]) | (uint32_t)narrow<bf16_t>(f[3]) << 16};
      }
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < left) out[j] = narrow<T>(f[j]);
    }
  } else {
    const T *top = p.dy + t * p.ldy + o;
    T dy[4] = {};
    if (left >= 4) {
      __builtin_memcpy(dy, top, sizeof dy);
    } else {
#pragma unroll
      for (int j = 0; j < 3; ++j)
        if (j < left) dy[j] = top[j];
    }
    T dg[4], du[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float v, s;
      act_of<T, ACT>(g[j], v, s);
      const float d = widen(dy[j]);
      dg[j] = narrow<T>(j < left ? d * u[j] * s : 0.f), du[j] = narrow<T>(j < left ? d * v : 0.f);
    }
    T *at = p.d + t * p.parts * 2 * p.room + o;  // (o and the room are multiples of 4)
    __builtin_memcpy(__builtin_assume_aligned(at, 4 * sizeof(T)), dg, sizeof dg);
    __builtin_memcpy(__builtin_assume_aligned(at + p.room, 4 * sizeof(T)), du, sizeof du);
    if constexpr (sizeof(T) == 2) {
      if (p.parts == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v, s;
          act_of<T, ACT>(g[j], v, s);
          const float d = widen(dy[j]);
          dg[j] = narrow<T>(left_of(j < left ? d * u[j] * s : 0.f, dg[j])), du[j] = narrow<T>(left_of(j < left ? d * v : 0.f, du[j]));
        }
        at += 2 * p.room;
        __builtin_memcpy(__builtin_assume_aligned(at, 4 * sizeof(T)), dg, sizeof dg);
        __builtin_memcpy(__builtin_assume_aligned(at + p.room, 4 * sizeof(T)), du, sizeof du);
      }
    }
  }
}

// A line of an operand is at p + line * s (k contiguous) or p + line (lines contiguous, k s apart).
template <class T>
struct Side {
  const T *p;
  int64_t s;
  int64_t lines;
};
// result[row of a][line of b] = sum over phases and k of a(row, k) b(line, k)
template <class T>
struct Product {
  Side<T> a[4], b[4];  // of phase f and batch i at f * batches + i
  int phases, second;  // from `second` on phases are of second parts
  int64_t k;           // of each phase
  T *out[2];           // of each batch
  int64_t ld;
  int batches;
};

// fp32 sums of ranges of k that the calls below leave in the workspace, in bytes; size: of an element
size_t tile_gate_parts(int64_t rows, int64_t outs, int64_t k, int size);
size_t tile_product_parts(int64_t rows, int64_t lines, int64_t k, int batches, int size);

// (all three ways to a pair of projections leave as many parts of dg and du as p.parts says)
template <class T>
hipError_t tile_gate(const Gate<T> &p, int act, bool back, const Side<T> &x, const T *w_gate, const T *w_up, int64_t ldw, int64_t k,
                     float *part, hipStream_t s);
// the sums of `splits` ranges of k, [splits][rows][2][room], joined
template <class T>
hipError_t join_gate(const Gate<T> &p, int act, bool back, int splits, const float *part, hipStream_t s);
template <class T, bool AT>
hipError_t tile_product(const Product<T> &p, float *part, hipStream_t s);

// Straight from memory (gated_gemm.hip).  Operands whose k or lines are contiguous and 16 bytes a load: pointers and strides are multiples.
bool gemm_takes(const void *p, int64_t ld, int64_t width, int size);
size_t gemm_gate_parts(int64_t rows, int64_t outs, int64_t k, int size);
template <class T>
hipError_t gemm_gate(const Gate<T> &p, int act, bool back, const Side<T> &x, const T *w_gate, const T *w_up, int64_t ldw, int64_t k, float *part,
                     hipStream_t s);
// dx and the weights' gradients from dg and du, all in one launch, and one that joins ranges of k.
template <class T>
struct Backward {
  const T *d;
  int64_t room, rows;
  int parts;
  const T *w_gate, *w_up;
  int64_t ldw;
  const T *x;
  int64_t ldx, width;
  int64_t C_in, C_out;
  T *dx;  // nullable, as the two below
  int64_t ld;
  T *dw_gate, *dw_up;
};
size_t gemm_back_parts(int64_t rows, int64_t C_in, int64_t C_out, int parts, int size);
template <class T>
hipError_t gemm_back(const Backward<T> &b, float *part, hipStream_t s);

// The two projections for few rows of bf16 (gated_thin.hip), operands as above.
size_t thin_gate_parts(int64_t rows, int64_t outs, int64_t k);
hipError_t thin_gate(const Gate<bf16_t> &p, int act, bool back, const Side<bf16_t> &x, const bf16_t *w_gate, const bf16_t *w_up, int64_t ldw,
                     int64_t k, float *part, hipStream_t s);

}  // namespace wcc

// The gated feed-forward block: routes, and the slopes from kept projections.
#include <algorithm>

#include "gated.h"

namespace wcc {
namespace {

// dg and du from what the projections are kept as: a lane has 16 bytes of dy.  Bound by memory: 4096 x 5632 bf16 in 33 us,
// 5.6 TB/s.
template <class T, int ACT>
__global__ __launch_bounds__(256) void kept_slopes_kernel(Gate<T> p) {
  constexpr int VE = VecOf<T>::N;
  const int64_t per_row = p.room / VE, blocks = (p.outs + kKept - 1) / kKept, up = p.rows * blocks;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < p.rows * per_row; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per_row;
    const int o = (int)(i - t * per_row) * VE, left = p.outs - o;
    float dg[VE] = {}, du[VE] = {};
    if (left > 0) {
      const u32x4 top = load_part<T>(p.dy + t * p.ldy + o, left);
      const int64_t block = t * blocks + o / kKept, at = block * kKept + o % kKept;
      const float gs = step_value(p.steps[block]), us = step_value(p.steps[up + block]);
#pragma unroll
      for (int h = 0; h < VE / 4; ++h) {
        const uint32_t gc = reinterpret_cast<const uint32_t *>(p.codes + at)[h], uc = reinterpret_cast<const uint32_t *>(p.codes + up * kKept + at)[h];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float v, s;
          act_of<T, ACT>(kept_value(gc, j, gs), v, s);
          const float dy = elem<T>(top, 4 * h + j);
          if (4 * h + j < left) dg[4 * h + j] = dy * kept_value(uc, j, us) * s, du[4 * h + j] = dy * v;
        }
      }
    }
    T *d = p.d + t * p.parts * 2 * p.room + o;
    *reinterpret_cast<u32x4 *>(d) = pack<T>(dg);
    *reinterpret_cast<u32x4 *>(d + p.room) = pack<T>(du);
    if constexpr (sizeof(T) == 2) {
      if (p.parts == 2) {
#pragma unroll
        for (int j = 0; j < VE; ++j) dg[j] = left_of(dg[j], narrow<T>(dg[j])), du[j] = left_of(du[j], narrow<T>(du[j]));
        *reinterpret_cast<u32x4 *>(d + 2 * p.room) = pack<T>(dg);
        *reinterpret_cast<u32x4 *>(d + 3 * p.room) = pack<T>(du);
      }
    }
  }
}

// zeros: what the weights' gradients are without rows
__global__ __launch_bounds__(256) void zeros_kernel(uint16_t *p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// Matrices copied to rows of a stride that 16-byte loads take, zeros behind their width.  Three at most in one launch.
template <class T>
struct Copy {
  const T *from;
  T *to;
  int64_t ld, rows;
};
template <class T>
struct Copies {
  Copy<T> c[3];
  int width;
  int64_t room;
};
template <class T>
__global__ __launch_bounds__(256) void copy_kernel(Copies<T> a) {
  constexpr int VE = VecOf<T>::N;
  const Copy<T> c = a.c[blockIdx.y];
  const int64_t per_row = a.room / VE;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < c.rows * per_row; i += (int64_t)gridDim.x * 256) {
    const int64_t t = i / per_row, e = (i - t * per_row) * VE;
    *reinterpret_cast<u32x4 *>(c.to + t * a.room + e) = load_part<T>(c.from + t * c.ld + e, (int)(a.width - e));
  }
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

// Which kernels a call takes, and what the workspace holds: dg and du; x where it comes as codes or has to be copied; the weights where
// they have to be copied; sums of ranges of k.
struct Plan {
  bool gemm, copy_x, copy_w;  // tiles fed straight from memory
  int parts;                  // of dg and du
  bool few;                   // they are two because dg and du are few
  size_t d, x, w, part, bytes;
  int64_t room, ldx, k;  // of d's halves; of rows and weights that were copied; C_in in whole chunks of 16 bytes
};

constexpr int kThin = 64;  // rows of few

// A backward pass has its products in tiles fed straight from memory, rows and weights that 16-byte loads do not take copied for it: as many
// launches as by way of registers or fewer, and 1.2 to 2.5 times as fast from 2^13 products on (65 rows 64 <-> 64 bf16 14.8 us against
// 31.0, 777 rows 1000 <-> 1537 at odd strides 43.8 and 102, in fp32 173 and 312; 30 rows 4001 <-> 8000 234 and 252; one row 3001 <-> 5001,
// all copies, 166 and 163).  A pair of projections has less to win: bf16 from 2^25 products on (128 rows 128 -> 256, 2^23, 4.6 us and
// 4.4, 256 -> 256 5.4 and 7.1), with copies from 2^27 on (500 rows 301 -> 743 9.3 and 11.2, 512 rows 33 -> 64 6.3 and 4.5), fp32 always, with
// copies from 3 * 2^27 on (777 rows 333 -> 1000 21.9 and 26.7, 300 rows 301 -> 743 18.1 and 13.4).  Made again for few dg and du (kFew) they
// stay in tiles by way of registers: whole backward passes of 100 rows 1024 <-> 640 take 27 us so and 32, 1000 rows 1001 <-> 120 40 and 45, 1000 rows
// 4096 <-> 130 60 and 57.
Plan plan_of(const wcc_gated_desc &g, bool backward) {
  Plan p = {};
  const int size = g.dtype == WCC_F32 ? 4 : 2;
  const double products = 2.0 * g.rows * g.C_in * g.C_out;
  const int each = 16 / size;
  p.room = room_of(g.C_out), p.ldx = room_of(g.C_in), p.k = (g.C_in + each - 1) / each * each;
  p.copy_w = g.C_in % each != 0, p.copy_x = p.copy_w || g.ldx % each != 0;
  const bool thin = size == 2 && g.rows <= kThin;
  const double least = size == 2 ? (p.copy_x && !backward ? 1 << 27 : 1 << 25) : p.copy_x && !backward ? 3 << 27 : 0;
  p.gemm = !thin && products >= least;
  p.few = size == 2 && g.rows * (int64_t)g.C_out < kFew;
  p.parts = size == 2 && (p.few || g.train == WCC_TRAIN_FINE) ? 2 : 1;
  if (!backward && !p.gemm) p.copy_x = p.copy_w = false;
  size_t parts = tile_gate_parts(g.rows, g.C_out, g.C_in, size), at = 0;  // (tensors at odd addresses take these tiles)
  if (size == 2 && g.rows <= kThin) parts = std::max(parts, thin_gate_parts(g.rows, g.C_out, p.k));
  if (p.gemm) parts = std::max(parts, gemm_gate_parts(g.rows, g.C_out, p.k, size));
  if (backward) at += up((size_t)g.rows * p.parts * 2 * p.room * size);
  p.x = at;
  if (backward || p.copy_x) at += up((size_t)g.rows * p.ldx * size);
  p.w = at;
  if (p.copy_w) at += 2 * up((size_t)g.C_out * p.ldx * size);
  p.part = at;
  if (backward) {
    parts = std::max({parts, gemm_back_parts(g.rows, g.C_in, g.C_out, p.parts, size), tile_product_parts(g.rows, g.C_in, g.C_out, 1, size),
                      tile_product_parts(g.C_out, g.C_in, g.rows, 2, size)});
  }
  p.bytes = p.part + up(parts);
  return p;
}

// The operands of a call as its products take them.
template <class T>
struct Operands {
  bool takes;  // 16-byte loads
  Side<T> x;
  const T *wg, *wu;
  int64_t ldw;
};
template <class T>
hipError_t prepare(const wcc_gated_desc &d, const Plan &p, const GatedArgs &g, bool x_used, bool w_used, Operands<T> &o, hipStream_t s) {
  o.wg = static_cast<const T *>(g.w_gate), o.wu = static_cast<const T *>(g.w_up), o.ldw = d.C_in;
  o.x = Side<T>{static_cast<const T *>(g.x), d.ldx, d.rows};
  o.takes = true;
  hipError_t e = hipSuccess;
  if (x_used && !g.x) {  // (whole blocks: zeros behind the width)
    wcc_rows_desc r = {};
    r.rows = d.rows, r.width = (int32_t)(kept_blocks(d.C_in) * kKept), r.dtype = d.dtype, r.ld = p.ldx;
    KeepArgs k = {};
    k.back = g.ws + p.x, k.codes = const_cast<int8_t *>(g.x_codes), k.steps = const_cast<uint8_t *>(g.x_steps);
    if ((e = launch_restore(r, k, s)) != hipSuccess) return e;
    o.x = Side<T>{static_cast<const T *>(k.back), p.ldx, d.rows};
  }
  Copies<T> c = {};
  int n = 0;
  c.width = d.C_in, c.room = p.ldx;
  if (x_used && g.x && p.copy_x) {
    T *to = reinterpret_cast<T *>(g.ws + p.x);
    c.c[n++] = Copy<T>{o.x.p, to, d.ldx, d.rows};
    o.x = Side<T>{to, p.ldx, d.rows};
  }
  if (w_used && p.copy_w) {
    T *to = reinterpret_cast<T *>(g.ws + p.w), *next = reinterpret_cast<T *>(g.ws + p.w + up((size_t)d.C_out * p.ldx * sizeof(T)));
    c.c[n++] = Copy<T>{o.wg, to, d.C_in, d.C_out}, c.c[n++] = Copy<T>{o.wu, next, d.C_in, d.C_out};
    o.wg = to, o.wu = next, o.ldw = p.ldx;
  }
  if (n > 0) {
    const int64_t most = std::max<int64_t>(d.rows, d.C_out) * (p.ldx / VecOf<T>::N);
    copy_kernel<T><<<dim3((unsigned)std::min<int64_t>((most + 255) / 256, 2048), n), 256, 0, s>>>(c);
    e = hipGetLastError();
  }
  if (x_used) o.takes = gemm_takes(o.x.p, o.x.s, p.k, sizeof(T));
  if (w_used) o.takes = o.takes && gemm_takes(o.wg, o.ldw, p.k, sizeof(T)) && gemm_takes(o.wu, o.ldw, p.k, sizeof(T));
  return e;
}

template <class T>
hipError_t gate_of(const wcc_gated_desc &d, const Plan &p, const Gate<T> &gate, bool back, const Operands<T> &o, float *part, hipStream_t s) {
  if constexpr (sizeof(T) == 2) {
    if (d.rows <= kThin && o.takes) return thin_gate(gate, d.act, back, o.x, o.wg, o.wu, o.ldw, p.k, part, s);
  }
  if (p.gemm && o.takes && !(back && p.few)) return gemm_gate<T>(gate, d.act, back, o.x, o.wg, o.wu, o.ldw, p.k, part, s);
  return tile_gate<T>(gate, d.act, back, o.x, o.wg, o.wu, o.ldw, d.C_in, part, s);
}

template <class T>
hipError_t forward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  const Plan p = plan_of(d, false);
  Operands<T> o;
  hipError_t e = prepare<T>(d, p, g, true, true, o, s);
  if (e != hipSuccess) return e;
  Gate<T> gate = {};
  gate.rows = d.rows, gate.outs = d.C_out, gate.y = static_cast<T *>(g.y), gate.ldy = d.ldy, gate.codes = g.codes, gate.steps = g.steps;
  gate.room = p.room, gate.parts = p.parts;
  return gate_of<T>(d, p, gate, false, o, reinterpret_cast<float *>(g.ws + p.part), s);
}

template <class T, int ACT>
void kept_slopes(const Gate<T> &gate, hipStream_t s) {
  const int64_t n = gate.rows * (gate.room / VecOf<T>::N);
  kept_slopes_kernel<T, ACT><<<(unsigned)std::min<int64_t>((n + 255) / 256, 8192), 256, 0, s>>>(gate);
}

template <class T>
hipError_t backward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  const Plan p = plan_of(d, true);
  float *part = reinterpret_cast<float *>(g.ws + p.part);
  const bool dw = g.dw_gate || g.dw_up, again = !g.codes;
  Operands<T> o;
  hipError_t e = prepare<T>(d, p, g, dw || again, g.dx || again, o, s);
  if (e != hipSuccess) return e;
  Gate<T> gate = {};
  gate.rows = d.rows, gate.outs = d.C_out, gate.ldy = d.ldy, gate.codes = g.codes, gate.steps = g.steps;
  gate.dy = static_cast<const T *>(g.dy), gate.d = reinterpret_cast<T *>(g.ws + p.d), gate.room = p.room, gate.parts = p.parts;
  if (again) {
    e = gate_of<T>(d, p, gate, true, o, part, s);
  } else {
    switch (d.act) {
      case WCC_ACT_RELU: kept_slopes<T, WCC_ACT_RELU>(gate, s); break;
      case WCC_ACT_SILU: kept_slopes<T, WCC_ACT_SILU>(gate, s); break;
      case WCC_ACT_GELU: kept_slopes<T, WCC_ACT_GELU>(gate, s); break;
      default: kept_slopes<T, WCC_ACT_NONE>(gate, s);
    }
    e = hipGetLastError();
  }
  if (e != hipSuccess) return e;
  const T *dg = gate.d, *du = gate.d + p.room;
  if (o.takes) {
    const Backward<T> b{dg, p.room, d.rows, p.parts, o.wg, o.wu, o.ldw, o.x.p, o.x.s, p.k, d.C_in, d.C_out, static_cast<T *>(g.dx), d.ldx,
                        static_cast<T *>(g.dw_gate), static_cast<T *>(g.dw_up)};
    return gemm_back<T>(b, part, s);
  }
  const int64_t ldd = p.parts * 2 * p.room, next = 2 * p.room;
  if (g.dx) {
    Product<T> m = {};
    m.phases = 2 * p.parts, m.second = 2, m.batches = 1, m.k = d.C_out, m.ld = d.ldx, m.out[0] = static_cast<T *>(g.dx);
    for (int i = 0; i < p.parts; ++i) {
      m.a[2 * i] = Side<T>{dg + i * next, ldd, d.rows}, m.a[2 * i + 1] = Side<T>{du + i * next, ldd, d.rows};
      m.b[2 * i] = Side<T>{o.wg, o.ldw, d.C_in}, m.b[2 * i + 1] = Side<T>{o.wu, o.ldw, d.C_in};
    }
    if ((e = tile_product<T, false>(m, part, s)) != hipSuccess) return e;
  }
  if (dw) {
    Product<T> m = {};
    m.phases = p.parts, m.second = 1, m.k = d.rows, m.ld = d.C_in;
    if (g.dw_gate) m.out[m.batches++] = static_cast<T *>(g.dw_gate);
    if (g.dw_up) m.out[m.batches++] = static_cast<T *>(g.dw_up);
    for (int i = 0; i < p.parts; ++i) {
      int n = i * m.batches;
      if (g.dw_gate) m.a[n] = Side<T>{dg + i * next, ldd, d.C_out}, m.b[n++] = Side<T>{o.x.p, o.x.s, d.C_in};
      if (g.dw_up) m.a[n] = Side<T>{du + i * next, ldd, d.C_out}, m.b[n] = Side<T>{o.x.p, o.x.s, d.C_in};
    }
    if ((e = tile_product<T, true>(m, part, s)) != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t gated_bytes(const wcc_gated_desc &d, bool backward) { return d.rows > 0 ? plan_of(d, backward).bytes : 0; }

hipError_t launch_gated_forward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  return d.dtype == WCC_F32 ? forward<float>(d, g, s) : forward<bf16_t>(d, g, s);
}
hipError_t launch_gated_backward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  if (d.rows == 0) {
    const int64_t n = (int64_t)d.C_in * d.C_out * (d.dtype == WCC_F32 ? 2 : 1);
    for (void *p : {g.dw_gate, g.dw_up})
      if (p) zeros_kernel<<<(unsigned)std::min<int64_t>((n + 255) / 256, 8192), 256, 0, s>>>(static_cast<uint16_t *>(p), n);
    return hipGetLastError();
  }
  return d.dtype == WCC_F32 ? backward<float>(d, g, s) : backward<bf16_t>(d, g, s);
}

}  // namespace wcc

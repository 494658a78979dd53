// The gated feed-forward block: routes, and the slopes from kept projections.
#include <algorithm>

#include "gated.h"

namespace wcc {
namespace {

// dg and du from what the projections are kept as: a lane has 16 bytes of dy.  Bound by memory.
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
    T *d = p.d + t * 2 * p.room + o;
    *reinterpret_cast<u32x4 *>(d) = pack<T>(dg);
    *reinterpret_cast<u32x4 *>(d + p.room) = pack<T>(du);
  }
}

// zeros: what the weights' gradients are without rows
__global__ __launch_bounds__(256) void zeros_kernel(uint16_t *p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

size_t up(size_t v) { return (v + 255) / 256 * 256; }

struct Plan {
  size_t d, x, part, bytes;  // of the backward pass: dg and du; x where it is kept in codes; sums of ranges of k
  int64_t room, ldx;
};

Plan plan_of(const wcc_gated_desc &g, bool backward) {
  Plan p = {};
  const size_t size = g.dtype == WCC_F32 ? 4 : 2;
  p.room = room_of(g.C_out), p.ldx = room_of(g.C_in);
  size_t parts = tile_gate_parts(g.rows, g.C_out, g.C_in);
  if (backward) {
    p.x = up((size_t)g.rows * 2 * p.room * size);
    p.part = p.x + up((size_t)g.rows * p.ldx * size);
    parts = std::max({parts, tile_product_parts(g.rows, g.C_in, g.C_out, 1), tile_product_parts(g.C_out, g.C_in, g.rows, 2)});
  }
  p.bytes = p.part + up(parts);
  return p;
}

template <class T>
hipError_t forward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  const Plan p = plan_of(d, false);
  Gate<T> gate = {};
  gate.rows = d.rows, gate.outs = d.C_out, gate.y = static_cast<T *>(g.y), gate.ldy = d.ldy, gate.codes = g.codes, gate.steps = g.steps;
  gate.room = p.room;
  const Side<T> x{static_cast<const T *>(g.x), d.ldx, d.rows};
  return tile_gate<T>(gate, d.act, false, x, static_cast<const T *>(g.w_gate), static_cast<const T *>(g.w_up), d.C_in,
                      reinterpret_cast<float *>(g.ws + p.part), s);
}

template <class T, int ACT>
void kept_slopes(const Gate<T> &gate, hipStream_t s) {
  const int64_t n = gate.rows * (gate.room / VecOf<T>::N);
  kept_slopes_kernel<T, ACT><<<(unsigned)std::min<int64_t>((n + 255) / 256, 8192), 256, 0, s>>>(gate);
}

template <class T>
hipError_t backward(const wcc_gated_desc &d, const GatedArgs &g, hipStream_t s) {
  const Plan p = plan_of(d, true);
  const T *wg = static_cast<const T *>(g.w_gate), *wu = static_cast<const T *>(g.w_up);
  float *part = reinterpret_cast<float *>(g.ws + p.part);
  Side<T> x{static_cast<const T *>(g.x), d.ldx, d.rows};
  hipError_t e = hipSuccess;
  const bool dw = g.dw_gate || g.dw_up;
  if (!g.x && (dw || !g.codes)) {
    wcc_rows_desc r = {};
    r.rows = d.rows, r.width = d.C_in, r.dtype = d.dtype, r.ld = p.ldx;
    KeepArgs k = {};
    k.back = g.ws + p.x, k.codes = const_cast<int8_t *>(g.x_codes), k.steps = const_cast<uint8_t *>(g.x_steps);
    if ((e = launch_restore(r, k, s)) != hipSuccess) return e;
    x = Side<T>{static_cast<const T *>(k.back), p.ldx, d.rows};
  }
  Gate<T> gate = {};
  gate.rows = d.rows, gate.outs = d.C_out, gate.ldy = d.ldy, gate.codes = g.codes, gate.steps = g.steps;
  gate.dy = static_cast<const T *>(g.dy), gate.d = reinterpret_cast<T *>(g.ws + p.d), gate.room = p.room;
  if (g.codes) {
    switch (d.act) {
      case WCC_ACT_RELU: kept_slopes<T, WCC_ACT_RELU>(gate, s); break;
      case WCC_ACT_SILU: kept_slopes<T, WCC_ACT_SILU>(gate, s); break;
      case WCC_ACT_GELU: kept_slopes<T, WCC_ACT_GELU>(gate, s); break;
      default: kept_slopes<T, WCC_ACT_NONE>(gate, s);
    }
    e = hipGetLastError();
  } else {
    e = tile_gate<T>(gate, d.act, true, x, wg, wu, d.C_in, part, s);
  }
  if (e != hipSuccess) return e;
  const T *dg = gate.d, *du = gate.d + p.room;
  if (g.dx) {
    Product<T> m = {};
    m.phases = 2, m.batches = 1, m.k = d.C_out, m.ld = d.ldx, m.out[0] = static_cast<T *>(g.dx);
    m.a[0] = Side<T>{dg, 2 * p.room, d.rows}, m.a[1] = Side<T>{du, 2 * p.room, d.rows};
    m.b[0] = Side<T>{wg, d.C_in, d.C_in}, m.b[1] = Side<T>{wu, d.C_in, d.C_in};
    if ((e = tile_product<T, false>(m, part, s)) != hipSuccess) return e;
  }
  if (dw) {
    Product<T> m = {};
    m.phases = 1, m.k = d.rows, m.ld = d.C_in;
    int n = 0;
    if (g.dw_gate) m.a[n] = Side<T>{dg, 2 * p.room, d.C_out}, m.out[n++] = static_cast<T *>(g.dw_gate);
    if (g.dw_up) m.a[n] = Side<T>{du, 2 * p.room, d.C_out}, m.out[n++] = static_cast<T *>(g.dw_up);
    m.batches = n;
    m.b[0] = m.b[1] = Side<T>{x.p, x.s, d.C_in};
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

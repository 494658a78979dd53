// The two projections of the gated block for few rows of bf16: what counts is the weights on their way.
//
// A workgroup has 32 outputs of both weights and 32 rows of x; its four waves take stages of 64 k in turn and add up at the end.  A wave's
// stages go to LDS of its own straight from memory, 1 KiB a load in whole lines of memory, a ring of D of them ahead: the waves wait for
// nobody until the end, and nothing but their own loads.  The rows' part of a stage goes the same way, so that loads arrive in the order
// they are waited for.  One launch: the activation, the product and the codes are made where the sums are.
// Bound by memory.
#include <algorithm>

#include "gated.h"

namespace wcc {
namespace {

constexpr uint32_t kNowhere = 0x80000000u;  // beyond any descriptor here

// XR: loads of 8 rows of x a stage.  PARTS: a range of `range` stages, whose sums go to part [splits][rows][2][room].
template <int XR, int D, int ACT, bool BACK, bool PARTS>
__global__ __launch_bounds__(256) void gate_thin_kernel(Gate<bf16_t> p, Side<bf16_t> x, const bf16_t *__restrict__ w_gate,
                                                        const bf16_t *__restrict__ w_up, int64_t ldw, int k, int range,
                                                        float *__restrict__ part) {
  constexpr int Stage = (8 + XR) * 1024, L = 8 + XR;
  __shared__ __align__(1024) unsigned char ring[4][D][Stage];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane & 31, half = lane >> 5;
  const int o0 = blockIdx.x * 32;
  const int64_t t0 = (int64_t)blockIdx.y * 32;
  auto buffer = [&](const bf16_t *q, int64_t lines, int64_t ld) {  // (in the backward pass outputs go on up to d's room: no lines)
    const int64_t bytes = lines > 0 ? ((min(lines, (int64_t)32) - 1) * ld + k) * 2 : 0;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16_t *>(q), 0, (int)(uint32_t)bytes, 0x00020000);
  };
  const __amdgpu_buffer_rsrc_t rg = buffer(w_gate + o0 * ldw, p.outs - o0, ldw), ru = buffer(w_up + o0 * ldw, p.outs - o0, ldw),
                               rx = buffer(x.p + t0 * x.s, p.rows - t0, x.s);
  uint32_t wo[2], xo[2];
  int chunk[2];
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    chunk[b] = (lane % 8) ^ chunk_key(b * 8 + lane / 8);
    wo[b] = (uint32_t)((b * 8 + lane / 8) * ldw * 2 + chunk[b] * 16);
    xo[b] = (uint32_t)((b * 8 + lane / 8) * x.s * 2 + chunk[b] * 16);
  }
  const int first = PARTS ? (int)blockIdx.z * range : 0, stages = PARTS ? min((k + kK - 1) / kK, first + range) : (k + kK - 1) / kK;
  auto load = [&](int s, int slot) {  // (a stage past the last: loads of nothing, so that the counts hold)
    uint32_t at[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) at[b] = s < stages && chunk[b] * 8 < k - s * kK ? (uint32_t)(s * kLine) : kNowhere;
    unsigned char *to = ring[wv][slot];
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const int b = i & 1, line = i < 8 ? (i & 3) >> 1 : (i - 8) >> 1;
      const uint32_t off = i < 8 ? wo[b] + (uint32_t)(line * 32 * ldw) : xo[b] + (uint32_t)(line * 32 * x.s);  // (16 lines further)
      const uint32_t where = at[b] == kNowhere ? kNowhere : off + at[b];
      auto *dst = (__attribute__((address_space(3))) void *)(to + i * 1024);
      if (i < 4) __builtin_amdgcn_raw_ptr_buffer_load_lds(rg, dst, 16, where, 0, 0, 0);
      else if (i < 8) __builtin_amdgcn_raw_ptr_buffer_load_lds(ru, dst, 16, where, 0, 0, 0);
      else __builtin_amdgcn_raw_ptr_buffer_load_lds(rx, dst, 16, where, 0, 0, 0);
    }
  };
  f32x16 g = {}, u = {};
#pragma unroll
  for (int i = 0; i < D; ++i) load(first + wv + 4 * i, i);
  int slot = 0;
  for (int s = first + wv; s < stages; s += 4) {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * L) : "memory");
    const unsigned char *at = ring[wv][slot];
    u32x4 gf[4], uf[4], xf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      gf[i] = chunk_of(at, ln, i * 2 + half);
      uf[i] = chunk_of(at + 4096, ln, i * 2 + half);
      xf[i] = chunk_of(at + 8192, ln % (XR * 8), i * 2 + half);  // (rows past XR * 8 repeat others, and go nowhere)
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    load(s + 4 * D, slot);
#pragma unroll
    for (int i = 0; i < 4; ++i) g = mma<bf16_t>(gf[i], xf[i], g), u = mma<bf16_t>(uf[i], xf[i], u);
    slot = slot + 1 == D ? 0 : slot + 1;
  }
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing is on its way to LDS from here on
  __syncthreads();
  // the waves' sums: register i of both at [wave][i][lane]
  float *sums = reinterpret_cast<float *>(&ring[0][0][0]);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    sums[(wv * 32 + i) * 64 + lane] = g[i];
    sums[(wv * 32 + 16 + i) * 64 + lane] = u[i];
  }
  __syncthreads();
  float ga[4], ua[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    ga[j] = ua[j] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      ga[j] += sums[(w * 32 + 4 * wv + j) * 64 + lane];
      ua[j] += sums[(w * 32 + 16 + 4 * wv + j) * 64 + lane];
    }
  }
  const int64_t t = t0 + ln;
  const int o = o0 + result_line(4 * wv, half);
  if constexpr (PARTS) {
    if (ln < XR * 8 && t < p.rows && o < p.room) {
      float *q = part + ((blockIdx.z * p.rows + t) * 2) * p.room + o;
      *reinterpret_cast<f32x4_any *>(q) = f32x4_any{ga[0], ga[1], ga[2], ga[3]};
      *reinterpret_cast<f32x4_any *>(q + p.room) = f32x4_any{ua[0], ua[1], ua[2], ua[3]};
    }
    return;
  }
  uint32_t gb = 0, ub = 0;
  if (!BACK && p.codes) {  // (lines behind the last are 0)
    uint32_t(*tops)[2][32] = reinterpret_cast<uint32_t(*)[2][32]>(sums + 4 * 32 * 64);
#pragma unroll
    for (int j = 0; j < 4; ++j) gb = max(gb, __float_as_uint(ga[j]) & 0x7fffffffu), ub = max(ub, __float_as_uint(ua[j]) & 0x7fffffffu);
    gb = max(gb, (uint32_t)__shfl_xor((int)gb, 32, 64)), ub = max(ub, (uint32_t)__shfl_xor((int)ub, 32, 64));
    tops[wv][half][ln] = half ? ub : gb;
    __syncthreads();
    gb = step_of(max(max(tops[0][0][ln], tops[1][0][ln]), max(tops[2][0][ln], tops[3][0][ln])));
    ub = step_of(max(max(tops[0][1][ln], tops[1][1][ln]), max(tops[2][1][ln], tops[3][1][ln])));
  }
  if (ln < XR * 8 && t < p.rows && o < p.room) finish<bf16_t, ACT, BACK>(p, t, o, ga, ua, gb, ub);
}

}  // namespace

namespace {

// Ranges of 16 stages and more of long rows where there are few workgroups (16 of them, a step of 2 rows 7744 <-> 512 with two such launches:
// 54 us, 46 in ranges; 2624 -> 320 would lose by the second launch).
struct ThinPlan {
  int blocks, splits, chunk;
};
ThinPlan thin_plan(int64_t rows, int64_t room, int64_t k) {
  const int stages = (int)((k + kK - 1) / kK);
  ThinPlan p;
  p.blocks = (int)((room + 31) / 32);
  const int64_t n = p.blocks * ((rows + 31) / 32);
  const int want = n < 64 && stages >= 64 ? std::min<int64_t>(256 / n, stages / 16) : 1;
  p.chunk = (stages + want - 1) / want;
  p.splits = (stages + p.chunk - 1) / p.chunk;
  return p;
}

}  // namespace

size_t thin_gate_parts(int64_t rows, int64_t outs, int64_t k) {
  const ThinPlan p = thin_plan(rows, room_of(outs), k);
  return p.splits > 1 ? (size_t)p.splits * rows * 2 * room_of(outs) * sizeof(float) : 0;
}

// x's rows up to 8, 16 or 32 a workgroup, 9 to 12 KiB a stage, and as many stages as leave LDS to it alone: up to 144 KiB.
// One row, 2048 -> 5632 (46 MB of weights): 8.4 us on weights that stay in the caches, 10.8 on weights in turn (4.3 TB/s); tiles of
// 128 rows in five ranges of k and their join 13.0 + 3.9.
hipError_t thin_gate(const Gate<bf16_t> &p, int act, bool back, const Side<bf16_t> &x, const bf16_t *w_gate, const bf16_t *w_up, int64_t ldw,
                     int64_t k, float *part, hipStream_t s) {
  const ThinPlan plan = thin_plan(p.rows, p.room, k);
  const dim3 blocks((unsigned)plan.blocks, (unsigned)((p.rows + 31) / 32), (unsigned)plan.splits);
  auto go = [&](auto xr, auto d, auto a, auto b, auto parts) {
    gate_thin_kernel<decltype(xr)::value, decltype(d)::value, decltype(a)::value, decltype(b)::value, decltype(parts)::value>
        <<<blocks, 256, 0, s>>>(p, x, w_gate, w_up, ldw, (int)k, plan.chunk, part);
  };
  auto by_rows = [&](auto a, auto b, auto parts) {
    if (p.rows <= 8) go(std::integral_constant<int, 1>(), std::integral_constant<int, 4>(), a, b, parts);
    else if (p.rows <= 16) go(std::integral_constant<int, 2>(), std::integral_constant<int, 3>(), a, b, parts);
    else go(std::integral_constant<int, 4>(), std::integral_constant<int, 3>(), a, b, parts);
  };
  if (plan.splits > 1) {
    by_rows(std::integral_constant<int, WCC_ACT_NONE>(), std::false_type(), std::true_type());
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : join_gate<bf16_t>(p, act, back, plan.splits, part, s);
  }
  auto by_way = [&](auto a) { back ? by_rows(a, std::true_type(), std::false_type()) : by_rows(a, std::false_type(), std::false_type()); };
  switch (act) {
    case WCC_ACT_RELU: by_way(std::integral_constant<int, WCC_ACT_RELU>()); break;
    case WCC_ACT_SILU: by_way(std::integral_constant<int, WCC_ACT_SILU>()); break;
    case WCC_ACT_GELU: by_way(std::integral_constant<int, WCC_ACT_GELU>()); break;
    default: by_way(std::integral_constant<int, WCC_ACT_NONE>());
  }
  return hipGetLastError();
}

}  // namespace wcc

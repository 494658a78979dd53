// The products of the gated block fed straight from memory: projections of many rows (bf16, from 2^25 products on) or of any (fp32), and all
// products of a backward pass, down to one row, wherever operands begin on 16 bytes and their lines lie a multiple of it apart.
//
// A workgroup of four waves has BT x BO results and two stages of 128 bytes of k (64 bf16, 32 fp32) in LDS; loads (16 bytes a lane) go
// there without passing registers.  A wave's operands of a whole stage fit its registers beside the results, so a stage's half of LDS is
// free after a quarter of its products: from there on the loads of the stage after the next go out, one between every few products.  Two
// barriers a stage: LDS is read; the next stage is there.
// LDS has no padding (such a load writes 1 KiB in a row), so the 16-byte chunks of a line are exchanged by a key of the line, at the load
// by choosing which chunk of memory a lane asks for: the lines that a read takes at once are on different banks.  Operands come
// either with k contiguous, or with their lines contiguous (the weights for dx; both for the weights' gradients): LDS holds lines of k then
// and the reads transpose 4 x 16 blocks.
// Loads go through buffer descriptors that end where the operand does: what lies behind the last line or the last k is 0 without a
// branch, and the stages past the last are loads of nothing.
//
// bf16 is bound by the matrix cores, whose clock falls to 1.65 GHz under them: 8192 rows 2048 -> 2 x 8192 bf16 take 424 to 487 us by card
// and temperature (1.3 to 1.13 PFLOP/s; the library's product by itself, without activation and join, 426), 69 % of the cycles a product.
// The gradients of 4096 rows 2048 <-> 2 x 5632, dx and the weights', 365 (1.03 PFLOP/s; the library's two 344): there operands whose lines
// are contiguous take twice as many reads of LDS, and a product is on its way in 47 % of the cycles; the ends of these 256-wide tiles, a
// bf16 and a fp32 one in one kernel, spill 178 registers, which shows in 108 MB written for 63 MB of results.  Four stages of 128-wide
// tiles in place of two, and tiles of 64 rows, were slower.  fp32: 8192 rows 2048 <-> 2048 3010 us backward, projections too (137 of 153
// TFLOP/s); 1156 rows 160 -> 2 x 960 17.5 for 4.6 of products, 285 tiles of five stages on 256 compute units.
#include <algorithm>

#include "gated.h"

namespace wcc {
namespace {

constexpr uint32_t kNowhere = 0x80000000u;  // beyond any descriptor here

using Rsrc = __amdgpu_buffer_rsrc_t;
__device__ __forceinline__ Rsrc buffer(const char *p, int64_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), 0, (int)(uint32_t)max(bytes, (int64_t)0), 0x00020000);
}
__device__ __forceinline__ void buffer_to_lds(Rsrc r, uint32_t off, unsigned char *to) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 16, off, 0, 0, 0);
}

// An operand in memory as a tile sees it.
//   along:  line l at p + l * ld, k contiguous; `lines` of them there, `k` long
//   across: k at p + k * ld, lines contiguous; `lines` of them there
// In bytes but for the counts.  Two halves: along, lines in turns of 32 from p[0] and p[1] (the two weights); across, k from `turn` on in
// p[1], from its first line on (dx: the two weights again), and from `again` on the same once more (second parts).
struct Operand {
  const char *p[2];
  int64_t ld;
  int64_t lines, k;
  int64_t turn, again;
};

template <class T, int B, bool ACROSS, bool TURNS>
struct Feed {
  static constexpr int Size = sizeof(T), VE = 16 / Size, KS = kLine / Size;  // KS: k of a stage
  static constexpr int Bytes = B * kLine, L = Bytes / 4096;                  // of a stage; loads of a wave
  static constexpr int C = B / VE, R = 64 / C;                               // across: chunks of a line of k, lines of a load
  static constexpr int PerLoad = ACROSS ? R : 8;
  static_assert(!ACROSS || Size == 4 || C >= 16, "keys of lines reach chunk 15");
  uint32_t off[2], at[2];  // the lane's places in loads of even and odd number; at: this stage's (along)
  int chunk[2];
  uint32_t step;
  Rsrc r[2];

  __device__ __forceinline__ void aim(const Operand &o) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    step = (uint32_t)(PerLoad * o.ld);
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if constexpr (ACROSS) {
        const int row = b * R + lane / C;
        chunk[b] = 0;
        off[b] = (uint32_t)((wv * L * R + lane / C) * o.ld + ((lane % C) ^ (Size == 2 ? (row & 3) * 4 : 0)) * 16);
      } else {
        const int row = b * 8 + lane / 8;
        chunk[b] = (lane % 8) ^ chunk_key(row);
        // (in turns of 32 lines a wave's loads are at the lines of both halves that its 64 lie in, or of the one that its 32 lie in)
        const int first = TURNS ? (B == 256 ? wv * 32 : (wv >> 1) * 32) : wv * L * 8;  // (TURNS: B is 128 or 256)
        off[b] = (uint32_t)((first + lane / 8) * o.ld + chunk[b] * 16);
      }
    }
    if constexpr (!ACROSS) {
      const int64_t bytes = o.lines > 0 ? (min(o.lines, (int64_t)B) - 1) * o.ld + o.k * Size : 0;
      r[0] = buffer(o.p[0], bytes);
      if constexpr (TURNS) {
        r[1] = buffer(o.p[1], bytes);
        if (B == 128 && (wv & 1)) r[0] = r[1];
      }
    }
  }
  // before the loads of a stage
  __device__ __forceinline__ void turn_to(const Operand &o, int64_t stage) {
    int64_t k = stage * KS;
    if constexpr (ACROSS) {
      const char *p = o.p[0];
      if constexpr (TURNS) {
        if (k >= o.again) k -= o.again;
        if (k >= o.turn) p = o.p[1], k -= o.turn;
      }
      const int64_t n = min(o.k - k, (int64_t)KS);
      const bool some = n > 0 && o.lines > 0;
      r[0] = buffer(some ? p + k * o.ld : p, some ? (n - 1) * o.ld + min(o.lines, (int64_t)B) * Size : 0);
    } else {
      const int64_t left = o.k - k;
#pragma unroll
      for (int b = 0; b < 2; ++b) at[b] = chunk[b] * VE < left ? off[b] + (uint32_t)(k * Size) : kNowhere;
    }
  }
  template <int i>
  __device__ __forceinline__ void load(unsigned char *to) const {
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned char *place = to + (wv * L + i) * 1024;
    if constexpr (ACROSS) {
      buffer_to_lds(r[0], off[i & 1] + i * step, place);
    } else {
      // (turns: the second half of a wave's loads is at the other weight's lines)
      constexpr int n = TURNS && B == 256 ? i % (L / 2) : i, which = TURNS && B == 256 ? i / (L / 2) : 0;
      buffer_to_lds(r[which], at[i & 1] + n * step, place);
    }
  }
};

// The barrier by itself (a fence would wait for all loads); the clobbers keep the reads of LDS on their sides of it.
__device__ __forceinline__ void bare_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
// all but the last n loads of every wave have arrived
template <int n>
__device__ __forceinline__ void arrived() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
  bare_barrier();
}

// The first operand of the matrix cores is W (outputs), the second X (rows): a lane has one row's results, four neighbouring outputs at a
// time.
// TWO: from stage `second` on X is of second parts, by what is finite in W.
template <class T, int BT, int BO, bool XA, bool WA, bool XTURNS, bool WTURNS, bool TWO>
struct Gemm {
  static constexpr int WT = 2, WO = 2, ET = BT / WT / 32, EO = BO / WO / 32;
  using X = Feed<T, BT, XA, XTURNS>;
  using W = Feed<T, BO, WA, WTURNS>;
  static constexpr int XL = X::L, WL = W::L, L = XL + WL;
  struct Operands {
    u32x4 x[ET], w[EO];
  };
  X x;
  W w;
  int64_t second;

  template <int from, int to>
  __device__ __forceinline__ void load(unsigned char *xs, unsigned char *ws) const {
    if constexpr (from < to) {
      if constexpr (from < XL) x.template load<from>(xs);
      else w.template load<from - XL>(ws);
      load<from + 1, to>(xs, ws);
    }
  }
  // 32 lines from `line` on, the k of a step, of lines of k that are B lines wide
  template <int B>
  __device__ static __forceinline__ u32x4 across(const unsigned char *s, int line, int step) {
    const int lane = threadIdx.x & 63;
    u32x4 v;
    if constexpr (sizeof(T) == 4) {
      const unsigned char *at = s + (step * 8 + (lane >> 5) * 4) * (B * 4) + (line + (lane & 31)) * 4;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const uint32_t *>(at + i * (B * 4));
    } else {
      const int g = lane >> 4, q = lane & 15;
      const int n = line + (g & 1) * 16 + (q & 3) * 4, kk = step * 16 + (g >> 1) * 8 + (q >> 2);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int row = kk + h * 4;
        const uint2 u = turned(s + row * (B * 2) + (((n >> 3) ^ ((row & 3) * 4)) << 4) + (n & 7) * 2);
        v[2 * h] = u.x, v[2 * h + 1] = u.y;
      }
    }
    return v;
  }
  __device__ __forceinline__ void fetch(const unsigned char *xs, const unsigned char *ws, int step, int64_t stage, Operands &f) const {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
    const int tw = (wv / WO) * (ET * 32), ow = (wv % WO) * (EO * 32);
#pragma unroll
    for (int e = 0; e < EO; ++e) f.w[e] = WA ? across<BO>(ws, ow + e * 32, step) : chunk_of(ws, ow + e * 32 + ln, step * 2 + half);
#pragma unroll
    for (int r = 0; r < ET; ++r) f.x[r] = XA ? across<BT>(xs, tw + r * 32, step) : chunk_of(xs, tw + r * 32 + ln, step * 2 + half);
    if constexpr (TWO) {
      if (stage >= second) {
#pragma unroll
        for (int e = 0; e < EO; ++e) f.w[e] = finite_of(f.w[e]);
      }
    }
  }
  __device__ static __forceinline__ void multiply(const Operands &f, f32x16 (&acc)[EO][ET]) {
#pragma unroll
    for (int e = 0; e < EO; ++e)
#pragma unroll
      for (int r = 0; r < ET; ++r) acc[e][r] = mma<T>(f.w[e], f.x[r], acc[e][r]);
  }
  // The order of a step: its reads of LDS two at a time between the first products (the rest of which hide the last one's way),
  // its loads between the others, as far apart as they get: a load takes 16 cycles on its way out, a product 32.
  template <int reads, int loads>
  __device__ static __forceinline__ void spread() {
    constexpr int M = ET * EO, N = (reads + 1) / 2;
    if constexpr (M < 16 || sizeof(T) == 4) {  // (two workgroups a compute unit hide each other's)
      __builtin_amdgcn_sched_barrier(0);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      if (i < M) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    }
    constexpr int each = loads > 0 && M > N ? (M - N) / loads : 0;
#pragma unroll
    for (int i = 0; i < loads; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
      if (each > 0) __builtin_amdgcn_sched_group_barrier(0x008, each, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, M, 0);
    __builtin_amdgcn_sched_barrier(0);
  }
  // The stage in (xs, ws), whose first two steps' operands are on their way to f; the next one is in (xn, wn), and `later` is loaded
  // where this one was.
  __device__ __forceinline__ void stage(const Operand &xo, const Operand &wo, int64_t now, int64_t later, unsigned char *xs, unsigned char *ws,
                                        const unsigned char *xn, const unsigned char *wn, Operands (&f)[4], f32x16 (&acc)[EO][ET]) {
    constexpr int Reads = ET * (XA ? 2 : 1) + EO * (WA ? 2 : 1), L1 = (L + 2) / 3, L2 = 2 * L1;
    x.turn_to(xo, later), w.turn_to(wo, later);
    fetch(xs, ws, 2, now, f[2]);
    fetch(xs, ws, 3, now, f[3]);
    multiply(f[0], acc);
    spread<2 * Reads, 0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    bare_barrier();
    load<0, L1>(xs, ws);
    multiply(f[1], acc);
    spread<0, L1>();
    load<L1, L2>(xs, ws);
    multiply(f[2], acc);
    spread<0, L2 - L1>();
    arrived<L2>();
    fetch(xn, wn, 0, now + 1, f[0]);
    fetch(xn, wn, 1, now + 1, f[1]);
    load<L2, L>(xs, ws);
    multiply(f[3], acc);
    spread<2 * Reads, L - L2>();
  }
  // acc += the products over stages s0 .. s1
  __device__ __forceinline__ void run(const Operand &xo, const Operand &wo, int64_t s0, int64_t s1, unsigned char *xs0, unsigned char *ws0,
                                      unsigned char *xs1, unsigned char *ws1, f32x16 (&acc)[EO][ET]) {
    const int64_t none = (int64_t)1 << 40;  // (a stage of nothing)
    auto at = [&](int64_t s) { return s < s1 ? s : none; };
    x.aim(xo), w.aim(wo);
    Operands f[4];
    x.turn_to(xo, s0), w.turn_to(wo, s0);
    load<0, L>(xs0, ws0);
    x.turn_to(xo, at(s0 + 1)), w.turn_to(wo, at(s0 + 1));
    load<0, L>(xs1, ws1);
    arrived<L>();
    fetch(xs0, ws0, 0, s0, f[0]);
    fetch(xs0, ws0, 1, s0, f[1]);
    int64_t s = s0;
    for (; s + 1 < s1; s += 2) {
      stage(xo, wo, s, at(s + 2), xs0, ws0, xs1, ws1, f, acc);
      stage(xo, wo, s + 1, at(s + 3), xs1, ws1, xs0, ws0, f, acc);
    }
    if (s < s1) stage(xo, wo, s, none, xs0, ws0, xs1, ws1, f, acc);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing is on its way to LDS from here on
    bare_barrier();
  }
};

__device__ __forceinline__ uint2 narrow4(float a, float b, float c, float d) {
  return uint2{(uint32_t)narrow<bf16_t>(a) | (uint32_t)narrow<bf16_t>(b) << 16, (uint32_t)narrow<bf16_t>(c) | (uint32_t)narrow<bf16_t>(d) << 16};
}

// 32 rows of `Row` bytes that a wave has written to LDS in 8-byte pieces, exchanged by a key of the row (even, so that pairs of them stay
// together): 16 bytes a lane, f(row, byte in the row, the 16 bytes).  (A wave reads what it wrote itself: LDS is in order.)
template <int Row>
__device__ __forceinline__ int twist(int row) { return row % (Row / 16) * 2; }
template <int Row>
__device__ __forceinline__ void put(unsigned char *lds, int row, int piece, const uint2 &v) {
  *reinterpret_cast<uint2 *>(lds + row * Row + ((piece ^ twist<Row>(row)) << 3)) = v;
}
template <int Row, class F>
__device__ __forceinline__ void leave(const unsigned char *lds, F f) {
  constexpr int Lanes = Row / 16, Rows = 64 / Lanes;
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int r0 = 0; r0 < 32; r0 += Rows) {
    const int row = r0 + lane / Lanes, c = lane % Lanes;
    f(row, c * 16, *reinterpret_cast<const u32x4 *>(lds + row * Row + (((2 * c) ^ twist<Row>(row)) << 3)));
  }
}

// ---- the two projections -------------------------------------------------------------------------------------
// PARTS: a range of k, whose sums go to part [splits][rows][2][room].  NP: parts of dg and du in d (known here: a loop over p.parts makes
// the one that nearly all calls have 1 to 2 % slower, 560 to 571 us for 4096 rows 2048 <-> 2 x 5632).
template <class T, int BT, int BO, int ACT, bool BACK, bool PARTS, int NP = 1>
__global__ __launch_bounds__(256, BO == 128 ? 2 : 1) void gate_gemm_kernel(Gate<T> p, Operand x, Operand w, int64_t tiles_t, int tiles_o,
                                                                         int64_t chunk, float *__restrict__ part) {
  using G = Gemm<T, BT, BO, false, false, false, true, false>;
  constexpr int ET = G::ET, EO = G::EO, Pairs = EO / 2, Row = Pairs * 64;
  __shared__ __align__(1024) unsigned char xs0[G::X::Bytes], ws0[G::W::Bytes], xs1[G::X::Bytes], ws1[G::W::Bytes];
  const int64_t tiles = tiles_t * tiles_o, at = in_runs(blockIdx.x, gridDim.x), split = PARTS ? at / tiles : 0;
  int64_t tt;
  int to;
  tile_of(at - split * tiles, tiles_t, tiles_o, tt, to);
  const int64_t t0 = tt * BT;
  const int o0 = to * (BO / 2);
  x.p[0] += t0 * x.ld, x.lines -= t0;
  w.p[0] += o0 * w.ld, w.p[1] += o0 * w.ld, w.lines -= o0;
  w.lines = min(w.lines, (int64_t)(BO / 2));
  f32x16 acc[EO][ET] = {};
  G g;
  const int64_t stages = (x.k + G::X::KS - 1) / G::X::KS;
  g.run(x, w, split * chunk, PARTS ? min(stages, (split + 1) * chunk) : stages, xs0, ws0, xs1, ws1, acc);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  const int64_t tw = t0 + (wv / G::WO) * (ET * 32);
  const int ow = o0 + (wv % G::WO) * (Pairs * 32);
  unsigned char *own = wv == 0 ? xs0 : wv == 1 ? ws0 : wv == 2 ? xs1 : ws1;  // (8 KiB each at least)
  const int64_t blocks = (p.outs + kKept - 1) / kKept;
  if constexpr (PARTS) {
#pragma unroll
    for (int r = 0; r < ET; ++r) {
      const int64_t t = tw + r * 32 + ln;
      if (t >= p.rows) continue;
#pragma unroll
      for (int e = 0; e < EO; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int o = ow + (e >> 1) * 32 + result_line(i, half);
          float *q = part + ((split * p.rows + t) * 2 + (e & 1)) * p.room + o;
          if (o < p.room) *reinterpret_cast<f32x4_any *>(q) = f32x4_any{acc[e][r][i], acc[e][r][i + 1], acc[e][r][i + 2], acc[e][r][i + 3]};
        }
    }
    return;
  } else if constexpr (sizeof(T) == 4) {  // (bound by the matrix cores: straight to memory)
#pragma unroll
    for (int r = 0; r < ET; ++r)
#pragma unroll
      for (int j = 0; j < Pairs; ++j) {
        const f32x16 &ga = acc[2 * j][r], &ua = acc[2 * j + 1][r];  // (lines behind the last are 0)
        uint32_t m[2] = {0, 0};
        if (!BACK && p.codes) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            m[0] = max(m[0], __float_as_uint(ga[i]) & 0x7fffffffu);
            m[1] = max(m[1], __float_as_uint(ua[i]) & 0x7fffffffu);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) m[h] = step_of(max(m[h], (uint32_t)__shfl_xor((int)m[h], 32, 64)));
        }
        const int64_t t = tw + r * 32 + ln;
        if (t < p.rows) {
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            float gv[4] = {ga[i], ga[i + 1], ga[i + 2], ga[i + 3]}, uv[4] = {ua[i], ua[i + 1], ua[i + 2], ua[i + 3]};
            const int o = ow + j * 32 + result_line(i, half);
            if (o < p.room) finish<T, ACT, BACK>(p, t, o, gv, uv, m[0], m[1]);
          }
        }
      }
    return;
  } else {
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    const int64_t t = tw + r * 32 + ln;
    unsigned char *second = own + 32 * Row;
    if constexpr (BACK) {
#pragma unroll 1
      for (int part = 0; part < NP; ++part) {
        int outs = p.outs;
        if constexpr (NP > 1) asm volatile("" : "+s"(outs));  // (comparisons with it made anew for each part, or they would be held for both)
#pragma unroll
        for (int j = 0; j < Pairs; ++j) {
          const f32x16 &ga = acc[2 * j][r], &ua = acc[2 * j + 1][r];  // (lines behind the last are 0)
          const int o = ow + j * 32;
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const int at = o + result_line(i, half);
            float dg[4], du[4];
            uint2 top = {0, 0};
            if (t < p.rows && at < outs) {
              const bf16_t *q = p.dy + t * p.ldy + at;
              if (at + 4 <= outs) {
                const u32x2_any v = *reinterpret_cast<const u32x2_any *>(q);
                top = uint2{v.x, v.y};
              } else {
                top.x = q[0];
                if (at + 1 < outs) top.x |= (uint32_t)q[1] << 16;
                if (at + 2 < outs) top.y = q[2];
              }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float v, s;
              act_of<bf16_t, ACT>(ga[i + k], v, s);
              const uint32_t word = k < 2 ? top.x : top.y;
              const float dy = __uint_as_float(k & 1 ? word & 0xffff0000u : word << 16);
              dg[k] = dy * ua[i + k] * s, du[k] = dy * v;
              if (at + k >= outs) dg[k] = du[k] = 0.f;  // (what lies behind is 0)
              if (part > 0) dg[k] = left_of(dg[k], narrow<bf16_t>(dg[k])), du[k] = left_of(du[k], narrow<bf16_t>(du[k]));
            }
            put<Row>(own, ln, j * 8 + (i >> 1) + half, narrow4(dg[0], dg[1], dg[2], dg[3]));
            put<Row>(second, ln, j * 8 + (i >> 1) + half, narrow4(du[0], du[1], du[2], du[3]));
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
          leave<Row>(h ? second : own, [&](int row, int b, const u32x4 &v) {
            const int o = ow + b / 2;
            if (tw + r * 32 + row < p.rows && o < p.room)
              *reinterpret_cast<u32x4 *>(p.d + (((tw + r * 32 + row) * NP + part) * 2 + h) * p.room + o) = v;
          });
      }
    } else {
#pragma unroll
      for (int j = 0; j < Pairs; ++j) {
        const f32x16 &ga = acc[2 * j][r], &ua = acc[2 * j + 1][r];  // (lines behind the last are 0)
        if (p.codes) {
          uint32_t m[2] = {0, 0};
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            m[0] = max(m[0], __float_as_uint(ga[i]) & 0x7fffffffu);
            m[1] = max(m[1], __float_as_uint(ua[i]) & 0x7fffffffu);
          }
          const int64_t block = ow / kKept + j;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t b = step_of(max(m[h], (uint32_t)__shfl_xor((int)m[h], 32, 64)));
            const float per = per_step(b);
            const f32x16 &v = h ? ua : ga;
            if (half == h && t < p.rows && block < blocks) p.steps[((int64_t)h * p.rows + t) * blocks + block] = (uint8_t)b;
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
              const uint32_t c = b == 255 ? 0 : codes_of(v[i], v[i + 1], v[i + 2], v[i + 3], per);
              *reinterpret_cast<uint32_t *>(second + (h * Pairs + j) * 1024 + ln * 32 + result_line(i, half)) = c;
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          float f[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            float v, s;
            act_of<bf16_t, ACT>(ga[i + k], v, s);
            f[k] = v * ua[i + k];
          }
          put<Row>(own, ln, j * 8 + (i >> 1) + half, narrow4(f[0], f[1], f[2], f[3]));
        }
      }
      leave<Row>(own, [&](int row, int b, const u32x4 &v) {
        const int o = ow + b / 2;
        if (tw + r * 32 + row < p.rows && o < p.outs) store_part<bf16_t>(p.y + (tw + r * 32 + row) * p.ldy + o, p.outs - o, v);
      });
      if (p.codes) {  // blocks of 32 rows of 32 bytes: 16 bytes a lane
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < Pairs; ++j) {
            const int row = lane / 2, b = lane % 2 * 16;
            const int64_t t2 = tw + r * 32 + row, block = ow / kKept + j;
            const u32x4 v = *reinterpret_cast<const u32x4 *>(second + (h * Pairs + j) * 1024 + row * 32 + b);
            if (t2 < p.rows && block < blocks) *reinterpret_cast<u32x4 *>(p.codes + (((int64_t)h * p.rows + t2) * blocks + block) * kKept + b) = v;
          }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  }
}

// ---- dx and the weights' gradients -----------------------------------------------------------------------------
template <class T>
struct Result {
  T *out[2];  // rows from `turn` on go to out[1], from its first on
  int64_t ld, rows, outs, turn;
  float *part;     // PARTS: [splits][turns * rows][outs]
};

template <class T>
struct Job {
  Result<T> r;
  Operand x, w;
  int64_t tiles_t;
  int tiles_o, splits;
  int64_t chunk, stages, from;  // from: the stage that second parts begin with
  int64_t blocks;               // 0: none
};

template <class T, int BT, int BO, bool XA, bool TWO>
__device__ __forceinline__ void product_tile(const Job<T> &job, int64_t block, unsigned char *xs0, unsigned char *ws0, unsigned char *xs1,
                                             unsigned char *ws1) {
  using G = Gemm<T, BT, BO, XA, true, XA && TWO, !XA || TWO, TWO>;
  constexpr int ET = G::ET, EO = G::EO, Row = EO * 64;
  const Result<T> &p = job.r;
  Operand x = job.x, w = job.w;
  const int64_t tiles = job.tiles_t * job.tiles_o, split = block / tiles;
  int64_t tt;
  int to;
  tile_of(block % tiles, job.tiles_t, job.tiles_o, tt, to);
  // rows of the second half begin with a tile of their own
  const int64_t tiles_half = (p.rows + BT - 1) / BT, second = tt >= tiles_half ? 1 : 0;
  const int64_t t0 = (tt - second * tiles_half) * BT;
  const int64_t o0 = (int64_t)to * BO;
  if constexpr (XA) x.p[0] += (second * p.turn + t0) * (int64_t)sizeof(T), x.p[1] += (second * p.turn + t0) * (int64_t)sizeof(T);
  else x.p[0] += t0 * x.ld;
  x.lines -= t0;
  w.p[0] += o0 * sizeof(T), w.p[1] += o0 * sizeof(T), w.lines -= o0;
  f32x16 acc[EO][ET] = {};
  G g;
  g.second = job.from;
  g.run(x, w, split * job.chunk, min(job.stages, (split + 1) * job.chunk), xs0, ws0, xs1, ws1, acc);
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  const int64_t tw = t0 + (wv / G::WO) * (ET * 32), ow = o0 + (wv % G::WO) * (EO * 32);
  unsigned char *own = wv == 0 ? xs0 : wv == 1 ? ws0 : wv == 2 ? xs1 : ws1;
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    if (sizeof(T) == 4 || job.splits > 1) {
      const int64_t t = tw + r * 32 + ln, halves = p.out[1] ? 2 : 1;
      if (t < p.rows) {
        float *q;
        if (job.splits > 1) q = p.part + ((split * halves + second) * p.rows + t) * p.outs;
        else q = reinterpret_cast<float *>(p.out[second]) + t * p.ld;
#pragma unroll
        for (int e = 0; e < EO; ++e)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const int64_t o = ow + e * 32 + result_line(i, half);
            if (o + 4 <= p.outs) {
              *reinterpret_cast<f32x4_any *>(q + o) = f32x4_any{acc[e][r][i], acc[e][r][i + 1], acc[e][r][i + 2], acc[e][r][i + 3]};
            } else {
#pragma unroll
              for (int k = 0; k < 3; ++k)
                if (o + k < p.outs) q[o + k] = acc[e][r][i + k];
            }
          }
      }
    } else if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < EO; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          put<Row>(own, ln, e * 8 + (i >> 1) + half, narrow4(acc[e][r][i], acc[e][r][i + 1], acc[e][r][i + 2], acc[e][r][i + 3]));
      leave<Row>(own, [&](int row, int b, const u32x4 &v) {
        const int64_t o = ow + b / 2, t = tw + r * 32 + row;
        if (t < p.rows && o < p.outs) store_part<bf16_t>(p.out[second] + t * p.ld + o, (int)min(p.outs - o, (int64_t)8), v);
      });
    }
    __builtin_amdgcn_sched_barrier(0);
  }
}

// dx's tiles, the longer ones, before the weights'
template <class T, int BT, int BO, bool TWO>
__global__ __launch_bounds__(256, BO == 64 ? 4 : BO == 128 ? 2 : 1) void product_gemm_kernel(Job<T> dx, Job<T> dw) {
  __shared__ __align__(1024) unsigned char xs0[BT * kLine], ws0[BO * kLine], xs1[BT * kLine], ws1[BO * kLine];
  const int64_t b = blockIdx.x;
  if (b < dx.blocks) product_tile<T, BT, BO, false, TWO>(dx, in_runs(b, dx.blocks), xs0, ws0, xs1, ws1);
  else product_tile<T, BT, BO, true, TWO>(dw, in_runs(b - dx.blocks, dw.blocks), xs0, ws0, xs1, ws1);
}

// Sums of ranges of k joined in their order: dx, then the one or two of the weights.
template <class T>
__global__ __launch_bounds__(256) void product_gemm_join_kernel(Job<T> dx, Job<T> dw, int first) {
  const int which = first + blockIdx.y, h = which > 0 ? which - 1 : 0;
  const Job<T> &job = which == 0 ? dx : dw;
  const Result<T> &p = job.r;
  const int64_t all = p.rows * p.outs, halves = p.out[1] ? 2 : 1;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < all; i += (int64_t)gridDim.x * 1024) {
    f32x4_any v = {};
    const int n = (int)min(all - i, (int64_t)4);
    if (n == 4) {
#pragma unroll 4
      for (int s = 0; s < job.splits; ++s) v += *reinterpret_cast<const f32x4_any *>(p.part + (s * halves + h) * all + i);
    } else {
      for (int s = 0; s < job.splits; ++s)
        for (int j = 0; j < n; ++j) v[j] += p.part[(s * halves + h) * all + i + j];
    }
    int64_t row = i / p.outs, o = i - row * p.outs;
    for (int j = 0; j < n; ++j) {
      p.out[h][row * p.ld + o] = narrow<T>(v[j]);
      if (++o == p.outs) o = 0, ++row;
    }
  }
}

bool on_16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t tiles(int64_t n, int64_t size) { return (n + size - 1) / size; }

template <class F>
hipError_t by_act(int act, F f) {
  switch (act) {
    case WCC_ACT_RELU: return f(std::integral_constant<int, WCC_ACT_RELU>());
    case WCC_ACT_SILU: return f(std::integral_constant<int, WCC_ACT_SILU>());
    case WCC_ACT_GELU: return f(std::integral_constant<int, WCC_ACT_GELU>());
    default: return f(std::integral_constant<int, WCC_ACT_NONE>());
  }
}

// How the products of a backward pass are cut.  dx: rows x C_in over 2 room; the weights' gradients, both: 2 C_out x C_in over the rows.
// Each workgroup has about as many stages as there are for every place (256, or 512 and 1024 of the smaller tiles).
struct ProductPlan {
  int bt, bo;
  struct Part {
    int64_t stages, chunk;
    int splits;
    size_t bytes;
  } dx, dw;
};
ProductPlan plan_of(int64_t rows, int64_t C_in, int64_t C_out, int64_t room, int parts, int size) {
  ProductPlan p = {};
  const int each = kLine / size;
  p.dx.stages = parts * 2 * room / each, p.dw.stages = parts * tiles(rows, each);
  auto tiles_of = [&](int64_t bt, int64_t bo, int64_t &dx, int64_t &dw) {
    dx = tiles(rows, bt) * tiles(C_in, bo), dw = 2 * tiles(C_out, bt) * tiles(C_in, bo);
    return dx + dw;
  };
  int64_t dx, dw;
  p.bt = p.bo = 128;
  // (the larger ones where three quarters of the compute units have one, and four fifths of them lie within the results)
  if (size == 2 && tiles_of(256, 256, dx, dw) >= 200 && 5 * C_in * (rows + 2 * C_out) >= 4 * 65536 * (dx + dw)) p.bt = p.bo = 256;
  // (fp32: the smaller ones where the larger are few, and where a fifth of those would lie past C_in, 40000 rows 160 <-> 960 in 928 us against
  // 1123; 8192 rows 320 <-> 640 take 222 in them and 219 in the larger, 4096 rows 512 <-> 2048 426 and 409, 1024 <-> 2048 820 and 762)
  if (size == 4 && (tiles_of(128, 128, dx, dw) < 192 || 5 * C_in <= 4 * 128 * tiles(C_in, 128))) p.bt = p.bo = 64;
  tiles_of(p.bt, p.bo, dx, dw);
  // Ranges for the shortest time by a rough count: a workgroup takes its stages and as much as four for its beginning and end; more of them
  // than there are places wait.
  const int64_t slots = p.bt == 256 ? 256 : p.bt == 64 ? 1024 : 512, mean = std::max<int64_t>(tiles(dx * p.dx.stages + dw * p.dw.stages, slots), 4);
  int64_t best = 0;
  for (int i = 0; i < 16; ++i) {
    const int64_t has = mean + i * mean / 8;
    auto cut = [&](int64_t stages) { return std::min<int64_t>(std::max<int64_t>((stages + has / 2) / has, 1), 64); };
    const int64_t n = cut(p.dx.stages), m = cut(p.dw.stages), blocks = dx * n + dw * m;
    const int64_t a = tiles(p.dx.stages, n) + 4, b = tiles(p.dw.stages, m) + 4;
    const int64_t time = blocks <= slots ? std::max(a, b) : std::max(std::max(a, b), (dx * n * a + dw * m * b) / slots + std::min(a, b));
    if (best == 0 || time < best) {
      best = time;
      p.dx.chunk = tiles(p.dx.stages, n), p.dw.chunk = tiles(p.dw.stages, m);
    }
  }
  p.dx.splits = (int)tiles(p.dx.stages, p.dx.chunk), p.dw.splits = (int)tiles(p.dw.stages, p.dw.chunk);
  p.dx.bytes = p.dx.splits > 1 ? (size_t)p.dx.splits * rows * C_in * sizeof(float) : 0;
  p.dx.bytes = (p.dx.bytes + 255) / 256 * 256;
  p.dw.bytes = p.dw.splits > 1 ? (size_t)p.dw.splits * 2 * C_out * C_in * sizeof(float) : 0;
  return p;
}

// The two projections: tiles of 256 x 128 outputs of both where three quarters of the compute units have one and
// their end is not most of the work, else of 128 x 64 (fp32, few:
// of 64 x 64).
struct GatePlan {
  int bt, bo, splits;
  int64_t stages, chunk;
};
GatePlan gate_plan(int64_t rows, int64_t outs, int64_t k, int size) {
  GatePlan p = {};
  p.stages = tiles(k, kLine / size);
  p.bt = p.bo = 128;
  if (size == 2 && p.stages >= 12 && tiles(rows, 256) * tiles(outs, 128) >= 200) p.bt = p.bo = 256;
  if (size == 4 && tiles(rows, 128) * tiles(outs, 64) < 256) p.bt = 64;
  const int64_t n = tiles(rows, p.bt) * tiles(outs, p.bo / 2);
  // Ranges for the shortest time by a rough count, in stages: rounds of 256, four for a workgroup's beginning and end, and the join, 4 us and
  // the sums written and read at 4 TB/s (a stage takes 0.35 us, of fp32 0.93 or 1.86).
  int64_t want = 1;
  if (p.bt < 256) {
    const double stage = size == 2 ? 0.35 : p.bt == 64 ? 0.93 : 1.86, sums = 16e-6 * rows * room_of(outs) / 4 / stage;
    double best = 0;
    for (int64_t splits = 1; splits <= 16 && (splits == 1 || p.stages >= 4 * splits); ++splits) {
      const double time = tiles(n * splits, 256) * (tiles(p.stages, splits) + 4.0) + (splits > 1 ? 4 / stage + sums * splits : 0.0);
      if (splits == 1 || time < best) best = time, want = splits;
    }
  }
  p.chunk = tiles(p.stages, want);
  p.splits = (int)tiles(p.stages, p.chunk);
  return p;
}

}  // namespace

// 16-byte loads, tiles within a descriptor
bool gemm_takes(const void *p, int64_t ld, int64_t width, int size) {
  const int each = 16 / size;
  return on_16(p) && ld % each == 0 && ld * size < 1 << 22 && width % each == 0;
}

template <class T>
hipError_t gemm_gate(const Gate<T> &p, int act, bool back, const Side<T> &x, const T *w_gate, const T *w_up, int64_t ldw, int64_t k,
                     float *part, hipStream_t s) {
  const GatePlan plan = gate_plan(p.rows, p.outs, k, sizeof(T));
  Operand xo = {}, wo = {};
  xo.p[0] = reinterpret_cast<const char *>(x.p), xo.ld = x.s * sizeof(T), xo.lines = x.lines, xo.k = k;
  wo.p[0] = reinterpret_cast<const char *>(w_gate), wo.p[1] = reinterpret_cast<const char *>(w_up), wo.ld = ldw * sizeof(T);
  wo.lines = p.outs, wo.k = k;
  return by_act(plan.splits > 1 ? (int)WCC_ACT_NONE : act, [&](auto a) {  // (ranges: sums as they are)
    constexpr int ACT = decltype(a)::value;
    auto go = [&](auto bt, auto bo) {
      constexpr int BT = decltype(bt)::value, BO = decltype(bo)::value;
      const int64_t tiles_t = tiles(p.rows, BT);
      const int tiles_o = (int)tiles(p.outs, BO / 2);
      const unsigned n = (unsigned)(tiles_t * tiles_o * plan.splits);
      if (plan.splits > 1) {
        if constexpr (BO == 128 && ACT == WCC_ACT_NONE) gate_gemm_kernel<T, BT, BO, ACT, false, true><<<n, 256, 0, s>>>(p, xo, wo, tiles_t, tiles_o, plan.chunk, part);
      } else if (back && sizeof(T) == 2 && p.parts == 2) {
        if constexpr (sizeof(T) == 2) gate_gemm_kernel<T, BT, BO, ACT, true, false, 2><<<n, 256, 0, s>>>(p, xo, wo, tiles_t, tiles_o, 0, nullptr);
      } else if (back) {
        gate_gemm_kernel<T, BT, BO, ACT, true, false><<<n, 256, 0, s>>>(p, xo, wo, tiles_t, tiles_o, 0, nullptr);
      } else {
        gate_gemm_kernel<T, BT, BO, ACT, false, false><<<n, 256, 0, s>>>(p, xo, wo, tiles_t, tiles_o, 0, nullptr);
      }
    };
    const std::integral_constant<int, 256> L;
    const std::integral_constant<int, 128> M;
    const std::integral_constant<int, 64> S;
    if constexpr (sizeof(T) == 2) {
      if (plan.bt == 256) go(L, L);
      else go(M, M);
    } else {
      if (plan.bt == 64) go(S, M);
      else go(M, M);
    }
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || plan.splits == 1 ? e : join_gate<T>(p, act, back, plan.splits, part, s);
  });
}

size_t gemm_gate_parts(int64_t rows, int64_t outs, int64_t k, int size) {
  const GatePlan p = gate_plan(rows, outs, k, size);
  return p.splits > 1 ? (size_t)p.splits * rows * 2 * room_of(outs) * sizeof(float) : 0;
}
size_t gemm_back_parts(int64_t rows, int64_t C_in, int64_t C_out, int parts, int size) {
  const ProductPlan p = plan_of(rows, C_in, C_out, room_of(C_out), parts, size);
  return p.dx.bytes + p.dw.bytes;
}

template <class T>
hipError_t gemm_back(const Backward<T> &b, float *part, hipStream_t s) {
  const int64_t size = sizeof(T), never = (int64_t)1 << 60;
  const ProductPlan p = plan_of(b.rows, b.C_in, b.C_out, b.room, b.parts, sizeof(T));  // (whichever gradients are asked for)
  Job<T> dx = {}, dw = {};
  if (b.dx) {
    Operand &x = dx.x, &w = dx.w;
    x.p[0] = reinterpret_cast<const char *>(b.d), x.ld = b.parts * 2 * b.room * size, x.lines = b.rows, x.k = b.parts * 2 * b.room;
    w.p[0] = reinterpret_cast<const char *>(b.w_gate), w.p[1] = reinterpret_cast<const char *>(b.w_up);
    w.ld = b.ldw * size, w.lines = b.ldw, w.k = b.C_out, w.turn = b.room, w.again = 2 * b.room;
    dx.r = Result<T>{{b.dx, nullptr}, b.ld, b.rows, b.C_in, 0, part};
    dx.from = 2 * b.room * size / kLine;
    dx.tiles_t = tiles(b.rows, p.bt), dx.tiles_o = (int)tiles(b.C_in, p.bo);
    dx.splits = p.dx.splits, dx.chunk = p.dx.chunk, dx.stages = p.dx.stages;
    dx.blocks = dx.tiles_t * dx.tiles_o * dx.splits;
  }
  if (b.dw_gate || b.dw_up) {
    Operand &x = dw.x, &w = dw.w;
    const int halves = b.dw_gate && b.dw_up ? 2 : 1;
    const T *d = b.dw_gate ? b.d : b.d + b.room;
    const int64_t turn = p.dw.stages / b.parts * (kLine / size);  // rows of a part, in whole stages
    x.p[0] = reinterpret_cast<const char *>(d), x.p[1] = reinterpret_cast<const char *>(d + 2 * b.room);
    x.ld = b.parts * 2 * b.room * size, x.lines = b.room, x.k = b.rows, x.turn = turn, x.again = never;
    w.p[0] = w.p[1] = reinterpret_cast<const char *>(b.x), w.ld = b.ldx * size, w.lines = b.width, w.k = b.rows, w.turn = turn, w.again = never;
    dw.r = Result<T>{{b.dw_gate ? b.dw_gate : b.dw_up, halves == 2 ? b.dw_up : nullptr}, b.C_in, b.C_out, b.C_in, b.room,
                     part + p.dx.bytes / sizeof(float)};
    dw.from = p.dw.stages / b.parts;
    dw.tiles_t = halves * tiles(b.C_out, p.bt), dw.tiles_o = (int)tiles(b.C_in, p.bo);
    dw.splits = p.dw.splits, dw.chunk = p.dw.chunk, dw.stages = p.dw.stages;
    dw.blocks = dw.tiles_t * dw.tiles_o * dw.splits;
  }
  const unsigned n = (unsigned)(dx.blocks + dw.blocks);
  if (n == 0) return hipSuccess;
  if constexpr (sizeof(T) == 2) {
    if (p.bt == 256 && b.parts == 2) product_gemm_kernel<T, 256, 256, true><<<n, 256, 0, s>>>(dx, dw);
    else if (p.bt == 256) product_gemm_kernel<T, 256, 256, false><<<n, 256, 0, s>>>(dx, dw);
    else if (b.parts == 2) product_gemm_kernel<T, 128, 128, true><<<n, 256, 0, s>>>(dx, dw);
    else product_gemm_kernel<T, 128, 128, false><<<n, 256, 0, s>>>(dx, dw);
  } else {
    if (p.bt == 64) product_gemm_kernel<T, 64, 64, false><<<n, 256, 0, s>>>(dx, dw);
    else product_gemm_kernel<T, 128, 128, false><<<n, 256, 0, s>>>(dx, dw);
  }
  const bool join_dx = dx.splits > 1, join_dw = dw.splits > 1;
  if (join_dx || join_dw) {
    const int64_t most = std::max(join_dx ? dx.r.rows * dx.r.outs : 0, join_dw ? dw.r.rows * dw.r.outs : 0);
    const int first = join_dx ? 0 : 1, count = (join_dx ? 1 : 0) + (join_dw ? dw.r.out[1] ? 2 : 1 : 0);
    product_gemm_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(tiles(most, 1024), 4096), count), 256, 0, s>>>(dx, dw, first);
  }
  return hipGetLastError();
}

#define WCC_GEMM(T)                                                                                                                          \
  template hipError_t gemm_gate<T>(const Gate<T> &, int, bool, const Side<T> &, const T *, const T *, int64_t, int64_t, float *, hipStream_t); \
  template hipError_t gemm_back<T>(const Backward<T> &, float *, hipStream_t);
WCC_GEMM(float)
WCC_GEMM(bf16_t)
#undef WCC_GEMM

}  // namespace wcc

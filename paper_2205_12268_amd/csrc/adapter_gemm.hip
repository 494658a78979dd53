// The projection for many rows of bf16: the matrix cores fed from LDS, which loads go to straight from memory.
//
// A workgroup of four waves has BT rows x BO outputs and two stages of 64 k in LDS; loads (16 bytes a lane) go there without
// passing registers.  A wave's operands of a whole stage fit its registers beside the results, so a stage's half of LDS is
// free after a quarter of its products: from there on the loads of the stage after the next go out, one between every three
// products.  Two barriers a stage: LDS is read; the next stage is there.
// LDS has no padding (such a load writes 1 KiB in a row), so the 16-byte chunks of a line are exchanged by a key of the line, at
// the load by choosing which chunk of memory a lane asks for: the 16 lines that a read takes at once are on different banks.
// Where W's outputs are contiguous and not its k (NN), LDS holds lines of k and the reads transpose 4 x 16 blocks.
// The first operand of the matrix cores is W, the second x: a lane has one row's results, four neighbouring outputs at a time,
// which leave through LDS as whole lines.
// The last stages, which the end of k cuts, are not overlapped; chunks past the end (and, NN, past the last output) come from 16
// bytes of zeros.
// Bound by the matrix cores and what feeds them: 8192 rows, 4096 -> 4096 236 us on inputs that stay in the caches (1.17 PFLOP/s), the
// other order of W 225 (1.22), 8192 in all three 0.90 ms (1.22 PFLOP/s); 128 x 128 tiles 1024 rows, 4096 -> 4096 44 us; with 8 adapters
// of rank 32 and inputs in turn the 8192 rows take 259 to 287.  24 adapters in mixed order add 17 us to 1024 rows.  Not kept: four stages of 32 k (300 us), bands of 4 or 16 row tiles (270 to 277), a priority for waves that multiply.
#include "adapter.h"

namespace wcc {
namespace {

constexpr int Line = kLine, Chunks = kChunks, PerLoad = 1024 / Line;  // lines of a load

// FULL: a tile lies within the rows and outputs (the last ones are moved back, over others: rows, whose results they repeat, are
// stored twice, outputs by the one tile whose they are, since where an adapter is not finite the order of its sums goes by all outputs
// of a wave).  With NN, outputs count up to whole chunks of 8 there, which W's rows hold: its loads begin at a chunk.
template <int BT, int BO, int WT, bool NN, bool FULL>
struct Gemm {
  static constexpr int Waves = 4, WO = Waves / WT;
  static constexpr int ET = BT / WT / 32, EO = BO / WO / 32;            // 32 x 32 results of a wave
  static constexpr int XB = BT * kK * 2, WB = BO * kK * 2;              // bytes of a stage
  static constexpr int XL = XB / 1024 / Waves, WL = WB / 1024 / Waves;  // loads of a wave
  static constexpr int C = BO / 8, R = 64 / C;                          // NN: chunks of a line of k, lines of a load

  // Where a wave's loads begin.  Load i is at x + i * x_step + k, and a lane's place in it depends on i's last bit alone; without
  // FULL the rows are held to the last one, each load's by itself.
  struct Loader {
    const char *x, *w;
    int64_t x_step, w_step, w_stage;  // bytes between loads; NN: between stages
    uint32_t xo[2], wo[2];
    const char *xr[FULL ? 1 : XL], *wr[FULL || NN ? 1 : WL];
    int o_left;                       // NN: outputs from o0 on
  };

  __device__ static __forceinline__ void aim(const Project<bf16_t> &p, int64_t t0, int o0, int k0, Loader &l) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    l.x = reinterpret_cast<const char *>(p.x + (t0 + wv * XL * PerLoad) * p.ldx + k0);
    l.x_step = (int64_t)PerLoad * p.ldx * 2;
    l.o_left = p.outs - o0;
    if constexpr (NN) {
      l.w = reinterpret_cast<const char *>(p.w + (int64_t)(k0 + wv * WL * R) * p.wk + o0);
      l.w_step = R * p.wk * 2;
      l.w_stage = kK * p.wk * 2;
    } else {
      l.w = reinterpret_cast<const char *>(p.w + (int64_t)(o0 + wv * WL * PerLoad) * p.wo + k0);
      l.w_step = PerLoad * p.wo * 2;
      l.w_stage = Line;
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int row = b * PerLoad + lane / Chunks, chunk = (lane % Chunks) ^ chunk_key(row);
      l.xo[b] = (uint32_t)((lane / Chunks) * p.ldx * 2 + chunk * 16);
      if constexpr (NN) l.wo[b] = (uint32_t)((lane / C) * p.wk * 2 + ((lane % C) ^ (((b * R + lane / C) & 3) * 4)) * 16);
      else l.wo[b] = (uint32_t)((lane / Chunks) * p.wo * 2 + chunk * 16);
    }
    if constexpr (!FULL) {
#pragma unroll
      for (int i = 0; i < XL; ++i) {
        const int row = (wv * XL + i) * PerLoad + lane / Chunks, chunk = (lane % Chunks) ^ chunk_key(row);
        l.xr[i] = reinterpret_cast<const char *>(p.x + min(t0 + row, p.rows - 1) * p.ldx + k0 + chunk * 8);
      }
      if constexpr (!NN) {
#pragma unroll
        for (int i = 0; i < WL; ++i) {
          const int row = (wv * WL + i) * PerLoad + lane / Chunks, chunk = (lane % Chunks) ^ chunk_key(row);
          l.wr[i] = reinterpret_cast<const char *>(p.w + (int64_t)min(o0 + row, p.outs - 1) * p.wo + k0 + chunk * 8);
        }
      }
    }
  }

  __device__ static __forceinline__ const char *x_at(const Loader &l, int i, int stage) {
    if constexpr (FULL) return l.x + i * l.x_step + (int64_t)stage * Line + l.xo[i & 1];
    else return l.xr[i] + (int64_t)stage * Line;
  }
  __device__ static __forceinline__ const char *w_at(const Loader &l, int i, int stage) {
    if constexpr (FULL || NN) return l.w + i * l.w_step + stage * l.w_stage + l.wo[i & 1];
    else return l.wr[i] + (int64_t)stage * Line;
  }
  // NN without FULL: whether the lane's chunk of load i lies before the last output
  __device__ static __forceinline__ bool w_there(const Loader &l, int i) {
    const int lane = threadIdx.x & 63, row = (i & 1) * R + lane / C;
    return ((lane % C) ^ ((row & 3) * 4)) * 8 < l.o_left;
  }

  // loads from..to of a stage all of whose k are there
  template <int from, int to>
  __device__ static __forceinline__ void load(const Loader &l, int stage, unsigned char *xs, unsigned char *ws) {
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
    for (int i = from; i < to; ++i) {
      if (i < XL) {
        to_lds(x_at(l, i, stage), xs + (wv * XL + i) * 1024);
      } else {
        const char *at = w_at(l, i - XL, stage);
        if constexpr (NN && !FULL) at = w_there(l, i - XL) ? at : reinterpret_cast<const char *>(&kZeros);
        to_lds(at, ws + (wv * WL + i - XL) * 1024);
      }
    }
  }
  // a stage of which `left` k are there (a multiple of 8)
  __device__ static __forceinline__ void load_cut(const Loader &l, int stage, int left, unsigned char *xs, unsigned char *ws) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const char *zeros = reinterpret_cast<const char *>(&kZeros);
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const int chunk = (lane % Chunks) ^ chunk_key((wv * XL + i) * PerLoad + lane / Chunks);
      to_lds(chunk * 8 < left ? x_at(l, i, stage) : zeros, xs + (wv * XL + i) * 1024);
    }
#pragma unroll
    for (int i = 0; i < WL; ++i) {
      bool there;
      if constexpr (NN) there = (wv * WL + i) * R + lane / C < left && w_there(l, i);
      else there = ((lane % Chunks) ^ chunk_key((wv * WL + i) * PerLoad + lane / Chunks)) * 8 < left;
      to_lds(there ? w_at(l, i, stage) : zeros, ws + (wv * WL + i) * 1024);
    }
  }

  // 32 outputs from o on, 16 k from k on, of lines of k
  __device__ static __forceinline__ u32x4 across(const unsigned char *s, int o, int k) {
    const int lane = threadIdx.x & 63, g = lane >> 4, q = lane & 15;
    const int n = o + (g & 1) * 16 + (q & 3) * 4, kk = k + (g >> 1) * 8 + (q >> 2);
    u32x4 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = kk + h * 4;
      const uint2 u = turned(s + row * (BO * 2) + (((n >> 3) ^ ((row & 3) * 4)) << 4) + (n & 7) * 2);
      v[2 * h] = u.x, v[2 * h + 1] = u.y;
    }
    return v;
  }

  struct Operands {
    u32x4 x[ET], w[EO];
  };
  __device__ static __forceinline__ void fetch(const unsigned char *xs, const unsigned char *ws, int step, Operands &f) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
    const int tw = (wv / WO) * (ET * 32), ow = (wv % WO) * (EO * 32);
#pragma unroll
    for (int e = 0; e < EO; ++e) f.w[e] = NN ? across(ws, ow + e * 32, step * 16) : chunk_of(ws, ow + e * 32 + ln, step * 2 + half);
#pragma unroll
    for (int r = 0; r < ET; ++r) f.x[r] = chunk_of(xs, tw + r * 32 + ln, step * 2 + half);
  }
  __device__ static __forceinline__ void multiply(const Operands &f, f32x16 (&acc)[EO][ET]) {
#pragma unroll
    for (int e = 0; e < EO; ++e)
#pragma unroll
      for (int r = 0; r < ET; ++r) acc[e][r] = mma<bf16_t>(f.w[e], f.x[r], acc[e][r]);
  }
  // The barrier by itself (a fence would wait for all loads); the clobbers keep the reads of LDS on their sides of it.
  __device__ static __forceinline__ void barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  }
  // all but the last n loads of every wave have arrived
  template <int n>
  __device__ static __forceinline__ void arrived() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory");
    barrier();
  }
  // The order of a step: its reads of LDS two at a time between the first products (the rest of which hide the last one's way),
  // its loads between the others, as far apart as they get: a load takes 16 cycles on its way out, a product 32.
  template <int reads, int loads>
  __device__ static __forceinline__ void spread() {
    constexpr int M = ET * EO, N = (reads + 1) / 2;
    if constexpr (M < 16) {  // (two workgroups a compute unit hide each other's: 1024 x 4096 -> 4096 50 us with, 44.5 without)
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
  __device__ static __forceinline__ void stage(const Loader &l, int later, unsigned char *xs, unsigned char *ws, const unsigned char *xn,
                                               const unsigned char *wn, Operands (&f)[4], f32x16 (&acc)[EO][ET]) {
    constexpr int Reads = ET + EO * (NN ? 2 : 1), L = XL + WL, L1 = (L + 2) / 3, L2 = 2 * L1;
    fetch(xs, ws, 2, f[2]);
    fetch(xs, ws, 3, f[3]);
    multiply(f[0], acc);
    spread<2 * Reads, 0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    barrier();
    load<0, L1>(l, later, xs, ws);
    multiply(f[1], acc);
    spread<0, L1>();
    load<L1, L2>(l, later, xs, ws);
    multiply(f[2], acc);
    spread<0, L2 - L1>();
    arrived<L2>();
    fetch(xn, wn, 0, f[0]);
    fetch(xn, wn, 1, f[1]);
    load<L2, L>(l, later, xs, ws);
    multiply(f[3], acc);
    spread<2 * Reads, L - L2>();
  }

  // acc += x W^T over k0 .. k1
  __device__ static __forceinline__ void run(const Project<bf16_t> &p, int64_t t0, int o0, int k0, int k1, unsigned char *xs0,
                                             unsigned char *ws0, unsigned char *xs1, unsigned char *ws1, f32x16 (&acc)[EO][ET]) {
    constexpr int L = XL + WL;
    Loader l;
    aim(p, t0, o0, k0, l);
    const int pairs = (k1 - k0) / (2 * kK);
    Operands f[4];
    if (pairs > 0) {
      load<0, L>(l, 0, xs0, ws0);
      load<0, L>(l, 1, xs1, ws1);
      arrived<L>();
      fetch(xs0, ws0, 0, f[0]);
      fetch(xs0, ws0, 1, f[1]);
      const int last = 2 * pairs - 1;  // (what would be loaded beyond it is loaded again, for nothing)
      for (int s = 0; s < last; s += 2) {
        stage(l, min(s + 2, last), xs0, ws0, xs1, ws1, f, acc);
        stage(l, min(s + 3, last), xs1, ws1, xs0, ws0, f, acc);
      }
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");  // nothing is on its way to LDS from here on
      barrier();
    }
    for (int s = 2 * pairs, left = k1 - k0 - s * kK; left > 0; ++s, left -= kK) {
      load_cut(l, s, left, xs0, ws0);
      arrived<0>();
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        fetch(xs0, ws0, i, f[0]);
        multiply(f[0], acc);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      barrier();
    }
  }

  // The wave's results to y, rows from tw and outputs from ow on, without those before `from`, through its part of LDS: a row's 8-byte
  // pieces are exchanged by a key of the row (even, so that pairs of them stay together).
  __device__ static __forceinline__ void store(const Project<bf16_t> &p, int64_t tw, int ow, int from, const f32x16 (&acc)[EO][ET],
                                               unsigned char *lds) {
    constexpr int Row = EO * 64, Pieces = Row / 8, Lanes = Row / 16, Rows = 64 / Lanes;  // bytes of a row; rows of a store
    const int lane = threadIdx.x & 63, ln = lane & 31, half = lane >> 5;
    auto twist = [](int row) { return row % (Pieces / 2) * 2; };
#pragma unroll
    for (int r = 0; r < ET; ++r) {
#pragma unroll
      for (int e = 0; e < EO; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const int row = r * 32 + ln, piece = e * 8 + (i >> 1) + half;
          const uint2 v = {(uint32_t)narrow<bf16_t>(acc[e][r][i]) | (uint32_t)narrow<bf16_t>(acc[e][r][i + 1]) << 16,
                           (uint32_t)narrow<bf16_t>(acc[e][r][i + 2]) | (uint32_t)narrow<bf16_t>(acc[e][r][i + 3]) << 16};
          *reinterpret_cast<uint2 *>(lds + row * Row + ((piece ^ twist(row)) << 3)) = v;
        }
      __builtin_amdgcn_sched_barrier(0);
    }
    // (a wave reads what it wrote itself: LDS is in order)
#pragma unroll 4
    for (int r0 = 0; r0 < ET * 32; r0 += Rows) {
      const int row = r0 + lane / Lanes, c = lane % Lanes, o = ow + c * 8;
      const u32x4 v = *reinterpret_cast<const u32x4 *>(lds + row * Row + (((2 * c) ^ twist(row)) << 3));
      bf16_t *y = p.y + (tw + row) * p.ldy + o;
      if ((FULL || tw + row < p.rows) && (!FULL || o >= from) && ((FULL && !NN) || o + 8 <= p.outs)) {
        *reinterpret_cast<u32x4_any *>(y) = v;
      } else if (FULL || tw + row < p.rows) {
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if ((!FULL || o + q >= from) && o + q < p.outs) y[q] = (bf16_t)(v[q >> 1] >> (16 * (q & 1)));
      }
    }
  }
};

template <int BT, int BO, bool NN, bool FULL>
__global__ __launch_bounds__(256, BT == 128 ? 2 : 1) void project_gemm_kernel(Project<bf16_t> p, int64_t tiles_t, int tiles_o) {
  using G = Gemm<BT, BO, 2, NN, FULL>;
  constexpr int ET = G::ET, EO = G::EO;
  __shared__ __align__(1024) unsigned char xs0[G::XB], ws0[G::WB], xs1[G::XB], ws1[G::WB];
  int64_t tt;
  int to;
  tile_of(in_runs(blockIdx.x, tiles_t * tiles_o), tiles_t, tiles_o, tt, to);
  int64_t t0 = tt * BT;
  int o0 = to * BO;
  const int from = o0;
  if constexpr (FULL) t0 = min(t0, p.rows - BT), o0 = min(o0, (NN ? (p.outs + 7) / 8 * 8 : p.outs) - BO);
  const int wv = threadIdx.x >> 6;
  const int64_t tw = t0 + (wv / G::WO) * (ET * 32);
  const int ow = o0 + (wv % G::WO) * (EO * 32);
  f32x16 acc[EO][ET] = {};
  if (p.low.of_row) {  // (first: beside the operands its registers would not fit)
    constexpr int Quarter = BT / 4;
    auto room = [&](int row) {
      const int q = row / Quarter;
      return reinterpret_cast<bf16_t *>(q == 0 ? xs0 : q == 1 ? ws0 : q == 2 ? xs1 : ws1) + row % Quarter * PartsOf<bf16_t>::Out * p.h.ld;
    };
    gather_lines<bf16_t, BT>(p.low, p.h, room, t0, p.rows);
    __syncthreads();
    auto lines_of = [&](int r) { return room(__builtin_amdgcn_readfirstlane((wv / G::WO) * (ET * 32) + r * 32)); };
    int o[EO];
#pragma unroll
    for (int e = 0; e < EO; ++e) o[e] = ow + e * 32 + (threadIdx.x & 31);
    add_thin<bf16_t, EO, ET, false, 1>(p.low, p.m, p.h.ld, lines_of, p.rows, p.outs, tw, o, acc);
    __syncthreads();
  }
  G::run(p, t0, o0, 0, p.width, xs0, ws0, xs1, ws1, acc);
  unsigned char *own = wv == 0 ? xs0 : wv == 1 ? ws0 : wv == 2 ? xs1 : ws1;
  G::store(p, tw, ow, from, acc, own);
}

// Ranges of k: a workgroup leaves its sums as they are.  Before the tiles, workgroups of rank lines.
template <int BT, int BO, int WT, bool NN>
__global__ __launch_bounds__(256, 2) void project_gemm_split_kernel(Project<bf16_t> p, int64_t tiles_t, int tiles_o, int splits, int chunk,
                                                                    float *__restrict__ part, ThinJob<bf16_t> thin, ThinJob<bf16_t> other) {
  using G = Gemm<BT, BO, WT, NN, false>;
  constexpr int ET = G::ET, EO = G::EO;
  __shared__ __align__(1024) unsigned char xs0[G::XB], ws0[G::WB], xs1[G::XB], ws1[G::WB];
  const int64_t block = blockIdx.x;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  if (block < thin.blocks + other.blocks) {
    __shared__ ThinLds lds;
    unsigned char *own = wv == 0 ? xs0 : wv == 1 ? ws0 : wv == 2 ? xs1 : ws1;  // (16 KiB each where rows come by ranges)
    if (block < thin.blocks) thin_block<bf16_t>(thin, p.low, block, lds, own);
    else thin_block<bf16_t>(other, p.low, block - thin.blocks, lds, own);
    return;
  }
  const int64_t at = block - thin.blocks - other.blocks;
  const int split = (int)(at % splits);
  const int64_t tile = at / splits, t0 = tile % tiles_t * BT;
  const int o0 = (int)(tile / tiles_t) * BO;
  f32x16 acc[EO][ET] = {};
  G::run(p, t0, o0, split * chunk, min(p.width, (split + 1) * chunk), xs0, ws0, xs1, ws1, acc);
  const int64_t tw = t0 + (wv / G::WO) * (ET * 32);
  const int ow = o0 + (wv % G::WO) * (EO * 32);
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    const int64_t t = tw + r * 32 + ln;
    if (t >= p.rows) continue;
#pragma unroll
    for (int e = 0; e < EO; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int o = ow + e * 32 + (i >> 2) * 8 + half * 4;
        float *y = part + ((int64_t)split * p.rows + t) * p.outs + o;
        if (o + 4 <= p.outs) {
          *reinterpret_cast<f32x4_any *>(y) = f32x4_any{acc[e][r][i], acc[e][r][i + 1], acc[e][r][i + 2], acc[e][r][i + 3]};
        } else {
#pragma unroll
          for (int q = 0; q < 3; ++q)
            if (o + q < p.outs) y[q] = acc[e][r][i + q];
        }
      }
  }
}

bool on_16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t tiles(int64_t n, int size) { return (n + size - 1) / size; }

template <int B, bool FULL>
void launch(const Project<bf16_t> &p, hipStream_t s) {
  const int64_t tiles_t = tiles(p.rows, B);
  const int tiles_o = (int)tiles(p.outs, B);
  const unsigned blocks = (unsigned)(tiles_t * tiles_o);
  if (p.wk == 1) project_gemm_kernel<B, B, false, FULL><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o);
  else project_gemm_kernel<B, B, true, FULL><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o);
}

}  // namespace

// Rows of x and W that 16-byte loads can take, lanes' offsets within 32 bits, and no more tiles than a launch has workgroups.
bool gemm_takes(const Project<bf16_t> &p) {
  const int64_t w_row = p.wk == 1 ? p.wo : p.wk;
  return on_16(p.x) && on_16(p.w) && p.ldx % 8 == 0 && p.ldx < 1 << 27 && w_row % 8 == 0 && p.width % 8 == 0 &&
         tiles(p.rows, 128) * tiles(p.outs, 128) < 1 << 22;
}

// Tiles in ranges of k: 32, 64 or 128 rows by 128 outputs.
int split_rows(int64_t rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

// Whole tiles where they give three quarters of the compute units work; else ranges of 256 k at least, and two (few rows: what counts
// is W on its way) workgroups a compute unit.  (1024 rows, with 4 adapters, whole and in ranges: 4096 -> 1536 62 and 36 us, 4096 -> 3200
// 63 and 72, 1024 -> 3200 34 and 43.)
int gemm_splits(int64_t rows, int width, int outs) {
  const int64_t n = tiles(rows, split_rows(rows)) * tiles(outs, 128);
  if (rows > 64 && n >= 192) return 1;
  const int64_t want = std::min<int64_t>(((rows > 64 ? 384 : 512) + n - 1) / n, std::max(width / 256, 1));
  const int64_t chunk = tiles(tiles(width, (int)std::min<int64_t>(want, 16)), 128) * 128;
  return (int)tiles(width, (int)chunk);
}

// 256 x 256 tiles, of which a compute unit holds one, where three quarters of them have one.  (4 adapters, 256 and 128: 4096 rows,
// 4096 -> 4096 172 and 187 us; 2048 rows, 4096 -> 2048, which gives 64, 133 and 69.)
void launch_gemm(const Project<bf16_t> &p, hipStream_t s) {
  if (p.rows >= 256 && p.outs >= 256 && tiles(p.rows, 256) * tiles(p.outs, 256) >= 200) launch<256, true>(p, s);
  else launch<128, false>(p, s);
}

template <int BT, int WT>
void launch_split(const Project<bf16_t> &p, int splits, float *part, const ThinJob<bf16_t> &thin, const ThinJob<bf16_t> &other, hipStream_t s) {
  const int64_t tiles_t = tiles(p.rows, BT);
  const int tiles_o = (int)tiles(p.outs, 128), chunk = (int)tiles(tiles(p.width, splits), 128) * 128;
  const unsigned blocks = (unsigned)(tiles_t * tiles_o * splits + thin.blocks + other.blocks);
  if (p.wk == 1) project_gemm_split_kernel<BT, 128, WT, false><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
  else project_gemm_split_kernel<BT, 128, WT, true><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
}

void launch_gemm_split(const Project<bf16_t> &p, int splits, float *part, const ThinJob<bf16_t> &thin, const ThinJob<bf16_t> &other,
                       hipStream_t s) {
  const int rows = split_rows(p.rows);
  if (rows == 32) launch_split<32, 1>(p, splits, part, thin, other, s);
  else if (rows == 64) launch_split<64, 1>(p, splits, part, thin, other, s);
  else launch_split<128, 2>(p, splits, part, thin, other, s);
}

}  // namespace wcc

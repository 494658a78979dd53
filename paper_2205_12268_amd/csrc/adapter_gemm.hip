// The projection for many rows of bf16: the matrix cores fed from LDS, which loads go to straight from memory.
//
// A workgroup has BT rows x BO outputs, stages of 64 k, two of them in LDS: while one is multiplied, the other's loads
// (16 bytes a lane, into LDS without passing registers) are in flight.  LDS has no padding (such a load writes 1 KiB in a row),
// so the 16-byte chunks of a line are exchanged by a key of the line, at the load by choosing which chunk of memory a lane
// asks for: the 16 lines that a read takes at once are then on different banks.
// Where W's outputs are contiguous and not its k (NN), LDS holds lines of k and the reads transpose 4 x 16 blocks.
// The first operand of the matrix cores is W, the second x: a lane has one row's results, four neighbouring outputs at a time.
// Chunks past the end of k, and outputs past the last (NN), are loaded from 16 bytes of zeros.
#include "adapter.h"

namespace wcc {
namespace {

__device__ const uint4 kZeros = {0, 0, 0, 0};

typedef __attribute__((address_space(3))) unsigned char lds_byte;
typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;

__device__ __forceinline__ void to_lds(const bf16_t *from, unsigned char *to) {
  __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                   (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

constexpr int kK = 64;  // k of a stage: lines of 128 bytes

// (see adapter_tile.hip)
__device__ __forceinline__ void tile_of(int64_t b, int64_t tiles, int64_t tiles_t, int tiles_o, int64_t &tt, int &to) {
  const int64_t each = tiles / 8;
  if (b < each * 8) b = b % 8 * each + b / 8;
  const int64_t band = (int64_t)8 * tiles_o, first = b / band * 8, in = b % band;
  const int64_t high = min(tiles_t - first, (int64_t)8);
  tt = first + in % high;
  to = (int)(in / high);
}

template <int BT, int BO, int WT, int WO, bool NN>
struct Gemm {
  static constexpr int Waves = WT * WO, Threads = Waves * 64;
  static constexpr int ET = BT / WT / 32, EO = BO / WO / 32;       // 32 x 32 results of a wave
  static constexpr int XB = BT * kK * 2, WB = BO * kK * 2;         // bytes of a stage
  static constexpr int XL = XB / 1024 / Waves, WL = WB / 1024 / Waves;  // loads of a wave

  struct Loader {
    const bf16_t *x[XL], *w[WL];
    int xk[XL], wk[WL];  // first k of the lane's chunk (NN: of w, the line of k), or far off where there is none
    int64_t w_step;
  };

  __device__ static __forceinline__ void aim(const Project<bf16_t> &p, int64_t t0, int o0, int k0, Loader &l) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      const int row = (wv * XL + i) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
      l.x[i] = p.x + min(t0 + row, p.rows - 1) * p.ldx + k0 + chunk * 8;
      l.xk[i] = chunk * 8;
    }
#pragma unroll
    for (int i = 0; i < WL; ++i) {
      if constexpr (!NN) {
        const int row = (wv * WL + i) * 8 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
        l.w[i] = p.w + (int64_t)min(o0 + row, p.outs - 1) * p.wo + k0 + chunk * 8;
        l.wk[i] = chunk * 8;
      } else {
        constexpr int C = BO / 8, R = 64 / C;  // chunks of a line, lines of a load
        const int row = (wv * WL + i) * R + lane / C, chunk = (lane % C) ^ ((row & 3) * 4);
        const int o = o0 + chunk * 8;
        l.w[i] = p.w + (int64_t)(k0 + row) * p.wk + o;
        l.wk[i] = o < p.outs ? row : 1 << 30;
      }
    }
    l.w_step = NN ? kK * p.wk : kK;
  }

  // the stage that begins at k
  __device__ static __forceinline__ void load(Loader &l, int k, int end, unsigned char *xs, unsigned char *ws) {
    const int wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bf16_t *zeros = reinterpret_cast<const bf16_t *>(&kZeros);
#pragma unroll
    for (int i = 0; i < XL; ++i) {
      to_lds(k + l.xk[i] < end ? l.x[i] : zeros, xs + (wv * XL + i) * 1024);
      l.x[i] += kK;
    }
#pragma unroll
    for (int i = 0; i < WL; ++i) {
      to_lds(k + l.wk[i] < end ? l.w[i] : zeros, ws + (wv * WL + i) * 1024);
      l.w[i] += l.w_step;
    }
  }

  __device__ static __forceinline__ u32x4 line(const unsigned char *s, int row, int chunk) {
    return *reinterpret_cast<const u32x4 *>(s + row * 128 + ((chunk ^ ((row >> 1) & 7)) << 4));
  }
  // 32 outputs from o on, 16 k from k on, of lines of k
  __device__ static __forceinline__ u32x4 across(const unsigned char *s, int o, int k) {
    const int lane = threadIdx.x & 63, g = lane >> 4, q = lane & 15;
    const int n = o + (g & 1) * 16 + (q & 3) * 4, kk = k + (g >> 1) * 8 + (q >> 2);
    u32x4 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int row = kk + h * 4;
      const unsigned char *at = s + row * (BO * 2) + (((n >> 3) ^ ((row & 3) * 4)) << 4) + (n & 7) * 2;
      const bf16x4 r = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
          (__attribute__((address_space(3))) bf16x4 *)(__attribute__((address_space(3))) void *)at);
      const uint2 u = __builtin_bit_cast(uint2, r);
      v[2 * h] = u.x, v[2 * h + 1] = u.y;
    }
    return v;
  }

  __device__ static __forceinline__ void multiply(const unsigned char *xs, const unsigned char *ws, f32x16 (&acc)[EO][ET]) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
    const int tw = (wv / WO) * (ET * 32), ow = (wv % WO) * (EO * 32);
    u32x4 xf[2][ET], wf[2][EO];
    auto fetch = [&](int ks) {
#pragma unroll
      for (int e = 0; e < EO; ++e)
        wf[ks & 1][e] = NN ? across(ws, ow + e * 32, ks * 16) : line(ws, ow + e * 32 + ln, ks * 2 + half);
#pragma unroll
      for (int r = 0; r < ET; ++r) xf[ks & 1][r] = line(xs, tw + r * 32 + ln, ks * 2 + half);
    };
    fetch(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      if (ks < 3) fetch(ks + 1);
#pragma unroll
      for (int e = 0; e < EO; ++e)
#pragma unroll
        for (int r = 0; r < ET; ++r) acc[e][r] = mma<bf16_t>(wf[ks & 1][e], xf[ks & 1][r], acc[e][r]);
      __builtin_amdgcn_sched_barrier(0);  // (the reads of one step ahead, no more: registers)
    }
  }

  // As adapter.h's add_thin, with rows and outputs exchanged: a lane's own row is t0 + lane % 32.
  __device__ static __forceinline__ void add_rank(const Project<bf16_t> &p, int64_t t0, int o0, f32x16 (&acc)[EO][ET], int r) {
    constexpr int P = PartsOf<bf16_t>::Out;
    const int ln = threadIdx.x & 31, half = (threadIdx.x >> 5) & 1;
    const int64_t t = min(t0 + ln, p.rows - 1);
    const int id = t0 + ln < p.rows ? p.low.of(t) : -1;
    uint32_t rest = (uint32_t)__ballot(id >= 0);
    while (rest != 0) {
      const int a = __builtin_amdgcn_readlane(id, __builtin_ctz(rest));
      rest &= ~(uint32_t)__ballot(id == a);
      const int lines = p.low.lines(a);
      f32x16 d[EO] = {};
      for (int j0 = 0; j0 < lines; j0 += 16) {
        const int j = j0 + half * 8, left = lines - j;
        u32x4 hf[P] = {}, mf[EO] = {};
        if (left > 0) {
          float hv[8];
          p.h.eight(t, j, hv);
          split_to<bf16_t, P>(hv, hf);
#pragma unroll
          for (int e = 0; e < EO; ++e) mf[e] = thin_k(p.m, a, min(o0 + e * 32 + ln, p.outs - 1), j, left);
        }
#pragma unroll
        for (int e = 0; e < EO; ++e)
#pragma unroll
          for (int q = P - 1; q >= 0; --q) d[e] = mma<bf16_t>(mf[e], hf[q], d[e]);
      }
#pragma unroll
      for (int e = 0; e < EO; ++e)
#pragma unroll
        for (int i = 0; i < 16; ++i) acc[e][r][i] += id == a ? d[e][i] : 0.f;
    }
  }
};

// The results of a tile: acc += x W^T over k0 .. k1.
template <class G>
__device__ __forceinline__ void run_tile(const Project<bf16_t> &p, int64_t t0, int o0, int k0, int k1, unsigned char *xs0, unsigned char *ws0,
                                         unsigned char *xs1, unsigned char *ws1, f32x16 (&acc)[G::EO][G::ET]) {
  typename G::Loader l;
  G::aim(p, t0, o0, k0, l);
  G::load(l, k0, k1, xs0, ws0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int k = k0; k < k1; k += 2 * kK) {  // (an odd last stage has one of zeros beside it)
    G::load(l, k + kK, k1, xs1, ws1);
    G::multiply(xs0, ws0, acc);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (k + 2 * kK < k1) G::load(l, k + 2 * kK, k1, xs0, ws0);
    G::multiply(xs1, ws1, acc);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
}

template <int BT, int BO, int WT, int WO, bool NN>
__global__ __launch_bounds__(WT *WO * 64, 2) void project_gemm_kernel(Project<bf16_t> p, int64_t tiles_t, int tiles_o) {
  using G = Gemm<BT, BO, WT, WO, NN>;
  constexpr int ET = G::ET, EO = G::EO;
  __shared__ __align__(1024) unsigned char xs0[G::XB], ws0[G::WB], xs1[G::XB], ws1[G::WB];
  int64_t tt;
  int to;
  tile_of(blockIdx.x, tiles_t * tiles_o, tiles_t, tiles_o, tt, to);
  const int64_t t0 = tt * BT;
  const int o0 = to * BO;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  const int64_t tw = t0 + (wv / WO) * (ET * 32);
  const int ow = o0 + (wv % WO) * (EO * 32);
  f32x16 acc[EO][ET] = {};
  if (p.low.of_row) {  // (first: beside the loads' addresses its registers would not fit)
#pragma unroll
    for (int r = 0; r < ET; ++r) G::add_rank(p, tw + r * 32, ow, acc, r);
  }
  run_tile<G>(p, t0, o0, 0, p.width, xs0, ws0, xs1, ws1, acc);
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    __builtin_amdgcn_sched_barrier(0);
    const int64_t t = tw + r * 32 + ln;
    if (t >= p.rows) continue;
#pragma unroll
    for (int e = 0; e < EO; ++e)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int o = ow + e * 32 + (i >> 2) * 8 + half * 4;
        bf16_t *y = p.y + t * p.ldy + o;
        if (o + 4 <= p.outs) {
          const uint64_t v = (uint64_t)narrow<bf16_t>(acc[e][r][i]) | (uint64_t)narrow<bf16_t>(acc[e][r][i + 1]) << 16 |
                             (uint64_t)narrow<bf16_t>(acc[e][r][i + 2]) << 32 | (uint64_t)narrow<bf16_t>(acc[e][r][i + 3]) << 48;
          typedef uint64_t u64_2 __attribute__((aligned(2)));
          *reinterpret_cast<u64_2 *>(y) = v;
        } else {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            if (o + q < p.outs) y[q] = narrow<bf16_t>(acc[e][r][i + q]);
        }
      }
  }
}

// Ranges of k: a workgroup leaves its sums as they are.  Before the tiles, workgroups of rank lines.
template <int BT, int BO, int WT, int WO, bool NN>
__global__ __launch_bounds__(WT *WO * 64, 2) void project_gemm_split_kernel(Project<bf16_t> p, int64_t tiles_t, int tiles_o, int splits,
                                                                            int chunk, float *__restrict__ part, ThinJob<bf16_t> thin,
                                                                            ThinJob<bf16_t> other) {
  using G = Gemm<BT, BO, WT, WO, NN>;
  constexpr int ET = G::ET, EO = G::EO;
  __shared__ __align__(1024) unsigned char xs0[G::XB], ws0[G::WB], xs1[G::XB], ws1[G::WB];
  const int64_t block = blockIdx.x;
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6, ln = lane & 31, half = lane >> 5;
  if (block < thin.blocks) return thin_block<bf16_t>(thin, p.low, block, xs0);
  if (block < thin.blocks + other.blocks) return thin_block<bf16_t>(other, p.low, block - thin.blocks, xs0);
  const int64_t at = block - thin.blocks - other.blocks;
  const int split = (int)(at % splits);
  const int64_t tile = at / splits, t0 = tile % tiles_t * BT;
  const int o0 = (int)(tile / tiles_t) * BO;
  f32x16 acc[EO][ET] = {};
  run_tile<G>(p, t0, o0, split * chunk, min(p.width, (split + 1) * chunk), xs0, ws0, xs1, ws1, acc);
  const int64_t tw = t0 + (wv / WO) * (ET * 32);
  const int ow = o0 + (wv % WO) * (EO * 32);
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
          for (int q = 0; q < 4; ++q)
            if (o + q < p.outs) y[q] = acc[e][r][i + q];
        }
      }
  }
}

bool on_16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t tiles(int64_t n, int size) { return (n + size - 1) / size; }

template <int BT, int BO, int WT, int WO>
void launch(const Project<bf16_t> &p, hipStream_t s) {
  const int64_t tiles_t = tiles(p.rows, BT);
  const int tiles_o = (int)tiles(p.outs, BO);
  const unsigned blocks = (unsigned)(tiles_t * tiles_o);
  if (p.wk == 1) project_gemm_kernel<BT, BO, WT, WO, false><<<blocks, WT * WO * 64, 0, s>>>(p, tiles_t, tiles_o);
  else project_gemm_kernel<BT, BO, WT, WO, true><<<blocks, WT * WO * 64, 0, s>>>(p, tiles_t, tiles_o);
}

}  // namespace

// Rows of x and W that 16-byte loads can take, and no more tiles than a launch has workgroups.
bool gemm_takes(const Project<bf16_t> &p) {
  const int64_t w_row = p.wk == 1 ? p.wo : p.wk;
  return on_16(p.x) && on_16(p.w) && p.ldx % 8 == 0 && w_row % 8 == 0 && p.width % 8 == 0 &&
         tiles(p.rows, 128) * tiles(p.outs, 128) < 1 << 22;
}

int gemm_splits(int64_t rows, int width, int outs) {
  const int64_t n = tiles(rows, 128) * tiles(outs, 128);
  if (n >= 192) return 1;
  const int64_t want = std::min<int64_t>((384 + n - 1) / n, std::max(width / 256, 1));
  const int64_t chunk = tiles(tiles(width, (int)std::min<int64_t>(want, 16)), 128) * 128;
  return (int)tiles(width, (int)chunk);
}

void launch_gemm(const Project<bf16_t> &p, hipStream_t s) {
  if (tiles(p.rows, 256) * tiles(p.outs, 256) >= 200) launch<256, 256, 2, 4>(p, s);
  else launch<128, 128, 2, 2>(p, s);
}

void launch_gemm_split(const Project<bf16_t> &p, int splits, float *part, const ThinJob<bf16_t> &thin, const ThinJob<bf16_t> &other,
                       hipStream_t s) {
  const int64_t tiles_t = tiles(p.rows, 128);
  const int tiles_o = (int)tiles(p.outs, 128), chunk = (int)tiles(tiles(p.width, splits), 128) * 128;
  const unsigned blocks = (unsigned)(tiles_t * tiles_o * splits + thin.blocks + other.blocks);
  if (p.wk == 1) project_gemm_split_kernel<128, 128, 2, 2, false><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
  else project_gemm_split_kernel<128, 128, 2, 2, true><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
}

}  // namespace wcc

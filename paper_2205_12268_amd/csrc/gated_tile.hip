// The products of the gated block in tiles of 128 (or 64) x 128 through LDS by way of registers: any type, alignment and stride.
// Projections come here that are too small for tiles fed straight from memory to win, or whose copies would cost more than they give; the
// gradients' products (tile_product) only where a tensor does not begin on 16 bytes or a row is 4 MiB and longer.
//
// Four waves of 64 (32) x 64 results; stages of 128 bytes of k (64 bf16 or 32 fp32), two in LDS, the next one's loads in flight while one is
// multiplied.  LDS lines are 144 bytes apart, which spreads the 16-byte reads of 32 lines over all banks.  Where lines are contiguous
// in memory and not their k, a thread loads pairs of lines of eight (four) k and exchanges halves, so that LDS holds the same either way.
// For the two projections a tile's second operand is 64 lines of each weight; a wave has the same 32 outputs of both, so that the
// activation, the product, their slopes and the codes are made where the sums are.
// Few tiles are cut into ranges of k, whose sums another launch joins in their order.
#include "gated.h"

namespace wcc {
namespace {

constexpr int kTile = 128, kRowBytes = 144, kStage = 128;

// B lines of an operand, 64 or 128
template <class T, bool ACROSS, int B>
struct Loader {
  static constexpr int VE = VecOf<T>::N, N = B / 32, Pairs = B / 2, Groups = 256 / Pairs;  // Groups of threads over k
  const T *p[ACROSS ? 1 : N];
  int64_t s;
  bool both;
  // line(i): which line the tile's i-th is
  template <class F>
  __device__ __forceinline__ void aim(const F &line_at, int64_t stride) {
    const int tid = threadIdx.x;
    s = stride;
    if constexpr (ACROSS) {
      bool one;
      p[0] = line_at(2 * (tid % Pairs), one);
      line_at(2 * (tid % Pairs) + 1, both);
    } else {
      bool there;
#pragma unroll
      for (int i = 0; i < N; ++i) p[i] = line_at((tid >> 3) + 32 * i, there) + (tid & 7) * VE;
    }
  }
  __device__ __forceinline__ void load(int64_t k, int64_t k1, u32x4 (&st)[N]) const {
    const int tid = threadIdx.x;
    if constexpr (ACROSS) {
      const int kg = tid / Pairs;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        const int64_t kk = k + (kg + Groups * i) * VE;
        const int left = (int)max(min(k1 - kk, (int64_t)VE), (int64_t)0);
        load_k_pair(p[0] + (left > 0 ? kk : 0) * s, s, left, both, st[2 * i], st[2 * i + 1]);
      }
    } else {
      const int left = (int)min(k1 - k - (tid & 7) * VE, (int64_t)VE);
#pragma unroll
      for (int i = 0; i < N; ++i) st[i] = load_k(p[i] + k, left);
    }
  }
  __device__ __forceinline__ static void store(unsigned char *lds, const u32x4 (&st)[N]) {
    const int tid = threadIdx.x;
    if constexpr (ACROSS) {
      const int pair = tid % Pairs, kg = tid / Pairs;
#pragma unroll
      for (int i = 0; i < N / 2; ++i) {
        *reinterpret_cast<u32x4 *>(lds + (2 * pair) * kRowBytes + (kg + Groups * i) * 16) = st[2 * i];
        *reinterpret_cast<u32x4 *>(lds + (2 * pair + 1) * kRowBytes + (kg + Groups * i) * 16) = st[2 * i + 1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) *reinterpret_cast<u32x4 *>(lds + ((tid >> 3) + 32 * i) * kRowBytes + (tid & 7) * 16) = st[i];
    }
  }
};

// acc[e][r] += the products over k0 .. k1 (second: of a's second part, by what is finite in b); wave (wm, wn) has rows (wm * ET + r) * 32 and lines first(e) of the second operand
template <class T, bool AT, bool BT, int ET, class F>
__device__ __forceinline__ void multiply(const Loader<T, AT, 64 * ET> &a, const Loader<T, BT, kTile> &b, int64_t k0, int64_t k1, int wm, F first, bool second,
                                         unsigned char (&lds)[2][(64 * ET + kTile) * kRowBytes], f32x16 (&acc)[2][ET]) {
  constexpr int KB = kStage / (int)sizeof(T), Rows = 64 * ET;
  const int lane = threadIdx.x & 63, ln = lane & 31, half = lane >> 5;
  u32x4 sa[2 * ET], sb[4];
  a.load(k0, k1, sa), b.load(k0, k1, sb);
  __syncthreads();  // (whoever read LDS before)
  a.store(lds[0], sa), b.store(lds[0] + Rows * kRowBytes, sb);
  __syncthreads();
  int buf = 0;
  for (int64_t k = k0; k < k1; k += KB, buf ^= 1) {
    const bool more = k + KB < k1;
    if (more) a.load(k + KB, k1, sa), b.load(k + KB, k1, sb);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
      u32x4 af[ET], bf[2];
#pragma unroll
      for (int r = 0; r < ET; ++r)
        af[r] = *reinterpret_cast<const u32x4 *>(lds[buf] + ((wm * ET + r) * 32 + ln) * kRowBytes + ks * 32 + half * 16);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        bf[e] = *reinterpret_cast<const u32x4 *>(lds[buf] + (Rows + first(e) + ln) * kRowBytes + ks * 32 + half * 16);
        if constexpr (sizeof(T) == 2) {
          if (second) bf[e] = finite_of(bf[e]);
        }
      }
#pragma unroll
      for (int r = 0; r < ET; ++r)
#pragma unroll
        for (int e = 0; e < 2; ++e) acc[e][r] = mma<T>(bf[e], af[r], acc[e][r]);
    }
    if (more) a.store(lds[buf ^ 1], sa), b.store(lds[buf ^ 1] + Rows * kRowBytes, sb);
    __syncthreads();
  }
}

struct Grid {
  int et;       // rows of a tile / 64
  int64_t tiles_r, tiles_o, tiles;
  int splits;
  int64_t chunk;  // k of a range
};

// ---- the two projections -------------------------------------------------------------------------------------
template <class T, int ET, int ACT, bool BACK, bool PARTS>
__global__ __launch_bounds__(256, 2) void gate_tile_kernel(Gate<T> p, Side<T> x, const T *__restrict__ w_gate, const T *__restrict__ w_up,
                                                           int64_t ldw, int64_t k, Grid n, float *__restrict__ part) {
  __shared__ __align__(16) unsigned char lds[2][(64 * ET + kTile) * kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5, wm = wv >> 1, wn = wv & 1;
  const int64_t at = in_runs(blockIdx.x, n.tiles * n.splits), split = at / n.tiles;
  int64_t tt;
  int to;
  tile_of(at % n.tiles, n.tiles_r, (int)n.tiles_o, tt, to);
  const int64_t t0 = tt * (64 * ET);
  const int o0 = to * (kTile / 2);
  Loader<T, false, 64 * ET> a;
  Loader<T, false, kTile> b;
  a.aim([&](int i, bool &there) { there = true; return x.p + min(t0 + i, x.lines - 1) * x.s; }, 1);
  b.aim([&](int i, bool &there) {
    there = true;
    return (i < kTile / 2 ? w_gate : w_up) + (int64_t)min(o0 + i % (kTile / 2), p.outs - 1) * ldw;
  }, 1);
  f32x16 acc[2][ET] = {};
  multiply<T, false, false, ET>(a, b, split * n.chunk, min(k, (split + 1) * n.chunk), wm, [&](int e) { return e * (kTile / 2) + wn * 32; }, false, lds, acc);
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    const int64_t t = t0 + (wm * ET + r) * 32 + ln;
    const int ow = o0 + wn * 32;
    if constexpr (PARTS) {
      if (t >= p.rows) continue;
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          float *q = part + ((split * p.rows + t) * 2 + e) * p.room + ow + result_line(i, half);
          *reinterpret_cast<f32x4_any *>(q) = f32x4_any{acc[e][r][i], acc[e][r][i + 1], acc[e][r][i + 2], acc[e][r][i + 3]};
        }
    } else {
      uint32_t gb = 0, ub = 0;
      if (!BACK && p.codes) {
        uint32_t m[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            if (ow + result_line(i, half) >= p.outs) acc[e][r][i] = 0.f;
            m[e] = max(m[e], __float_as_uint(acc[e][r][i]) & 0x7fffffffu);
          }
          m[e] = max(m[e], (uint32_t)__shfl_xor((int)m[e], 32, 64));
        }
        gb = step_of(m[0]), ub = step_of(m[1]);
      }
      if (t >= p.rows) continue;
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        float g[4], u[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) g[j] = acc[0][r][i + j], u[j] = acc[1][r][i + j];
        finish<T, ACT, BACK>(p, t, ow + result_line(i, half), g, u, gb, ub);
      }
    }
  }
}

// the ranges' sums joined: 4 outputs a thread, 8 neighbours a block
template <class T, int ACT, bool BACK>
__global__ __launch_bounds__(256) void gate_join_kernel(Gate<T> p, int splits, const float *__restrict__ part) {
  const int64_t quads = p.room / 4, i = (int64_t)blockIdx.x * 256 + threadIdx.x, t = i / quads;
  const int o = (int)(i % quads) * 4;
  if (t >= p.rows) return;
  float g[4] = {}, u[4] = {};
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    const float *q = part + (s * p.rows + t) * 2 * p.room + o;
    const f32x4_any a = *reinterpret_cast<const f32x4_any *>(q), b = *reinterpret_cast<const f32x4_any *>(q + p.room);
#pragma unroll
    for (int j = 0; j < 4; ++j) g[j] += a[j], u[j] += b[j];
  }
  uint32_t gb = 0, ub = 0;
  if (!BACK && p.codes) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (o + j >= p.outs) g[j] = u[j] = 0.f;
      gb = max(gb, __float_as_uint(g[j]) & 0x7fffffffu), ub = max(ub, __float_as_uint(u[j]) & 0x7fffffffu);
    }
#pragma unroll
    for (int off = 1; off < 8; off <<= 1)
      gb = max(gb, (uint32_t)__shfl_xor((int)gb, off, 64)), ub = max(ub, (uint32_t)__shfl_xor((int)ub, off, 64));
    gb = step_of(gb), ub = step_of(ub);
  }
  finish<T, ACT, BACK>(p, t, o, g, u, gb, ub);
}

// ---- products of one result ----------------------------------------------------------------------------------
template <class T, int ET, bool AT, bool PARTS>
__global__ __launch_bounds__(256, 2) void product_tile_kernel(Product<T> p, Grid n, float *__restrict__ part) {
  __shared__ __align__(16) unsigned char lds[2][(64 * ET + kTile) * kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5, wm = wv >> 1, wn = wv & 1;
  const int64_t at = in_runs(blockIdx.x, n.tiles * n.splits), split = at / n.tiles;
  int64_t tt;
  int to;
  tile_of(at % n.tiles, n.tiles_r, (int)n.tiles_o, tt, to);
  const int batch = blockIdx.y;
  const int64_t r0 = tt * (64 * ET), o0 = (int64_t)to * kTile, rows = p.a[0].lines, lines = p.b[0].lines;
  f32x16 acc[2][ET] = {};
  for (int f = 0; f < p.phases; ++f) {
    const Side<T> sa = p.a[f * p.batches + batch], sb = p.b[f * p.batches + batch];
    Loader<T, AT, 64 * ET> a;
    Loader<T, true, kTile> b;
    a.aim([&](int i, bool &there) {
      there = r0 + i < rows;
      return sa.p + min(r0 + i, rows - 1) * (AT ? 1 : sa.s);
    }, sa.s);
    b.aim([&](int i, bool &there) {
      there = o0 + i < lines;
      return sb.p + min(o0 + i, lines - 1);
    }, sb.s);
    multiply<T, AT, true, ET>(a, b, split * n.chunk, min(p.k, (split + 1) * n.chunk), wm, [&](int e) { return wn * 64 + e * 32; }, f >= p.second, lds, acc);
  }
#pragma unroll
  for (int r = 0; r < ET; ++r) {
    const int64_t t = r0 + (wm * ET + r) * 32 + ln;
    if (t >= rows) continue;
#pragma unroll
    for (int e = 0; e < 2; ++e)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t o = o0 + wn * 64 + e * 32 + result_line(i, half);
        if (o >= lines) continue;
        if constexpr (PARTS) part[((split * p.batches + batch) * rows + t) * lines + o] = acc[e][r][i];
        else p.out[batch][t * p.ld + o] = narrow<T>(acc[e][r][i]);
      }
  }
}

template <class T>
__global__ __launch_bounds__(256) void product_join_kernel(Product<T> p, int splits, const float *__restrict__ part) {
  const int64_t rows = p.a[0].lines, lines = p.b[0].lines, all = rows * lines;
  const int batch = blockIdx.y;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    float v = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v += part[(s * p.batches + batch) * all + i];
    p.out[batch][i / lines * p.ld + i % lines] = narrow<T>(v);
  }
}

int64_t tiles(int64_t n, int64_t size) { return (n + size - 1) / size; }

// Tiles of 64 rows where those of 128 leave compute units without work; ranges of k, two stages at least, up to two workgroups a
// compute unit.
Grid grid_of(int64_t rows, int64_t lines, int64_t width, int64_t k, int batches, int size) {
  Grid g;
  g.tiles_o = tiles(lines, width);
  g.et = rows <= 64 || tiles(rows, 128) * g.tiles_o * batches < 256 ? 1 : 2;
  g.tiles_r = tiles(rows, 64 * g.et), g.tiles = g.tiles_r * g.tiles_o;
  const int64_t least = 2 * kStage / size;
  const int64_t want = std::min<int64_t>({512 / std::max<int64_t>(g.tiles * batches, 1), std::max<int64_t>(k / least, 1), 16});
  g.chunk = tiles(tiles(k, std::max<int64_t>(want, 1)), kStage / size) * (kStage / size);
  g.splits = (int)tiles(k, g.chunk);
  return g;
}

template <class F>
hipError_t by_act(int act, F f) {
  switch (act) {
    case WCC_ACT_RELU: return f(std::integral_constant<int, WCC_ACT_RELU>());
    case WCC_ACT_SILU: return f(std::integral_constant<int, WCC_ACT_SILU>());
    case WCC_ACT_GELU: return f(std::integral_constant<int, WCC_ACT_GELU>());
    default: return f(std::integral_constant<int, WCC_ACT_NONE>());
  }
}

}  // namespace

size_t tile_gate_parts(int64_t rows, int64_t outs, int64_t k, int size) {
  const Grid n = grid_of(rows, outs, kTile / 2, k, 1, size);
  return n.splits > 1 ? (size_t)n.splits * rows * 2 * room_of(outs) * sizeof(float) : 0;
}
size_t tile_product_parts(int64_t rows, int64_t lines, int64_t k, int batches, int size) {
  const Grid n = grid_of(rows, lines, kTile, k, batches, size);
  return n.splits > 1 ? (size_t)n.splits * batches * rows * lines * sizeof(float) : 0;
}

template <class T>
hipError_t join_gate(const Gate<T> &p, int act, bool back, int splits, const float *part, hipStream_t s) {
  const unsigned n = (unsigned)tiles(p.rows * (p.room / 4), 256);
  return by_act(act, [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    if (back) gate_join_kernel<T, ACT, true><<<n, 256, 0, s>>>(p, splits, part);
    else gate_join_kernel<T, ACT, false><<<n, 256, 0, s>>>(p, splits, part);
    return hipGetLastError();
  });
}
template hipError_t join_gate<float>(const Gate<float> &, int, bool, int, const float *, hipStream_t);
template hipError_t join_gate<bf16_t>(const Gate<bf16_t> &, int, bool, int, const float *, hipStream_t);

template <class T>
hipError_t tile_gate(const Gate<T> &p, int act, bool back, const Side<T> &x, const T *w_gate, const T *w_up, int64_t ldw, int64_t k,
                     float *part, hipStream_t s) {
  const Grid n = grid_of(p.rows, p.outs, kTile / 2, k, 1, sizeof(T));
  const unsigned blocks = (unsigned)(n.tiles * n.splits);
  return by_act(act, [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    auto go = [&](auto size) {
      constexpr int ET = decltype(size)::value;
      if (n.splits > 1) {
        gate_tile_kernel<T, ET, WCC_ACT_NONE, false, true><<<blocks, 256, 0, s>>>(p, x, w_gate, w_up, ldw, k, n, part);
      } else if (back) {
        gate_tile_kernel<T, ET, ACT, true, false><<<blocks, 256, 0, s>>>(p, x, w_gate, w_up, ldw, k, n, part);
      } else {
        gate_tile_kernel<T, ET, ACT, false, false><<<blocks, 256, 0, s>>>(p, x, w_gate, w_up, ldw, k, n, part);
      }
    };
    if (n.et == 1) go(std::integral_constant<int, 1>());
    else go(std::integral_constant<int, 2>());
    const hipError_t e = hipGetLastError();
    return e != hipSuccess || n.splits == 1 ? e : join_gate<T>(p, act, back, n.splits, part, s);
  });
}

template <class T, bool AT>
hipError_t tile_product(const Product<T> &p, float *part, hipStream_t s) {
  const int64_t rows = p.a[0].lines, lines = p.b[0].lines;
  const Grid n = grid_of(rows, lines, kTile, p.k, AT ? 2 : 1, sizeof(T));  // (the same for one of the weights' gradients as for both)
  const dim3 blocks((unsigned)(n.tiles * n.splits), p.batches);
  auto go = [&](auto size) {
    constexpr int ET = decltype(size)::value;
    if (n.splits > 1) {
      product_tile_kernel<T, ET, AT, true><<<blocks, 256, 0, s>>>(p, n, part);
      product_join_kernel<T><<<dim3((unsigned)std::min<int64_t>(tiles(rows * lines, 256), 1 << 16), p.batches), 256, 0, s>>>(p, n.splits, part);
    } else {
      product_tile_kernel<T, ET, AT, false><<<blocks, 256, 0, s>>>(p, n, part);
    }
  };
  if (n.et == 1) go(std::integral_constant<int, 1>());
  else go(std::integral_constant<int, 2>());
  return hipGetLastError();
}

template hipError_t tile_gate<float>(const Gate<float> &, int, bool, const Side<float> &, const float *, const float *, int64_t, int64_t,
                                     float *, hipStream_t);
template hipError_t tile_gate<bf16_t>(const Gate<bf16_t> &, int, bool, const Side<bf16_t> &, const bf16_t *, const bf16_t *, int64_t,
                                      int64_t, float *, hipStream_t);
template hipError_t tile_product<float, false>(const Product<float> &, float *, hipStream_t);
template hipError_t tile_product<float, true>(const Product<float> &, float *, hipStream_t);
template hipError_t tile_product<bf16_t, false>(const Product<bf16_t> &, float *, hipStream_t);
template hipError_t tile_product<bf16_t, true>(const Product<bf16_t> &, float *, hipStream_t);

}  // namespace wcc

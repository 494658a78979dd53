// The projection for many rows: tiles of 128 rows x 128 outputs through LDS, any type, alignment and order of W.
//
// Four waves of 64 x 64 each; stages of 128 bytes of k (64 bf16 or 32 fp32), two in LDS, the next one's loads in flight
// while one is multiplied.  LDS rows are 144 bytes apart, which spreads the 16-byte reads of 32 rows over all banks.
// Where W's outputs are contiguous and not its k (the gradient of x), a thread loads pairs of outputs of eight (four) k and
// exchanges halves, so that LDS holds the same rows of k either way.
// The thin product of the rank lines comes last (add_thin); with ranges of k it is left, with their sum, to another launch.
// fp32 is bound by the matrix cores: 2048 rows, 2048 -> 4096 316 us, 79% of their cycles at the clock the card keeps (2.13 GHz).  bf16
// rows at odd addresses are bound by their loads: 1172 rows, 2816 -> 4224 98 us, 0.28 PFLOP/s (large products: copied, adapter.hip).
#include "adapter.h"

namespace wcc {
namespace {

constexpr int kTile = 128, kRowBytes = 144, kStage = 128;

template <class T, bool NN, bool PARTS>
__global__ __launch_bounds__(256, 2) void project_tile_kernel(Project<T> p, int64_t tiles_t, int tiles_o, int splits, int chunk,
                                                              float *__restrict__ part, ThinJob<T> thin, ThinJob<T> other) {
  constexpr int VE = VecOf<T>::N, KB = kStage / (int)sizeof(T);
  __shared__ __align__(1024) unsigned char lds[2][2 * kTile][kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5;
  const int wm = wv >> 1, wn = wv & 1;
  const int64_t lines = PARTS ? thin.blocks + other.blocks : 0;
  if constexpr (PARTS) {
    if (blockIdx.x < lines) {
      __shared__ ThinLds order;
      unsigned char *own = &lds[0][0][0] + wv * kThinRoom;
      if (blockIdx.x < thin.blocks) thin_block<T>(thin, p.low, blockIdx.x, order, own);
      else thin_block<T>(other, p.low, blockIdx.x - thin.blocks, order, own);
      return;
    }
  }
  const int64_t tiles = tiles_t * tiles_o;
  for (int64_t b = blockIdx.x - lines; b < tiles * splits; b += gridDim.x - lines) {
    const int64_t at = in_runs(b, tiles * splits);
    const int split = (int)(at / tiles), k0 = split * chunk, k1 = min(p.width, k0 + chunk);
    int64_t tt;
    int to;
    tile_of(at % tiles, tiles_t, tiles_o, tt, to);
    const int64_t t0 = tt * kTile;
    const int o0 = to * kTile;
    const int row = tid >> 3, chunk8 = tid & 7;
    const T *px[4], *pw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      px[i] = p.x + min(t0 + row + 32 * i, p.rows - 1) * p.ldx + chunk8 * VE;
      if (!NN) pw[i] = p.w + (int64_t)min(o0 + row + 32 * i, p.outs - 1) * p.wo + chunk8 * VE;
    }
    const int pair = tid & 63, kg = tid >> 6;
    const bool both = o0 + 2 * pair + 1 < p.outs;
    if (NN) pw[0] = p.w + min(o0 + 2 * pair, p.outs - 1);
    const bool all = o0 + kTile <= p.outs;
    u32x4 st[8];
    auto load = [&](int k) {
      if (k + KB <= k1 && (!NN || all)) {  // (nothing to check: no branch between the loads)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          st[i] = *reinterpret_cast<const u32x4_any *>(px[i] + k);
          if (!NN) st[4 + i] = *reinterpret_cast<const u32x4_any *>(pw[i] + k);
        }
        if (NN) {
#pragma unroll
          for (int i = 0; i < 2; ++i) load_k_pair(pw[0] + (k + (kg + 4 * i) * VE) * p.wk, p.wk, VE, true, st[4 + 2 * i], st[5 + 2 * i]);
        }
        return;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int left = k1 - k - chunk8 * VE;
        st[i] = load_k(px[i] + k, left);
        if (!NN) st[4 + i] = load_k(pw[i] + k, left);
      }
      if (NN) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int kk = k + (kg + 4 * i) * VE;
          load_k_pair(pw[0] + kk * p.wk, p.wk, k1 - kk, both, st[4 + 2 * i], st[5 + 2 * i]);
        }
      }
    };
    auto store = [&](int buf) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<u32x4 *>(&lds[buf][row + 32 * i][chunk8 * 16]) = st[i];
        if (!NN) *reinterpret_cast<u32x4 *>(&lds[buf][kTile + row + 32 * i][chunk8 * 16]) = st[4 + i];
      }
      if (NN) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          *reinterpret_cast<u32x4 *>(&lds[buf][kTile + 2 * pair][(kg + 4 * i) * 16]) = st[4 + 2 * i];
          *reinterpret_cast<u32x4 *>(&lds[buf][kTile + 2 * pair + 1][(kg + 4 * i) * 16]) = st[5 + 2 * i];
        }
      }
    };
    f32x16 acc[2][2] = {};
    load(k0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int k = k0; k < k1; k += KB, buf ^= 1) {
      if (k + KB < k1) load(k + KB);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        u32x4 xf[2], wf[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          xf[r] = *reinterpret_cast<const u32x4 *>(&lds[buf][wm * 64 + r * 32 + ln][ks * 32 + half * 16]);
          wf[r] = *reinterpret_cast<const u32x4 *>(&lds[buf][kTile + wn * 64 + r * 32 + ln][ks * 32 + half * 16]);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < 2; ++e) acc[e][r] = mma<T>(xf[r], wf[e], acc[e][r]);
      }
      if (k + KB < k1) store(buf ^ 1);
      __syncthreads();
    }
    const int o[2] = {o0 + wn * 64 + ln, o0 + wn * 64 + 32 + ln};
    T *h = reinterpret_cast<T *>(&lds[0][0][0]);
    if constexpr (!PARTS) {
      if (p.low.of_row) {
        auto room = [&](int row) { return h + row * PartsOf<T>::Out * p.h.ld; };
        gather_lines<T, kTile>(p.low, p.h, room, t0, p.rows);
        __syncthreads();
        auto lines_of = [&](int r) { return room(wm * 64 + r * 32); };
        add_thin<T, 2, 2, true, 2>(p.low, p.m, p.h.ld, lines_of, p.rows, p.outs, t0 + wm * 64, o, acc);
        __syncthreads();
      }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t tr = t0 + wm * 64 + r * 32;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t t = tr + result_line(i, half);
        if (t >= p.rows) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (o[e] < p.outs) {
            if constexpr (PARTS) part[(split * p.rows + t) * p.outs + o[e]] = acc[e][r][i];
            else p.y[t * p.ldy + o[e]] = narrow<T>(acc[e][r][i]);
          }
      }
    }
  }
}

}  // namespace

int64_t tiles_of(int64_t rows, int outs) { return ((rows + kTile - 1) / kTile) * ((outs + kTile - 1) / kTile); }
// Ranges of k of 512 bytes at least: as many as have places at once, 16 at most.
int tile_splits(int64_t rows, int width, int outs, int size) {
  const int64_t tiles = tiles_of(rows, outs);
  const int64_t want = std::clamp<int64_t>(kPlaces / tiles, 1, std::clamp<int64_t>((int64_t)width * size / 512, 1, 16));
  const int unit = kStage / size;
  const int64_t chunk = ((width + want - 1) / want + unit - 1) / unit * unit;
  return (int)((width + chunk - 1) / chunk);
}

template <class T>
void launch_tiles(const Project<T> &p, int splits, float *part, const ThinJob<T> &thin, const ThinJob<T> &other, hipStream_t s) {
  constexpr int unit = kStage / (int)sizeof(T);
  const int64_t tiles_t = (p.rows + kTile - 1) / kTile;
  const int tiles_o = (p.outs + kTile - 1) / kTile, chunk = ((p.width + splits - 1) / splits + unit - 1) / unit * unit;
  const unsigned blocks = (unsigned)(std::min<int64_t>(tiles_t * tiles_o * splits, 1 << 20) + (splits > 1 ? thin.blocks + other.blocks : 0));
  if (splits > 1) {
    if (p.wk == 1) project_tile_kernel<T, false, true><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
    else project_tile_kernel<T, true, true><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, splits, chunk, part, thin, other);
  } else {
    if (p.wk == 1) project_tile_kernel<T, false, false><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, 1, chunk, nullptr, {}, {});
    else project_tile_kernel<T, true, false><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o, 1, chunk, nullptr, {}, {});
  }
}
template void launch_tiles<bf16_t>(const Project<bf16_t> &, int, float *, const ThinJob<bf16_t> &, const ThinJob<bf16_t> &, hipStream_t);
template void launch_tiles<float>(const Project<float> &, int, float *, const ThinJob<float> &, const ThinJob<float> &, hipStream_t);

}  // namespace wcc

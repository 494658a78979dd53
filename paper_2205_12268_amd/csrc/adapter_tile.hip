// The projection for many rows: tiles of 128 rows x 128 outputs through LDS, any type, alignment and order of W.
//
// Four waves of 64 x 64 each; stages of 128 bytes of k (64 bf16 or 32 fp32), two in LDS, the next one's loads in flight
// while one is multiplied.  LDS rows are 144 bytes apart, which spreads the 16-byte reads of 32 rows over all banks.
// Where W's outputs are contiguous and not its k (the gradient of x), a thread loads pairs of outputs of eight (four) k and
// exchanges halves, so that LDS holds the same rows of k either way.
// The thin product of the rank lines comes last (add_thin).
#include "adapter.h"

namespace wcc {
namespace {

constexpr int kTile = 128, kRowBytes = 144, kStage = 128;

// Tiles in an order that leaves each of the eight XCDs (workgroups go to them in turn) a run of neighbours, and within a run
// blocks of up to eight row tiles, so that what neighbours share is in their L2.
__device__ __forceinline__ void tile_of(int64_t b, int64_t tiles, int64_t tiles_t, int tiles_o, int64_t &tt, int &to) {
  const int64_t each = tiles / 8;
  if (b < each * 8) b = b % 8 * each + b / 8;
  const int64_t band = (int64_t)8 * tiles_o, first = b / band * 8, in = b % band;
  const int64_t high = min(tiles_t - first, (int64_t)8);
  tt = first + in % high;
  to = (int)(in / high);
}

template <class T, bool NN>
__global__ __launch_bounds__(256, 2) void project_tile_kernel(Project<T> p, int64_t tiles_t, int tiles_o) {
  constexpr int VE = VecOf<T>::N, KB = kStage / (int)sizeof(T);
  __shared__ __align__(16) unsigned char lds[2][2 * kTile][kRowBytes];
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, ln = lane & 31, half = lane >> 5;
  const int wm = wv >> 1, wn = wv & 1;
  const int64_t tiles = tiles_t * tiles_o;
  for (int64_t b = blockIdx.x; b < tiles; b += gridDim.x) {
    int64_t tt;
    int to;
    tile_of(b, tiles, tiles_t, tiles_o, tt, to);
    const int64_t t0 = tt * kTile;
    const int o0 = to * kTile;
    const int row = tid >> 3, chunk = tid & 7;
    const T *px[4], *pw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      px[i] = p.x + min(t0 + row + 32 * i, p.rows - 1) * p.ldx + chunk * VE;
      if (!NN) pw[i] = p.w + (int64_t)min(o0 + row + 32 * i, p.outs - 1) * p.wo + chunk * VE;
    }
    const int pair = tid & 63, kg = tid >> 6;
    const bool both = o0 + 2 * pair + 1 < p.outs;
    if (NN) pw[0] = p.w + min(o0 + 2 * pair, p.outs - 1);
    u32x4 st[8];
    auto load = [&](int k) {
      const int left = p.width - k - chunk * VE;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        st[i] = load_k(px[i] + k, left);
        if (!NN) st[4 + i] = load_k(pw[i] + k, left);
      }
      if (NN) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int kk = k + (kg + 4 * i) * VE;
          load_k_pair(pw[0] + kk * p.wk, p.wk, p.width - kk, both, st[4 + 2 * i], st[5 + 2 * i]);
        }
      }
    };
    auto store = [&](int buf) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        *reinterpret_cast<u32x4 *>(&lds[buf][row + 32 * i][chunk * 16]) = st[i];
        if (!NN) *reinterpret_cast<u32x4 *>(&lds[buf][kTile + row + 32 * i][chunk * 16]) = st[4 + i];
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
    load(0);
    store(0);
    __syncthreads();
    int buf = 0;
    for (int k = 0; k < p.width; k += KB, buf ^= 1) {
      if (k + KB < p.width) load(k + KB);
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
          for (int e = 0; e < 2; ++e) acc[r][e] = mma<T>(xf[r], wf[e], acc[r][e]);
      }
      if (k + KB < p.width) store(buf ^ 1);
      __syncthreads();
    }
    const int o[2] = {o0 + wn * 64 + ln, o0 + wn * 64 + 32 + ln};
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const int64_t tr = t0 + wm * 64 + r * 32;
      if (p.low.of_row) add_thin<T, 2, true>(p.low, p.m, p.h, p.rows, p.outs, tr, o, acc[r]);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int64_t t = tr + result_line(i, half);
        if (t >= p.rows) continue;
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (o[e] < p.outs) p.y[t * p.ldy + o[e]] = narrow<T>(acc[r][e][i]);
      }
    }
  }
}

}  // namespace

template <class T>
void launch_tiles(const Project<T> &p, hipStream_t s) {
  const int64_t tiles_t = (p.rows + kTile - 1) / kTile;
  const int tiles_o = (p.outs + kTile - 1) / kTile;
  const unsigned blocks = (unsigned)std::min<int64_t>(tiles_t * tiles_o, 1 << 20);
  if (p.wk == 1) project_tile_kernel<T, false><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o);
  else project_tile_kernel<T, true><<<blocks, 256, 0, s>>>(p, tiles_t, tiles_o);
}
template void launch_tiles<bf16_t>(const Project<bf16_t> &, hipStream_t);
template void launch_tiles<float>(const Project<float> &, hipStream_t);

}  // namespace wcc

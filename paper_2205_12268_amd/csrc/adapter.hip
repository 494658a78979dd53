// One projection with a low-rank adapter for each row (wcc_adapter_forward, wcc_adapter_backward).
//
// Both directions are a product with W beside two thin ones that go through the rank lines of the row's adapter:
//   forward   h[t,j] = s_a sum_c A_a[j,c] x[t,c],    y[t,o]  = sum_c W[o,c] x[t,c]   + sum_j B_a[o,j] h[t,j]
//   backward  g[t,j] = s_a sum_o B_a[o,j] dy[t,o],   dx[t,c] = sum_o W[o,c] dy[t,o]  + sum_j A_a[j,c] g[t,j]
//   gradients dA_a[j,c] = sum_t g[t,j] x[t,c],       dB_a[o,j] = sum_t h[t,j] dy[t,o]
#include "head.h"

namespace wcc {
namespace {

// The adapters as the kernels see them.
struct Low {
  const int32_t *of_row;  // nullptr: none
  const int32_t *ranks;
  const float *scale;
  int n, rank;
  __device__ __forceinline__ int of(int64_t t) const {
    const int a = of_row ? of_row[t] : -1;
    return (uint32_t)a < (uint32_t)n ? a : -1;
  }
  __device__ __forceinline__ int lines(int a) const { return ranks ? min(max(ranks[a], 0), rank) : rank; }
  __device__ __forceinline__ float factor(int a) const { return scale ? scale[a] : 1.f; }
};

// h[t, j] for all rows, 0 past the adapter's rank or without one; one wave an entry.  m: lines [n, ...] with element
// (a, j, c) at (a * major + j * sj + c * sc).
template <class T>
__global__ __launch_bounds__(256) void low_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int width, Low low,
                                                  const T *__restrict__ m, int64_t major, int64_t sj, int64_t sc,
                                                  float *__restrict__ h) {
  const int lane = threadIdx.x & 63;
  const int64_t total = rows * low.rank, step = (int64_t)gridDim.x * 4;
  for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < total; i += step) {
    const int64_t t = i / low.rank;
    const int j = (int)(i - t * low.rank), a = low.of(t);
    float v = 0.f;
    if (a >= 0 && j < low.lines(a)) {
      const T *line = m + a * major + j * sj;
      for (int c = lane; c < width; c += 64) v = fmaf(widen(line[c * sc]), widen(x[t * ldx + c]), v);
      for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
      v *= low.factor(a);
    }
    if (lane == 0) h[i] = v;
  }
}

// y[t, o] = sum_c w(o, c) x[t, c] + sum_j m(a, j, o) h[t, j];  w(o, c) at o * wo + c * wc, m as above.
// 64 x 64 results a workgroup, 4 x 4 a thread, both operands through LDS in steps of 16.
template <class T>
__global__ __launch_bounds__(256) void project_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int width,
                                                      const T *__restrict__ w, int64_t wo, int64_t wc, int outs, Low low,
                                                      const T *__restrict__ m, int64_t major, int64_t sj, int64_t so,
                                                      const float *__restrict__ h, T *__restrict__ y, int64_t ldy) {
  __shared__ float xs[16][65], ws[16][65];
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int tiles_o = (outs + 63) / 64;
  const int64_t tiles = (rows + 63) / 64 * tiles_o;
  for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
  const int64_t t0 = tile / tiles_o * 64;
  const int o0 = (int)(tile % tiles_o) * 64;
  float acc[4][4] = {};
  for (int c0 = 0; c0 < width; c0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      const int r = i >> 4, c = c0 + (i & 15);
      xs[i & 15][r] = t0 + r < rows && c < width ? widen(x[(t0 + r) * ldx + c]) : 0.f;
      ws[i & 15][r] = o0 + r < outs && c < width ? widen(w[(o0 + r) * wo + c * wc]) : 0.f;
    }
    __syncthreads();
    for (int c = 0; c < 16; ++c)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(xs[c][ty * 4 + i], ws[c][tx * 4 + j], acc[i][j]);
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const int64_t t = t0 + ty * 4 + i;
    if (t >= rows) break;
    const int a = low.of(t), lines = a >= 0 ? low.lines(a) : 0;
    for (int j = 0; j < 4; ++j) {
      const int o = o0 + tx * 4 + j;
      if (o >= outs) break;
      float v = acc[i][j];
      for (int l = 0; l < lines; ++l) v = fmaf(widen(m[a * major + l * sj + o * so]), h[t * low.rank + l], v);
      y[t * ldy + o] = narrow<T>(v);
    }
  }
  }
}

// grad(a, j, c) = sum over the rows of adapter a of h[t, j] x[t, c], to a * major + j * sj + c * sc; a thread an entry.
template <class T>
__global__ __launch_bounds__(256) void low_grad_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int width, Low low,
                                                       const float *__restrict__ h, float *__restrict__ grad, int64_t major,
                                                       int64_t sj, int64_t sc) {
  const int64_t total = (int64_t)low.n * low.rank * width, step = (int64_t)gridDim.x * 256;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += step) {
    const int c = (int)(i % width), line = (int)(i / width), a = line / low.rank, j = line % low.rank;
    float v = 0.f;
    if (j < low.lines(a))
      for (int64_t t = 0; t < rows; ++t)
        if (low.of(t) == a) v = fmaf(h[t * low.rank + j], widen(x[t * ldx + c]), v);
    grad[a * major + j * sj + c * sc] = v;
  }
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }
size_t thin_bytes(const wcc_adapter_desc &d) { return align256((size_t)d.rows * d.rank * 4); }

Low low_of(const wcc_adapter_desc &d, const AdapterArgs &g) { return Low{g.of_row, g.ranks, g.scale, d.adapters, d.rank}; }

template <class T>
void thin(const wcc_adapter_desc &d, const AdapterArgs &g, bool back, float *h, hipStream_t s) {
  const int64_t total = d.rows * d.rank;
  if (!g.of_row || total == 0) return;
  const unsigned blocks = (unsigned)std::min<int64_t>((total + 3) / 4, 1 << 20);
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank;
  if (!back)
    low_kernel<T><<<blocks, 256, 0, s>>>((const T *)g.x, d.ldx, d.rows, d.C_in, low_of(d, g), (const T *)g.a, r * ci, ci, 1, h);
  else
    low_kernel<T><<<blocks, 256, 0, s>>>((const T *)g.dy, d.ldy, d.rows, d.C_out, low_of(d, g), (const T *)g.b, co * r, 1, r, h);
}

template <class T>
void forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  float *h = (float *)g.ws;
  thin<T>(d, g, false, h, s);
  const unsigned grid = (unsigned)std::min<int64_t>((int64_t)((d.C_out + 63) / 64) * ((d.rows + 63) / 64), 1 << 20);
  project_kernel<T><<<grid, 256, 0, s>>>((const T *)g.x, d.ldx, d.rows, d.C_in, (const T *)g.w, d.C_in, 1, d.C_out, low_of(d, g),
                                         (const T *)g.b, (int64_t)d.C_out * d.rank, 1, d.rank, h, (T *)g.y, d.ldy);
}

template <class T>
void backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  float *gr = (float *)g.ws, *h = (float *)(g.ws + thin_bytes(d));
  const int64_t ci = d.C_in, co = d.C_out, r = d.rank;
  if (g.y || g.da) thin<T>(d, g, true, gr, s);
  if (g.db) thin<T>(d, g, false, h, s);
  if (g.y) {
    const unsigned grid = (unsigned)std::min<int64_t>((int64_t)((d.C_in + 63) / 64) * ((d.rows + 63) / 64), 1 << 20);
    project_kernel<T><<<grid, 256, 0, s>>>((const T *)g.dy, d.ldy, d.rows, d.C_out, (const T *)g.w, 1, d.C_in, d.C_in, low_of(d, g),
                                           (const T *)g.a, r * ci, ci, 1, gr, (T *)g.y, d.ldx);
  }
  auto blocks = [&](int width) { return (unsigned)std::min<int64_t>((d.adapters * r * width + 255) / 256, 1 << 20); };
  if (g.da)
    low_grad_kernel<T><<<blocks(d.C_in), 256, 0, s>>>((const T *)g.x, d.ldx, d.rows, d.C_in, low_of(d, g), gr,
                                                                        g.da, r * ci, ci, 1);
  if (g.db)
    low_grad_kernel<T><<<blocks(d.C_out), 256, 0, s>>>((const T *)g.dy, d.ldy, d.rows, d.C_out, low_of(d, g),
                                                                         h, g.db, co * r, 1, r);
}

}  // namespace

size_t adapter_bytes(const wcc_adapter_desc &d) { return 2 * thin_bytes(d); }

hipError_t launch_adapter_forward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  if (d.dtype == WCC_BF16) forward<bf16_t>(d, g, s);
  else forward<float>(d, g, s);
  return hipGetLastError();
}

hipError_t launch_adapter_backward(const wcc_adapter_desc &d, const AdapterArgs &g, hipStream_t s) {
  if (d.dtype == WCC_BF16) backward<bf16_t>(d, g, s);
  else backward<float>(d, g, s);
  return hipGetLastError();
}

}  // namespace wcc

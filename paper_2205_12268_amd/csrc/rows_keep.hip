// Rows in 8 bits and back (the format: block.h).
//
// A lane has 16 bytes of x; the 4 (bf16) or 8 (fp32) lanes of a block exchange their largest magnitude.  Rows of codes are whole
// blocks, zeros behind the last value, so that whoever reads them needs no edge.  Bound by memory: 131072 rows of 256 bf16 take 22 us to codes and 16
// back (4.7 and 6.3 TB/s, the codes still in the caches; a large copy reaches 5.3), 1777 of 1001 fp32 at odd strides 4.2 and 3.9.
#include "block.h"

namespace wcc {
namespace {

// Vector i of a matrix whose rows have `per_row` vectors, in steps of `step`: row and place move by whole numbers made once, so that no
// lane divides but at its start.
struct Walk {
  int64_t row, d_row;
  int at, d_at, per_row;
  __device__ __forceinline__ Walk(int64_t i, int64_t step, int per_row_) : per_row(per_row_) {
    row = i / per_row, at = (int)(i - row * per_row);
    d_row = step / per_row, d_at = (int)(step - d_row * per_row);
  }
  __device__ __forceinline__ void next() {
    row += d_row, at += d_at;
    if (at >= per_row) at -= per_row, ++row;
  }
};

template <class T>
__global__ __launch_bounds__(256) void keep_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int width, int per_row,
                                                   int8_t *__restrict__ codes, uint8_t *__restrict__ steps) {
  constexpr int VE = VecOf<T>::N, Lanes = kKept / VE;
  // (256 is whole blocks, so a block's lanes are neighbours in one wave and leave the loop together)
  Walk w((int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, per_row);
  for (; w.row < rows; w.next()) {
    const u32x4 v = load_part<T>(x + w.row * ld + w.at * VE, width - w.at * VE);
    const uint32_t b = step_of(top_of_block<T>(v));
    const int64_t flat = w.row * per_row + w.at;
    store_codes<T>(codes + flat * VE, v, per_step(b));
    if ((threadIdx.x & (Lanes - 1)) == 0) steps[flat / Lanes] = (uint8_t)b;
  }
}

template <class T>
__global__ __launch_bounds__(256) void restore_kernel(const int8_t *__restrict__ codes, const uint8_t *__restrict__ steps, int64_t ld,
                                                      int64_t rows, int width, int per_row, T *__restrict__ x) {
  constexpr int VE = VecOf<T>::N, Lanes = kKept / VE;
  Walk w((int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, per_row);
  for (; w.row < rows; w.next()) {
    const int64_t flat = w.row * per_row + w.at;
    const float step = step_value(steps[flat / Lanes]);
    float f[VE];
#pragma unroll
    for (int h = 0; h < VE / 4; ++h) {
      const uint32_t c = reinterpret_cast<const uint32_t *>(codes + flat * VE)[h];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * h + j] = kept_value(c, j, step);
    }
    store_part<T>(x + w.row * ld + w.at * VE, width - w.at * VE, pack<T>(f));
  }
}

template <class T>
unsigned grid_of(const wcc_rows_desc &d, int &per_row) {
  per_row = (int)(kept_blocks(d.width) * (kKept / VecOf<T>::N));
  return (unsigned)std::min<int64_t>((d.rows * per_row + 255) / 256, 256 * 8 * 4);
}

}  // namespace

hipError_t launch_keep(const wcc_rows_desc &d, const KeepArgs &g, hipStream_t s) {
  int per_row;
  if (d.dtype == WCC_F32) {
    const unsigned n = grid_of<float>(d, per_row);
    keep_kernel<float><<<n, 256, 0, s>>>(static_cast<const float *>(g.x), d.ld, d.rows, d.width, per_row, g.codes, g.steps);
  } else {
    const unsigned n = grid_of<bf16_t>(d, per_row);
    keep_kernel<bf16_t><<<n, 256, 0, s>>>(static_cast<const bf16_t *>(g.x), d.ld, d.rows, d.width, per_row, g.codes, g.steps);
  }
  return hipGetLastError();
}

hipError_t launch_restore(const wcc_rows_desc &d, const KeepArgs &g, hipStream_t s) {
  int per_row;
  if (d.dtype == WCC_F32) {
    const unsigned n = grid_of<float>(d, per_row);
    restore_kernel<float><<<n, 256, 0, s>>>(g.codes, g.steps, d.ld, d.rows, d.width, per_row, static_cast<float *>(g.back));
  } else {
    const unsigned n = grid_of<bf16_t>(d, per_row);
    restore_kernel<bf16_t><<<n, 256, 0, s>>>(g.codes, g.steps, d.ld, d.rows, d.width, per_row, static_cast<bf16_t *>(g.back));
  }
  return hipGetLastError();
}

}  // namespace wcc

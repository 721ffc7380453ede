// Dropout with a counter-based generator (gfx950): element (r, j) of a
// [rows][cols] tensor is kept if bits [16 (j % 4), +16) of SplitMix64's output
// number r ceil(cols / 4) + j / 4 are at least the threshold.  Nothing is
// stored: the backward pass draws the same numbers again.
#include "runtime.h"
#include "ops.h"

namespace {

// one thread per word of four draws
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(int64_t rows, int64_t cols, const T *x, int64_t ldx, T *y,
                                                      int64_t ldy, Drop d) {
  const int64_t words = (cols + 3) >> 2, total = rows * words;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / words, c = (i - r * words) * 4;
    const uint64_t w = drop_word(d.key, r, words, (int)(c >> 2));
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < cols) {
        const float v = ElemT<T>::to_f(x[r * ldx + c + j]);
        y[r * ldy + c + j] = ElemT<T>::from_f(drop_keeps(w, j, d.thr) ? v * d.scale : 0.f);
      }
  }
}

template <typename T>
hipError_t run(int64_t rows, int64_t cols, const void *x, int64_t ldx, void *y, int64_t ldy, const Drop &d,
               hipStream_t s) {
  const int64_t total = rows * ((cols + 3) >> 2), blocks = (total + 255) / 256;
  hipLaunchKernelGGL(dropout_kernel<T>, dim3((uint32_t)(blocks < 16384 ? blocks : 16384)), dim3(256), 0, s, rows, cols,
                     (const T *)x, ldx, (T *)y, ldy, d);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *y, int64_t ldy,
                          const Drop &d, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(rows, cols, x, ldx, y, ldy, d, s)
                             : run<float>(rows, cols, x, ldx, y, ldy, d, s);
}

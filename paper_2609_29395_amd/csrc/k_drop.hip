// Dropout with a counter-based generator (gfx950): element (r, j) of a
// [rows][cols] tensor is kept if bits [16 (j % 4), +16) of SplitMix64's output
// number r ceil(cols / 4) + j / 4 are at least the threshold.  Nothing is
// stored: the backward pass draws the same numbers again.
//
// A thread takes eight elements, two words of draws, at a time: the finaliser's
// two 64-bit products (24 of its 40 or so lane cycles) are spread over four
// elements, so that reading and writing bounds the kernel.  Four such pieces a
// thread are loaded before the first is used; 16-byte accesses at any
// alignment.
//
// Bound: memory; 32,768 x 4096, bf16, 96 us (5.6 TB/s, a copy of 1 GiB 5.05),
// where a draw for every element took 193.
#include <algorithm>

#include "runtime.h"
#include "ops.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // global memory takes 16-byte accesses at any alignment

constexpr int PER = 8;  // elements of a piece

template <typename T, int PIECES>
__global__ void __launch_bounds__(256) dropout_kernel(uint32_t total, FastDiv fd_row, int64_t row0, int cols,
                                                      const T *x, int64_t ldx, T *y, int64_t ldy, Drop d) {
  constexpr int NW = PER * sizeof(T) / 16, VEC = 16 / sizeof(T);  // 16-byte vectors of a piece, elements of one
  const int64_t words = (cols + 3) >> 2;
  u32x4 w[PIECES][NW];
  int64_t row[PIECES];
  int col[PIECES];
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    const uint32_t u = (blockIdx.x * PIECES + p) * 256 + threadIdx.x;
    const uint32_t r = fdiv(u, fd_row);
    row[p] = row0 + r;
    col[p] = u < total ? (int)(u - r * fd_row.d) * PER : cols;
    const T *in = x + row[p] * ldx + col[p];
    if (col[p] + PER <= cols) {
#pragma unroll
      for (int i = 0; i < NW; ++i) w[p][i] = *(const u32x4_any *)(in + i * VEC);
    } else if (col[p] < cols) {  // the row's end: elements past it are taken as its last one
#pragma unroll
      for (int i = 0; i < NW; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const auto bits = [&](int k) -> uint32_t {
            const T v = in[min(k, cols - 1 - col[p])];
            if constexpr (sizeof(T) == 2) return v;
            else return __float_as_uint(v);
          };
          if constexpr (sizeof(T) == 2) w[p][i][j] = bits(2 * j) | bits(2 * j + 1) << 16;
          else w[p][i][j] = bits(4 * i + j);
        }
    }
  }
#pragma unroll
  for (int p = 0; p < PIECES; ++p) {
    if (col[p] >= cols) continue;
    const uint64_t state = d.key + (uint64_t)(row[p] * words + (col[p] >> 2) + 1) * GCPSL_GOLDEN;
    const uint64_t draw[2] = {gc_mix64(state), gc_mix64(state + GCPSL_GOLDEN)};
    const auto value = [&](float v, int j) { return drop_keeps(draw[j >> 2], j & 3, d.thr) ? v * d.scale : 0.f; };
    T *out = y + row[p] * ldy + col[p];
    const bool whole = col[p] + PER <= cols;
#pragma unroll
    for (int i = 0; i < NW; ++i) {
      u32x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t b = w[p][i][j];
        if constexpr (sizeof(T) == 2)
          o[j] = pack2_bf16(value(__uint_as_float(b << 16), 2 * j), value(__uint_as_float(b & 0xffff0000u), 2 * j + 1));
        else
          o[j] = __float_as_uint(value(__uint_as_float(b), 4 * i + j));
      }
      if (whole) {
        *(u32x4_any *)(out + i * VEC) = o;
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (col[p] + i * VEC + j < cols) {
            if constexpr (sizeof(T) == 2) out[j] = (T)(o[j >> 1] >> (j & 1) * 16);
            else out[i * VEC + j] = __uint_as_float(o[j]);
          }
      }
    }
  }
}

// Four pieces a thread, but one where that leaves CUs without eight waves.
constexpr int PIECES = 4;
constexpr uint32_t kFew = 256 * 512 * PIECES;

template <typename T>
hipError_t run(int64_t rows, int64_t cols, const void *x, int64_t ldx, void *y, int64_t ldy, const Drop &d,
               hipStream_t s) {
  const int64_t row_pieces = (cols + PER - 1) / PER;
  const FastDiv fd = make_fastdiv((uint32_t)row_pieces);
  // launches of at most 2^30 pieces, whose number is a 32-bit one
  const int64_t slab = std::max<int64_t>(1, (1 << 30) / row_pieces);
  for (int64_t r = 0; r < rows; r += slab) {
    const uint32_t total = (uint32_t)(std::min(slab, rows - r) * row_pieces);
    const auto launch = [&](auto kernel, uint32_t threads) {
      hipLaunchKernelGGL(kernel, dim3((threads + 255) / 256), dim3(256), 0, s, total, fd, r, (int)cols, (const T *)x, ldx,
                         (T *)y, ldy, d);
    };
    if (total <= kFew) launch(dropout_kernel<T, 1>, total);
    else launch(dropout_kernel<T, PIECES>, (total + PIECES - 1) / PIECES);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(int dtype, int64_t rows, int64_t cols, const void *x, int64_t ldx, void *y, int64_t ldy,
                          const Drop &d, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(rows, cols, x, ldx, y, ldy, d, s)
                             : run<float>(rows, cols, x, ldx, y, ldy, d, s);
}

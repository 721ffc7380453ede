// Forward products and input gradients of few rows, or of few results in all,
// grouped by cluster (gfx950): serving a row or so of every cluster, where the
// time is that of reading the weights, and products with fewer 128 x 128 tiles
// than CUs.
//
// A workgroup gives 16 or 32 rows x some columns of the result.  Its four waves
// share the sum: each streams its quarter of the operands' rows from memory to
// registers, 16 bytes a lane and 16 to 20 loads at a time, at any alignment,
// and multiplies them with MFMAs (fp32: the fp32 MFMA), with no LDS; the four
// partial sums meet in LDS.
//
// Input gradient: a weight row runs across the sum.  A lane loads VEC rows of
// VEC columns (a 16-byte vector) and fragment j takes column j of every lane, so
// that lane i's column is VEC i + j; in bf16, pairs of rows are interleaved by a
// byte permute for each two elements.  A lane ends with VEC consecutive columns.
//
// Bound: few rows, by memory: 16 rows of 16 groups, 4096 -> 4096, bf16, 68 us
// (5.4 TB/s).  Otherwise by what a CU loads, about 36 bytes a ns.
#include "group.h"

#include <type_traits>

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int WAVES = 4;  // (eight or sixteen were no faster anywhere)

template <typename T> struct Few;
template <> struct Few<bf16_t> {
  static constexpr int VEC = 8, STEP = 32;  // k of a lane's vector, of a step of four lanes
  static __device__ __forceinline__ void mma(f32x4_t &acc, const u32x4 &w, const u32x4 &x) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, w), __builtin_bit_cast(bf16x8_t, x), acc, 0,
                                                  0, 0);
  }
};
template <> struct Few<float> {
  static constexpr int VEC = 4, STEP = 16;
  // product j takes element j of every lane's vector, of both operands alike
  static __device__ __forceinline__ void mma(f32x4_t &acc, const u32x4 &w, const u32x4 &x) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), __uint_as_float(x[j]), acc, 0, 0, 0);
  }
};

// The vector's elements moved n of them down, zeros above.
template <typename T> __device__ __forceinline__ u32x4 shift_down(u32x4 v, int n) {
  constexpr int VEC = Few<T>::VEC;
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = 0;
#pragma unroll
  for (int s = 0; s < VEC; ++s)  // (once a sum, by one wave)
    if (s == n) {
#pragma unroll
      for (int e = 0; e + s < VEC; ++e) {
        if constexpr (VEC == 4) r[e] = v[e + s];
        else r[e >> 1] |= ((v[(e + s) >> 1] >> (((e + s) & 1) * 16)) & 0xffffu) << ((e & 1) * 16);
      }
    }
  return r;
}

// One operand's vectors of a step (the sum's positions lg VEC .. + VEC - 1 for
// this lane), whose rows run along the sum: F rows 16 apart.
template <typename T, int F> struct Along {
  using W = Few<T>;
  const T *at[F];
  u32x4 v[F];
  // rows of stride ld from p on, `n` inside: those outside are taken as the last one
  __device__ __forceinline__ void init(const T *p, int64_t ld, int n, int li, int lg) {
#pragma unroll
    for (int f = 0; f < F; ++f) at[f] = p + (int64_t)min(16 * f + li, n - 1) * ld + lg * W::VEC;
  }
  __device__ __forceinline__ void load(int s) {
#pragma unroll
    for (int f = 0; f < F; ++f) v[f] = *(const u32x4_any *)(at[f] + (int64_t)s * W::STEP);
  }
  // what is left of Q after s steps: a vector past the end is the last whole one, shifted
  __device__ __forceinline__ void rest(int s, int Q, int lg) {
    const int over = max(s * W::STEP + (lg + 1) * W::VEC - Q, 0);
#pragma unroll
    for (int f = 0; f < F; ++f)
      v[f] = shift_down<T>(*(const u32x4_any *)(at[f] + (int64_t)s * W::STEP - over), min(over, W::VEC));
  }
  __device__ __forceinline__ u32x4 frag(int f) const { return v[f]; }
};

// One whose rows run across the sum: VEC rows of VEC columns, of which
// fragment j takes column j of every lane.
template <typename T> struct Across {
  using W = Few<T>;
  const T *at;
  int64_t ld;
  u32x4 v[W::VEC];
  // columns of p, `n` of them: a vector past the end is the last whole one
  __device__ __forceinline__ void init(const T *p, int64_t ld_, int n, int li, int lg) {
    ld = ld_;
    at = p + min(li * W::VEC, n - W::VEC) + lg * W::VEC * ld;
  }
  __device__ __forceinline__ void load(int s) {
#pragma unroll
    for (int i = 0; i < W::VEC; ++i) v[i] = *(const u32x4_any *)(at + ((int64_t)s * W::STEP + i) * ld);
  }
  __device__ __forceinline__ void rest(int s, int Q, int lg) {
#pragma unroll
    for (int i = 0; i < W::VEC; ++i) {
      const int q = s * W::STEP + lg * W::VEC + i, over = max(q - Q + 1, 0);
      v[i] = *(const u32x4_any *)(at + ((int64_t)s * W::STEP + i - over) * ld);
      if (over) v[i] = u32x4{0, 0, 0, 0};
    }
  }
  __device__ __forceinline__ u32x4 frag(int j) const {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if constexpr (sizeof(T) == 2)
        r[i] = __builtin_amdgcn_perm(v[2 * i + 1][j >> 1], v[2 * i][j >> 1], j & 1 ? 0x07060302u : 0x05040100u);
      else r[i] = v[i][j];
    return r;
  }
};

// 16 FR rows x 16 FC columns of the result (FC vectors' columns where the
// weights' rows run across the sum).
template <typename T, int MODE, int FR, int FC>
__global__ void __launch_bounds__(64 * WAVES) group_few_kernel(GroupArgs a, int NT) {
  using F = Few<T>;
  constexpr bool BT = MODE == GROUP_DX;
  constexpr int AHEAD = (BT ? 20 : 16) / (FR + FC);  // steps whose loads are in flight
  static_assert(!BT || FC == F::VEC, "");
  __shared__ f32x4_t part[WAVES / 2][FR * FC][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  int g, row0, row1, nt;
  if (!tile_of<false>(a.off, a.G, a.M, 16 * FR, NT, blockIdx.x, g, row0, row1, nt)) return;
  const int c0 = nt * 16 * FC, Q = a.Q;
  const T *w = (const T *)a.b + g * a.b_gs, *x = (const T *)a.a + (int64_t)row0 * a.lda;
  Along<T, FR> ax[AHEAD];
  std::conditional_t<BT, Across<T>, Along<T, FC>> bw[AHEAD];
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) {
    ax[i].init(x, a.lda, row1 - row0, li, lg);
    bw[i].init(w + (BT ? c0 : (int64_t)c0 * a.ldb), a.ldb, a.N - c0, li, lg);
  }
  f32x4_t acc[FR][FC];
#pragma unroll
  for (int f = 0; f < FR; ++f)
#pragma unroll
    for (int c = 0; c < FC; ++c) acc[f][c] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const auto multiply = [&](int i) {
#pragma unroll
    for (int c = 0; c < FC; ++c) {
      const u32x4 b = bw[i].frag(c);
#pragma unroll
      for (int f = 0; f < FR; ++f) F::mma(acc[f][c], b, ax[i].frag(f));
    }
  };
  const int steps = Q / F::STEP;  // whole ones
  const int s1 = (int)((int64_t)steps * (wave + 1) / WAVES);
  int s = (int)((int64_t)steps * wave / WAVES);
  for (; s + AHEAD <= s1; s += AHEAD) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      bw[i].load(s + i);
      ax[i].load(s + i);
    }
    __builtin_amdgcn_sched_barrier(0);  // (the loads stay together)
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) multiply(i);
  }
  for (; s < s1; ++s) {
    bw[0].load(s);
    ax[0].load(s);
    multiply(0);
  }
  if (wave == WAVES - 1 && steps * F::STEP < Q) {
    bw[0].rest(steps, Q, lg);
    ax[0].rest(steps, Q, lg);
    multiply(0);
  }

  // the waves' sums: those of the second half join those of the first
  const int place = wave % (WAVES / 2);
  if (wave >= WAVES / 2) {
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
      for (int c = 0; c < FC; ++c) part[place][f * FC + c][lane] = acc[f][c];
  }
  __syncthreads();
  if (wave < WAVES / 2) {
#pragma unroll
    for (int f = 0; f < FR; ++f)
#pragma unroll
      for (int c = 0; c < FC; ++c) part[place][f * FC + c][lane] += acc[f][c];
  }
  __syncthreads();
  // four columns of a row at a time: of fragment fc, or of index 4 lg + i of fragments j .. j + 3
  constexpr int QUADS = FR * FC * 64;
#pragma unroll
  for (int e = threadIdx.x; e < QUADS; e += 64 * WAVES) {
    const int f = e / (FC * 64), fc = e / 64 % FC, m = row0 + 16 * f + li;
    f32x4_t v = f32x4_t{0.f, 0.f, 0.f, 0.f};
    int c;
    if constexpr (BT) {
      const int i = fc & 3, first = c0 + (4 * lg + i) * F::VEC, over = max(first + F::VEC - a.N, 0);
      c = first + (fc & ~3);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int j = min((fc & ~3) + r + over, FC - 1);  // (more: outside)
#pragma unroll
        for (int p = 0; p < WAVES / 2; ++p) v[r] += part[p][f * FC + j][lane][i];
      }
    } else {
      c = c0 + 16 * fc + 4 * lg;
#pragma unroll
      for (int p = 0; p < WAVES / 2; ++p) v += part[p][f * FC + fc][lane];
    }
    if (m < row1 && c < a.N) finish<T, MODE>(a, g, m, c, v);
  }
}

template <typename T, int MODE, int FR, int FC> hipError_t run(const GroupArgs &a, hipStream_t s) {
  const int64_t NT = (a.N + 16 * FC - 1) / (16 * FC), blocks = tile_blocks(a.M, a.G, 16 * FR, NT);
  if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((group_few_kernel<T, MODE, FR, FC>), dim3((uint32_t)blocks), dim3(64 * WAVES), 0, s, a, (int)NT);
  return hipGetLastError();
}

// Workgroups if each has 32 rows and 32 columns (input gradient: 16 vectors'),
// a group's last one half full on average.
int64_t tiles32(int dtype, const GroupArgs &a, int mode) {
  const int cols = mode == GROUP_FWD ? 32 : dtype == GCPSL_BF16 ? 128 : 64;
  return ((int64_t)a.M + 16 * a.G) / 32 * ((a.N + cols - 1) / cols);
}

// Forward: at most four rows a group on average (or 16 in all), and few enough
// that all of them in one group would read its weights no more than 16 times.
bool few_rows(const GroupArgs &a) { return a.M <= std::max(16, std::min(4 * a.G, 256)); }

// The largest tile that leaves the chip enough workgroups: us for tiles of
// 16 x 16, 32 x 16 and 32 x 32, bf16, 1 group,
//   rows 128, 512 -> 512 (64 tiles of 32 x 32):     4.8   5.3   5.9
//   rows 32, 4096 -> 4096 (128):                   19.2  15.7  18.8
//   rows 128, 1024 -> 4096 (512):                  22.4  14.9  11.4
// input gradient, 16 and 32 rows: 32 rows, 4096 -> 4096 (32), 18.6 and 22.3;
// 8 groups, 1,024 rows, 1024 -> 1024 (256), 11.1 and 9.9.
template <typename T> hipError_t run(int dtype, int mode, const GroupArgs &a, hipStream_t s) {
  const int64_t tiles = tiles32(dtype, a, mode);
  if (mode == GROUP_DX)
    return tiles <= 128 ? run<T, GROUP_DX, 1, Few<T>::VEC>(a, s) : run<T, GROUP_DX, 2, Few<T>::VEC>(a, s);
  if (tiles <= 64 || few_rows(a)) return run<T, GROUP_FWD, 1, 1>(a, s);
  return tiles <= 128 ? run<T, GROUP_FWD, 2, 1>(a, s) : run<T, GROUP_FWD, 2, 2>(a, s);
}

}  // namespace

// A vector at least in the operands' rows, and few rows or so few tiles that
// the kernels of 64 x 64, 64 x 128 and 128 x 128 tiles, of which a CU has one or
// none, take longer than this one, whose time goes with the tiles.  us here and
// there:
//   forward, fp32   1 group, 64 rows, 4096 -> 4096 (256 tiles)       33    56
//                   1 group, 1,000 rows, 2000 -> 300 (310)           41    37
//                   1 group, 1,307 rows, 512 -> 640 (827)            23    13
//      short sums   6 groups, 4,000 rows, 128 -> 64 (254)            5.3   6.8
//   forward, bf16   5 groups, 433 rows, 4096 -> 1024 (513)           34    40
//                   1 group, 1,307 rows, 512 -> 640 (827)            11.1  9.7
//   (rows at odd    1 group, 25 rows, 2013 -> 71 (3)                 13    22
//    addresses)     33 groups, 1,236 rows, 1687 -> 396 (716)         51    29
//   input grad.,    5 groups, 433 rows, 1024 <- 4096 (256)           46    60
//      fp32         4 groups, 500 rows, 1024 <- 4096 (272)           106   57
//   input grad.,    5 groups, 433 rows, 4096 <- 1024 (128)           22    42
//      bf16         8 groups, 1,024 rows, 1024 <- 1024 (288)         14.8  15.2
bool group_few_ok(int dtype, const GroupArgs &a, int mode) {
  const bool bf16 = dtype == GCPSL_BF16;
  const int vec = bf16 ? 8 : 4;
  if (mode == GROUP_DW || a.Q < vec) return false;
  const int64_t tiles = tiles32(dtype, a, mode);
  if (mode == GROUP_DX) return a.N >= vec && tiles <= (bf16 ? 320 : a.Q < 256 || !group_f32_deep_ok(a, mode) ? 512 : 256);
  return few_rows(a) || tiles <= (!bf16 ? (a.Q < 256 ? 768 : 304) : (a.lda | a.ldb) & 1 ? 256 : 640);
}

hipError_t launch_group_few(int dtype, int mode, const GroupArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(dtype, mode, a, s) : run<float>(dtype, mode, a, s);
}

// Products over rows grouped by cluster, fp32 (gfx950), on the bf16 matrix
// cores: 128 x 128 outputs a workgroup, any alignment and size.
//
// The fp32 MFMA runs at 1/16 of the bf16 rate.  An fp32 value is instead
// written exactly as the sum of three bf16 values,
//
//   x = h + m + l,  h = bf16(x), m = bf16(x - h), l = x - h - m
//
// (each difference is exact, |m| <= 2^-8 |x|, |l| <= 2^-17 |x|), and a product
// x y is the six terms l h' + h l' + m m' + m h' + h m' + h h'; the three left
// out reach 2^-24 |x y| at worst, the fp32 rounding of one product.  An MFMA
// rounds its sum about once per 8 products: h h' has a sum of its own and the
// five small terms another, so that the large one is rounded 4 times per 32
// values, less often than in a chain of fp32 products.  (Values below 2^-110
// run out of bf16's exponents: absolute precision 2^-133.)
//
// A workgroup that meets a value of kHuge or more (an infinity has no such
// split, and terms of opposite sign could overflow where the sum does not)
// takes its tile again with fp32 MFMAs.  A NaN is one in every term.
//
// Staging: threads 0..127 take the A operand, 128..255 the B operand, 32 values
// each of a 32-deep k tile, loaded to registers one tile ahead, split and
// written as 16-byte pieces of 8 consecutive k.  Operands whose rows run
// across the sum are loaded as 8 rows x 4 columns a thread, so that the 8 k of
// a column meet in one thread.  One 48 KB buffer: two workgroups share a CU
// and one's staging overlaps the other's MFMAs.
#include "group.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int BM = 128, BN = 128, BK = 32;
constexpr int PLANE = 128 * 64;  // bytes of one bf16 part of an operand's tile: 128 rows of 32
constexpr float kHuge = 1.125899906842624e15f;  // 2^50: products below 2^100, and any sum of them finite

// 16-byte piece c (8 k) of row r in a plane; the XOR spreads the 8 rows of a
// fragment read, and (2-way) the rows of transposed writes, over the banks.
__device__ __forceinline__ int at(int r, int c) { return r * 64 + ((c ^ (((r >> 1) ^ (r >> 3)) & 3)) * 16); }

// Two values -> their three parts, packed.
__device__ __forceinline__ void split2(float a, float b, uint32_t (&p)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    p[i] = pack2_bf16(a, b);
    a -= __uint_as_float(p[i] << 16);
    b -= __uint_as_float(p[i] & 0xffff0000u);
  }
}

// One thread's share of an operand's k tiles.  T: the operand's rows run
// across the sum (k = row); else along it.
template <bool T> struct Stage {
  const float *p;  // T: row k0 + 8 chunk, column 4 quad; else row t / 4, k0 + 8 (t % 4)
  int64_t ld;
  int n, t;        // rows or columns inside, thread of 128
  float v[4][8];   // [row or column][k]

  __device__ __forceinline__ void init(const float *base, int64_t ld_, int n_, int t_) {
    ld = ld_; n = n_; t = t_;
    p = T ? base + (int64_t)(t >> 5) * 8 * ld + (t & 31) * 4 : base + (int64_t)(t >> 2) * ld + (t & 3) * 8;
  }
  // k tile at k0, `left` deep from there (all of it past the end gives zeros)
  __device__ __forceinline__ void load(int k0, int left) {
    if constexpr (T) {
      const int k = (t >> 5) * 8, c = (t & 31) * 4;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float *q = p + (int64_t)(k0 + i) * ld;
        f32x4_any x{0.f, 0.f, 0.f, 0.f};
        if (k + i < left) {
          if (c + 4 <= n) {
            x = *(const f32x4_any *)q;
          } else {
#pragma unroll
            for (int j = 0; j < 3; ++j)
              if (c + j < n) x[j] = q[j];
          }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j][i] = x[j];
      }
    } else {
      const int k = (t & 3) * 8;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float *q = p + (int64_t)j * 32 * ld + k0;
        f32x4_any x{0.f, 0.f, 0.f, 0.f}, y{0.f, 0.f, 0.f, 0.f};
        if ((t >> 2) + j * 32 < n) {
          if (k + 8 <= left) {
            x = *(const f32x4_any *)q;
            y = *(const f32x4_any *)(q + 4);
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (k + i < left) x[i] = q[i];
              if (k + 4 + i < left) y[i] = q[4 + i];
            }
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[j][i] = x[i];
          v[j][4 + i] = y[i];
        }
      }
    }
  }
  // splits the values and writes them; returns the largest magnitude so far
  __device__ __forceinline__ float write(char *planes, float top) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = T ? (t & 31) * 4 + j : (t >> 2) + j * 32, c = T ? t >> 5 : t & 3;
      u32x4 w[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t s[3];
        split2(v[j][2 * i], v[j][2 * i + 1], s);
        top = fmaxf(fmaxf(top, fabsf(v[j][2 * i])), fabsf(v[j][2 * i + 1]));
#pragma unroll
        for (int k = 0; k < 3; ++k) w[k][i] = s[k];
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) *(u32x4 *)(planes + k * PLANE + at(r, c)) = w[k];
    }
    return top;
  }
};

__device__ __forceinline__ f32x4_t mma(const u32x4 &a, const u32x4 &b, const f32x4_t &c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                 0, 0);
}

template <int MODE>
__global__ void __launch_bounds__(256, 2) group_f32_kernel(GroupArgs a, int NT) {
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;
  __shared__ __attribute__((aligned(16))) char lds[6 * PLANE];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, li = lane & 15, lg = lane >> 4;
  int g, row0, rows, c0, Q, split = 0, nt;
  const float *A = (const float *)a.a, *B = (const float *)a.b;
  if constexpr (MODE == GROUP_DW) {
    const uint32_t MT = (uint32_t)(a.M + BM - 1) / BM, tiles = MT * (uint32_t)NT, part = blockIdx.x / tiles;
    int mt, q0, q1;
    block_order(xcd_swizzle(blockIdx.x - part * tiles, tiles), MT, (uint32_t)NT, mt, nt);
    row0 = mt * BM;
    split = __builtin_amdgcn_readfirstlane((int)(part % (uint32_t)a.splits));
    g = __builtin_amdgcn_readfirstlane((int)(part / (uint32_t)a.splits));
    group_piece(a, g, split, q0, q1);
    Q = q1 - q0;
    rows = min(BM, a.M - row0);
    c0 = nt * BN;
    A += (int64_t)q0 * a.lda + row0;
    B += (int64_t)q0 * a.ldb + c0;
  } else {
    int mt, row1;
    if (!tile_of(a.off, a.G, a.M, BM, NT, blockIdx.x, mt, nt)) return;
    if (!find_tile(a.off, a.G, a.M, BM, mt, g, row0, row1)) return;
    rows = row1 - row0;
    c0 = nt * BN;
    Q = a.Q;
    A += (int64_t)row0 * a.lda;
    B += g * a.b_gs + (BT ? (int64_t)c0 : (int64_t)c0 * a.ldb);
  }
  const int cols = min(BN, a.N - c0);
  const bool sums = MODE == GROUP_DW && a.db != nullptr && nt == 0;

  // [column fragment][row fragment], a lane holds 4 consecutive columns of one
  // row: the sums of h h' and of the small terms
  f32x4_t big[4][4], small[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) big[i][j] = small[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float top = 0.f, colsum[4] = {0.f, 0.f, 0.f, 0.f};

  // the fragments' multiplication for one k tile
  const auto multiply = [&] {
    u32x4 x[4][3];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int k = 0; k < 3; ++k) x[j][k] = *(const u32x4 *)(lds + k * PLANE + at(wm * 64 + j * 16 + li, lg));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      u32x4 w[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) w[k] = *(const u32x4 *)(lds + (3 + k) * PLANE + at(wn * 64 + i * 16 + li, lg));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        small[i][j] = mma(w[2], x[j][0], small[i][j]);
        small[i][j] = mma(w[0], x[j][2], small[i][j]);
        small[i][j] = mma(w[1], x[j][1], small[i][j]);
        small[i][j] = mma(w[1], x[j][0], small[i][j]);
        small[i][j] = mma(w[0], x[j][1], small[i][j]);
        big[i][j] = mma(w[0], x[j][0], big[i][j]);
      }
    }
  };
  const auto run = [&](auto &stage, bool is_a) {
    stage.load(0, Q);
    for (int k0 = 0; k0 < Q; k0 += BK) {
      __syncthreads();
      top = stage.write(lds + (is_a ? 0 : 3 * PLANE), top);
      if constexpr (MODE == GROUP_DW) {
        if (sums && is_a) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) colsum[j] += stage.v[j][i];
        }
      }
      __syncthreads();
      stage.load(k0 + BK, Q - k0 - BK);
      multiply();
    }
  };
  if constexpr (AT == BT) {
    Stage<AT> stage;
    if (wave < 2) stage.init(A, a.lda, rows, tid);
    else stage.init(B, a.ldb, cols, tid - 128);
    run(stage, wave < 2);
  } else if (wave < 2) {
    Stage<AT> stage;
    stage.init(A, a.lda, rows, tid);
    run(stage, true);
  } else {
    Stage<BT> stage;
    stage.init(B, a.ldb, cols, tid - 128);
    run(stage, false);
  }

  if (__syncthreads_or(top >= kHuge)) {
    // again in fp32, from memory: lane (li, lg) takes k = 4 s + lg of step s
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) big[i][j] = small[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < Q; k0 += 4) {
      const int k = k0 + lg;
      float x[4], w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = wm * 64 + j * 16 + li, c = wn * 64 + j * 16 + li;
        x[j] = r < rows && k < Q ? (AT ? A[(int64_t)k * a.lda + r] : A[(int64_t)r * a.lda + k]) : 0.f;
        w[j] = c < cols && k < Q ? (BT ? B[(int64_t)k * a.ldb + c] : B[(int64_t)c * a.ldb + k]) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) big[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[j], big[i][j], 0, 0, 0);
    }
  }

#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = wm * 64 + j * 16 + li;
    if (m >= rows) continue;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + wn * 64 + i * 16 + 4 * lg;
      if (c >= a.N) continue;
      const f32x4_t v = big[i][j] + small[i][j];
      if constexpr (MODE == GROUP_DW) store_grad(a, g, split, row0 + m, c, v);
      else finish<float, MODE>(a, g, row0 + m, c, v);
    }
  }
  if constexpr (MODE == GROUP_DW) {
    if (sums) {  // each column's four shares, of 8 of every 32 rows
      float *part = (float *)lds;
      __syncthreads();
      if (tid < 128)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[(tid >> 5) * 128 + (tid & 31) * 4 + j] = colsum[j];
      __syncthreads();
      if (tid < rows)
        store_bias_grad(a, g, split, row0 + tid, (part[tid] + part[128 + tid]) + (part[256 + tid] + part[384 + tid]));
    }
  }
}

template <int MODE> hipError_t run_mode(const GroupArgs &a, hipStream_t s) {
  const int64_t NT = (a.N + BN - 1) / BN;
  const int64_t blocks = MODE == GROUP_DW ? (int64_t)((a.M + BM - 1) / BM) * NT * a.splits * a.G
                                          : ((int64_t)a.M / BM + std::min(a.G, a.M)) * NT;
  if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(group_f32_kernel<MODE>, dim3((uint32_t)blocks), dim3(256), 0, s, a, (int)NT);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_group_f32(int mode, const GroupArgs &a, hipStream_t s) {
  return mode == GROUP_FWD ? run_mode<GROUP_FWD>(a, s)
                           : mode == GROUP_DX ? run_mode<GROUP_DX>(a, s) : run_mode<GROUP_DW>(a, s);
}

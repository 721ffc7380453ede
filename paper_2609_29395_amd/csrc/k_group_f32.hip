// Products over rows grouped by cluster, fp32 (gfx950), on the bf16 matrix
// cores: 128 x 128 outputs a workgroup, any alignment and size.
//
// How fp32 values are multiplied there: group_f32.h.
//
// Staging: threads 0..127 take the A operand, 128..255 the B operand, 16 values
// each of a 16-deep k tile, loaded to registers two tiles ahead, split and
// written to LDS one tile ahead as 16-byte pieces of 8 consecutive k; a tile
// costs one barrier.  Operands whose rows run across the sum are loaded as 8
// rows x 2 columns a thread, so that the 8 k of a column meet in one thread.
// Two 24 KB buffers; two workgroups share a CU and one's splitting overlaps the
// other's MFMAs.
//
// Bound: what a k tile costs beside its MFMAs, which the matrix cores are busy
// with 32 to 35 % of a launch: every value is split by each tile that reads it,
// and every 16 of the sum take fragment reads and a barrier.  8 groups of 1,024
// rows, 1024 -> 1024: forward 96 to 100 us (171 to 179 TFLOP/s, 42 % of what six
// bf16 products allow; fp32 MFMAs have a peak of 157), input gradient 97, weight
// gradient 105.  A workgroup alone on its CU takes 0.6 us a k tile where its
// MFMAs take 0.35.
#include "group_f32.h"

namespace {

constexpr int BM = 128, BN = 128, BK = 16;
constexpr int PLANE = 128 * 32;  // bytes of one bf16 part of an operand's tile: 128 rows of 16
constexpr int BUFFER = 6 * PLANE;

// 16-byte piece c (8 k) of row r in a plane; the XOR puts the 8 rows of a
// fragment read on all banks.
__device__ __forceinline__ int at(int r, int c) { return r * 32 + ((c ^ ((r >> 3) & 1)) * 16); }

// One thread's share of an operand's k tiles.  T: the operand's rows run
// across the sum (k = row): rows 8 chunk .. + 7 of a tile, two columns; else
// along it: rows t / 2 and (ROWS 2) t / 2 + 64, k = 8 (t % 2) .. + 7 of a tile.  Rows and
// columns past the n inside are taken as the last ones inside (what they give
// is not stored), so that loads need no test: a thread whose columns pass the
// end takes the last two instead.
template <bool T, int ROWS = 2> struct Stage {
  const char *base;  // of the next tile
  int64_t step;
  int row, chunk;                // first row (T: column) in LDS, 16-byte piece
  static constexpr int J = T ? 2 : ROWS;
  uint32_t off[T ? 1 : 2], ld;   // byte offsets of the thread's loads, bytes of a row
  float v[J][8];                 // [row or column][k]

  __device__ __forceinline__ void init(const float *p, int64_t ld_, int n, int t) {
    base = (const char *)p;
    ld = (uint32_t)ld_ * 4u;
    step = T ? ld_ * (4 * BK) : 4 * BK;
    if constexpr (T) {
      chunk = t >> 6;
      row = min((t & 63) * 2, n - 2);  // -1 in a tile of one column, which is not the first
      base -= 4;                       // offsets are not negative
      off[0] = (uint32_t)chunk * 8u * ld + (uint32_t)(row + 1) * 4u;
    } else {
      chunk = t & 1;
      row = t >> 1;
#pragma unroll
      for (int j = 0; j < 2; ++j) off[j] = (uint32_t)min(row + j * 64, n - 1) * ld + (uint32_t)chunk * 32u;
    }
  }
  // the next tile, all of it inside
  __device__ __forceinline__ void load_all() {
    if constexpr (T) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const f32x2_any x = *(const f32x2_any *)(base + (off[0] + (uint32_t)i * ld));
        v[0][i] = x[0];
        v[1][i] = x[1];
      }
    } else {
#pragma unroll
      for (int j = 0; j < J; ++j) {
        const f32x4_any x = *(const f32x4_any *)(base + off[j]), y = *(const f32x4_any *)(base + (off[j] + 16u));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[j][i] = x[i];
          v[j][4 + i] = y[i];
        }
      }
    }
    base += step;
  }
  // the same with `left` values of k inside
  __device__ __forceinline__ void load(int left) {
    if (left >= BK) {
      load_all();
    } else if (left > 0) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = min(chunk * 8 + i, left - 1), d = k - chunk * 8;  // a k inside
        const bool in = d == i;
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const int64_t o = T ? (int64_t)off[0] + (int64_t)d * ld + j * 4 : (int64_t)off[T ? 0 : j] + d * 4;
          const float x = *(const float *)(base + o);
          v[j][i] = in ? x : 0.f;
        }
      }
    }
  }
  // splits the values and writes them; returns the largest magnitude so far
  __device__ __forceinline__ float write(char *planes, float top) const {
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int r = T ? (row + j) & 127 : row + j * 64;  // (a negative row's place holds nothing of the tile)
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
      for (int k = 0; k < 3; ++k) *(u32x4 *)(planes + k * PLANE + at(r, chunk)) = w[k];
    }
    return top;
  }
};

// Where a workgroup's tile is: A and B from its first row, column and k on.
struct Tile {
  const float *A, *B;
  int g, row0, rows, c0, cols, Q, slot;
  bool sums;  // of A's columns, too (the bias gradient)
};

// The tile's sums and results; waves of 32 FJ x 64 outputs.
template <int MODE, int FJ>
__device__ __forceinline__ void group_f32_tile(const GroupArgs &a, const Tile &t, char *lds) {
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, li = lane & 31, lg = lane >> 5;
  const float *const A = t.A, *const B = t.B;
  const int g = t.g, row0 = t.row0, rows = t.rows, c0 = t.c0, cols = t.cols, Q = t.Q, slot = t.slot;
  const bool sums = t.sums;

  // [column fragment][row fragment] of 32 x 32: the sums of h h' and of the
  // small terms.  A lane holds, in four groups of four, columns 8 i + 4 lg ..
  // + 3 of row li.
  f32x16_t big[2][FJ], small[2][FJ];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < FJ; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) big[i][j][r] = small[i][j][r] = 0.f;
  float top = 0.f, colsum[2] = {0.f, 0.f};

  const auto run = [&](auto &stage, bool is_a) {
    char *const mine = lds + (is_a ? 0 : 3 * PLANE);
    const auto write = [&](int p) {  // to buffer p
      top = stage.write(mine + p * BUFFER, top);
      if constexpr (MODE == GROUP_DW) {
        if (sums && is_a) {
#pragma unroll
          for (int j = 0; j < 2; ++j) colsum[j] += sum8(stage.v[j]);
        }
      }
    };
    // k tile k0 of buffer p, the next one to LDS and the one after it to
    // registers; `all` says that the latter is inside as a whole (the loop of
    // such tiles has no branch, at whose end a load would be waited for)
    const auto tile = [&](int k0, int p, auto all) {
      u32x4 x[FJ][3], w[2][3];
      const char *now = lds + p * BUFFER;
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if (j < FJ) x[j][k] = *(const u32x4 *)(now + k * PLANE + at(wm * 32 * FJ + j * 32 + li, lg));
          w[j][k] = *(const u32x4 *)(now + (3 + k) * PLANE + at(wn * 64 + j * 32 + li, lg));
        }
      if constexpr (decltype(all)::value) {
        write(1 - p);
        stage.load_all();
      } else if (Q - k0 > BK) {
        write(1 - p);
        stage.load(Q - k0 - 2 * BK);
      }
      // term by term, so that a sum's next product is four MFMAs away
      constexpr int kw[6] = {2, 0, 1, 1, 0, 0}, kx[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
      for (int k = 0; k < 6; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < FJ; ++j) {
            if (k < 5) small[i][j] = mma(w[i][kw[k]], x[j][kx[k]], small[i][j]);
            else big[i][j] = mma(w[i][kw[k]], x[j][kx[k]], big[i][j]);
          }
      __syncthreads();
    };
    stage.load(Q);
    if (Q > 0) write(0);
    stage.load(Q - BK);
    __syncthreads();
    int k0 = 0, p = 0;
    for (; k0 + 3 * BK <= Q; k0 += BK, p ^= 1) tile(k0, p, std::true_type{});
    for (; k0 < Q; k0 += BK, p ^= 1) tile(k0, p, std::false_type{});
  };
  if constexpr (AT == BT) {
    Stage<AT> stage;
    if (wave < 2) stage.init(A, a.lda, rows, tid);
    else stage.init(B, a.ldb, cols, tid - 128);
    run(stage, wave < 2);
  } else if (wave < 2) {
    Stage<AT, FJ> stage;
    stage.init(A, a.lda, rows, tid);
    run(stage, true);
  } else {
    Stage<BT> stage;
    stage.init(B, a.ldb, cols, tid - 128);
    run(stage, false);
  }

  if (__syncthreads_or(top >= kHuge)) {
    // again in fp32, from memory: lane (li, lg) takes k = 2 s + lg of step s
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) big[i][j][r] = small[i][j][r] = 0.f;
    for (int k0 = 0; k0 < Q; k0 += 2) {
      const int k = k0 + lg;
      float x[FJ], w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int r = wm * 32 * FJ + j * 32 + li, c = wn * 64 + j * 32 + li;
        if (j < FJ) x[j] = r < rows && k < Q ? (AT ? A[(int64_t)k * a.lda + r] : A[(int64_t)r * a.lda + k]) : 0.f;
        w[j] = c < cols && k < Q ? (BT ? B[(int64_t)k * a.ldb + c] : B[(int64_t)c * a.ldb + k]) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < FJ; ++j) big[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(w[i], x[j], big[i][j], 0, 0, 0);
    }
  }

  // The results go through LDS, the rows of two waves (32 FJ of 512 bytes) at a
  // time, so that whole rows of the tile are written at once.
  const auto place = [&](int r, int c) { return lds + r * 512 + ((c >> 2) ^ ((r & 15) << 1)) * 16; };
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int m0 = h * 32 * FJ, r0 = tid >> 5, c4 = (tid & 31) * 4;
    if (m0 >= rows) break;
    const FinishRows<float, MODE == GROUP_DW ? GROUP_FWD : MODE, 4 * FJ> out(a, g, row0 + m0 + r0, 8, row0 + rows, c0 + c4);
    __syncthreads();
    if (wm == h)
#pragma unroll
      for (int j = 0; j < FJ; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            f32x4_t v;
#pragma unroll
            for (int r = 0; r < 4; ++r) v[r] = big[i][j][4 * q + r] + small[i][j][4 * q + r];
            *(f32x4_t *)place(j * 32 + li, wn * 64 + i * 32 + 8 * q + 4 * lg) = v;
          }
    __syncthreads();
    const auto sum = [&](int i, int) { return *(const f32x4_t *)place(r0 + 8 * i, c4); };
    if constexpr (MODE == GROUP_DW) {
      if (c0 + c4 < a.N)
        for (int i = 0; i < 4 * FJ && m0 + r0 + 8 * i < rows; ++i)
          store_grad(a, g, slot, row0 + m0 + r0 + 8 * i, c0 + c4, sum(i, 0));
    } else {
      out.store(a, sum);
    }
  }
  if constexpr (MODE == GROUP_DW) {
    if (sums) {  // each column's two shares, of 8 of every 16 rows
      float *part = (float *)lds;
      __syncthreads();
      if (tid < 128)
#pragma unroll
        for (int j = 0; j < 2; ++j) part[(tid >> 6) * 128 + ((min((tid & 63) * 2, rows - 2) + j) & 127)] = colsum[j];
      __syncthreads();
      if (tid < rows) store_bias_grad(a, g, slot, row0 + tid, part[tid] + part[128 + tid]);
    }
  }
}

template <int MODE>
__global__ void __launch_bounds__(256, 2) group_f32_kernel(GroupArgs a, int NT) {
  constexpr bool BT = MODE != GROUP_FWD;
  __shared__ __attribute__((aligned(16))) char lds[2 * BUFFER];
  Tile t{(const float *)a.a, (const float *)a.b, 0, 0, 0, 0, 0, a.Q, -1, false};
  int nt;
  if constexpr (MODE == GROUP_DW) {
    const uint32_t MT = (uint32_t)(a.M + BM - 1) / BM;
    uint32_t tile;
    int mt, q0, q1;
    if (!piece_of(a, MT * (uint32_t)NT, blockIdx.x, t.g, q0, q1, t.slot, tile)) return;
    block_order(tile, MT, (uint32_t)NT, mt, nt);
    t.row0 = mt * BM;
    t.Q = q1 - q0;
    t.rows = min(BM, a.M - t.row0);
    t.c0 = nt * BN;
    t.A += (int64_t)q0 * a.lda + t.row0;
    t.B += (int64_t)q0 * a.ldb + t.c0;
  } else {
    int row1;
    if (!tile_of(a.off, a.G, a.M, BM, NT, blockIdx.x, t.g, t.row0, row1, nt)) return;
    t.rows = row1 - t.row0;
    t.c0 = nt * BN;
    t.A += (int64_t)t.row0 * a.lda;
    t.B += t.g * a.b_gs + (BT ? (int64_t)t.c0 : (int64_t)t.c0 * a.ldb);
  }
  t.cols = min(BN, a.N - t.c0);
  t.sums = MODE == GROUP_DW && a.db != nullptr && nt == 0;
  if (MODE != GROUP_DW && t.rows <= BM / 2) group_f32_tile<MODE, 1>(a, t, lds);
  else group_f32_tile<MODE, 2>(a, t, lds);
}

template <int MODE> hipError_t run_mode(const GroupArgs &a, hipStream_t s) {
  const int64_t NT = (a.N + BN - 1) / BN;
  const int64_t blocks = MODE == GROUP_DW ? piece_blocks(a, (int64_t)((a.M + BM - 1) / BM) * NT)
                                          : tile_blocks(a.M, a.G, BM, NT);
  if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(group_f32_kernel<MODE>, dim3((uint32_t)blocks), dim3(256), 0, s, a, (int)NT);
  return hipGetLastError();
}

}  // namespace

// Two columns at least wherever the operands' rows run across the sum, and
// row strides whose offsets within a tile fit 32 bits.
bool group_f32_ok(const GroupArgs &a, int mode) {
  return a.lda <= kMaxTileLd && a.ldb <= kMaxTileLd && (mode == GROUP_FWD || a.N >= 2) && (mode != GROUP_DW || a.M >= 2);
}

hipError_t launch_group_f32(int mode, const GroupArgs &a, hipStream_t s) {
  return mode == GROUP_FWD ? run_mode<GROUP_FWD>(a, s)
                           : mode == GROUP_DX ? run_mode<GROUP_DX>(a, s) : run_mode<GROUP_DW>(a, s);
}

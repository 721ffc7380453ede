// Products over rows grouped by cluster, fp32 (gfx950), where 128 x 128 tiles
// are fewer than CUs: 64 x 64 outputs a workgroup, on the bf16 matrix cores
// (group_f32.h).
//
// Two teams of four waves share the sum: of the k tiles, 32 deep, one takes the
// even ones and the other the odd ones, each with two LDS buffers of its own,
// so that on every SIMD one team's splitting of values runs beside the other's
// MFMAs.  A thread stages 16 values of a k tile, loaded to registers three of
// its team's tiles ahead and written to LDS, split, one ahead; a step costs one
// barrier.  The teams' sums meet in LDS.
//
// A k tile's small terms go to two sums in turn, as a wave has only one 32 x 32
// fragment and an MFMA that waits for the one before it loses half its time.
//
// Bound: by a step's length, about 1.1 us for 64 of the sum, in which the MFMAs
// take 0.37 of every SIMD: each wave reads fragments, splits, multiplies and
// waits at the barrier.  (One team multiplying while the other splits, by the
// order of the two in their code, took 15 % longer: the compiler interleaves
// them within a wave.)  1 group of 1,000 rows, 4096 -> 1024, 256 tiles: forward
// 70 us (120 TFLOP/s), where 128 x 128 tiles took 137; input gradient of as
// many tiles 70.
#include "group_f32.h"

namespace {

constexpr int BM = 64, BN = 64, BK = 32;
constexpr int PLANE = 64 * BK * 2;  // bytes of one bf16 part of an operand's tile: 64 rows of 32
constexpr int BUFFER = 6 * PLANE;
constexpr int LDS_BYTES = 4 * BUFFER;  // two for each team
constexpr int SUMS = BM * BN * 4;      // bytes of a team's sums
static_assert(2 * SUMS + 8 * BM * 4 <= LDS_BYTES, "the teams' sums");

// 16-byte piece c (8 k) of row r in a plane; the XOR puts the 16 rows that a
// fragment read takes at a time on all banks.
__device__ __forceinline__ int at(int r, int c) { return r * 64 + ((c ^ ((r >> 2) & 3)) * 16); }

// One thread's share of its team's k tiles, for 128 threads an operand.  T: the
// operand's rows run across the sum (k = row): rows 8 chunk .. + 7 of a tile,
// two columns; else along it: row t / 2, k = 16 (t % 2) .. + 15.  Rows and
// columns past the n inside are taken as the last ones inside (what they give
// is not stored).
template <bool T> struct Stage {
  const char *base;  // of the team's next tile
  int64_t step;
  int row, chunk;    // row (T: first column) and first 16-byte piece in LDS
  uint32_t off, ld;  // byte offset of the thread's first load, bytes of a row
  float v[2][2][8];  // [set][T: column, else piece][k]

  __device__ __forceinline__ void init(const float *p, int64_t ld_, int n, int t, int first) {
    ld = (uint32_t)ld_ * 4u;
    base = (const char *)p + (T ? ld_ * first : first) * 4;
    step = (T ? ld_ : 1) * (2 * BK * 4);
    if constexpr (T) {
      chunk = t >> 5;
      row = min((t & 31) * 2, n - 2);  // -1 in a tile of one column, which is not the first
      base -= 4;                       // offsets are not negative
      off = (uint32_t)chunk * 8u * ld + (uint32_t)(row + 1) * 4u;
    } else {
      chunk = (t & 1) * 2;
      row = t >> 1;
      off = (uint32_t)min(row, n - 1) * ld + (uint32_t)chunk * 32u;
    }
  }
  // the next tile, all of it inside
  __device__ __forceinline__ void load_all(int set) {
    if constexpr (T) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const f32x2_any x = *(const f32x2_any *)(base + (off + (uint32_t)i * ld));
        v[set][0][i] = x[0];
        v[set][1][i] = x[1];
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4_any x = *(const f32x4_any *)(base + (off + (uint32_t)i * 16u));
#pragma unroll
        for (int r = 0; r < 4; ++r) v[set][i >> 1][(i & 1) * 4 + r] = x[r];
      }
    }
    base += step;
  }
  // the same with `left` values of k inside, zeros behind them
  __device__ __forceinline__ void load(int left, int set) {
    if (left >= BK) return load_all(set);
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int k = (chunk + (T ? 0 : j)) * 8 + i, in = min(k, left - 1) - chunk * 8;
        float x = 0.f;
        if (left > 0) x = *(const float *)(base + (T ? (int64_t)off + (int64_t)in * ld + j * 4 : (int64_t)off + in * 4));
        v[set][j][i] = k < left ? x : 0.f;
      }
  }
  // T: the sums of the thread's two columns in a set
  __device__ __forceinline__ void sum(int set, float (&s)[2]) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) s[j] += sum8(v[set][j]);
  }
  // splits the values and writes them; returns the largest magnitude so far
  __device__ __forceinline__ float write(char *planes, int set, float top) const {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int r = T ? (row + j) & 63 : row;  // (a negative row's place holds nothing of the tile)
      u32x4 w[3];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t s[3];
        split2(v[set][j][2 * i], v[set][j][2 * i + 1], s);
        top = fmaxf(fmaxf(top, fabsf(v[set][j][2 * i])), fabsf(v[set][j][2 * i + 1]));
#pragma unroll
        for (int k = 0; k < 3; ++k) w[k][i] = s[k];
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) *(u32x4 *)(planes + k * PLANE + at(r, chunk + (T ? 0 : j))) = w[k];
    }
    return top;
  }
};

template <int MODE>
__global__ void __launch_bounds__(512, 2) group_f32_deep_kernel(GroupArgs a, int NT) {
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;
  extern __shared__ __attribute__((aligned(1024))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, t = tid & 255;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int team = wave >> 2, wm = wave >> 1 & 1, wn = wave & 1, li = lane & 31, lg = lane >> 5;
  int g, row0, row1, nt, Q = a.Q, slot = -1;
  const float *A = (const float *)a.a, *B = (const float *)a.b;
  if constexpr (MODE == GROUP_DW) {
    const uint32_t MT = (uint32_t)(a.M + BM - 1) / BM;
    uint32_t tile;
    int mt, q0, q1;
    if (!piece_of(a, MT * (uint32_t)NT, blockIdx.x, g, q0, q1, slot, tile)) return;
    block_order(tile, MT, (uint32_t)NT, mt, nt);
    row0 = mt * BM;
    row1 = min(a.M, row0 + BM);
    Q = q1 - q0;
    A += (int64_t)q0 * a.lda + row0;
    B += (int64_t)q0 * a.ldb + nt * BN;
  } else {
    if (!tile_of<false>(a.off, a.G, a.M, BM, NT, blockIdx.x, g, row0, row1, nt)) return;
    A += (int64_t)row0 * a.lda;
    B += g * a.b_gs + (BT ? (int64_t)nt * BN : (int64_t)nt * BN * a.ldb);
  }
  const int rows = row1 - row0, c0 = nt * BN, cols = min(BN, a.N - c0);
  const bool sums = MODE == GROUP_DW && a.db != nullptr && nt == 0;  // of A's columns, too (the bias gradient)
  float colsum[2] = {0.f, 0.f};

  f32x16_t big, small[2];
#pragma unroll
  for (int r = 0; r < 16; ++r) big[r] = small[0][r] = small[1][r] = 0.f;
  float top = 0.f;
  const int steps = (Q + 2 * BK - 1) / (2 * BK);  // of each team; the odd one's last tile may be all zeros

  const auto run = [&](auto &stage, bool is_a) {
    char *const mine = lds + team * 2 * BUFFER, *const part = mine + (is_a ? 0 : 3 * PLANE);
    const auto write = [&](int to) {  // from the set of the same number
      top = stage.write(part + to * BUFFER, to, top);
      if constexpr (MODE == GROUP_DW) {
        if (sums && is_a) stage.sum(to, colsum);
      }
    };
    const auto left = [&](int i) { return Q - (2 * i + team) * BK; };
    // the team's k tile i of buffer p, the next one to LDS and the one two after
    // that to the registers this frees; `all` says that the latter is inside as a
    // whole
    const auto step = [&](int i, int p, auto all) {
      const char *now = mine + p * BUFFER;
      u32x4 x[2][3], w[2][3];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          x[h][k] = *(const u32x4 *)(now + k * PLANE + at(wm * 32 + li, 2 * h + lg));
          w[h][k] = *(const u32x4 *)(now + (3 + k) * PLANE + at(wn * 32 + li, 2 * h + lg));
        }
      if constexpr (decltype(all)::value) {
        write(1 - p);
        stage.load_all(1 - p);
      } else if (i + 1 < steps) {
        write(1 - p);
        if (i + 3 < steps) stage.load(left(i + 3), 1 - p);
      }
      constexpr int kw[6] = {2, 0, 1, 1, 0, 0}, kx[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int k = 0; k < 6; ++k) {
          if (k < 5) small[k & 1] = mma(w[h][kw[k]], x[h][kx[k]], small[k & 1]);
          else big = mma(w[h][kw[k]], x[h][kx[k]], big);
        }
      if constexpr (decltype(all)::value) {  // the fragments' reads, then splitting between the MFMAs
        __builtin_amdgcn_sched_group_barrier(0x100, 12, 0);
#pragma unroll
        for (int k = 0; k < 12; ++k) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 9, 0);
        }
      }
      __syncthreads();
    };
    stage.load(left(0), 0);
    if (steps > 1) stage.load(left(1), 1);
    write(0);
    if (steps > 2) stage.load(left(2), 0);
    __syncthreads();
    int i = 0;
    for (; (2 * i + 10) * BK <= Q; i += 2) {
      step(i, 0, std::true_type{});
      step(i + 1, 1, std::true_type{});
    }
    for (; i < steps; i += 2) {
      step(i, 0, std::false_type{});
      if (i + 1 < steps) step(i + 1, 1, std::false_type{});
    }
  };
  const bool is_a = (wave & 2) == 0;
  if constexpr (AT == BT) {
    Stage<AT> stage;
    if (is_a) stage.init(A, a.lda, rows, t, team * BK);
    else stage.init(B, a.ldb, cols, t - 128, team * BK);
    run(stage, is_a);
  } else if (is_a) {
    Stage<false> stage;
    stage.init(A, a.lda, rows, t, team * BK);
    run(stage, true);
  } else {
    Stage<true> stage;
    stage.init(B, a.ldb, cols, t - 128, team * BK);
    run(stage, false);
  }

  if (__syncthreads_or(top >= kHuge)) {
    // again in fp32, from memory, in pairs of k that the teams take in turn:
    // lane (li, lg) takes k = k0 + lg
#pragma unroll
    for (int r = 0; r < 16; ++r) big[r] = small[0][r] = small[1][r] = 0.f;
    const int m = wm * 32 + li, c = wn * 32 + li;
    for (int k0 = 2 * team; k0 < Q; k0 += 4) {
      const int k = k0 + lg;
      const float x = m < rows && k < Q ? (AT ? A[(int64_t)k * a.lda + m] : A[(int64_t)m * a.lda + k]) : 0.f;
      const float w = c < cols && k < Q ? (BT ? B[(int64_t)k * a.ldb + c] : B[(int64_t)c * a.ldb + k]) : 0.f;
      big = __builtin_amdgcn_mfma_f32_32x32x2f32(w, x, big, 0, 0, 0);
    }
  }

  // The teams' sums, and whole rows of the tile written at once.  A lane holds,
  // in four groups of four, columns 8 q + 4 lg .. + 3 of row li.
  const auto place = [&](int which, int r, int c) { return lds + which * SUMS + r * 256 + ((c >> 2) ^ (r & 15)) * 16; };
  const int r0 = tid >> 4, c4 = (tid & 15) * 4;
  const FinishRows<float, MODE == GROUP_DW ? GROUP_FWD : MODE, 2> out(a, g, row0 + r0, 32, row1, c0 + c4);
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    f32x4_t v;
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = big[4 * q + r] + (small[0][4 * q + r] + small[1][4 * q + r]);
    *(f32x4_t *)place(team, wm * 32 + li, wn * 32 + 8 * q + 4 * lg) = v;
  }
  // each column's shares: two teams, four pieces of 8 of their k tiles' 32
  float *const shares = (float *)(lds + 2 * SUMS);
  if (sums && is_a)
#pragma unroll
    for (int j = 0; j < 2; ++j) shares[(team * 4 + (t >> 5)) * 64 + ((min((t & 31) * 2, rows - 2) + j) & 63)] = colsum[j];
  __syncthreads();
  const auto sum = [&](int i, int) {
    return *(const f32x4_t *)place(0, r0 + 32 * i, c4) + *(const f32x4_t *)place(1, r0 + 32 * i, c4);
  };
  if constexpr (MODE == GROUP_DW) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (r0 + 32 * i < rows && c0 + c4 < a.N) store_grad(a, g, slot, row0 + r0 + 32 * i, c0 + c4, sum(i, 0));
    if (sums && tid < rows) {
      float v = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) v += shares[i * 64 + tid];
      store_bias_grad(a, g, slot, row0 + tid, v);
    }
  } else {
    out.store(a, sum);
  }
}

template <int MODE> hipError_t run_mode(const GroupArgs &a, hipStream_t s) {
  static PerDeviceOnce once;
  if (once.needed()) {
    const hipError_t e = hipFuncSetAttribute((const void *)group_f32_deep_kernel<MODE>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);
    if (e != hipSuccess) return e;
    once.mark();
  }
  const int64_t NT = (a.N + BN - 1) / BN;
  const int64_t blocks = MODE == GROUP_DW ? piece_blocks(a, (int64_t)((a.M + BM - 1) / BM) * NT)
                                          : tile_blocks(a.M, a.G, BM, NT);
  if (blocks > kMaxBlocks / 2) return hipErrorInvalidConfiguration;  // (of 512 threads)
  hipLaunchKernelGGL(group_f32_deep_kernel<MODE>, dim3((uint32_t)blocks), dim3(512), LDS_BYTES, s, a, (int)NT);
  return hipGetLastError();
}

}  // namespace

// At most one tile a CU (a CU holds one workgroup), a group's last tile half
// full on average.  us so and with the kernel taken otherwise: forward, 1 group
// of 200 rows, 4096 -> 4096 (192 tiles), 71 and 164; 1 of 1,307, 512 -> 640
// (200), 13 and 23; input gradient, 4 of 500, 1024 <- 4096 (144), 57 and 106;
// with more, 16 of 3,000 rows, 600 -> 600 (540), 45 and 37.
bool group_f32_deep_ok(const GroupArgs &a, int mode) {
  if (a.N < 32 || !group_f32_ok(a, mode)) return false;
  if (mode == GROUP_DW) return group_f32_deep_grad(a.G, a.Q, a.M, a.N);
  return ((int64_t)a.M + 32 * a.G) / 64 * ((a.N + BN - 1) / BN) <= kCUs;
}

hipError_t launch_group_f32_deep(int mode, const GroupArgs &a, hipStream_t s) {
  return mode == GROUP_FWD ? run_mode<GROUP_FWD>(a, s)
                           : mode == GROUP_DX ? run_mode<GROUP_DX>(a, s) : run_mode<GROUP_DW>(a, s);
}

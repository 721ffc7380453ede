// Products over rows grouped by cluster, bf16, on gfx950: 128 x 128 outputs a
// workgroup (64 x 128 in small launches), any alignment and size from 8 on, and
// the launches too small for tiles of 256 x 256.
//
// A k tile is 64 deep and goes through registers, loaded as 16-byte pieces at
// any alignment, to LDS as it lies in memory: an operand whose rows run along
// the sum as 128 rows of 128 bytes, one whose rows run across it as 64 rows of
// 256 bytes, from which ds_read_b64_tr_b16 makes fragments.  16-byte pieces are
// XOR-swizzled within a row so that a fragment read uses every bank.  Two
// buffers, one barrier a tile: tile t is multiplied while t + 1 is written to
// the other buffer and t + 2 (64 rows: and t + 3) loaded to registers.
//
// A piece that passes the end of the rows (the last k tile) or of the columns
// is the row's last 8 elements shifted into place, so that nothing outside the
// operand is read and what lies behind k is zero.
//
// Bound: the loads' time, which one k tile's MFMAs (0.25 us) do not cover: a
// workgroup alone on its CU takes 0.7 us a k tile, two share one better.  8
// groups of 512 rows, 1024 -> 1024: forward 22 us (383 TFLOP/s), input gradient
// 20 (442); 17,450 rows of 2 groups, 551 -> 1293 (rows at odd addresses): 67, 62
// and 87 us (369, 399, 287 TFLOP/s).  Tiles of 64 rows leave registers for loads
// two k tiles ahead (with 128 rows they spilled at the ends of odd sums).
#include "group.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short i16x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint64_t u64x2 __attribute__((ext_vector_type(2)));

constexpr int BN = 128, BK = 64;
constexpr int OPERAND = 128 * BK * 2, BUFFER = 2 * OPERAND;  // bytes of an operand's tile, of both

__device__ __forceinline__ int swz_row(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swz_col(int row) { return ((row & 3) | ((row >> 1) & 4)) << 1; }

// The vector's elements moved n places down, zeros above (n in 0 .. 8).
__device__ __forceinline__ u32x4 shift_down(const u32x4 &w, int n) {
  u64x2 v = __builtin_bit_cast(u64x2, w);
  if (n >= 4) v = u64x2{v[1], 0};
  const int b = (n & 3) * 16;
  v[0] = v[0] >> b | v[1] << 1 << (63 - b);
  v[1] >>= b;
  if (n >= 8) v = u64x2{0, 0};
  return __builtin_bit_cast(u32x4, v);
}

// One thread's four 16-byte pieces of an operand's k tiles.  T: the operand's
// rows run across the sum: k = tid / 16 + 16 j, columns 8 (tid % 16) .. + 7;
// else along it: rows tid / 8 + 32 j, k = 8 (tid % 8) .. + 7.  Rows past the n
// inside are taken as the last one inside (what they give is not stored).
// SETS: tiles whose loads may be in flight.
template <bool T, int PIECES, int SETS> struct Stage {
  const char *base;  // of the next tile
  int64_t step;
  uint32_t off[PIECES];
  int at, shift;     // byte in LDS, elements to shift the pieces down (T, at the columns' end)
  bool edge;         // some thread shifts
  u32x4 v[SETS][PIECES];
  static constexpr int NEXT = T ? 16 * 256 : 32 * 128;  // bytes from piece to piece in LDS

  __device__ __forceinline__ void init(const void *p, int64_t ld, int n, int tid) {
    base = (const char *)p;
    step = T ? ld * (2 * BK) : 2 * BK;
    if constexpr (T) {
      const int k = tid >> 4, chunk = tid & 15, col = min(chunk * 8, n - 8);  // below 0 in a tile that is not the first
      base -= 16;
      shift = min(chunk * 8 - col, 8);
      edge = n < 128 && n % 8 != 0;
      at = k * 256 + (chunk ^ swz_col(k)) * 16;
#pragma unroll
      for (int j = 0; j < PIECES; ++j) off[j] = (uint32_t)(k + 16 * j) * (uint32_t)ld * 2u + (uint32_t)(col + 8) * 2u;
    } else {
      const int row = tid >> 3, chunk = tid & 7;
      shift = 0;
      edge = false;
      at = row * 128 + (chunk ^ swz_row(row)) * 16;
#pragma unroll
      for (int j = 0; j < PIECES; ++j)
        off[j] = (uint32_t)min(row + 32 * j, n - 1) * (uint32_t)ld * 2u + (uint32_t)chunk * 16u;
    }
  }
  __device__ __forceinline__ void load_all(int set) {
#pragma unroll
    for (int j = 0; j < PIECES; ++j) v[set][j] = *(const u32x4_any *)(base + off[j]);
    base += step;
  }
  // the next tile, of which `left` values of k are inside; its pieces are whole
  // (T false: and shifted) when this returns
  __device__ __forceinline__ void load(int left, int tid, int set) {
    if (left >= BK) return load_all(set);
    if (left <= 0) return;
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      if constexpr (T) {
        const int k = (tid >> 4) + 16 * j, in = min(k, left - 1);
        v[set][j] = *(const u32x4_any *)(base + (off[j] - (uint32_t)(k - in) * (uint32_t)(step >> 6)));
        if (k >= left) v[set][j] = u32x4{0, 0, 0, 0};
      } else {
        const int over = min(max((tid & 7) * 8 + 8 - left, 0), 64);  // elements past the row's end
        const u32x4 w = *(const u32x4_any *)(base + (int64_t)off[j] - over * 2);
        v[set][j] = shift_down(w, min(over, 8));
      }
    }
  }
  __device__ __forceinline__ void write(char *lds, int set) {
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
      if (T && edge) v[set][j] = shift_down(v[set][j], shift);
      *(u32x4 *)(lds + at + j * NEXT) = v[set][j];
    }
  }
};

// Fragment i (16 rows or columns of the operand from `first` on) of k group g.
template <bool T> __device__ __forceinline__ bf16x8_t fragment(const char *lds, int first, int g, int lane) {
  const int li = lane & 15, lg = lane >> 4;
  if constexpr (T) {
    typedef __attribute__((address_space(3))) i16x4_t *P;
    const int row = 8 * lg + (li >> 2);
    const char *p = lds + (g * 32 + row) * 256 + (((first >> 3) + ((li & 3) >> 1)) ^ swz_col(row)) * 16 + (li & 1) * 8;
    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
    const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 1024));  // 4 rows on
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    return *(const bf16x8_t *)(lds + (first + li) * 128 + ((4 * g + lg) ^ swz_row(li)) * 16);
  }
}

// Where a workgroup's tile is: A and B from its first row, column and k on.
struct Tile {
  const bf16_t *A, *B;
  int g, row0, rows, c0, cols, Q, slot;
  bool sums;  // of A's columns, too (the bias gradient)
};

// The tile's sums and results; waves of 16 FM x 64 outputs.
template <int MODE, int FM, int SETS>
__device__ __forceinline__ void group_mid_tile(const GroupArgs &a, const Tile &t, char *lds) {
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;
  constexpr int FN = 4;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1, li = lane & 15, lg = lane >> 4;
  const int Q = t.Q;
  Stage<AT, FM, SETS> sa;  // half a tile has half of A's rows
  Stage<BT, 4, SETS> sb;
  sa.init(t.A, a.lda, t.rows, tid);
  sb.init(t.B, a.ldb, t.cols, tid);
  f32x4_t acc[FM][FN], bacc[2];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  bacc[0] = bacc[1] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  const auto write = [&](int to, int from) {
    sa.write(lds + to * BUFFER, from);
    sb.write(lds + to * BUFFER + OPERAND, from);
  };
  const auto load = [&](int left, int to) {
    sa.load(left, tid, to);
    sb.load(left, tid, to);
  };
  // k tile k0, of buffer p: the next one to LDS and the one SETS
  // after that to the registers this frees; `all` says that the latter is
  // inside as a whole (the loop of such tiles has no branch, at whose end a
  // load would be waited for)
  const auto tile = [&](int k0, int p, auto all) {
    const int set = SETS == 1 ? 0 : 1 - p;
    const char *now = lds + p * BUFFER;
    if (Q - k0 > BK) write(1 - p, set);
    if constexpr (decltype(all)::value) {
      sa.load_all(set);
      sb.load_all(set);
    } else {
      load(Q - k0 - (SETS + 1) * BK, set);
    }
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      bf16x8_t x[FM], w[FN];
#pragma unroll
      for (int i = 0; i < FM; ++i) x[i] = fragment<AT>(now, (wm * FM + i) * 16, g, lane);
#pragma unroll
      for (int j = 0; j < FN; ++j) w[j] = fragment<BT>(now + OPERAND, (wn * FN + j) * 16, g, lane);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], x[i], acc[i][j], 0, 0, 0);
      if constexpr (MODE == GROUP_DW) {
        if (t.sums) {  // A's columns against ones, wave wn taking every other fragment
          const uint32_t one2 = 0x3F803F80u;
          const bf16x8_t ones = __builtin_bit_cast(bf16x8_t, u32x4{one2, one2, one2, one2});
#pragma unroll
          for (int i = 0; i < FM; ++i)
            if ((i & 1) == wn) bacc[i >> 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, x[i], bacc[i >> 1], 0, 0, 0);
        }
      }
    }
    __syncthreads();
  };
#pragma unroll
  for (int i = 0; i < SETS; ++i) load(Q - i * BK, i);
  if (Q > 0) write(0, 0);
  load(Q - SETS * BK, 0);
  __syncthreads();
  int k0 = 0, p = 0;
  if constexpr (SETS == 1) {
    for (; k0 + 3 * BK <= Q; k0 += BK, p ^= 1) tile(k0, p, std::true_type{});
    for (; k0 < Q; k0 += BK, p ^= 1) tile(k0, p, std::false_type{});
  } else {  // (registers are chosen by constants)
    for (; k0 + 5 * BK <= Q; k0 += 2 * BK) {
      tile(k0, 0, std::true_type{});
      tile(k0 + BK, 1, std::true_type{});
    }
    for (; k0 < Q; k0 += 2 * BK) {
      tile(k0, 0, std::false_type{});
      if (k0 + BK < Q) tile(k0 + BK, 1, std::false_type{});
    }
  }

  // The results go through LDS, 32 FM rows of 512 bytes, so that whole rows of
  // the tile are written at once.
  const auto place = [&](int r, int c) { return lds + r * 512 + ((c >> 2) ^ ((r & 7) << 2)) * 16; };
  const int r0 = tid >> 4, c8 = (tid & 15) * 8;  // forward, input gradient: this thread's first row and its columns
  const FinishRows<bf16_t, MODE == GROUP_DW ? GROUP_FWD : MODE, 2 * FM> out(a, t.g, t.row0 + r0, 16, t.row0 + t.rows,
                                                                            t.c0 + c8);
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j) *(f32x4_t *)place((wm * FM + i) * 16 + li, (wn * FN + j) * 16 + 4 * lg) = acc[i][j];
  __syncthreads();
  if constexpr (MODE == GROUP_DW) {
    const int c = t.c0 + (tid & 31) * 4;
    if (c < a.N)
      for (int r = tid >> 5; r < t.rows; r += 8)
        store_grad(a, t.g, t.slot, t.row0 + r, c, *(const f32x4_t *)place(r, (tid & 31) * 4));
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int m = (wm * FM + i) * 16 + li;
      if (t.sums && lg == 0 && (i & 1) == wn && m < t.rows) store_bias_grad(a, t.g, t.slot, t.row0 + m, bacc[i >> 1][0]);
    }
  } else {
    out.store(a, [&](int i, int j) { return *(const f32x4_t *)place(r0 + 16 * i, c8 + 4 * j); });
  }
}

// BM: rows of a tile, 128 or 64.
template <int MODE, int BM>
__global__ void __launch_bounds__(256, 2) group_mid_kernel(GroupArgs a, int NT) {
  constexpr bool BT = MODE != GROUP_FWD;
  __shared__ __attribute__((aligned(1024))) char lds[2 * BUFFER];
  Tile t{(const bf16_t *)a.a, (const bf16_t *)a.b, 0, 0, 0, 0, 0, a.Q, -1, false};
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
    if (!tile_of<BM == 128>(a.off, a.G, a.M, BM, NT, blockIdx.x, t.g, t.row0, row1, nt)) return;
    t.rows = row1 - t.row0;
    t.c0 = nt * BN;
    t.A += (int64_t)t.row0 * a.lda;
    t.B += t.g * a.b_gs + (BT ? (int64_t)t.c0 : (int64_t)t.c0 * a.ldb);
  }
  t.cols = min(BN, a.N - t.c0);
  t.sums = MODE == GROUP_DW && a.db != nullptr && nt == 0;
  if constexpr (BM == 64) group_mid_tile<MODE, 2, 2>(a, t, lds);
  else if (MODE != GROUP_DW && t.rows <= BM / 2) group_mid_tile<MODE, 2, 1>(a, t, lds);
  else group_mid_tile<MODE, 4, 1>(a, t, lds);
}

template <int MODE, int BM> hipError_t run_tiles(const GroupArgs &a, hipStream_t s) {
  const int64_t NT = (a.N + BN - 1) / BN;
  const int64_t blocks = MODE == GROUP_DW ? piece_blocks(a, (int64_t)((a.M + BM - 1) / BM) * NT)
                                          : tile_blocks(a.M, a.G, BM, NT);
  if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL((group_mid_kernel<MODE, BM>), dim3((uint32_t)blocks), dim3(256), 0, s, a, (int)NT);
  return hipGetLastError();
}

// Tiles of 64 rows, and loads two k tiles ahead, if a CU has at most two of
// them: us for 64 and for 128 rows, forward, 20 groups, 1,500 rows, 800 -> 700
// (198 tiles of 64 rows), 14.9 and 20.4; 1 group, 2,000, 2048 -> 512 (124), 19.9
// and 25.1; 6, 16,000, 646 -> 191 (506), 18.7 and 20.2; but 4, 4,096, 1024 ->
// 1024 (528), 30.8 and 24.9.
template <int MODE> hipError_t run_mode(const GroupArgs &a, hipStream_t s) {
  if constexpr (MODE != GROUP_DW) {
    // a group's last tile half full on average
    const int64_t tiles = ((int64_t)a.M + 32 * a.G) / 64 * ((a.N + BN - 1) / BN);
    if (tiles <= 2 * kCUs) return run_tiles<MODE, 64>(a, s);
  }
  return run_tiles<MODE, 128>(a, s);
}

}  // namespace

// Eight elements at least in the operands' rows, and row strides whose offsets
// within a tile fit 32 bits.
bool group_mid_ok(int dtype, const GroupArgs &a, int mode) {
  return dtype == GCPSL_BF16 && a.lda <= kMaxTileLd && a.ldb <= kMaxTileLd && (mode == GROUP_FWD || a.N >= 8) &&
         (mode == GROUP_DW ? a.M >= 8 : a.Q >= 8);
}

hipError_t launch_group_mid(int mode, const GroupArgs &a, hipStream_t s) {
  return mode == GROUP_FWD ? run_mode<GROUP_FWD>(a, s)
                           : mode == GROUP_DX ? run_mode<GROUP_DX>(a, s) : run_mode<GROUP_DW>(a, s);
}

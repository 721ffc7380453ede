// Products over rows grouped by cluster, bf16, on gfx950: 256 x 256 outputs a
// workgroup from operands whose rows are 16-byte aligned.
//
// A k tile is 64 deep.  Each operand's 256 rows (or columns) are two halves of
// 128, each copied to LDS by loads that write LDS directly, as it lies in
// memory: an operand whose rows run along the sum as 128 rows of 128 bytes,
// one whose rows run across it as 64 rows of 256 bytes, from which
// ds_read_b64_tr_b16 makes fragments (within 16 lanes, lane 4 r + q reads 4
// columns of row r and lane i receives column i of the 4 rows).  16-byte
// chunks are XOR-swizzled within a row so that a fragment read uses every
// bank.
//
// Eight waves, two teams of four (one of each team on a SIMD): while one team
// multiplies, the other reads its next fragments, and they change places at
// every barrier.  A k tile has two phases: X multiplies the wave's 64 rows of
// the first A half by its 32 + 32 columns of both B halves, Y those of the
// second A half; 32 MFMAs (512 cycles) against 12 fragment reads a wave (192
// cycles of the LDS for a team at 256 bytes a cycle).  X reads the fragments of A's first half and
// of B's second, Y those of A's second half and of B's first half for the next
// tile.  A half is free as soon as both teams have read it and is refilled at
// once with what it holds two tiles on, so a copy has three phases (3,072
// MFMA cycles) to land.
//
// The MFMA takes B fragments as its first operand, so that a lane holds four
// consecutive columns of one row of the result.
//
// Bound: the matrix cores, at a clock that their power brings down to 1.5 to
// 1.8 GHz.  A k tile's two phases for both teams take about 2,270 cycles where
// the MFMAs alone take 2,048; a tile has about 10 us besides (offsets and first
// copies, results).  Even groups, 32,768 rows of 16, 4096 -> 4096: forward 844
// us (1,303 TFLOP/s), input gradient 819 (1,342), weight gradient 1,033 (1,064;
// 1.07 GB of fp32 results take 240 by themselves).  Ragged groups leave a last
// round partly empty: forward 937.
#include "group.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define LDS_PTR(p) ((__attribute__((address_space(3))) void *)(p))

constexpr int BM = 256, BN = 256, BK = 64, HALF = 128;  // rows and columns of a tile, depth, rows of a half
constexpr int HALF_BYTES = HALF * BK * 2;               // 16 KB: two 16-byte copies a thread
constexpr int STAGE = 4 * HALF_BYTES;                   // A's halves, B's halves
constexpr int OUT_ROW = BN * 4 + 16;      // bytes of a row of results in LDS (padded against bank conflicts)
constexpr int LDS_BYTES = 9 * HALF_BYTES;  // two stages, or three of half a tile
static_assert(HALF * OUT_ROW <= LDS_BYTES, "half a tile of results");
constexpr int FM = 4, FN = 2;  // 16-row and 16-column fragments of a wave in a half

// XOR on the 16-byte chunk of LDS row `row`: rows of 128 bytes (8 chunks) and
// of 256 (16 chunks).
__device__ __forceinline__ int swz_row(int row) { return (row >> 1) & 7; }
__device__ __forceinline__ int swz_col(int row) { return ((row & 3) | ((row >> 1) & 4)) << 1; }

// One operand's copies: this thread's two byte offsets into each half (kOob
// where there is no such row or column), and their depths within a tile.
template <bool T> struct Copies {
  uint32_t off[2][2];
  int q[2];
  // T: columns [0, n) of rows of stride ld; else rows [0, n)
  __device__ __forceinline__ Copies(int wave, int lane, int64_t ld, int n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int byte = j * 8192 + wave * 1024 + lane * 16;
      if constexpr (T) {
        const int row = byte / 256, chunk = (byte % 256 / 16) ^ swz_col(row);
        q[j] = row;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int col = h * HALF + chunk * 8;
          off[h][j] = col < n ? ((uint32_t)row * (uint32_t)ld + (uint32_t)col) * 2u : kOob;
        }
      } else {
        const int row = byte / 128, chunk = (byte % 128 / 16) ^ swz_row(row);
        q[j] = chunk * 8;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int r = h * HALF + row;
          off[h][j] = r < n ? ((uint32_t)r * (uint32_t)ld + (uint32_t)(chunk * 8)) * 2u : kOob;
        }
      }
    }
  }
};

// Copies half h of k tile kt of an operand (first element at base, step bytes
// from tile to tile, Q deep) to its place.
template <bool T>
__device__ __forceinline__ void issue(const Copies<T> &c, const char *base, int64_t step, int kt, int Q, int h,
                                      char *lds) {
  const __amdgpu_buffer_rsrc_t rs = make_rsrc(base + kt * step, kOob);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    uint32_t off = c.off[h][j];
    if (kt * BK + BK > Q) off = kt * BK + c.q[j] < Q ? off : kOob;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, LDS_PTR(lds + j * 8192), 16, off, 0, 0, 0);
  }
}

// Fragments of a wave in one half: [k group][16 rows or columns].
struct FragA {
  u32x4 f[2][FM];
};
struct FragB {
  u32x4 f[2][FN];
};
__device__ __forceinline__ u32x4 join(const u32x2 &lo, const u32x2 &hi) {
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
}

// Reads a phase's fragments and waits for them (in one block of assembly, so
// that no register is used before its data is there, and the compiler adds no
// wait for copies in flight).  a, b: LDS byte addresses of the fragments; rows
// along the sum have one for each k group, those across it one for each
// fragment.
#define ROW_A "ds_read_b128 %0, %12\n\tds_read_b128 %1, %12 offset:2048\n\t"                    \
              "ds_read_b128 %2, %12 offset:4096\n\tds_read_b128 %3, %12 offset:6144\n\t"        \
              "ds_read_b128 %4, %13\n\tds_read_b128 %5, %13 offset:2048\n\t"                    \
              "ds_read_b128 %6, %13 offset:4096\n\tds_read_b128 %7, %13 offset:6144\n\t"
__device__ __forceinline__ void read_phase(FragA &A, FragB &B, const uint32_t (&a)[2], const uint32_t (&b)[2],
                                           std::integral_constant<int, GROUP_FWD>) {
  asm volatile(ROW_A
               "ds_read_b128 %8, %14\n\tds_read_b128 %9, %14 offset:2048\n\t"
               "ds_read_b128 %10, %15\n\tds_read_b128 %11, %15 offset:2048\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(A.f[0][0]), "=&v"(A.f[0][1]), "=&v"(A.f[0][2]), "=&v"(A.f[0][3]), "=&v"(A.f[1][0]),
                 "=&v"(A.f[1][1]), "=&v"(A.f[1][2]), "=&v"(A.f[1][3]), "=&v"(B.f[0][0]), "=&v"(B.f[0][1]),
                 "=&v"(B.f[1][0]), "=&v"(B.f[1][1])
               : "v"(a[0]), "v"(a[1]), "v"(b[0]), "v"(b[1])
               : "memory");
}
// k group g and half fragment h of a transposed fragment: 32 g + 4 h rows of 256 bytes on
#define TR(d, s)                                                                                      \
  "ds_read_b64_tr_b16 %" #d "0, %" #s "\n\t"
__device__ __forceinline__ void read_phase(FragA &A, FragB &B, const uint32_t (&a)[2], const uint32_t (&b)[2],
                                           std::integral_constant<int, GROUP_DX>) {
  u32x2 p[8];
  asm volatile("ds_read_b128 %0, %16\n\tds_read_b128 %1, %16 offset:2048\n\t"
               "ds_read_b128 %2, %16 offset:4096\n\tds_read_b128 %3, %16 offset:6144\n\t"
               "ds_read_b128 %4, %17\n\tds_read_b128 %5, %17 offset:2048\n\t"
               "ds_read_b128 %6, %17 offset:4096\n\tds_read_b128 %7, %17 offset:6144\n\t"
               "ds_read_b64_tr_b16 %8, %18\n\tds_read_b64_tr_b16 %9, %18 offset:1024\n\t"
               "ds_read_b64_tr_b16 %10, %18 offset:8192\n\tds_read_b64_tr_b16 %11, %18 offset:9216\n\t"
               "ds_read_b64_tr_b16 %12, %19\n\tds_read_b64_tr_b16 %13, %19 offset:1024\n\t"
               "ds_read_b64_tr_b16 %14, %19 offset:8192\n\tds_read_b64_tr_b16 %15, %19 offset:9216\n\t"
               "s_waitcnt lgkmcnt(0)"
               : "=&v"(A.f[0][0]), "=&v"(A.f[0][1]), "=&v"(A.f[0][2]), "=&v"(A.f[0][3]), "=&v"(A.f[1][0]),
                 "=&v"(A.f[1][1]), "=&v"(A.f[1][2]), "=&v"(A.f[1][3]), "=&v"(p[0]), "=&v"(p[1]), "=&v"(p[2]),
                 "=&v"(p[3]), "=&v"(p[4]), "=&v"(p[5]), "=&v"(p[6]), "=&v"(p[7])
               : "v"(a[0]), "v"(a[1]), "v"(b[0]), "v"(b[1])
               : "memory");
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int g = 0; g < 2; ++g) B.f[g][i] = join(p[4 * i + 2 * g], p[4 * i + 2 * g + 1]);
}
__device__ __forceinline__ void read_phase(FragA &A, FragB &B, const uint32_t (&a)[4], const uint32_t (&b)[2],
                                           std::integral_constant<int, GROUP_DW>) {
  u32x2 p[24];
#define FOUR(d0, d1, d2, d3, s)                                                                     \
  "ds_read_b64_tr_b16 %" d0 ", %" s "\n\tds_read_b64_tr_b16 %" d1 ", %" s " offset:1024\n\t"        \
  "ds_read_b64_tr_b16 %" d2 ", %" s " offset:8192\n\tds_read_b64_tr_b16 %" d3 ", %" s " offset:9216\n\t"
  asm volatile(FOUR("0", "1", "2", "3", "24") FOUR("4", "5", "6", "7", "25") FOUR("8", "9", "10", "11", "26")
                   FOUR("12", "13", "14", "15", "27") FOUR("16", "17", "18", "19", "28")
                       FOUR("20", "21", "22", "23", "29") "s_waitcnt lgkmcnt(0)"
               : "=&v"(p[0]), "=&v"(p[1]), "=&v"(p[2]), "=&v"(p[3]), "=&v"(p[4]), "=&v"(p[5]), "=&v"(p[6]),
                 "=&v"(p[7]), "=&v"(p[8]), "=&v"(p[9]), "=&v"(p[10]), "=&v"(p[11]), "=&v"(p[12]), "=&v"(p[13]),
                 "=&v"(p[14]), "=&v"(p[15]), "=&v"(p[16]), "=&v"(p[17]), "=&v"(p[18]), "=&v"(p[19]), "=&v"(p[20]),
                 "=&v"(p[21]), "=&v"(p[22]), "=&v"(p[23])
               : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1])
               : "memory");
#undef FOUR
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int g = 0; g < 2; ++g) A.f[g][i] = join(p[4 * i + 2 * g], p[4 * i + 2 * g + 1]);
#pragma unroll
  for (int i = 0; i < FN; ++i)
#pragma unroll
    for (int g = 0; g < 2; ++g) B.f[g][i] = join(p[16 + 4 * i + 2 * g], p[17 + 4 * i + 2 * g]);
}
// B's first half of the first tile.
__device__ __forceinline__ void read_first(FragB &B, const uint32_t (&b)[2], bool transposed) {
  if (transposed) {
    u32x2 p[8];
    asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:1024\n\t"
                 "ds_read_b64_tr_b16 %2, %8 offset:8192\n\tds_read_b64_tr_b16 %3, %8 offset:9216\n\t"
                 "ds_read_b64_tr_b16 %4, %9\n\tds_read_b64_tr_b16 %5, %9 offset:1024\n\t"
                 "ds_read_b64_tr_b16 %6, %9 offset:8192\n\tds_read_b64_tr_b16 %7, %9 offset:9216\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(p[0]), "=&v"(p[1]), "=&v"(p[2]), "=&v"(p[3]), "=&v"(p[4]), "=&v"(p[5]), "=&v"(p[6]), "=&v"(p[7])
                 : "v"(b[0]), "v"(b[1])
                 : "memory");
#pragma unroll
    for (int i = 0; i < FN; ++i)
#pragma unroll
      for (int g = 0; g < 2; ++g) B.f[g][i] = join(p[4 * i + 2 * g], p[4 * i + 2 * g + 1]);
  } else {
    asm volatile("ds_read_b128 %0, %4\n\tds_read_b128 %1, %4 offset:2048\n\t"
                 "ds_read_b128 %2, %5\n\tds_read_b128 %3, %5 offset:2048\n\t"
                 "s_waitcnt lgkmcnt(0)"
                 : "=&v"(B.f[0][0]), "=&v"(B.f[0][1]), "=&v"(B.f[1][0]), "=&v"(B.f[1][1])
                 : "v"(b[0]), "v"(b[1])
                 : "memory");
  }
}
#undef ROW_A
#undef TR

__device__ __forceinline__ void barrier() { asm volatile("s_barrier" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <int MODE>
__global__ void __launch_bounds__(512, 2) group_tile_kernel(GroupArgs a, int NT) {
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;
  constexpr int NA = AT ? FM : 2;  // fragment addresses of A
  extern __shared__ __attribute__((aligned(1024))) char smem[];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 2, wn = wave & 3, li = lane & 15, lg = lane >> 4;

  int g, row0, rows, c0, Q, slot = -1, nt;
  const char *A, *B;
  if constexpr (MODE == GROUP_DW) {
    const int MT = (a.M + BM - 1) / BM;
    int mt, q0, q1;
    uint32_t t;
    if (!piece_of(a, (uint32_t)MT * (uint32_t)NT, blockIdx.x, g, q0, q1, slot, t)) return;
    block_order(t, (uint32_t)MT, (uint32_t)NT, mt, nt);
    row0 = mt * BM;
    Q = q1 - q0;
    rows = min(BM, a.M - row0);
    c0 = nt * BN;
    A = (const char *)a.a + ((int64_t)q0 * a.lda + row0) * 2;
    B = (const char *)a.b + ((int64_t)q0 * a.ldb + c0) * 2;
  } else {
    int row1;
    if (!tile_of(a.off, a.G, a.M, BM, NT, blockIdx.x, g, row0, row1, nt)) return;
    rows = row1 - row0;
    c0 = nt * BN;
    Q = a.Q;
    A = (const char *)a.a + (int64_t)row0 * a.lda * 2;
    B = (const char *)a.b + (g * a.b_gs + (BT ? (int64_t)c0 : (int64_t)c0 * a.ldb)) * 2;
  }
  const int cols = min(BN, a.N - c0), nk = (Q + BK - 1) / BK;
  const int64_t stepA = AT ? a.lda * (BK * 2) : BK * 2, stepB = BT ? a.ldb * (BK * 2) : BK * 2;
  const Copies<AT> ca(wave, lane, a.lda, rows);
  const Copies<BT> cb(wave, lane, a.ldb, cols);
  char *const dst = smem + wave * 1024;
  const auto copyA = [&](int kt, int h) { issue<AT>(ca, A, stepA, kt, Q, h, dst + (kt & 1) * STAGE + h * HALF_BYTES); };
  const auto copyB = [&](int kt, int h) {
    issue<BT>(cb, B, stepB, kt, Q, h, dst + (kt & 1) * STAGE + (2 + h) * HALF_BYTES);
  };

  // fragment addresses in the first halves of the first stage
  const uint32_t lds0 = (uint32_t)(size_t)LDS_PTR(smem);
  uint32_t ra[NA], rb[2];
  const int trow = 8 * lg + (li >> 2), tswz = swz_col(trow);  // transposed: row and its swizzle
  if constexpr (AT) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
      ra[i] = lds0 + trow * 256 + (((2 * (wm * FM + i) + ((li & 3) >> 1)) ^ tswz) * 16) + (li & 1) * 8;
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k) ra[k] = lds0 + (wm * FM * 16 + li) * 128 + (((4 * k + lg) ^ swz_row(li)) * 16);
  }
  if constexpr (BT) {
#pragma unroll
    for (int i = 0; i < FN; ++i)
      rb[i] = lds0 + 2 * HALF_BYTES + trow * 256 + (((2 * (wn * FN + i) + ((li & 3) >> 1)) ^ tswz) * 16) + (li & 1) * 8;
  } else {
#pragma unroll
    for (int k = 0; k < 2; ++k)
      rb[k] = lds0 + 2 * HALF_BYTES + (wn * FN * 16 + li) * 128 + (((4 * k + lg) ^ swz_row(li)) * 16);
  }

  f32x4_t acc[2][FM][2][FN];  // [A half][fragment][B half][fragment]
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[h][i][k][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  // weight gradient: sums of A's columns (the bias gradient) ride along in the
  // workgroups of the first column tile, wave wn taking fragment wn of each half
  const bool sums = MODE == GROUP_DW && a.db != nullptr && nt == 0;
  f32x4_t bacc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};

  FragA fa;
  FragB first[2], second;  // B's halves; the first one of this tile and of the next
  const auto multiply = [&](int h, const FragB &b0) {
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) {
          acc[h][i][0][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8_t, b0.f[k][j]), __builtin_bit_cast(bf16x8_t, fa.f[k][i]), acc[h][i][0][j], 0, 0, 0);
          acc[h][i][1][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
              __builtin_bit_cast(bf16x8_t, second.f[k][j]), __builtin_bit_cast(bf16x8_t, fa.f[k][i]), acc[h][i][1][j], 0, 0,
              0);
        }
      if constexpr (MODE == GROUP_DW) {
        if (sums) {
          const uint32_t one2 = 0x3F803F80u;  // two bf16 ones
          const u32x4 ones{one2, one2, one2, one2};
#pragma unroll
          for (int i = 0; i < FM; ++i)
            if (i == wn)
              bacc[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, ones),
                                                                __builtin_bit_cast(bf16x8_t, fa.f[k][i]), bacc[h], 0, 0, 0);
        }
      }
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
  };
  using Mode = std::integral_constant<int, MODE>;
  // addresses d bytes on
  const auto at_a = [&](uint32_t d, uint32_t(&r)[NA]) {
#pragma unroll
    for (int i = 0; i < NA; ++i) r[i] = ra[i] + d;
  };
  const auto at_b = [&](uint32_t d, uint32_t(&r)[2]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) r[i] = rb[i] + d;
  };
  if (MODE != GROUP_DW && rows <= HALF) {
    // Tiles of the first A half only: one phase a k tile, 32 MFMAs against 16
    // fragment reads, in three buffers of A's half and B's two.  A k tile is
    // copied two phases before it is read.
    const auto copy = [&](int kt, int p) {
      char *const d = dst + p * (3 * HALF_BYTES);
      issue<AT>(ca, A, stepA, kt, Q, 0, d);
      issue<BT>(cb, B, stepB, kt, Q, 0, d + HALF_BYTES);
      issue<BT>(cb, B, stepB, kt, Q, 1, d + 2 * HALF_BYTES);
    };
    copy(0, 0);
    copy(1, 1);
    wait_copies<6>();
    barrier();
    if (wm == 1) barrier();
    for (int kt = 0, p = 0; kt < nk; ++kt) {
      copy(kt + 2, p == 0 ? 2 : p - 1);
      uint32_t xa[NA], xb[2];
      at_a(p * (3 * HALF_BYTES), xa);
      at_b(p * (3 * HALF_BYTES), xb);  // (rb is past A's two halves: this is B's second one)
      read_phase(fa, second, xa, xb, Mode{});
      at_b(p * (3 * HALF_BYTES) - HALF_BYTES, xb);
      read_first(first[0], xb, BT);
      wait_copies<6>();
      barrier();
      multiply(0, first[0]);
      barrier();
      p = p == 2 ? 0 : p + 1;
    }
    if (wm == 0) barrier();
  } else {
  // what the phases before the first would have copied
  copyB(0, 0);
  copyA(0, 0);
  copyB(0, 1);
  copyA(0, 1);
  copyB(1, 0);
  copyA(1, 0);
  copyB(1, 1);
  wait_copies<8>();
  barrier();
  read_first(first[0], rb, BT);
  barrier();
  if (wm == 1) barrier();  // the second team is one slot behind

  const auto tile = [&](int kt, auto P) {
    constexpr int p = decltype(P)::value;  // kt % 2
    uint32_t xa[NA], xb[2];
    // X
    copyA(kt + 1, 1);
    copyB(kt + 2, 0);
    at_a(p * STAGE, xa);
    at_b(p * STAGE + HALF_BYTES, xb);
    read_phase(fa, second, xa, xb, Mode{});
    wait_copies<8>();
    barrier();
    multiply(0, first[p]);
    barrier();
    // Y
    copyA(kt + 2, 0);
    copyB(kt + 2, 1);
    at_a(p * STAGE + HALF_BYTES, xa);
    at_b((1 - p) * STAGE, xb);
    read_phase(fa, first[1 - p], xa, xb, Mode{});
    wait_copies<8>();
    barrier();
    multiply(1, first[p]);
    barrier();
  };
  int kt = 0;
  for (; kt + 1 < nk; kt += 2) {
    tile(kt, std::integral_constant<int, 0>{});
    tile(kt + 1, std::integral_constant<int, 1>{});
  }
  if (kt < nk) tile(kt, std::integral_constant<int, 0>{});
  if (wm == 0) barrier();
  }
  wait_copies<0>();  // no copy may land in LDS after the workgroup's end

  // The results go through LDS, a half at a time, so that whole rows of the
  // tile are written at once.
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (h * HALF >= rows) break;
    const int high = min(HALF, rows - h * HALF), m0 = row0 + h * HALF;
    // forward, input gradient: two rows a wave, eight columns a lane
    const int r0 = wave * 2 + (lane >> 5), c = (lane & 31) * 8;
    const FinishRows<bf16_t, MODE == GROUP_DW ? GROUP_FWD : MODE, HALF / 16, false> out(a, g, m0 + r0, 16, m0 + high,
                                                                                        c0 + c);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          *(f32x4_t *)(smem + ((wm * FM + i) * 16 + li) * OUT_ROW + (k * HALF + (wn * FN + j) * 16 + 4 * lg) * 4) =
              acc[h][i][k][j];
    __syncthreads();
    if constexpr (MODE == GROUP_DW) {  // a row a wave
      const int c4 = c0 + lane * 4;
      if (c4 < a.N)
        for (int r = wave; r < high; r += 8)
          store_grad(a, g, slot, m0 + r, c4, *(const f32x4_t *)(smem + r * OUT_ROW + lane * 16));
    } else {
      out.store(a, [&](int i, int j) { return *(const f32x4_t *)(smem + (r0 + 16 * i) * OUT_ROW + (c + 4 * j) * 4); });
    }
  }
  if (sums && lg == 0) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int m = h * HALF + (wm * FM + wn) * 16 + li;
      if (m < rows) store_bias_grad(a, g, slot, row0 + m, bacc[h][0]);
    }
  }
}

template <int MODE> hipError_t run(const GroupArgs &a, hipStream_t s) {
  static PerDeviceOnce once;
  if (once.needed()) {
    const hipError_t e = hipFuncSetAttribute((const void *)group_tile_kernel<MODE>,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);
    if (e != hipSuccess) return e;
    once.mark();
  }
  const int64_t NT = (a.N + BN - 1) / BN;
  const int64_t blocks = MODE == GROUP_DW ? piece_blocks(a, (int64_t)((a.M + BM - 1) / BM) * NT)
                                          : tile_blocks(a.M, a.G, BM, NT);
  if (blocks > kMaxBlocks / 2) return hipErrorInvalidConfiguration;  // (of 512 threads)
  hipLaunchKernelGGL(group_tile_kernel<MODE>, dim3((uint32_t)blocks), dim3(512), LDS_BYTES, s, a, (int)NT);
  return hipGetLastError();
}

}  // namespace

bool group_tile_ok(int dtype, const GroupArgs &a, int mode) {
  if (dtype != GCPSL_BF16 || a.N % 8 || a.lda % 8 || a.ldb % 8 || a.b_gs % 8) return false;
  if (mode == GROUP_DW ? a.M % 8 : a.Q % 8) return false;
  if ((reinterpret_cast<uintptr_t>(a.a) | reinterpret_cast<uintptr_t>(a.b)) % 16) return false;
  return a.lda <= kMaxTileLd && a.ldb <= kMaxTileLd;
}

hipError_t launch_group_tile(int mode, const GroupArgs &a, hipStream_t s) {
  return mode == GROUP_FWD ? run<GROUP_FWD>(a, s) : mode == GROUP_DX ? run<GROUP_DX>(a, s) : run<GROUP_DW>(a, s);
}

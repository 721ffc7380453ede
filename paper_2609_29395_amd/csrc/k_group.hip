// Products over rows grouped by cluster (gfx950): forward, input gradient and
// weight gradient of one linear layer per group, and a gated layer's forward pass
// and gradient, the groups' rows one after another and of any counts.
//
// The group offsets are read on the device, so a launch depends on the number
// of rows and groups only: it has as many row tiles as any offsets can need,
// and a workgroup finds its group and rows by a scan of the offsets.
#include "group.h"

#include <cmath>
#include <type_traits>

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------ any alignment
// 64 x 64 outputs, four waves of 32 x 32.  A k tile is staged through
// registers element by element, so any stride and size will do, into LDS rows
// of consecutive q; both operands' fragments are 16-byte LDS reads.
//
// What is left to it: narrow fp32 results (fewer than 64 columns, 32 where there
// are few tiles), operands of fewer
// elements than a vector, row strides past 2^22.  Bound by the element loads:
// 65,536 rows of 8 groups, 128 -> 10, fp32, 20 us, 1.8 TB/s (7 us at a copy's
// rate); the kernels of 128 columns would waste most of their products on it.
template <typename T> struct Any;
template <> struct Any<bf16_t> {
  static constexpr int BQ = 64, LD = 72;  // q a tile; elements per LDS row (padded against bank conflicts)
  static __device__ __forceinline__ void mma(f32x4_t &acc, const bf16_t *a, const bf16_t *b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8_t *)a, *(const bf16x8_t *)b, acc, 0, 0, 0);
  }
  static constexpr int PER = 8, STEP = 32;  // consecutive q of one lane's fragment, q of a product
};
template <> struct Any<float> {
  static constexpr int BQ = 64, LD = 68;
  // four products of four q each: q = 4 (lane / 16) + j in product j, the same for both operands
  static __device__ __forceinline__ void mma(f32x4_t &acc, const float *a, const float *b) {
    const float4 x = *(const float4 *)a, y = *(const float4 *)b;
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, y.x, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, y.y, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, y.z, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, y.w, acc, 0, 0, 0);
  }
  static constexpr int PER = 4, STEP = 16;
};

template <typename T, int MODE>
__global__ void __launch_bounds__(256) group_any_kernel(GroupArgs a, int NT) {
  using K = Any<T>;
  constexpr int BQ = K::BQ, LD = K::LD, BM = 64, BN = 64;
  constexpr bool AT = MODE == GROUP_DW, BT = group_across(MODE);  // q runs over the operand's rows
  constexpr bool PAIR = MODE == GROUP_GATED;
  constexpr int COLS = PAIR ? BN / 2 : BN;                       // outputs of a tile
  constexpr int PT = BM * BQ / 256;                              // elements per thread and operand
  __shared__ __attribute__((aligned(16))) T la[BM * LD], lb[BN * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int li = lane & 15, lg = lane >> 4;
  int g, row0, row1, q0 = 0, q1 = a.Q, slot = -1, nt;
  if constexpr (MODE == GROUP_DW) {
    const uint32_t MT = (uint32_t)(a.M + BM - 1) / BM;
    uint32_t t;
    int mt;
    if (!piece_of(a, MT * (uint32_t)NT, blockIdx.x, g, q0, q1, slot, t)) return;
    block_order(t, MT, (uint32_t)NT, mt, nt);
    row0 = mt * BM;
    row1 = min(a.M, row0 + BM);
  } else {
    if (!tile_of(a.off, a.G, a.M, BM, NT, blockIdx.x, g, row0, row1, nt)) return;
  }
  const int c0 = nt * COLS;
  const T *A = (const T *)a.a, *B = (const T *)a.b + g * a.b_gs;
  // b's row (BT: column) at column j of the tile
  const auto col = [&](int j) { return PAIR ? min(c0 + j % COLS, a.N - 1) + (j < COLS ? 0 : a.N) : min(c0 + j, a.N - 1); };

  f32x4_t acc[2][2];  // [column fragment][row fragment]
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int wm = wave >> 1, wn = wave & 1;
  float rowsum = 0.f;  // weight grad: this thread's row of A (threads below BM)

  for (int q = q0; q < q1; q += BQ) {
    // consecutive threads take consecutive addresses of the operand; rows,
    // columns and q outside are loaded as the last ones inside, so that all
    // loads are in flight together
    T va[PT], vb[PT];
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int e = i * 256 + tid;
      const int ra = min(row0 + (AT ? e % BM : e / BQ), row1 - 1), qa = min(q + (AT ? e / BM : e % BQ), q1 - 1);
      const int rb = col(BT ? e % BN : e / BQ), qb = min(q + (BT ? e / BN : e % BQ), q1 - 1);
      va[i] = AT ? A[(int64_t)qa * a.lda + ra] : A[(int64_t)ra * a.lda + qa];
      vb[i] = BT ? B[(int64_t)qb * a.ldb + rb] : B[(int64_t)rb * a.ldb + qb];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int e = i * 256 + tid;
      const int ra = AT ? e % BM : e / BQ, qa = AT ? e / BM : e % BQ;
      const int rb = BT ? e % BN : e / BQ, qb = BT ? e / BN : e % BQ;
      la[ra * LD + qa] = q + qa < q1 ? va[i] : T(0);
      lb[rb * LD + qb] = q + qb < q1 ? vb[i] : T(0);
    }
    __syncthreads();
    for (int k = 0; k < min(BQ, q1 - q); k += K::STEP)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
          K::mma(acc[i][j], lb + (wn * 32 + i * 16 + li) * LD + k + lg * K::PER,
                 la + (wm * 32 + j * 16 + li) * LD + k + lg * K::PER);
    if (MODE == GROUP_DW && tid < BM)
      for (int i = 0; i < BQ; i += 8) {
        float v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = ElemT<T>::to_f(la[tid * LD + i + j]);
        rowsum += sum8(v);
      }
  }

  // lane (li, lg) holds columns 4 lg .. 4 lg + 3 of row li of each fragment
  if constexpr (PAIR) {  // the values' waves hand their sums over
    __shared__ f32x4_t values[2][2][2][64];  // [wm][column fragment][row fragment]
    if (wn == 1) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) values[wm][i][j][lane] = acc[i][j];
    }
    __syncthreads();
    if (wn == 1) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int m = row0 + wm * 32 + j * 16 + li, c = c0 + i * 16 + 4 * lg;
        if (m < row1) finish_pair<T, MODE>(a, g, m, c, acc[i][j], values[wm][i][j][lane]);
      }
    return;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int m = row0 + wm * 32 + j * 16 + li, c = c0 + wn * 32 + i * 16 + 4 * lg;
      if (m >= row1) continue;
      if constexpr (MODE == GROUP_DW) {
        if (c < a.N) store_grad(a, g, slot, m, c, acc[i][j]);
      } else if constexpr (MODE == GROUP_GATED_GRAD) {
        finish_pair<T, MODE>(a, g, m, c, acc[i][j], acc[i][j]);
      } else {
        if (c < a.N) finish<T, MODE>(a, g, m, c, acc[i][j]);
      }
    }
  if (MODE == GROUP_DW && a.db && nt == 0 && tid < BM && row0 + tid < row1)
    store_bias_grad(a, g, slot, row0 + tid, rowsum);
}

// out[0 .. per) = the sum of n partials of `per` entries each.  SPLIT: each wave
// takes a quarter of the partials, eight loads in flight (1 group of 8,192
// rows, 64 -> 64, in 27 pieces: 33 -> 18 us with the products); else a thread
// takes all of them (pieces of large results: 57 against 68 us for 1 group of
// 3,448 rows, 1024 -> 4096, in 2).
template <bool SPLIT>
__device__ __forceinline__ void join(const float *p, int64_t per, uint32_t n, float *out, uint32_t block,
                                     uint32_t blocks, f32x4_t (&quarter)[3][64]) {
  constexpr int ENTRIES = SPLIT ? 256 : 1024, AHEAD = SPLIT ? 8 : 4;
  const uint32_t wave = threadIdx.x >> 6, at = SPLIT ? threadIdx.x & 63 : threadIdx.x;
  const uint32_t k0 = SPLIT ? n * wave / 4 : 0, k1 = SPLIT ? n * (wave + 1) / 4 : n;
  for (int64_t base = (int64_t)block * ENTRIES; base < per; base += (int64_t)blocks * ENTRIES) {
    const int64_t i = base + at * 4;
    f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
    if (i + 4 <= per) {
      uint32_t k = k0;
      for (; k + AHEAD <= k1; k += AHEAD) {
        f32x4_any v[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) v[u] = *(const f32x4_any *)(p + (int64_t)(k + u) * per + i);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) s += v[u];
      }
#pragma unroll 2
      for (; k < k1; ++k) s += *(const f32x4_any *)(p + (int64_t)k * per + i);
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (i + r < per)
          for (uint32_t k = k0; k < k1; ++k) s[r] += p[(int64_t)k * per + i + r];
    }
    if (SPLIT) {
      if (wave) quarter[wave - 1][at] = s;
      __syncthreads();
      s = (s + quarter[0][at]) + (quarter[1][at] + quarter[2][at]);
      __syncthreads();
    }
    if (SPLIT && wave) continue;
    if (i + 4 <= per) *(f32x4_any *)(out + i) = s;
    else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (i + r < per) out[i + r] = s[r];
    }
  }
}

// Weight gradient in pieces: the pieces' sums, in an order of their own.
// `blocks` workgroups for each group, whose weights and biases they share;
// those of a group of one piece end at once.
__global__ void __launch_bounds__(256) group_join_kernel(GroupArgs a, uint32_t blocks) {
  __shared__ f32x4_t quarter[3][64];
  const int g = (int)(blockIdx.x / blocks);
  uint32_t before = 0, slots = 0, n = 0, first = 0;
  for (int base = 0; base <= g; base += 64) {
    LaneTiles l;
    before = lane_tiles<true>(a.off, a.G, a.Q, a.piece, base, before, l);
    const uint32_t own = l.tiles > 1 ? l.tiles : 0, sum = lane_scan(own);
    if (g < base + 64) {
      n = (uint32_t)of_lane((int)own, g - base);
      first = slots + (uint32_t)of_lane((int)(sum - own), g - base);
    }
    slots += (uint32_t)of_lane((int)sum, 63);
  }
  n = __builtin_amdgcn_readfirstlane(n);
  first = __builtin_amdgcn_readfirstlane(first);
  if (n == 0 || first + n > (uint32_t)a.slots) return;
  const int64_t per = (int64_t)a.M * a.N;
  const uint32_t block = blockIdx.x - g * blocks;
  const auto both = [&](auto SPLIT) {
    join<decltype(SPLIT)::value>(a.part + first * per, per, n, (float *)a.out + g * a.out_gs, block, blocks, quarter);
    if (a.db)
      join<decltype(SPLIT)::value>(a.part_db + (int64_t)first * a.M, a.M, n, a.db + g * a.db_gs, block, blocks, quarter);
  };
  if (n > 8) both(std::true_type());
  else both(std::false_type());
}

template <typename T>
hipError_t launch_any(int mode, const GroupArgs &a, hipStream_t s) {
  const int NT = mode == GROUP_GATED ? (a.N + 31) / 32 : (a.N + 63) / 64;
  if (mode == GROUP_DW) {
    const int64_t blocks = piece_blocks(a, (int64_t)((a.M + 63) / 64) * NT);
    if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((group_any_kernel<T, GROUP_DW>), dim3((uint32_t)blocks), dim3(256), 0, s, a, NT);
    return hipGetLastError();
  }
  const int64_t blocks = tile_blocks(a.M, a.G, 64, NT);
  if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
  const auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, s, a, NT); };
  if (mode == GROUP_FWD) launch(group_any_kernel<T, GROUP_FWD>);
  else if (mode == GROUP_DX) launch(group_any_kernel<T, GROUP_DX>);
  else if (mode == GROUP_GATED) launch(group_any_kernel<T, GROUP_GATED>);
  else launch(group_any_kernel<T, GROUP_GATED_GRAD>);
  return hipGetLastError();
}

}  // namespace

namespace {

// Whether tiles of 256 x 256 (a group's last one half full on average) give half
// of the CUs one.  With fewer the 128 x 128 kernel's are faster: 64 tiles,
// 4 groups of 128 rows, 4096 -> 4096, 47 against 55 us; 16, 8 groups of 256, 512
// -> 512, 12 against 16; as fast at 128, and slower from 144 on, 8 groups of
// 1,024, 1024 -> 1024, 32 against 27.
bool tiles_fill_half(int64_t row_tiles, int64_t cols) { return row_tiles * ((cols + 255) / 256) >= kCUs / 2; }
bool fills_half(const GroupArgs &a, int mode) {
  return tiles_fill_half(mode == GROUP_DW ? (int64_t)((a.M + 255) / 256) * a.G : ((int64_t)a.M + 128 * a.G) / 256,
                         group_cols(a, mode));
}

}  // namespace

// A piece takes the rows that a workgroup has if they are shared evenly over
// one round of workgroups on the chip, but enough of them that its products
// take longer than its partial, written and read again: 1,024 for tiles of
// 256 x 256 (15 us against 10).  For the others a piece of p rows costs about
// p a in products and, over all of the rows, rows tiles b / p in partials, the
// sum of which is least at p = sqrt(rows tiles b / a), b / a about 4 for bf16, 1
// for fp32 tiles of 128 x 128 and 0.5 for those of 64 x 64; 128 at least (two
// steps of the bf16 kernel; 64 are no faster) and 512 at most.  us with this and
// with 512 throughout: 1 group of 8,192 rows, 64 -> 64, bf16, 14 and 16; 1 of
// 1,024, 1024 -> 1024, fp32 in 128 x 128, 31 and 43.  The tile is the one that
// the operands most likely take.
//
// No group is cut, and the join's launch saved (1.5 to 2 us), where the largest
// one, taken as three times the average, has no more rows than that is worth,
// and all of them in one group would not take much longer.  With the input
// gradient, us so and in pieces, bf16: 8 groups of 1,024 rows, 1000 -> 500, 25.3
// and 27.6; 4 of 256, 256 -> 256, 12.9 and 14.5.
GroupPieces group_pieces(int dtype, int G, int64_t rows, int n, int k) {
  const bool big = dtype == GCPSL_BF16 && n % 8 == 0 && k % 8 == 0 &&
                   tiles_fill_half((int64_t)((n + 255) / 256) * G, k);
  const bool deep = dtype == GCPSL_F32 && group_f32_deep_grad(G, rows, n, k);
  const int64_t tile = big ? 256 : deep ? 64 : 128, slots = big || deep ? kCUs : 2 * kCUs;
  const int64_t tiles = ((n + tile - 1) / tile) * ((k + tile - 1) / tile);
  // (a CU holds one workgroup of the 64 x 64 kernel: no more of them than CUs)
  const int64_t even = tiles >= slots ? rows : deep ? rows / (slots / tiles) : rows * tiles / slots;
  const double b_by_a = dtype == GCPSL_BF16 ? 4 : deep ? 0.5 : 1;
  const int64_t least =
      big ? 1024 : std::min<int64_t>(512, std::max<int64_t>(128, (int64_t)std::sqrt(b_by_a * (double)rows * (double)tiles)));
  const int64_t whole = dtype == GCPSL_BF16 || deep ? 384 : 192;
  const bool one = rows <= 4 * whole && std::min(rows, 3 * rows / G) <= whole;
  const int64_t piece = one ? rows + 1 : std::min<int64_t>(std::max<int64_t>(even, least), 1 << 30);
  // a group of p > 1 pieces has more than (p - 1/2) piece >= 3/4 p piece rows
  return {(int)piece, rows * 2 >= piece * 3 ? (int)(rows * 4 / (piece * 3)) : 0};
}

hipError_t launch_group(int dtype, int mode, const GroupArgs &a, hipStream_t s) {
  hipError_t e;
  if (group_few_ok(dtype, a, mode)) e = launch_group_few(dtype, mode, a, s);
  else if (group_tile_ok(dtype, a, mode) && fills_half(a, mode)) e = launch_group_tile(mode, a, s);
  else if (group_mid_ok(dtype, a, mode)) e = launch_group_mid(mode, a, s);
  else if (dtype == GCPSL_F32 && group_f32_deep_ok(a, mode)) e = launch_group_f32_deep(mode, a, s);
  else if (dtype == GCPSL_F32 && group_cols(a, mode) >= 64 && group_f32_ok(a, mode)) e = launch_group_f32(mode, a, s);
  else e = dtype == GCPSL_BF16 ? launch_any<bf16_t>(mode, a, s) : launch_any<float>(mode, a, s);
  if (e == hipSuccess && mode == GROUP_DW && a.slots > 0) {
    // about eight workgroups a CU in all, of 256 entries or more
    const int64_t most = ((int64_t)a.M * a.N + 255) / 256, share = std::max(1, 2048 / a.G);
    const uint32_t n = (uint32_t)std::min(most, share);
    hipLaunchKernelGGL(group_join_kernel, dim3(n * (uint32_t)a.G), dim3(256), 0, s, a, n);
    e = hipGetLastError();
  }
  return e;
}

// Products over rows grouped by cluster (gfx950): forward, input gradient and
// weight gradient of one linear layer per group, the groups' rows one after
// another and of any counts.
//
// The group offsets are read on the device, so a launch depends on the number
// of rows and groups only: it has as many row tiles as any offsets can need,
// and a workgroup finds its group and rows by a scan of the offsets.
#include "runtime.h"
#include "ops.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

// Rows [begin, end) of group g, inside [0, rows) whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t *off, int g, int rows, int &begin, int &end) {
  begin = clampi(off[g], 0, rows);
  end = clampi(off[g + 1], begin, rows);
}

// Group and first row of row tile t (bm rows a tile, no tile spans groups);
// false if there are not that many.  Every wave scans by itself.  (A tile is
// checked against its group's own rows, so offsets that decrease can make
// groups overlap but no row outside [0, rows) is touched.)
__device__ __forceinline__ bool find_tile(const int32_t *off, int G, int rows, int bm, int t, int &g, int &row0,
                                          int &row1) {
  const int lane = threadIdx.x & 63;
  uint32_t before = 0;
  for (int base = 0; base < G; base += 64) {
    const int i = base + lane;
    int b = 0, e = 0;
    if (i < G) group_rows(off, i, rows, b, e);
    const uint32_t tiles = (uint32_t)(e - b + bm - 1) / (uint32_t)bm;
    uint32_t sum = tiles;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const uint32_t v = __shfl_up(sum, d, 64);
      if (lane >= d) sum += v;
    }
    const uint32_t first = before + sum - tiles;  // the group's first tile
    const uint64_t hit = __ballot((uint32_t)t - first < tiles);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      g = base + l;
      row0 = __shfl(b, l, 64) + (t - (int)__shfl(first, l, 64)) * bm;
      row1 = min(__shfl(e, l, 64), row0 + bm);
      g = __builtin_amdgcn_readfirstlane(g);
      row0 = __builtin_amdgcn_readfirstlane(row0);
      row1 = __builtin_amdgcn_readfirstlane(row1);
      return true;
    }
    before += __shfl(sum, 63, 64);
  }
  return false;
}

// ------------------------------------------------------------ any alignment
// 64 x 64 outputs, four waves of 32 x 32.  A k tile is staged through
// registers element by element, so any stride and size will do, into LDS rows
// of consecutive q; both operands' fragments are 16-byte LDS reads.
template <typename T> struct Any;
template <> struct Any<bf16_t> {
  static constexpr int BQ = 32, LD = 40;  // q a tile; elements per LDS row (padded against bank conflicts)
  static __device__ __forceinline__ void mma(f32x4_t &acc, const bf16_t *a, const bf16_t *b) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8_t *)a, *(const bf16x8_t *)b, acc, 0, 0, 0);
  }
  static constexpr int PER = 8;  // consecutive q of one lane's fragment
};
template <> struct Any<float> {
  static constexpr int BQ = 16, LD = 20;
  // four products of four q each: q = 4 (lane / 16) + j in product j, the same for both operands
  static __device__ __forceinline__ void mma(f32x4_t &acc, const float *a, const float *b) {
    const float4 x = *(const float4 *)a, y = *(const float4 *)b;
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, y.x, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, y.y, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, y.z, acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, y.w, acc, 0, 0, 0);
  }
  static constexpr int PER = 4;
};

// Four consecutive columns c .. c + 3 of row m of the result (forward, input
// gradient): bias, ReLU (a NaN stays one), dropout or gate, one rounding.
template <typename T, int MODE>
__device__ __forceinline__ void finish(const GroupArgs &a, int g, int m, int c, f32x4_t v) {
  if (c >= a.N) return;
  uint64_t word = 0;
  if (MODE == GROUP_FWD && a.drop.thr) word = drop_word(a.drop.key, m, (a.N + 3) >> 2, c >> 2);
  T *out = (T *)a.out + (int64_t)m * a.ldo + c;
  const T *gate = (const T *)a.gate + (int64_t)m * a.ldg + c;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (c + r >= a.N) break;
    float x = v[r];
    if constexpr (MODE == GROUP_FWD) {
      if (a.bias) x += a.bias[g * a.bias_gs + c + r];
      if (a.relu) x = x <= 0.f ? 0.f : x;
      if (a.drop.thr) x = drop_keeps(word, r, a.drop.thr) ? x * a.drop.scale : 0.f;
    } else {
      if (a.gate) x = ElemT<T>::to_f(gate[r]) > 0.f ? x * a.drop.scale : 0.f;
    }
    out[r] = ElemT<T>::from_f(x);
  }
}

template <typename T, int MODE>
__global__ void __launch_bounds__(256) group_any_kernel(GroupArgs a, int NT) {
  using K = Any<T>;
  constexpr int BQ = K::BQ, LD = K::LD, BM = 64, BN = 64;
  constexpr bool AT = MODE == GROUP_DW, BT = MODE != GROUP_FWD;  // q runs over the operand's rows
  constexpr int PT = BM * BQ / 256;                              // elements per thread and operand
  __shared__ __attribute__((aligned(16))) T la[BM * LD], lb[BN * LD];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int li = lane & 15, lg = lane >> 4;
  const int nt = blockIdx.x % NT;
  int g, row0, row1, q0 = 0, q1 = a.Q, mt = blockIdx.x / NT, split = 0;
  if constexpr (MODE == GROUP_DW) {
    const int MT = (a.M + BM - 1) / BM;
    split = mt / MT % a.splits;
    g = mt / MT / a.splits;
    row0 = mt % MT * BM;
    row1 = min(a.M, row0 + BM);
    group_rows(a.off, g, a.Q, q0, q1);
    const int piece = ((q1 - q0 + a.splits - 1) / a.splits + BQ - 1) / BQ * BQ;
    const int64_t at = q0 + (int64_t)split * piece;  // may pass the group's end, and 31 bits
    q0 = (int)min(at, (int64_t)q1);
    q1 = (int)min(at + piece, (int64_t)q1);
  } else {
    if (!find_tile(a.off, a.G, a.M, BM, mt, g, row0, row1)) return;
  }
  const int c0 = nt * BN;
  const T *A = (const T *)a.a, *B = (const T *)a.b + g * a.b_gs;

  f32x4_t acc[2][2];  // [column fragment][row fragment]
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  const int wm = wave >> 1, wn = wave & 1;
  float rowsum = 0.f;  // weight grad: this thread's row of A (threads below BM)

  for (int q = q0; q < q1; q += BQ) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PT; ++i) {
      const int e = i * 256 + tid;
      // consecutive threads take consecutive addresses of the operand
      const int ra = AT ? e % BM : e / BQ, qa = AT ? e / BM : e % BQ;
      const int rb = BT ? e % BN : e / BQ, qb = BT ? e / BN : e % BQ;
      T va = 0, vb = 0;
      if (row0 + ra < row1 && q + qa < q1)
        va = AT ? A[(int64_t)(q + qa) * a.lda + row0 + ra] : A[(int64_t)(row0 + ra) * a.lda + q + qa];
      if (c0 + rb < a.N && q + qb < q1)
        vb = BT ? B[(int64_t)(q + qb) * a.ldb + c0 + rb] : B[(int64_t)(c0 + rb) * a.ldb + q + qb];
      la[ra * LD + qa] = va;
      lb[rb * LD + qb] = vb;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        K::mma(acc[i][j], lb + (wn * 32 + i * 16 + li) * LD + lg * K::PER, la + (wm * 32 + j * 16 + li) * LD + lg * K::PER);
    if (MODE == GROUP_DW && tid < BM)
      for (int i = 0; i < BQ; ++i) rowsum += ElemT<T>::to_f(la[tid * LD + i]);
  }

  // lane (li, lg) holds columns 4 lg .. 4 lg + 3 of row li of each fragment
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int m = row0 + wm * 32 + j * 16 + li, c = c0 + wn * 32 + i * 16 + 4 * lg;
      if (m >= row1) continue;
      if constexpr (MODE == GROUP_DW) {
        float *out = a.splits > 1 ? a.part + (((int64_t)split * a.G + g) * a.M + m) * a.N + c
                                  : (float *)a.out + g * a.out_gs + (int64_t)m * a.ldo + c;
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (c + r < a.N) out[r] = acc[i][j][r];
      } else {
        finish<T, MODE>(a, g, m, c, acc[i][j]);
      }
    }
  if (MODE == GROUP_DW && a.db && nt == 0 && tid < BM && row0 + tid < row1) {
    if (a.splits > 1) a.part_db[((int64_t)split * a.G + g) * a.M + row0 + tid] = rowsum;
    else a.db[g * a.db_gs + row0 + tid] = rowsum;
  }
}

// Weight gradient in pieces: the pieces' sums, in order.
__global__ void __launch_bounds__(256) group_join_kernel(GroupArgs a) {
  const int64_t per = (int64_t)a.M * a.N, all = per * a.G, all_db = (int64_t)a.M * a.G;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i < all) {
    float s = 0.f;
    for (int k = 0; k < a.splits; ++k) s += a.part[k * all + i];
    const int64_t g = i / per, r = i - g * per;
    ((float *)a.out)[g * a.out_gs + r / a.N * a.ldo + r % a.N] = s;
  } else if (a.db && i - all < all_db) {
    const int64_t j = i - all;
    float s = 0.f;
    for (int k = 0; k < a.splits; ++k) s += a.part_db[k * all_db + j];
    a.db[j / a.M * a.db_gs + j % a.M] = s;
  }
}

template <typename T>
hipError_t launch_any(int mode, const GroupArgs &a, hipStream_t s) {
  const int NT = (a.N + 63) / 64;
  if (mode == GROUP_DW) {
    const int64_t blocks = (int64_t)((a.M + 63) / 64) * NT * a.splits * a.G;
    if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((group_any_kernel<T, GROUP_DW>), dim3((uint32_t)blocks), dim3(256), 0, s, a, NT);
    if (a.splits > 1) {
      const int64_t n = (int64_t)a.G * a.M * (a.N + (a.db ? 1 : 0));
      hipLaunchKernelGGL(group_join_kernel, dim3((uint32_t)((n + 255) / 256)), dim3(256), 0, s, a);
    }
    return hipGetLastError();
  }
  const int64_t blocks = ((int64_t)a.M / 64 + min(a.G, a.M)) * NT;
  if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
  if (blocks == 0) return hipSuccess;
  if (mode == GROUP_FWD)
    hipLaunchKernelGGL((group_any_kernel<T, GROUP_FWD>), dim3((uint32_t)blocks), dim3(256), 0, s, a, NT);
  else
    hipLaunchKernelGGL((group_any_kernel<T, GROUP_DX>), dim3((uint32_t)blocks), dim3(256), 0, s, a, NT);
  return hipGetLastError();
}

}  // namespace

int group_splits(int dtype, int G, int64_t rows, int n, int k) {
  (void)dtype;
  // pieces of a group's rows until about two workgroups per CU have a tile each, of 128 rows or more on average
  const int64_t tiles = (int64_t)((n + 63) / 64) * ((k + 63) / 64) * G;
  const int64_t want = (512 + tiles - 1) / tiles, most = rows / ((int64_t)128 * G);
  return (int)(want < most ? want : most > 1 ? most : 1);
}

hipError_t launch_group(int dtype, int mode, const GroupArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? launch_any<bf16_t>(mode, a, s) : launch_any<float>(mode, a, s);
}

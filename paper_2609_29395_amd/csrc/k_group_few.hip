// Forward products of few rows grouped by cluster (gfx950): serving a row or
// so of every cluster, where the time is that of reading the weights.
//
// A workgroup gives 16 rows x 16 columns of the result.  Its four waves share
// the sum: each streams its quarter of the 16 weight rows from memory to
// registers, 16 bytes a lane and eight loads ahead, at any alignment, and
// multiplies them by the activations with MFMAs (which need no LDS and cost
// nothing beside the loads); the four partial sums meet in LDS.  fp32 takes the
// fp32 MFMA.
#include "group.h"

namespace {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int TILE = 16, AHEAD = 8;

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

template <typename T>
__global__ void __launch_bounds__(256) group_few_kernel(GroupArgs a, int NT) {
  using F = Few<T>;
  __shared__ f32x4_t part[4][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int li = lane & 15, lg = lane >> 4;
  int g, row0, row1, nt;
  if (!tile_of<false>(a.off, a.G, a.M, TILE, NT, blockIdx.x, g, row0, row1, nt)) return;
  const int c0 = nt * TILE, Q = a.Q;
  // rows and columns outside are taken as the last ones inside, and not stored
  const T *w = (const T *)a.b + g * a.b_gs + (int64_t)min(c0 + li, a.N - 1) * a.ldb + lg * F::VEC;
  const T *x = (const T *)a.a + (int64_t)min(row0 + li, row1 - 1) * a.lda + lg * F::VEC;
  const int steps = Q / F::STEP;  // whole ones
  const int s0 = (int)((int64_t)steps * wave / 4), s1 = (int)((int64_t)steps * (wave + 1) / 4);
  f32x4_t acc[2] = {f32x4_t{0.f, 0.f, 0.f, 0.f}, f32x4_t{0.f, 0.f, 0.f, 0.f}};
  int s = s0;
  for (; s + AHEAD <= s1; s += AHEAD) {
    u32x4 vw[AHEAD], vx[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) vw[i] = *(const u32x4_any *)(w + (int64_t)(s + i) * F::STEP);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) vx[i] = *(const u32x4_any *)(x + (int64_t)(s + i) * F::STEP);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) F::mma(acc[i & 1], vw[i], vx[i]);
  }
  for (; s < s1; ++s) {
    const u32x4 vw = *(const u32x4_any *)(w + (int64_t)s * F::STEP), vx = *(const u32x4_any *)(x + (int64_t)s * F::STEP);
    F::mma(acc[0], vw, vx);
  }
  if (wave == 3 && steps * F::STEP < Q) {  // what is left: a vector past the end is the last whole one, shifted
    const int k = steps * F::STEP + lg * F::VEC, over = max(k + F::VEC - Q, 0);
    const u32x4 vw = *(const u32x4_any *)(w + steps * F::STEP - over), vx = *(const u32x4_any *)(x + steps * F::STEP - over);
    F::mma(acc[0], shift_down<T>(vw, min(over, F::VEC)), shift_down<T>(vx, min(over, F::VEC)));
  }
  part[wave][lane] = acc[0] + acc[1];
  __syncthreads();
  const int m = row0 + li, c = c0 + 4 * lg;
  if (wave == 0 && m < row1 && c < a.N)
    finish<T, GROUP_FWD>(a, g, m, c, (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]));
}

template <typename T> hipError_t run(const GroupArgs &a, hipStream_t s) {
  const int64_t NT = (a.N + TILE - 1) / TILE, blocks = tile_blocks(a.M, a.G, TILE, NT);
  if (blocks > INT32_MAX) return hipErrorInvalidConfiguration;
  hipLaunchKernelGGL(group_few_kernel<T>, dim3((uint32_t)blocks), dim3(256), 0, s, a, (int)NT);
  return hipGetLastError();
}

}  // namespace

// A vector at least in the operands' rows; at most four rows a group on average
// (or one tile of them), and few enough that all of them in one group would
// read its weights no more than 16 times.
bool group_few_ok(int dtype, const GroupArgs &a, int mode) {
  return mode == GROUP_FWD && a.Q >= (dtype == GCPSL_BF16 ? 8 : 4) &&
         a.M <= std::max(TILE, std::min(4 * a.G, 16 * TILE));
}

hipError_t launch_group_few(int dtype, const GroupArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(a, s) : run<float>(a, s);
}

// Label scores (gfx950): per row of logits the log probability of a label,
// the entropy, the log sum of exponentials and the most likely classes; and
// the logits' gradient.
#include "runtime.h"
#include "ops.h"

namespace {

// Order of the classes of a row: by value, then by the lower index.  A NaN is
// above every number, -0 equals 0.
__device__ __forceinline__ uint64_t order_key(float v, int i) {
  uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);
  if (v != v) b = 0x7f800001u;  // one above +inf
  b = b & 0x80000000u ? ~b : b | 0x80000000u;
  return (uint64_t)b << 32 | (uint32_t)~i;
}

template <typename F> __device__ __forceinline__ float block_reduce(float v, F f, float *buf) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
  __syncthreads();
  return f(f(buf[0], buf[1]), f(buf[2], buf[3]));
}

template <typename T>
__global__ void __launch_bounds__(256) score_kernel(ScoreArgs a) {
  __shared__ float buf[4];
  __shared__ uint64_t kbuf[4];
  const int64_t r = blockIdx.x;
  const T *z = (const T *)a.z + r * a.ldz;
  float m = -INFINITY;
  for (int i = threadIdx.x; i < a.L; i += 256) m = fmaxf(m, ElemT<T>::to_f(z[i]));
  m = block_reduce(m, [](float x, float y) { return fmaxf(x, y); }, buf);
  const float base = m == -INFINITY ? 0.f : m;
  float s = 0.f, t = 0.f;
  for (int i = threadIdx.x; i < a.L; i += 256) {
    const float d = ElemT<T>::to_f(z[i]) - base, e = expf(d);
    s += e;
    t += e * fmaxf(d, -1e4f);  // where e is 0, d may be infinite
  }
  const auto add = [](float x, float y) { return x + y; };
  s = block_reduce(s, add, buf);
  t = block_reduce(t, add, buf);
  const bool empty = m == -INFINITY && s == 0.f;  // every class is ruled out
  const float ls = logf(s), lse = empty ? -INFINITY : base + ls;
  if (threadIdx.x == 0) {
    if (a.lse) a.lse[r] = lse;
    if (a.entropy) a.entropy[r] = empty ? 0.f : ls - t / s;
    if (a.logp) {
      const int y = a.labels[r];
      a.logp[r] = (unsigned)y >= (unsigned)a.L ? 0.f : empty ? -INFINITY : (ElemT<T>::to_f(z[y]) - base) - ls;
    }
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t best = 0;
    for (int i = threadIdx.x; i < a.L; i += 256) {
      const uint64_t key = order_key(ElemT<T>::to_f(z[i]), i);
      if (key < last && key > best) best = key;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, d, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) kbuf[threadIdx.x >> 6] = best;
    __syncthreads();
    last = max(max(kbuf[0], kbuf[1]), max(kbuf[2], kbuf[3]));
    if (threadIdx.x == 0) {
      const int i = (int)~(uint32_t)last;
      a.top_class[r * a.top + k] = i;
      a.top_logp[r * a.top + k] = empty ? -INFINITY : (ElemT<T>::to_f(z[i]) - base) - ls;
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(256) score_grad_kernel(ScoreGradArgs a) {
  const int64_t r = blockIdx.x;
  const T *z = (const T *)a.z + r * a.ldz;
  T *dz = (T *)a.dz + r * a.lddz;
  const float lse = a.lse[r];
  const int y = a.g_logp ? a.labels[r] : -1;
  const float gl = (unsigned)y < (unsigned)a.L ? a.g_logp[r] : 0.f;
  const float gh = a.g_entropy ? a.g_entropy[r] : 0.f, H = a.g_entropy ? a.entropy[r] : 0.f;
  for (int i = threadIdx.x; i < a.L; i += 256) {
    float d = 0.f;
    if (!(lse < -1e30f)) {
      const float lp = ElemT<T>::to_f(z[i]) - lse, p = expf(lp);
      d = (i == y ? gl : 0.f) - gl * p - gh * p * (fmaxf(lp, -1e4f) + H);
    }
    dz[i] = ElemT<T>::from_f(d);
  }
}

}  // namespace

size_t score_work_bytes(int, int64_t, int, int) { return 0; }

hipError_t launch_score(int dtype, const ScoreArgs &a, hipStream_t s) {
  if (dtype == GCPSL_BF16) hipLaunchKernelGGL(score_kernel<bf16_t>, dim3((uint32_t)a.rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(score_kernel<float>, dim3((uint32_t)a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_score_grad(int dtype, const ScoreGradArgs &a, hipStream_t s) {
  if (dtype == GCPSL_BF16) hipLaunchKernelGGL(score_grad_kernel<bf16_t>, dim3((uint32_t)a.rows), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(score_grad_kernel<float>, dim3((uint32_t)a.rows), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Label scores (gfx950): per row of logits the log probability of a label,
// the entropy, the log sum of exponentials and the most likely classes; and
// the logits' gradient.
//
// Scores are one pass over the logits.  A row is cut into chunks that a group
// of threads holds in registers (16-byte loads at any alignment); each chunk
// gives its maximum m, s = sum e^d and t = sum e^d d, d = x - m, and its `top`
// largest classes.  A row of one chunk is done then; the chunks of a longer
// row are joined by a second kernel from 16 + 8 top bytes each.
//
// Top classes of a chunk: the top-th largest of a wave's 64 lane maxima (found
// on the upper 16 bits of its order, bit by bit, by ballots) is a lower bound
// of the chunk's top-th largest value, as each of those lanes has an element
// at least as large.  The few elements that reach the largest wave's bound go
// to a list in LDS and every one counts how many are above it.  Where the list
// overflows (many equal values) or the chunk holds a NaN or infinity, the top
// classes are taken one at a time by a maximum over the chunk.
//
// Bound: reading the logits.  4,096 rows of 131,072 classes, bf16, top 8: 203 to
// 208 us (5.2 TB/s; reads alone reach 6.2).  One row of as many, top 20: 6 + 4.4
// us in two kernels, launches and latency.  The gradient reads and writes once:
// 4,096 x 50,021, fp32, 298 us (5.5 TB/s), bf16 143 (5.7).  Its short rows are
// bound by workgroups, one or more a row: 65,536 x 10, fp32, 49 us, bf16 43.
#include <algorithm>

#include "runtime.h"
#include "ops.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // global memory takes 16-byte accesses at any alignment

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float log_of(float s) { return __builtin_amdgcn_logf(s) * kLn2; }
constexpr float kNear = 1048576.f;  // 2^20: maxima up to which differences come from products with log2e
constexpr float kFar = -1e4f;  // e^kFar is 0: stands for any smaller difference where that is multiplied by e^d = 0

// Largest of three values; a NaN may or may not show.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}

template <typename T> struct Bits;  // the elements of a 16-byte vector
template <> struct Bits<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ float at(const u32x4 &w, int j) { return __uint_as_float(w[j]); }
  static __device__ __forceinline__ void drop_first(u32x4 &w, int n) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (j < n) w[j] = 0xff800000u;  // -inf
  }
};
template <> struct Bits<bf16_t> {
  static constexpr int VEC = 8;
  static __device__ __forceinline__ float at(const u32x4 &w, int j) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
  static __device__ __forceinline__ void drop_first(u32x4 &w, int n) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) w[j >> 1] = j & 1 ? (w[j >> 1] & 0xffffu) | 0xff800000u : (w[j >> 1] & 0xffff0000u) | 0xff80u;
  }
};

// Order of the classes of a row: by value, then by the lower index.  A NaN is
// above every number, -0 equals 0.  0 is below every class.
__device__ __forceinline__ uint32_t order_of(float v) {
  uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);
  if (v != v) b = 0x7f800001u;  // one above +inf
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) {
  return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t key_of(float v, int i) { return (uint64_t)order_of(v) << 32 | (uint32_t)~i; }

template <typename F> __device__ __forceinline__ float wave_all(float v, F f) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = f(v, __shfl_xor(v, d, 64));
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_all(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
  return wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ uint64_t wave_max(uint64_t v) {
#pragma unroll
  for (int d = 32; d; d >>= 1) v = max(v, (uint64_t)__shfl_xor((unsigned long long)v, d, 64));
  return v;
}
// Largest key of the group of TPR threads (256: the workgroup, all of which calls it).
template <int TPR> __device__ __forceinline__ uint64_t group_max(uint64_t v, uint64_t *buf) {
  v = wave_max(v);
  if constexpr (TPR == 256) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = max(max(buf[0], buf[1]), max(buf[2], buf[3]));
  }
  return v;
}

// The largest bound, on the upper 16 bits of an order, that at least n lanes
// reach (n <= 64).
__device__ __forceinline__ uint32_t bound_of(uint32_t order, int n) {
  uint32_t at = 0;
#pragma unroll
  for (int bit = 15; bit >= 0; --bit) {
    const uint32_t next = at | 1u << bit;
    if (__popcll(__ballot((order >> 16) >= next)) >= n) at = next;
  }
  return at << 16;
}

// Sums of a set of logits: maximum, sum of e^d, sum of e^d d.
struct Sums {
  float m, s, t;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// The sums as those below the maximum m instead of their own.
__device__ __forceinline__ void rebase(Sums &p, float m) {
  const float d = fmaxf(p.m - base_of(m), kFar), f = exp_of(d);
  p.t = f * (p.t + p.s * d);
  p.s *= f;
  p.m = m;
}

// A row's results from its sums; rows without a class left are -inf or 0
// throughout, those with a NaN or +inf NaN.
struct RowScore {
  float base, ls, lse, entropy;
  bool empty;
  __device__ __forceinline__ explicit RowScore(const Sums &p) {
    empty = p.s == 0.f;
    base = base_of(p.m);
    ls = p.s < INFINITY ? log_of(p.s) : NAN;
    lse = empty ? -INFINITY : base + ls;
    entropy = empty ? 0.f : ls - p.t / p.s;
  }
  __device__ __forceinline__ float logp(float x) const { return empty ? -INFINITY : (x - base) - ls; }
};
template <typename T>
__device__ __forceinline__ void write_row(const ScoreArgs &a, int64_t row, const RowScore &r) {
  if (a.lse) a.lse[row] = r.lse;
  if (a.entropy) a.entropy[row] = r.entropy;
  if (a.logp) {
    const int y = a.labels[row];
    a.logp[row] = (unsigned)y < (unsigned)a.L ? r.logp(ElemT<T>::to_f(((const T *)a.z)[row * a.ldz + y])) : 0.f;
  }
}
__device__ __forceinline__ void write_top(const ScoreArgs &a, int64_t row, int k, uint64_t key, const RowScore &r) {
  a.top_class[row * a.top + k] = (int)~(uint32_t)key;
  a.top_logp[row * a.top + k] = r.logp(value_of((uint32_t)(key >> 32)));
}

// Workspace of a row of several chunks: its chunks' sums, then their top keys.
__device__ __forceinline__ float4 *part_sums(const ScoreArgs &a, int64_t row, int chunks) {
  return (float4 *)a.work + row * chunks;
}
__device__ __forceinline__ uint64_t *part_keys(const ScoreArgs &a, int64_t row, int chunks) {
  return (uint64_t *)((float4 *)a.work + a.rows * chunks) + row * chunks * a.top;
}

// TPR threads (64 or 256) hold a chunk of TPR * NV 16-byte vectors.
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(256, 4) score_kernel(ScoreArgs a, uint32_t jobs, FastDiv fd_chunks) {
  using B = Bits<T>;
  constexpr int VEC = B::VEC, GROUPS = 256 / TPR, WAVES = TPR / 64;
  constexpr int VCAP = 128 * (TPR == 256 ? 2 : 1), CAP = VCAP;  // room for vectors and for keys
  __shared__ float4 wsum[4];
  __shared__ u32x4 vlist_[GROUPS * VCAP];
  __shared__ uint64_t list_[GROUPS * CAP], buf[4];
  __shared__ int vindex_[GROUPS * VCAP], count_[2 * GROUPS];
  const int t = threadIdx.x % TPR, wave = threadIdx.x >> 6;
  const int grp = TPR == 256 ? 0 : __builtin_amdgcn_readfirstlane(wave);
  u32x4 *vlist = vlist_ + grp * VCAP;
  int *vindex = vindex_ + grp * VCAP, *count = count_ + 2 * grp;
  uint64_t *list = list_ + grp * CAP;
  const int chunks = (int)fd_chunks.d;
  const uint32_t job = blockIdx.x * GROUPS + grp;
  const bool live = job < jobs;
  const int64_t row = live ? fdiv(job, fd_chunks) : 0;
  const int c = live ? (int)(job - (uint32_t)row * fd_chunks.d) : 0;
  const T *z = (const T *)a.z + row * a.ldz;
  const int L = a.L, i0 = (c * NV * TPR + t) * VEC;

  // Vector v starts at element i0 + v TPR VEC.  One that passes the row's end
  // is the row's last one instead, without what it shares with the vectors
  // before it.
  u32x4 w[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) w[v] = *(const u32x4_any *)(z + min(i0 + v * TPR * VEC, L - VEC));
  if ((c + 1) * NV * TPR * VEC > L) {
#pragma unroll
    for (int v = 0; v < NV; ++v) B::drop_first(w[v], i0 + v * TPR * VEC + VEC - L);
  }
  float vmax[NV], lmax = -INFINITY;
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    vmax[v] = -INFINITY;
#pragma unroll
    for (int j = 0; j < VEC; j += 2) vmax[v] = max3(vmax[v], B::at(w[v], j), B::at(w[v], j + 1));
    lmax = fmaxf(lmax, vmax[v]);
  }
  // In units of log 2, d = x log2e - base log2e with the second product
  // rounded: what that rounding is off by (`off`) is the same for every
  // element and is taken out of the sums.  It is at most 2^-24 of the product,
  // below 0.1 up to kNear; further out, from 10^9 on, 2^off would pass fp32's
  // range.  (`base` is that of the wave: of a finite fill, where its classes
  // are all ruled out.)
  Sums p{wave_max(lmax), 0.f, 0.f};
  const float base = base_of(p.m), prod = base * kLog2e, off = fmaf(base, kLog2e, -prod);
  float s2[2] = {0.f, 0.f}, t2[2] = {0.f, 0.f};
#pragma unroll
  for (int v = 0; v < NV; ++v)
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float d = fmaf(B::at(w[v], j), kLog2e, -prod), e = __builtin_amdgcn_exp2f(d);
      s2[j & 1] += e;
      t2[j & 1] = fmaf(e, fmaxf(d, kFar), t2[j & 1]);
    }
  const float f = __builtin_amdgcn_exp2f(-off);
  p.s = wave_sum(s2[0] + s2[1]);
  p.t = kLn2 * f * fmaf(-off, p.s, wave_sum(t2[0] + t2[1]));
  p.s *= f;
  if (fabsf(base) > kNear) {  // the difference first, which is exact near the maximum
    p.s = p.t = 0.f;
    for (int k = 0; k < NV * VEC; ++k) {  // the thread's own elements, again from memory
      const int i = i0 + k / VEC * TPR * VEC + k % VEC;
      if (i >= L) break;
      const float d = ElemT<T>::to_f(z[i]) - base, e = exp_of(d);
      p.s += e;
      p.t = fmaf(e, fmaxf(d, kFar), p.t);
    }
    p.s = wave_sum(p.s);
    p.t = wave_sum(p.t);
  }

  float bound = -INFINITY;
  if (a.top) {
    const uint32_t at = bound_of(order_of(lmax), a.top);
    if (at > order_of(-INFINITY)) bound = value_of(at);
  }
  if (t == 0) count[0] = count[1] = 0;
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0) wsum[wave] = make_float4(p.m, p.s, p.t, bound);
    __syncthreads();
    Sums q[4];
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      q[i] = Sums{wsum[i].x, wsum[i].y, wsum[i].z};
      m = fmaxf(m, q[i].m);
      bound = fmaxf(bound, wsum[i].w);
    }
    p = Sums{m, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      rebase(q[i], m);
      p.s += q[i].s;
      p.t += q[i].t;
    }
  } else {
    __syncthreads();
  }
  const RowScore r(p);
  if (t == 0 && live) {
    if (chunks > 1) part_sums(a, row, chunks)[c] = make_float4(p.m, p.s, p.t, 0.f);
    else write_row<T>(a, row, r);
  }
  if (a.top == 0) return;

  // the vectors that reach the bound, then their elements that do
  uint64_t *keys = part_keys(a, row, chunks) + (int64_t)c * a.top;
  if (lmax >= bound) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (vmax[v] >= bound) {
        const int n = atomicAdd(count, 1);
        if (n < VCAP) {
          vlist[n] = w[v];
          vindex[n] = i0 + v * TPR * VEC;
        }
      }
  }
  __syncthreads();
  const int nv = __builtin_amdgcn_readfirstlane(count[0]);
  if (nv <= VCAP)
    for (int e = t; e < nv * VEC; e += TPR) {
      const int i = vindex[e / VEC], k = min(i, L - VEC) + e % VEC;  // below i: not the vector's own
      const float x = ElemT<T>::to_f(((const T *)vlist)[e]);
      if (x >= bound && k >= i) {
        const int n = atomicAdd(count + 1, 1);
        if (n < CAP) list[n] = key_of(x, k);
      }
    }
  __syncthreads();
  const int n = __builtin_amdgcn_readfirstlane(count[1]);
  if (nv <= VCAP && n <= CAP && p.s < INFINITY) {
    for (int i = t; i < n; i += TPR) {
      const uint64_t key = list[i];
      int above = 0;
      for (int j = 0; j < n; ++j) above += list[j] > key;
      if (above < a.top && live) {
        if (chunks > 1) keys[above] = key;
        else write_top(a, row, above, key, r);
      }
    }
    // a chunk of fewer classes
    if (chunks > 1 && live && t < a.top && t >= n) keys[t] = 0;
    return;
  }
  const int c1 = min(L, (c + 1) * NV * TPR * VEC);
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t best = 0;
    for (int i = c * NV * TPR * VEC + t; i < c1; i += TPR) {
      const uint64_t key = key_of(ElemT<T>::to_f(z[i]), i);
      if (key < last && key > best) best = key;
    }
    last = group_max<TPR>(best, buf);
    if (t == 0 && live) {
      if (chunks > 1) keys[k] = last;
      else write_top(a, row, k, last, r);
    }
  }
}

// A row of several chunks from their sums and top keys, at most 1,024 of them:
// a wave a row holds the keys in registers and takes the top classes as the
// chunks' kernel does (a maximum over all keys for each class cost 0.7 us a
// class: 15 us for 20).
constexpr int kHeld = 16, kCandidates = 128;
template <typename T>
__global__ void __launch_bounds__(256) score_join_kernel(ScoreArgs a, int chunks) {
  __shared__ uint64_t list_[4 * kCandidates];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint64_t *list = list_ + wave * kCandidates;
  const int64_t row = (int64_t)blockIdx.x * 4 + wave;
  if (row >= a.rows) return;
  const float4 *sums = part_sums(a, row, chunks);
  const uint64_t *keys = part_keys(a, row, chunks);
  const int n = chunks * a.top;
  uint64_t held[kHeld], best = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) held[i] = lane + i * 64 < n ? keys[lane + i * 64] : 0;
  float m = -INFINITY;
  for (int c = lane; c < chunks; c += 64) m = fmaxf(m, sums[c].x);
  Sums p{wave_max(m), 0.f, 0.f};
  for (int c = lane; c < chunks; c += 64) {
    Sums q{sums[c].x, sums[c].y, sums[c].z};
    rebase(q, p.m);
    p.s += q.s;
    p.t += q.t;
  }
  p.s = wave_sum(p.s);
  p.t = wave_sum(p.t);
  const RowScore r(p);
  if (lane == 0) write_row<T>(a, row, r);
  if (a.top == 0) return;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) best = max(best, held[i]);
  const uint64_t bound = max((uint64_t)bound_of((uint32_t)(best >> 32), a.top) << 32, (uint64_t)1);
  int count = 0;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const bool in = held[i] >= bound;
    const uint64_t lanes = __ballot(in);
    if (in) {
      const int at = count + __popcll(lanes & ((1ull << lane) - 1));
      if (at < kCandidates) list[at] = held[i];
    }
    count += __popcll(lanes);
  }
  if (count <= kCandidates) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int i = lane; i < count; i += 64) {
      const uint64_t key = list[i];
      int above = 0;
      for (int j = 0; j < count; ++j) above += list[j] > key;
      if (above < a.top) write_top(a, row, above, key, r);
    }
    return;
  }
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    best = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i)
      if (held[i] < last && held[i] > best) best = held[i];
    last = wave_max(best);
    if (lane == 0) write_top(a, row, k, last, r);
  }
}

// The same for more keys, a workgroup a row, one class at a time.
template <typename T>
__global__ void __launch_bounds__(256) score_join_many_kernel(ScoreArgs a, int chunks) {
  __shared__ float4 wsum[4];
  __shared__ uint64_t buf[4];
  const int64_t row = blockIdx.x;
  const int t = threadIdx.x;
  const float4 *sums = part_sums(a, row, chunks);
  const uint64_t *keys = part_keys(a, row, chunks);
  const int64_t n = (int64_t)chunks * a.top;
  float m = -INFINITY;
  for (int c = t; c < chunks; c += 256) m = fmaxf(m, sums[c].x);
  m = wave_max(m);
  Sums p{m, 0.f, 0.f};
  for (int c = t; c < chunks; c += 256) {
    Sums q{sums[c].x, sums[c].y, sums[c].z};
    rebase(q, m);
    p.s += q.s;
    p.t += q.t;
  }
  p.s = wave_sum(p.s);
  p.t = wave_sum(p.t);
  if ((t & 63) == 0) wsum[t >> 6] = make_float4(p.m, p.s, p.t, 0.f);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i) m = fmaxf(m, wsum[i].x);
  p = Sums{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Sums q{wsum[i].x, wsum[i].y, wsum[i].z};
    rebase(q, m);
    p.s += q.s;
    p.t += q.t;
  }
  const RowScore r(p);
  if (t == 0) write_row<T>(a, row, r);
  uint64_t last = ~0ull;
  for (int k = 0; k < a.top; ++k) {
    uint64_t best = 0;
    for (int64_t i = t; i < n; i += 256)
      if (keys[i] < last && keys[i] > best) best = keys[i];
    last = group_max<256>(best, buf);
    if (t == 0) write_top(a, row, k, last, r);
  }
}

// Rows of at most 64 classes: 16 lanes a row, every class counts those above
// it.
template <typename T>
__global__ void __launch_bounds__(256) score_small_kernel(ScoreArgs a) {
  const int lane = threadIdx.x & 15;
  const int64_t job = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const bool live = job < a.rows;
  const int64_t row = live ? job : 0;
  const T *z = (const T *)a.z + row * a.ldz;
  const int n = (a.L + 15) >> 4;
  float x[4], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = i * 16 + lane < a.L ? ElemT<T>::to_f(z[i * 16 + lane]) : -INFINITY;
    m = fmaxf(m, x[i]);
  }
#pragma unroll
  for (int d = 8; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 16));
  Sums p{m, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float d = x[i] - base_of(m), e = exp_of(d);
    p.s += e;
    p.t = fmaf(e, fmaxf(d, kFar), p.t);
  }
#pragma unroll
  for (int d = 8; d; d >>= 1) {
    p.s += __shfl_xor(p.s, d, 16);
    p.t += __shfl_xor(p.t, d, 16);
  }
  const RowScore r(p);
  if (lane == 0 && live) write_row<T>(a, row, r);
  if (a.top == 0) return;
  uint64_t key[4];
  int above[4] = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i) key[i] = i * 16 + lane < a.L ? key_of(x[i], i * 16 + lane) : 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n)
      for (int l = 0; l < 16; ++l) {
        const uint64_t other = __shfl((unsigned long long)key[i], l, 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) above[j] += other > key[j];
      }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (live && i * 16 + lane < a.L && above[i] < a.top) write_top(a, row, above[i], key[i], r);
}

// A row's lse from which on its classes count as ruled out: -2^23, where fp32's
// steps are 1 and lse no longer holds the logarithm of how many share it, so that
// z - lse would make e^0 of every class.
constexpr float kRuledOut = -8388608.f;

// dz: NV 16-byte vectors a thread, chunks of 256 NV vectors of a row.
template <typename T, int NV>
__global__ void __launch_bounds__(256) score_grad_kernel(ScoreGradArgs a, FastDiv fd_chunks) {
  using B = Bits<T>;
  constexpr int VEC = B::VEC;
  const int64_t row = fdiv(blockIdx.x, fd_chunks);
  const int c = (int)(blockIdx.x - (uint32_t)row * fd_chunks.d), L = a.L;
  const T *z = (const T *)a.z + row * a.ldz;
  T *dz = (T *)a.dz + row * a.lddz;
  const int i0 = (c * NV * 256 + (int)threadIdx.x) * VEC;
  u32x4 w[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int i = i0 + v * 256 * VEC;
    w[v] = u32x4{0, 0, 0, 0};
    if (i + VEC <= L) w[v] = *(const u32x4_any *)(z + i);
  }
  const float lse = a.lse[row];
  const int y = a.g_logp ? a.labels[row] : -1;
  const float gl = (unsigned)y < (unsigned)L ? a.g_logp[row] : 0.f;
  const float gh = a.g_entropy ? a.g_entropy[row] : 0.f, H = a.g_entropy ? a.entropy[row] : 0.f;
  const bool empty = lse <= kRuledOut;
  const float g0 = -gl - gh * H;  // dz = p (g0 - gh log p) off the label
  const auto grad = [&](float x, int i) {
    if (empty) return 0.f;
    const float lp = x - lse, p = exp_of(lp);
    const float d = p * fmaf(-gh, fmaxf(lp, kFar), g0);
    return i == y ? d + gl : d;
  };
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int i = i0 + v * 256 * VEC;
    if (i + VEC <= L) {
      u32x4 o;
      if constexpr (VEC == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __float_as_uint(grad(B::at(w[v], j), i + j));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          o[j] = pack2_bf16(grad(B::at(w[v], 2 * j), i + 2 * j), grad(B::at(w[v], 2 * j + 1), i + 2 * j + 1));
      }
      *(u32x4_any *)(dz + i) = o;
    } else {
      for (int k = i; k < L; ++k) dz[k] = ElemT<T>::from_f(grad(ElemT<T>::to_f(z[k]), k));
    }
  }
}

// Chunks of a long row: as much as a workgroup holds in registers (16,384
// classes), or a quarter (bf16) or eighth (fp32) of it where the rows are too
// few to give every CU two such chunks.  But a row that one large chunk holds
// is not cut: 1 row of 6,058 classes of bf16 takes 5.5 us so, and 8.0 as two
// small chunks and their join.  Nor is one whose small chunks' keys are more
// than a wave holds for the join: 1 row of 600,000, top 8, 9.7 against 15.0
// us; below that small chunks are faster, 7.9 against 9.1 us for 17,000.
struct Chunks {
  bool large;
  int64_t n;  // of a row
};
template <typename T> constexpr int kLargeNV = sizeof(T) == 2 ? 8 : 16;
constexpr int kSmallNV = 2;
template <typename T> Chunks chunks_of(int64_t rows, int L, int top) {
  constexpr int64_t per = 256 * Bits<T>::VEC;
  const int64_t large = (L + per * kLargeNV<T> - 1) / (per * kLargeNV<T>);
  const int64_t small = (L + per * kSmallNV - 1) / (per * kSmallNV);
  if (rows * large >= 512 || (large == 1 && small > 1) || small * top > 64 * kHeld) return {true, large};
  return {false, small};
}
// Rows that one wave each takes: those it holds in 4 vectors a lane, and in 8
// where there are rows enough for all SIMDs: us so and by four waves a row, 4,096
// rows of 4,096 classes, bf16, 10.0 and 13.8, of 2,048, fp32, 8.1 and 12.6; 1,024
// rows 6.5 and 6.3, 5.8 and 6.0.
template <typename T> bool wave_rows(int64_t rows, int L) {
  return L <= 64 * (rows >= 1024 ? 8 : 4) * Bits<T>::VEC;
}

template <typename T> size_t work_of(int64_t rows, int L, int top) {
  if (wave_rows<T>(rows, L)) return 0;
  const int64_t n = chunks_of<T>(rows, L, top).n;
  return n > 1 ? (size_t)rows * n * (16 + 8 * (size_t)top) : 0;
}

// Rows of one launch; `wave` and `ch` are chosen by all the rows of the call.
template <typename T> hipError_t run_rows(const ScoreArgs &a, bool wave, const Chunks &ch, hipStream_t s) {
  if (a.L <= 64) {
    hipLaunchKernelGGL(score_small_kernel<T>, dim3((uint32_t)((a.rows + 15) / 16)), dim3(256), 0, s, a);
    return hipGetLastError();
  }
  const uint32_t n = (uint32_t)(a.rows * ch.n);
  const auto launch = [&](auto kernel, uint32_t groups) {
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(256), 0, s, a, n, make_fastdiv((uint32_t)ch.n));
  };
  // a row that is not cut: as many vectors a thread as it needs (the most, always:
  // 4,096 rows of 3,000 classes, fp32, 28 us where 15 do, of 100, bf16, 7.6 and 6.0)
  const int vectors = (a.L + Bits<T>::VEC - 1) / Bits<T>::VEC;
  if (wave) {
    if (vectors <= 64) launch(score_kernel<T, 64, 1>, (n + 3) / 4);
    else if (vectors <= 128) launch(score_kernel<T, 64, 2>, (n + 3) / 4);
    else if (vectors <= 256) launch(score_kernel<T, 64, 4>, (n + 3) / 4);
    else launch(score_kernel<T, 64, 8>, (n + 3) / 4);
  } else if (ch.n > 1 ? !ch.large : vectors <= 256 * kSmallNV) {
    launch(score_kernel<T, 256, kSmallNV>, n);
  } else if (ch.n == 1 && vectors <= 1024) {
    launch(score_kernel<T, 256, 4>, n);
  } else if (ch.n == 1 && vectors <= 2048) {
    launch(score_kernel<T, 256, 8>, n);
  } else {
    launch(score_kernel<T, 256, kLargeNV<T>>, n);
  }
  if (ch.n > 1 && ch.n * a.top <= 64 * kHeld)
    hipLaunchKernelGGL(score_join_kernel<T>, dim3((uint32_t)((a.rows + 3) / 4)), dim3(256), 0, s, a, (int)ch.n);
  else if (ch.n > 1)
    hipLaunchKernelGGL(score_join_many_kernel<T>, dim3((uint32_t)a.rows), dim3(256), 0, s, a, (int)ch.n);
  return hipGetLastError();
}

// p's entry r, or null.
template <typename P> P *entry_at(P *p, int64_t r) { return p ? p + r : nullptr; }

template <typename T> hipError_t run(const ScoreArgs &a, hipStream_t s) {
  const bool wave = wave_rows<T>(a.rows, a.L);
  const Chunks ch = wave || a.L <= 64 ? Chunks{false, 1} : chunks_of<T>(a.rows, a.L, a.top);
  const int64_t slab = kMaxBlocks / ch.n;  // (launches of less than a workgroup a row would hold more)
  for (int64_t r = 0; r < a.rows; r += slab) {
    ScoreArgs b = a;
    b.z = (const T *)a.z + r * a.ldz;
    b.rows = std::min(slab, a.rows - r);
    b.labels = entry_at(a.labels, r);
    b.logp = entry_at(a.logp, r);
    b.entropy = entry_at(a.entropy, r);
    b.lse = entry_at(a.lse, r);
    b.top_logp = entry_at(a.top_logp, r * a.top);
    b.top_class = entry_at(a.top_class, r * a.top);
    const hipError_t e = run_rows<T>(b, wave, ch, s);  // (one after another on the stream: the workspace serves each)
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T> hipError_t run_grad(const ScoreGradArgs &a, hipStream_t s) {
  constexpr int NV = 4;
  const int64_t per = 256 * NV * Bits<T>::VEC, n = (a.L + per - 1) / per, slab = kMaxBlocks / n;
  for (int64_t r = 0; r < a.rows; r += slab) {
    ScoreGradArgs b = a;
    b.z = (const T *)a.z + r * a.ldz;
    b.rows = std::min(slab, a.rows - r);
    b.labels = entry_at(a.labels, r);
    b.lse = a.lse + r;
    b.entropy = entry_at(a.entropy, r);
    b.g_logp = entry_at(a.g_logp, r);
    b.g_entropy = entry_at(a.g_entropy, r);
    b.dz = (T *)a.dz + r * a.lddz;
    hipLaunchKernelGGL((score_grad_kernel<T, NV>), dim3((uint32_t)(b.rows * n)), dim3(256), 0, s, b,
                       make_fastdiv((uint32_t)n));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

size_t score_work_bytes(int dtype, int64_t rows, int L, int top) {
  return dtype == GCPSL_BF16 ? work_of<bf16_t>(rows, L, top) : work_of<float>(rows, L, top);
}

hipError_t launch_score(int dtype, const ScoreArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(a, s) : run<float>(a, s);
}

hipError_t launch_score_grad(int dtype, const ScoreGradArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run_grad<bf16_t>(a, s) : run_grad<float>(a, s);
}

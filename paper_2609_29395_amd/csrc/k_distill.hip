// Distillation of rows of logits from a teacher's best classes (gfx950): the
// divergence beside the label's log probability, and the logits' gradient.
//
//   kl = sum_k q_k (log q_k - log p_k),  q = softmax(v / T),  p = softmax(z / T)
//   dz = g_kl (p - q) / T + g_logp (1[c = y] - softmax(z))
//
// Forward, one pass over the logits: every thread keeps a running maximum m of its
// own and the sums of e^((z - m) / T) and, where both are asked for, e^(z - m), and
// brings them to a larger maximum once for a batch of 16-byte vectors.  A row is a
// workgroup's, or a wave's where it is short; where the rows are fewer than the
// chip holds workgroups, each is cut into parts that a second kernel joins.  With
// w_k = e^((v_k - max v) / T) and W their sum, kl = sum_k w_k (log w_k - log p_k) / W
// - log W, from `top` logits of the row.
//
// Gradient: the dense terms go over the part; then, behind a barrier, the
// teacher's classes in it are written again with their q_k, which all entries of a
// class sum in the same order (no atomics: the same bits always).
//
// Bound: memory.  bf16, 4,096 rows: 131,072 classes at T = 2 190 us forward (5.6
// TB/s), 355 the gradient (6.0, where a copy reaches 5.0); 50,021 classes 76 and 152
// (5.4 both).  Short rows by their latency, the teacher's entries and their logits
// being loads after loads: 65,536 rows of 1,000 classes 43 and 68 us.  One row of
// 131,072 classes 7 and 6 us.
#include <algorithm>
#include <type_traits>

#include "ops.h"
#include "runtime.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));  // global memory takes 16-byte accesses at any alignment
template <int N> using Count = std::integral_constant<int, N>;

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.693147180559945309417f;
__device__ __forceinline__ float exp_of(float d) { return __builtin_amdgcn_exp2f(d * kLog2e); }
__device__ __forceinline__ float log_of(float s) { return __builtin_amdgcn_logf(s) * kLn2; }
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

// An lse from which on a row's classes count as ruled out, as for the score gradient.
constexpr float kRuledOut = -8388608.f;

template <typename T> struct Bits;  // the elements of a 16-byte vector
template <> struct Bits<float> {
  static constexpr int VEC = 4;
  static __device__ __forceinline__ float at(const u32x4 &w, int j) { return __uint_as_float(w[j]); }
  static __device__ __forceinline__ u32x4 none() { return u32x4{0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u}; }  // -inf
};
template <> struct Bits<bf16_t> {
  static constexpr int VEC = 8;
  static __device__ __forceinline__ float at(const u32x4 &w, int j) {
    return __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
  }
  static __device__ __forceinline__ u32x4 none() { return u32x4{0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u}; }
};

// A part of a row: vectors [v0, v1) of those that lie on 16-byte boundaries of
// `base` and, the first part, the row's classes before and behind them, one by one.
// (Vectors from the row's first class on, at odd addresses: 4,096 rows of 50,021
// classes, bf16, 93 and 195 us where 78 and 180 do.)
template <typename T> struct Part {
  static constexpr int VEC = Bits<T>::VEC;
  int head, behind, L;  // classes before the vectors, the first behind them
  uint32_t v0, v1;
  bool ends;            // takes them
  __device__ __forceinline__ Part(const T *base, int L_, uint32_t part, uint32_t per) : L(L_) {
    const int past = (int)(reinterpret_cast<uintptr_t>(base) / sizeof(T)) & (VEC - 1);
    head = (VEC - past) & (VEC - 1);
    const uint32_t all = (uint32_t)(L - head) / VEC;  // (rows here have more than 64 classes)
    behind = head + (int)(all * VEC);
    v0 = min(part * per, all);
    v1 = min(v0 + per, all);
    ends = part == 0;
  }
  // Class of the t-th one by itself, -1 if there is none.
  __device__ __forceinline__ int single(int t) const {
    if (!ends) return -1;
    if (t < head) return t;
    const int c = behind + (t - head);
    return c < L ? c : -1;
  }
  __device__ __forceinline__ bool has(int c) const {
    if ((unsigned)c >= (unsigned)L) return false;
    if (c < head || c >= behind) return ends;
    const uint32_t v = (uint32_t)(c - head) / VEC;
    return v >= v0 && v < v1;
  }
};

// Over groups of W lanes (16 or 64).
template <int W> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int d = W / 2; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d, W));
  return v;
}
template <int W> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
  for (int d = W / 2; d; d >>= 1) v += __shfl_xor(v, d, W);
  return v;
}
// Over a row's TPR threads; buf [4], each used once.
template <int TPR> __device__ __forceinline__ float row_max(float v, float *buf) {
  v = lanes_max<TPR == 256 ? 64 : TPR>(v);
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = fmaxf(fmaxf(buf[0], buf[1]), fmaxf(buf[2], buf[3]));
  }
  return v;
}
template <int TPR> __device__ __forceinline__ float row_sum(float v, float *buf) {
  v = lanes_sum<TPR == 256 ? 64 : TPR>(v);
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (buf[0] + buf[1]) + (buf[2] + buf[3]);
  }
  return v;
}
template <int TPR> __device__ __forceinline__ void row_sync() {
  if constexpr (TPR == 256) __syncthreads();
  else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// Sums of a set of logits below its maximum m: of e^((z - m) / T), of e^(z - m).
struct Sums {
  float m, t, s;
};
__device__ __forceinline__ void rebase(Sums &p, float m, float inv_t) {
  const float d = p.m - base_of(m);  // (-inf or less where nothing was summed: t = s = 0)
  p.t *= exp_of(d * inv_t);
  p.s *= exp_of(d);
  p.m = m;
}
__device__ __forceinline__ void join(Sums &p, Sums q, float inv_t) {
  const float m = fmaxf(p.m, q.m);
  rebase(p, m, inv_t);
  rebase(q, m, inv_t);
  p.t += q.t;
  p.s += q.s;
}
template <int W> __device__ __forceinline__ void lanes_join(Sums &p, float inv_t) {
  rebase(p, lanes_max<W>(p.m), inv_t);
  p.t = lanes_sum<W>(p.t);
  p.s = lanes_sum<W>(p.s);
}

// Logarithms of a row's probabilities at one temperature; rows without a class
// left have -inf throughout, those with a NaN or +inf NaN.
struct RowLog {
  float base, ls, lse, inv;
  bool empty;
  __device__ __forceinline__ RowLog(float m, float s, float inv_) : inv(inv_) {
    empty = s == 0.f;
    base = base_of(m);
    ls = s < INFINITY ? log_of(s) : NAN;
    lse = empty ? -INFINITY : fmaf(base, inv, ls);
  }
  __device__ __forceinline__ float logp(float x) const { return empty ? -INFINITY : fmaf(x - base, inv, -ls); }
};

// What a row's results need beside its sums: the label's logit (lane 0), the lane's
// first entry and its class's logit, loaded before the row is read, as each takes
// a load after another.
template <typename T> struct RowEnds {
  int y, c;
  float label, v, x;
  __device__ __forceinline__ RowEnds(const DistillArgs &a, int64_t row, int t) : y(-1), c(-1), label(0.f), v(0.f), x(0.f) {
    const T *z = (const T *)a.z + row * a.ldz;
    if (a.logp && t == 0) y = a.labels[row];
    if (a.kl && t < a.top) entry(a, row, t, c, v, x);
    if ((unsigned)y < (unsigned)a.L) label = ElemT<T>::to_f(z[y]);
  }
  // entry k of the row; c -1 if it is left out
  static __device__ __forceinline__ void entry(const DistillArgs &a, int64_t row, int k, int &c, float &v, float &x) {
    c = a.t_class[row * a.top + k];
    v = a.t_value[row * a.top + k];
    if ((unsigned)c < (unsigned)a.L) x = ElemT<T>::to_f(((const T *)a.z)[row * a.ldz + c]);
    else c = -1;
  }
};

// Results of a row from its sums, by W lanes (this one is lane t).  a.temperature 1: the two sums are one.
template <typename T, int W>
__device__ __forceinline__ void write_row(const DistillArgs &a, int64_t row, const Sums &p, int t, const RowEnds<T> &ends) {
  const float inv_t = 1.f / a.temperature;
  const RowLog soft(p.m, p.t, inv_t);
  if (t == 0) {
    const RowLog plain(p.m, a.temperature == 1.f ? p.t : p.s, 1.f);
    if (a.lse_t) a.lse_t[row] = soft.lse;
    if (a.lse) a.lse[row] = plain.lse;
    if (a.logp) a.logp[row] = (unsigned)ends.y < (unsigned)a.L ? plain.logp(ends.label) : 0.f;
  }
  if (!a.kl) return;
  float best = ends.c >= 0 ? fmaxf(-INFINITY, ends.v) : -INFINITY;
  for (int k = t + W; k < a.top; k += W)
    if ((unsigned)a.t_class[row * a.top + k] < (unsigned)a.L) best = fmaxf(best, a.t_value[row * a.top + k]);
  best = base_of(lanes_max<W>(best));
  float sum = 0.f, part = 0.f;
  int c = ends.c;
  float v = ends.v, x = ends.x;
  for (int k = t; k < a.top; k += W) {
    if (k != t) RowEnds<T>::entry(a, row, k, c, v, x);
    if (c < 0) continue;
    const float d = (v - best) * inv_t, w = exp_of(d);
    if (w == 0.f) continue;  // (-inf, or so far below that its term is 0)
    sum += w;
    part = fmaf(w, d - soft.logp(x), part);
  }
  sum = lanes_sum<W>(sum);
  part = lanes_sum<W>(part);
  if (t == 0) a.kl[row] = sum == 0.f ? 0.f : part / sum - log_of(sum);
}

// f(N, whole, v) for a thread's vectors of [v0, v1): N of them from v + t on, TPR apart,
// four while all threads have as many, then as many as any has left (whole false).
template <int TPR, typename F> __device__ __forceinline__ void each_batch(uint32_t v0, uint32_t v1, F f) {
  uint32_t v = v0;
  for (; v + 4 * TPR <= v1; v += 4 * TPR) f(Count<4>{}, std::true_type{}, v);
  const uint32_t left = v1 - v;
  if (left > 3 * TPR) f(Count<4>{}, std::false_type{}, v);
  else if (left > 2 * TPR) f(Count<3>{}, std::false_type{}, v);
  else if (left > TPR) f(Count<2>{}, std::false_type{}, v);
  else if (left > 0) f(Count<1>{}, std::false_type{}, v);
}
// The row of this thread among those of its workgroup, in a scalar register where a wave has one.
template <int TPR> __device__ __forceinline__ int row_in_block() {
  const int i = (int)threadIdx.x / TPR;
  return TPR >= 64 ? __builtin_amdgcn_readfirstlane(i) : i;
}

// Part `job` % parts of row `job` / parts by TPR threads; a part is `per` vectors.  TWO: both sums.
template <typename T, int TPR, bool TWO>
__global__ void __launch_bounds__(256) distill_kernel(DistillArgs a, uint32_t jobs, FastDiv fd_parts, uint32_t per) {
  using B = Bits<T>;
  constexpr int VEC = B::VEC, GROUPS = 256 / TPR, LANES = TPR < 64 ? TPR : 64;
  __shared__ float4 wsum[4];
  const int t = threadIdx.x % TPR, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t job = blockIdx.x * GROUPS + row_in_block<TPR>();
  if (job >= jobs) return;  // (rows that share a workgroup share no barrier, those that share a wave no shuffle)
  const int64_t row = fdiv(job, fd_parts);
  const T *z = (const T *)a.z + row * a.ldz;
  const Part<T> part(z, a.L, job - (uint32_t)row * fd_parts.d, per);
  const T *vectors = z + part.head;
  const float inv_t = 1.f / a.temperature, ct = kLog2e * inv_t;
  Sums p{-INFINITY, 0.f, 0.f};
  const bool last = fd_parts.d == 1 && (TPR < 256 || wave == 0);  // writes the results
  const RowEnds<T> ends(a, row, last ? t : INT32_MAX);
  const int single = part.single(t);
  if (single >= 0) {
    const float x = ElemT<T>::to_f(z[single]);
    p.m = fmaxf(p.m, x);
    const float d = x - base_of(p.m);
    p.t = exp_of(d * inv_t);
    p.s = exp_of(d);
  }
  each_batch<TPR>(part.v0, part.v1, [&](auto count, auto whole, uint32_t v) {
    constexpr int N = decltype(count)::value;
    constexpr bool WHOLE = decltype(whole)::value;
    u32x4 w[N];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const uint32_t i = v + u * TPR + t;
      w[u] = *(const u32x4 *)(vectors + (WHOLE ? i : min(i, part.v1 - 1)) * VEC);
    }
    if (!WHOLE && v + (N - 1) * TPR + t >= part.v1) w[N - 1] = B::none();
    float m = p.m;
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int j = 0; j < VEC; ++j) m = fmaxf(m, B::at(w[u], j));
    rebase(p, m, inv_t);
    const float base = base_of(m);
    float t2[2] = {0.f, 0.f}, s2[2] = {0.f, 0.f};
#pragma unroll
    for (int u = 0; u < N; ++u)
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float d = B::at(w[u], j) - base;
        t2[j & 1] += __builtin_amdgcn_exp2f(d * ct);
        if (TWO) s2[j & 1] += __builtin_amdgcn_exp2f(d * kLog2e);
      }
    p.t += t2[0] + t2[1];
    p.s += s2[0] + s2[1];
  });
  lanes_join<LANES>(p, inv_t);
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0) wsum[wave] = make_float4(p.m, p.t, p.s, 0.f);
    __syncthreads();
    if (wave) return;
    p = Sums{wsum[0].x, wsum[0].y, wsum[0].z};
#pragma unroll
    for (int i = 1; i < 4; ++i) join(p, Sums{wsum[i].x, wsum[i].y, wsum[i].z}, inv_t);
  }
  if (fd_parts.d > 1) {
    if (t == 0) ((float4 *)a.work)[job] = make_float4(p.m, p.t, p.s, 0.f);
  } else {
    write_row<T, LANES>(a, row, p, t, ends);
  }
}

// Rows of several parts, a wave each.
template <typename T> __global__ void __launch_bounds__(256) distill_join_kernel(DistillArgs a, uint32_t parts) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row >= a.rows) return;
  const float inv_t = 1.f / a.temperature;
  const float4 *work = (const float4 *)a.work + row * parts;
  const RowEnds<T> ends(a, row, lane);
  Sums p{-INFINITY, 0.f, 0.f};
  for (uint32_t i = lane; i < parts; i += 64) join(p, Sums{work[i].x, work[i].y, work[i].z}, inv_t);
  lanes_join<64>(p, inv_t);
  write_row<T, 64>(a, row, p, lane, ends);
}

// Rows of at most 64 classes: 16 lanes a row.
template <typename T> __global__ void __launch_bounds__(256) distill_small_kernel(DistillArgs a) {
  const int lane = threadIdx.x & 15;
  const int64_t job = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (job >= a.rows) return;  // (shuffles stay within the 16 lanes)
  const T *z = (const T *)a.z + job * a.ldz;
  const float inv_t = 1.f / a.temperature;
  const RowEnds<T> ends(a, job, lane);
  float x[4], m = -INFINITY;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[i] = i * 16 + lane < a.L ? ElemT<T>::to_f(z[i * 16 + lane]) : -INFINITY;
    m = fmaxf(m, x[i]);
  }
  Sums p{lanes_max<16>(m), 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float d = x[i] - base_of(p.m);
    p.t += exp_of(d * inv_t);
    p.s += exp_of(d);
  }
  p.t = lanes_sum<16>(p.t);
  p.s = lanes_sum<16>(p.s);
  write_row<T, 16>(a, job, p, lane, ends);
}

// --------------------------------------------------------------- gradient
// What an element's gradient takes of its row; ruled-out rows and those without label or teacher have weights 0.
struct GradRow {
  float gk, lse_t, gl, lse, inv_t;
  int y;
  __device__ __forceinline__ GradRow(const DistillGradArgs &a, int64_t row) {
    inv_t = 1.f / a.temperature;
    gk = a.g_kl ? a.g_kl[row] * inv_t : 0.f;
    lse_t = a.g_kl ? a.lse_t[row] : 0.f;
    gl = a.g_logp ? a.g_logp[row] : 0.f;
    lse = a.g_logp ? a.lse[row] : 0.f;
    y = a.g_logp ? a.labels[row] : -1;
    if (lse <= kRuledOut || (unsigned)y >= (unsigned)a.L) {
      gl = lse = 0.f;
      y = -1;
    }
  }
  __device__ __forceinline__ void teach(bool teacher) {
    if (lse_t <= kRuledOut || !teacher) gk = lse_t = 0.f;
  }
  // of the dense terms and the label
  __device__ __forceinline__ float operator()(float x, int i) const {
    float d = 0.f;
    if (gk != 0.f) d = gk * exp_of(fmaf(x, inv_t, -lse_t));
    if (gl != 0.f) d = fmaf(-gl, exp_of(x - lse), d);
    return i == y ? d + gl : d;
  }
};

// Part of a row by TPR threads, as in the forward pass.
template <typename T, int TPR>
__global__ void __launch_bounds__(256) distill_grad_kernel(DistillGradArgs a, uint32_t jobs, FastDiv fd_parts, uint32_t per) {
  using B = Bits<T>;
  constexpr int VEC = B::VEC, GROUPS = 256 / TPR;
  __shared__ float buf[2][4];
  extern __shared__ float teacher[];  // of every row: weights, logits and classes [top]
  const int t = threadIdx.x % TPR, grp = row_in_block<TPR>(), top = a.g_kl ? a.top : 0;
  float *weight = teacher + grp * 3 * top, *logit = weight + top;
  int *cls = (int *)(logit + top);
  const uint32_t job = blockIdx.x * GROUPS + grp;
  if (job >= jobs) return;
  const int64_t row = fdiv(job, fd_parts);
  const T *z = (const T *)a.z + row * a.ldz;
  T *dz = (T *)a.dz + row * a.lddz;
  const Part<T> part(dz, a.L, job - (uint32_t)row * fd_parts.d, per);  // (z may lie otherwise: loads at any alignment)
  const float inv_t = 1.f / a.temperature;

  const auto load = [&](auto count, auto whole, uint32_t v, auto &w) {
#pragma unroll
    for (int u = 0; u < decltype(count)::value; ++u) {
      const uint32_t i = v + u * TPR + t;
      w[u] = *(const u32x4_any *)(z + part.head + (decltype(whole)::value ? i : min(i, part.v1 - 1)) * VEC);
    }
  };
  GradRow grad(a, row);
  float sum = 0.f;
  // the teacher's classes: weights, and the logits of those in this part (read before anything of it is written)
  const auto teach = [&] {
    float best = -INFINITY;
    for (int k = t; k < top; k += TPR) {
      int c = a.t_class[row * a.top + k];
      const float v = a.t_value[row * a.top + k];
      if ((unsigned)c >= (unsigned)a.L || v == -INFINITY) c = -1;
      cls[k] = c;
      weight[k] = v;
      if (c >= 0) best = fmaxf(best, v);
      logit[k] = part.has(c) ? ElemT<T>::to_f(z[c]) : 0.f;
    }
    const int single = part.single(t);
    const float x = single >= 0 ? ElemT<T>::to_f(z[single]) : 0.f;
    if (top) {
      best = base_of(row_max<TPR>(best, buf[0]));
      for (int k = t; k < top; k += TPR) {
        const float w = cls[k] >= 0 ? exp_of((weight[k] - best) * inv_t) : 0.f;
        weight[k] = w;
        sum += w;
      }
      sum = row_sum<TPR>(sum, buf[1]);
    }
    grad.teach(sum != 0.f);  // (an entry left has weight 1, or makes the sum NaN)
    row_sync<TPR>();
    if (single >= 0) dz[single] = ElemT<T>::from_f(grad(x, single));
  };
  const auto finish = [&](auto count, auto whole, uint32_t v, const auto &w) {
    constexpr int N = decltype(count)::value;
#pragma unroll
    for (int u = 0; u < N; ++u) {
      if (!decltype(whole)::value && u == N - 1 && v + u * TPR + t >= part.v1) break;
      const int i = part.head + (int)((v + u * TPR + t) * VEC);
      u32x4 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (VEC == 4) o[j] = __float_as_uint(grad(B::at(w[u], j), i + j));
        else o[j] = pack2_bf16(grad(B::at(w[u], 2 * j), i + 2 * j), grad(B::at(w[u], 2 * j + 1), i + 2 * j + 1));
      }
      *(u32x4 *)(dz + i) = o;
    }
  };
  // Rows of a wave load their first vectors before the teacher's entries are taken,
  // which is a chain of loads (65,536 rows of 1,000 classes, bf16: 73 and 68 us); a
  // workgroup would wait for them at its barriers (4,096 rows of 6,000: 24 and 28).
  bool taught = TPR == 256;
  if (taught) teach();
  each_batch<TPR>(part.v0, part.v1, [&](auto count, auto whole, uint32_t v) {
    u32x4 w[decltype(count)::value];
    load(count, whole, v, w);
    if (!taught) {  // (the same in all the row's threads)
      teach();
      taught = true;
    }
    finish(count, whole, v, w);
  });
  if (!taught) teach();
  if (grad.gk == 0.f) return;  // (the same in all the row's threads)
  row_sync<TPR>();
  for (int k = t; k < top; k += TPR) {
    const int c = cls[k];
    if (!part.has(c)) continue;
    float q = 0.f;
    for (int j = 0; j < top; ++j)
      if (cls[j] == c) q += weight[j];
    dz[c] = ElemT<T>::from_f(fmaf(-grad.gk, q / sum, grad(logit[k], c)));
  }
}

// Rows of at most 64 classes: 16 lanes a row.
template <typename T> __global__ void __launch_bounds__(256) distill_grad_small_kernel(DistillGradArgs a) {
  const int lane = threadIdx.x & 15;
  const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (row >= a.rows) return;  // (shuffles stay within the 16 lanes)
  const T *z = (const T *)a.z + row * a.ldz;
  T *dz = (T *)a.dz + row * a.lddz;
  const int top = a.g_kl ? a.top : 0;
  const int32_t *tc = a.t_class + row * a.top;
  const float *tv = a.t_value + row * a.top;
  const float inv_t = 1.f / a.temperature;
  float x[4], q[4] = {0.f, 0.f, 0.f, 0.f}, best = -INFINITY, sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = i * 16 + lane < a.L ? ElemT<T>::to_f(z[i * 16 + lane]) : 0.f;
  for (int k = lane; k < top; k += 16)
    if ((unsigned)tc[k] < (unsigned)a.L) best = fmaxf(best, tv[k]);
  best = base_of(lanes_max<16>(best));
  for (int k = 0; k < top; ++k) {  // every lane all entries, in the same order
    const int c = tc[k];
    if ((unsigned)c >= (unsigned)a.L || tv[k] == -INFINITY) continue;
    const float w = exp_of((tv[k] - best) * inv_t);
    sum += w;
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] += c == i * 16 + lane ? w : 0.f;
  }
  GradRow grad(a, row);
  grad.teach(sum != 0.f);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = i * 16 + lane;
    if (c >= a.L) continue;
    float d = grad(x[i], c);
    if (grad.gk != 0.f) d = fmaf(-grad.gk, q[i] / sum, d);
    dz[c] = ElemT<T>::from_f(d);
  }
}

// Vectors of a part, and parts of a row: whole rows where they are enough for
// every CU to have four workgroups, else parts of 1,024 vectors at least; the
// gradient, which has no parts to join, in such parts always: of 4,096 rows of
// 50,021 classes, bf16, in whole rows 180 us, in parts of 2,048 166, of 1,024 152 and
// of 512 200.
struct Parts {
  int threads;  // of a row: 16 and 64 with more of them in a workgroup
  uint32_t n, per;
};
template <typename T> Parts parts_of_row(int64_t rows, int L, int64_t groups = 1024) {
  const uint32_t vectors = ((uint32_t)L + Bits<T>::VEC - 1) / Bits<T>::VEC;
  if (vectors <= 32) return {16, 1, vectors};
  if (vectors <= 256) return {64, 1, vectors};
  const uint32_t step = 1024;
  const int64_t most = (vectors + step - 1) / step, want = (groups + rows - 1) / std::max<int64_t>(rows, 1);
  const uint32_t n = (uint32_t)std::max<int64_t>(1, std::min(most, want));
  const uint32_t per = ((vectors + n - 1) / n + step - 1) / step * step;
  return {256, (vectors + per - 1) / per, per};
}

template <typename P> P *entry_at(P *p, int64_t r) { return p ? p + r : nullptr; }

template <typename T> hipError_t run(const DistillArgs &all, hipStream_t s) {
  const Parts parts = parts_of_row<T>(all.rows, all.L);
  const bool two = all.temperature != 1.f && (all.lse || all.logp);
  const int64_t slab = kMaxBlocks / parts.n;
  for (int64_t r = 0; r < all.rows; r += slab) {
    DistillArgs a = all;
    a.z = (const T *)all.z + r * all.ldz;
    a.rows = std::min(slab, all.rows - r);
    a.t_class = all.t_class + r * all.top;
    a.t_value = all.t_value + r * all.top;
    a.labels = entry_at(all.labels, r);
    a.kl = entry_at(all.kl, r);
    a.lse_t = entry_at(all.lse_t, r);
    a.logp = entry_at(all.logp, r);
    a.lse = entry_at(all.lse, r);
    if (a.L <= 64) {
      hipLaunchKernelGGL(distill_small_kernel<T>, dim3((uint32_t)((a.rows + 15) / 16)), dim3(256), 0, s, a);
    } else {
      const uint32_t jobs = (uint32_t)(a.rows * parts.n);
      const uint32_t at_once = 256 / parts.threads;
      const auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((jobs + at_once - 1) / at_once), dim3(256), 0, s, a, jobs, make_fastdiv(parts.n),
                           parts.per);
      };
      if (parts.threads == 16) two ? launch(distill_kernel<T, 16, true>) : launch(distill_kernel<T, 16, false>);
      else if (parts.threads == 64) two ? launch(distill_kernel<T, 64, true>) : launch(distill_kernel<T, 64, false>);
      else two ? launch(distill_kernel<T, 256, true>) : launch(distill_kernel<T, 256, false>);
      if (parts.n > 1)
        hipLaunchKernelGGL(distill_join_kernel<T>, dim3((uint32_t)((a.rows + 3) / 4)), dim3(256), 0, s, a, parts.n);
    }
    const hipError_t e = hipGetLastError();  // (one after another on the stream: the workspace serves each)
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T> hipError_t run_grad(const DistillGradArgs &all, hipStream_t s) {
  const Parts parts = parts_of_row<T>(all.rows, all.L, (int64_t)1 << 40);
  const int64_t slab = kMaxBlocks / parts.n;
  for (int64_t r = 0; r < all.rows; r += slab) {
    DistillGradArgs a = all;
    a.z = (const T *)all.z + r * all.ldz;
    a.dz = (T *)all.dz + r * all.lddz;
    a.rows = std::min(slab, all.rows - r);
    a.t_class = entry_at(all.t_class, r * all.top);
    a.t_value = entry_at(all.t_value, r * all.top);
    a.labels = entry_at(all.labels, r);
    a.lse_t = entry_at(all.lse_t, r);
    a.lse = entry_at(all.lse, r);
    a.g_kl = entry_at(all.g_kl, r);
    a.g_logp = entry_at(all.g_logp, r);
    if (a.L <= 64) {
      hipLaunchKernelGGL(distill_grad_small_kernel<T>, dim3((uint32_t)((a.rows + 15) / 16)), dim3(256), 0, s, a);
    } else {
      const uint32_t jobs = (uint32_t)(a.rows * parts.n);
      const uint32_t at_once = 256 / parts.threads;
      const size_t lds = sizeof(float) * 3 * at_once * (a.g_kl ? a.top : 0);
      const auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((jobs + at_once - 1) / at_once), dim3(256), lds, s, a, jobs, make_fastdiv(parts.n),
                           parts.per);
      };
      if (parts.threads == 16) launch(distill_grad_kernel<T, 16>);
      else if (parts.threads == 64) launch(distill_grad_kernel<T, 64>);
      else launch(distill_grad_kernel<T, 256>);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename T> size_t work_of(int64_t rows, int L) {
  const Parts parts = parts_of_row<T>(rows, L);
  return L > 64 && parts.n > 1 ? sizeof(float4) * (size_t)rows * parts.n : 0;
}

}  // namespace

size_t distill_work_bytes(int dtype, int64_t rows, int L) {
  return dtype == GCPSL_BF16 ? work_of<bf16_t>(rows, L) : work_of<float>(rows, L);
}
hipError_t launch_distill(int dtype, const DistillArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(a, s) : run<float>(a, s);
}
hipError_t launch_distill_grad(int dtype, const DistillGradArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run_grad<bf16_t>(a, s) : run_grad<float>(a, s);
}

// Residual updates of rows grouped by cluster with the norms round a block, and
// their gradients (gfx950).
//
//   out = alpha x + beta s t,  s = sigmoid(gate),  t = w1 y r1  (or y)
//   h   = w2 out r2,           r = 1 / sqrt(mean of the row's squares + eps)
//
// A row is held in registers by a wave or a workgroup, as 16-byte vectors loaded
// at any alignment; longer rows are read again for every pass over them.
//
// Gradient: with o = out r2, v = y r1, a = w2 g_h and means over the row,
//
//   D  = g_out + r2 (a - o c2),   c2 = mean(a o)
//   dy = r1 (c - v c1),           c = beta s w1 D,  c1 = mean(c v)
//
// c1 needs D, which needs c2: but it is linear in D, so that one pass gives both
// from mean(a o), mean(p (g_out + r2 a)) and mean(p o) with p = beta s w1 v.  The
// weights' gradients are summed by the threads over the rows of a piece of a
// group; pieces are joined in their order by a second kernel.
//
// Bound: memory.
#include <algorithm>

#include "group.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Sum over the 64 lanes, the same in all of them.
__device__ __forceinline__ float wave_sum(float v) {
  const auto add = [&](auto ctrl, auto rows) {
    v += __uint_as_float(dpp<decltype(ctrl)::value, decltype(rows)::value>(__float_as_uint(v)));
  };
  using std::integral_constant;
  add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});
  add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Sums of N values over a row's TPR threads.  `buf` [4][N] is not to be written
// again before all threads have passed a later barrier.
template <int TPR, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float (*buf)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = wave_sum(v[i]);
  if constexpr (TPR == 256) {
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[threadIdx.x >> 6][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (buf[0][i] + buf[1][i]) + (buf[2][i] + buf[3][i]);
  }
}

// Group of row r, -1 if it is in none.
__device__ __forceinline__ int group_of(const int32_t *off, int G, int rows, int r) {
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < G; base += 64) {
    int begin = 0, end = 0;
    if (base + lane < G) group_rows(off, base + lane, rows, begin, end);
    const uint64_t hit = __ballot(begin <= r && r < end);
    if (hit) return __builtin_amdgcn_readfirstlane(base + __ffsll((unsigned long long)hit) - 1);
  }
  return -1;
}

// A thread's VEC columns from i on; those past the row's end are 0 and not stored.
// HELD, rows of n >= VEC: a vector that passes the end is the row's last one, of
// which the first `drop` columns are not its own (VEC: none is).
template <typename T, bool HELD> struct Cols {
  static constexpr int VEC = Vec16<T>::N;
  int i, drop, n;
  __device__ __forceinline__ Cols(int at, int n_) : i(at), drop(0), n(n_) {
    if constexpr (HELD) {
      i = min(at, n - VEC);
      drop = min(at - i, VEC);
    }
  }
  __device__ __forceinline__ bool own(int j) const { return HELD ? j >= drop : i + j < n; }
  __device__ __forceinline__ u32x4_any load(const T *p) const {
    u32x4_any v;
    if (HELD || i + VEC <= n) {
      v = *(const u32x4_any *)(p + i);
      return v;
    }
    v = u32x4_any{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (i + j < n) {
        if constexpr (sizeof(T) == 2) v[j >> 1] |= (uint32_t)p[i + j] << (16 * (j & 1));
        else v[j] = __float_as_uint(p[i + j]);
      }
    return v;
  }
  // zeros for what is not its own (after all loads, so that none is waited for before the others are sent)
  __device__ __forceinline__ void clear(u32x4_any &v) const {
    if (!HELD || drop == 0) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (j < drop) {
        if constexpr (sizeof(T) == 2) v[j >> 1] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
        else v[j] = 0;
      }
  }
  __device__ __forceinline__ void load_weights(const float *p, float (&w)[VEC]) const {
    if (HELD || i + VEC <= n) {
#pragma unroll
      for (int j = 0; j < VEC; j += 4) {
        const f32x4_any v = *(const f32x4_any *)(p + i + j);
#pragma unroll
        for (int r = 0; r < 4; ++r) w[j + r] = v[r];
      }
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) w[j] = i + j < n ? p[i + j] : 0.f;
    }
  }
  __device__ __forceinline__ void store(T *p, const float (&v)[VEC]) const {
    if (HELD ? drop == 0 : i + VEC <= n) {
      u32x4_any o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 2) o[j] = pack2_bf16(v[2 * j], v[2 * j + 1]);
        else o[j] = __float_as_uint(v[j]);
      }
      *(u32x4_any *)(p + i) = o;
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (own(j)) p[i + j] = ElemT<T>::from_f(v[j]);
    }
  }
  __device__ __forceinline__ void store_sums(float *p, const float (&v)[VEC]) const {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (own(j)) p[i + j] = v[j];
  }
};

__device__ __forceinline__ float rms_of(float squares, int n, float eps) {
  return 1.f / sqrtf(squares / (float)n + eps);
}

// A row by TPR threads (64: four rows a workgroup), NV vectors a thread; NV 0: any length.
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(256) residual_kernel(ResidualArgs a) {
  constexpr bool HELD = NV > 0;
  constexpr int VEC = Vec16<T>::N, H = HELD ? NV : 1;
  __shared__ float buf[2][2][4][1];
  const int t = threadIdx.x % TPR, n = a.n;
  const int64_t first = (int64_t)blockIdx.x * (256 / TPR) + (TPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0);
  int parity = 0;
  // (rows that share a workgroup are a wave's each: no barrier then)
  for (int64_t row = first; row < a.rows; row += (int64_t)gridDim.x * (256 / TPR), parity ^= 1) {
    const T *x = (const T *)a.x + row * a.ldx, *y = (const T *)a.y + row * a.ldy, *gate = (const T *)a.gate + row * a.ldg;
    T *out = (T *)a.out + row * a.ldo, *h = (T *)a.h + row * a.ldh;
    u32x4_any wx[H], wy[H], wg[H];
    const auto load = [&](int v, const Cols<T, HELD> &c) {
      wx[v] = c.load(x);
      if (a.y) wy[v] = c.load(y);
      if (a.gate) wg[v] = c.load(gate);
    };
    // f(v, columns) for all of the thread's vectors
    const auto each = [&](auto f) {
      if constexpr (HELD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) f(v, Cols<T, true>((v * TPR + t) * VEC, n));
      } else {
        for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) f(0, Cols<T, false>((int)i, n));
      }
    };
    if constexpr (HELD) {
      each(load);
      each([&](int v, const Cols<T, HELD> &c) {
        c.clear(wx[v]);
        if (a.y) c.clear(wy[v]);
      });
    }
    const int g = group_of(a.off, a.G, (int)a.rows, (int)row);
    if (g < 0) continue;
    const float *w1 = a.w_block ? a.w_block + g * a.wb_gs : nullptr, *w2 = a.w_next ? a.w_next + g * a.wn_gs : nullptr;
    float r1 = 1.f;
    if (w1) {
      float s[1] = {0.f};
      each([&](int v, const Cols<T, HELD> &c) {
        if constexpr (!HELD) wy[v] = c.load(y);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float e = Vec16<T>::at(wy[v], j);
          s[0] = fmaf(e, e, s[0]);
        }
      });
      row_sum<TPR>(s, buf[parity][0]);
      r1 = rms_of(s[0], n, a.eps);
      if (a.r_block && t == 0) a.r_block[row] = r1;
    }
    // the updated columns of vector v
    const auto update = [&](int v, const Cols<T, HELD> &c, float (&o)[VEC]) {
      if constexpr (!HELD) load(v, c);
      if (!a.y) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = Vec16<T>::at(wx[v], j);
        return;
      }
      float w[VEC];
      if (w1) c.load_weights(w1, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        float tj = Vec16<T>::at(wy[v], j), rest;
        if (w1) tj = w[j] * (tj * r1);
        if (a.gate) tj *= sigmoid_of(Vec16<T>::at(wg[v], j), rest);
        o[j] = fmaf(a.beta, tj, a.alpha * Vec16<T>::at(wx[v], j));
      }
    };
    float held[H][VEC];
    float s[1] = {0.f};
    if (HELD || w2) {
      each([&](int v, const Cols<T, HELD> &c) {
        update(v, c, held[v]);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] = fmaf(held[v][j], held[v][j], s[0]);
        if (HELD && a.out) c.store(out, held[v]);
      });
    }
    float r2 = 0.f;
    if (w2) {
      row_sum<TPR>(s, buf[parity][1]);
      r2 = rms_of(s[0], n, a.eps);
      if (a.r_next && t == 0) a.r_next[row] = r2;
    }
    if (HELD && !w2) continue;
    each([&](int v, const Cols<T, HELD> &c) {
      if constexpr (!HELD) {
        update(v, c, held[v]);
        if (a.out) c.store(out, held[v]);
        if (!w2) return;
      }
      float w[VEC];
      c.load_weights(w2, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) w[j] *= held[v][j] * r2;
      c.store(h, w);
    });
  }
}

// --------------------------------------------------------------- gradients
// What a thread has of a row: vectors of out, g_out, g_h, y and the gate.
struct GradVec {
  u32x4_any x, go, gh, y, g;
};

// Rows of a piece by a workgroup; NV vectors a thread, or (0) any length.
constexpr int kPieceRows = 256;  // of a piece, at most
template <typename T, int NV>
__global__ void __launch_bounds__(256) residual_grad_kernel(ResidualGradArgs a) {
  constexpr bool HELD = NV > 0;
  constexpr int VEC = Vec16<T>::N, H = HELD ? NV : 1, TPR = 256;
  __shared__ float buf[2][4][3];
  __shared__ float means[HELD ? 1 : kPieceRows][2];
  const int t = threadIdx.x, n = a.n;
  int g, q0, q1, slot;
  uint32_t tile;
  {
    GroupArgs p{};  // what piece_of takes of it
    p.off = a.off;
    p.G = a.G;
    p.Q = (int)a.rows;
    p.piece = a.piece;
    p.slots = a.slots;
    if (!piece_of<1>(p, 1, blockIdx.x, g, q0, q1, slot, tile)) return;
  }
  const float *w1 = a.w_block ? a.w_block + g * a.wb_gs : nullptr, *w2 = a.w_next ? a.w_next + g * a.wn_gs : nullptr;
  const float inv_n = 1.f / (float)n;
  const auto load = [&](int row, const Cols<T, HELD> &c, GradVec &w) {
    if (a.g_h) {
      w.x = c.load((const T *)a.x + (int64_t)row * a.ldx);
      w.gh = c.load((const T *)a.g_h + (int64_t)row * a.ldgh);
    }
    if (a.g_out) w.go = c.load((const T *)a.g_out + (int64_t)row * a.ldgo);
    if (a.y) w.y = c.load((const T *)a.y + (int64_t)row * a.ldy);
    if (a.gate) w.g = c.load((const T *)a.gate + (int64_t)row * a.ldg);
  };
  // the row's three sums from one vector
  const auto sums = [&](const Cols<T, HELD> &c, const GradVec &w, const float (&b1)[VEC], const float (&b2)[VEC], float r1,
                        float r2, float (&s)[3]) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const float o = a.g_h ? Vec16<T>::at(w.x, j) * r2 : 0.f, e = a.g_h ? b2[j] * Vec16<T>::at(w.gh, j) : 0.f;
      s[0] = fmaf(e, o, s[0]);
      if (w1) {
        float p = b1[j] * (Vec16<T>::at(w.y, j) * r1), rest;
        if (a.gate) p *= sigmoid_of(Vec16<T>::at(w.g, j), rest);
        s[1] = fmaf(p, fmaf(r2, e, a.g_out ? Vec16<T>::at(w.go, j) : 0.f), s[1]);
        s[2] = fmaf(p, o, s[2]);
      }
    }
  };
  // results of one vector of a row, c2 and c1 the row's means (of c v without beta)
  const auto finish = [&](int row, const Cols<T, HELD> &c, const GradVec &w, const float (&b1)[VEC], const float (&b2)[VEC],
                          float r1, float r2, float c2, float c1, float (&d1)[VEC], float (&d2)[VEC]) {
    float dx[VEC], dy[VEC], dg[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      float D = a.g_out ? Vec16<T>::at(w.go, j) : 0.f;
      if (a.g_h) {
        const float o = Vec16<T>::at(w.x, j) * r2, gh = Vec16<T>::at(w.gh, j);
        D = fmaf(r2, fmaf(-o, c2, b2[j] * gh), D);
        d2[j] = fmaf(gh, o, d2[j]);
      }
      dx[j] = a.alpha * D;
      if (!a.y) continue;
      float s = 1.f, rest = 0.f;
      if (a.gate) s = sigmoid_of(Vec16<T>::at(w.g, j), rest);
      const float e = a.beta * D, es = e * s;
      const float v = Vec16<T>::at(w.y, j) * r1;
      float tj = v;
      dy[j] = es;
      if (w1) {
        tj *= b1[j];
        dy[j] = r1 * fmaf(-v, a.beta * c1, es * b1[j]);
        d1[j] = fmaf(es, v, d1[j]);
      }
      dg[j] = es * tj * rest;
    }
    c.store((T *)a.dx + (int64_t)row * a.lddx, dx);
    if (a.y) c.store((T *)a.dy + (int64_t)row * a.lddy, dy);
    if (a.dgate) c.store((T *)a.dgate + (int64_t)row * a.lddg, dg);
  };
  const auto means_of = [&](const float (&s)[3], float r2, float &c2, float &c1) {
    c2 = s[0] * inv_n;
    c1 = fmaf(-r2 * c2, s[2], s[1]) * inv_n;
  };
  const auto r1_of = [&](int row) { return w1 ? a.r_block[row] : 1.f; };
  const auto r2_of = [&](int row) { return a.g_h ? a.r_next[row] : 0.f; };
  // a vector's weight gradients, to their place or to a partial
  const auto store_grads = [&](const Cols<T, HELD> &c, const float (&d1)[VEC], const float (&d2)[VEC]) {
    if (a.dw_block) c.store_sums(slot >= 0 ? a.part + (int64_t)slot * 2 * n : a.dw_block + g * a.dwb_gs, d1);
    if (a.dw_next) c.store_sums(slot >= 0 ? a.part + ((int64_t)slot * 2 + 1) * n : a.dw_next + g * a.dwn_gs, d2);
  };

  if constexpr (HELD) {
    float b1[H][VEC], b2[H][VEC], d1[H][VEC], d2[H][VEC];
    GradVec w[H];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<T, true> c((v * TPR + t) * VEC, n);
      if (w1) c.load_weights(w1, b1[v]);
      if (w2) c.load_weights(w2, b2[v]);
#pragma unroll
      for (int j = 0; j < VEC; ++j) d1[v][j] = d2[v][j] = 0.f;
    }
    for (int row = q0; row < q1; ++row) {
      const float r1 = r1_of(row), r2 = r2_of(row);
      float s[3] = {0.f, 0.f, 0.f}, c2, c1;
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Cols<T, true> c((v * TPR + t) * VEC, n);
        load(row, c, w[v]);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const Cols<T, true> c((v * TPR + t) * VEC, n);
        if (a.g_h) c.clear(w[v].gh);  // (then every sum's terms are 0)
        if (a.y) c.clear(w[v].y);
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) sums(Cols<T, true>((v * TPR + t) * VEC, n), w[v], b1[v], b2[v], r1, r2, s);
      row_sum<TPR>(s, buf[row & 1]);
      means_of(s, r2, c2, c1);
#pragma unroll
      for (int v = 0; v < NV; ++v)
        finish(row, Cols<T, true>((v * TPR + t) * VEC, n), w[v], b1[v], b2[v], r1, r2, c2, c1, d1[v], d2[v]);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) store_grads(Cols<T, true>((v * TPR + t) * VEC, n), d1[v], d2[v]);
  } else {
    GradVec w;
    for (int row = q0; row < q1; ++row) {
      const float r1 = r1_of(row), r2 = r2_of(row);
      float s[3] = {0.f, 0.f, 0.f}, b1[VEC], b2[VEC];
      for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) {
        const Cols<T, false> c((int)i, n);
        if (w1) c.load_weights(w1, b1);
        if (w2) c.load_weights(w2, b2);
        load(row, c, w);
        sums(c, w, b1, b2, r1, r2, s);
      }
      row_sum<TPR>(s, buf[row & 1]);
      if (t == 0) means_of(s, r2, means[row - q0][0], means[row - q0][1]);
    }
    __syncthreads();
    for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) {
      const Cols<T, false> c((int)i, n);
      float b1[VEC], b2[VEC], d1[VEC], d2[VEC];
      if (w1) c.load_weights(w1, b1);
      if (w2) c.load_weights(w2, b2);
#pragma unroll
      for (int j = 0; j < VEC; ++j) d1[j] = d2[j] = 0.f;
      for (int row = q0; row < q1; ++row) {
        load(row, c, w);
        finish(row, c, w, b1, b2, r1_of(row), r2_of(row), means[row - q0][0], means[row - q0][1], d1, d2);
      }
      store_grads(c, d1, d2);
    }
  }
}

// The weights' gradients of a group of several pieces: a column a thread.
__global__ void __launch_bounds__(256) residual_join_kernel(ResidualGradArgs a, uint32_t blocks) {
  const int g = (int)(blockIdx.x / blocks);
  uint32_t before = 0, slots = 0, n = 0, first = 0;
  for (int base = 0; base <= g; base += 64) {
    LaneTiles l;
    before = lane_tiles<true>(a.off, a.G, (int)a.rows, a.piece, base, before, l);
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
  const int64_t c = (int64_t)(blockIdx.x - g * blocks) * 256 + threadIdx.x;  // of both weights' columns
  if (c >= 2 * (int64_t)a.n) return;
  const bool second = c >= a.n;
  float *out = second ? a.dw_next : a.dw_block;
  if (!out) return;
  const float *p = a.part + (int64_t)first * 2 * a.n + c;
  float s = 0.f;
  for (uint32_t k = 0; k < n; ++k) s += p[(int64_t)k * 2 * a.n];
  out[second ? g * a.dwn_gs + (c - a.n) : g * a.dwb_gs + c] = s;
}

template <typename T> hipError_t run(const ResidualArgs &a, hipStream_t s) {
  constexpr int VEC = Vec16<T>::N;
  const int vectors = a.n < VEC ? INT32_MAX : (a.n + VEC - 1) / VEC;
  const auto launch = [&](auto kernel, int64_t blocks) {
    blocks = std::min<int64_t>(blocks, 8 * kCUs);  // as many as the chip holds
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
  };
  if (vectors <= 64) return launch(residual_kernel<T, 64, 1>, (a.rows + 3) / 4);
  if (vectors <= 128) return launch(residual_kernel<T, 64, 2>, (a.rows + 3) / 4);
  if (vectors <= 256) return launch(residual_kernel<T, 256, 1>, a.rows);
  if (vectors <= 512) return launch(residual_kernel<T, 256, 2>, a.rows);
  if (vectors <= 1024) return launch(residual_kernel<T, 256, 4>, a.rows);
  return launch(residual_kernel<T, 256, 0>, a.rows);
}

template <typename T> hipError_t run_grad(const ResidualGradArgs &a, hipStream_t s) {
  constexpr int VEC = Vec16<T>::N;
  const int vectors = a.n < VEC ? INT32_MAX : (a.n + VEC - 1) / VEC;
  const int64_t blocks = a.rows / a.piece + a.G;
  if (blocks > kMaxBlocks) return hipErrorInvalidConfiguration;
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(256), 0, s, a);
    return hipGetLastError();
  };
  hipError_t e;
  if (vectors <= 256) e = launch(residual_grad_kernel<T, 1>);
  else if (vectors <= 512) e = launch(residual_grad_kernel<T, 2>);
  else e = launch(residual_grad_kernel<T, 0>);
  if (e == hipSuccess && a.slots > 0 && (a.dw_block || a.dw_next)) {
    const int64_t per = (2 * (int64_t)a.n + 255) / 256;
    if (per * a.G > kMaxBlocks) return hipErrorInvalidConfiguration;
    hipLaunchKernelGGL(residual_join_kernel, dim3((uint32_t)(per * a.G)), dim3(256), 0, s, a, (uint32_t)per);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// Rows of a piece: enough pieces for two workgroups a CU, at most kPieceRows - kPieceRows / 3.
GroupPieces residual_pieces(int G, int64_t rows, int n) {
  const int64_t piece = std::min<int64_t>(std::max<int64_t>((rows + 511) / 512, 4), kPieceRows / 2);
  // a group of p > 1 pieces has more than (p - 1/2) piece >= 3/4 p piece rows
  return {(int)piece, rows * 2 >= piece * 3 ? (int)(rows * 4 / (piece * 3)) : 0};
}

hipError_t launch_residual(int dtype, const ResidualArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(a, s) : run<float>(a, s);
}
hipError_t launch_residual_grad(int dtype, const ResidualGradArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run_grad<bf16_t>(a, s) : run_grad<float>(a, s);
}

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
// from three sums (GradRow).  The
// weights' gradients are summed by the threads over the rows of a piece of a
// group; pieces are joined in their order by a second kernel.
//
// Bound: memory.  bf16, n 4,096: 32,768 rows of 16 groups 268 to 274 us by card (5.0 to
// 4.9 TB/s), norms alone 5.4 TB/s; the gradient of 16,384 rows 237 us (4.5), of the
// norm alone 90 (4.5).  A row's instructions, about 60 an element in the gradient,
// take nearly as long: sigmoids are taken twice, once for the sums and once for the
// results.  Rows of four or two a wave, 16 groups: 2,048 of n 64 5.4 us in either type,
// which is the launch; 1,000,000 in fp32 275 (4.7 TB/s) and in bf16 224 (2.9, as half
// the lanes hold no vector of such rows); 262,144 of n 256, bf16, 141 (4.8).
#include <algorithm>

#include "group.h"

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Threads of a row and of a workgroup; a workgroup takes R rows at a time.
constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// This thread's row of those that its workgroup takes at a time: in a scalar register where a wave has one.
template <int TPR> __device__ __forceinline__ int row_in_block() {
  const int i = (int)threadIdx.x / TPR;
  return TPR >= 64 ? __builtin_amdgcn_readfirstlane(i) : i;
}

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
// Over W neighbouring lanes of 16 that hold W values over and over, by rotations, the same in all of them.
template <int W> __device__ __forceinline__ float lanes_sum(float v) {
  if (W >= 16) v += __uint_as_float(dpp<0x128, 0xf>(__float_as_uint(v)));
  if (W >= 8) v += __uint_as_float(dpp<0x124, 0xf>(__float_as_uint(v)));
  if (W >= 4) v += __uint_as_float(dpp<0x122, 0xf>(__float_as_uint(v)));
  return v + __uint_as_float(dpp<0x121, 0xf>(__float_as_uint(v)));
}

// Sums of N values over a row's TPR threads.  Rows of more than a wave meet in
// `buf`, one of 16 waves an entry, which is not to be written again before all
// threads have passed a later barrier.
template <int TPR, int N> __device__ __forceinline__ void row_sum(float (&v)[N], float (*buf)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (TPR >= 64) v[i] = wave_sum(v[i]);
    else v[i] = lanes_sum<16>(v[i]);
    if (TPR == 32) v[i] += __shfl_xor(v[i], 16);
  }
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) buf[wave][i] = v[i];
    __syncthreads();
    const float(&own)[N] = buf[wave / W * W + (threadIdx.x & (W - 1))];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = lanes_sum<W>(own[i]);
  }
}

// Groups of rows: the first 64 groups' bounds stay in the lanes, a group a lane.  So
// all 64 lanes have to be active in every lookup, those too that have no row (any
// row will do for them): a group whose lane is switched off would not be seen.
struct Finder {
  const int32_t *off;
  int G, rows, begin, end;
  __device__ __forceinline__ Finder(const int32_t *off_, int G_, int rows_) : off(off_), G(G_), rows(rows_) { load(0, begin, end); }
  __device__ __forceinline__ void load(int base, int &b, int &e) const {
    const int i = base + (int)(threadIdx.x & 63);
    b = e = 0;
    if (i < G) group_rows(off, i, rows, b, e);
  }
  // group of row r, the same r in all lanes, -1 if it is in none
  __device__ __forceinline__ int of(int r) const {
    uint64_t hit = __ballot(begin <= r && r < end);
    int base = 0;
    while (!hit && base + 64 < G) {
      base += 64;
      int b, e;
      load(base, b, e);
      hit = __ballot(b <= r && r < e);
    }
    return hit ? __builtin_amdgcn_readfirstlane(base + __ffsll((unsigned long long)hit) - 1) : -1;
  }
  // of every lane's row, TPR lanes or more having the same
  template <int TPR> __device__ __forceinline__ int of_lane_rows(int r) const {
    if constexpr (TPR >= 64) {
      return of(__builtin_amdgcn_readfirstlane(r));
    } else {
      int g = -1;
#pragma unroll
      for (int k = 0; k < 64; k += TPR) {
        const int own = of(__builtin_amdgcn_readlane(r, k));
        if ((int)(threadIdx.x & 63) / TPR == k / TPR) g = own;
      }
      return g;
    }
  }
};

// A thread's VEC columns from i on; those past the row's end are 0 and not stored.
// HELD, rows of n >= VEC: a vector that passes the end is the row's last one, of
// which the first `drop` columns are not its own (VEC: none is).
template <typename T, bool HELD> struct Cols {
  static constexpr int VEC = Vec16<T>::N;
  int i, drop, n;
  Cols() = default;
  __device__ __forceinline__ Cols(int first, int n_) : i(first), drop(0), n(n_) {
    if constexpr (HELD) {
      i = min(first, n - VEC);
      drop = min(first - i, VEC);
    }
  }
  // To the compiler another i from here on: else a loop over rows carries a 64-bit
  // address a lane for each of its tensors (16 registers, spilled) where the row's
  // scalar one and this offset will do.
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(i)); }
  // p + i; held rows are short: an offset of 32 bits next to a scalar base
  template <typename E> __device__ __forceinline__ E *at(E *p) const {
    if constexpr (HELD) return (E *)((char *)p + (uint32_t)i * (uint32_t)sizeof(E));
    return p + i;
  }
  template <typename E> __device__ __forceinline__ const E *at(const E *p) const { return at(const_cast<E *>(p)); }
  __device__ __forceinline__ bool own(int j) const { return HELD ? j >= drop : i + j < n; }
  __device__ __forceinline__ u32x4_any load(const T *p) const {
    u32x4_any v;
    if (HELD || i + VEC <= n) {
      v = *(const u32x4_any *)at(p);
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
  __device__ __forceinline__ void clear(u32x4 &v) const {
    if (!HELD || drop == 0) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (j < drop) {
        if constexpr (sizeof(T) == 2) v[j >> 1] &= j & 1 ? 0x0000ffffu : 0xffff0000u;
        else v[j] = 0;
      }
  }
  // 0 for what is not its own: an infinite one times a cleared value would be NaN.
  __device__ __forceinline__ void load_weights(const float *p, float (&w)[VEC]) const {
    if (HELD || i + VEC <= n) {
#pragma unroll
      for (int j = 0; j < VEC; j += 4) {
        const f32x4_any v = *(const f32x4_any *)(at(p) + j);
#pragma unroll
        for (int r = 0; r < 4; ++r) w[j + r] = v[r];
      }
      if (HELD && __builtin_expect(drop > 0, 0))  // (a branch, so that no other thread waits for the loads here)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (j < drop) w[j] = 0.f;
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
      *(u32x4_any *)at(p) = o;
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (own(j)) at(p)[j] = ElemT<T>::from_f(v[j]);
    }
  }
  __device__ __forceinline__ void store_sums(float *p, const float (&v)[VEC]) const {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (own(j)) at(p)[j] = v[j];
  }
};

__device__ __forceinline__ float rms_of(float squares, int n, float eps) {
  return 1.f / sqrtf(squares / (float)n + eps);
}

// Rows [blockIdx `per`, + per), each by TPR threads that hold NV vectors of it; the
// next row's loads go out before this one's sums.  A group's weights stay in
// registers as long as the rows are its own.
template <typename T, int TPR, int NV>
__global__ void __launch_bounds__(block_of(TPR)) residual_kernel(ResidualArgs a, int per) {
  constexpr int VEC = Vec16<T>::N, R = block_of(TPR) / TPR;
  __shared__ float buf[2][2][16][1];
  const int t = threadIdx.x % TPR, n = a.n, rows = (int)a.rows;
  const int r0 = (int)min((int64_t)blockIdx.x * per, a.rows), r1 = (int)min((int64_t)r0 + per, a.rows);
  const Finder finder(a.off, a.G, rows);
  struct Raw {
    u32x4 x, y, g;
  };
  Raw now[NV], next[NV];
  Cols<T, true> cols_[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) cols_[v] = Cols<T, true>((v * TPR + t) * VEC, n);
  const auto cols = [&](int v) -> const Cols<T, true> & { return cols_[v]; };
  const auto load = [&](int row, Raw(&w)[NV]) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<T, true> c = cols(v);
      w[v].x = c.load((const T *)a.x + row * a.ldx);
      if (a.y) w[v].y = c.load((const T *)a.y + row * a.ldy);
      if (a.gate) w[v].g = c.load((const T *)a.gate + row * a.ldg);
    }
  };
  const int mine = r0 + row_in_block<TPR>();  // the first row
  if (r0 < r1) load(min(mine, r1 - 1), next);
  float w1[NV][VEC], w2[NV][VEC];
  int held = -1, parity = 0;
  for (int first = r0; first < r1; first += R, parity ^= 1) {
    const int row = mine + (first - r0);
#pragma unroll
    for (int v = 0; v < NV; ++v) cols_[v].fresh();
#pragma unroll
    for (int v = 0; v < NV; ++v) now[v] = next[v];
    if (first + R < r1) load(min(row + R, r1 - 1), next);
    const int g = finder.of_lane_rows<TPR>(min(row, r1 - 1));
    const bool live = row < r1 && g >= 0;
    if (g >= 0 && g != held) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        if (a.w_block) cols(v).load_weights(a.w_block + g * a.wb_gs, w1[v]);
        if (a.w_next) cols(v).load_weights(a.w_next + g * a.wn_gs, w2[v]);
      }
      held = g;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const Cols<T, true> c = cols(v);
      c.clear(now[v].x);
      if (a.y) c.clear(now[v].y);
    }
    float r = 1.f;
    if (a.w_block) {
      float s[1] = {0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
          const float e = Vec16<T>::at(now[v].y, j);
          s[0] = fmaf(e, e, s[0]);
        }
      row_sum<TPR>(s, buf[parity][0]);
      r = rms_of(s[0], n, a.eps);
      if (a.r_block && t == 0 && live) a.r_block[row] = r;
    }
    float o[NV][VEC], s[1] = {0.f};
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        o[v][j] = Vec16<T>::at(now[v].x, j);
        if (a.y) {
          float y = Vec16<T>::at(now[v].y, j), rest;
          if (a.w_block) y = w1[v][j] * (y * r);
          if (a.gate) y *= sigmoid_of(Vec16<T>::at(now[v].g, j), rest);
          o[v][j] = fmaf(a.beta, y, a.alpha * o[v][j]);
        }
        s[0] = fmaf(o[v][j], o[v][j], s[0]);
      }
      if (a.out && live) cols(v).store((T *)a.out + row * a.ldo, o[v]);
    }
    if (!a.w_next) continue;  // (the same in all threads)
    row_sum<TPR>(s, buf[parity][1]);
    r = rms_of(s[0], n, a.eps);
    if (!live) continue;  // (barriers are passed)
    if (a.r_next && t == 0) a.r_next[row] = r;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) o[v][j] = w2[v][j] * (o[v][j] * r);
      cols(v).store((T *)a.h + row * a.ldh, o[v]);
    }
  }
}

// Rows that no workgroup holds (or of less than a vector), a workgroup each: read for every pass.
template <typename T> __global__ void __launch_bounds__(256) residual_long_kernel(ResidualArgs a) {
  constexpr int VEC = Vec16<T>::N, TPR = 256;
  __shared__ float buf[2][2][16][1];
  const int t = threadIdx.x, n = a.n;
  const Finder finder(a.off, a.G, (int)a.rows);
  int parity = 0;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const int g = finder.of((int)row);
    if (g < 0) continue;
    parity ^= 1;  // (of the rows that are taken: two in turn must not share a buffer, as only one of the sums may be asked for)
    const T *x = (const T *)a.x + row * a.ldx, *y = (const T *)a.y + row * a.ldy, *gate = (const T *)a.gate + row * a.ldg;
    const float *w1 = a.w_block ? a.w_block + g * a.wb_gs : nullptr, *w2 = a.w_next ? a.w_next + g * a.wn_gs : nullptr;
    const auto each = [&](auto f) {
      for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) f(Cols<T, false>((int)i, n));
    };
    float r1 = 1.f, r2 = 0.f;
    if (w1) {
      float s[1] = {0.f};
      each([&](const Cols<T, false> &c) {
        const u32x4_any v = c.load(y);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] = fmaf(Vec16<T>::at(v, j), Vec16<T>::at(v, j), s[0]);
      });
      row_sum<TPR>(s, buf[parity][0]);
      r1 = rms_of(s[0], n, a.eps);
      if (a.r_block && t == 0) a.r_block[row] = r1;
    }
    const auto update = [&](const Cols<T, false> &c, float(&o)[VEC]) {
      const u32x4_any vx = c.load(x);
      u32x4_any vy, vg;
      if (a.y) vy = c.load(y);
      if (a.gate) vg = c.load(gate);
      float w[VEC];
      if (w1) c.load_weights(w1, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        o[j] = Vec16<T>::at(vx, j);
        if (!a.y) continue;
        float v = Vec16<T>::at(vy, j), rest;
        if (w1) v = w[j] * (v * r1);
        if (a.gate) v *= sigmoid_of(Vec16<T>::at(vg, j), rest);
        o[j] = fmaf(a.beta, v, a.alpha * o[j]);
      }
    };
    float o[VEC];
    if (w2) {
      float s[1] = {0.f};
      each([&](const Cols<T, false> &c) {
        update(c, o);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s[0] = fmaf(o[j], o[j], s[0]);
      });
      row_sum<TPR>(s, buf[parity][1]);
      r2 = rms_of(s[0], n, a.eps);
      if (a.r_next && t == 0) a.r_next[row] = r2;
    }
    each([&](const Cols<T, false> &c) {
      update(c, o);
      if (a.out) c.store((T *)a.out + row * a.ldo, o);
      if (!w2) return;
      float w[VEC];
      c.load_weights(w2, w);
#pragma unroll
      for (int j = 0; j < VEC; ++j) w[j] *= o[j] * r2;
      c.store((T *)a.h + row * a.ldh, w);
    });
  }
}

// --------------------------------------------------------------- gradients
// What a thread has of a row: vectors of out, g_out, g_h, y and the gate.  What a
// call does not have is 0 (its weights 1, its reciprocal rms 0 or 1, its gate
// open), so that all calls go the same way.
struct GradVec {
  u32x4 x, go, gh, y, g;
  __device__ __forceinline__ GradVec() { x = go = gh = y = g = u32x4{0, 0, 0, 0}; }
  // The values below are taken from here again, not kept from before: registers for
  // as many again of them (of a bf16 vector's, 171 in all) would halve the waves.
  __device__ __forceinline__ void again() { asm volatile("" : "+v"(x), "+v"(go), "+v"(gh), "+v"(y), "+v"(g)); }
};
// BLOCK: with a block's output; else the norm alone, which has no y, gate or w_block.
template <bool BLOCK, typename T, bool HELD>
__device__ __forceinline__ void load_grad(const ResidualGradArgs &a, int row, const Cols<T, HELD> &c, GradVec &w) {
  if (a.g_h) {
    w.x = c.load((const T *)a.x + (int64_t)row * a.ldx);
    w.gh = c.load((const T *)a.g_h + (int64_t)row * a.ldgh);
  }
  if (a.g_out) w.go = c.load((const T *)a.g_out + (int64_t)row * a.ldgo);
  if constexpr (BLOCK) {
    w.y = c.load((const T *)a.y + (int64_t)row * a.ldy);
    if (a.gate) w.g = c.load((const T *)a.gate + (int64_t)row * a.ldg);
  }
}
// What a row's elements take of it.  With e = w2 g_h, f = g_out + r2 e and p = w1 y s,
// the means c2 and c1 are those of r2 e x and of r1 p (f - r2 c2 r2 x) (x the updated
// row), so that only sums of products of the loaded values are needed; and
//   D = f - k2 x,  k2 = r2^2 c2;   dy = r1 beta s D w1 - k1 y,  k1 = beta r1^2 c1.
struct GradRow {
  float r1, r2, k1, k2;
  __device__ __forceinline__ GradRow(const ResidualGradArgs &a, int row) : k1(0.f), k2(0.f) {
    r1 = a.w_block ? a.r_block[row] : 1.f;
    r2 = a.g_h ? a.r_next[row] : 0.f;
  }
  // s: sums of e x, p f, p x
  __device__ __forceinline__ void means(const ResidualGradArgs &a, const float (&s)[3]) {
    const float inv_n = 1.f / (float)a.n;
    k2 = r2 * r2 * (r2 * s[0] * inv_n);
    if (a.w_block) k1 = a.beta * r1 * r1 * (r1 * fmaf(-k2, s[2], s[1]) * inv_n);
  }
};
// s = sigmoid(g), and 1 - s = e^-g s: g below -87, where that would be infinity times 0, is taken as that.  (A NaN stays one.)
__device__ __forceinline__ float open_of(float g) {
  return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2E * g));
}
__device__ __forceinline__ float open_of(float g, float &rest) {
  const float e = __builtin_amdgcn_exp2f(-kLog2E * (g < -87.f ? -87.f : g)), s = __builtin_amdgcn_rcpf(1.f + e);
  rest = e * s;
  return s;
}
// The row's three sums from one vector.
template <bool BLOCK, typename T, int VEC>
__device__ __forceinline__ void grad_sums(const ResidualGradArgs &a, const GradVec &w, const float (&b1)[VEC],
                                          const float (&b2)[VEC], const GradRow &r, float (&s)[3]) {
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    const float x = Vec16<T>::at(w.x, j), e = b2[j] * Vec16<T>::at(w.gh, j);
    s[0] = fmaf(e, x, s[0]);
    if constexpr (BLOCK) {
      const float open = open_of(Vec16<T>::at(w.g, j)), p = b1[j] * Vec16<T>::at(w.y, j) * (a.gate ? open : 1.f);
      s[1] = fmaf(p, fmaf(r.r2, e, Vec16<T>::at(w.go, j)), s[1]);
      s[2] = fmaf(p, x, s[2]);
    }
  }
}
// Results of one vector of a row, and what it adds to the weights' gradients.
template <bool BLOCK, typename T, bool HELD, int VEC>
__device__ __forceinline__ void grad_finish(const ResidualGradArgs &a, int row, const Cols<T, HELD> &c, const GradVec &w,
                                            const float (&b1)[VEC], const float (&b2)[VEC], const GradRow &r,
                                            float (&d1)[VEC], float (&d2)[VEC]) {
  float dx[VEC], dy[VEC], dg[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) {
    const float x = Vec16<T>::at(w.x, j), gh = Vec16<T>::at(w.gh, j);
    const float D = fmaf(-r.k2, x, fmaf(r.r2, b2[j] * gh, Vec16<T>::at(w.go, j)));
    d2[j] = fmaf(gh * r.r2, x, d2[j]);
    dx[j] = BLOCK ? a.alpha * D : D;
    if constexpr (BLOCK) {
      float rest;
      const float y = Vec16<T>::at(w.y, j), open = open_of(Vec16<T>::at(w.g, j), rest);
      const float es = D * (a.gate ? a.beta * open : a.beta), t = r.r1 * (es * b1[j]);
      dy[j] = fmaf(-r.k1, y, t);
      d1[j] = fmaf(es * r.r1, y, d1[j]);
      dg[j] = t * y * rest;
      if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (four at a time: fewer registers)
    }
  }
  c.store((T *)a.dx + (int64_t)row * a.lddx, dx);
  if constexpr (BLOCK) {
    c.store((T *)a.dy + (int64_t)row * a.lddy, dy);
    if (a.dgate) c.store((T *)a.dgate + (int64_t)row * a.lddg, dg);
  }
}
// Where a piece's sums of the weights' gradients go.
struct GradPlace {
  float *d1, *d2;
  __device__ __forceinline__ GradPlace(const ResidualGradArgs &a, int g, int slot) {
    d1 = !a.dw_block ? nullptr : slot >= 0 ? a.part + (int64_t)slot * 2 * a.n : a.dw_block + g * a.dwb_gs;
    d2 = !a.dw_next ? nullptr : slot >= 0 ? a.part + ((int64_t)slot * 2 + 1) * a.n : a.dw_next + g * a.dwn_gs;
  }
};
__device__ __forceinline__ bool grad_piece(const ResidualGradArgs &a, int &g, int &q0, int &q1, int &slot) {
  GroupArgs p{};  // what piece_of takes of it
  p.off = a.off;
  p.G = a.G;
  p.Q = (int)a.rows;
  p.piece = a.piece;
  p.slots = a.slots;
  uint32_t tile;
  return piece_of<1>(p, 1, blockIdx.x, g, q0, q1, slot, tile);
}

// Rows of a piece, R at a time, each by TPR threads that hold NV vectors of it; AHEAD:
// the next rows' loads go out before these ones' sums.
template <typename T, int TPR, int NV, bool AHEAD, bool BLOCK>
__global__ void __launch_bounds__(block_of(TPR), TPR < 64 ? 3 : 4) residual_grad_kernel(ResidualGradArgs a) {
  constexpr int VEC = Vec16<T>::N, R = block_of(TPR) / TPR;
  __shared__ float buf[2][16][3];
  __shared__ float shares[R > 1 ? R - 1 : 1][R > 1 ? TPR * NV * VEC : 1];
  const int t = threadIdx.x % TPR, rg = row_in_block<TPR>(), n = a.n;
  int g, q0, q1, slot;
  if (!grad_piece(a, g, q0, q1, slot)) return;
  Cols<T, true> cols_[NV];
#pragma unroll
  for (int v = 0; v < NV; ++v) cols_[v] = Cols<T, true>((v * TPR + t) * VEC, n);
  const auto cols = [&](int v) -> const Cols<T, true> & { return cols_[v]; };
  float b1[NV][VEC], b2[NV][VEC], d1[NV][VEC], d2[NV][VEC];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      b1[v][j] = b2[v][j] = 1.f;
      d1[v][j] = d2[v][j] = 0.f;
    }
    if (a.w_block) cols(v).load_weights(a.w_block + g * a.wb_gs, b1[v]);
    if (a.g_h) cols(v).load_weights(a.w_next + g * a.wn_gs, b2[v]);
  }
  if (q0 < q1) {
    GradVec now[NV], next[AHEAD ? NV : 1];
    const auto load = [&](int row, auto &w) {
#pragma unroll
      for (int v = 0; v < NV; ++v) load_grad<BLOCK>(a, row, cols(v), w[v]);
    };
    if constexpr (AHEAD) load(min(q0 + rg, q1 - 1), next);
    GradRow r_next(a, min(q0 + rg, q1 - 1));
    int parity = 0;
    for (int first = q0; first < q1; first += R, parity ^= 1) {
      const int row = first + rg;
      GradRow r = r_next;
#pragma unroll
      for (int v = 0; v < NV; ++v) cols_[v].fresh();
      if constexpr (AHEAD) {
#pragma unroll
        for (int v = 0; v < NV; ++v) now[v] = next[v];
        if (first + R < q1) load(min(row + R, q1 - 1), next);
      } else {
        load(min(row, q1 - 1), now);
      }
      if (first + R < q1) r_next = GradRow(a, min(row + R, q1 - 1));
      float s[3] = {0.f, 0.f, 0.f};
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        cols(v).clear(now[v].gh);  // (then every sum's terms are 0, those of an infinite g_out too)
        cols(v).clear(now[v].go);
        if (BLOCK) cols(v).clear(now[v].y);
        grad_sums<BLOCK, T>(a, now[v], b1[v], b2[v], r, s);
      }
      row_sum<TPR>(s, buf[parity]);
      r.means(a, s);
      if (row >= q1) continue;  // (barriers are passed)
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (BLOCK) now[v].again();
#pragma unroll
      for (int v = 0; v < NV; ++v) grad_finish<BLOCK>(a, row, cols(v), now[v], b1[v], b2[v], r, d1[v], d2[v]);
    }
  }
  const GradPlace to(a, g, slot);
  const auto finish = [&](float *p, float(&d)[NV][VEC]) {
    if (!p) return;
    if constexpr (R > 1) {  // the rows' shares, in their order
      __syncthreads();
      if (rg > 0)
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
          for (int j = 0; j < VEC; ++j) shares[rg - 1][(v * VEC + j) * TPR + t] = d[v][j];
      __syncthreads();
      if (rg > 0) return;
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          for (int i = 0; i < R - 1; ++i) d[v][j] += shares[i][(v * VEC + j) * TPR + t];
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) cols(v).store_sums(p, d[v]);
  };
  finish(to.d1, d1);
  finish(to.d2, d2);
}

// The same for rows that no workgroup holds (or of less than a vector): the means
// of a piece's rows first, then its columns, each over all rows.
constexpr int kLongPiece = 128, kLongRows = 256;  // rows of a piece, and that it may have
template <typename T, bool BLOCK> __global__ void __launch_bounds__(256) residual_grad_long_kernel(ResidualGradArgs a) {
  constexpr int VEC = Vec16<T>::N, TPR = 256;
  __shared__ float buf[2][16][3];
  __shared__ float means[kLongRows][2];
  const int t = threadIdx.x, n = a.n;
  int g, q0, q1, slot;
  if (!grad_piece(a, g, q0, q1, slot)) return;
  const float *w1 = a.w_block ? a.w_block + g * a.wb_gs : nullptr, *w2 = a.g_h ? a.w_next + g * a.wn_gs : nullptr;
  GradVec w;
  float b1[VEC], b2[VEC];
#pragma unroll
  for (int j = 0; j < VEC; ++j) b1[j] = b2[j] = 1.f;
  for (int row = q0; row < q1; ++row) {
    GradRow r(a, row);
    float s[3] = {0.f, 0.f, 0.f};
    for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) {
      const Cols<T, false> c((int)i, n);
      if (w1) c.load_weights(w1, b1);
      if (w2) c.load_weights(w2, b2);
      load_grad<BLOCK>(a, row, c, w);
      grad_sums<BLOCK, T>(a, w, b1, b2, r, s);
    }
    row_sum<TPR>(s, buf[row & 1]);
    r.means(a, s);
    if (t == 0) {
      means[row - q0][0] = r.k2;
      means[row - q0][1] = r.k1;
    }
  }
  __syncthreads();
  const GradPlace to(a, g, slot);
  for (int64_t i = (int64_t)t * VEC; i < n; i += TPR * VEC) {
    const Cols<T, false> c((int)i, n);
    float d1[VEC], d2[VEC];
    if (w1) c.load_weights(w1, b1);
    if (w2) c.load_weights(w2, b2);
#pragma unroll
    for (int j = 0; j < VEC; ++j) d1[j] = d2[j] = 0.f;
    for (int row = q0; row < q1; ++row) {
      load_grad<BLOCK>(a, row, c, w);
      GradRow r(a, row);
      r.k2 = means[row - q0][0];
      r.k1 = means[row - q0][1];
      grad_finish<BLOCK>(a, row, c, w, b1, b2, r, d1, d2);
    }
    if (to.d1) c.store_sums(to.d1, d1);
    if (to.d2) c.store_sums(to.d2, d2);
  }
}

// The weights' gradients of a group of several pieces: 128 columns of both together a
// workgroup, four a thread and LANES threads a column that take every LANES-th
// piece; their shares meet in LDS.
constexpr int kJoinCols = 128;
template <int LANES>
__global__ void __launch_bounds__(kJoinCols / 4 * LANES) residual_join_kernel(ResidualGradArgs a, uint32_t blocks) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  __shared__ f32x4_t shares[LANES][kJoinCols / 4];
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
  const int in = threadIdx.x % (kJoinCols / 4), lane = threadIdx.x / (kJoinCols / 4);
  const int64_t all = 2 * (int64_t)a.n, c = (int64_t)(blockIdx.x - g * blocks) * kJoinCols + in * 4;
  const float *p = a.part + (int64_t)first * all + c;
  f32x4_t s = f32x4_t{0.f, 0.f, 0.f, 0.f};
  if (c + 4 <= all) {
#pragma unroll 4
    for (uint32_t k = lane; k < n; k += LANES) s += *(const f32x4_any *)(p + (int64_t)k * all);
  } else {
#pragma unroll
    for (int r = 0; r < 3; ++r)
      if (c + r < all)
        for (uint32_t k = lane; k < n; k += LANES) s[r] += p[(int64_t)k * all + r];
  }
  shares[lane][in] = s;
  __syncthreads();
  if (lane) return;
#pragma unroll
  for (int i = 1; i < LANES; ++i) s += shares[i][in];
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const bool second = c + r >= a.n;
    float *out = second ? a.dw_next : a.dw_block;  // (a partial of what is not asked for holds anything)
    if (c + r < all && out) out[second ? g * a.dwn_gs + (c + r - a.n) : g * a.dwb_gs + c + r] = s[r];
  }
}

// 16-byte vectors of a row; rows of less than one go with those that nothing holds.
int64_t vectors_of(int dtype, int n) {
  const int vec = dtype == GCPSL_BF16 ? 8 : 4;
  return n < vec ? INT32_MAX : (n + vec - 1) / vec;
}

template <typename T> hipError_t run(int dtype, const ResidualArgs &a, hipStream_t s) {
  const int64_t vectors = vectors_of(dtype, a.n);
  const auto launch = [&](auto kernel, int tpr) {
    // as many workgroups as the chip holds, of the same number of rows
    const int block = block_of(tpr);
    const int64_t at_once = block / tpr, most = kCUs * 2048 / block;
    const int64_t per = ((a.rows + most - 1) / most + at_once - 1) / at_once * at_once;
    hipLaunchKernelGGL(kernel, dim3((uint32_t)((a.rows + per - 1) / per)), dim3(block), 0, s, a, (int)per);
    return hipGetLastError();
  };
  if (vectors <= 16) return launch(residual_kernel<T, 16, 1>, 16);
  if (vectors <= 32) return launch(residual_kernel<T, 32, 1>, 32);
  if (vectors <= 64) return launch(residual_kernel<T, 64, 1>, 64);
  if (vectors <= 128) return launch(residual_kernel<T, 64, 2>, 64);
  if (vectors <= 256) return launch(residual_kernel<T, 256, 1>, 256);
  if (vectors <= 512) return launch(residual_kernel<T, 256, 2>, 256);
  if (vectors <= 1024) return launch(residual_kernel<T, 512, 2>, 512);
  if (vectors <= 2048) return launch(residual_kernel<T, 1024, 2>, 1024);
  hipLaunchKernelGGL(residual_long_kernel<T>, dim3((uint32_t)std::min<int64_t>(a.rows, 8 * kCUs)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Threads of a row in the gradient's kernels, 0 for those that nothing holds.
int grad_threads(int dtype, int n) {
  const int64_t vectors = vectors_of(dtype, n);
  for (int tpr : {16, 32, 64, 128, 256, 512, 1024})
    if (vectors <= tpr) return tpr;
  return dtype == GCPSL_F32 && vectors <= 2048 ? 1024 : 0;
}

template <typename T, bool BLOCK> hipError_t run_grad(int dtype, const ResidualGradArgs &a, hipStream_t s) {
  const int64_t blocks = a.rows / a.piece + a.G, joins = (2 * (int64_t)a.n + kJoinCols - 1) / kJoinCols * a.G;
  if (blocks > kMaxBlocks / 4 || joins > kMaxBlocks) return hipErrorInvalidConfiguration;  // (of up to 1,024 threads; 256)
  const int tpr = grad_threads(dtype, a.n);
  const auto launch = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((uint32_t)blocks), dim3(block_of(tpr)), 0, s, a);
    return hipGetLastError();
  };
  // Registers for the next rows' loads: not beside all that bf16 rows of a block need
  // (with their weights in LDS for it they were no faster).
  constexpr bool A = sizeof(T) == 4 || !BLOCK;
  hipError_t e;
  if (tpr == 16) e = launch(residual_grad_kernel<T, 16, 1, A, BLOCK>);
  else if (tpr == 32) e = launch(residual_grad_kernel<T, 32, 1, A, BLOCK>);
  else if (tpr == 64) e = launch(residual_grad_kernel<T, 64, 1, A, BLOCK>);
  else if (tpr == 128) e = launch(residual_grad_kernel<T, 128, 1, A, BLOCK>);
  else if (tpr == 256) e = launch(residual_grad_kernel<T, 256, 1, A, BLOCK>);
  else if (tpr == 512) e = launch(residual_grad_kernel<T, 512, 1, A, BLOCK>);
  else if (tpr == 1024 && vectors_of(dtype, a.n) <= 1024) e = launch(residual_grad_kernel<T, 1024, 1, A, BLOCK>);
  else if (tpr == 1024) {
    if constexpr (sizeof(T) == 4) e = launch(residual_grad_kernel<T, 1024, 2, false, BLOCK>);
    else e = hipErrorInvalidValue;  // (grad_threads gives fp32 rows only)
  }
  else e = launch(residual_grad_long_kernel<T, BLOCK>);
  if (e == hipSuccess && a.slots > 0 && (a.dw_block || a.dw_next)) {
    const auto join = [&](auto kernel, int lanes) {
      hipLaunchKernelGGL(kernel, dim3((uint32_t)joins), dim3(kJoinCols / 4 * lanes), 0, s, a, (uint32_t)(joins / a.G));
    };
    if (a.slots >= 64 * a.G && joins <= kMaxBlocks / 4) join(residual_join_kernel<32>, 32);
    else join(residual_join_kernel<8>, 8);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

// Rows of a piece: a few pieces less than the chip holds workgroups at once (16
// waves a CU), as groups round their number up or down and one more would be a
// round of its own (8,192 rows of 4 unequal groups, n 8,192, bf16: 324 us with as
// many, 234 so); a quarter of that where 16 rows are left, so that unequal ones end
// together (65,536 rows of 8 groups, n 256, bf16: 58 and 55 us).  Smaller ones
// cost more in partials (16,384 rows of 16 groups, n 4,096, bf16: 32 rows a piece
// 237 us, 16 rows 248).  Four rows at least for each of those that a workgroup
// takes at a time; us with at least 2, 4 and 8: 777 rows of 7 groups, n 1,001, fp32,
// 13.1, 13.9 and 17.7, n 4,096, bf16, 25.7, 22.5 and 27.2; 4,096 of 16, n 1,024, bf16,
// 23.8, 21.4 and 23.8; 2,000 of 16, n 4,096, bf16, 37.7, 37.5 and 34.9; 16,384 of 16, n
// 64, fp32, 11.4, 12.2 and 14.8.
GroupPieces residual_pieces(int dtype, int G, int64_t rows, int n) {
  const int tpr = grad_threads(dtype, n);
  const int64_t block = tpr ? block_of(tpr) : 256, full = kCUs * 1024 / block * 15 / 16,
                target = rows >= 64 * full ? 4 * full : full;
  const int64_t least = tpr ? 4 * block / tpr : 4;
  int64_t piece = std::max<int64_t>((rows + target - 1) / target, least);
  if (!tpr) piece = std::min<int64_t>(piece, kLongPiece);  // (a piece has at most 1.6 times as many rows)
  if (rows <= 2 * least) piece = std::max<int64_t>(rows, 1);  // one piece a group, and no join to launch
  // a group of p > 1 pieces has more than (p - 1/2) piece >= 3/4 p piece rows
  return {(int)piece, rows * 2 >= piece * 3 ? (int)(rows * 4 / (piece * 3)) : 0};
}

hipError_t launch_residual(int dtype, const ResidualArgs &a, hipStream_t s) {
  return dtype == GCPSL_BF16 ? run<bf16_t>(dtype, a, s) : run<float>(dtype, a, s);
}
hipError_t launch_residual_grad(int dtype, const ResidualGradArgs &a, hipStream_t s) {
  if (a.y) return dtype == GCPSL_BF16 ? run_grad<bf16_t, true>(dtype, a, s) : run_grad<float, true>(dtype, a, s);
  return dtype == GCPSL_BF16 ? run_grad<bf16_t, false>(dtype, a, s) : run_grad<float, false>(dtype, a, s);
}

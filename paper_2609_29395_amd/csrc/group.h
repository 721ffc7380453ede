// What the kernels of grouped products share: which rows a workgroup has, and
// what happens to a finished sum.
#pragma once

#include <algorithm>
#include <utility>

#include "ops.h"
#include "runtime.h"

constexpr uint32_t kCUs = 256;

// Row stride up to which the offsets within 256 rows stay below 2^31 bytes.
constexpr int64_t kMaxTileLd = 1 << 22;

bool group_tile_ok(int dtype, const GroupArgs &a, int mode);
hipError_t launch_group_tile(int mode, const GroupArgs &a, hipStream_t s);
bool group_few_ok(int dtype, const GroupArgs &a, int mode);
hipError_t launch_group_few(int dtype, int mode, const GroupArgs &a, hipStream_t s);
bool group_mid_ok(int dtype, const GroupArgs &a, int mode);
hipError_t launch_group_mid(int mode, const GroupArgs &a, hipStream_t s);
bool group_f32_ok(const GroupArgs &a, int mode);
hipError_t launch_group_f32(int mode, const GroupArgs &a, hipStream_t s);
bool group_f32_deep_ok(const GroupArgs &a, int mode);
// fp32 weight gradients [n][k] of G groups, `rows` in all, that tiles of 64 x 64
// take: at most one a CU, and so few rows for each of the pieces that fit beside
// each other that the larger tiles' rate does not pass their quicker beginning
// and end.  us so and with 128 x 128: 1 group of 813 rows, 64 -> 256, 11 and 19;
// 1 of 2,000, 1024 -> 1024 (1 piece), 41 and 50; 1 of 10,000, 512 -> 512 (4 of
// 2,500), 50 and 57; 1 of 20,000 (4 of 5,000), 97 and 80.
inline bool group_f32_deep_grad(int G, int64_t rows, int n, int k) {
  const int64_t tiles = (int64_t)((n + 63) / 64) * ((k + 63) / 64);
  return tiles * G <= kCUs && rows <= 2560 * (kCUs / tiles);
}
hipError_t launch_group_f32_deep(int mode, const GroupArgs &a, hipStream_t s);

#define GROUP_DEVICE __device__ __forceinline__

// Rows [begin, end) of group g, inside [0, rows) whatever the offsets hold.
GROUP_DEVICE void group_rows(const int32_t *off, int g, int rows, int &begin, int &end) {
  begin = min(max(off[g], 0), rows);
  end = min(max(off[g + 1], begin), rows);
}

// A group of `count` rows in tiles of bm rows, or (pieces) in about count / bm
// equal parts, at least one.
template <bool PIECES> GROUP_DEVICE uint32_t parts_of(int count, int bm) {
  return PIECES ? max(((uint32_t)count + (uint32_t)bm / 2u) / (uint32_t)bm, 1u)
                : (uint32_t)(count + bm - 1) / (uint32_t)bm;
}

// Row tiles (bm rows, none spans groups) or pieces of groups [base, base +
// 64), one group a lane: its rows, the parts before it (`before` are those
// before the first) and its own.  Returns the parts up to the last.
struct LaneTiles {
  int begin, end;
  uint32_t first, tiles;
};
// v moved across lanes by DPP control CTRL, 0 where nothing arrives or the row of 16 is not in ROWS.
template <int CTRL, int ROWS> GROUP_DEVICE uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
// Inclusive sum over the 64 lanes, all of them active: within rows of 16 by shifts of 1, 2, 4 and 8, then the row
// before (into rows 1 and 3) and the two before (rows 2 and 3) from their last lane.  (Shuffles go through the LDS: a
// launch took 0.3 to 0.5 us longer with them.)
GROUP_DEVICE uint32_t lane_scan(uint32_t v) {
  v += dpp<0x111, 0xf>(v);
  v += dpp<0x112, 0xf>(v);
  v += dpp<0x114, 0xf>(v);
  v += dpp<0x118, 0xf>(v);
  v += dpp<0x142, 0xa>(v);
  v += dpp<0x143, 0xc>(v);
  return v;
}
// Lane i's v, i the same in every lane.
GROUP_DEVICE int of_lane(int v, int i) {
  return __builtin_amdgcn_readlane(v, __builtin_amdgcn_readfirstlane(i));
}

template <bool PIECES = false>
GROUP_DEVICE uint32_t lane_tiles(const int32_t *off, int G, int rows, int bm, int base, uint32_t before, LaneTiles &l) {
  const int i = base + (int)(threadIdx.x & 63);
  l.begin = l.end = 0;
  l.tiles = 0;
  if (i < G) {
    group_rows(off, i, rows, l.begin, l.end);
    l.tiles = parts_of<PIECES>(l.end - l.begin, bm);
  }
  const uint32_t sum = lane_scan(l.tiles);
  l.first = before + sum - l.tiles;
  return before + (uint32_t)of_lane((int)sum, 63);
}

// Tile t of MT x NT in blocks of 8 row tiles by all column tiles, rows
// fastest: 32 tiles in order are about 8 x 4 and share their operands.
GROUP_DEVICE void block_order(uint32_t t, uint32_t MT, uint32_t NT, int &mt, int &nt) {
  const uint32_t block = t < 8u * NT ? 0u : t / (8u * NT), in = t - block * 8u * NT;
  const uint32_t high = min(8u, MT - block * 8u);  // row tiles of this block
  const uint32_t n = high == 8u ? in >> 3 : in / high;
  nt = __builtin_amdgcn_readfirstlane((int)n);
  mt = __builtin_amdgcn_readfirstlane((int)(block * 8u + in - n * high));
}

// Lane whose group has part t, -1 if none.  (A part is checked against its
// group's own ones: offsets that decrease can make groups overlap, but no row
// outside [0, rows) is touched.)
GROUP_DEVICE int lane_of(const LaneTiles &l, uint32_t t) {
  const uint64_t hit = __ballot(t - l.first < l.tiles);
  return __ffsll((unsigned long long)hit) - 1;
}

// Piece and tile of workgroup b of a weight gradient of `tiles` tiles: the
// piece's group, rows [q0, q1) and place among the partials (-1 if the group is
// one piece); false if there is none.  Every XCD has an eighth of every piece's
// tiles, so that unequal groups do not make unequal XCDs.  (Each XCD beginning
// with another piece, so that their writing did not coincide, cost more in
// operands read from memory: 716 against 640 us for 16 groups of 1,024 rows.)
// (Offsets that decrease can make more partials than there is room for: those
// are left out.)
GROUP_DEVICE bool piece_of(const GroupArgs &a, uint32_t tiles, uint32_t b, int &g, int &q0, int &q1, int &slot,
                           uint32_t &tile) {
  LaneTiles l;
  const uint32_t first64 = lane_tiles<true>(a.off, a.G, a.Q, a.piece, 0, 0, l);
  uint32_t P = first64;
  for (int base = 64; base < a.G; base += 64) {
    LaneTiles m;
    P = lane_tiles<true>(a.off, a.G, a.Q, a.piece, base, P, m);
  }
  P = __builtin_amdgcn_readfirstlane(P);
  const uint32_t t = b / tiles;
  if (t >= P) return false;
  tile = xcd_swizzle(b - t * tiles, tiles);
  uint32_t before = first64, slots = 0, own = l.tiles > 1 ? l.tiles : 0, sum = lane_scan(own);
  int base = 0, i = lane_of(l, t);
  while (i < 0) {
    base += 64;
    if (base >= a.G) return false;
    slots += (uint32_t)of_lane((int)sum, 63);
    before = lane_tiles<true>(a.off, a.G, a.Q, a.piece, base, before, l);
    own = l.tiles > 1 ? l.tiles : 0;
    sum = lane_scan(own);
    i = lane_of(l, t);
  }
  const int begin = of_lane(l.begin, i), end = of_lane(l.end, i);
  const int n = of_lane((int)l.tiles, i), k = (int)(t - (uint32_t)of_lane((int)l.first, i));
  const int part = ((end - begin + n - 1) / n + 63) / 64 * 64;
  const int64_t at = begin + (int64_t)k * part;  // may pass the group's end, and 31 bits
  g = __builtin_amdgcn_readfirstlane(base + i);
  q0 = __builtin_amdgcn_readfirstlane((int)min(at, (int64_t)end));
  q1 = __builtin_amdgcn_readfirstlane((int)min(at + part, (int64_t)end));
  slot = __builtin_amdgcn_readfirstlane(n > 1 ? (int)(slots + (uint32_t)of_lane((int)(sum - own), i)) + k : -1);
  return slot < a.slots;
}

// Group, rows [row0, row1) and column tile of workgroup b of a product whose
// row tiles (bm rows) the offsets make; false if it has none.  The tiles are
// dealt to the XCDs in contiguous runs of block_order, so that an XCD's
// workgroups share their operands in its L2.  The tiles past the last whole
// round of one per CU are halved if they still make no more than a round: a CU
// that takes one tile more than the others makes them wait for half as long.
// (What a result is the sum of, and in which order, does not depend on it.)
template <bool HALVES = true>
GROUP_DEVICE bool tile_of(const int32_t *off, int G, int rows, int bm, int NT_, uint32_t b, int &g, int &row0, int &row1,
                          int &nt) {
  LaneTiles l;
  const uint32_t NT = (uint32_t)NT_, first64 = lane_tiles(off, G, rows, bm, 0, 0, l);
  uint32_t MT = first64;
  for (int base = 64; base < G; base += 64) {
    LaneTiles m;
    MT = lane_tiles(off, G, rows, bm, base, MT, m);
  }
  MT = __builtin_amdgcn_readfirstlane(MT);
  const uint32_t all = MT * NT, full = all / kCUs * kCUs, rest = all - full;
  uint32_t t = b;
  int half = -1, mt;
  if (b < full) {
    t = xcd_swizzle(b, full);
  } else if (HALVES && 2 * rest <= kCUs) {
    if (b >= full + 2 * rest) return false;
    t = xcd_swizzle(b - full, 2 * rest);
    half = __builtin_amdgcn_readfirstlane((int)(t & 1));
    t = full + (t >> 1);
  } else {
    if (b >= all) return false;
    t = full + xcd_swizzle(b - full, rest);
  }
  block_order(t, MT, NT, mt, nt);
  uint32_t before = first64;
  int base = 0, i = lane_of(l, (uint32_t)mt);
  while (i < 0) {
    base += 64;
    if (base >= G) return false;
    before = lane_tiles(off, G, rows, bm, base, before, l);
    i = lane_of(l, (uint32_t)mt);
  }
  g = __builtin_amdgcn_readfirstlane(base + i);
  row0 = __builtin_amdgcn_readfirstlane(of_lane(l.begin, i) + (mt - of_lane((int)l.first, i)) * bm);
  row1 = __builtin_amdgcn_readfirstlane(min(of_lane(l.end, i), row0 + bm));
  if (half == 0) row1 = min(row1, row0 + bm / 2);
  if (half == 1) row0 += bm / 2;
  return row0 < row1;
}
// Workgroups of such a launch: as many tiles as any offsets can make, and the
// halves.
inline int64_t tile_blocks(int64_t rows, int G, int bm, int64_t NT) {
  return (rows / bm + std::min<int64_t>(G, rows)) * NT + kCUs / 2;
}

// Four consecutive columns c .. c + 3 of row m of the result (forward, input
// gradient): bias, ReLU (a NaN stays one), dropout or gate.
template <typename T, int MODE>
GROUP_DEVICE void epilogue(const GroupArgs &a, int m, int c, const float *bias, const float *gate, float (&v)[4]) {
  if constexpr (MODE == GROUP_FWD) {
    uint64_t word = 0;
    if (a.drop.thr) word = drop_word(a.drop.key, m, (a.N + 3) >> 2, c >> 2);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[r] += bias[r];
      if (a.relu) v[r] = v[r] <= 0.f ? 0.f : v[r];
      if (a.drop.thr) v[r] = drop_keeps(word, r, a.drop.thr) ? v[r] * a.drop.scale : 0.f;
    }
  } else if (a.gate) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = gate[r] > 0.f ? v[r] * a.drop.scale : 0.f;
  }
}

typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// One rounding and a store, all four columns inside the result (their number
// is a multiple of 4); any alignment.
template <typename T, int MODE, typename V>
GROUP_DEVICE void finish4(const GroupArgs &a, int g, int m, int c, const V &acc) {
  float v[4] = {acc[0], acc[1], acc[2], acc[3]}, bias[4] = {0.f, 0.f, 0.f, 0.f}, gate[4];
  if constexpr (MODE == GROUP_FWD) {
    if (a.bias) {
      const f32x4_any b = *(const f32x4_any *)(a.bias + g * a.bias_gs + c);
#pragma unroll
      for (int r = 0; r < 4; ++r) bias[r] = b[r];
    }
  } else if (a.gate) {
    const T *p = (const T *)a.gate + (int64_t)m * a.ldg + c;
    if constexpr (sizeof(T) == 2) {
      const u32x2_any b = *(const u32x2_any *)p;
#pragma unroll
      for (int r = 0; r < 4; ++r) gate[r] = __uint_as_float(r & 1 ? b[r >> 1] & 0xffff0000u : b[r >> 1] << 16);
    } else {
      const f32x4_any b = *(const f32x4_any *)p;
#pragma unroll
      for (int r = 0; r < 4; ++r) gate[r] = b[r];
    }
  }
  epilogue<T, MODE>(a, m, c, bias, gate, v);
  T *out = (T *)a.out + (int64_t)m * a.ldo + c;
  if constexpr (sizeof(T) == 2)
    *(u32x2_any *)out = u32x2_any{pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3])};
  else
    *(f32x4_any *)out = f32x4_any{v[0], v[1], v[2], v[3]};
}

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T> struct Vec16;  // the elements of a 16-byte vector
template <> struct Vec16<bf16_t> {
  static constexpr int N = 8;
  static GROUP_DEVICE float at(const u32x4_any &v, int j) {
    return __uint_as_float(j & 1 ? v[j >> 1] & 0xffff0000u : v[j >> 1] << 16);
  }
};
template <> struct Vec16<float> {
  static constexpr int N = 4;
  static GROUP_DEVICE float at(const u32x4_any &v, int j) { return __uint_as_float(v[j]); }
};

// The same where columns may lie outside.
template <typename T, int MODE, typename V>
GROUP_DEVICE void finish(const GroupArgs &a, int g, int m, int c, const V &acc) {
  if (c + 4 <= a.N) return finish4<T, MODE>(a, g, m, c, acc);
  float v[4] = {acc[0], acc[1], acc[2], acc[3]}, bias[4] = {0.f, 0.f, 0.f, 0.f}, gate[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (c + r < a.N) {
      if constexpr (MODE == GROUP_FWD) {
        if (a.bias) bias[r] = a.bias[g * a.bias_gs + c + r];
      } else {
        if (a.gate) gate[r] = ElemT<T>::to_f(((const T *)a.gate)[(int64_t)m * a.ldg + c + r]);
      }
    }
  epilogue<T, MODE>(a, m, c, bias, gate, v);
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (c + r < a.N) ((T *)a.out)[(int64_t)m * a.ldo + c + r] = ElemT<T>::from_f(v[r]);
}

// A thread's 16 bytes of columns, c on (EDGES false: all inside or all outside), of ROWS rows m0, m0 + step, ... below
// m1: the bias and the gate's rows are loaded together before the sums are
// there, so that no row waits for its own.
template <typename T, int MODE, int ROWS, bool EDGES = true> struct FinishRows {
  static constexpr int VEC = Vec16<T>::N;
  int m0, step, m1, c;
  float bias[VEC];
  u32x4_any gate[ROWS];
  GROUP_DEVICE FinishRows(const GroupArgs &a, int g, int m0_, int step_, int m1_, int c_)
      : m0(m0_), step(step_), m1(m1_), c(c_) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) bias[j] = 0.f;
    if (c >= a.N) return;
    const bool whole = !EDGES || c + VEC <= a.N;  // else what is past the columns is taken as the last one
    if constexpr (MODE == GROUP_FWD) {
      if (!a.bias) return;
      const float *p = a.bias + g * a.bias_gs;
      if (whole) {
#pragma unroll
        for (int j = 0; j < VEC; j += 4) {
          const f32x4_any b = *(const f32x4_any *)(p + c + j);
#pragma unroll
          for (int r = 0; r < 4; ++r) bias[j + r] = b[r];
        }
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) bias[j] = p[min(c + j, a.N - 1)];
      }
    } else if (a.gate) {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const T *p = (const T *)a.gate + (int64_t)min(m0 + i * step, m1 - 1) * a.ldg;
        if (whole) {
          gate[i] = *(const u32x4_any *)(p + c);
        } else {
          const auto bits = [&](int j) -> uint32_t {
            const T v = p[min(c + j, a.N - 1)];
            if constexpr (sizeof(T) == 2) return v;
            else return __float_as_uint(v);
          };
#pragma unroll
          for (int j = 0; j < 4; ++j) gate[i][j] = sizeof(T) == 2 ? bits(2 * j) | bits(2 * j + 1) << 16 : bits(j);
        }
      }
    }
  }
  // the sums of row i, columns 4 j on, at acc(i, j)
  template <typename F> GROUP_DEVICE void store_row(const GroupArgs &a, int i, const u32x4_any &gates, const F &acc) const {
    const int m = m0 + i * step;
    if (m >= m1) return;
    u32x4_any o;
#pragma unroll
    for (int j = 0; j < VEC / 4; ++j) {
      const f32x4_any v = acc(i, j);
      float x[4], b[4], gt[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[r] = v[r];
        b[r] = bias[4 * j + r];
        gt[r] = MODE == GROUP_FWD ? 0.f : Vec16<T>::at(gates, 4 * j + r);
      }
      epilogue<T, MODE>(a, m, c + 4 * j, b, gt, x);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (sizeof(T) == 4) o[r] = __float_as_uint(x[r]);
        else if (r & 1) o[2 * j + (r >> 1)] = pack2_bf16(x[r - 1], x[r]);
      }
    }
    T *out = (T *)a.out + (int64_t)m * a.ldo + c;
    if (!EDGES || c + VEC <= a.N) {
      *(u32x4_any *)out = o;
    } else {
#pragma unroll
      for (int j = 0; j < VEC - 1; ++j)
        if (c + j < a.N) {
          if constexpr (sizeof(T) == 2) out[j] = (T)(o[j >> 1] >> (j & 1) * 16);
          else out[j] = __uint_as_float(o[j]);
        }
    }
  }
  template <typename F> GROUP_DEVICE void store(const GroupArgs &a, const F &acc) const {
    if (c >= a.N) return;
    if constexpr (MODE == GROUP_FWD) {  // (copies of the draws' code for every row cost more in fetching it)
#pragma unroll 1
      for (int i = 0; i < ROWS; ++i) store_row(a, i, u32x4_any{}, acc);
    } else {
#pragma unroll
      for (int i = 0; i < ROWS; ++i) store_row(a, i, gate[i], acc);
    }
  }
};

// Four columns of a weight gradient, to its place or (slot >= 0) to a partial.
template <typename V> GROUP_DEVICE void store_grad(const GroupArgs &a, int g, int slot, int m, int c, const V &acc) {
  float *out = slot >= 0 ? a.part + ((int64_t)slot * a.M + m) * a.N + c
                         : (float *)a.out + g * a.out_gs + (int64_t)m * a.ldo + c;
  if (c + 4 <= a.N) {
    *(f32x4_any *)out = f32x4_any{acc[0], acc[1], acc[2], acc[3]};
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (c + r < a.N) out[r] = acc[r];
  }
}
// Eight values in a tree, which a bias gradient adds to the sum it carries.  (1,024
// normal values in the 128 x 128 tiles' order: off by 1.6e-7 of the result in the
// mean square so, by 4.0e-7 one after another, for as many additions.)
GROUP_DEVICE float sum8(const float (&v)[8]) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}
GROUP_DEVICE void store_bias_grad(const GroupArgs &a, int g, int slot, int m, float v) {
  if (slot >= 0) a.part_db[(int64_t)slot * a.M + m] = v;
  else a.db[g * a.db_gs + m] = v;
}

// Workgroups of a weight gradient of `tiles` tiles a piece: as many pieces as
// any offsets can make.
inline int64_t piece_blocks(const GroupArgs &a, int64_t tiles) { return ((int64_t)a.Q / a.piece + a.G) * tiles; }

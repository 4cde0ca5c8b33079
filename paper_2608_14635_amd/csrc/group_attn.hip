// Attention over the retained arena, a group's shared prefix read once (kvr_attention.h).
//
// Query rows that share a kv head are columns: column i g + h is row i of q head h of the
// group of heads.  There are two kinds of entities: a group of requests, whose rows all see
// the group's prefix, and a request, whose rows see what follows it.  An entity's columns in
// tiles of 16 NT make items, the work of an item comes in units of positions.  Every
// workgroup takes an equal stretch of the units of all items, entity after entity, whatever
// the lengths (they are known on the device alone); its four waves share out each item's part
// of it and merge their sums in LDS.  A second kernel joins what is there of a column: the
// workgroups' sums over its group's prefix and over its own positions.
//
// A unit in a wave's registers, lane (q, c) = (lane / 16, lane % 16):
//   S^T = K Q^T, 16 positions a tile: the lane gets the scores of positions 4q .. 4q+3 for
//   column c.
//   Online softmax per column, exp2 domain, rescaled only where the maximum rose by more
//   than 2^SLACK.
//   O^T = V^T P^T: the lane's weights are the B operand as they are; for the A operand it
//   holds dims c d/16 .. of its own positions 4q .., which in bf16 it pairs into that
//   operand's order.  It gets d/4 neighbouring dims of column c: sums, maxima and weights of
//   a column stay in its four lanes.
//   In bf16 (v_mfma_f32_16x16x32_bf16, units of 32 positions) a weight enters the product as
//   a bf16 number and the bf16 rest, 2^-17 of it lost: rounding it once would cost more
//   than the output's own rounding where few positions weigh.  In fp32 (units of 16,
//   v_mfma_f32_16x16x4_f32) nothing is rounded.
//   A weight may be 2^SLACK and 2^31 of them add up, so the sums of large V could pass the
//   largest fp32 number where their quotient, which lies between the V's, does not: all
//   weights, and their sum, are taken 2^-LIFT as large.  In bf16 the maxima are LIFT too high
//   for it (exponents are then rounded to 2^-19, below the 2^-17 above), in fp32 weights are
//   multiplied.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "host.h"
#include "kvr_attention.h"

namespace kvr {
namespace {

constexpr int GA_NT = 256, WAVES = GA_NT / 64;
constexpr float SLACK = 8.0f, LIFT = 40.0f;  // log2 units
constexpr int MOST_ROWS = 1 << 24;           // query rows, requests and groups of a call
constexpr int START = 4;                     // units that an item's start counts as
constexpr int CUS = 256;
constexpr int KNOWN = 512;                   // groups whose offsets are kept in LDS

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

template <typename T> struct Unit;
template <> struct Unit<bf16_t> { static constexpr int POS = 32; };
template <> struct Unit<float> { static constexpr int POS = 16; };

// What the second kernel has to know of an entity: where its items' units begin, what each
// counts, its first item among its kind, its first query row and its columns, its request's group.
struct Entity {
  uint32_t base, item;
  int first, row, cols, group, pad[2];
};
struct Plan {
  uint32_t size, longer, workers, pad[5];
};

struct GroupAttnParams {
  const char *plane_k, *plane_v;
  int64_t row_bytes;             // of a slot: nkv d elements
  uint32_t num_blocks;
  int block_size;
  uint32_t block_inv;            // ceil(2^16 / block_size) where that is below 32, else 0: n / block_size of n < 64
  const char* q;
  char* out;
  int64_t q_stride, out_stride;  // bytes
  const int32_t* q_offsets;      // null: row r is request r's
  int rows;
  const int32_t* lens;
  const int32_t* tables;
  int R, max_blocks;
  const int32_t* group_offsets;
  const int32_t* prefix_lens;
  int G;
  int nkv, g;                    // q heads of a kv head
  uint32_t g_inv;                // ceil(2^32 / g), 0 for g = 1: n / g of n < 2^28 is the product's high half
  int max_query;
  int most_len;                  // positions of a request: max_len, or what its table holds
  int workers;                   // workgroups of a kv head
  Plan* plan;
  Entity* entities;              // [G + R]
  // sums of kinds 0 (prefixes) and 1: [nkv][slots][cols][ROW]
  float* part[2];
  int part_cols[2];
  int64_t slots[2];
};

__device__ __forceinline__ int by_g(const GroupAttnParams& p, int n) {
  return p.g_inv ? (int)__umulhi((uint32_t)n, p.g_inv) : n;
}
__device__ __forceinline__ int clamp_to(int v, int lo, int hi) { return max(lo, min(v, hi)); }
// Inclusive sums over the wave's lanes: within rows of 16, then the rows' last into those
// behind.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);   // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);   // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);   // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return v;
}
// a / b of whole numbers: a correctly rounded quotient of such small ones never reaches
// the next whole number
__device__ __forceinline__ uint32_t quotient(uint32_t a, uint32_t b) { return (uint32_t)((double)a / (double)b); }
// The maximum, the sum over the four lanes (q, c) of a c.
__device__ __forceinline__ float max_over_q(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_over_q(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// All units in `workers` stretches, the first `longer` of them a unit longer.
struct Stretches {
  uint32_t size, longer, workers;
  __device__ __forceinline__ Stretches(uint32_t most, uint32_t total) {
    workers = min(most, total);
    size = total ? quotient(total, workers) : 0;
    longer = total - size * workers;
  }
  __device__ __forceinline__ explicit Stretches(const Plan& p) : size(p.size), longer(p.longer), workers(p.workers) {}
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * size + min(w, longer); }
  __device__ __forceinline__ int holder(uint32_t u) const {  // whose unit u is
    const uint32_t head = longer * (size + 1);
    return (int)(u < head ? quotient(u, size + 1) : longer + quotient(u - head, size));
  }
};

// A request's query rows, and the position after the last of them.
struct Rows {
  int row, all, used, end;  // used: at most max_query of all
};
__device__ __forceinline__ Rows rows_of(const GroupAttnParams& p, int r) {
  Rows x{r, 1, 1, 0};
  if (p.q_offsets) {
    x.row = clamp_to(p.q_offsets[r], 0, p.rows);
    x.all = max(min(p.q_offsets[r + 1], p.rows) - x.row, 0);
    x.used = min(x.all, p.max_query);
  }
  x.end = max(p.lens[r], 0) - (x.all - x.used);  // the rows left out are the last ones
  return x;
}

// An entity: columns that see positions lo .. hi - 1 through a table.
struct Shape {
  int row, cols, lo, hi, table, group;
  int tiles;      // of columns; 0: nothing to do
  uint32_t item;  // what an item counts: its units and its start
  __device__ __forceinline__ uint32_t units() const { return (uint32_t)tiles * item; }
};

// Group offsets, of the first KNOWN groups in LDS.
struct Groups {
  const int32_t* lds;
  __device__ __forceinline__ int offset(const GroupAttnParams& p, int e) const {
    return p.G < KNOWN ? lds[e] : p.group_offsets[e];
  }
  // The group that request r is in, -1: none.  One of a single request shares nothing.
  __device__ __forceinline__ int of(const GroupAttnParams& p, int r) const {
    if (p.G == 0) return -1;
    int a = 0, b = p.G - 1;
    while (a < b) {
      const int m = (a + b + 1) / 2;
      if (offset(p, m) <= r) a = m;
      else b = m - 1;
    }
    const int lo = clamp_to(offset(p, a), 0, p.R), hi = clamp_to(offset(p, a + 1), lo, p.R);
    return r >= lo && r < hi && hi - lo > 1 ? a : -1;
  }
};

template <int COLS, int POS>
__device__ __forceinline__ Shape finish_shape(const GroupAttnParams& p, Shape s) {
  const int n = s.hi - s.lo;
  s.tiles = n > 0 ? (int)(((int64_t)s.cols + COLS - 1) / COLS) : 0;
  s.item = (uint32_t)(((int64_t)max(n, 0) + POS - 1) / POS) + START;
  return s;
}
template <int COLS, int POS>
__device__ __forceinline__ Shape shape_of(const GroupAttnParams& p, const Groups& groups, int e) {
  Shape s{};
  s.group = -1;
  if (e < p.G) {
    const int r0 = clamp_to(groups.offset(p, e), 0, p.R), r1 = clamp_to(groups.offset(p, e + 1), r0, p.R);
    s.table = r0;
    s.hi = r1 - r0 > 1 ? clamp_to(p.prefix_lens[e], 0, p.most_len) : 0;
    if (s.hi > 0) {
      s.row = p.q_offsets ? clamp_to(p.q_offsets[r0], 0, p.rows) : r0;
      s.cols = ((p.q_offsets ? clamp_to(p.q_offsets[r1], s.row, p.rows) : r1) - s.row) * p.g;
    }
    return finish_shape<COLS, POS>(p, s);
  }
  s.table = e - p.G;
  const Rows x = rows_of(p, s.table);
  s.row = x.row;
  s.cols = x.used * p.g;
  s.group = groups.of(p, s.table);
  s.hi = clamp_to(x.end, 0, p.most_len);
  s.lo = s.group >= 0 ? clamp_to(p.prefix_lens[s.group], 0, s.hi) : 0;
  return finish_shape<COLS, POS>(p, s);
}

// Positions that a query row of a prefix's columns sees.
__device__ __forceinline__ int limit_in_group(const GroupAttnParams& p, const Groups& groups, int e, int row) {
  if (!p.q_offsets) return p.lens[row];
  const int r0 = clamp_to(groups.offset(p, e), 0, p.R), r1 = clamp_to(groups.offset(p, e + 1), r0, p.R);
  int a = r0, b = max(r1 - 1, r0);
  // the last request whose rows begin at or before it
  while (a < b) {
    const int m = (a + b + 1) / 2;
    if (p.q_offsets[m] <= row) a = m;
    else b = m - 1;
  }
  const Rows x = rows_of(p, a);
  return max(p.lens[a], 0) - x.all + (row - x.row) + 1;
}

// Floats of a partial's row: d sums, a maximum and a sum of weights, on boundaries of 16 bytes.
template <int D>
constexpr int ROW = D + 4;

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// N consecutive values of a sum as they go out.
template <typename T, int N>
__device__ __forceinline__ void store_out(T* dst, const float* v) {
  if constexpr (sizeof(T) == 2) {
    static_assert(N % 4 == 0, "whole words");
    typedef uint32_t u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<u32x2_a4*>(dst + i) = u32x2_a4{pack_bf16(v[i], v[i + 1]), pack_bf16(v[i + 2], v[i + 3])};
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) dst[i] = v[i];
  }
}

// Keys and values of a unit in a lane's registers.  bf16: K words of two tiles' position c,
// dims 32 kk + 8 q ..; V words of positions 4q + i of both tiles, dims 8 c ..  fp32: one tile, K's
// dims q d/4 .., V's c d/16 ...
template <typename T, int D> struct Regs;
template <int D> struct Regs<bf16_t, D> {
  static constexpr int TILES = 2, NK = D / 32, NV = 4 * TILES;
  u32x4 k[TILES][NK];
  u32x4 v[NV];
};
template <int D> struct Regs<float, D> {
  static constexpr int TILES = 1, NK = D / 16, NV = 4;
  static constexpr int VW = D / 16;  // floats of a position
  f32x4 k[TILES][NK];
  float v[NV][VW];
};

// A part of an item: its unit range of a wave, and the columns.
template <typename T, int D, int NT>
struct Part {
  using R = Regs<T, D>;
  static constexpr int POS = Unit<T>::POS, TILES = R::TILES, NS = 4 * TILES, JN = D / 16;
  f32x4 o[NT][JN];        // [j][r]: dim q d/4 + r d/16 + j of column c
  float top[NT], l[NT];   // what weights are relative to; the lane's own weights' sum
};

// The arena slots of a stretch of positions, 64 blocks' table entries in a wave's lanes.
struct Table {
  const int32_t* entries;
  int max_blocks;
  int first;   // block of lane 0's entry
  int mine;
  __device__ __forceinline__ void load(int block, int lane) {
    first = block;
    mine = (uint32_t)(block + lane) < (uint32_t)max_blocks ? entries[block + lane] : -1;
  }
};

template <typename T, int D, int NT>
__device__ void attend_part(const GroupAttnParams& p, const Groups& groups, const Shape& s, int entity, int tile,
                            int cols_tile, int first, int upto, int kvh, Part<T, D, NT>& x) {
  using R = Regs<T, D>;
  constexpr int POS = Unit<T>::POS, TILES = R::TILES, NS = 4 * TILES, JN = D / 16;
  const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    x.top[nt] = -INFINITY;
    x.l[nt] = 0.0f;
#pragma unroll
    for (int j = 0; j < JN; ++j) x.o[nt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  if (first >= upto) return;
  // ---- queries, and the positions that each column sees ----
  typename std::conditional<sizeof(T) == 2, u32x4, f32x4>::type qr[NT][R::NK];
  int limit[NT], all = s.hi, some = 0;
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int cc = tile + nt * 16 + c, i = by_g(p, min(cc, s.cols - 1));
    const bool there = nt * 16 + c < cols_tile;
    const char* src = p.q + (int64_t)(s.row + i) * p.q_stride + (int64_t)(kvh * p.g + min(cc, s.cols - 1) - i * p.g) * D * sizeof(T);
#pragma unroll
    for (int kk = 0; kk < R::NK; ++kk) {
      if constexpr (sizeof(T) == 2) {
        qr[nt][kk] = there ? (u32x4)*reinterpret_cast<const u32x4_a4*>(src + kk * 64 + q * 16) : u32x4{0, 0, 0, 0};
      } else {
        qr[nt][kk] = there ? (f32x4)*reinterpret_cast<const f32x4_a4*>(src + (q * (D / 4) + kk * 4) * 4)
                           : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
    }
    int lim;
    if (entity < p.G) {
      lim = limit_in_group(p, groups, entity, s.row + i);
    } else {
      const Rows y = rows_of(p, s.table);
      lim = max(p.lens[s.table], 0) - y.all + i + 1;
    }
    limit[nt] = clamp_to(lim, 0, s.hi);
    all = there ? min(all, limit[nt]) : all;
    some = there ? max(some, limit[nt]) : some;
  }
#pragma unroll
  for (int o = 1; o < 16; o *= 2) {
    all = min(all, __shfl_xor(all, o, 64));
    some = max(some, __shfl_xor(some, o, 64));
  }
  all = __builtin_amdgcn_readfirstlane(all);
  some = __builtin_amdgcn_readfirstlane(some);
  upto = min(upto, (int)(((int64_t)max(some - s.lo, 0) + POS - 1) / POS));
  if (first >= upto) return;

  // ---- addresses ----
  const int B = p.block_size;
  const int pos0 = s.lo + first * POS;
  int blk = pos0 / B, off = pos0 - blk * B;  // of the unit to be loaded next
  Table table{p.tables + (int64_t)s.table * p.max_blocks, p.max_blocks, 0, 0};
  table.load(blk, lane);
  const char* head_k = p.plane_k + (int64_t)kvh * D * sizeof(T);
  const char* head_v = p.plane_v + (int64_t)kvh * D * sizeof(T);
  R u;
  uint32_t valid = 0;  // bit i: position i of the lane's own NS is there
  bool whole = true;   // every position of the unit is
  int next = pos0;
  // the unit's slots: lane x mod POS has position x's, -1: not there
  const auto slots_of_unit = [&]() {
    const int at = off + lane % POS;
    int n;
    if (p.block_inv) {
      n = (int)((uint32_t)at * p.block_inv >> 16);
    } else {
      n = at >= B ? 1 : 0;
    }
    // the unit's last block
    const int last = p.block_inv ? (int)((uint32_t)(off + POS - 1) * p.block_inv >> 16) : off + POS - 1 >= B ? 1 : 0;
    if (blk + last - table.first >= 64) table.load(blk, lane);
    const int entry = __shfl(table.mine, blk + n - table.first, 64);
    const int slot = (uint32_t)entry < p.num_blocks && (uint32_t)(next + lane % POS) < (uint32_t)some ? entry * B + (at - n * B) : -1;
    next += POS;
    off += POS;
    const int step = p.block_inv ? (int)((uint32_t)off * p.block_inv >> 16) : off >= B ? 1 : 0;
    blk += step;
    off -= step * B;
    return slot;
  };
  const auto load_k = [&](int slot) {
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int mine = max(__shfl(slot, t * 16 + c, 64), 0);
      const char* src = head_k + mine * p.row_bytes;
#pragma unroll
      for (int kk = 0; kk < R::NK; ++kk) {
        if constexpr (sizeof(T) == 2) u.k[t][kk] = *reinterpret_cast<const u32x4_a4*>(src + kk * 64 + q * 16);
        else u.k[t][kk] = *reinterpret_cast<const f32x4_a4*>(src + (q * (D / 4) + kk * 4) * 4);
      }
    }
  };
  const auto load_v = [&](int slot) {
    valid = 0;
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      const int mine = __shfl(slot, (i / 4) * 16 + 4 * q + i % 4, 64);
      valid |= (mine >= 0 ? 1u : 0u) << i;
      const char* src = head_v + max(mine, 0) * p.row_bytes;
      if constexpr (sizeof(T) == 2) {
        u.v[i] = *reinterpret_cast<const u32x4_a4*>(src + c * 16);
      } else {
#pragma unroll
        for (int j = 0; j < R::VW; ++j) u.v[i][j] = reinterpret_cast<const float*>(src)[c * R::VW + j];
      }
    }
    whole = __all(valid == (1u << NS) - 1);
  };
  int slot = slots_of_unit();
  load_k(slot);
  load_v(slot);
#pragma unroll 1
  for (int unit = first; unit < upto; ++unit) {
    const int pos = s.lo + unit * POS;
    const bool more = unit + 1 < upto;
    const bool edge = !whole || (uint32_t)(pos + POS) > (uint32_t)all;
    // ---- scores ----
    f32x4 sc[NT][TILES];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int kk = 0; kk < R::NK; ++kk)
            a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u.k[t][kk]),
                                                        __builtin_bit_cast(bf16x8, qr[nt][kk]), a, 0, 0, 0);
        } else {
#pragma unroll
          for (int kk = 0; kk < R::NK; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(u.k[t][kk][e], qr[nt][kk][e], a, 0, 0, 0);
        }
        sc[nt][t] = a;
      }
    if (more) {
      slot = slots_of_unit();
      load_k(slot);
    }
    uint32_t seen[NT];
    if (edge) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        seen[nt] = 0;
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const bool ok = (valid >> i & 1) && (uint32_t)(pos + (i / 4) * 16 + 4 * q + i % 4) < (uint32_t)limit[nt];
          seen[nt] |= (ok ? 1u : 0u) << i;
          sc[nt][i / 4][i % 4] = ok ? sc[nt][i / 4][i % 4] : -INFINITY;
        }
      }
    }
    // ---- weights ----
    float w[NT][NS];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float most = sc[nt][0][0];
#pragma unroll
      for (int i = 1; i < NS; ++i) most = fmaxf(most, sc[nt][i / 4][i % 4]);
      most = max_over_q(most) * scale_log2;
      constexpr float lift = sizeof(T) == 2 ? LIFT : 0.0f;
      const float rise = most + lift;
      if (__any(rise > x.top[nt] + SLACK)) {
        const float now = rise > x.top[nt] + SLACK ? rise : x.top[nt];
        const float f = x.top[nt] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(x.top[nt] - now);
        const float keep = now == x.top[nt] ? 1.0f : f;
        x.top[nt] = now;
        x.l[nt] *= keep;
#pragma unroll
        for (int j = 0; j < JN; ++j) x.o[nt][j] *= keep;
      }
      const float base = x.top[nt] == -INFINITY ? 0.0f : x.top[nt];
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        float e = __builtin_amdgcn_exp2f(fmaf(sc[nt][i / 4][i % 4], scale_log2, -base));
        if constexpr (sizeof(T) == 4) e *= 0x1p-40f;
        w[nt][i] = e;
        x.l[nt] += e;
      }
    }
    // ---- sums of values ----
    if (edge) {
      // what no column sees becomes zero, whatever lies there; values that are not finite at
      // positions that only some columns see are taken out and counted for those that do
      bool odd = false;
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const bool ok = valid >> i & 1;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t y = ok ? u.v[i][e] : 0u;
            u.v[i][e] = y;
            odd |= (y & 0x7f80u) == 0x7f80u || (y & 0x7f800000u) == 0x7f800000u;
          }
        } else {
#pragma unroll
          for (int j = 0; j < R::VW; ++j) {
            const float y = ok ? u.v[i][j] : 0.0f;
            u.v[i][j] = y;
            odd |= !(fabsf(y) < INFINITY);
          }
        }
      }
      if (__any(odd)) {
#pragma unroll 1
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int j = 0; j < JN; ++j) {
            f32x4 n = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              // products of ones, four positions of a tile at a time
#pragma unroll
              for (int t = 0; t < TILES; ++t) {
                bool bad;
                if constexpr (sizeof(T) == 2) {
                  const uint32_t y = j % 2 ? u.v[t * 4 + i][j / 2] >> 16 : u.v[t * 4 + i][j / 2] & 0xffffu;
                  bad = (y & 0x7f80u) == 0x7f80u;
                } else {
                  bad = !(fabsf(u.v[t * 4 + i][j]) < INFINITY);
                }
                uint32_t sn = 0;
#pragma unroll
                for (int k = 0; k < NT; ++k) sn = k == nt ? seen[k] : sn;
                const float b = sn >> (t * 4 + i) & 1 ? 1.0f : 0.0f;
                n = __builtin_amdgcn_mfma_f32_16x16x4f32(bad ? 1.0f : 0.0f, b, n, 0, 0, 0);
              }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
              for (int k = 0; k < NT; ++k)
                if (k == nt) x.o[k][j][r] = n[r] > 0.0f ? NAN : x.o[k][j][r];
          }
        }
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t y = u.v[i][e];
              if ((y & 0x7f80u) == 0x7f80u) y &= 0xffff0000u;
              if ((y & 0x7f800000u) == 0x7f800000u) y &= 0xffffu;
              u.v[i][e] = y;
            }
          } else {
#pragma unroll
            for (int j = 0; j < R::VW; ++j) u.v[i][j] = fabsf(u.v[i][j]) < INFINITY ? u.v[i][j] : 0.0f;
          }
        }
      }
    }
    if constexpr (sizeof(T) == 2) {
      u32x4 hi[NT], lo[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = w[nt][2 * i], b = w[nt][2 * i + 1];
          const uint32_t h = pack_bf16(a, b);
          hi[nt][i] = h;
          lo[nt][i] = pack_bf16(a - __uint_as_float(h << 16), b - __uint_as_float(h & 0xffff0000u));
        }
#pragma unroll
      for (int j = 0; j < JN; ++j) {
        u32x4 a;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          a[i] = __builtin_amdgcn_perm(u.v[2 * i + 1][j / 2], u.v[2 * i][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
        const bf16x8 av = __builtin_bit_cast(bf16x8, a);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          x.o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, hi[nt]), x.o[nt][j], 0, 0, 0);
          x.o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, lo[nt]), x.o[nt][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            x.o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(u.v[i][j], w[nt][i], x.o[nt][j], 0, 0, 0);
    }
    if (more) load_v(slot);
  }
}

// An output row's quotient.
template <int N>
__device__ __forceinline__ void divide(float* v, float l) {
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = l == 0.0f ? 0.0f : v[i] * inv;
}

template <typename T>
__device__ __forceinline__ T* out_of(const GroupAttnParams& p, int row, int col, int kvh, int d, int dim) {
  const int i = by_g(p, col);
  return reinterpret_cast<T*>(p.out + (int64_t)(row + i) * p.out_stride) + (int64_t)(kvh * p.g + col - i * p.g) * d + dim;
}

template <int D>
struct MergeScratch {
  float o[WAVES][16][ROW<D>];
};

// A part of an item of NT tiles of 16 columns: the waves' shares, merged, to `dst` ([column][ROW])
// or, where that is null, to the output rows.
template <typename T, int D, int NT>
__device__ void run_part(const GroupAttnParams& p, const Groups& groups, const Shape& s, int entity, int tile,
                         int cols_tile, int first, int upto, int kvh, float* dst, MergeScratch<D>& scratch) {
  constexpr int JN = D / 16;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = lane & 15, q = lane >> 4;
  const int n = upto - first;
  Part<T, D, NT> x;
  attend_part<T, D, NT>(p, groups, s, entity, tile, cols_tile, first + (int)((int64_t)n * wave / WAVES),
                        first + (int)((int64_t)n * (wave + 1) / WAVES), kvh, x);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (nt * 16 < cols_tile) {
      float* mine = scratch.o[wave][c];
      const float l = sum_over_q(x.l[nt]);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < JN; ++j) mine[q * (D / 4) + r * JN + j] = x.o[nt][j][r];
      if (q == 0) {
        mine[D] = x.top[nt];
        mine[D + 1] = l;
      }
      __syncthreads();
      const int col = t / 16, dim = t % 16 * JN;
      if (nt * 16 + col < cols_tile) {
        float top = -INFINITY, sum = 0.0f, v[JN];
#pragma unroll
        for (int i = 0; i < WAVES; ++i) top = fmaxf(top, scratch.o[i][col][D]);
        const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
        for (int j = 0; j < JN; ++j) v[j] = 0.0f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
          const float f = __builtin_amdgcn_exp2f(scratch.o[i][col][D] - base);
          sum = fmaf(scratch.o[i][col][D + 1], f, sum);
#pragma unroll
          for (int j = 0; j < JN; ++j) v[j] = fmaf(scratch.o[i][col][dim + j], f, v[j]);
        }
        if (dst) {
          float* to = dst + (int64_t)(nt * 16 + col) * ROW<D>;
#pragma unroll
          for (int j = 0; j < JN; ++j) to[dim + j] = v[j];
          if (dim == 0) {
            to[D] = top;
            to[D + 1] = sum;
          }
        } else {
          divide<JN>(v, sum);
          T* to = out_of<T>(p, s.row, tile + nt * 16 + col, kvh, D, dim);
          if constexpr (sizeof(T) == 2) {
            store_out<T, JN>(to, v);
          } else {
#pragma unroll
            for (int j = 0; j < JN; ++j) to[j] = v[j];
          }
        }
      }
      __syncthreads();
    }
  }
}

constexpr int occupancy_of(int nt) { return nt == 4 ? 1 : 2; }

template <typename T, int D, int NT>
__global__ __launch_bounds__(GA_NT, occupancy_of(NT)) void group_attn_kernel(GroupAttnParams p) {
  constexpr int COLS = 16 * NT, POS = Unit<T>::POS;
  __shared__ int32_t s_groups[KNOWN];
  __shared__ uint32_t s_sum[3][WAVES];
  __shared__ int s_begin[4];  // the stretch's first entity, units, prefixes' and other items before it
  __shared__ MergeScratch<D> s_merge;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int kvh = blockIdx.x % p.nkv, w = blockIdx.x / p.nkv;
  const Groups groups{s_groups};
  if (p.G > 0 && p.G < KNOWN)
    for (int i = t; i <= p.G; i += GA_NT) s_groups[i] = p.group_offsets[i];
  if (t == 0) s_begin[0] = -1;
  __syncthreads();

  // ---- the units and items before each thread's entities ----
  const int E = p.G + p.R, per = (E + GA_NT - 1) / GA_NT;
  uint32_t mine[3] = {0, 0, 0};  // units, items of prefixes, of requests
  for (int i = 0; i < per; ++i) {
    const int e = t * per + i;
    if (e < E) {
      const Shape s = shape_of<COLS, POS>(p, groups, e);
      mine[0] += s.units();
      mine[e < p.G ? 1 : 2] += s.tiles;
    }
  }
  uint32_t pre[3], total = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    pre[k] = wave_scan(mine[k]);
    if (lane == 63) s_sum[k][wave] = pre[k];
    pre[k] -= mine[k];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (i < wave) pre[k] += s_sum[k][i];
    total += s_sum[0][i];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const Stretches st(p.workers, total);
  const uint32_t u0 = st.begin(w), u1 = st.begin(w + 1);
  if ((uint32_t)w < st.workers && u0 >= pre[0] && u0 - pre[0] < mine[0]) {
    s_begin[0] = t * per;
    s_begin[1] = (int)pre[0];
    s_begin[2] = (int)pre[1];
    s_begin[3] = (int)pre[2];
  }
  if (blockIdx.x == 0) {  // what the second kernel reads
    if (t == 0) {
      Plan h{};
      h.size = st.size;
      h.longer = st.longer;
      h.workers = st.workers;
      *p.plan = h;
    }
    for (int i = 0; i < per; ++i) {
      const int e = t * per + i;
      if (e < E) {
        const Shape s = shape_of<COLS, POS>(p, groups, e);
        p.entities[e] = Entity{pre[0], s.item, (int)pre[e < p.G ? 1 : 2], s.row, s.tiles ? s.cols : 0, s.group, {s.lo, 0}};
        pre[0] += s.units();
        pre[e < p.G ? 1 : 2] += s.tiles;
      }
    }
  }
  __syncthreads();
  int e = __builtin_amdgcn_readfirstlane(s_begin[0]);
  if (e < 0) return;
  uint32_t base = __builtin_amdgcn_readfirstlane(s_begin[1]);
  int items[2] = {__builtin_amdgcn_readfirstlane(s_begin[2]), __builtin_amdgcn_readfirstlane(s_begin[3])};
  Shape s = shape_of<COLS, POS>(p, groups, e);
  for (uint32_t u = u0; u < u1;) {
    while (u - base >= s.units() && e + 1 < E) {
      base += s.units();
      items[e < p.G ? 0 : 1] += s.tiles;
      s = shape_of<COLS, POS>(p, groups, ++e);
    }
    const uint32_t tile = quotient(u - base, s.item);
    if (tile >= (uint32_t)s.tiles) break;  // offsets that overlap so far that the units passed 2^32
    const uint32_t from = u - base - tile * s.item, to = min(s.item, from + (u1 - u));
    u += to - from;
    const int first = max((int)from - START, 0), upto = (int)to - START;
    if (upto <= 0) continue;  // of the start alone
    const int kind = e < p.G ? 0 : 1, cols = min(COLS, s.cols - (int)tile * COLS);
    // a request's item that is all here, with no prefix before it, goes straight out
    float* dst = nullptr;
    if (kind == 0 || s.lo > 0 || from > START || to < s.item) {
      const int64_t slot = (int64_t)items[kind] + tile + w;
      if (slot >= p.slots[kind]) break;  // offsets that overlap: more items than rows make
      dst = p.part[kind] + (kvh * p.slots[kind] + slot) * p.part_cols[kind] * ROW<D>;
    }
    const int at = (int)tile * COLS;
    if (NT == 1 || cols <= 16) run_part<T, D, 1>(p, groups, s, e, at, cols, first, upto, kvh, dst, s_merge);
    else if (NT == 2 || cols <= 32) run_part<T, D, 2>(p, groups, s, e, at, cols, first, upto, kvh, dst, s_merge);
    else run_part<T, D, NT == 4 ? 4 : 2>(p, groups, s, e, at, cols, first, upto, kvh, dst, s_merge);
  }
}

// Columns whose sums lie in several places: D / 4 lanes a column.
template <typename T, int D, int NT>
__global__ __launch_bounds__(GA_NT) void group_merge_kernel(GroupAttnParams p) {
  constexpr int COLS = 16 * NT, LANES = D / 4, AT_ONCE = GA_NT / LANES, CHUNK = 8;
  const Stretches st(*p.plan);
  const int64_t all = (int64_t)p.R * p.nkv;
  for (int64_t b = blockIdx.x; b < all; b += gridDim.x) {
    const int kvh = (int)(b % p.nkv), r = (int)(b / p.nkv);
    const Entity own = p.entities[p.G + r];
    Entity pre{};
    if (own.group >= 0) pre = p.entities[own.group];
    const Rows x = rows_of(p, r);
    const int cols = x.used * p.g, lane = threadIdx.x % LANES, dim = lane * 4;
    for (int col = threadIdx.x / LANES; col < cols; col += AT_ONCE) {
      // its partials: of the prefix, then of its own positions
      const float* src[2];
      int n[2] = {0, 0};
      const int at[2] = {(x.row - pre.row) * p.g + col, col};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const Entity& y = k ? own : pre;
        src[k] = nullptr;
        if (at[k] < 0 || at[k] >= y.cols) continue;
        const int tile = at[k] / COLS;
        const uint32_t begin = y.base + (uint32_t)tile * y.item;
        const int a = st.holder(begin + START), z = st.holder(begin + y.item - 1);
        const int64_t slot = (int64_t)y.first + tile + a;
        if (slot < 0 || slot + (z - a) >= p.slots[k]) continue;
        n[k] = z - a + 1;
        src[k] = p.part[k] + ((kvh * p.slots[k] + slot) * p.part_cols[k] + (at[k] - tile * COLS)) * ROW<D>;
      }
      if (n[1] == 1 && own.pad[0] == 0) continue;  // written by the first kernel
      float top = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const int total = n[0] + n[1];
      for (int i0 = 0; i0 < total; i0 += CHUNK) {
        float m[CHUNK], ls[CHUNK];
        f32x4 v[CHUNK];
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {  // past the last: the last again, not counted below
          const int k = min(i0 + i, total - 1);
          const float* part = k < n[0] ? src[0] + (int64_t)k * p.part_cols[0] * ROW<D>
                                       : src[1] + (int64_t)(k - n[0]) * p.part_cols[1] * ROW<D>;
          v[i] = *reinterpret_cast<const f32x4*>(part + dim);
          m[i] = part[D];
          ls[i] = part[D + 1];
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) now = fmaxf(now, m[i]);
        const float base = now == -INFINITY ? 0.0f : now;
        const float was = __builtin_amdgcn_exp2f(top - base);
        top = now;
        l *= was;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= was;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
          if (i0 + i < total) {
            const float f = __builtin_amdgcn_exp2f(m[i] - base);
            l = fmaf(ls[i], f, l);
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] = fmaf(v[i][d], f, o[d]);
          }
      }
      divide<4>(o, l);
      store_out<T, 4>(out_of<T>(p, x.row, col, kvh, D, dim), o);
    }
  }
}

struct Sizes {
  int64_t R, rows, G, max_query, max_len;
  int g;
};

// Column tiles of an item: as many as the average of what shares it fills.
int tiles_of(const Sizes& z) {
  const int64_t cols = z.G > 0 ? (z.rows * z.g + z.G - 1) / z.G : z.g * z.max_query;
  return cols > 32 ? 4 : cols > 16 ? 2 : 1;
}
int most_workers(int nkv, int nt) { return std::max(1, CUS * occupancy_of(nt) / nkv); }

// The workspace: the plan, the entities, the sums of prefixes and those of requests.  Their
// numbers grow with every size of a call, whichever kernel it takes.
struct GroupLayout {
  uint64_t entities, part[2], total;
  int part_cols[2];   // for the call's own kernel
  int64_t slots[2];
};
GroupLayout layout_of(const kv_model_desc& d, const Sizes& z, int nt) {
  const int64_t columns = z.rows * z.g, row = d.head_dim + 4, most = most_workers(d.num_kv_heads, 1);
  const int64_t entity[2] = {z.G, z.R}, widest[2] = {std::min<int64_t>(64, columns), std::min<int64_t>(64, z.g * std::min(z.max_query, z.rows))};
  GroupLayout L;
  L.entities = 256;
  L.part[0] = L.entities + (uint64_t)round_up((z.G + z.R) * (int64_t)sizeof(Entity), 256);
  for (int k = 0; k < 2; ++k) {
    const int64_t floats = k == 0 && z.G == 0 ? 0 : d.num_kv_heads * (columns + (entity[k] + most) * widest[k]) * row;
    (k == 0 ? L.part[1] : L.total) = L.part[k] + (uint64_t)round_up(4 * floats, 256);
    L.part_cols[k] = (int)std::min<int64_t>(16 * nt, widest[k]);
    L.slots[k] = floats ? columns / (16 * nt) + entity[k] + most_workers(d.num_kv_heads, nt) : 0;
  }
  return L;
}

bool takes(const Sizes& z) {
  if (z.R > MOST_ROWS || z.rows > MOST_ROWS || z.G > MOST_ROWS || z.max_len > INT32_MAX) return false;
  return (z.R + z.G + z.rows * z.g / 8) * (z.max_len / 16 + 16) <= INT32_MAX;
}

template <typename T, int D, int NT>
void launch_tiles(const GroupAttnParams& p, hipStream_t s) {
  hipLaunchKernelGGL((group_attn_kernel<T, D, NT>), dim3((unsigned)(p.workers * p.nkv)), dim3(GA_NT), 0, s, p);
  const int64_t blocks = std::min<int64_t>((int64_t)p.R * p.nkv, 1 << 20);
  hipLaunchKernelGGL((group_merge_kernel<T, D, NT>), dim3((unsigned)blocks), dim3(GA_NT), 0, s, p);
}
template <typename T, int D>
void launch(int nt, const GroupAttnParams& p, hipStream_t s) {
  if (nt == 1) launch_tiles<T, D, 1>(p, s);
  else if (nt == 2) launch_tiles<T, D, 2>(p, s);
  else launch_tiles<T, D, 4>(p, s);
}

bool head_sizes(const kv_model_desc& d) { return d.head_dim % 32 == 0 && d.num_q_heads / d.num_kv_heads <= 16; }

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

uint64_t kv_group_attention_workspace_bytes(const kv_model_desc* desc, int32_t num_requests, int64_t rows,
                                            int32_t num_groups, int32_t max_query, int64_t max_len) {
  if (check_desc(desc) != KV_OK || !head_sizes(*desc)) return 0;
  if (num_requests <= 0 || num_requests > MOST_ROWS || rows <= 0 || rows > MOST_ROWS || num_groups < 0 ||
      num_groups > MOST_ROWS || max_query <= 0 || max_len <= 0 || max_len > INT32_MAX)
    return 0;
  return layout_of(*desc, {num_requests, rows, num_groups, max_query, max_len, desc->num_q_heads / desc->num_kv_heads}, 1)
      .total;
}

kv_status kv_group_attention(kv_arena_t arena, int32_t layer, const void* q, int64_t q_stride,
                             const int32_t* q_offsets, int64_t rows, const int32_t* lens, const int32_t* tables,
                             int32_t R, int32_t max_blocks, const int32_t* group_offsets, const int32_t* prefix_lens,
                             int32_t num_groups, int32_t max_query, int64_t max_len, void* out, int64_t out_stride,
                             void* workspace, uint64_t ws_bytes, void* stream) {
  if (!live_arena(arena)) return kvr_err::set(KV_ESTATE, "unknown or released arena handle");
  const kv_model_desc& d = arena->desc;
  const int64_t e = elem_bytes(d.dtype), row = (int64_t)d.num_q_heads * d.head_dim;
  if (!head_sizes(d))
    return kvr_err::set(KV_EINVAL, "group attention needs head_dim in {32, 64, 128} and at most 16 q heads per kv head");
  if (arena->num_blocks > INT32_MAX / arena->block_size)
    return kvr_err::set(KV_EINVAL, "group attention takes arenas below 2^31 slots");
  if (layer < 0 || layer >= d.num_layers)
    return kvr_err::set(KV_EINVAL, "layer %d outside [0, %d)", layer, d.num_layers);
  if (R < 0 || R > MOST_ROWS || rows < 0 || rows > MOST_ROWS || num_groups < 0 || num_groups > MOST_ROWS || max_blocks < 0)
    return kvr_err::set(KV_EINVAL, "num_requests, rows and num_groups are 0 .. 2^24, max_blocks_per_req is not negative");
  if (!q_offsets && rows != R) return kvr_err::set(KV_EINVAL, "without q_offsets rows must equal num_requests");
  if (R == 0 || rows == 0) return kvr_err::clear();
  if (max_query < 1 || max_len < 1) return kvr_err::set(KV_EINVAL, "max_query and max_len must be positive");
  if (!q || !out || !lens || (max_blocks > 0 && !tables) || (num_groups > 0 && (!group_offsets || !prefix_lens)))
    return kvr_err::set(KV_EINVAL, "null q, out, lens, block_tables, group_offsets or prefix_lens");
  const int64_t most_stride = INT64_MAX / 8 / rows;
  if (q_stride < row || out_stride < row || q_stride > most_stride || out_stride > most_stride)
    return kvr_err::set(KV_EINVAL, "a stride is below the row's %lld elements, or beyond the addresses there are",
                        (long long)row);
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)(q_stride * e) | (uintptr_t)(out_stride * e) | (uintptr_t)q_offsets |
       (uintptr_t)lens | (uintptr_t)tables | (uintptr_t)group_offsets | (uintptr_t)prefix_lens |
       (uintptr_t)arena->base) % 4 != 0)
    return kvr_err::set(KV_EINVAL, "the arrays, the strides and the arena need boundaries of 4 bytes");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
  const int g = d.num_q_heads / d.num_kv_heads;
  const Sizes z{R, rows, num_groups, max_query, max_len, g};
  if (!takes(z)) return kvr_err::set(KV_EINVAL, "max_len or the work of one call above 2^31: split the query rows");
  const int nt = tiles_of(z);
  const GroupLayout L = layout_of(d, z, nt);
  if (L.total > ws_bytes)
    return kvr_err::set(KV_ENOMEM, "workspace of %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                        (unsigned long long)L.total);
  DeviceGuard dg(arena->device);
  const kv_status st = device_ready(dg, arena->device);
  if (st != KV_OK) return st;
  GroupAttnParams p{};
  p.row_bytes = (int64_t)d.num_kv_heads * d.head_dim * e;
  const int64_t plane = arena->num_blocks * arena->block_size * p.row_bytes;
  p.plane_k = static_cast<const char*>(arena->base) + 2 * layer * plane;
  p.plane_v = p.plane_k + plane;
  p.num_blocks = (uint32_t)arena->num_blocks;
  p.block_size = arena->block_size;
  p.block_inv = p.block_size < 32 ? (uint32_t)(((1 << 16) + p.block_size - 1) / p.block_size) : 0;
  p.q = static_cast<const char*>(q);
  p.out = static_cast<char*>(out);
  p.q_stride = q_stride * e;
  p.out_stride = out_stride * e;
  p.q_offsets = q_offsets;
  p.rows = (int)rows;
  p.lens = lens;
  p.tables = tables;
  p.R = R;
  p.max_blocks = max_blocks;
  p.group_offsets = group_offsets;
  p.prefix_lens = prefix_lens;
  p.G = num_groups;
  p.nkv = d.num_kv_heads;
  p.g = g;
  p.g_inv = g == 1 ? 0 : (uint32_t)(((1ull << 32) + g - 1) / g);
  p.max_query = max_query;
  p.most_len = (int)std::min<int64_t>({max_len, (int64_t)max_blocks * arena->block_size, INT32_MAX});
  p.workers = most_workers(d.num_kv_heads, nt);
  char* ws = static_cast<char*>(workspace);
  p.plan = reinterpret_cast<Plan*>(ws);
  p.entities = reinterpret_cast<Entity*>(ws + L.entities);
  for (int k = 0; k < 2; ++k) {
    p.part[k] = reinterpret_cast<float*>(ws + L.part[k]);
    p.part_cols[k] = L.part_cols[k];
    p.slots[k] = L.slots[k];
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d.dtype == KV_BF16) launch<bf16_t, 128>(nt, p, s);
  else if (d.head_dim == 128) launch<float, 128>(nt, p, s);
  else if (d.head_dim == 64) launch<float, 64>(nt, p, s);
  else launch<float, 32>(nt, p, s);
  return launched();
}

}  // extern "C"

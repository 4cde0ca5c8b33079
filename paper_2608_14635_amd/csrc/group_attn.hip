// Attention over the retained arena, a group's shared prefix read once (kvr_attention.h).
//
// Query rows that share a kv head are columns: column i g + h is row i of q head h of the
// group of heads.  There are two kinds of entities: a group of requests, whose rows all see
// the group's prefix, and a request, whose rows see what follows it.  An entity's columns in
// tiles (of 16, or 128 in bf16 and 32 in fp32) make items, the work of an item comes in units of
// positions.  Every workgroup takes an equal stretch of the units of all items, entity after
// entity, whatever the lengths (they are known on the device alone); a unit counts by the
// columns of its item, an item's start as eight costs more.  Up to 16 (32) columns the four waves
// share out an item's units and merge their sums in LDS; of more they share out the columns, and
// units come to all of them through LDS, read once.  A second kernel joins what is there of a
// column: the workgroups' sums over its group's prefix and over its own positions.  Short calls
// have a workgroup to an item and no second kernel.
//
// Bound by memory with few columns: 64 requests of 1004 - 5980 positions in eight groups, 8 kv
// heads, 667 MB in 130 us (5.1 TB/s; a read reaches 6.0) + 5.8.  With many (48 requests on one
// prefix of 24011, 240 columns, 297 MB in 83 - 95 + 9) a workgroup's unit of 32 positions and 128
// columns takes 3500 cycles: 770 of matrix instructions, some 1300 of others, the rest are waits for
// each other with two waves a SIMD.  Calls of some 20 us by what follows one another: plan 3,
// first unit 6, the last merges 3, the second kernel 4 to 7.
//
// A unit in a wave's registers, lane (q, c) = (lane / 16, lane % 16):
//   S^T = K Q^T, 16 positions a tile: the lane gets the scores of positions 4q .. 4q+3 for
//   column c.
//   Online softmax per column, rescaled only where the maximum rose by more than 2^SLACK.
//   Weights are 2^((s - m) log2 e / sqrt d) with m a score as it came: the difference of near
//   scores is exact, however large they are.  (A multiple of m, rounded, as the base of one
//   multiply-add: from scores of 2^33 on its rounding moves the largest weight out of what
//   fp32 holds.)
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
//   weights, and their sum, are taken 2^-LIFT as large.  In bf16 exponents are LIFT less for it
//   (and then rounded to 2^-19, below the 2^-17 above), in fp32 weights are multiplied.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "dma.h"
#include "host.h"
#include "kvr_attention.h"

namespace kvr {
namespace {

constexpr int GA_NT = 256, WAVES = GA_NT / 64;
constexpr float SLACK = 8.0f, LIFT = 40.0f;  // log2 units
// log2 e / sqrt d
template <int D>
constexpr float LOG2_SCALE = 1.4426950408889634 / (D == 128 ? 11.313708498984760390 : D == 64 ? 8.0 : 5.6568542494923801952);
constexpr int MOST_ROWS = 1 << 24;           // query rows, requests and groups of a call
constexpr int START = 8;                     // what an item's start costs
constexpr int CUS = 256, A_CU = 2;           // workgroups of a CU, by their registers and LDS

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));

// What the second kernel has to know of an entity: where its items begin, what each
// costs, its first item among its kind, its first query row and its columns, its request's group.
struct Entity {
  uint32_t base, item;
  int first, row, cols, group, lo, cost;
};
struct Plan {
  uint32_t more, half, size, longer, workers, pad[3];
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

// What a unit of an item of so many columns costs: two for one whose waves have a unit each.  (Four
// and six of the wider: 98 us, not 94, for 48 requests on one prefix; five and eight 106; four and
// five 93, but 39.5, not 36.6, where columns are up to 64.)
constexpr int MOST_COST = 4;
__host__ __device__ constexpr int cost_of(int cols, int most_cols) {
  return most_cols <= 32 || cols <= 16 ? 2 : cols <= 64 ? 3 : MOST_COST;
}

// All costs in stretches: of the first `half` workers `more` each, then the first `longer` of
// size + 1, then of `size`.  A unit is the worker's that has the first of its cost; none has less
// than a unit's, so that of an item that several hold each one between the first and the last holds
// a unit.  Where all are there and have much to do, the first half, on each CU the older of its two
// workgroups, which is served first, takes 1 + 1/SKEW of the average, the rest as much less (64
// requests of 1000 - 6000 positions in eight groups: 130 us, evenly 134, with 1/16 132).
constexpr uint32_t SKEW = 8, SKEWED = 32;
struct Stretches {
  uint32_t more, half, size, longer, workers;
  __device__ __forceinline__ Stretches(uint32_t most, uint32_t total) {
    workers = max(1u, min(most, total / MOST_COST));
    const uint32_t even = quotient(total, workers);
    half = workers == most && even >= SKEWED ? workers / 2 : 0;
    more = even + even / SKEW;
    const uint32_t rest = total - half * more;
    size = quotient(rest, workers - half);
    longer = rest - size * (workers - half);
  }
  __device__ __forceinline__ explicit Stretches(const Plan& p)
      : more(p.more), half(p.half), size(p.size), longer(p.longer), workers(p.workers) {}
  __device__ __forceinline__ uint32_t begin(uint32_t w) const {
    return w < half ? w * more : half * more + (w - half) * size + min(w - half, longer);
  }
  __device__ __forceinline__ int holder(uint32_t u) const {  // whose u is
    if (u < half * more) return (int)quotient(u, more);
    const uint32_t v = u - half * more, head = longer * (size + 1);
    return (int)(half + (v < head ? quotient(v, size + 1) : longer + quotient(v - head, size)));
  }
};

// The lists of groups and requests: where they are short, in LDS.
constexpr int KNOWN_GROUPS = 512, KNOWN_REQUESTS = 1024;
struct Known {
  int32_t offsets[KNOWN_GROUPS], prefixes[KNOWN_GROUPS], rows[KNOWN_REQUESTS], lens[KNOWN_REQUESTS];
};
template <bool LDS>
struct Lists {
  const GroupAttnParams& p;
  const Known* known;
  __device__ __forceinline__ bool groups() const { return LDS && p.G < KNOWN_GROUPS; }
  __device__ __forceinline__ bool requests() const { return LDS && p.R < KNOWN_REQUESTS; }
  __device__ __forceinline__ int offset(int e) const { return groups() ? known->offsets[e] : p.group_offsets[e]; }
  __device__ __forceinline__ int prefix(int e) const { return groups() ? known->prefixes[e] : p.prefix_lens[e]; }
  __device__ __forceinline__ int row(int r) const {
    return !p.q_offsets ? r : requests() ? known->rows[r] : p.q_offsets[r];
  }
  __device__ __forceinline__ int len(int r) const { return requests() ? known->lens[r] : p.lens[r]; }
};
// Into LDS, the first 256 of each on their way together.
__device__ __forceinline__ void fill_known(const GroupAttnParams& p, Known& k) {
  const int t = threadIdx.x, G = p.G < KNOWN_GROUPS ? p.G : 0, R = p.R < KNOWN_REQUESTS ? p.R : 0;
  const int groups = G > 0 ? G + 1 : 0, rows = R > 0 && p.q_offsets ? R + 1 : 0;
  int a = 0, b = 0, c = 0, d = 0;
  if (t < groups) a = p.group_offsets[t];
  if (t < G) b = p.prefix_lens[t];
  if (t < rows) c = p.q_offsets[t];
  if (t < R) d = p.lens[t];
  if (t < groups) k.offsets[t] = a;
  if (t < G) k.prefixes[t] = b;
  if (t < rows) k.rows[t] = c;
  if (t < R) k.lens[t] = d;
  for (int i = t + GA_NT; i < groups; i += GA_NT) k.offsets[i] = p.group_offsets[i];
  for (int i = t + GA_NT; i < G; i += GA_NT) k.prefixes[i] = p.prefix_lens[i];
  for (int i = t + GA_NT; i < rows; i += GA_NT) k.rows[i] = p.q_offsets[i];
  for (int i = t + GA_NT; i < R; i += GA_NT) k.lens[i] = p.lens[i];
}

// A request's query rows, and the position after the last of them.
struct Rows {
  int row, all, used, end;  // used: at most max_query of all
  int start;                // position of the first
};
template <bool LDS>
__device__ __forceinline__ Rows rows_of(const Lists<LDS>& lists, int r) {
  const GroupAttnParams& p = lists.p;
  Rows x{r, 1, 1, 0, 0};
  if (p.q_offsets) {
    x.row = clamp_to(lists.row(r), 0, p.rows);
    x.all = max(min(lists.row(r + 1), p.rows) - x.row, 0);
    x.used = min(x.all, p.max_query);
  }
  x.start = max(lists.len(r), 0) - x.all;
  x.end = x.start + x.used;  // the rows left out are the last ones
  return x;
}

// An entity: columns that see positions lo .. hi - 1 through a table.  Units begin at multiples
// of their positions, the first with the one that lo lies in.
struct Shape {
  int row, cols, lo, hi, table, group;
  int tiles;      // of columns; 0: nothing to do
  int units;      // of an item
  int cost;       // of a unit
  uint32_t item;  // what an item costs: its start and its units
  __device__ __forceinline__ uint32_t all() const { return (uint32_t)tiles * item; }
};

// The group that request r is in, -1: none.  One of a single request shares nothing.
__device__ __forceinline__ int group_of(const Lists<true>& lists, int r) {
  const GroupAttnParams& p = lists.p;
  if (p.G == 0) return -1;
  int a = 0, b = p.G - 1;
  while (a < b) {
    const int m = (a + b + 1) / 2;
    if (lists.offset(m) <= r) a = m;
    else b = m - 1;
  }
  const int lo = clamp_to(lists.offset(a), 0, p.R), hi = clamp_to(lists.offset(a + 1), lo, p.R);
  return r >= lo && r < hi && hi - lo > 1 ? a : -1;
}

template <int COLS, int POS>
__device__ __forceinline__ Shape finish_shape(const GroupAttnParams& p, Shape s) {
  s.tiles = s.hi > s.lo ? (int)(((int64_t)s.cols + COLS - 1) / COLS) : 0;
  s.units = s.hi > s.lo ? (s.hi - 1) / POS - s.lo / POS + 1 : 0;
  s.cost = cost_of(min(s.cols, COLS), COLS);
  s.item = (uint32_t)(START + s.units * s.cost);
  return s;
}
template <int COLS, int POS>
__device__ __forceinline__ Shape shape_of(const Lists<true>& lists, int e) {
  const GroupAttnParams& p = lists.p;
  Shape s{};
  s.group = -1;
  if (e < p.G) {
    const int r0 = clamp_to(lists.offset(e), 0, p.R), r1 = clamp_to(lists.offset(e + 1), r0, p.R);
    s.table = r0;
    s.hi = r1 - r0 > 1 ? clamp_to(lists.prefix(e), 0, p.most_len) : 0;
    if (s.hi > 0) {
      s.row = p.q_offsets ? clamp_to(lists.row(r0), 0, p.rows) : r0;
      s.cols = ((p.q_offsets ? clamp_to(lists.row(r1), s.row, p.rows) : r1) - s.row) * p.g;
    }
    return finish_shape<COLS, POS>(p, s);
  }
  s.table = e - p.G;
  const Rows x = rows_of(lists, s.table);
  s.row = x.row;
  s.cols = x.used * p.g;
  s.group = group_of(lists, s.table);
  s.hi = clamp_to(x.end, 0, p.most_len);
  s.lo = s.group >= 0 ? clamp_to(lists.prefix(s.group), 0, s.hi) : 0;
  return finish_shape<COLS, POS>(p, s);
}

// The same in every lane, and known to be.
__device__ __forceinline__ Shape uniform(Shape s) {
  const auto u = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  return Shape{u(s.row),   u(s.cols),  u(s.lo),    u(s.hi),   u(s.table),
               u(s.group), u(s.tiles), u(s.units), u(s.cost), (uint32_t)u((int)s.item)};
}

// Positions that a query row of a prefix's columns sees.
__device__ __forceinline__ int limit_in_group(const Lists<true>& lists, int e, int row) {
  const GroupAttnParams& p = lists.p;
  if (!p.q_offsets) return lists.len(row);
  const int r0 = clamp_to(lists.offset(e), 0, p.R), r1 = clamp_to(lists.offset(e + 1), r0, p.R);
  int a = r0, b = max(r1 - 1, r0);
  // the last request whose rows begin at or before it
  while (a < b) {
    const int m = (a + b + 1) / 2;
    if (lists.row(m) <= row) a = m;
    else b = m - 1;
  }
  const Rows x = rows_of(lists, a);
  return x.start + (row - x.row) + 1;
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
  static constexpr int POS = 32, TILES = 2, NK = D / 32, NS = 4 * TILES;
  typedef u32x4 Word;
  u32x4 k[TILES][NK];
  u32x4 v[NS];
  __device__ __forceinline__ void load_k(int t, const char* row, int q) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) k[t][kk] = *reinterpret_cast<const u32x4_a4*>(row + kk * 64 + q * 16);
  }
  __device__ __forceinline__ void load_v(int i, const char* row, int c) {
    v[i] = *reinterpret_cast<const u32x4_a4*>(row + c * 16);
  }
  __device__ __forceinline__ void put_v(int i, char* row, int c) const { *reinterpret_cast<u32x4*>(row + c * 16) = v[i]; }
  __device__ __forceinline__ void keep_v(int i, bool ok) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[i][e] = ok ? v[i][e] : 0u;
  }
  // whether a value is not finite; such values as zero
  __device__ __forceinline__ bool odd() const {
    bool y = false;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) y |= (v[i][e] & 0x7f80u) == 0x7f80u || (v[i][e] & 0x7f800000u) == 0x7f800000u;
    return y;
  }
  __device__ __forceinline__ void without_odd() {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if ((v[i][e] & 0x7f80u) == 0x7f80u) v[i][e] &= 0xffff0000u;
        if ((v[i][e] & 0x7f800000u) == 0x7f800000u) v[i][e] &= 0xffffu;
      }
  }
};
template <int D> struct Regs<float, D> {
  static constexpr int POS = 16, TILES = 1, NK = D / 16, NS = 4;
  static constexpr int VW = D / 16;  // floats of a position
  typedef f32x4 Word;
  f32x4 k[TILES][NK];
  float v[NS][VW];
  __device__ __forceinline__ void load_k(int t, const char* row, int q) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) k[t][kk] = *reinterpret_cast<const f32x4_a4*>(row + (q * (D / 4) + kk * 4) * 4);
  }
  __device__ __forceinline__ void load_v(int i, const char* row, int c) {
#pragma unroll
    for (int j = 0; j < VW; ++j) v[i][j] = reinterpret_cast<const float*>(row)[c * VW + j];
  }
  __device__ __forceinline__ void put_v(int i, char* row, int c) const {
#pragma unroll
    for (int j = 0; j < VW; ++j) reinterpret_cast<float*>(row)[c * VW + j] = v[i][j];
  }
  __device__ __forceinline__ void keep_v(int i, bool ok) {
#pragma unroll
    for (int j = 0; j < VW; ++j) v[i][j] = ok ? v[i][j] : 0.0f;
  }
  __device__ __forceinline__ bool odd() const {
    bool y = false;
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int j = 0; j < VW; ++j) y |= !(fabsf(v[i][j]) < INFINITY);
    return y;
  }
  __device__ __forceinline__ void without_odd() {
#pragma unroll
    for (int i = 0; i < NS; ++i)
#pragma unroll
      for (int j = 0; j < VW; ++j) v[i][j] = fabsf(v[i][j]) < INFINITY ? v[i][j] : 0.0f;
  }
};

// Position of a lane's i-th score within its unit.
__device__ __forceinline__ int at_of(int i, int q) { return (i / 4) * 16 + 4 * q + i % 4; }

// A part of an item: its first column and their number, the units of a wave.
struct Span {
  int entity, tile, cols, first, upto, kvh;
};

// NT tiles of 16 columns in a wave's registers.
template <typename T, int D, int NT>
struct Columns {
  using R = Regs<T, D>;
  static constexpr int POS = R::POS, TILES = R::TILES, NS = R::NS, JN = D / 16;
  typename R::Word q[NT][R::NK];
  int limit[NT];         // positions that column c sees
  int all;               // that every column does
  f32x4 o[NT][JN];       // [j][r]: dim q d/4 + r d/16 + j of column c
  float top[NT], l[NT];  // the score that weights are relative to; the lane's own weights' sum

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      top[nt] = -INFINITY;
      l[nt] = 0.0f;
#pragma unroll
      for (int j = 0; j < JN; ++j) o[nt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }

  // Queries and limits of columns x.tile + skip ..
  __device__ __forceinline__ void load(const Lists<true>& lists, const Shape& s, const Span& x,
                                       int skip) {
    const GroupAttnParams& p = lists.p;
    const int lane = threadIdx.x & 63, c = lane & 15, qq = lane >> 4;
    all = s.hi;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int in = skip + nt * 16 + c, cc = min(x.tile + in, s.cols - 1), i = by_g(p, cc);
      const bool there = in < x.cols;
      const char* src = p.q + (int64_t)(s.row + i) * p.q_stride + (int64_t)(x.kvh * p.g + cc - i * p.g) * D * sizeof(T);
#pragma unroll
      for (int kk = 0; kk < R::NK; ++kk) {
        if constexpr (sizeof(T) == 2)
          q[nt][kk] = there ? (u32x4)*reinterpret_cast<const u32x4_a4*>(src + kk * 64 + qq * 16) : u32x4{0, 0, 0, 0};
        else
          q[nt][kk] = there ? (f32x4)*reinterpret_cast<const f32x4_a4*>(src + (qq * (D / 4) + kk * 4) * 4)
                            : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }
      int lim;
      if (x.entity < p.G) {
        lim = limit_in_group(lists, x.entity, s.row + i);
      } else {
        lim = rows_of(lists, s.table).start + i + 1;
      }
      limit[nt] = clamp_to(lim, 0, s.hi);
      all = there ? min(all, limit[nt]) : all;
    }
#pragma unroll
    for (int o = 1; o < 16; o *= 2) all = min(all, __shfl_xor(all, o, 64));
    all = __builtin_amdgcn_readfirstlane(all);
  }

  __device__ __forceinline__ void scores(const R& u, f32x4 (&sc)[NT][TILES]) const {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f};
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int kk = 0; kk < R::NK; ++kk)
            a = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, u.k[t][kk]),
                                                        __builtin_bit_cast(bf16x8, q[nt][kk]), a, 0, 0, 0);
        } else {
#pragma unroll
          for (int kk = 0; kk < R::NK; ++kk)
#pragma unroll
            for (int e = 0; e < 4; ++e) a = __builtin_amdgcn_mfma_f32_16x16x4f32(u.k[t][kk][e], q[nt][kk][e], a, 0, 0, 0);
        }
        sc[nt][t] = a;
      }
  }

  // Scores of positions from `pos` on that are not there (`there`: a bit each), or that a column
  // does not see.
  __device__ __forceinline__ void mask(f32x4 (&sc)[NT][TILES], int pos, uint32_t there) const {
    const int qq = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < NS; ++i)
        if (!(there >> at_of(i, qq) & 1) || (uint32_t)(pos + at_of(i, qq)) >= (uint32_t)limit[nt])
          sc[nt][i / 4][i % 4] = -INFINITY;
  }

  // Scores become weights.
  __device__ __forceinline__ void weigh(f32x4 (&sc)[NT][TILES]) {
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float most = sc[nt][0][0];
#pragma unroll
      for (int i = 1; i < NS; ++i) most = fmaxf(most, sc[nt][i / 4][i % 4]);
      const float rise = max_over_q(most);
      const bool higher = (rise - top[nt]) * LOG2_SCALE<D> > SLACK;
      if (__any(higher)) {
        const float now = higher ? rise : top[nt];
        const float f = now == top[nt] ? 1.0f : __builtin_amdgcn_exp2f((top[nt] - now) * LOG2_SCALE<D>);
        top[nt] = now;
        l[nt] *= f;
#pragma unroll
        for (int j = 0; j < JN; ++j) o[nt][j] *= f;
      }
      const float base = top[nt] == -INFINITY ? 0.0f : top[nt];
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const float x = sc[nt][i / 4][i % 4] - base;
        float e;
        if constexpr (sizeof(T) == 2) e = __builtin_amdgcn_exp2f(fmaf(x, LOG2_SCALE<D>, -LIFT));
        else e = __builtin_amdgcn_exp2f(x * LOG2_SCALE<D>) * 0x1p-40f;
        sc[nt][i / 4][i % 4] = e;
        l[nt] += e;
      }
    }
  }

  // Values at positions that are not there become zero, whatever they are.  Values that are not
  // finite, at positions that only some columns see: NaN in those, and taken out.  rows: LDS for
  // the unit's values, or where they lie.
  __device__ __forceinline__ void mask_values(R& u, int pos, uint32_t there, char* rows, bool in_rows) {
    const int lane = threadIdx.x & 63, c = lane & 15, qq = lane >> 4;
#pragma unroll
    for (int i = 0; i < NS; ++i) u.keep_v(i, there >> at_of(i, qq) & 1);
    if (!__any(u.odd())) return;
    constexpr int BYTES = D * sizeof(T);
    if (!in_rows) {
#pragma unroll
      for (int i = 0; i < NS; ++i) u.put_v(i, rows + at_of(i, qq) * BYTES, c);
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
#pragma unroll 1
    for (int at = 0; at < POS; ++at) {
      if (!(there >> at & 1)) continue;
      const T* mine = reinterpret_cast<const T*>(rows + at * BYTES) + qq * (D / 4);
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < JN; ++j) {
          const float y = Elem<T>::load(mine, r * JN + j);
          if (!(fabsf(y) < INFINITY)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if ((uint32_t)(pos + at) < (uint32_t)limit[nt]) o[nt][j][r] = NAN;
          }
        }
    }
    u.without_odd();
  }

  __device__ __forceinline__ void sums(const R& u, const f32x4 (&w)[NT][TILES]) {
    if constexpr (sizeof(T) == 2) {
      u32x4 hi[NT], lo[NT];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float a = w[nt][i / 2][2 * i % 4], b = w[nt][i / 2][2 * i % 4 + 1];
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
        for (int nt = 0; nt < NT; ++nt)
          o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, hi[nt]), o[nt][j], 0, 0, 0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(bf16x8, lo[nt]), o[nt][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
            o[nt][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(u.v[i][j], w[nt][i / 4][i % 4], o[nt][j], 0, 0, 0);
    }
  }
};

// The arena's slots of positions pos .., unit after unit: a window of 256 blocks' table
// entries in a wave's lanes.  (They are waited for where they are loaded, which waits for the
// units on their way too: seldom, with four a lane.)
template <int POS>
struct Slots {
  static constexpr int WIN = 4;
  const int32_t* entries;
  int first, a, b, c, d;  // block of lane 0's first entry; the lane's own, 64 apart
  int held;               // of those four
  int blk, off, next;   // of the next unit's first position
  int lo, hi;
  __device__ __forceinline__ Slots(const GroupAttnParams& p, const Shape& s, int pos, int end)
      : entries(p.tables + (int64_t)s.table * p.max_blocks), blk(pos / p.block_size), off(pos - blk * p.block_size),
        next(pos), lo(s.lo), hi(end) {
    fill(p);
  }
  __device__ __forceinline__ void fill(const GroupAttnParams& p) {
    const auto entry = [&](int i) {
      const uint32_t x = (uint32_t)blk + 64 * i + (threadIdx.x & 63);
      return x < (uint32_t)p.max_blocks ? entries[x] : -1;
    };
    first = blk;
    held = WIN;
    a = entry(0);
    b = entry(1);
    c = entry(2);
    d = entry(3);
    asm volatile("" : "+v"(a), "+v"(b), "+v"(c), "+v"(d));
  }
  // blocks to the right of `blk` that position off + n of it lies in
  __device__ __forceinline__ int blocks(const GroupAttnParams& p, int n) const {
    const uint32_t x = (uint32_t)(off + n);
    return p.block_inv ? (int)(x * p.block_inv >> 16) : x >= (uint32_t)p.block_size ? 1 : 0;
  }
  // The next unit's: lane x has position x mod POS's, slot 0 where the table names none; bits of
  // those positions that are there.
  __device__ __forceinline__ int take(const GroupAttnParams& p, uint32_t& there) {
    if (blk - first >= 64) {
      first += 64;
      a = b;
      b = c;
      c = d;
      --held;
    }
    const int last = blk + blocks(p, POS - 1) - first;
    if (last >= 64 * held) fill(p);
    const int x = threadIdx.x & (POS - 1), n = blocks(p, x), at = blk + n - first;
    int named = __shfl(a, at & 63, 64);
    if (last >= 64) {
      const int right = __shfl(b, at & 63, 64);
      named = at >= 64 ? right : named;
    }
    const bool ok = (uint32_t)named < p.num_blocks;
    const int slot = ok ? named * p.block_size + (off + x - n * p.block_size) : 0;
    there = (uint32_t)(__ballot(ok && (uint32_t)(next + x) < (uint32_t)hi && next + x >= lo) & ((1ull << POS) - 1));
    const int step = blocks(p, POS);
    next += POS;
    blk += step;
    off += POS - step * p.block_size;
    return slot;
  }
};

// The same where four positions on a boundary of four lie in one block, for a wave that brings the
// fours `four` and four + 1 of every unit: 64 units ahead, a lane each, so that a unit's are read
// from a lane.  (By the window of entries above it takes 590 of a unit's 3600 cycles, 94 us, not
// 88, for 48 requests of 24000 shared and 200 - 2000 own positions.)
template <int POS>
struct Fours {
  const int32_t* entries;
  int lo, hi, four;
  int first;           // position of lane 0's unit
  int slot_a, slot_b;  // of the two fours, 0 where the table names none
  uint32_t bits;       // positions that are there
  __device__ __forceinline__ Fours(const GroupAttnParams& p, const Shape& s, int pos, int end, int wave)
      : entries(p.tables + (int64_t)s.table * p.max_blocks), lo(s.lo), hi(end), four(2 * wave) {
    fill(p, pos);
  }
  __device__ __forceinline__ void fill(const GroupAttnParams& p, int pos) {
    constexpr int N = POS / 4;
    first = pos;
    const uint32_t mine = (uint32_t)pos + (threadIdx.x & 63) * POS;
    int named[N];
    uint32_t blk = mine / (uint32_t)p.block_size, off = mine - blk * p.block_size, my_off[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      my_off[i] = off;
      named[i] = blk < (uint32_t)p.max_blocks && mine + 4 * i < (uint32_t)hi ? entries[blk] : -1;
      off += 4;
      if (off >= (uint32_t)p.block_size) {
        off = 0;
        ++blk;
      }
    }
    bits = 0;
    slot_a = slot_b = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool ok = (uint32_t)named[i] < p.num_blocks;
      const int slot = ok ? named[i] * p.block_size + (int)my_off[i] : 0;
      slot_a = i == four ? slot : slot_a;
      slot_b = i == four + 1 ? slot : slot_b;
      bits |= ok ? 15u << 4 * i : 0u;
    }
    const int from = lo - (int)mine, to = hi - (int)mine;  // of the unit's positions
    bits &= from <= 0 ? 0xffffffffu : from >= POS ? 0u : 0xffffffffu << from;
    bits &= to >= POS ? 0xffffffffu : to <= 0 ? 0u : ~(0xffffffffu << to);
    asm volatile("" : "+v"(slot_a), "+v"(slot_b), "+v"(bits));  // waited for here
  }
  // Of the unit that begins at position pos: the fours' slots, the positions that are there.
  __device__ __forceinline__ void take(const GroupAttnParams& p, int pos, int (&slot)[2], uint32_t& there) {
    static_assert(POS == 32, "a bit a position");
    if (pos - first >= 64 * POS) fill(p, pos);
    const int at = (pos - first) / POS;
    slot[0] = __builtin_amdgcn_readlane(slot_a, at);
    slot[1] = __builtin_amdgcn_readlane(slot_b, at);
    there = __builtin_amdgcn_readlane(bits, at);
  }
};

// Sums of the waves, a tile of 16 columns at a time (a wave's part is room for a unit's values
// too), and units of bf16 K and V on their way and in use.
constexpr int RING = 4, UNIT_BYTES = 2 * 32 * 256;
template <int D, bool SHARED>
struct Scratch {
  union {
    float o[WAVES][16][ROW<D>];
    char ring[SHARED ? RING : 1][SHARED ? UNIT_BYTES : 16];
  };
};

// All that a workgroup has in LDS, as one object: of several the compiler knows which one the
// direct loads write, and waits for all of them before every read of it.
template <int D, bool SHARED>
struct Shared {
  Scratch<D, SHARED> scratch;
  Known known;
  uint32_t sum[3][WAVES];
  // the stretch's first entity (-1: none), costs and items of its kind and of the requests before it
  struct {
    int entity, items[2];
    uint32_t cost;
    Shape shape;
  } begin;
};

// The last position, and one more, that a part's columns see.
__device__ __forceinline__ int end_of(const Lists<true>& lists, const Shape& s, const Span& x) {
  if (x.entity < lists.p.G) return s.hi;
  return clamp_to(rows_of(lists, s.table).start + by_g(lists.p, x.tile + x.cols - 1) + 1, 0, s.hi);
}
// Units of an entity up to a position that its columns see.
__device__ __forceinline__ int units_to(const Shape& s, int end, int pos) {
  return end > s.lo ? (end - 1) / pos - s.lo / pos + 1 : 0;
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

// A part of an item of up to 16 NT columns, its units shared out to the waves: their sums,
// merged, to `dst` ([column][ROW]) or, where that is null, to the output rows.
template <typename T, int D, int NT, typename S, typename SlotsOf>
__device__ __forceinline__ void run_split(const Lists<true>& lists, const Shape& s, const Span& x,
                                          float* dst, S& scratch, SlotsOf slots_of) {
  const GroupAttnParams& p = lists.p;
  using R = Regs<T, D>;
  constexpr int JN = D / 16, POS = R::POS, TILES = R::TILES, NS = R::NS;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = lane & 15, q = lane >> 4;
  Columns<T, D, NT> cl;
  cl.clear();
  const int end = __builtin_amdgcn_readfirstlane(end_of(lists, s, x));
  const int n = min(x.upto, units_to(s, end, POS)) - x.first, pos0 = s.lo / POS * POS;
  const int first = x.first + (int)((int64_t)max(n, 0) * wave / WAVES);
  const int upto = x.first + (int)((int64_t)max(n, 0) * (wave + 1) / WAVES);
  if (first < upto) {
    const char* head_k = p.plane_k + (int64_t)x.kvh * D * sizeof(T);
    const char* head_v = p.plane_v + (int64_t)x.kvh * D * sizeof(T);
    auto slots = slots_of(pos0 + first * POS, end);
    R u;
    uint32_t there, coming;
    int slot = slots.take(p, there);
    const auto load_k = [&]() {
#pragma unroll
      for (int i = 0; i < TILES; ++i) u.load_k(i, head_k + __shfl(slot, i * 16 + c, 64) * p.row_bytes, q);
    };
    const auto load_v = [&]() {
#pragma unroll
      for (int i = 0; i < NS; ++i) u.load_v(i, head_v + __shfl(slot, at_of(i, q), 64) * p.row_bytes, c);
    };
    load_k();
    load_v();
    cl.load(lists, s, x, 0);
#pragma unroll 1
    for (int unit = first; unit < upto; ++unit) {
      const int pos = pos0 + unit * POS;
      const bool more = unit + 1 < upto;
      const bool edge = there != (uint32_t)((1ull << POS) - 1) || (uint32_t)(pos + POS) > (uint32_t)cl.all;
      f32x4 w[NT][TILES];
      cl.scores(u, w);
      if (more) {
        slot = slots.take(p, coming);
        load_k();
      }
      if (edge) cl.mask(w, pos, there);
      cl.weigh(w);
      if (edge) cl.mask_values(u, pos, there, reinterpret_cast<char*>(scratch.o[wave]), false);
      cl.sums(u, w);
      if (more) load_v();
      there = coming;
    }
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    if (nt * 16 >= x.cols) break;
    float* mine = scratch.o[wave][c];
    const float l = sum_over_q(cl.l[nt]);
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < JN; ++j) mine[q * (D / 4) + r * JN + j] = cl.o[nt][j][r];
    if (q == 0) {
      mine[D] = cl.top[nt];
      mine[D + 1] = l;
    }
    __syncthreads();
    const int col = t / 16, dim = t % 16 * JN;
    if (nt * 16 + col < x.cols) {
      float top = -INFINITY, sum = 0.0f, v[JN];
#pragma unroll
      for (int i = 0; i < WAVES; ++i) top = fmaxf(top, scratch.o[i][col][D]);
      const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
      for (int j = 0; j < JN; ++j) v[j] = 0.0f;
#pragma unroll
      for (int i = 0; i < WAVES; ++i) {
        const float f = __builtin_amdgcn_exp2f((scratch.o[i][col][D] - base) * LOG2_SCALE<D>);
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
        store_out<T, JN>(out_of<T>(p, s.row, x.tile + nt * 16 + col, x.kvh, D, dim), v);
      }
    }
    __syncthreads();
  }
}

// A part of an item of up to 64 NT columns of a bf16 model, its columns shared out to the waves:
// units come to them through a ring in LDS, by direct-to-LDS loads; a wave brings eight positions
// of a unit, four a load, which lie in one block.  K's 16-byte words of row r lie at word ^ r
// mod 16, so that the 16 rows that are read at once lie on different banks; V's rows are read
// whole.
template <int D, int NT, typename S>
__device__ __forceinline__ void run_shared(const Lists<true>& lists, const Shape& s, const Span& x,
                                           float* dst, S& scratch) {
  const GroupAttnParams& p = lists.p;
  using R = Regs<bf16_t, D>;
  constexpr int JN = D / 16, POS = R::POS, TILES = R::TILES, NS = R::NS, ROWB = D * 2;
  static_assert(ROWB == 256 && UNIT_BYTES == 2 * POS * ROWB, "sixteen words a row");
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = lane & 15, q = lane >> 4;
  Columns<bf16_t, D, NT> cl;
  cl.clear();
  const int skip = wave * 16 * NT;  // of the part's columns
  const int end = __builtin_amdgcn_readfirstlane(end_of(lists, s, x));
  const int upto = min(x.upto, units_to(s, end, POS)), pos0 = s.lo / POS * POS;
  if (x.first < upto) {
    const char* head_k = p.plane_k + (int64_t)x.kvh * ROWB;
    const char* head_v = p.plane_v + (int64_t)x.kvh * ROWB;
    Fours<POS> fours(p, s, pos0 + x.first * POS, end, wave);
    const int bytes = 3 * (int)p.row_bytes + ROWB, row_off = q * (int)p.row_bytes;
    uint32_t there[RING];  // bits of the units in the ring, oldest first
    // a unit's loads; nothing past the last, so that the waits of the last RING - 2 units are for all
    int fetched = x.first;
    const auto fetch = [&](uint32_t& bits) {
      if (fetched < upto) {
        int slot[2];
        fours.take(p, pos0 + fetched * POS, slot, bits);
        char* ring = scratch.ring[(fetched - x.first) % RING];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = wave * 8 + i * 4;
          const int64_t at = slot[i] * p.row_bytes;
          load_lds(head_k + at, bytes, ring + row * ROWB, row_off + ((c ^ ((row + q) & 15)) * 16), 0);
          load_lds(head_v + at, bytes, ring + POS * ROWB + row * ROWB, row_off + c * 16, 0);
        }
      }
      ++fetched;
    };
    fetch(there[0]);
    cl.load(lists, s, x, skip);
#pragma unroll
    for (int i = 1; i < RING - 1; ++i) fetch(there[i]);
#pragma unroll 1
    for (int unit = x.first; unit < upto; ++unit) {
      // this unit's loads have landed, those of the later ones may be on their way
      asm volatile("" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      if (unit + RING - 1 <= upto) KVR_WAIT_VMCNT(4 * (RING - 2));
      else KVR_WAIT_VMCNT(0);
      KVR_WAIT_LGKM0();
      __builtin_amdgcn_s_barrier();  // ... and the other waves', who are done with the unit before
      __builtin_amdgcn_sched_barrier(0);
      asm volatile("" ::: "memory");
      fetch(there[RING - 1]);
      char* ring = scratch.ring[(unit - x.first) % RING];
      const int pos = pos0 + unit * POS;
      const bool edge = there[0] != 0xffffffffu || (uint32_t)(pos + POS) > (uint32_t)cl.all;
      if (skip < x.cols) {
        f32x4 w[NT][TILES];
        R u;
#pragma unroll
        for (int i = 0; i < TILES; ++i)
#pragma unroll
          for (int kk = 0; kk < R::NK; ++kk)
            u.k[i][kk] = *reinterpret_cast<const u32x4*>(ring + (i * 16 + c) * ROWB + (((kk * 4 + q) ^ c) * 16));
        cl.scores(u, w);
        if (edge) cl.mask(w, pos, there[0]);
        cl.weigh(w);
#pragma unroll
        for (int i = 0; i < NS; ++i)
          u.v[i] = *reinterpret_cast<const u32x4*>(ring + POS * ROWB + at_of(i, q) * ROWB + c * 16);
        if (edge) cl.mask_values(u, pos, there[0], ring + POS * ROWB, true);
        cl.sums(u, w);
      }
#pragma unroll
      for (int i = 0; i + 1 < RING; ++i) there[i] = there[i + 1];
    }
    asm volatile("" ::: "memory");
    KVR_WAIT_VMCNT(0);
    KVR_WAIT_LGKM0();
    __builtin_amdgcn_s_barrier();  // the ring is free
    asm volatile("" ::: "memory");
  }
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int in = skip + nt * 16 + c;
    float l = sum_over_q(cl.l[nt]);
    if (in < x.cols) {
      float v[D / 4];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < JN; ++j) v[r * JN + j] = cl.o[nt][j][r];
      if (dst) {
        float* to = dst + (int64_t)in * ROW<D>;
#pragma unroll
        for (int i = 0; i < D / 4; i += 4)
          *reinterpret_cast<f32x4*>(to + q * (D / 4) + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
        if (q == 0) {
          to[D] = cl.top[nt];
          to[D + 1] = l;
        }
      } else {
        divide<D / 4>(v, l);
        store_out<bf16_t, D / 4>(out_of<bf16_t>(p, s.row, x.tile + in, x.kvh, D, q * (D / 4)), v);
      }
    }
  }
}

template <typename T, int D, int COLS>
__global__ __launch_bounds__(GA_NT, A_CU) void group_attn_kernel(GroupAttnParams p) {
  constexpr int POS = Regs<T, D>::POS;
  __shared__ __attribute__((aligned(1024))) Shared<D, (COLS > 32)> shared;
  auto& scratch = shared.scratch;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  // A CU's two workgroups read different heads (256 of a slot's 2 KB, say): reads of some heads take
  // longer, and a CU's return in order, so that all workgroups end nearer together (135 us, not 140,
  // for 64 requests of 600 - 6500 positions).
  const int w = blockIdx.x / p.nkv, kvh = (blockIdx.x + (w >= p.workers / 2 ? 1 : 0)) % p.nkv;
  const Lists<true> lists{p, &shared.known};
  fill_known(p, shared.known);
  if (t == 0) shared.begin.entity = -1;
  __syncthreads();

  // ---- the costs and items before each thread's entities ----
  const int E = p.G + p.R, per = (E + GA_NT - 1) / GA_NT;
  uint32_t mine[3] = {0, 0, 0};  // costs, items of prefixes, of requests
  Shape s{};
  for (int i = 0; i < per; ++i) {
    const int e = t * per + i;
    if (e < E) {
      s = shape_of<COLS, POS>(lists, e);
      mine[0] += s.all();
      mine[e < p.G ? 1 : 2] += s.tiles;
    }
  }
  uint32_t pre[3], total = 0;
#pragma unroll
  for (int k = 0; k < 3; ++k) {
    pre[k] = wave_scan(mine[k]);
    if (lane == 63) shared.sum[k][wave] = pre[k];
    pre[k] -= mine[k];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
#pragma unroll
    for (int k = 0; k < 3; ++k)
      if (i < wave) pre[k] += shared.sum[k][i];
    total += shared.sum[0][i];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const Stretches st(p.workers, total);
  const uint32_t u0 = st.begin(w), u1 = st.begin(w + 1);
  const bool starts = (uint32_t)w < st.workers && u0 >= pre[0] && u0 - pre[0] < mine[0];
  if (blockIdx.x == 0 && t == 0) {
    Plan h{};
    h.more = st.more;
    h.half = st.half;
    h.size = st.size;
    h.longer = st.longer;
    h.workers = st.workers;
    *p.plan = h;
  }
  // the thread whose entities the stretch begins in says so, and one workgroup what the second
  // kernel reads
  if (starts || blockIdx.x == 0)
    for (int i = 0; i < per; ++i) {
      const int e = t * per + i;
      if (e >= E) break;
      if (per > 1) s = shape_of<COLS, POS>(lists, e);
      const int kind = e < p.G ? 0 : 1;
      if (starts && u0 >= pre[0] && u0 - pre[0] < s.all()) {
        shared.begin.entity = e;
        shared.begin.items[0] = (int)pre[1];
        shared.begin.items[1] = (int)pre[2];
        shared.begin.cost = pre[0];
        shared.begin.shape = s;
      }
      if (blockIdx.x == 0)
        p.entities[e] = Entity{pre[0], s.item, (int)pre[1 + kind], s.row, s.tiles ? s.cols : 0, s.group, s.lo, s.cost};
      pre[0] += s.all();
      pre[1 + kind] += s.tiles;
    }
  __syncthreads();
  int e = __builtin_amdgcn_readfirstlane(shared.begin.entity);
  if (e < 0) return;
  uint32_t base = __builtin_amdgcn_readfirstlane(shared.begin.cost);
  int items[2] = {__builtin_amdgcn_readfirstlane(shared.begin.items[0]),
                  __builtin_amdgcn_readfirstlane(shared.begin.items[1])};
  s = uniform(shared.begin.shape);
  for (uint32_t u = u0; u < u1;) {
    while (u - base >= s.all() && e + 1 < E) {
      base += s.all();
      items[e < p.G ? 0 : 1] += s.tiles;
      s = uniform(shape_of<COLS, POS>(lists, ++e));
    }
    const uint32_t tile = quotient(u - base, s.item);
    if (tile >= (uint32_t)s.tiles) break;  // offsets that overlap so far that the costs passed 2^32
    const uint32_t from = u - base - tile * s.item, to = min(s.item, from + (u1 - u));
    u += to - from;
    // units whose first is here
    const int first = (max((int)from - START, 0) + s.cost - 1) / s.cost;
    const int upto = (max((int)to - START, 0) + s.cost - 1) / s.cost;
    if (upto <= first) continue;
    const int kind = e < p.G ? 0 : 1;
    // a request's item that is all here, with no prefix before it, goes straight out
    float* dst = nullptr;
    if (kind == 0 || s.lo > 0 || first > 0 || upto < s.units) {
      const int64_t slot = (int64_t)items[kind] + tile + w;
      if (slot >= p.slots[kind]) break;  // offsets that overlap: more items than rows make
      dst = p.part[kind] + (kvh * p.slots[kind] + slot) * p.part_cols[kind] * ROW<D>;
    }
    const Span x{e, (int)tile * COLS, min(COLS, s.cols - (int)tile * COLS), first, upto, kvh};
    const auto slots_of = [&](int pos, int end) { return Slots<POS>(p, s, pos, end); };
    if (COLS == 16 || x.cols <= 16) {
      run_split<T, D, 1>(lists, s, x, dst, scratch, slots_of);
    } else if constexpr (COLS == 32) {
      run_split<T, D, 2>(lists, s, x, dst, scratch, slots_of);
    } else if constexpr (COLS == 128) {
      if (x.cols <= 64) run_shared<D, 1>(lists, s, x, dst, scratch);
      else run_shared<D, 2>(lists, s, x, dst, scratch);
    }
  }
}

// Short calls: a workgroup to 16 columns of a request and kv head, all positions there, whose sums
// go straight out; a prefix is read by every request, through the first one's table, and there is
// no second kernel.
constexpr int SHORT_UNITS = 32;
// The slots of a wave's units, a quarter of those at most, looked up together.
template <int POS>
struct ShortSlots {
  static constexpr int N = SHORT_UNITS / WAVES * POS / 64;
  int slot[N], first, next;  // of positions first + 64 i + lane, -1 where none is
  __device__ __forceinline__ ShortSlots(const GroupAttnParams& p, const int32_t* head, const int32_t* own, int prefix,
                                        int pos, int end)
      : first(pos), next(pos) {
    int named[N], blk[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = pos + 64 * i + (threadIdx.x & 63);
      blk[i] = at / p.block_size;
      named[i] = at < end && blk[i] < p.max_blocks ? (at < prefix ? head : own)[blk[i]] : -1;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int at = pos + 64 * i + (threadIdx.x & 63);
      slot[i] = (uint32_t)named[i] < p.num_blocks ? named[i] * p.block_size + (at - blk[i] * p.block_size) : -1;
      asm volatile("" : "+v"(slot[i]));
    }
  }
  __device__ __forceinline__ int take(const GroupAttnParams&, uint32_t& there) {
    const int at = next - first, x = threadIdx.x & (POS - 1);
    int from = slot[0];
#pragma unroll
    for (int i = 1; i < N; ++i) from = at >= 64 * i ? slot[i] : from;
    const int mine = __shfl(from, (at & 63) + x, 64);
    there = (uint32_t)(__ballot(mine >= 0) & ((1ull << POS) - 1));
    next += POS;
    return max(mine, 0);
  }
};
template <typename T, int D>
__global__ __launch_bounds__(GA_NT, A_CU) void group_short_kernel(GroupAttnParams p) {
  constexpr int POS = Regs<T, D>::POS;
  static_assert(SHORT_UNITS / WAVES * POS % 64 == 0 && 64 % POS == 0, "whole units of a wave in its lanes");
  __shared__ struct {
    Scratch<D, false> scratch;
    Known known;
  } shared;
  const Lists<true> lists{p, &shared.known};
  fill_known(p, shared.known);
  __syncthreads();
  const int r = blockIdx.z, kvh = blockIdx.y, tile = blockIdx.x * 16;
  const Rows rows = rows_of(lists, r);
  Shape s{};
  s.row = rows.row;
  s.cols = rows.used * p.g;
  s.table = r;
  s.group = group_of(lists, r);
  s.hi = clamp_to(rows.end, 0, p.most_len);
  s = uniform(s);
  if (tile >= s.cols) return;
  const int prefix = s.group >= 0 ? lists.prefix(s.group) : 0;
  const int head = s.group >= 0 ? clamp_to(lists.offset(s.group), 0, p.R) : r;
  const int32_t *own = p.tables + (int64_t)r * p.max_blocks, *first = p.tables + (int64_t)head * p.max_blocks;
  const Span x{p.G + r, tile, min(16, s.cols - tile), 0, SHORT_UNITS, kvh};
  run_split<T, D, 1>(lists, s, x, nullptr, shared.scratch,
                     [&](int pos, int end) { return ShortSlots<POS>(p, first, own, prefix, pos, end); });
}

// Columns whose sums lie in several places: D / 4 lanes a column, a workgroup the next few
// columns of a request's kv head.  (All of them in one workgroup: 14.1 us, not 7.1, for 20 requests
// of 8 - 32 columns in five groups.)
template <int D>
constexpr int AT_ONCE = GA_NT / (D / 4);
template <typename T, int D, int COLS>
__global__ __launch_bounds__(GA_NT) void group_merge_kernel(GroupAttnParams p) {
  constexpr int LANES = D / 4, CHUNK = 8;
  const Stretches st(*p.plan);
  const Lists<false> lists{p, nullptr};
  const int64_t all = (int64_t)p.R * p.nkv;
  for (int64_t b = blockIdx.y; b < all; b += gridDim.y) {
    const int kvh = (int)(b % p.nkv), r = (int)(b / p.nkv);
    const Entity own = p.entities[p.G + r];
    const Rows x = rows_of(lists, r);
    const int cols = x.used * p.g, lane = threadIdx.x % LANES, dim = lane * 4;
    Entity pre{};
    if (own.group >= 0) pre = p.entities[own.group];
    for (int col = blockIdx.x * AT_ONCE<D> + threadIdx.x / LANES; col < cols; col += gridDim.x * AT_ONCE<D>) {
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
        const int a = st.holder(begin + START), z = st.holder(begin + y.item - y.cost);
        const int64_t slot = (int64_t)y.first + tile + a;
        if (slot < 0 || slot + (z - a) >= p.slots[k]) continue;
        n[k] = z - a + 1;
        src[k] = p.part[k] + ((kvh * p.slots[k] + slot) * p.part_cols[k] + (at[k] - tile * COLS)) * ROW<D>;
      }
      if (n[1] == 1 && own.lo == 0) continue;  // written by the first kernel
      float top = -INFINITY, l = 0.0f, o[4] = {0.0f, 0.0f, 0.0f, 0.0f};
      const int total = n[0] + n[1];
#pragma unroll 1
      for (int i0 = 0; i0 < total; i0 += CHUNK) {
        float2 ml[CHUNK];
        f32x4 v[CHUNK];
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) {  // past the last: the last again, not counted below
          const int k = min(i0 + i, total - 1);
          const float* part = k < n[0] ? src[0] + (int64_t)k * p.part_cols[0] * ROW<D>
                                       : src[1] + (int64_t)(k - n[0]) * p.part_cols[1] * ROW<D>;
          v[i] = *reinterpret_cast<const f32x4*>(part + dim);
          ml[i] = *reinterpret_cast<const float2*>(part + D);
        }
        float now = top;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i) now = fmaxf(now, ml[i].x);
        const float base = now == -INFINITY ? 0.0f : now;
        const float was = __builtin_amdgcn_exp2f((top - base) * LOG2_SCALE<D>);
        top = now;
        l *= was;
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] *= was;
#pragma unroll
        for (int i = 0; i < CHUNK; ++i)
          if (i0 + i < total) {
            const float f = __builtin_amdgcn_exp2f((ml[i].x - base) * LOG2_SCALE<D>);
            l = fmaf(ml[i].y, f, l);
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

// Columns of an item: the fewest that the average of what shares it fills (the groups' own sizes
// are known on the device alone; a large group among many small ones gets their narrow items).  More
// than 16 go through LDS in bf16, by loads that take rows on boundaries of 16 bytes, four to a block
// (128 at most: a wave's two tiles, with their sums, fill its registers; 64 gain nothing for what
// they fit).  Other arenas and block sizes have 16, and a prefix's reads up to eight times over.
int cols_of(const kv_model_desc& d, const Sizes& z, bool fours) {
  const int64_t cols = z.G > 0 ? (z.rows * z.g + z.G - 1) / z.G : z.g * std::min(z.max_query, z.rows);
  if (d.dtype == KV_BF16 && !fours) return 16;
  if (d.dtype != KV_BF16) return cols > 16 && d.head_dim < 128 ? 32 : 16;
  return cols > 16 ? 128 : 16;
}
// Workgroups of a kv head, a multiple of eight.
int most_workers(int nkv) { return std::max(8, CUS * A_CU / nkv / 8 * 8); }

// The workspace: the plan, the entities, the sums of prefixes and those of requests.  Their
// numbers grow with every size of a call, whichever kernel it takes.
struct GroupLayout {
  uint64_t entities, part[2], total;
  int part_cols[2];   // for the call's own kernel
  int64_t slots[2];
};
GroupLayout layout_of(const kv_model_desc& d, const Sizes& z, int cols) {
  const int64_t columns = z.rows * z.g, row = d.head_dim + 4, most = most_workers(d.num_kv_heads);
  const int64_t entity[2] = {z.G, z.R}, widest[2] = {std::min<int64_t>(128, columns),
                                                     std::min<int64_t>(128, z.g * std::min(z.max_query, z.rows))};
  GroupLayout L;
  L.entities = 256;
  L.part[0] = L.entities + (uint64_t)round_up((z.G + z.R) * (int64_t)sizeof(Entity), 256);
  for (int k = 0; k < 2; ++k) {
    const int64_t floats = k == 0 && z.G == 0 ? 0 : d.num_kv_heads * (columns + (entity[k] + most) * widest[k]) * row;
    (k == 0 ? L.part[1] : L.total) = L.part[k] + (uint64_t)round_up(4 * floats, 256);
    L.part_cols[k] = (int)std::min<int64_t>(cols, widest[k]);
    L.slots[k] = floats ? columns / cols + entity[k] + most_workers(d.num_kv_heads) : 0;
  }
  return L;
}

bool takes(const Sizes& z) {
  if (z.R > MOST_ROWS || z.rows > MOST_ROWS || z.G > MOST_ROWS || z.max_len > INT32_MAX) return false;
  return (z.R + z.G + z.rows * z.g / 8) * (z.max_len / 8 + 16) <= INT32_MAX;
}

// Whether a call is short, by the units that its bounds let an item have and by its items.  In us of
// a call, so and by the other two kernels, 32 q and 8 kv heads in bf16, prefix + own positions: 440
// + 60 of 4 requests (32 items) 10.3 and 14.3, of 64 (512) 16.7 and 25.8, of 256 (2048) 62.9
// and 63.0, of 512 122 and 113; 60 + 440 of 256 80 and 118; 900 + 100 of 4 requests 14.7 and
// 15.3, of 64 26.5 and 28.5, of 128 (1024) 47 and 38.
int64_t short_tiles(const GroupAttnParams& p) { return ((int64_t)p.g * std::min(p.max_query, p.rows) + 15) / 16; }
bool is_short(const GroupAttnParams& p, int pos) {
  const int units = (int)(((int64_t)p.most_len + pos - 1) / pos);
  return units <= SHORT_UNITS && p.R * (int64_t)p.nkv * short_tiles(p) <= (units <= SHORT_UNITS / 2 ? 2048 : 512);
}

template <typename T, int D, int COLS>
void launch_cols(const GroupAttnParams& p, hipStream_t s) {
  hipLaunchKernelGGL((group_attn_kernel<T, D, COLS>), dim3((unsigned)(p.workers * p.nkv)), dim3(GA_NT), 0, s, p);
  const int64_t columns = (int64_t)p.g * std::min(p.max_query, p.rows);
  const int64_t wide = std::min<int64_t>((columns + AT_ONCE<D> - 1) / AT_ONCE<D>, 1 << 14);
  const int64_t high = std::min<int64_t>({(int64_t)p.R * p.nkv, 65535, (1 << 22) / wide});
  hipLaunchKernelGGL((group_merge_kernel<T, D, COLS>), dim3((unsigned)wide, (unsigned)high), dim3(GA_NT), 0, s, p);
}
template <typename T, int D>
void launch(int cols, const GroupAttnParams& p, hipStream_t s) {
  if (is_short(p, Regs<T, D>::POS)) {
    hipLaunchKernelGGL((group_short_kernel<T, D>), dim3((unsigned)short_tiles(p), (unsigned)p.nkv, (unsigned)p.R),
                       dim3(GA_NT), 0, s, p);
  } else if (cols == 16) {
    launch_cols<T, D, 16>(p, s);
  } else if constexpr (sizeof(T) == 2) {
    launch_cols<T, D, 128>(p, s);
  } else if constexpr (D < 128) {
    launch_cols<T, D, 32>(p, s);
  }
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
  return layout_of(*desc, {num_requests, rows, num_groups, max_query, max_len, desc->num_q_heads / desc->num_kv_heads}, 16)
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
  if (q == out && rows > 1 && q_stride != out_stride)
    return kvr_err::set(KV_EINVAL, "out over q needs the same stride");
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)(q_stride * e) | (uintptr_t)(out_stride * e) | (uintptr_t)q_offsets |
       (uintptr_t)lens | (uintptr_t)tables | (uintptr_t)group_offsets | (uintptr_t)prefix_lens |
       (uintptr_t)arena->base) % 4 != 0)
    return kvr_err::set(KV_EINVAL, "the arrays, the strides and the arena need boundaries of 4 bytes");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
  const int g = d.num_q_heads / d.num_kv_heads;
  const Sizes z{R, rows, num_groups, max_query, max_len, g};
  if (!takes(z)) return kvr_err::set(KV_EINVAL, "max_len or the work of one call above 2^31: split the query rows");
  const int cols = cols_of(d, z, (uintptr_t)arena->base % 16 == 0 && arena->block_size % 4 == 0);
  const GroupLayout L = layout_of(d, z, cols);
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
  p.workers = most_workers(d.num_kv_heads);
  char* ws = static_cast<char*>(workspace);
  p.plan = reinterpret_cast<Plan*>(ws);
  p.entities = reinterpret_cast<Entity*>(ws + L.entities);
  for (int k = 0; k < 2; ++k) {
    p.part[k] = reinterpret_cast<float*>(ws + L.part[k]);
    p.part_cols[k] = L.part_cols[k];
    p.slots[k] = L.slots[k];
  }
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d.dtype == KV_BF16) launch<bf16_t, 128>(cols, p, s);
  else if (d.head_dim == 128) launch<float, 128>(cols, p, s);
  else if (d.head_dim == 64) launch<float, 64>(cols, p, s);
  else launch<float, 32>(cols, p, s);
  return launched();
}

}  // extern "C"

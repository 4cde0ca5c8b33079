// Attention over a packed arena (kvr_packed.h).
//
// The query rows of a request that share a kv head are columns: column i g + h is
// query i of q head h of the group.  An item is one request's next 16 NT columns of one
// kv head; its work comes in units of 32 positions.  Every wave takes an equal
// stretch of the units of all items, request after request, whatever the lengths (they
// are known on the device alone), so that all waves end together.  Where a stretch
// ends inside an item the wave leaves the item's sums so far; the four waves of a
// workgroup, whose stretches follow each other, merge theirs, and a second kernel
// merges what is left between workgroups.
//
// A unit in a wave's registers, lane (q, c) = (lane / 16, lane % 16):
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16, 16 positions a tile: position c's dims
//   q d/4 .. are the lane's K operand, d/8 bytes and one scale; the conversions to bf16
//   are exact.  The lane gets the scores of positions 4q .. 4q+3 for column c.
//   Online softmax per column, exp2 domain, rescaled only where the maximum rose by
//   more than 2^SLACK.
//   O = P V: the lane's weights of the unit's two tiles are the A operand as they are,
//   positions 4q .. 4q+3 of both being its eight k's; V's layout gives the lane the dims
//   c d/16 .. of the same positions, which it pairs into the B operands of d/16 products.
//   A weight may be 2^SLACK and 2^31 of them add up, so the sums of large V could pass the
//   largest fp32 number where their quotient, which lies between the V's, does not.  From
//   the first unit with a scale of 2^65 or more on, a wave takes an item's maxima LIFT too high
//   and so all weights and their sum that much smaller: 2^31 2^SLACK 2^-LIFT 1.5 2^127 is below
//   2^127, 2^31 2^SLACK 6 2^64 without it.  (Exponents are then rounded to 2^-19 and V below
//   2^-86 may be lost.  Scores of 2^30 have no room for LIFT.)
//   (Up to 8 columns, a softmax a tile in the two halves of the 16, merged at the end,
//   spares half the exponentials and took as long: 30.2 us against 29.5 below.)
// Records reach a wave through a ring of its own in LDS, by direct-to-LDS loads: a
// record is 17 d contiguous bytes, K's and V's lane by lane in the operands' order, so
// the reads back are linear, and records are on their way without a register.
// Weights enter the product as a bf16 number and the bf16 rest (2^-17 of a weight lost),
// in fp32 models as three (as do the queries): rounding them once would cost more than
// the output's own rounding where few positions weigh, and the products are not what
// bounds the kernel.
//
// What bounds it: the records' way from HBM and what a call costs once.  16 requests of
// 2048 - 16384 positions (8 kv heads of 128, 4 q heads each, 124 MB of records), one query
// row each: 29.7 us.  1.8 of them are the plan (2.8 with 1100 requests, 9.7 with 4000, which
// every workgroup reads), 4.6 the way to the first record (three loads that follow each other,
// while other waves' records keep the memory busy), 2 - 3 the merges.  Two requests of
// 150 - 200 thousand positions (403 MB): 78 us, of which the records' way at a large read's
// rate is 67.  One to five query rows of 40 requests of 300 - 4000 positions (5 q heads a kv
// head, 88 MB, 34 of them twice): 29.6 us, 106 MB past the L2 caches.
//   Workgroups a CU and records a ring: three and four.  Three and six took 31.2 us, two
// and eight 33.7, four and four 31.1 (the long ones 79, 85 and 81).  Two column tiles need
// the registers of two a CU: with three, registers spill, 56 us against 35 on the 40
// requests.
//   As many waves as run at once: half as many more took 38 us, twice as many 37; the
// stretches are equal, so more of them only merge more.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "dma.h"
#include "host.h"
#include "kvr_packed.h"
#include "launch.h"
#include "packed.h"

namespace kvr {
namespace {

constexpr int PA_NT = 256;         // four waves
constexpr float SLACK = 8.0f;      // rescale slack, log2 units
constexpr float LIFT = 40.0f;      // of maxima over large values, log2 units
constexpr int MOST_ROWS = 1 << 24; // query rows and requests of a call

constexpr int TILES = 2;           // tiles of a unit
constexpr int UNIT = 16 * TILES;   // positions of a unit

template <typename T> struct Split;  // bf16 numbers that stand for a query, for a weight
template <> struct Split<bf16_t> { static constexpr int Q = 1, P = 2; };
template <> struct Split<float> { static constexpr int Q = 3, P = 3; };

// The item that a workgroup began and left open, for the second kernel: its columns (0:
// none), first query row and column tile, the wave that began it, and the workgroups
// that hold sums of it.
struct OpenItem {
  int cols, row, tile, wave, groups;
};

struct PackedAttnParams {
  PackedLayer packed;
  uint32_t num_blocks;           // of the arena, or all that an entry can name
  const char* q;                 // rows of queries, model dtype
  char* out;
  int64_t q_stride, out_stride;  // bytes
  const int32_t* q_offsets;      // null: row r is request r's
  int64_t rows;
  const int32_t* lens;
  const int32_t* tables;
  int R, max_blocks;
  int g;                         // q heads of a kv head
  uint32_t g_inv;                // ceil(2^32 / g), 0 for g = 1: n / g of n < 2^28 is the product's high half
  int max_query;                 // rows of a request past it are left out: the sums have no room
  int most_len;                  // positions of a request: max_len, or what its table holds
  int start;                     // units that an item's start counts as
  int whole;                     // units of a stretch where a workgroup has an item to itself, else 0
  int workers;                   // stretches per kv head, a multiple of four
  int part_cols;                 // columns of a slot of sums
  OpenItem* open;                // [workers / 4]
  float* part;                   // [nkv][workers][2][part_cols][ROW]: an item begun before, one left open
};

// f(0), f(1), .. with the index a constant
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

// Workgroups a CU holds by their registers, and the records of a wave's ring that
// then fit its LDS.
constexpr int occupancy_of(bool f32, int d, int nt) {
  return f32 && d == 128 ? 3 - nt : 4 - nt;
}
constexpr int ring_of(int occupancy) { return occupancy == 3 ? 4 : 8; }

__device__ __forceinline__ int by_g(const PackedAttnParams& p, int n) {
  return p.g_inv ? (int)__umulhi((uint32_t)n, p.g_inv) : n;
}
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
// Stretches: all units in workers parts, equal but for LATER units: the waves of a CU's
// second workgroup take that many fewer than those of its first, its third's twice as
// many fewer.  (Workgroups come to the CUs in their order; the oldest on a CU is served
// first.)  Two requests of 150 - 200 thousand positions 77.0 us, 16 of 2048 - 16384 29.6,
// 64 of 2 heads 19.5; equal parts 78.3, 30.7 and 20.9, three units 76.6, 30.5 and 21.2.
// Parts too short for that are equal.
constexpr uint32_t LATER = 2;
template <int OCC>
struct Stretches {
  // the first `longer` ones are a unit longer; turn: waves of the CUs' first workgroups
  uint32_t workers, size, longer, turn, later;
  __device__ __forceinline__ Stretches(uint32_t most, uint32_t total, uint32_t whole) {
    turn = most / OCC;
    if (whole) {
      workers = most;
      size = whole;
      longer = later = 0;
      return;
    }
    workers = min(most, total);  // a unit each at least
    later = OCC > 1 && total / (2 * LATER) >= most ? LATER : 0;
    total += less(workers);
    size = total ? quotient(total, workers) : 0;
    longer = total - size * workers;
  }
  __device__ __forceinline__ uint32_t less(uint32_t w) const {  // of all before w
    return later * ((uint32_t)max((int)(w - turn), 0) + (uint32_t)max((int)(w - 2 * turn), 0));
  }
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * size + min(w, longer) - less(w); }
  __device__ __forceinline__ uint32_t holder(uint32_t u) const {  // whose unit u is
    uint32_t a = 0, b = workers - 1;
    while (a < b) {
      const uint32_t m = (a + b + 1) / 2;
      if (begin(m) <= u) a = m;
      else b = m - 1;
    }
    return a;
  }
};

struct Request {
  int row, m, len, want;  // first query row, rows, positions there are, position after the last of these rows
  int tiles, steps;       // column tiles, units of each
  uint32_t item;          // what an item counts: its units and its start
  __device__ __forceinline__ uint32_t units() const { return (uint32_t)tiles * item; }
};
template <int COLS>
__device__ __forceinline__ Request make_request(const PackedAttnParams& p, int row, int m, int want) {
  Request q;
  q.row = row;
  q.m = m;
  q.want = want;
  q.len = max(0, min(want, p.most_len));
  q.tiles = (int)(((int64_t)m * p.g + COLS - 1) / COLS);
  q.steps = max(1, (int)(((int64_t)q.len + UNIT - 1) / UNIT));
  q.item = (uint32_t)(p.whole ? p.whole * (PA_NT / 64) : q.steps + p.start);
  return q;
}
template <int COLS>
__device__ __forceinline__ Request get_request(const PackedAttnParams& p, int r) {
  int row = r, m = 1, want = p.lens[r];
  if (p.q_offsets) {
    const int a = p.q_offsets[r], b = p.q_offsets[r + 1];
    row = min(max(a, 0), (int)p.rows);
    const int all = max(min(b, (int)p.rows) - row, 0);
    m = min(all, p.max_query);
    want = max(want, 0) - (all - m);  // the rows left out are the last ones
  }
  return make_request<COLS>(p, row, m, want);
}

// The scale of byte i of a word.  The conversions read the exponent alone, whatever the
// neighbouring bytes leave in the sign and the mantissa.
__device__ __forceinline__ float scale_of(uint32_t word, int i) {
  return __uint_as_float(i == 3 ? word >> 1 : word << (23 - 8 * i));
}

// Masks of a word's first n bytes, and of its bytes that are 255.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << 8 * n) - 1; }
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  return (((w & 0x7f7f7f7fu) + 0x01010101u) & w & 0x80808080u) >> 7;  // 1 in each
}

template <int BYTES>
__device__ __forceinline__ void load_words(const char* p, uint32_t* w) {
  if constexpr (BYTES == 16) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
  } else if constexpr (BYTES == 8) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    w[0] = u.x; w[1] = u.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// two values of a word's byte SEL as bf16, exactly
template <int SEL>
__device__ __forceinline__ uint32_t pair_of(uint32_t word, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, SEL));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

// The nearest number to a query's that does not round to an infinite bf16 one (of an infinite
// query it leaves an infinite rest).
__device__ __forceinline__ float near_bf16(float v) { return __builtin_amdgcn_fmed3f(v, -0x1.fep127f, 0x1.fep127f); }

// What a wave's stretch holds of items that are not its own alone: of one begun before
// it ([0]), of one it leaves open ([1]).
struct Stretch {
  int cols[2];   // columns, 0: no such item
  int row[2], tile[2];
  int flags;     // 1: the item begun before ends in it; 2, 4: [0]'s, [1]'s sums are in the wave's ring
  uint32_t end;  // the open item's units' end
};

// Floats of a partial's row: on boundaries of 16 bytes, of 8 where 16 rows have to fit a
// ring of the smallest heads.
constexpr int row_of(int d) { return d == 32 ? d + 2 : d + 4; }
template <int D>
constexpr int ROW = row_of(D);

// Columns are merged 256 / D at a time: a lane has four dims of one of them.  A partial
// is D sums, a maximum and a sum of weights; n of them go in their order.
template <int D>
constexpr int LANES = D / 4;
template <int D>
constexpr int AT_ONCE = 64 / LANES<D>;
struct Column {
  float m, l, o[4];
};
template <int D>
__device__ __forceinline__ int dim_of(int lane) { return lane % LANES<D> * 4; }
template <int D>
__device__ __forceinline__ void load_part(const float* part, int dim, float2& ml, float* o) {
  ml = *reinterpret_cast<const float2*>(part + D);
  if constexpr (ROW<D> % 4 == 0) {
    const float4 a = *reinterpret_cast<const float4*>(part + dim);
    o[0] = a.x; o[1] = a.y; o[2] = a.z; o[3] = a.w;
  } else {
    const float2 a = *reinterpret_cast<const float2*>(part + dim), b = *reinterpret_cast<const float2*>(part + dim + 2);
    o[0] = a.x; o[1] = a.y; o[2] = b.x; o[3] = b.y;
  }
}
template <int D>
__device__ __forceinline__ void store_part(float* part, int dim, const float* o) {
  if constexpr (ROW<D> % 4 == 0) {
    *reinterpret_cast<float4*>(part + dim) = make_float4(o[0], o[1], o[2], o[3]);
  } else {
    reinterpret_cast<float2*>(part + dim)[0] = make_float2(o[0], o[1]);
    reinterpret_cast<float2*>(part + dim)[1] = make_float2(o[2], o[3]);
  }
}
template <int D, int CHUNK, typename SRC>  // CHUNK: partials whose loads are on their way together
__device__ __forceinline__ Column merge_column(SRC src, int n, int lane) {
  Column x{-INFINITY, 0.0f, {0.0f, 0.0f, 0.0f, 0.0f}};
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += CHUNK) {
    float2 ml[CHUNK];
    float o[CHUNK][4];
#pragma unroll
    for (int i = 0; i < CHUNK; ++i)  // past the last: the last again, not counted below
      src(min(i0 + i, n - 1), [&](const float* part) { load_part<D>(part, dim_of<D>(lane), ml[i], o[i]); });
    float top = x.m;
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) top = fmaxf(top, ml[i].x);
    const float base = top == -INFINITY ? 0.0f : top;
    const float was = __builtin_amdgcn_exp2f(x.m - base);
    x.m = top;
    x.l *= was;
#pragma unroll
    for (int d = 0; d < 4; ++d) x.o[d] *= was;
#pragma unroll
    for (int i = 0; i < CHUNK; ++i) {
      const float f = i0 + i < n ? __builtin_amdgcn_exp2f(ml[i].x - base) : 0.0f;
      x.l = fmaf(ml[i].y, f, x.l);
#pragma unroll
      for (int d = 0; d < 4; ++d) x.o[d] = fmaf(o[i][d], f, x.o[d]);
    }
  }
  return x;
}

// A merged column of a tile as its output row at kv head kvh, the tile's request's query
// rows from `row` on, or as a partial.
template <typename T, int D, int COLS>
__device__ __forceinline__ void put_out(const PackedAttnParams& p, int row, int tile, int col, int kvh, int lane,
                                        const Column& v) {
  const int gc = tile * COLS + col, i = by_g(p, gc);
  T* dst = reinterpret_cast<T*>(p.out + (int64_t)(row + i) * p.out_stride) +
           (int64_t)(kvh * p.g + gc - i * p.g) * D + dim_of<D>(lane);
  const float inv = v.l == 0.0f ? 0.0f : 1.0f / v.l;
  float x[4];
#pragma unroll
  for (int d = 0; d < 4; ++d) x[d] = v.l == 0.0f ? 0.0f : v.o[d] * inv;
  if constexpr (sizeof(T) == 2) {
    typedef uint32_t u32x2_a4 __attribute__((ext_vector_type(2), aligned(4)));
    *reinterpret_cast<u32x2_a4*>(dst) = u32x2_a4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3])};
  } else {
    *reinterpret_cast<f32x4_a4*>(dst) = f32x4{x[0], x[1], x[2], x[3]};
  }
}
template <int D>
__device__ __forceinline__ void put_part(float* dst, int lane, const Column& v) {
  store_part<D>(dst, dim_of<D>(lane), v.o);
  if (dim_of<D>(lane) == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(v.m, v.l);
}

template <typename T, int D, int NT, int OCC>
__global__ __launch_bounds__(PA_NT, OCC) void packed_attn_kernel(PackedAttnParams p) {
  constexpr int COLS = 16 * NT;           // columns of an item
  constexpr int W = D / 32, DT = D / 16;  // words a tile; dims a lane, P.V products
  constexpr int QP = Split<T>::Q, PP = Split<T>::P;
  constexpr int NV = 4 * TILES;           // scores of a lane and column
  constexpr int REC = 17 * D, RING = ring_of(OCC), LOADS = (16 * D + 1023) / 1024 + 1;
  __shared__ __attribute__((aligned(16))) char s_ring[PA_NT / 64][RING * REC];
  static_assert(RING % TILES == 0, "units do not wrap in the ring");
  static_assert(RING * REC >= NT * 64 * ROW<D>, "all columns' rows fit the ring");
  constexpr int WAVES = PA_NT / 64;
  __shared__ uint32_t s_wave[WAVES];
  __shared__ Stretch s_str[WAVES];
  __shared__ int s_begin[WAVES][5];  // where a wave's stretch begins: request, its first unit, row, rows, length
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), c = lane & 15, q = lane >> 4;
  const int nkv = p.packed.nkv, g = p.g;
  const int kvh = blockIdx.x % nkv, w = blockIdx.x / nkv * WAVES + wave;

  // ---- the units before each thread's requests ----
  const int per = (p.R + PA_NT - 1) / PA_NT;
  uint32_t mine = 0;
  Request rq{};
  for (int i = 0; i < per; ++i)
    if (t * per + i < p.R) {
      rq = get_request<COLS>(p, t * per + i);
      mine += rq.units();
    }
  uint32_t pre = wave_scan(mine);
  if (lane == 63) s_wave[wave] = pre;
  if (lane == 0) {
    s_str[wave] = Stretch{};
    s_begin[wave][0] = -1;
  }
  __syncthreads();
  uint32_t total = 0;
  pre -= mine;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    if (i < wave) pre += s_wave[i];
    total += s_wave[i];
  }
  total = __builtin_amdgcn_readfirstlane(total);
  const Stretches<OCC> st(p.workers, total, p.whole);
  // the thread whose requests hold a wave's first unit says so
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    const uint32_t v = blockIdx.x / nkv * WAVES + i, first = st.begin(v);
    if (v < st.workers && first >= pre && first - pre < mine) {
      s_begin[i][0] = t * per;
      s_begin[i][1] = (int)pre;
      s_begin[i][2] = rq.row;
      s_begin[i][3] = rq.m;
      s_begin[i][4] = rq.want;
    }
  }
  __syncthreads();

  float* const slots = p.part + ((int64_t)kvh * p.workers + w) * 2 * p.part_cols * ROW<D>;
  const auto begin_of = [&](int i) { return __builtin_amdgcn_readfirstlane(s_begin[wave][i]); };
  int r = begin_of(0);
  if (r >= 0) {
    const uint32_t u0 = st.begin(w), u1 = st.begin(w + 1);
    uint32_t base = begin_of(1);
    rq = per == 1 ? make_request<COLS>(p, begin_of(2), begin_of(3), begin_of(4)) : get_request<COLS>(p, r);

    const int B = p.packed.block_size, tpb = B / PK_TILE;
    const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
    const char* head = p.packed.base + (int64_t)kvh * tpb * (17 * D);
    const int64_t block_bytes = (int64_t)nkv * tpb * (17 * D);
    char* const ring = s_ring[wave];
    const int k_off = c * (D / 2) + q * (D / 8), v_off = 8 * D + q * (2 * D) + c * (D / 8);
    const int ks_off = 16 * D + c * (D / 32) + q * D / 128, vs_off = 16 * D + D / 2 + q * (D / 8) + c * D / 512 * 4;

    for (uint32_t u = u0; u < u1;) {
      // ---- the stretch's part of one item ----
      while (u - base >= rq.units() && r + 1 < p.R) {
        base += rq.units();
        rq = get_request<COLS>(p, ++r);
      }
      const uint32_t item = quotient(u - base, rq.item);
      if (item >= (uint32_t)rq.tiles) break;  // offsets that overlap so far that the units passed 2^32
      const int tile = (int)item;
      const uint32_t from = u - base - item * rq.item, to = min(rq.item, from + (u1 - u));
      const int start = (int)rq.item - rq.steps, first = max((int)from - start, 0), upto = (int)to - start;
      u += to - from;
      if (upto <= 0) continue;  // of the start alone
      const int cols = min(COLS, rq.m * g - tile * COLS);  // of this tile
      // positions that every column sees, and that any does
      const int i_lo = by_g(p, tile * COLS), i_hi = by_g(p, tile * COLS + cols - 1);
      const int all = min(rq.len, rq.want - rq.m + i_lo + 1), some = min(rq.len, rq.want - rq.m + i_hi + 1);
      const int stop = min(upto, (int)(((uint32_t)max(some, 0) + UNIT - 1) / UNIT));

      // 64 table entries, one a lane, and the queries: on their way ahead of the records
      const int32_t* table = p.tables + (int64_t)r * p.max_blocks;
      int next = first * TILES, bi = next / tpb, ti = next - bi * tpb;  // the next record, its block and place in it
      int window = bi, tab = bi + lane < p.max_blocks ? table[bi + lane] : -1;
      constexpr int QV = 8 * (int)sizeof(T) / 16;  // 16-byte pieces of eight dims
      f32x4 qraw[NT][W][QV];
      int limit[NT];  // positions the lane's column sees
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int col = nt * 16 + c, gc = tile * COLS + min(col, cols - 1), i = by_g(p, gc);
        limit[nt] = col < cols ? min(rq.len, rq.want - rq.m + i + 1) : some;
        const T* src = reinterpret_cast<const T*>(p.q + (int64_t)(rq.row + i) * p.q_stride) +
                       (int64_t)(kvh * g + gc - i * g) * D + q * (D / 4);
#pragma unroll
        for (int s = 0; s < W; ++s)
#pragma unroll
          for (int e = 0; e < QV; ++e) qraw[nt][s][e] = reinterpret_cast<const f32x4_a4*>(src + 8 * s)[e];
      }

      // the ring.  Entries are waited for where they are loaded, not at every use: that
      // would wait for the ring's loads too.
      asm volatile("" : "+v"(tab));
      auto entries = [&](int b0) {
        int e = b0 + lane < p.max_blocks ? table[b0 + lane] : -1;
        asm volatile("" : "+v"(e));
        return e;
      };
      const int last = stop * TILES;
      int put = 0, get = 0;   // bytes into the ring
      bool broken = false;    // a block is not in the arena
      auto issue = [&]() {
        if (bi - window >= 64) {
          window = bi;
          tab = entries(bi);
        }
        const int e = __builtin_amdgcn_readlane(tab, bi - window);
        const bool in = (uint32_t)e < p.num_blocks;
        broken |= !in;
        const char* rec = head + (in ? e : 0) * block_bytes + (int64_t)ti * REC;
        constexpr int FULL = 16 * D / 1024;
#pragma unroll
        for (int i = 0; i < FULL; ++i) load_lds(rec, REC, ring + put + 1024 * i, lane * 16, 1024 * i);
        if (FULL == 0 && lane < D) load_lds(rec, REC, ring + put, lane * 16, 0);
        if (lane < D / 16) load_lds(rec, REC, ring + put + 16 * D, lane * 16, 16 * D);
        put = put == (RING - 1) * REC ? 0 : put + REC;
        ++next;
        if (++ti == tpb) {
          ti = 0;
          ++bi;
        }
      };
#pragma unroll 1
      for (int i = 0; i < RING && next < last; ++i) issue();

      bf16x8 qf[NT][QP][W];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const bool used = nt * 16 + c < cols;
#pragma unroll
        for (int s = 0; s < W; ++s) {
          if constexpr (QP == 1) {
            qf[nt][0][s] = used ? __builtin_bit_cast(bf16x8, qraw[nt][s][0]) : bf16x8{};
          } else {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = used ? qraw[nt][s][e / 4 % QV][e % 4] : 0.0f;
#pragma unroll
            for (int part = 0; part < QP; ++part) {
              union { uint32_t w[4]; bf16x8 f; } f;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                f.w[e] = part ? pack_bf16(x[2 * e], x[2 * e + 1]) : pack_bf16(near_bf16(x[2 * e]), near_bf16(x[2 * e + 1]));
                x[2 * e] -= __uint_as_float(f.w[e] << 16);
                x[2 * e + 1] -= __uint_as_float(f.w[e] & 0xffff0000u);
              }
              qf[nt][part][s] = f.f;
            }
          }
        }
      }
      float m_run[NT], l_run[NT];
      f32x4 o[NT][DT];
      float lift = 0.0f;             // LIFT from the first large scale on
      uint32_t watch = 0x80808080u;  // and then 0
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m_run[nt] = -INFINITY;
        l_run[nt] = 0.0f;
#pragma unroll
        for (int j = 0; j < DT; ++j) o[nt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      }

      // sums relative to other maxima
      auto rescale = [&](int nt, float m_new) {
        const float alpha = m_new == m_run[nt] ? 1.0f : __builtin_amdgcn_exp2f(m_run[nt] - m_new);
        l_run[nt] *= alpha;
        m_run[nt] = m_new;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f = __shfl(alpha, 4 * q + j, 64);  // column 4q + j's
#pragma unroll
          for (int d = 0; d < DT; ++d) o[nt][d][j] *= f;
        }
      };

      for (int kt = first; kt < stop; ++kt) {
        // this unit's records have landed; of those behind it, RING - TILES at most are on their way
        const int behind = next - (kt + 1) * TILES;
        if (behind >= RING - TILES) KVR_WAIT_VMCNT((RING - TILES) * LOADS);
        else if (RING - TILES > TILES && behind >= RING - 2 * TILES) KVR_WAIT_VMCNT((RING - 2 * TILES) * LOADS);
        else KVR_WAIT_VMCNT(0);
        asm volatile("" ::: "memory");  // the reads below stay below
        // record x of the unit: TILES divides the ring into whole units
        auto at = [&](int x) { return ring + get + x * REC; };
        const bool whole = (int64_t)(kt + 1) * UNIT <= all && !broken;
        // scores
        uint32_t kw[TILES][W], ks[TILES];
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
          load_words<D / 8>(at(x) + k_off, kw[x]);
          ks[x] = (uint8_t)at(x)[ks_off];
        }
        f32x4 st[NT][TILES];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int x = 0; x < TILES; ++x) st[nt][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int s = 0; s < W; ++s)
#pragma unroll
          for (int x = 0; x < TILES; ++x) {
            const float scale = scale_of(ks[x], 0);
            union { uint32_t w[4]; bf16x8 f; } kf;
            kf.w[0] = pair_of<0>(kw[x][s], scale);
            kf.w[1] = pair_of<1>(kw[x][s], scale);
            kf.w[2] = pair_of<2>(kw[x][s], scale);
            kf.w[3] = pair_of<3>(kw[x][s], scale);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int part = 0; part < QP; ++part)
                st[nt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.f, qf[nt][part][s], st[nt][x], 0, 0, 0);
          }
        float sc[NT][NV];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < NV; ++i) sc[nt][i] = st[nt][i / 4][i % 4];
        const int p0 = kt * UNIT + 4 * q;  // the lane's first position of the unit's first tile
        uint32_t vw[TILES][W], vs[TILES];
#pragma unroll
        for (int x = 0; x < TILES; ++x) {
          load_words<D / 8>(at(x) + v_off, vw[x]);
          vs[x] = *reinterpret_cast<const uint32_t*>(at(x) + vs_off);
        }
        bool nan_v = false;
        if (!whole) {
          // positions past a column's limit and in blocks that are not there leave its
          // softmax; V there may hold any bits, and 0 times them is not 0
          int in = (1 << TILES) - 1;  // the unit's tiles whose blocks are in the arena
          if (broken) {
            in = 0;
#pragma unroll 1
            for (int x = 0; x < TILES; ++x) {
              const int b = (kt * TILES + x) / tpb;
              in |= (int)(b < p.max_blocks && (uint32_t)table[b] < p.num_blocks) << x;
            }
          }
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            const bool gone = !(in >> (i / 4) & 1);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if (gone || p0 + 16 * (i / 4) + i % 4 >= limit[nt]) sc[nt][i] = -INFINITY;
          }
          uint32_t nan = 0;
#pragma unroll
          for (int x = 0; x < TILES; ++x) {
            const int n = in >> x & 1 ? some - (p0 + 16 * x) : 0;  // of the lane's four positions
            constexpr int KB = D / 32;                             // bytes of one
#pragma unroll
            for (int i = 0; i < W; ++i) vw[x][i] &= first_bytes(min(n, 4) * KB - 4 * i);
            vs[x] &= first_bytes(n);
            nan |= nan_bytes(vs[x]) & ~first_bytes(all - (p0 + 16 * x));  // seen by some columns only
          }
          nan_v = nan != 0;
        }
        // scales of 2^65 and more: their bytes start with two ones
        uint32_t large = 0;
#pragma unroll
        for (int x = 0; x < TILES; ++x) large |= vs[x] & vs[x] << 1;
        if (__any(large & watch)) {
          lift = LIFT;
          watch = 0;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) rescale(nt, m_run[nt] + LIFT);
        }
        // weights
        uint32_t pw[NT][PP][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float mx = -INFINITY;
#pragma unroll
          for (int i = 0; i < NV; ++i) mx = fmaxf(mx, sc[nt][i]);
          mx = fmaf(mx, scale_log2, lift);
          mx = max_over_q(mx);
          if (__any(mx > m_run[nt] + SLACK)) rescale(nt, fmaxf(m_run[nt], mx));
          // a column that has seen nothing yet: weights of 0
          const float m = m_run[nt] == -INFINITY ? 0.0f : m_run[nt];
          float e[NV];
#pragma unroll
          for (int i = 0; i < NV; ++i) {
            e[i] = __builtin_amdgcn_exp2f(fmaf(sc[nt][i], scale_log2, -m));
            l_run[nt] += e[i];
          }
#pragma unroll
          for (int part = 0; part < PP; ++part)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              pw[nt][part][i] = pack_bf16(e[2 * i], e[2 * i + 1]);
              e[2 * i] -= __uint_as_float(pw[nt][part][i] << 16);
              e[2 * i + 1] -= __uint_as_float(pw[nt][part][i] & 0xffff0000u);
            }
        }
        if (!whole && __any(nan_v)) {
          // A NaN of V that some columns see and some do not: a product of ones counts,
          // for each column and dim, the NaN it sees; then V is 0 there.
          uint32_t ind[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t two = nan_bytes(vs[i / 2]) >> (16 * (i % 2));  // of two positions
            ind[i] = (two & 1) * 0x3f80u | (two >> 8 & 1) * 0x3f800000u;
          }
          const bf16x8 nf = __builtin_bit_cast(bf16x8, make_uint4(ind[0], ind[1], ind[2], ind[3]));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            uint32_t seen[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int pos = p0 + 16 * (i / 2) + 2 * (i % 2);
              seen[i] = (pos < limit[nt] ? 0x3f80u : 0u) | (pos + 1 < limit[nt] ? 0x3f800000u : 0u);
            }
            const bf16x8 sf = __builtin_bit_cast(bf16x8, make_uint4(seen[0], seen[1], seen[2], seen[3]));
            const f32x4 hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf, nf, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float add = hits[j] > 0.0f ? __builtin_nanf("") : 0.0f;
#pragma unroll
              for (int d = 0; d < DT; ++d) o[nt][d][j] += add;
            }
          }
#pragma unroll
          for (int x = 0; x < TILES; ++x) {
            const uint32_t gone = nan_bytes(vs[x]) * 255u;
            vs[x] &= ~gone;
#pragma unroll
            for (int i = 0; i < W; ++i) {
              uint32_t bytes = 0;  // of word i, those of positions that are gone
#pragma unroll
              for (int y = 0; y < 4; ++y) bytes |= (gone >> (8 * ((4 * i + y) / (D / 32))) & 255u) << (8 * y);
              vw[x][i] &= ~bytes;
            }
          }
        }
        // O += P V
        bf16x8 pf[NT][PP];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int part = 0; part < PP; ++part)
            pf[nt][part] = __builtin_bit_cast(
                bf16x8, make_uint4(pw[nt][part][0], pw[nt][part][1], pw[nt][part][2], pw[nt][part][3]));
        static_for<DT / 2>([&](auto DS) {
          constexpr int s = DS;  // dims 2s and 2s + 1 of the lane
          uint32_t pr[8];
          static_for<8>([&](auto I) {
            constexpr int i = I, byte = i % 4 * (D / 32) + s;
            pr[i] = pair_of<byte % 4>(vw[i / 4][byte / 4], scale_of(vs[i / 4], i % 4));
          });
          union { uint32_t w[4]; bf16x8 f; } lo, hi;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            lo.w[i] = __builtin_amdgcn_perm(pr[2 * i + 1], pr[2 * i], 0x05040100u);
            hi.w[i] = __builtin_amdgcn_perm(pr[2 * i + 1], pr[2 * i], 0x07060302u);
          }
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int part = 0; part < PP; ++part) {
              o[nt][2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[nt][part], lo.f, o[nt][2 * s], 0, 0, 0);
              o[nt][2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pf[nt][part], hi.f, o[nt][2 * s + 1], 0, 0, 0);
            }
        });
        KVR_WAIT_LGKM0();  // the unit's records are in registers: the ring takes the next ones
        asm volatile("" ::: "memory");
        get = get == (RING - TILES) * REC ? 0 : get + TILES * REC;
#pragma unroll 1
        for (int x = 0; x < TILES && next < last; ++x) issue();
      }

      // ---- the columns' outputs, or what there is of them ----
      // Through the ring, a row's dims over the lanes.  What stays open goes to the workspace,
      // or at the stretch's end, where the ring has no more to take, stays where it is.
      const bool done = first == 0 && upto == rq.steps, stay = u >= u1;
      float* const rows = reinterpret_cast<float*>(ring);
      float* const part = stay ? rows : slots + (first > 0 ? 0 : 1) * p.part_cols * ROW<D>;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float* const tr = rows + nt * 16 * ROW<D>;
        const float l = sum_over_q(l_run[nt]);
        if (q == 0) *reinterpret_cast<float2*>(tr + c * ROW<D> + D) = make_float2(m_run[nt], l);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float* const row = tr + (4 * q + j) * ROW<D>;
          if constexpr (DT % 4 == 0) {
#pragma unroll
            for (int d = 0; d < DT; d += 4) {
              const float x[4] = {o[nt][d][j], o[nt][d + 1][j], o[nt][d + 2][j], o[nt][d + 3][j]};
              store_part<D>(row, c * DT + d, x);
            }
          } else {
#pragma unroll
            for (int d = 0; d < DT; ++d) row[c * DT + d] = o[nt][d][j];
          }
        }
      }
      asm volatile("" ::: "memory");
      const int used = stay && !done ? 0 : cols;  // 0: the rows are the partials
#pragma unroll 1
      for (int i0 = 0; i0 < used; i0 += AT_ONCE<D>) {
        const int i = i0 + lane / LANES<D>;
        if (i >= used) continue;
        Column v;
        float2 ml;
        load_part<D>(rows + i * ROW<D>, dim_of<D>(lane), ml, v.o);
        v.m = ml.x;
        v.l = ml.y;
        if (done) put_out<T, D, COLS>(p, rq.row, tile, i, kvh, lane, v);
        else put_part<D>(part + i * ROW<D>, lane, v);
      }
      KVR_WAIT_LGKM0();  // the rows have been read: the ring may be filled again
      asm volatile("" ::: "memory");
      if (!done && lane == 0) {
        Stretch& me = s_str[wave];
        const int which = first > 0 ? 0 : 1;
        me.cols[which] = cols;
        me.row[which] = rq.row;
        me.tile[which] = tile;
        me.flags |= (stay ? 2 << which : 0) | (first > 0 && upto == rq.steps ? 1 : 0);
        if (first == 0) me.end = base + (uint32_t)(tile + 1) * rq.item;
      }
    }
  }

  // ---- the workgroup's own merges: an item begun before it, and those its waves left
  // open, each over the waves that went on with it ----
  __syncthreads();
  const Stretch str = s_str[lane % WAVES];  // lane i: wave i's
  const auto of_waves = [](bool v) { return (uint32_t)__ballot(v) & ((1u << WAVES) - 1); };
  const uint32_t begun = of_waves(str.cols[0] != 0), left = of_waves(str.cols[1] != 0), ended = of_waves(str.flags & 1);
  const uint32_t near[2] = {of_waves(str.flags & 2), of_waves(str.flags & 4)};  // sums in the rings
  OpenItem open{0, 0, 0, 0, 0};
  const int64_t pitch = (int64_t)2 * p.part_cols * ROW<D>;
  float* const slots0 = slots - wave * pitch;
  int turn = wave;  // the wave's place among those that take the next columns
#pragma unroll 1
  for (int lead = -1; lead < WAVES; ++lead) {
    const int at = max(lead, 0), which = lead < 0 ? 0 : 1;
    if (!((which ? left : begun) >> at & 1)) continue;
    int n = 1;
    bool closed = lead < 0 && (ended & 1);
    while (!closed && at + n < WAVES && begun >> (at + n) & 1) closed = ended >> (at + n++) & 1;
    const int cols = __builtin_amdgcn_readlane(str.cols[which], at);
    const int row = __builtin_amdgcn_readlane(str.row[which], at);
    const int tile = __builtin_amdgcn_readlane(str.tile[which], at);
    closed &= lead >= 0;  // all of the item is here
    float* slot = slots0 + at * pitch + which * p.part_cols * ROW<D>;
    if (lead >= 0 && !closed) open = OpenItem{cols, row, tile, at, 0};
    if (n == 1 && !(near[which] >> at & 1)) continue;
    // A wave's sums are in its ring or, where its stretch went on behind them, in the
    // workspace: a branch for each, not loads that may be from either memory.
#pragma unroll 1
    for (int c0 = turn * AT_ONCE<D>; c0 < cols; c0 += WAVES * AT_ONCE<D>) {
      const int col = c0 + lane / LANES<D>;
      if (col >= cols) continue;
      const Column v = merge_column<D, WAVES>(
          [&](int i, auto load) {
            const int j = at + i;
            if ((i == 0 ? near[which] : near[0]) >> j & 1)
              load(reinterpret_cast<const float*>(&s_ring[0][0] + j * (RING * REC)) + col * ROW<D>);
            else
              load((i == 0 ? slot : slots0 + j * pitch) + col * ROW<D>);
          },
          n, lane);
      if (closed) put_out<T, D, COLS>(p, row, tile, col, kvh, lane, v);
      else put_part<D>(slot + col * ROW<D>, lane, v);
    }
    turn = (turn - (cols + AT_ONCE<D> - 1) / AT_ONCE<D>) & (WAVES - 1);
  }
  if (kvh == 0 && t == 0) {
    const int wg = blockIdx.x / nkv;
    if (open.cols) open.groups = min((int)st.holder(s_str[open.wave].end - 1), p.workers - 1) / WAVES - wg + 1;
    p.open[wg] = open;
  }
}

// Workgroup (kv head, workgroup of the first kernel): the item that it began and left
// open, merged over the workgroups that went on with it, in their order.  Its time is its
// loads' way from other chiplets' caches: 3 us with few partials, 6.8 with 48 of 5 columns.
// The loads on their way together are the least of four numbers that holds the partials:
// those past the last are loaded for nothing, and every round waits once.  At 32 always, 40
// requests of 4 - 25 columns take 12.3 us, not 4.9, 8 of up to 256 columns 17.6, not 5.4; at 16
// and more 6.9 and 10.2; at 8 and less the 48 partials 8.3.
constexpr int PM_NT = 256;
template <typename T, int D, int NT>
__global__ __launch_bounds__(PM_NT) void packed_attn_merge_kernel(PackedAttnParams p) {
  constexpr int WG = PA_NT / 64;
  const int nkv = p.packed.nkv, wg = blockIdx.x / nkv, kvh = blockIdx.x % nkv;
  const OpenItem it = p.open[wg];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t pitch = (int64_t)2 * p.part_cols * ROW<D>;
  const float* first = p.part + ((int64_t)kvh * p.workers + wg * WG) * pitch;
  const float* lead = first + it.wave * pitch + p.part_cols * ROW<D>;
  auto merge = [&](auto chunk) {
#pragma unroll 1
    for (int c0 = wave * AT_ONCE<D>; c0 < it.cols; c0 += PM_NT / 64 * AT_ONCE<D>) {
      const int col = c0 + lane / LANES<D>;
      if (col >= it.cols) continue;
      put_out<T, D, 16 * NT>(
          p, it.row, it.tile, col, kvh, lane,
          merge_column<D, chunk>(
              [&](int i, auto load) { load((i == 0 ? lead : first + i * WG * pitch) + col * ROW<D>); }, it.groups,
              lane));
    }
  };
  if (it.groups <= 4) merge(std::integral_constant<int, 4>{});
  else if (it.groups <= 8) merge(std::integral_constant<int, 8>{});
  else if (it.groups <= 16) merge(std::integral_constant<int, 16>{});
  else merge(std::integral_constant<int, 32>{});
}

// The kernel for a call's columns per request.  A request with more than 16 NT has several
// items, whose waves read its records again, about half of them from the L2 caches; two column tiles a
// wave spare half of that and cost the third workgroup of a CU.  16 requests of 2000 - 6000
// positions with 80 columns (8 kv heads) took 44 us with one and 52 with two, 8 with 128
// 41 and 47, 8 with 256 47.9 and 47.5, 4 with 512 78 and 72, one with 2048 94 and 84.  (Four
// tiles, one workgroup a CU: 84 with 80 columns, 124 with 2048.)
struct Plan {
  int nt, cols, occupancy;
};
Plan plan_of_tiles(int dtype, int d, int nt) { return Plan{nt, 16 * nt, occupancy_of(dtype == KV_F32, d, nt)}; }
Plan plan_of(int dtype, int d, int g, int64_t max_query) {
  return plan_of_tiles(dtype, d, g * max_query <= 256 ? 1 : 2);
}

// Items of one kv head, and their units, at most: of a call's R requests with `rows` query
// rows in all, max_query of one, and max_len positions.
struct Sizes {
  int R, g;
  int64_t rows, max_query, max_len;
  int64_t items(int cols) const {
    return std::min(R + rows * g / cols, R * ((max_query * g + cols - 1) / cols));
  }
  int64_t steps() const { return (max_len + UNIT - 1) / UNIT; }
};

// Stretches per kv head, whole workgroups.
//   A workgroup to an item, its four waves equal parts of it, where the chip holds all of
// them at once and a part is at most WHOLE units: nothing is left to merge between
// workgroups, and the second kernel is not launched.  A call on 90 requests of up to 250
// positions took 11.1 us so and 15.0 the other way, 16 of up to 500 9.7 and 11.6; parts of
// eight, 16 of up to 1000, 14.9 and 13.2.
//   Else a unit each where the chip holds as many waves at once, else those waves.  Then an
// item's start counts as START units more: a wave whose stretch goes on with another item
// ends the one and waits for the other's table, queries and first records, some 4 us, and
// the waves should end together.  None, two and four: 31.9, 30.1 and 29.4 us on 16 requests
// of one row, 32.4, 29.6 and 29.4 on 40 of one to five, 21.3, 18.8 and 18.3 on 64 of 2 kv
// heads, 71.7, 67.1 and 68.4 on 4 of 128 rows.
constexpr int START = 4;
constexpr int64_t WHOLE = 4;
struct Stretching {
  int workers, start, whole;
};
int64_t most_waves(const Plan& pl, int nkv) { return (256 * 4 * pl.occupancy + nkv - 1) / nkv; }
Stretching stretches_of(const Plan& pl, int nkv, const Sizes& z) {
  const int64_t items = z.items(pl.cols), units = items * z.steps(), waves = most_waves(pl, nkv);
  const int64_t part = (z.steps() + 3) / 4;
  if (part <= WHOLE && 4 * items <= waves) return {(int)(4 * items), 0, (int)part};
  if (units <= waves) return {(int)round_up(units, PA_NT / 64), 0, 0};
  return {(int)round_up(waves, PA_NT / 64), START, 0};
}

template <typename T, int D, int NT>
void launch_tiles(const PackedAttnParams& p, hipStream_t s) {
  constexpr int OCC = occupancy_of(std::is_same<T, float>::value, D, NT);
  const dim3 grid((unsigned)((int64_t)p.workers / (PA_NT / 64) * p.packed.nkv));
  hipLaunchKernelGGL((packed_attn_kernel<T, D, NT, OCC>), grid, dim3(PA_NT), 0, s, p);
  if (!p.whole) hipLaunchKernelGGL((packed_attn_merge_kernel<T, D, NT>), grid, dim3(PM_NT), 0, s, p);
}
template <typename T, int D>
void launch(const Plan& pl, const PackedAttnParams& p, hipStream_t s) {
  if (pl.nt == 1) launch_tiles<T, D, 1>(p, s);
  else launch_tiles<T, D, 2>(p, s);
}

// The workspace: what workgroups left open, then the waves' sums.  It is as large as any
// call of no larger sizes needs, whichever kernel that one takes.
struct AttnLayout {
  uint64_t part, total;
};
AttnLayout attn_layout(const kv_model_desc& d, const Sizes& z) {
  int64_t workers = 0, columns = 0;
  const Plan own = plan_of(d.dtype, d.head_dim, z.g, z.max_query);
  for (int nt = 1; nt <= own.nt; ++nt) {
    const Plan pl = plan_of_tiles(d.dtype, d.head_dim, nt);
    const int64_t units = z.items(pl.cols) * std::max<int64_t>(4, z.steps());
    const int64_t w = round_up(std::min(most_waves(pl, d.num_kv_heads), units), PA_NT / 64);
    workers = std::max(workers, w);
    columns = std::max(columns, w * std::min<int64_t>(pl.cols, z.g * z.max_query));
  }
  AttnLayout L;
  L.part = (uint64_t)round_up(workers / (PA_NT / 64) * (int64_t)sizeof(OpenItem), 256);
  L.total = L.part + (uint64_t)(4 * d.num_kv_heads * 2 * columns * row_of(d.head_dim));
  return L;
}

}  // namespace
}  // namespace kvr

using namespace kvr;

namespace {

void run(const kv_packed* packed, int32_t layer, const void* q, int64_t q_stride, const int32_t* q_offsets,
         int64_t rows, const int32_t* lens, const int32_t* tables, int R, int max_blocks, int32_t max_query,
         int64_t max_len, void* out, int64_t out_stride, void* workspace, hipStream_t s) {
  const kv_model_desc& d = packed->desc;
  const int64_t e = elem_bytes(d.dtype);
  PackedAttnParams p{};
  p.packed = packed_layer(packed, layer);
  p.num_blocks = (uint32_t)std::min<int64_t>(packed->num_blocks, (int64_t)INT32_MAX + 1);
  p.q = static_cast<const char*>(q);
  p.out = static_cast<char*>(out);
  p.q_stride = q_stride * e;
  p.out_stride = out_stride * e;
  p.q_offsets = q_offsets;
  p.rows = rows;
  p.lens = lens;
  p.tables = tables;
  p.R = R;
  p.max_blocks = max_blocks;
  p.g = d.num_q_heads / d.num_kv_heads;
  p.g_inv = p.g == 1 ? 0 : (uint32_t)(((1ull << 32) + p.g - 1) / p.g);
  const Sizes z{R, p.g, rows, max_query, max_len};
  const Plan plan = plan_of(d.dtype, d.head_dim, p.g, max_query);
  const Stretching st = stretches_of(plan, d.num_kv_heads, z);
  p.max_query = max_query;
  p.most_len = (int)std::min<int64_t>({max_len, (int64_t)max_blocks * packed->block_size, INT32_MAX});
  p.start = st.start;
  p.whole = st.whole;
  p.workers = st.workers;
  p.part_cols = (int)std::min<int64_t>(plan.cols, (int64_t)p.g * max_query);
  p.open = static_cast<OpenItem*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + attn_layout(d, z).part);
  if (d.dtype == KV_BF16) launch<bf16_t, 128>(plan, p, s);
  else if (d.head_dim == 128) launch<float, 128>(plan, p, s);
  else if (d.head_dim == 64) launch<float, 64>(plan, p, s);
  else launch<float, 32>(plan, p, s);
}

}  // namespace

bool kvr::packed_attention_takes(const kv_model_desc& d, int64_t R, int64_t rows, int64_t max_query, int64_t max_len) {
  if (R > MOST_ROWS || rows > MOST_ROWS || max_len > INT32_MAX) return false;
  const int g = d.num_q_heads / d.num_kv_heads;
  const Plan plan = plan_of(d.dtype, d.head_dim, g, max_query);
  const Sizes z{(int)R, g, rows, max_query, max_len};
  return (R + rows * g / plan.cols) * (z.steps() + START) <= INT32_MAX;
}

void kvr::packed_attention_step(const kv_packed* a, int32_t layer, const void* q, const int32_t* lens,
                                const int32_t* tables, int R, int max_blocks, int64_t max_len, void* out,
                                void* workspace, hipStream_t s) {
  const int64_t row = (int64_t)a->desc.num_q_heads * a->desc.head_dim;
  run(a, layer, q, row, nullptr, R, lens, tables, R, max_blocks, 1, max_len, out, row, workspace, s);
}

extern "C" {

uint64_t kv_packed_attention_workspace_bytes(const kv_model_desc* desc, int32_t num_requests, int64_t rows,
                                             int32_t max_query, int64_t max_len) {
  if (kv_packed_bytes(desc, PK_TILE, 1) == 0 || desc->num_q_heads / desc->num_kv_heads > 16) return 0;
  if (num_requests <= 0 || num_requests > MOST_ROWS || rows <= 0 || rows > MOST_ROWS || max_query <= 0 ||
      max_len <= 0 || max_len > INT32_MAX)
    return 0;
  return attn_layout(*desc, {num_requests, desc->num_q_heads / desc->num_kv_heads, rows, max_query, max_len}).total;
}

kv_status kv_packed_attention(kv_packed_t packed, int32_t layer, const void* q, int64_t q_stride,
                              const int32_t* q_offsets, int64_t rows, const int32_t* lens, const int32_t* tables,
                              int32_t R, int32_t max_blocks, int32_t max_query, int64_t max_len, void* out,
                              int64_t out_stride, void* workspace, uint64_t ws_bytes, void* stream) {
  if (!live_packed(packed)) return kvr_err::set(KV_ESTATE, "unknown or released packed arena handle");
  const kv_model_desc& d = packed->desc;
  const int64_t e = elem_bytes(d.dtype), row = (int64_t)d.num_q_heads * d.head_dim;
  if (d.num_q_heads / d.num_kv_heads > 16)
    return kvr_err::set(KV_EINVAL, "packed attention supports at most 16 q heads per kv head");
  if (layer < 0 || layer >= d.num_layers)
    return kvr_err::set(KV_EINVAL, "layer %d outside [0, %d)", layer, d.num_layers);
  if (R < 0 || R > MOST_ROWS || rows < 0 || rows > MOST_ROWS || max_blocks < 0)
    return kvr_err::set(KV_EINVAL, "num_requests and rows are 0 .. 2^24, max_blocks_per_req is not negative");
  if (!q_offsets && rows != R) return kvr_err::set(KV_EINVAL, "without q_offsets rows must equal num_requests");
  if (R == 0 || rows == 0) return kvr_err::clear();
  if (max_query < 1 || max_len < 1) return kvr_err::set(KV_EINVAL, "max_query and max_len must be positive");
  if (!q || !out || !lens || (max_blocks > 0 && !tables))
    return kvr_err::set(KV_EINVAL, "null q, out, lens or block_tables");
  if (q_stride < row || out_stride < row)
    return kvr_err::set(KV_EINVAL, "a stride is below the row's %lld elements", (long long)row);
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)(q_stride * e) | (uintptr_t)(out_stride * e) | (uintptr_t)q_offsets |
       (uintptr_t)lens | (uintptr_t)tables) % 4 != 0)
    return kvr_err::set(KV_EINVAL, "the arrays and the strides need boundaries of 4 bytes");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
  if (!packed_attention_takes(d, R, rows, max_query, max_len))
    return kvr_err::set(KV_EINVAL, "max_len or the work of one call above 2^31: split the query rows");
  const uint64_t need = kv_packed_attention_workspace_bytes(&d, R, rows, max_query, max_len);
  if (need > ws_bytes)
    return kvr_err::set(KV_ENOMEM, "workspace of %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                        (unsigned long long)need);
  DeviceGuard dg(packed->device);
  const kv_status st = device_ready(dg, packed->device);
  if (st != KV_OK) return st;
  run(packed, layer, q, q_stride, q_offsets, rows, lens, tables, R, max_blocks, max_query, max_len, out, out_stride,
      workspace, reinterpret_cast<hipStream_t>(stream));
  return launched();
}

}  // extern "C"

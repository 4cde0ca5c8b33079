// Attention over a packed arena (kvr_packed.h).
//
// The query rows of a request that share a kv head are columns: column i g + h is
// query i of q head h of the group.  An item is one request's 16 NT columns of one kv
// head; its work comes in units of 32 positions.  Every wave takes an equal stretch of
// the units of all items, request after request, whatever the lengths (they are known
// on the device alone), so that all waves end together; where a stretch ends inside an
// item, the wave leaves the item's sums so far, and a second kernel merges them.
//
// A unit in a wave's registers, lane (q, c) = (lane / 16, lane % 16):
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16, 16 positions a tile: position c's dims
//   q d/4 .. are the lane's K operand, d/8 bytes and one scale; the conversions to bf16
//   are exact.  It gets the scores of positions 4q .. 4q+3 for column c.
//   Online softmax per column, exp2 domain, rescaled only where the maximum rose by
//   more than 2^SLACK.
//   O = P V: the lane's weights of two tiles are the A operand as they are, positions
//   4q .. 4q+3 of both being its eight k's; V's layout gives the lane the dims
//   c d/16 .. of the same positions, which it pairs into the B operands of d/16
//   products.  Nothing passes through LDS.
// Weights enter the product as a bf16 number and the bf16 rest (2^-17 of a weight lost),
// in fp32 models as three (as do the queries): rounding them once would cost more than
// the output's own rounding where few positions weigh, and the products are not what
// bounds the kernel.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "host.h"
#include "kvr_packed.h"
#include "launch.h"
#include "packed.h"

namespace kvr {
namespace {

constexpr int PA_UNIT = 32;        // positions of a unit
constexpr int PA_NT = 256;         // four waves
constexpr float SLACK = 8.0f;      // rescale slack, log2 units
constexpr int PA_WAVES = 2048;     // waves of a call

template <typename T> struct Split;  // bf16 numbers that stand for a query, for a weight
template <> struct Split<bf16_t> { static constexpr int Q = 1, P = 2; };
template <> struct Split<float> { static constexpr int Q = 3, P = 3; };

// What a wave leaves of an item it did not finish: the item, its units' end, and the
// units of all items.
struct OpenItem {
  int64_t end, total;
  int request, tile;  // request -1: none
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

struct PackedAttnParams {
  PackedLayer packed;
  int64_t num_blocks;
  const char* q;                 // rows of queries, model dtype
  char* out;
  int64_t q_stride, out_stride;  // bytes
  const int32_t* q_offsets;      // null: row r is request r's
  int64_t rows;
  const int32_t* lens;
  const int32_t* tables;
  int R, max_blocks;
  int nq;
  int max_query;                 // rows of a request past it are left out: the sums have no room
  int workers;                   // stretches per kv head
  int part_cols;                 // columns of a slot of sums
  OpenItem* open;                // [workers]
  float* part;                   // [nkv][workers][2][part_cols][D + 2]
};

// f(0), f(1), .. with the index a constant
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    static_for<N, I + 1>(f);
  }
}

struct Request {
  int row, m, len, want;  // first query row, rows, positions there are, position after the last query
  int tiles, steps;       // column tiles, units of each
};
template <int NT>
__device__ __forceinline__ Request get_request(const PackedAttnParams& p, int r) {
  Request q;
  q.row = r;
  q.m = 1;
  if (p.q_offsets) {
    const int a = p.q_offsets[r], b = p.q_offsets[r + 1];
    q.row = min(max(a, 0), (int)p.rows);
    q.m = min(max(min(b, (int)p.rows) - q.row, 0), p.max_query);
  }
  q.want = p.lens[r];
  q.len = (int)max((int64_t)0, min((int64_t)q.want, (int64_t)p.max_blocks * p.packed.block_size));
  const int g = p.nq / p.packed.nkv;
  q.tiles = (int)(((int64_t)q.m * g + 16 * NT - 1) / (16 * NT));
  q.steps = max(1, (q.len + PA_UNIT - 1) / PA_UNIT);
  return q;
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

// A unit's bytes of a lane.
template <int D>
struct Unit {
  static constexpr int W = D / 32;  // words of K, and of V, a tile
  uint32_t k[2][W], v[2][W], ks[2], vs[2];
  bool there[2];  // the tile's block is in the arena
};

template <typename T, int D, int NT>
__global__ __launch_bounds__(PA_NT) void packed_attn_kernel(PackedAttnParams p) {
  constexpr int W = D / 32, DT = D / 16;  // words a tile; dims a lane, P.V products
  constexpr int QP = Split<T>::Q, PP = Split<T>::P;
  __shared__ int64_t s_pre[PA_NT + 1];
  __shared__ int64_t s_wave[PA_NT / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, c = lane & 15, q = lane >> 4;
  const int nkv = p.packed.nkv, g = p.nq / nkv;

  // ---- the units before each thread's requests ----
  const int per = (p.R + PA_NT - 1) / PA_NT;
  int64_t mine = 0;
  for (int i = 0; i < per; ++i) {
    const int r = t * per + i;
    if (r < p.R) {
      const Request x = get_request<NT>(p, r);
      mine += (int64_t)x.tiles * x.steps;
    }
  }
  int64_t incl = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t u = __shfl_up(incl, o, 64);
    if (lane >= o) incl += u;
  }
  if (lane == 63) s_wave[wave] = incl;
  __syncthreads();
  int64_t before = 0, total = 0;
#pragma unroll
  for (int i = 0; i < PA_NT / 64; ++i) {
    if (i < wave) before += s_wave[i];
    total += s_wave[i];
  }
  s_pre[t + 1] = before + incl;
  if (t == 0) s_pre[0] = 0;
  __syncthreads();

  const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * (PA_NT / 64) + wave);
  const int kvh = id % nkv, w = id / nkv;
  if (w >= p.workers) return;
  OpenItem* open = p.open + w;
  if (kvh == 0 && lane == 0) *open = OpenItem{0, total, -1, 0};
  const int64_t workers = min((int64_t)p.workers, total);  // a unit each at least
  if (w >= workers) return;
  const int64_t u0 = total * w / workers, u1 = total * (w + 1) / workers;

  int a = 0, b = PA_NT - 1;  // the last thread's requests that begin at or before u0
  while (a < b) {
    const int m = (a + b + 1) / 2;
    if (s_pre[m] <= u0) a = m;
    else b = m - 1;
  }
  int r = a * per;
  int64_t base = s_pre[a];
  Request rq = get_request<NT>(p, r);
  while (base + (int64_t)rq.tiles * rq.steps <= u0) {
    base += (int64_t)rq.tiles * rq.steps;
    rq = get_request<NT>(p, ++r);
  }

  const int B = p.packed.block_size, tpb = B / PK_TILE;
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)D);
  const char* head = p.packed.base + (int64_t)kvh * tpb * (17 * D);
  const int64_t block_bytes = (int64_t)nkv * tpb * (17 * D);
  const int k_off = c * (D / 2) + q * (D / 8), v_off = 8 * D + q * (2 * D) + c * (D / 8);
  const int ks_off = 16 * D + c * (D / 32) + q * D / 128, vs_off = 16 * D + D / 2 + q * (D / 8) + c * D / 512 * 4;

  for (int64_t u = u0; u < u1;) {
    // ---- the stretch's part of one item ----
    const int tile = (int)((u - base) / rq.steps), first = (int)(u - base - (int64_t)tile * rq.steps);
    const int upto = (int)min((int64_t)rq.steps, first + (u1 - u));
    const int cols = min(16 * NT, rq.m * g - tile * 16 * NT);  // of this tile
    // positions that every column sees, and that any does
    const int i_lo = tile * 16 * NT / g, i_hi = (tile * 16 * NT + cols - 1) / g;
    const int all = min(rq.len, rq.want - rq.m + i_lo + 1), some = min(rq.len, rq.want - rq.m + i_hi + 1);
    const int stop = min(upto, (max(some, 0) + PA_UNIT - 1) / PA_UNIT);

    bf16x8 qf[NT][QP][W];
    int limit[NT];  // positions column c of tile nt sees
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int col = nt * 16 + c, gc = tile * 16 * NT + col, i = gc / g;
      limit[nt] = col < cols ? min(rq.len, rq.want - rq.m + i + 1) : some;
      const T* src = reinterpret_cast<const T*>(p.q + (int64_t)(rq.row + min(i, rq.m - 1)) * p.q_stride) +
                     (int64_t)(kvh * g + gc % g) * D + q * (D / 4);
#pragma unroll
      for (int s = 0; s < W; ++s) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = col < cols ? Elem<T>::load(src, 8 * s + e) : 0.0f;
#pragma unroll
        for (int part = 0; part < QP; ++part) {
          union { uint32_t w[4]; bf16x8 f; } f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f.w[e] = pack_bf16(x[2 * e], x[2 * e + 1]);
            x[2 * e] -= __uint_as_float(f.w[e] << 16);
            x[2 * e + 1] -= __uint_as_float(f.w[e] & 0xffff0000u);
          }
          qf[nt][part][s] = f.f;
        }
      }
    }
    float m_run[NT], l_run[NT];
    f32x4 o[NT][DT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      m_run[nt] = -INFINITY;
      l_run[nt] = 0.0f;
#pragma unroll
      for (int j = 0; j < DT; ++j) o[nt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }

    // 64 table entries at a time, one a lane
    const int32_t* table = p.tables + (int64_t)r * p.max_blocks;
    auto entries = [&](int b0) { return b0 + lane < p.max_blocks ? table[b0 + lane] : -1; };
    int bi = first * 2 / tpb, ti = first * 2 % tpb;  // the next tile's block and place in it
    int window = bi, tab = entries(bi);
    auto fetch = [&](Unit<D>& n) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        if (bi - window >= 64) {
          window = bi;
          tab = entries(bi);
        }
        const int e = __builtin_amdgcn_readlane(tab, bi - window);
        n.there[x] = e >= 0 && e < p.num_blocks;
        const char* rec = head + (n.there[x] ? e : 0) * block_bytes + ti * (17 * D);
        load_words<D / 8>(rec + k_off, n.k[x]);
        load_words<D / 8>(rec + v_off, n.v[x]);
        n.ks[x] = (uint8_t)rec[ks_off];
        n.vs[x] = *reinterpret_cast<const uint32_t*>(rec + vs_off);
        if (++ti == tpb) {
          ti = 0;
          ++bi;
        }
      }
    };

    auto attend = [&](Unit<D>& n, int kt) {
      const int j0 = kt * PA_UNIT + 4 * q;  // the lane's first position of tile 0
      const bool whole = kt * PA_UNIT + PA_UNIT <= all && n.there[0] && n.there[1];
      // scores
      f32x4 st[NT][2];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) st[nt][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const float ks = scale_of(n.ks[x]);
#pragma unroll
        for (int s = 0; s < W; ++s) {
          union { uint32_t w[4]; bf16x8 f; } kf;
          kf.w[0] = pair_of<0>(n.k[x][s], ks);
          kf.w[1] = pair_of<1>(n.k[x][s], ks);
          kf.w[2] = pair_of<2>(n.k[x][s], ks);
          kf.w[3] = pair_of<3>(n.k[x][s], ks);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int part = 0; part < QP; ++part)
              st[nt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf.f, qf[nt][part][s], st[nt][x], 0, 0, 0);
        }
      }
      bool nan_v = false;
      if (!whole) {
        // positions past a column's limit and in blocks that are not there leave its
        // softmax; V there may hold any bits, and 0 times them is not 0
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int pos = j0 + 16 * x + j;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              if (pos >= limit[nt] || !n.there[x]) st[nt][x][j] = -INFINITY;
            if (pos >= some || !n.there[x]) {
              constexpr int KB = D / 32;  // bytes of a position
#pragma unroll
              for (int y = 0; y < KB; ++y) n.v[x][(j * KB + y) / 4] &= ~(0xffu << ((j * KB + y) % 4 * 8));
              n.vs[x] &= ~(0xffu << (8 * j));
            }
            nan_v |= (n.vs[x] >> (8 * j) & 0xff) == PK_NAN && pos >= all;
          }
      }
      // weights
      uint32_t pf[NT][PP][4];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float sc[8], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sc[i] = st[nt][i / 4][i % 4] * scale_log2;
          mx = fmaxf(mx, sc[i]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        if (__any(mx > m_run[nt] + SLACK)) {
          const float m_new = fmaxf(m_run[nt], mx);
          const float alpha = m_new == m_run[nt] ? 1.0f : __builtin_amdgcn_exp2f(m_run[nt] - m_new);
          l_run[nt] *= alpha;
          m_run[nt] = m_new;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float f = __shfl(alpha, 4 * q + j, 64);  // column 4q + j's
#pragma unroll
            for (int d = 0; d < DT; ++d) o[nt][d][j] *= f;
          }
        }
        // a column that has seen nothing yet: weights of 0
        const float m = m_run[nt] == -INFINITY ? 0.0f : m_run[nt];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sc[i] = __builtin_amdgcn_exp2f(sc[i] - m);
          l_run[nt] += sc[i];
        }
#pragma unroll
        for (int part = 0; part < PP; ++part)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pf[nt][part][i] = pack_bf16(sc[2 * i], sc[2 * i + 1]);
            sc[2 * i] -= __uint_as_float(pf[nt][part][i] << 16);
            sc[2 * i + 1] -= __uint_as_float(pf[nt][part][i] & 0xffff0000u);
          }
      }
      if (!whole && __any(nan_v)) {
        // A NaN of V that some columns see and some do not: a product of ones counts,
        // for each column and dim, the NaN it sees; then V is 0 there.
        uint32_t seen[NT][4], ind[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t word = 0;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int k = 2 * i + y, x = k / 4, j = k % 4;
            if ((n.vs[x] >> (8 * j) & 0xff) == PK_NAN) word |= 0x3f80u << (16 * y);
          }
          ind[i] = word;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            seen[nt][i] = 0;
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const int k = 2 * i + y;
              if (j0 + 16 * (k / 4) + k % 4 < limit[nt]) seen[nt][i] |= 0x3f80u << (16 * y);
            }
          }
        }
        const bf16x8 nf = __builtin_bit_cast(bf16x8, make_uint4(ind[0], ind[1], ind[2], ind[3]));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const bf16x8 sf = __builtin_bit_cast(bf16x8, make_uint4(seen[nt][0], seen[nt][1], seen[nt][2], seen[nt][3]));
          const f32x4 hits = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf, nf, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (hits[j] > 0.0f)
#pragma unroll
              for (int d = 0; d < DT; ++d) o[nt][d][j] = __builtin_nanf("");
        }
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if ((n.vs[x] >> (8 * j) & 0xff) == PK_NAN) {
              constexpr int KB = D / 32;
#pragma unroll
              for (int y = 0; y < KB; ++y) n.v[x][(j * KB + y) / 4] &= ~(0xffu << ((j * KB + y) % 4 * 8));
              n.vs[x] &= ~(0xffu << (8 * j));
            }
      }
      // O += P V
      float vs[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) vs[i] = scale_of(n.vs[i / 4] >> (8 * (i % 4)) & 0xff);
      static_for<DT / 2>([&](auto S) {
        constexpr int s = S;  // dims 2s and 2s + 1 of the lane
        uint32_t pr[8];
        static_for<8>([&](auto I) {
          constexpr int i = I, byte = i % 4 * (D / 32) + s;
          pr[i] = pair_of<byte % 4>(n.v[i / 4][byte / 4], vs[i]);
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
            const bf16x8 f = __builtin_bit_cast(bf16x8, make_uint4(pf[nt][part][0], pf[nt][part][1], pf[nt][part][2],
                                                                   pf[nt][part][3]));
            o[nt][2 * s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, lo.f, o[nt][2 * s], 0, 0, 0);
            o[nt][2 * s + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(f, hi.f, o[nt][2 * s + 1], 0, 0, 0);
          }
      });
    };

    Unit<D> now, next;
    if (first < stop) fetch(now);
    for (int kt = first; kt < stop; ++kt) {
      if (kt + 1 < stop) fetch(next);
      attend(now, kt);
      now = next;
    }

    // ---- the columns' outputs, or what there is of them ----
    const bool done = first == 0 && upto == rq.steps;
    float* part = p.part + (((int64_t)kvh * p.workers + w) * 2 + (first > 0 ? 0 : 1)) * p.part_cols * (D + 2);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float l = l_run[nt] + __shfl_xor(l_run[nt], 16, 64);
      l += __shfl_xor(l, 32, 64);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int col = nt * 16 + 4 * q + j;
        const float lj = __shfl(l, 4 * q + j, 64), mj = __shfl(m_run[nt], 4 * q + j, 64);
        if (col >= cols) continue;
        float x[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) x[d] = o[nt][d][j];
        if (done) {
          const int gc = tile * 16 * NT + col;
          T* dst = reinterpret_cast<T*>(p.out + (int64_t)(rq.row + gc / g) * p.out_stride) +
                   (int64_t)(kvh * g + gc % g) * D + c * DT;
          const float inv = lj == 0.0f ? 0.0f : 1.0f / lj;
#pragma unroll
          for (int d = 0; d < DT; ++d) Elem<T>::store(dst, d, lj == 0.0f ? 0.0f : x[d] * inv);
        } else {
          float* dst = part + col * (D + 2);
#pragma unroll
          for (int d = 0; d < DT; ++d) dst[c * DT + d] = x[d];
          if (c == 0) {
            dst[D] = mj;
            dst[D + 1] = lj;
          }
        }
      }
    }
    if (first == 0 && !done && kvh == 0 && lane == 0)
      *open = OpenItem{base + (int64_t)(tile + 1) * rq.steps, total, r, tile};
    u += upto - first;
    if (u < u1)
      while (base + (int64_t)rq.tiles * rq.steps <= u) {
        base += (int64_t)rq.tiles * rq.steps;
        rq = get_request<NT>(p, ++r);
      }
  }
}

// Workgroup (kv head, worker): the item that the worker began and left open, merged
// over the workers that went on with it, in their order.  A wave takes every fourth
// column, a lane D / 64 dims of it.
template <typename T, int D, int NT>
__global__ __launch_bounds__(PA_NT) void packed_attn_merge_kernel(PackedAttnParams p) {
  const int nkv = p.packed.nkv, g = p.nq / nkv, w = blockIdx.x / nkv, kvh = blockIdx.x % nkv;
  const OpenItem it = p.open[w];
  if (it.request < 0) return;
  const Request rq = get_request<NT>(p, it.request);
  const int cols = min(16 * NT, rq.m * g - it.tile * 16 * NT);
  const int64_t workers = min((int64_t)p.workers, it.total);
  int n = 1;  // with the workers after w whose stretches begin inside the item
  while (w + n < workers && it.total * (w + n) / workers < it.end) ++n;
  const int lane = threadIdx.x & 63;
  const int64_t pitch = (int64_t)2 * p.part_cols * (D + 2);
  const float* first = p.part + ((int64_t)kvh * p.workers + w) * pitch;
  for (int col = threadIdx.x >> 6; col < cols; col += PA_NT / 64) {
    // worker w's second slot, the others' first
    auto src = [&](int i) { return first + i * pitch + (i == 0 ? p.part_cols * (D + 2) : 0) + col * (D + 2); };
    float m = -INFINITY;
    for (int i = 0; i < n; ++i) m = fmaxf(m, src(i)[D]);
    const float base = m == -INFINITY ? 0.0f : m;
    float l = 0.0f, o[(D + 63) / 64] = {};
    for (int i = 0; i < n; ++i) {
      const float* x = src(i);
      const float f = __builtin_amdgcn_exp2f(x[D] - base);
      l = fmaf(x[D + 1], f, l);
#pragma unroll
      for (int d = 0; d < (D + 63) / 64; ++d)
        if (d * 64 + lane < D) o[d] = fmaf(x[d * 64 + lane], f, o[d]);
    }
    const int gc = it.tile * 16 * NT + col;
    T* dst = reinterpret_cast<T*>(p.out + (int64_t)(rq.row + gc / g) * p.out_stride) +
             (int64_t)(kvh * g + gc % g) * D;
#pragma unroll
    for (int d = 0; d < (D + 63) / 64; ++d)
      if (d * 64 + lane < D) Elem<T>::store(dst, d * 64 + lane, l == 0.0f ? 0.0f : o[d] / l);
  }
}

// Column tiles of a wave: as many as the rows of one request fill.
int column_tiles(int dtype, int g, int32_t max_query) {
  const int64_t cols = (int64_t)g * max_query;
  return cols <= 16 ? 1 : cols <= 32 || dtype == KV_F32 ? 2 : 4;
}

// Stretches per kv head: PA_WAVES waves in all, but no more than units there can be.
int workers_of(int nkv, int R, int64_t rows, int g, int nt, int64_t max_len) {
  const int64_t items = R + rows * g / (16 * nt);
  const int64_t units = items * ((max_len + PA_UNIT - 1) / PA_UNIT);
  return (int)std::max<int64_t>(1, std::min<int64_t>((PA_WAVES + nkv - 1) / nkv, units));
}

template <typename T, int D, int NT>
void launch_nt(const PackedAttnParams& p, hipStream_t s) {
  const int64_t waves = (int64_t)p.workers * p.packed.nkv;
  hipLaunchKernelGGL((packed_attn_kernel<T, D, NT>), dim3((unsigned)((waves + 3) / 4)), dim3(PA_NT), 0, s, p);
  hipLaunchKernelGGL((packed_attn_merge_kernel<T, D, NT>), dim3((unsigned)waves), dim3(PA_NT), 0, s, p);
}
template <typename T, int D>
void launch(int nt, const PackedAttnParams& p, hipStream_t s) {
  if (nt == 1) return launch_nt<T, D, 1>(p, s);
  if (nt == 2) return launch_nt<T, D, 2>(p, s);
  if constexpr (std::is_same<T, bf16_t>::value) launch_nt<T, D, 4>(p, s);
}

// The workspace: what workers left open, then their sums.
struct AttnLayout {
  int nt, workers, cols;
  uint64_t part, total;
};
AttnLayout attn_layout(const kv_model_desc& d, int32_t R, int64_t rows, int32_t max_query, int64_t max_len) {
  AttnLayout L;
  const int g = d.num_q_heads / d.num_kv_heads;
  L.nt = column_tiles(d.dtype, g, max_query);
  L.workers = workers_of(d.num_kv_heads, R, rows, g, L.nt, max_len);
  L.cols = (int)std::min<int64_t>(16 * L.nt, (int64_t)g * max_query);
  L.part = (uint64_t)round_up((int64_t)L.workers * (int64_t)sizeof(OpenItem), 256);
  L.total = L.part + (uint64_t)4 * d.num_kv_heads * L.workers * 2 * L.cols * (d.head_dim + 2);
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
  p.num_blocks = packed->num_blocks;
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
  p.nq = d.num_q_heads;
  const AttnLayout L = attn_layout(d, R, rows, max_query, max_len);
  p.max_query = max_query;
  p.workers = L.workers;
  p.part_cols = L.cols;
  p.open = static_cast<OpenItem*>(workspace);
  p.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.part);
  if (d.dtype == KV_BF16) launch<bf16_t, 128>(L.nt, p, s);
  else if (d.head_dim == 128) launch<float, 128>(L.nt, p, s);
  else if (d.head_dim == 64) launch<float, 64>(L.nt, p, s);
  else launch<float, 32>(L.nt, p, s);
}

}  // namespace

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
  if (num_requests <= 0 || rows <= 0 || max_query <= 0 || max_len <= 0) return 0;
  return attn_layout(*desc, num_requests, rows, max_query, max_len).total;
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
  if (R < 0 || rows < 0 || rows > INT32_MAX || max_blocks < 0)
    return kvr_err::set(KV_EINVAL, "num_requests, rows and max_blocks_per_req are 0 .. 2^31 - 1");
  if (!q_offsets && rows != R) return kvr_err::set(KV_EINVAL, "without q_offsets rows must equal num_requests");
  if (R == 0 || rows == 0) return kvr_err::clear();
  if (max_query < 1 || max_len < 1) return kvr_err::set(KV_EINVAL, "max_query and max_len must be positive");
  if (!q || !out || !lens || (max_blocks > 0 && !tables)) return kvr_err::set(KV_EINVAL, "null q, out, lens or block_tables");
  if (q_stride < row || out_stride < row)
    return kvr_err::set(KV_EINVAL, "a stride is below the row's %lld elements", (long long)row);
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)(q_stride * e) | (uintptr_t)(out_stride * e) | (uintptr_t)q_offsets |
       (uintptr_t)lens | (uintptr_t)tables) % 4 != 0)
    return kvr_err::set(KV_EINVAL, "the arrays and the strides need boundaries of 4 bytes");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
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

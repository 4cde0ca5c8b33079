// Rows of a layer's q, k and v products into the retained arena (kvr_append.h).
//
// A lane holds eight pairs (x_i, x_{i + d/2}) of a head, two loads of 16 bytes in bf16;
// d / 16 neighbouring lanes make a head and agree on its norm by exchanges.  The cosines
// and sines of a row are the same for all its heads: a workgroup computes those of its
// rows once, a pair a thread, into LDS, while its first loads are on their way.
//
// Angles.  In turns, t = p 2^(-(2i/d) log2 theta - log2 2 pi), fp64.  t less its nearest
// whole number is exact, and so is what is left after quarter turns; the sine and cosine
// of at most an eighth of a turn are their series to y^13 and y^14 (the next terms are
// below 2^-45), rounded to fp32 at the end.  t's own rounding is 2^-52 of it: 2^-34 of a turn
// at positions of a million.
//
// Every value is read once and written once, so long calls go at a copy's rate: 8191 rows of 40 q
// and 8 kv heads, 235 MB, in 48.9 us, 4.8 TB/s.  Short ones wait for their loads, one after
// the other: 64 rows of 32 + 16 heads 5.1 us, 23 rows of 12 + 4 heads 3.8.
#include <algorithm>

#include "common.h"
#include "host.h"
#include "kvr_append.h"

namespace kvr {
namespace {

constexpr int AP_NT = 256;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a4 __attribute__((aligned(4)));  // 16 bytes on any 4-byte boundary

// Eight consecutive values as they lie in memory.
template <typename T> struct Raw8;
template <> struct Raw8<bf16_t> {
  u32x4 u;
  __device__ __forceinline__ void load(const char* p) { u = *reinterpret_cast<const u32x4_a4*>(p); }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void store(char* p, const float* v) {
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      u[i] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[2 * i], (__bf16)v[2 * i + 1]});
    *reinterpret_cast<u32x4_a4*>(p) = u;
  }
};
template <> struct Raw8<float> {
  f32x4 a, b;
  __device__ __forceinline__ void load(const char* p) {
    a = reinterpret_cast<const f32x4_a4*>(p)[0];
    b = reinterpret_cast<const f32x4_a4*>(p)[1];
  }
  __device__ __forceinline__ void values(float* v) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = a[i];
      v[4 + i] = b[i];
    }
  }
  static __device__ __forceinline__ void store(char* p, const float* v) {
    reinterpret_cast<f32x4_a4*>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4_a4*>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
};

struct AppendParams {
  const char *q, *k, *v;  // q null: no q heads
  char *q_out, *plane_k, *plane_v;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // bytes
  const int32_t* positions;
  const int64_t* slots;
  int64_t rows, arena_slots;
  int nq, nkv;  // nq 0 without q
  const char *bq, *bk, *bv, *q_norm, *k_norm;  // null: none
  float eps;
  double log2_theta;
};

// Cosine and sine of a number of turns.
__device__ __forceinline__ float2 cos_sin_turns(double t) {
  const double r = t - rint(t), k = rint(4.0 * r);
  const double y = (r - 0.25 * k) * 6.283185307179586476925, z = y * y;
  double s = 1.0 / 6227020800.0;
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, y, y);
  double c = -1.0 / 87178291200.0;
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int n = (int)k & 3;  // k is -2 .. 2
  const double a = n & 1 ? s : c, b = n & 1 ? c : s;
  return make_float2((float)(n == 1 || n == 2 ? -a : a), (float)(n >= 2 ? -b : b));
}

// A lane's part of a head: where it comes from and goes to.
struct Part {
  const char* src;
  char* dst;          // null: passed over
  const char *bias, *gain;
  int row;            // of the workgroup's
  bool turned;
};

template <typename T, int D, int ROWS>
__global__ __launch_bounds__(AP_NT) void append_kernel(AppendParams p) {
  constexpr int HALF = D / 2, LANES = HALF / 8;  // lanes of a head
  __shared__ float2 s_turn[ROWS][HALF];
  const int t = threadIdx.x;
  const int heads = p.nq + 2 * p.nkv, lanes = heads * LANES, parts = ROWS * lanes;
  const int64_t groups = (p.rows + ROWS - 1) / ROWS;
#pragma unroll 1
  for (int64_t group = blockIdx.x; group < groups; group += gridDim.x) {
    const int64_t row0 = group * ROWS;
    const auto part_of = [&](int n) {
      Part a;
      a.row = ROWS == 1 ? 0 : n / lanes;
      const int in_row = n - a.row * lanes, h = in_row / LANES, c = in_row % LANES * 8;
      const int64_t row = row0 + a.row;
      const bool there = n < parts && row < p.rows;
      const int pos = there ? p.positions[row] : -1;
      a.dst = nullptr;
      a.src = nullptr;
      if (h < p.nq) {
        a.turned = true;
        a.bias = p.bq ? p.bq + (h * D + c) * sizeof(T) : nullptr;
        a.gain = p.q_norm ? p.q_norm + c * sizeof(T) : nullptr;
        if (pos >= 0) {
          a.src = p.q + row * p.q_stride + (h * D + c) * (int64_t)sizeof(T);
          a.dst = p.q_out + row * p.q_out_stride + (h * D + c) * (int64_t)sizeof(T);
        }
      } else {
        const bool is_v = h >= p.nq + p.nkv;
        const int at = (h - p.nq - (is_v ? p.nkv : 0)) * D + c;
        const char* bias = is_v ? p.bv : p.bk;
        a.turned = !is_v;
        a.bias = bias ? bias + at * sizeof(T) : nullptr;
        a.gain = !is_v && p.k_norm ? p.k_norm + c * sizeof(T) : nullptr;
        const int64_t slot = pos >= 0 ? p.slots[row] : -1;
        if (slot >= 0 && slot < p.arena_slots) {
          a.src = (is_v ? p.v + row * p.v_stride : p.k + row * p.k_stride) + at * (int64_t)sizeof(T);
          a.dst = (is_v ? p.plane_v : p.plane_k) + (slot * p.nkv * D + at) * (int64_t)sizeof(T);
        }
      }
      return a;
    };
    Raw8<T> lo, hi;
    Part cur = part_of(t);
    if (cur.dst) {
      lo.load(cur.src);
      hi.load(cur.src + HALF * sizeof(T));
    }
    for (int i = t; i < ROWS * HALF; i += AP_NT) {
      const int64_t row = row0 + i / HALF;
      const int pos = row < p.rows ? p.positions[row] : 0;
      const int pair = i % HALF;
      s_turn[i / HALF][pair] =
          cos_sin_turns(pos * exp2(-2.0 * pair / D * p.log2_theta - 2.651496129472318798043));
    }
    __syncthreads();
#pragma unroll 1
    for (int n = t; n < parts; n += AP_NT) {
      float a[8], b[8];
      lo.values(a);
      hi.values(b);
      const Part now = cur;
      cur = part_of(n + AP_NT);
      if (cur.dst) {
        lo.load(cur.src);
        hi.load(cur.src + HALF * sizeof(T));
      }
      const int c = n % LANES * 8;
      if (now.bias && now.dst) {
        Raw8<T> x, y;
        float u[8], w[8];
        x.load(now.bias);
        y.load(now.bias + HALF * sizeof(T));
        x.values(u);
        y.values(w);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          a[i] += u[i];
          b[i] += w[i];
        }
      }
      if constexpr (D >= 32) {
        // the lanes of a head share its row, so all of them are here or none
        if (now.gain && now.dst) {
          float ss = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) ss = fmaf(a[i], a[i], fmaf(b[i], b[i], ss));
#pragma unroll
          for (int o = 1; o < LANES; o *= 2) ss += __shfl_xor(ss, o, 64);
          const float inv = 1.0f / sqrtf(ss / (float)D + p.eps);
          Raw8<T> x, y;
          float u[8], w[8];
          x.load(now.gain);
          y.load(now.gain + HALF * sizeof(T));
          x.values(u);
          y.values(w);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            a[i] = a[i] * inv * u[i];
            b[i] = b[i] * inv * w[i];
          }
        }
      }
      if (now.turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = s_turn[now.row][c + i];
          const float x = a[i], y = b[i];
          a[i] = x * cs.x - y * cs.y;
          b[i] = y * cs.x + x * cs.y;
        }
      }
      if (now.dst) {
        Raw8<T>::store(now.dst, a);
        Raw8<T>::store(now.dst + HALF * sizeof(T), b);
      }
    }
    __syncthreads();  // the angles have been read
  }
}

template <typename T, int D, int ROWS>
void launch_rows(const AppendParams& p, hipStream_t s) {
  const int64_t groups = (p.rows + ROWS - 1) / ROWS;
  hipLaunchKernelGGL((append_kernel<T, D, ROWS>), dim3((unsigned)std::min<int64_t>(groups, 1 << 20)), dim3(AP_NT), 0, s,
                     p);
}
template <typename T, int D>
void launch_append(const AppendParams& p, hipStream_t s) {
  // rows of a workgroup, by the calls' us with one and with four: 1024 rows of 64 q and 8 kv heads of
  // 128 in bf16 11.0 and 16.4, 2048 18.4 and 19.7, 4096 43.9 and 40.2; of 32 + 8 heads 8.3 and
  // 10.0, 11.9 and 11.6, 25.8 and 22.1; of 8 + 2 heads 7.0 and 6.9, 8.1 and 7.2, 12.7 and 8.7
  if (p.rows > 2048) launch_rows<T, D, 4>(p, s);
  else launch_rows<T, D, 1>(p, s);
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" kv_status kv_append(kv_arena_t arena, int32_t layer, const kv_layer_weights* weights, const void* q,
                               int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               const int32_t* positions, const int64_t* slots, int64_t rows, void* q_out,
                               int64_t q_out_stride, void* stream) {
  if (!live_arena(arena)) return kvr_err::set(KV_ESTATE, "unknown or released arena handle");
  const kv_model_desc& d = arena->desc;
  const int64_t e = elem_bytes(d.dtype);
  const int64_t q_row = (int64_t)d.num_q_heads * d.head_dim, kv_row = (int64_t)d.num_kv_heads * d.head_dim;
  if (layer < 0 || layer >= d.num_layers)
    return kvr_err::set(KV_EINVAL, "layer %d outside [0, %d)", layer, d.num_layers);
  if (rows < 0 || rows > INT32_MAX) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^31 - 1");
  if (q_row + 2 * kv_row > 1 << 24) return kvr_err::set(KV_EINVAL, "more than 2^24 values a row");
  if (rows == 0) return kvr_err::clear();
  if (!k || !v || !positions || !slots) return kvr_err::set(KV_EINVAL, "null k, v, positions or slots");
  if (!q != !q_out) return kvr_err::set(KV_EINVAL, "q and q_out go together");
  if (k_stride < kv_row || v_stride < kv_row || (q && (q_stride < q_row || q_out_stride < q_row)))
    return kvr_err::set(KV_EINVAL, "a stride is below its row");
  if (k_stride > INT64_MAX / 8 / rows || v_stride > INT64_MAX / 8 / rows ||
      (q && (q_stride > INT64_MAX / 8 / rows || q_out_stride > INT64_MAX / 8 / rows)))
    return kvr_err::set(KV_EINVAL, "a stride beyond the addresses there are");
  if (q == q_out && q && q_stride != q_out_stride)
    return kvr_err::set(KV_EINVAL, "q_out over q needs the same stride");
  const auto bytes = [&](int64_t stride) { return (uintptr_t)(stride * e); };
  uintptr_t all = (uintptr_t)k | (uintptr_t)v | bytes(k_stride) | bytes(v_stride) | (uintptr_t)positions;
  if (q) all |= (uintptr_t)q | (uintptr_t)q_out | bytes(q_stride) | bytes(q_out_stride);
  AppendParams p{};
  if (d.qk_norm || d.qkv_bias) {
    if (!weights) return kvr_err::set(KV_EINVAL, "null weights of a model with norms or biases");
    if (d.qk_norm) {
      if (!weights->k_norm || (q && !weights->q_norm)) return kvr_err::set(KV_EINVAL, "null q_norm or k_norm");
      p.k_norm = static_cast<const char*>(weights->k_norm);
      p.q_norm = q ? static_cast<const char*>(weights->q_norm) : nullptr;
    }
    if (d.qkv_bias) {
      if (!weights->bk || !weights->bv || (q && !weights->bq)) return kvr_err::set(KV_EINVAL, "null bq, bk or bv");
      p.bk = static_cast<const char*>(weights->bk);
      p.bv = static_cast<const char*>(weights->bv);
      p.bq = q ? static_cast<const char*>(weights->bq) : nullptr;
    }
    all |= (uintptr_t)p.q_norm | (uintptr_t)p.k_norm | (uintptr_t)p.bq | (uintptr_t)p.bk | (uintptr_t)p.bv;
  }
  if (all % 4 != 0 || (uintptr_t)slots % 8 != 0)
    return kvr_err::set(KV_EINVAL, "arrays and strides need boundaries of 4 bytes, slots one of 8");
  if ((uintptr_t)arena->base % 4 != 0) return kvr_err::set(KV_EINVAL, "the arena does not start on a boundary of 4 bytes");
  DeviceGuard dg(arena->device);
  const kv_status st = device_ready(dg, arena->device);
  if (st != KV_OK) return st;
  p.q = static_cast<const char*>(q);
  p.k = static_cast<const char*>(k);
  p.v = static_cast<const char*>(v);
  p.q_out = static_cast<char*>(q_out);
  p.arena_slots = arena->num_blocks * arena->block_size;
  const int64_t plane = p.arena_slots * kv_row * e;
  p.plane_k = static_cast<char*>(arena->base) + 2 * layer * plane;
  p.plane_v = p.plane_k + plane;
  p.q_stride = q_stride * e;
  p.k_stride = k_stride * e;
  p.v_stride = v_stride * e;
  p.q_out_stride = q_out_stride * e;
  p.positions = positions;
  p.slots = slots;
  p.rows = rows;
  p.nq = q ? d.num_q_heads : 0;
  p.nkv = d.num_kv_heads;
  p.eps = (float)d.rms_eps;
  p.log2_theta = log2(d.rope_theta);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (d.dtype == KV_BF16) launch_append<bf16_t, 128>(p, s);
  else if (d.head_dim == 128) launch_append<float, 128>(p, s);
  else if (d.head_dim == 64) launch_append<float, 64>(p, s);
  else if (d.head_dim == 32) launch_append<float, 32>(p, s);
  else launch_append<float, 16>(p, s);
  return launched();
}

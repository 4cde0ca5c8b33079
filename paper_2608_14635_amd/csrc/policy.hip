// The clipped policy loss and the gradient of its logits (kvr_policy.h).
//
// With t_v = c (z_v - m) as in logits.h, e_v = 2^t_v, rest = sum over v != t of e_v and
// mine = e_t:
//   lp = -log1p(rest / mine),   p_v = e_v / (rest + mine),   1 - p_t = rest / (rest + mine)
// The token's own term stays out of the sum: for a token that is all but certain, what is
// left of 1 - p_t in a sum with its 1 is noise.  The gradient is one factor of the row times
// e_v, but for the token's entry.
//
// Many rows, or short ones: a workgroup a row.  Its threads pass over the row once for their
// largest logits and sums, join them, and pass over it again for the gradient, backwards: what
// was read last is in the L2 cache yet, the rest in the last-level one, which holds the rows of
// all workgroups at once.  A row that fits the threads' registers is read once.
// Few long rows: a row is cut into chunks; a workgroup reads its chunk once, into registers, and
// leaves its largest logit and sum.  A wave merges the chunks of a row in a fixed order.  A third
// kernel turns logits into gradients.
// What is done once a row is done in fp64, by short series: the library's exp, log, log1p and expm1
// are some hundred instructions each, which a row's only lane would wait for from memory.
#include <algorithm>

#include "common.h"
#include "host.h"
#include "kvr_policy.h"
#include "logits.h"

namespace kvr {
namespace {

constexpr int PL_NT = 256;
constexpr int PL_ITEMS = 32;                  // entries of a thread
constexpr int PL_CHUNK = PL_NT * PL_ITEMS;
constexpr int PL_MAX_VOCAB = 256 * PL_CHUNK;
constexpr int64_t PL_MOST_CHUNKS = (1 << 24) - 1;  // of a call: a grid holds 2^32 - 1 threads

// What the gradient of a row takes: for v != tok, mul 2^t_v with t_v relative to base; at_tok.
struct RowGrad {
  float base, mul, at_tok;
  int tok;  // -1: a row of zeros, whatever its logits
};

struct PolicyParams {
  const char* logits;
  char* grad;
  int64_t stride, grad_stride;  // bytes
  int64_t rows;
  int vocab, chunks;
  float scale, c, c_rest;  // c + c_rest = scale log2 e
  const int32_t* tokens;
  const float *old, *ref, *advantages, *weights;
  double low, high;  // clip bounds of rho
  float kl_coef;
  float *total, *losses, *logprobs, *kls;
  float2* stats;      // [rows][chunks] largest logit, sum without the token's
  RowGrad* row_grad;  // [rows]
  double* row_loss;   // [rows]
};

// t of a logit relative to a base whose C is cm.
__device__ __forceinline__ float t_of(const PolicyParams& p, float z, float base, float cm, bool by) {
  return by ? fmaf(z, p.c, -cm) : (z - base) * p.c;
}

// A thread's VECS pieces of the row's entries begin + i STEP + t VEC ..; entries past the row's
// end are -infinity.  A piece that crosses the end is loaded entry by entry.
template <typename T, int VECS>
__device__ __forceinline__ void load_pieces(const T* z, int begin, int vocab, Piece<T> (&v)[VECS]) {
  constexpr int VEC = Piece<T>::N, STEP = PL_NT * VEC;
  const int t = threadIdx.x;
  if (begin + VECS * STEP <= vocab) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) v[i].load(z + (begin + i * STEP) + (uint32_t)(t * VEC));
    return;
  }
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = begin + i * STEP + t * VEC;
    v[i] = Piece<T>{};
    if (at + VEC <= vocab) {
      v[i].load(z + at);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[i].set(j, at + j < vocab ? Elem<T>::load(z, at + j) : -INFINITY);
    }
  }
}

template <typename T>
__global__ __launch_bounds__(PL_NT) void policy_chunk_kernel(PolicyParams p) {
  constexpr int VEC = Piece<T>::N, VECS = PL_ITEMS / VEC, STEP = PL_NT * VEC;
  __shared__ float s_red[2][PL_NT / 64];
  const int t = threadIdx.x;
  const int c = blockIdx.x % p.chunks;
  const int64_t row = blockIdx.x / p.chunks;
  const int tok = p.tokens[row];
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int begin = c * PL_CHUNK;
  Piece<T> v[VECS];
  load_pieces(z, begin, p.vocab, v);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < VECS; ++i)
#pragma unroll
    for (int j = 0; j < VEC; ++j) m = fmaxf(m, v[i].value(j));
  m = max_over_wave(m);
  if ((t & 63) == 0) s_red[0][t >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PL_NT / 64; ++i) m = fmaxf(m, s_red[0][i]);
  if (tok >= begin && tok < begin + PL_CHUNK) {  // a NaN or +infinity of its own counts with the row's sums
    const int at = tok - begin;
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (at == i * STEP + t * VEC + j) v[i].set(j, -INFINITY);
  }
  const float base = base_of(m), cm = c_of(base, p.c);
  const bool by = by_c(cm);
  float l = 0.0f;
  if (by) {
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) l += __builtin_amdgcn_exp2f(fmaf(v[i].value(j), p.c, -cm));
  } else {
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) l += __builtin_amdgcn_exp2f((v[i].value(j) - base) * p.c);
  }
  l = sum_over_wave(l);
  if ((t & 63) == 0) s_red[1][t >> 6] = l;
  __syncthreads();
  if (t == 0) {
    l = 0.0f;
#pragma unroll
    for (int i = 0; i < PL_NT / 64; ++i) l += s_red[1][i];
    p.stats[row * p.chunks + c] = make_float2(m, l);
  }
}

__device__ __forceinline__ double sum_over_wave(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// e^x - 1: x = n ln 2 + r with |r| <= ln 2 / 2, 2^n (e^r - 1) + (2^n - 1), e^r - 1 by its series
// to r^13 (the next term is below 2^-57 of r).  `one`: e^x instead.
__device__ __forceinline__ double exp_less(double x, bool one) {
  const double n = rint(fmin(fmax(x, -800.0), 800.0) * 1.442695040888963407360);
  const double r = fma(-n, 1.90821492927058770002e-10, fma(-n, 6.93147180369123816490e-01, x));  // ln 2 in two parts
  double s = 1.0 / 6227020800.0;
  s = fma(s, r, 1.0 / 479001600.0);
  s = fma(s, r, 1.0 / 39916800.0);
  s = fma(s, r, 1.0 / 3628800.0);
  s = fma(s, r, 1.0 / 362880.0);
  s = fma(s, r, 1.0 / 40320.0);
  s = fma(s, r, 1.0 / 5040.0);
  s = fma(s, r, 1.0 / 720.0);
  s = fma(s, r, 1.0 / 120.0);
  s = fma(s, r, 1.0 / 24.0);
  s = fma(s, r, 1.0 / 6.0);
  s = fma(s, r, 0.5);
  s = fma(s * r, r, r);
  const int k = (int)n;
  const double y = ldexp(s, k), z = ldexp(1.0, k);
  const double v = one ? y + z : y + (z - 1.0);
  return x > 709.0 ? INFINITY : x < -750.0 ? (one ? 0.0 : -1.0) : x != x ? x : v;
}
// log(a / b) for 0.5 <= a / b <= 2: 2 atanh(s), s = (a - b) / (a + b), |s| <= 1/3, by its series
// to s^33 (the next term is below 2^-57 of s).  less: a - b.
__device__ __forceinline__ double log_ratio(double less, double sum) {
  const double s = less / sum, z = s * s;
  double y = 1.0 / 33.0;
#pragma unroll
  for (int i = 31; i >= 3; i -= 2) y = fma(y, z, 1.0 / i);
  return 2.0 * fma(y * z, s, s);
}
// log a, a > 0 and finite.
__device__ __forceinline__ double log_of(double a) {
  int k;
  const double m = frexp(a, &k);  // 0.5 .. 1
  return fma((double)k, 6.93147180559945309417e-01, log_ratio(m - 1.0, m + 1.0));
}

// What a chunk's t_v leave out, in log2 units: the rounding of its C.
__device__ __forceinline__ double c_rounding(const PolicyParams& p, float base) {
  const float cm = c_of(base, p.c);
  return by_c(cm) ? (double)base * p.c - cm : 0.0;
}

// 1 - 2^-x of that, |x| <= 2^-5 (C is below 2^20).
__device__ __forceinline__ double c_rounding_less(const PolicyParams& p, float base) {
  return -exp_less(-6.93147180559945309417e-01 * c_rounding(p, base), false);
}

// A row's inputs besides its logits.
struct RowIn {
  int tok;
  float z, old, ref, advantage, weight;
};
template <typename T>
__device__ __forceinline__ RowIn row_in(const PolicyParams& p, int64_t row, int tok) {
  RowIn r;
  r.tok = tok;
  r.old = p.old ? p.old[row] : 0.0f;
  r.ref = p.ref ? p.ref[row] : 0.0f;
  r.advantage = p.advantages[row];
  r.weight = p.weights ? p.weights[row] : 1.0f;
  r.z = tok >= 0 && tok < p.vocab ? Elem<T>::load(reinterpret_cast<const T*>(p.logits + row * p.stride), tok) : 0.0f;
  return r;
}

// A row's results from its largest logit m and the others' sum `rest`, relative to m.
__device__ __forceinline__ RowGrad finish_row(const PolicyParams& p, int64_t row, const RowIn& r, float m, double rest) {
  const double scale = p.scale, base = base_of(m);
  const float w = r.weight;
  const bool in = r.tok >= 0 && r.tok < p.vocab;
  double lp = 0.0, kl = 0.0, loss = 0.0, slope = 0.0, not_t = 0.0, all = 1.0;
  bool none = true;
  if (in) {
    const double x = scale * ((double)r.z - base), mine = exp_less(x, true);
    all = rest + mine;
    none = all == 0.0;  // every logit is -infinity
    lp = none ? -INFINITY : rest < mine ? -log_ratio(rest, mine + all) : x - log_of(all);
    if (all != all) lp = all;
    not_t = none ? 1.0 : rest / all;
  }
  if (in && w != 0.0f) {
    const double a = r.advantage;
    const double rho = p.old ? exp_less(lp - r.old, true) : lp != lp ? lp : 1.0;
    const double plain = rho * a, cut = fmin(fmax(rho, p.low), p.high) * a;
    const bool kept = !(plain > cut);
    double fall = 0.0;
    if (p.ref) {
      const double d = r.ref - lp, e = exp_less(d, false);
      kl = e == INFINITY ? e : e - d;
      if (p.kl_coef != 0.0f) fall = p.kl_coef * e;
    }
    loss = w * ((p.kl_coef != 0.0f ? p.kl_coef * kl : 0.0) - (kept ? plain : cut));
    slope = w * scale * (-(kept ? plain : 0.0) - fall);
  }
  if (p.losses) p.losses[row] = (float)loss;
  if (p.logprobs) p.logprobs[row] = (float)lp;
  if (p.kls) p.kls[row] = (float)kl;
  if (p.total) p.row_loss[row] = loss;
  RowGrad g;
  g.base = (float)base;
  g.mul = none ? 0.0f : (float)(-slope / all * (1.0 - c_rounding_less(p, g.base)));
  g.at_tok = (float)(slope * not_t);
  g.tok = in && w != 0.0f ? r.tok : -1;
  return g;
}

// A sum relative to its largest logit m, relative to `most` and without the rounding of its C.
// The exponent is taken in fp64, what fp32 leaves of it as a factor.
__device__ __forceinline__ float joined(const PolicyParams& p, float m, float l, float most) {
  const double x = ((double)base_of(m) - base_of(most)) * ((double)p.c + p.c_rest) - c_rounding(p, base_of(m));
  const float hi = (float)x, lo = (float)(x - hi);
  const float f = __builtin_amdgcn_exp2f(hi);
  return l == 0.0f || f == 0.0f ? (l != l ? l : 0.0f) : l * fmaf(f, lo * LN2, f);
}

// A wave a row.
template <typename T>
__global__ __launch_bounds__(PL_NT) void policy_row_kernel(PolicyParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (PL_NT / 64) + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  const RowIn in = row_in<T>(p, row, p.tokens[row]);
  const float2* stats = p.stats + row * p.chunks;
  float m = -INFINITY;
  for (int i = lane; i < p.chunks; i += 64) m = fmaxf(m, stats[i].x);
  m = max_over_wave(m);
  float sum = 0.0f;
  for (int i = lane; i < p.chunks; i += 64) {
    const float2 q = stats[i];
    sum += joined(p, q.x, q.y, m);
  }
  const double rest = sum_over_wave(sum);
  if (lane == 0) {
    const RowGrad g = finish_row(p, row, in, m, rest);
    if (p.grad) p.row_grad[row] = g;
  }
}

// The rows' losses, the threads of NT in turn.
template <int NT>
__device__ __forceinline__ void put_total(const PolicyParams& p) {
  __shared__ double s_sum[NT / 64];
  double v = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < p.rows; i += NT) v += p.row_loss[i];
  v = sum_over_wave(v);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = s_sum[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) v += s_sum[i];
    *p.total = (float)v;
  }
}
constexpr int TOTAL_NT = 512;
__global__ __launch_bounds__(TOTAL_NT) void policy_total_kernel(PolicyParams p) { put_total<TOTAL_NT>(p); }

__device__ __forceinline__ void put_entry(float* p, float v) { *p = v; }
__device__ __forceinline__ void put_entry(bf16_t* p, float v) { *p = f2bf(v); }

template <typename T>
__global__ __launch_bounds__(PL_NT) void policy_grad_kernel(PolicyParams p) {
  constexpr int VEC = Piece<T>::N, VECS = PL_ITEMS / VEC, STEP = PL_NT * VEC;
  const int t = threadIdx.x;
  const int c = blockIdx.x % p.chunks;
  const int64_t row = blockIdx.x / p.chunks;
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  T* out = reinterpret_cast<T*>(p.grad + row * p.grad_stride);
  const RowGrad g = p.row_grad[row];
  const int begin = c * PL_CHUNK;
  Piece<T> v[VECS];
  load_pieces(z, begin, p.vocab, v);
  const float cm = c_of(g.base, p.c);
  const bool by = by_c(cm);
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = begin + i * STEP + t * VEC;
    float y[VEC];
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      y[j] = g.mul * __builtin_amdgcn_exp2f(t_of(p, v[i].value(j), g.base, cm, by));
      if (at + j == g.tok) y[j] = g.at_tok;
      if (g.tok < 0) y[j] = 0.0f;
    }
    if (at + VEC <= p.vocab) {
      Piece<T> w;
      w.put(y);
      w.store(out + at);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j)
        if (at + j < p.vocab) put_entry(out + at + j, y[j]);
    }
  }
  if (p.total && blockIdx.x == 0) put_total<PL_NT>(p);
}

// Gradients of a piece's entries `at` .. of a row that is not left out; the token's own entry is
// put afterwards.
template <typename T>
__device__ __forceinline__ void put_grad(const PolicyParams& p, const RowGrad& g, float cm, bool by, const Piece<T>& v,
                                         T* out, int at) {
  constexpr int VEC = Piece<T>::N;
  float y[VEC];
  if (by) {
#pragma unroll
    for (int j = 0; j < VEC; ++j) y[j] = g.mul * __builtin_amdgcn_exp2f(fmaf(v.value(j), p.c, -cm));
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j) y[j] = g.mul * __builtin_amdgcn_exp2f((v.value(j) - g.base) * p.c);
  }
  if (at + VEC <= p.vocab) {
    Piece<T> w;
    w.put(y);
    w.store(out + at);
  } else {
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (at + j < p.vocab) put_entry(out + at + j, y[j]);
  }
}

// A workgroup of NT threads a row, U pieces of a thread at a time.  HELD: all of the row's.
template <typename T, int NT, int U, bool HELD>
__global__ __launch_bounds__(NT) void policy_whole_kernel(PolicyParams p) {
  constexpr int VEC = Piece<T>::N, WAVES = NT / 64, STEP = NT * VEC, TURN = U * STEP;
  __shared__ float s_most[WAVES], s_sum[WAVES];
  __shared__ RowGrad s_grad;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int tok = p.tokens[row];
  const int turns = HELD ? 1 : (p.vocab + TURN - 1) / TURN;
  Piece<T> v[U];
  const auto load = [&](int begin) {
    if (begin + TURN <= p.vocab) {
#pragma unroll
      for (int i = 0; i < U; ++i) v[i].load(z + (begin + i * STEP) + (uint32_t)(t * VEC));
      return;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = begin + i * STEP + t * VEC;
      v[i] = Piece<T>{};
      if (at + VEC <= p.vocab) {
        v[i].load(z + at);
      } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[i].set(j, at + j < p.vocab ? Elem<T>::load(z, at + j) : -INFINITY);
      }
    }
  };
  RowIn in;
  if (t == 0) in = row_in<T>(p, row, tok);
  float m = -INFINITY, l = 0.0f;
#pragma unroll 1
  for (int turn = 0; turn < turns; ++turn) {
    const int begin = turn * TURN;
    load(begin);
    float most = m;
#pragma unroll
    for (int i = 0; i < U; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) most = fmaxf(most, v[i].value(j));
    const float cm = c_of(base_of(most), p.c);
    if (most > m) {
      const float was = c_of(base_of(m), p.c);
      const float x = by_c(cm) && by_c(was) ? was - cm : (m - most) * p.c;
      l = l == 0.0f ? 0.0f : l * __builtin_amdgcn_exp2f(x);
      m = most;
    }
    const int at = tok - begin;  // the token's entry stays out of the sum
    if (at >= 0 && at < TURN) {
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j)
          if (at == i * STEP + t * VEC + j) v[i].set(j, -INFINITY);
    }
    if (by_c(cm)) {
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) l += __builtin_amdgcn_exp2f(fmaf(v[i].value(j), p.c, -cm));
    } else {
      const float base = base_of(m);
#pragma unroll
      for (int i = 0; i < U; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) l += __builtin_amdgcn_exp2f((v[i].value(j) - base) * p.c);
    }
  }
  // ---- the threads' sums, then the waves' ----
  const float wave_most = max_over_wave(m);
  const float wave_sum = sum_over_wave(joined(p, m, l, wave_most));
  if ((t & 63) == 0) {
    s_most[t >> 6] = wave_most;
    s_sum[t >> 6] = wave_sum;
  }
  __syncthreads();
  if (t < 64) {
    const int i = min(t, WAVES - 1);
    const float most = max_over_wave(s_most[i]);
    // a wave's sum has no rounded C in it
    const double x = ((double)base_of(s_most[i]) - base_of(most)) * ((double)p.c + p.c_rest);
    double sum = t < WAVES && s_sum[i] != 0.0f ? s_sum[i] * exp_less(x * 6.93147180559945309417e-01, true) : 0.0;
#pragma unroll
    for (int o = WAVES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (t == 0) s_grad = finish_row(p, row, in, most, sum);
  }
  if (!p.grad) return;
  __syncthreads();
  // ---- the gradient ----
  const RowGrad g = s_grad;
  T* out = reinterpret_cast<T*>(p.grad + row * p.grad_stride);
  if (g.tok < 0) {
    Piece<T> zero{};
    for (int at = t * VEC; at < p.vocab; at += STEP) {
      if (at + VEC <= p.vocab) {
        zero.store(out + at);
      } else {
        for (int j = at; j < p.vocab; ++j) put_entry(out + j, 0.0f);
      }
    }
    return;
  }
  const float cm = c_of(g.base, p.c);
  const bool by = by_c(cm);
#pragma unroll 1
  for (int turn = turns - 1; turn >= 0; --turn) {
    const int begin = turn * TURN;
    if (!HELD) load(begin);
#pragma unroll
    for (int i = 0; i < U; ++i) put_grad(p, g, cm, by, v[i], out, begin + i * STEP + t * VEC);
  }
  if (g.tok % STEP / VEC == t) put_entry(out + g.tok, g.at_tok);  // after the thread's own store there
}

int chunks_of(int vocab) { return (vocab + PL_CHUNK - 1) / PL_CHUNK; }

// Whether a call's rows are taken whole: they fit a workgroup's registers, or there are enough of
// them.
constexpr int WHOLE_ROWS = 160;
template <typename T, int NT, int U, bool HELD>
void launch_whole(const PolicyParams& p, hipStream_t s) {
  hipLaunchKernelGGL((policy_whole_kernel<T, NT, U, HELD>), dim3((unsigned)p.rows), dim3(NT), 0, s, p);
  if (p.total) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(TOTAL_NT), 0, s, p);
}
template <typename T>
void launch(const PolicyParams& p, hipStream_t s) {
  constexpr int VEC = Piece<T>::N, SMALL = 32 / VEC, U = 8;
  if (p.vocab <= 256 * 32) return launch_whole<T, 256, SMALL, true>(p, s);
  if (p.rows >= WHOLE_ROWS) {
    if (p.vocab <= 1024 * VEC * U) return launch_whole<T, 1024, U, true>(p, s);
    return launch_whole<T, 1024, U, false>(p, s);
  }
  const dim3 grid((unsigned)(p.rows * p.chunks)), nt(PL_NT);
  hipLaunchKernelGGL((policy_chunk_kernel<T>), grid, nt, 0, s, p);
  hipLaunchKernelGGL((policy_row_kernel<T>), dim3((unsigned)((p.rows + PL_NT / 64 - 1) / (PL_NT / 64))), nt, 0, s, p);
  if (p.grad) hipLaunchKernelGGL((policy_grad_kernel<T>), grid, nt, 0, s, p);
  else if (p.total) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(TOTAL_NT), 0, s, p);
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

uint64_t kv_policy_loss_workspace_bytes(int64_t rows, int32_t vocab) {
  if (rows <= 0 || rows > (1 << 20) || vocab <= 0 || vocab > PL_MAX_VOCAB) return 0;
  const int64_t chunks = chunks_of(vocab);
  if (rows * chunks > PL_MOST_CHUNKS) return 0;
  return (uint64_t)(rows * (sizeof(RowGrad) + sizeof(double) + chunks * sizeof(float2)));
}

kv_status kv_policy_loss(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t stride, float scale,
                         const int32_t* tokens, const float* old_logprobs, const float* ref_logprobs,
                         const float* advantages, const float* weights, float clip_low, float clip_high, float kl_coef,
                         float* total, float* losses, float* logprobs, float* kls, void* grad, int64_t grad_stride,
                         void* workspace, uint64_t ws_bytes, int32_t device, void* stream) {
  if (dtype != KV_F32 && dtype != KV_BF16) return kvr_err::set(KV_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > (1 << 20)) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^20");
  if (vocab < 1 || vocab > PL_MAX_VOCAB) return kvr_err::set(KV_EINVAL, "vocab must be 1 .. 2^21");
  if (rows * chunks_of(vocab) > PL_MOST_CHUNKS)
    return kvr_err::set(KV_EINVAL, "rows * vocab of one call above 2^37: split the rows");
  const int64_t most_stride = INT64_MAX / 8 / std::max<int64_t>(rows, 1);
  if (stride < vocab || stride > most_stride || (grad && (grad_stride < vocab || grad_stride > most_stride)))
    return kvr_err::set(KV_EINVAL, "a stride is below the vocabulary, or beyond the addresses there are");
  if (!(scale > 0.0f) || !(scale <= 0x1p127f))
    return kvr_err::set(KV_EINVAL, "scale must be positive and at most 2^127");
  if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f))
    return kvr_err::set(KV_EINVAL, "clip_low must be 0 .. 1, clip_high at least 0");
  if (!(kl_coef - kl_coef == 0.0f)) return kvr_err::set(KV_EINVAL, "kl_coef must be finite");
  if (!ref_logprobs && (kl_coef != 0.0f || kls))
    return kvr_err::set(KV_EINVAL, "kl_coef and kls need ref_logprobs");
  if (rows == 0 && !total) return kvr_err::clear();
  if (rows > 0 && (!logits || !tokens || !advantages))
    return kvr_err::set(KV_EINVAL, "null logits, tokens or advantages");
  if (!total && !losses && !logprobs && !kls && !grad) return kvr_err::clear();
  if (grad == logits && grad && grad_stride != stride)
    return kvr_err::set(KV_EINVAL, "grad over the logits needs the same stride");
  const uintptr_t words = (uintptr_t)tokens | (uintptr_t)old_logprobs | (uintptr_t)ref_logprobs |
                          (uintptr_t)advantages | (uintptr_t)weights | (uintptr_t)total | (uintptr_t)losses |
                          (uintptr_t)logprobs | (uintptr_t)kls;
  if (words % 4 != 0 || ((uintptr_t)logits | (uintptr_t)grad) % elem_bytes(dtype) != 0)
    return kvr_err::set(KV_EINVAL, "an array does not start on a boundary of its elements");
  PolicyParams p{};
  if (rows > 0) {
    if (!workspace || (uintptr_t)workspace % 16 != 0)
      return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
    const uint64_t need = kv_policy_loss_workspace_bytes(rows, vocab);
    if (need > ws_bytes)
      return kvr_err::set(KV_ENOMEM, "workspace of %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                          (unsigned long long)need);
  }
  DeviceGuard dg(device);
  const kv_status st = device_ready(dg, device);
  if (st != KV_OK) return st;
  p.logits = static_cast<const char*>(logits);
  p.grad = static_cast<char*>(grad);
  p.stride = stride * elem_bytes(dtype);
  p.grad_stride = grad_stride * elem_bytes(dtype);
  p.rows = rows;
  p.vocab = vocab;
  p.chunks = chunks_of(vocab);
  p.scale = scale;
  const double c = (double)scale * 1.442695040888963407360;
  p.c = (float)c;
  p.c_rest = (float)(c - p.c);
  p.tokens = tokens;
  p.old = old_logprobs;
  p.ref = ref_logprobs;
  p.advantages = advantages;
  p.weights = weights;
  p.low = 1.0 - clip_low;
  p.high = 1.0 + clip_high;
  p.kl_coef = kl_coef;
  p.total = total;
  p.losses = losses;
  p.logprobs = logprobs;
  p.kls = kls;
  p.row_grad = static_cast<RowGrad*>(workspace);
  p.row_loss = reinterpret_cast<double*>(p.row_grad + rows);
  p.stats = reinterpret_cast<float2*>(p.row_loss + rows);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (rows == 0) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(TOTAL_NT), 0, s, p);
  else if (dtype == KV_BF16) launch<bf16_t>(p, s);
  else launch<float>(p, s);
  return launched();
}

}  // extern "C"

// The clipped policy loss and the gradient of its logits (kvr_policy.h).
//
// With t_v = c (z_v - m) as in logits.h, e_v = 2^t_v, rest = sum over v != t of e_v and
// mine = e_t:
//   lp = -log1p(rest / mine),   p_v = e_v / (rest + mine),   1 - p_t = rest / (rest + mine)
// The token's own term stays out of the sum: for a token that is all but certain, what is
// left of 1 - p_t in a sum with its 1 is noise.  The gradient is one factor of the row times
// e_v, but for the token's entry.
//
// Rows that fit the registers of a workgroup, and many longer ones whose gradient is wanted: a
// workgroup a row, which it holds there, as much of it as fits.  Its threads take their largest
// logits and sums, join them, and turn what they hold into gradients: the logits are read once.
// Losses alone of a row to a CU: the same, without holding it.
// Few long rows, and losses of many: a row is cut into chunks; a workgroup reads its chunk once, into
// registers, and leaves its largest logit and sum.  A wave merges the chunks of a row in a fixed
// order.  A third kernel turns logits into gradients.
// What is done once a row is done in fp64, by short series: the library's exp, log, log1p and expm1
// are some hundred instructions each, which a row's only lane would wait for from memory.
//
// Bound by memory where there is much of it: 1024 rows of 151936 bf16 logits with gradient, 622 MB, in
// 149 us (4.2 TB/s; a copy reaches 4.7), 250 rows of 152064 fp32 ones 304 MB in 68 (4.5), losses
// of 384 rows of 128256 bf16 logits 98.5 MB in 22.6 (4.4) + 6.2 + 3.8.  By waiting where there is
// little: 171 rows of 1024 in 5.7 + 1.6.
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

// What the gradient of a row takes: for v != tok, mul 2^(t_v + more) with t_v relative to base; at_tok.
struct RowGrad {
  float base, mul, at_tok;
  float more;  // 0, but where mul would be large
  int tok;     // -1: a row of zeros, whatever its logits
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

// In fp64, for what is done once a row or a wave of it: a row's threads joined so and in fp32 by
// lane moves took the same 152.4 - 153.6 us (1024 rows of 151936 bf16 logits).
__device__ __forceinline__ double sum64_over_wave(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// The series' coefficients.  In memory, and read where they are used: as numbers of the code a loop
// over rows keeps all of them in registers that its pieces need.
__constant__ double EXP_SERIES[12] = {1.0 / 6227020800.0, 1.0 / 479001600.0, 1.0 / 39916800.0, 1.0 / 3628800.0,
                                      1.0 / 362880.0,     1.0 / 40320.0,     1.0 / 5040.0,     1.0 / 720.0,
                                      1.0 / 120.0,        1.0 / 24.0,        1.0 / 6.0,        0.5};
__constant__ double ATANH_SERIES[16] = {1.0 / 33.0, 1.0 / 31.0, 1.0 / 29.0, 1.0 / 27.0, 1.0 / 25.0, 1.0 / 23.0,
                                        1.0 / 21.0, 1.0 / 19.0, 1.0 / 17.0, 1.0 / 15.0, 1.0 / 13.0, 1.0 / 11.0,
                                        1.0 / 9.0,  1.0 / 7.0,  1.0 / 5.0,  1.0 / 3.0};
template <int N>
__device__ __forceinline__ double series(const double* c, double x) {
  asm volatile("" : "+s"(c));
  double s = c[0];
#pragma unroll
  for (int i = 1; i < N; ++i) s = fma(s, x, c[i]);
  return s;
}

// e^x - 1: x = n ln 2 + r with |r| <= ln 2 / 2, 2^n (e^r - 1) + (2^n - 1), e^r - 1 by its series
// to r^13 (the next term is below 2^-57 of r).  `one`: e^x instead.  n ln 2 is taken off by Cody and
// Waite's two steps: the first part of ln 2 is its first 32 bits, whose product with n is exact (the
// split that the public fdlibm has too).
__device__ __forceinline__ double exp_less(double x, bool one) {
  const double n = rint(fmin(fmax(x, -800.0), 800.0) * 1.442695040888963407360);
  const double r = fma(-n, 1.90821492927058770002e-10, fma(-n, 6.93147180369123816490e-01, x));
  const double s = fma(series<12>(EXP_SERIES, r) * r, r, r);
  const int k = (int)n;
  const double y = ldexp(s, k), z = ldexp(1.0, k);
  const double v = one ? y + z : y + (z - 1.0);
  return x > 709.0 ? INFINITY : x < -750.0 ? (one ? 0.0 : -1.0) : x != x ? x : v;
}
// log(a / b) for 0.5 <= a / b <= 2: 2 atanh(s), s = (a - b) / (a + b), |s| <= 1/3, by its series
// to s^33 (the next term is below 2^-57 of s).  less: a - b.
__device__ __forceinline__ double log_ratio(double less, double sum) {
  const double s = less / sum, z = s * s;
  return 2.0 * fma(series<16>(ATANH_SERIES, z) * z, s, s);
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

// Factors above this stay apart from their power of two: a factor near fp32's largest, or past it,
// times a 2^t that is 0 in fp32 may be any number.  (Of those up to here such products are below
// 2^-122.)
constexpr double MOST_MUL = 16.0;
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
  const double factor = none ? 0.0 : -slope / all;
  g.more = 0.0f;
  if (fabs(factor) > MOST_MUL) {
    const bool finite = fabs(factor) < INFINITY;
    const int k = finite ? ilogb(factor) : 1;
    g.more = (float)k;
    g.mul = (float)(finite ? ldexp(factor, -k) : factor);
  } else {
    g.mul = (float)(factor * (1.0 - c_rounding_less(p, g.base)));
  }
  // what has no probability has no gradient, also where the slope is infinite
  g.at_tok = not_t == 0.0 && slope == slope ? 0.0f : (float)(slope * not_t);
  g.tok = in && w != 0.0f ? r.tok : -1;
  return g;
}

// Whether a row's gradients take their exponents by its C, which its factor then allows for.
__device__ __forceinline__ bool plain_grads(const RowGrad& g, float cm) { return by_c(cm) && g.more == 0.0f; }
// Gradients of a piece's entries but for the token's.
template <typename T>
__device__ __forceinline__ void grads_of(const PolicyParams& p, const RowGrad& g, float cm, bool plain, const Piece<T>& x,
                                         float (&y)[Piece<T>::N]) {
  if (plain) {
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j) y[j] = g.mul * __builtin_amdgcn_exp2f(fmaf(x.value(j), p.c, -cm));
  } else {
#pragma unroll
    for (int j = 0; j < Piece<T>::N; ++j) {
      const float t = scaled_difference(x.value(j), g.base, p.c, -g.more);
      // by an infinite slope: of probabilities that fp64 holds
      y[j] = fabsf(g.mul) == INFINITY ? t < -1074.0f ? 0.0f : g.mul : g.mul * __builtin_amdgcn_exp2f(t);
    }
  }
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
  const double rest = sum64_over_wave(sum);
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
  v = sum64_over_wave(v);
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
  const bool plain = __all(plain_grads(g, cm));
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = begin + i * STEP + t * VEC;
    float y[VEC];
    grads_of(p, g, cm, plain, v[i], y);
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
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

// A thread's piece of entries `at` ..: where it crosses the row's end, entries from further left
// that others hold too.  First entry of what it holds.
template <typename T>
__device__ __forceinline__ int load_piece(const T* z, int at, int vocab, Piece<T>& v) {
  const int from = min(at, vocab - Piece<T>::N);
  v.load(z + from);
  return from;
}
// Keeps the compiler from holding the pieces' values of an earlier use, four times their registers.
template <typename T>
__device__ __forceinline__ void anew(Piece<T>& v) {
  asm volatile("" : "+v"(v.w));
}

// A number that the compiler takes for another one than before, so that nothing made of it is kept
// from piece to piece, in registers that the pieces need.
__device__ __forceinline__ int number_anew(int n) {
  n = __builtin_amdgcn_readfirstlane(n);
  asm volatile("" : "+s"(n));
  return n;
}
__device__ __forceinline__ int thread_anew() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// A thread's largest logit and sum of the entries it has seen: fp32 over a piece, then over the
// pieces of a call of see(): equal entries, added one by one, round one way (that took 151 us,
// not 154, for 1024 rows of 151936 bf16 logits).
struct Seen {
  float m = -INFINITY;
  double l = 0.0;
};
// U more pieces, the i-th at i STEP + t VEC of the `left` entries that the row has from there on.
// The first FULL of them are whole, those past the row's end not looked at.
template <typename T, int NT, int U, int FULL>
__device__ __forceinline__ void see(const PolicyParams& p, Piece<T> (&v)[U], int left, int tok, Seen& s) {
  constexpr int VEC = Piece<T>::N, STEP = NT * VEC;
  const int t = thread_anew();
  left = number_anew(left);
  // of a piece that crosses the row's end the first `skip` entries are others'
  const auto skip_of = [&](int i) { return max(i * STEP + t * VEC - (left - VEC), 0); };
  float most = s.m;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (i >= FULL && i * STEP >= left) continue;
    if (i < FULL || (i + 1) * STEP <= left) {
#pragma unroll
      for (int j = 0; j < VEC; ++j) most = fmaxf(most, v[i].value(j));
    } else {
      const int skip = skip_of(i);
#pragma unroll
      for (int j = 0; j < VEC; ++j) most = fmaxf(most, j >= skip ? v[i].value(j) : -INFINITY);
    }
  }
  const float base = base_of(most), cm = c_of(base, p.c);
  if (most > s.m) {
    // by the two C; where not both count, by the logits and the rounding of the one that does
    const float was = c_of(base_of(s.m), p.c), off = by_c(was) ? -fmaf(base_of(s.m), p.c, -was) : fmaf(base, p.c, -cm);
    const float x = by_c(cm) == by_c(was) ? by_c(cm) ? was - cm : (s.m - most) * p.c : fmaf(s.m - most, p.c, off);
    s.l = s.l == 0.0 ? 0.0 : s.l * __builtin_amdgcn_exp2f(x);
    s.m = most;
  }
  // the token's entry (of the pieces from the first on, negative: none) stays out of the sum
  const bool by = __all(by_c(cm));
  float l = 0.0f;
  left = number_anew(left);
  tok = number_anew(tok);
#pragma unroll
  for (int i = 0; i < U; ++i) anew(v[i]);
#pragma unroll
  for (int i = 0; i < U; ++i) {
    if (i >= FULL && i * STEP >= left) continue;
    if ((i < FULL || (i + 1) * STEP <= left) && (uint32_t)(tok - i * STEP) >= (uint32_t)STEP && by) {
      float sum = __builtin_amdgcn_exp2f(fmaf(v[i].value(0), p.c, -cm));
#pragma unroll
      for (int j = 1; j < VEC; ++j) sum += __builtin_amdgcn_exp2f(fmaf(v[i].value(j), p.c, -cm));
      l += sum;
    } else {
      float sum = 0.0f;
      const int skip = skip_of(i), own = tok - i * STEP - t * VEC + skip;
#pragma unroll
      for (int j = 0; j < VEC; ++j) {
        const float z = v[i].value(j);
        const float e = __builtin_amdgcn_exp2f(by_c(cm) ? fmaf(z, p.c, -cm) : (z - base) * p.c);
        sum += j >= skip && !(tok >= 0 && j == own) ? e : 0.0f;
      }
      l += sum;
    }
  }
  s.l += l;
#pragma unroll
  for (int i = 0; i < U; ++i) anew(v[i]);
}

// Gradients of a thread's piece of a row that is not left out; the token's own entry is put
// afterwards.
template <typename T>
__device__ __forceinline__ void put_grad(const PolicyParams& p, const RowGrad& g, float cm, bool plain, const Piece<T>& v,
                                         T* out, int at) {
  constexpr int VEC = Piece<T>::N;
  Piece<T> x = v;
  anew(x);
  float y[VEC];
  grads_of(p, g, cm, plain, x, y);
  if (at + VEC <= p.vocab) {
    x.put(y);
    x.store_past(out + at);
  } else {
    const int from = p.vocab - VEC;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
      if (from + j >= at) put_entry(out + from + j, y[j]);
  }
}

// The threads' sums of a row, joined: what its gradient takes, in every thread.
template <int NT>
struct JoinScratch {
  float most[NT / 64], sum[NT / 64];
  RowGrad grad;
};
template <int NT>
__device__ __forceinline__ RowGrad join_row(const PolicyParams& p, int64_t row, const RowIn& in, const Seen& s,
                                            JoinScratch<NT>& scratch) {
  constexpr int WAVES = NT / 64;
  const int t = threadIdx.x;
  const float wave_most = max_over_wave(s.m);
  const float wave_sum = (float)sum64_over_wave(joined(p, s.m, (float)s.l, wave_most));
  if ((t & 63) == 0) {
    scratch.most[t >> 6] = wave_most;
    scratch.sum[t >> 6] = wave_sum;
  }
  __syncthreads();
  if (t < 64) {
    const int i = min(t, WAVES - 1);
    const float most = max_over_wave(scratch.most[i]);
    // a wave's sum has no rounded C in it
    const double x = ((double)base_of(scratch.most[i]) - base_of(most)) * ((double)p.c + p.c_rest);
    double sum = t < WAVES && scratch.sum[i] != 0.0f ? scratch.sum[i] * exp_less(x * 6.93147180559945309417e-01, true) : 0.0;
#pragma unroll
    for (int o = WAVES / 2; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if (t == 0) scratch.grad = finish_row(p, row, in, most, sum);
  }
  __syncthreads();
  return scratch.grad;
}

// A row of zeros.
template <typename T, int NT>
__device__ __forceinline__ void put_zeros(const PolicyParams& p, T* out) {
  constexpr int VEC = Piece<T>::N;
  const Piece<T> zero{};
#pragma unroll 1
  for (int at = threadIdx.x * VEC; at < p.vocab; at += NT * VEC) {
    if (at + VEC <= p.vocab) zero.store_past(out + at);
    else
      for (int j = at; j < p.vocab; ++j) put_entry(out + j, 0.0f);
  }
}

// Short rows, of at most NT 32 entries: a workgroup a row, in its registers.  bf16 rows of the
// larger workgroups take 64 registers, for two of 1024 threads to a CU: 1024 rows of 32000 with
// gradient 35.1 us, of 86 registers 41.9.  fp32 rows would spill (256 rows of 32000: 19.9 and
// 17.3 us).
template <typename T, int NT>
__global__ __launch_bounds__(NT, sizeof(T) == 2 && NT > 256 ? 8 : 4) void policy_short_kernel(PolicyParams p) {
  constexpr int VEC = Piece<T>::N, U = 32 / VEC, STEP = NT * VEC;
  __shared__ JoinScratch<NT> scratch;
  const int t = threadIdx.x;
  const int64_t row = blockIdx.x;
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int tok = p.tokens[row];
  Piece<T> v[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int at = i * STEP + t * VEC;
    if (i * STEP >= p.vocab) continue;
    if (p.vocab >= VEC) {
      load_piece(z, at, p.vocab, v[i]);
    } else {  // in the place that entries from further left would have
      v[i] = Piece<T>{};
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[i].set(j, p.vocab - VEC + j >= 0 ? Elem<T>::load(z, p.vocab - VEC + j) : -INFINITY);
    }
  }
  const RowIn in = row_in<T>(p, row, tok);
  Seen s;
  see<T, NT, U, 0>(p, v, p.vocab, tok, s);
  const RowGrad g = join_row<NT>(p, row, in, s, scratch);
  if (!p.grad) return;
  T* out = reinterpret_cast<T*>(p.grad + row * p.grad_stride);
  if (g.tok < 0) return put_zeros<T, NT>(p, out);
  const float cm = c_of(g.base, p.c);
  const bool plain = __all(plain_grads(g, cm));
#pragma unroll
  for (int i = 0; i < U; ++i)
    if (i * STEP < p.vocab) put_grad(p, g, cm, plain, v[i], out, i * STEP + t * VEC);
  if (g.tok % STEP / VEC == t) put_entry(out + g.tok, g.at_tok);  // after the thread's own store there
}

// Losses of long rows alone: a workgroup a row, which its threads go through with the next four
// pieces on their way.
template <typename T>
__global__ __launch_bounds__(512, 4) void policy_losses_kernel(PolicyParams p) {
  constexpr int NT = 512, VEC = Piece<T>::N, STEP = NT * VEC, U = 4, TURN = U * STEP;
  __shared__ JoinScratch<NT> scratch;
  const int64_t row = blockIdx.x;
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int tok = p.tokens[row];
  Piece<T> v[U], w[U];
  const auto load = [&](int begin, Piece<T>(&x)[U]) {
    const int t = thread_anew();
#pragma unroll
    for (int i = 0; i < U; ++i) load_piece(z, min(begin, p.vocab) + i * STEP + t * VEC, p.vocab, x[i]);
  };
  const auto look = [&](int begin, Piece<T>(&x)[U], Seen& s) {
    see<T, NT, U, 0>(p, x, p.vocab - begin, tok >= begin ? tok - begin : -1, s);
  };
  load(0, v);
  const RowIn in = row_in<T>(p, row, tok);
  Seen s;
#pragma unroll 1
  for (int begin = 0; begin < p.vocab; begin += 2 * TURN) {
    load(begin + TURN, w);
    look(begin, v, s);
    load(begin + 2 * TURN, v);
    if (begin + TURN < p.vocab) look(begin + TURN, w, s);
  }
  join_row<NT>(p, row, in, s, scratch);
}

// Long rows with their gradient: a workgroup of 1024 threads to a row, H pieces of a thread in its
// registers, of which the last four may lie past the row's end, and what is further right read
// twice.  As pieces go out, those of the workgroup's next row come in.  Of 38 us a row of 151936
// bf16 logits (19 pieces held), sums took 13, the join 10 (it waits for the slowest of 16 waves),
// gradients 15.
// Read twice, whole, by 256 to 1024 threads: 162 to 182 us, not 154, for 1024 such rows.
template <typename T, int H>
__global__ __launch_bounds__(1024, 4) void policy_rows_kernel(PolicyParams p) {
  constexpr int NT = 1024, VEC = Piece<T>::N, STEP = NT * VEC, U = 4, TURN = U * STEP, FULL = H - 4;
  __shared__ JoinScratch<NT> scratch;
  const auto row_of = [&](int64_t row) { return reinterpret_cast<const T*>(p.logits + row * p.stride); };
  Piece<T> v[H];
  int64_t row = blockIdx.x;
  int tok = p.tokens[row];
#pragma unroll
  for (int i = 0; i < H; ++i) load_piece(row_of(row), i * STEP + (int)threadIdx.x * VEC, p.vocab, v[i]);
#pragma unroll 1
  for (; row < p.rows; row += gridDim.x) {
    const RowIn in = row_in<T>(p, row, tok);
    const T* z = row_of(row);
    Seen s;
    see<T, NT, H, FULL>(p, v, p.vocab, tok, s);
#pragma unroll 1
    for (int begin = H * STEP; begin < p.vocab; begin += TURN) {
      Piece<T> w[U];
      const int t = thread_anew();
#pragma unroll
      for (int i = 0; i < U; ++i) load_piece(z, begin + i * STEP + t * VEC, p.vocab, w[i]);
      see<T, NT, U, 0>(p, w, p.vocab - begin, tok >= begin ? tok - begin : -1, s);
    }
    const RowGrad g = join_row<NT>(p, row, in, s, scratch);
    T* out = reinterpret_cast<T*>(p.grad + row * p.grad_stride);
    const float cm = c_of(g.base, p.c);
    const bool plain = __all(plain_grads(g, cm)), more = row + gridDim.x < p.rows, kept = __any(g.tok >= 0);
    const T* next = row_of(more ? row + gridDim.x : row);
    tok = p.tokens[more ? row + gridDim.x : row];
    if (!kept) put_zeros<T, NT>(p, out);
    const int t = thread_anew(), vocab = number_anew(p.vocab);
#pragma unroll
    for (int i = 0; i < H; ++i) {
      if (kept && (i < FULL || i * STEP < vocab)) put_grad(p, g, cm, plain, v[i], out, i * STEP + t * VEC);
      // after the last row one piece again and again, which is in the cache
      load_piece(next, more ? i * STEP + t * VEC : t * VEC, vocab, v[i]);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!kept) continue;
#pragma unroll 1
    for (int begin = H * STEP; begin < p.vocab; begin += TURN) {
      Piece<T> w[U];
      const int t = thread_anew();
#pragma unroll
      for (int i = 0; i < U; ++i) load_piece(z, begin + i * STEP + t * VEC, p.vocab, w[i]);
#pragma unroll
      for (int i = 0; i < U; ++i)
        if (begin + i * STEP < p.vocab) put_grad(p, g, cm, plain, w[i], out, begin + i * STEP + t * VEC);
    }
    if (g.tok % STEP / VEC == (int)threadIdx.x) put_entry(out + g.tok, g.at_tok);  // after the thread's own store there
  }
}

int chunks_of(int vocab) { return (vocab + PL_CHUNK - 1) / PL_CHUNK; }

// With their gradient, rows from which on each is given to one workgroup.  In us, so and by
// chunks: of 65536 bf16 logits 96 rows 17.5 and 17.2, 128 rows 18.2 and 19.1, 256 rows 21.1 and
// 26.1; of 152064 128 rows 28.6 and 28.8, 160 rows 31.7 and 34.1; of 128256 fp32 logits 96 rows
// 32.1 and 31.0, 128 rows 35.5 and 43.5.
constexpr int WHOLE_ROWS = 128, CUS = 256;
// Losses alone of middling rows go by chunks above this many: of 18000 bf16 logits, whole and by
// chunks, 512 rows 15.2 and 15.5 us, 1024 rows 23.9 and 19.2.
constexpr int WHOLE_LOSSES = 512;
// Losses of longer rows: a row to a CU, so and by chunks, of 65536 bf16 logits 16 rows 12.1 and 13.8,
// 256 rows 13.5 and 18.4; of 128256 64 rows 17.5 and 15.4, 128 rows 17.8 and 17.4, 256 rows 18.6 and
// 22.3, but 384, of which a CU has two, 34.4 and 30.8; of 152064 fp32 logits 128 rows 23.0 and 22.0,
// 192 rows 28.0 and 30.0.
template <typename T>
void launch(const PolicyParams& p, hipStream_t s) {
  constexpr int VEC = Piece<T>::N;
  const dim3 nt(PL_NT);
  bool total = p.total;
  const auto whole = [&](auto n) {
    constexpr int NT = decltype(n)::value;
    hipLaunchKernelGGL((policy_short_kernel<T, NT>), dim3((unsigned)p.rows), dim3(NT), 0, s, p);
  };
  if (p.vocab <= 256 * 32) {
    whole(std::integral_constant<int, 256>{});
  } else if (p.vocab <= 512 * 32) {
    whole(std::integral_constant<int, 512>{});
  } else if (p.vocab <= 1024 * 32 && (p.grad || p.rows <= WHOLE_LOSSES)) {
    whole(std::integral_constant<int, 1024>{});
  } else if (!p.grad && p.rows <= CUS && (p.vocab <= 65536 || p.rows >= WHOLE_ROWS)) {
    hipLaunchKernelGGL((policy_losses_kernel<T>), dim3((unsigned)p.rows), dim3(512), 0, s, p);
  } else if (p.grad && p.rows >= WHOLE_ROWS) {
    const dim3 grid((unsigned)std::min<int64_t>(p.rows, CUS));
    const int pieces = (p.vocab + 1024 * VEC - 1) / (1024 * VEC);  // more than 32 / VEC
    const auto go = [&](auto h) {
      hipLaunchKernelGGL((policy_rows_kernel<T, decltype(h)::value>), grid, dim3(1024), 0, s, p);
    };
    // 16 at most, which fill a thread's 128 registers: with 16, 17, 19 and 20 held (those spill) 1024
    // rows of 151936 bf16 logits take 151, 154, 154 and 159 us, of 200000 194, 196, 204 and 210; 250
    // rows of 152064 fp32 ones with 16, 18 and 20 67.4, 68.3 and 70.8
    constexpr int LEAST = VEC == 8 ? 8 : 12;
    if (pieces <= LEAST) go(std::integral_constant<int, LEAST>{});
    else if (pieces <= 12) go(std::integral_constant<int, 12>{});
    else go(std::integral_constant<int, 16>{});
  } else {
    const dim3 grid((unsigned)(p.rows * p.chunks));
    hipLaunchKernelGGL((policy_chunk_kernel<T>), grid, nt, 0, s, p);
    hipLaunchKernelGGL((policy_row_kernel<T>), dim3((unsigned)((p.rows + PL_NT / 64 - 1) / (PL_NT / 64))), nt, 0, s, p);
    if (p.grad) {
      hipLaunchKernelGGL((policy_grad_kernel<T>), grid, nt, 0, s, p);
      total = false;
    }
  }
  if (total) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(TOTAL_NT), 0, s, p);
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
  p.row_loss = static_cast<double*>(workspace);
  p.stats = reinterpret_cast<float2*>(p.row_loss + rows);
  p.row_grad = reinterpret_cast<RowGrad*>(p.stats + rows * p.chunks);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (rows == 0) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(TOTAL_NT), 0, s, p);
  else if (dtype == KV_BF16) launch<bf16_t>(p, s);
  else launch<float>(p, s);
  return launched();
}

}  // extern "C"

// The clipped policy loss and the gradient of its logits (kvr_policy.h).
//
// With t_v = c (z_v - m) as in logits.h, e_v = 2^t_v, rest = sum over v != t of e_v and
// mine = e_t:
//   lp = -log1p(rest / mine),   p_v = e_v / (rest + mine),   1 - p_t = rest / (rest + mine)
// The token's own term stays out of the sum: for a token that is all but certain, what is
// left of 1 - p_t in a sum with its 1 is noise.  The gradient is one factor of the row times
// e_v, but for the token's entry.
//
// A row is cut into chunks; a workgroup reads its chunk once, into registers, and leaves its
// largest logit and sum.  A wave merges the chunks of a row in a fixed order, in fp64 as all
// that is done once a row.  A third kernel turns logits into gradients.
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

// What a chunk's t_v leave out, in log2 units: the rounding of its C.
__device__ __forceinline__ double c_rounding(const PolicyParams& p, float base) {
  const float cm = c_of(base, p.c);
  return by_c(cm) ? (double)base * p.c - cm : 0.0;
}

// A row's results from its largest logit m, the others' sum `rest` and the token's logit z;
// rest is relative to m, in exact units.
__device__ __forceinline__ void finish_row(const PolicyParams& p, int64_t row, int tok, float m, double rest, float z) {
  const double scale = p.scale, base = base_of(m);
  const float w = p.weights ? p.weights[row] : 1.0f;
  const bool in = tok >= 0 && tok < p.vocab;
  double lp = 0.0, kl = 0.0, loss = 0.0, slope = 0.0, not_t = 0.0, all = 1.0;
  bool none = true;
  if (in) {
    const double x = scale * ((double)z - base), mine = exp(x);
    all = rest + mine;
    none = all == 0.0;  // every logit is -infinity
    lp = none ? -INFINITY : rest < mine ? -log1p(rest / mine) : x - log(all);
    not_t = none ? 1.0 : rest / all;
  }
  if (in && w != 0.0f) {
    const double a = p.advantages[row];
    const double rho = p.old ? exp(lp - p.old[row]) : lp != lp ? lp : 1.0;
    const double plain = rho * a, cut = fmin(fmax(rho, p.low), p.high) * a;
    const bool kept = !(plain > cut);
    double fall = 0.0;
    if (p.ref) {
      const double d = p.ref[row] - lp, e = expm1(d);
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
  if (p.grad) {
    RowGrad g;
    g.base = (float)base;
    g.mul = none ? 0.0f : (float)(-slope / all * exp2(-c_rounding(p, g.base)));
    g.at_tok = (float)(slope * not_t);
    g.tok = in && w != 0.0f ? tok : -1;
    p.row_grad[row] = g;
  }
}

// A wave a row.
template <typename T>
__global__ __launch_bounds__(PL_NT) void policy_row_kernel(PolicyParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * (PL_NT / 64) + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  const int tok = p.tokens[row];
  const float z = tok >= 0 && tok < p.vocab ? Elem<T>::load(reinterpret_cast<const T*>(p.logits + row * p.stride), tok)
                                            : 0.0f;
  const float2* stats = p.stats + row * p.chunks;
  float m = -INFINITY;
  for (int i = lane; i < p.chunks; i += 64) m = fmaxf(m, stats[i].x);
  m = max_over_wave(m);
  double rest = 0.0;
  for (int i = lane; i < p.chunks; i += 64) {
    const float2 q = stats[i];
    const double b = base_of(q.x), x = (b - base_of(m)) * ((double)p.c + p.c_rest);
    rest += q.y == 0.0f ? 0.0 : q.y * exp2(x - c_rounding(p, q.x));
  }
  rest = sum_over_wave(rest);
  if (lane == 0) finish_row(p, row, tok, m, rest, z);
}

// The rows' losses, a workgroup's threads in turn.
__device__ __forceinline__ void put_total(const PolicyParams& p) {
  __shared__ double s_sum[PL_NT / 64];
  double v = 0.0;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < p.rows; i += PL_NT) v += p.row_loss[i];
  v = sum_over_wave(v);
  if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = v;
  __syncthreads();
  if (threadIdx.x == 0) {
    v = s_sum[0];
#pragma unroll
    for (int i = 1; i < PL_NT / 64; ++i) v += s_sum[i];
    *p.total = (float)v;
  }
}
__global__ __launch_bounds__(PL_NT) void policy_total_kernel(PolicyParams p) { put_total(p); }

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
  if (p.total && blockIdx.x == 0) put_total(p);
}

int chunks_of(int vocab) { return (vocab + PL_CHUNK - 1) / PL_CHUNK; }

template <typename T>
void launch(const PolicyParams& p, hipStream_t s) {
  const dim3 grid((unsigned)(p.rows * p.chunks)), nt(PL_NT);
  hipLaunchKernelGGL((policy_chunk_kernel<T>), grid, nt, 0, s, p);
  hipLaunchKernelGGL((policy_row_kernel<T>), dim3((unsigned)((p.rows + PL_NT / 64 - 1) / (PL_NT / 64))), nt, 0, s, p);
  if (p.grad) hipLaunchKernelGGL((policy_grad_kernel<T>), grid, nt, 0, s, p);
  else if (p.total) hipLaunchKernelGGL(policy_total_kernel, dim3(1), nt, 0, s, p);
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
  if (rows == 0) hipLaunchKernelGGL(policy_total_kernel, dim3(1), dim3(PL_NT), 0, s, p);
  else if (dtype == KV_BF16) launch<bf16_t>(p, s);
  else launch<float>(p, s);
  return launched();
}

}  // extern "C"

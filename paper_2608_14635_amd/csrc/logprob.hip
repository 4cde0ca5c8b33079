// Log probabilities of given tokens, entropy and likeliest tokens (kvr_logprob.h).
//
// With m the largest logit of a row, e_v = exp(scale (z_v - m)), l = sum e_v and
// s = sum (z_v - m) e_v:
//   log p_t = scale (z_t - m) - log l,   entropy = log l - scale s / l
// (both terms of the entropy are of one sign, so nothing cancels).  A row is cut into
// chunks; a workgroup reads its chunk once, into registers, takes the chunk's m, l and
// s from there and, where asked, its top_n entries; a second kernel merges the
// chunks of each row in a fixed order.
//
// Top entries.  (value, lower index first) is one 64-bit key, so that all keys of a
// row differ and the order is total.  The top_n-th largest of the 256 threads' own
// largest keys is a bound that at least top_n entries reach, and only entries of
// top_n threads can: those are collected in LDS (a few more than top_n as a rule, at
// most top_n * ITEMS) and ranked by counting.
//
// Bound by HBM where rows are many (4 or 2 bytes a logit against one exp and some
// eight other operations), by latency where they are few.
#include <algorithm>

#include "common.h"
#include "host.h"
#include "kvr_logprob.h"

namespace kvr {
namespace {

constexpr int LP_NT = 256;
constexpr float LOG2E = 1.4426950408889634f;
constexpr int LP_MAX_VOCAB = 1 << 22;
constexpr int LP_KEYS = 4096;  // collected keys: top_n * ITEMS, and top_n * chunks * top_n / 256, at most

struct LogprobParams {
  const char* logits;
  int64_t stride;  // bytes
  int vocab, chunks, top;
  float scale;
  const int32_t* tokens;
  float* logprobs;
  float* entropy;
  float* top_logprobs;
  int32_t* top_tokens;
  float4* stats;   // [rows][chunks] m, l, s
  uint64_t* keys;  // [rows][chunks][top]
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_a2 __attribute__((aligned(2)));

// 16 bytes of logits as values, from any boundary of their elements
__device__ __forceinline__ void get_vec(const float* p, float* v) {
  const f32x4 a = *reinterpret_cast<const f32x4_a4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = a[i];
}
__device__ __forceinline__ void get_vec(const bf16_t* p, float* v) {
  const u32x4 u = *reinterpret_cast<const u32x4_a2*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(u[i] << 16);
    v[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}

// Unsigned numbers that order as the values do; -0 as +0, NaN below all.
__device__ __forceinline__ uint32_t order_bits(float z) {
  const uint32_t b = __float_as_uint(z + 0.0f);
  return z != z ? 0u : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float ordered_value(uint32_t u) {
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ __forceinline__ uint64_t make_key(uint32_t order, uint32_t index) {
  return (uint64_t)order << 32 | (0xffffffffu - index);
}
__device__ __forceinline__ uint32_t key_index(uint64_t k) { return 0xffffffffu - (uint32_t)k; }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
  return v;
}

// Ranks by counting: how many of the n keys in LDS are larger.
__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t* keys, int n) {
  int r = 0;
  for (int i = 0; i < n; ++i) r += keys[i] > key;
  return r;
}

struct TopScratch {
  uint64_t keys[LP_KEYS];
  uint64_t own[LP_NT];
  uint64_t bound;
  int count;
};

// The bound: the top-th largest of the threads' own largest keys.
__device__ __forceinline__ uint64_t top_bound(uint64_t own, int top, TopScratch& s) {
  const int t = threadIdx.x;
  s.own[t] = own;
  if (t == 0) s.count = 0;
  __syncthreads();
  if (rank_of(own, s.own, LP_NT) == top - 1) s.bound = own;
  __syncthreads();
  return s.bound;
}
__device__ __forceinline__ void collect(uint64_t key, TopScratch& s) {
  const int at = atomicAdd(&s.count, 1);  // any order: the ranks settle it
  if (at < LP_KEYS) s.keys[at] = key;
}

template <typename T, int ITEMS>
__global__ __launch_bounds__(LP_NT) void logprob_chunk_kernel(LogprobParams p) {
  constexpr int VEC = 16 / (int)sizeof(T), VECS = ITEMS / VEC;
  __shared__ float s_red[3][LP_NT / 64];
  __shared__ TopScratch s_top;
  const int t = threadIdx.x, w = t >> 6, lane = t & 63;
  const int c = blockIdx.x % p.chunks;
  const int64_t row = blockIdx.x / p.chunks;
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int first = c * (LP_NT * ITEMS) + t * VEC;
  float v[ITEMS];
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    const int at = first + i * (LP_NT * VEC);
    if (at + VEC <= p.vocab) {
      get_vec(z + at, v + i * VEC);
    } else {
#pragma unroll
      for (int j = 0; j < VEC; ++j) v[i * VEC + j] = at + j < p.vocab ? Elem<T>::load(z, at + j) : -INFINITY;
    }
  }
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) m = fmaxf(m, v[i]);
  m = wave_max(m);
  if (lane == 0) s_red[0][w] = m;
  __syncthreads();
  m = s_red[0][0];
#pragma unroll
  for (int i = 1; i < LP_NT / 64; ++i) m = fmaxf(m, s_red[0][i]);
  // nothing but -infinity (or NaN): sums of zeros (or NaN)
  const float base = m == -INFINITY ? 0.0f : m, scale2 = p.scale * LOG2E;
  float l = 0.0f, s = 0.0f;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const float x = v[i] - base, e = __builtin_amdgcn_exp2f(x * scale2);
    l += e;
    s += e == 0.0f ? 0.0f : x * e;
  }
  l = wave_sum(l);
  s = wave_sum(s);
  if (lane == 0) {
    s_red[1][w] = l;
    s_red[2][w] = s;
  }
  __syncthreads();
  if (t == 0) {
    l = s = 0.0f;
    for (int i = 0; i < LP_NT / 64; ++i) {
      l += s_red[1][i];
      s += s_red[2][i];
    }
    p.stats[row * p.chunks + c] = make_float4(m, l, s, 0.0f);
  }
  if (p.top == 0) return;
  // entries past the vocabulary order as NaN of higher indices: below all others
  uint64_t own = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int at = first + i / VEC * (LP_NT * VEC) + i % VEC;
    const uint64_t k = make_key(at < p.vocab ? order_bits(v[i]) : 0u, at);
    own = k > own ? k : own;
  }
  const uint64_t bound = top_bound(own, p.top, s_top);
  if (own >= bound) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int at = first + i / VEC * (LP_NT * VEC) + i % VEC;
      const uint64_t k = make_key(at < p.vocab ? order_bits(v[i]) : 0u, at);
      if (k >= bound) collect(k, s_top);
    }
  }
  __syncthreads();
  const int n = min(s_top.count, LP_KEYS);
  uint64_t* out = p.keys + (row * p.chunks + c) * p.top;
  for (int i = t; i < n; i += LP_NT) {
    const int r = rank_of(s_top.keys[i], s_top.keys, n);
    if (r < p.top) out[r] = s_top.keys[i];
  }
}

template <typename T>
__global__ __launch_bounds__(LP_NT) void logprob_row_kernel(LogprobParams p) {
  __shared__ float s_red[3][LP_NT / 64];
  __shared__ TopScratch s_top;
  const int t = threadIdx.x, w = t >> 6, lane = t & 63;
  const int64_t row = blockIdx.x;
  const float4* stats = p.stats + row * p.chunks;
  float m = -INFINITY;
  for (int c = t; c < p.chunks; c += LP_NT) m = fmaxf(m, stats[c].x);
  m = wave_max(m);
  if (lane == 0) s_red[0][w] = m;
  __syncthreads();
  m = s_red[0][0];
#pragma unroll
  for (int i = 1; i < LP_NT / 64; ++i) m = fmaxf(m, s_red[0][i]);
  const float scale2 = p.scale * LOG2E;
  float l = 0.0f, s = 0.0f;
  for (int c = t; c < p.chunks; c += LP_NT) {
    // a chunk of -infinity alone adds l = s = 0 (or its NaN)
    const float4 q = stats[c];
    const float x = q.x == -INFINITY ? 0.0f : q.x - m, e = __builtin_amdgcn_exp2f(x * scale2);
    l = fmaf(q.y, e, l);
    s += e == 0.0f ? 0.0f * q.z : e * fmaf(x, q.y, q.z);
  }
  l = wave_sum(l);
  s = wave_sum(s);
  if (lane == 0) {
    s_red[1][w] = l;
    s_red[2][w] = s;
  }
  __syncthreads();
  l = s = 0.0f;
#pragma unroll
  for (int i = 0; i < LP_NT / 64; ++i) {
    l += s_red[1][i];
    s += s_red[2][i];
  }
  const bool none = l == 0.0f;  // every logit -infinity
  const float log_l = none ? 0.0f : logf(l);
  auto logprob = [&](float z) { return none ? -INFINITY : (z - m) * p.scale - log_l; };
  if (t == 0) {
    if (p.logprobs) {
      const int tok = p.tokens[row];
      float lp = tok < 0 ? 0.0f : l != l ? l : -INFINITY;
      if (tok >= 0 && tok < p.vocab)
        lp = logprob(Elem<T>::load(reinterpret_cast<const T*>(p.logits + row * p.stride), tok));
      p.logprobs[row] = lp;
    }
    if (p.entropy) {
      const float h = log_l - p.scale * s / l;
      p.entropy[row] = none || h < 0.0f ? 0.0f : h;  // NaN stays
    }
  }
  if (p.top == 0) return;
  const uint64_t* keys = p.keys + row * p.chunks * p.top;
  const int total = p.chunks * p.top;
  uint64_t own = t;  // threads without a key: below all of them, and different
  for (int i = t; i < total; i += LP_NT) own = max(own, keys[i]);
  const uint64_t bound = top_bound(own, p.top, s_top);
  if (own >= bound)
    for (int i = t; i < total; i += LP_NT)
      if (keys[i] >= bound) collect(keys[i], s_top);
  __syncthreads();
  const int n = min(s_top.count, LP_KEYS);
  for (int i = t; i < n; i += LP_NT) {
    const uint64_t k = s_top.keys[i];
    const int r = rank_of(k, s_top.keys, n);
    if (r < p.top) {
      p.top_tokens[row * p.top + r] = (int32_t)key_index(k);
      p.top_logprobs[row * p.top + r] = logprob(ordered_value((uint32_t)(k >> 32)));
    }
  }
}

// Entries a thread takes: 64 where rows are many (a workgroup's 64 KB of fp32 in
// flight), 16 where they would leave CUs idle.
int items_of(int64_t rows, int vocab) {
  const int64_t wide = (vocab + LP_NT * 64 - 1) / (LP_NT * 64);
  return rows * wide >= 512 || vocab > LP_NT * 16 * 256 ? 64 : 16;
}
int chunks_of(int items, int vocab) { return (vocab + LP_NT * items - 1) / (LP_NT * items); }

template <typename T>
void launch(const LogprobParams& p, int64_t rows, int items, hipStream_t s) {
  const dim3 grid((unsigned)(rows * p.chunks));
  if (items == 64)
    hipLaunchKernelGGL((logprob_chunk_kernel<T, 64>), grid, dim3(LP_NT), 0, s, p);
  else
    hipLaunchKernelGGL((logprob_chunk_kernel<T, 16>), grid, dim3(LP_NT), 0, s, p);
  hipLaunchKernelGGL(logprob_row_kernel<T>, dim3((unsigned)rows), dim3(LP_NT), 0, s, p);
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

uint64_t kv_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top_n) {
  if (rows <= 0 || rows > (1 << 20) || vocab <= 0 || vocab > LP_MAX_VOCAB || top_n < 0 ||
      top_n > KV_LOGPROBS_MAX_TOP || top_n > vocab)
    return 0;
  const int64_t chunks = chunks_of(items_of(rows, vocab), vocab);
  return (uint64_t)(rows * chunks * (16 + 8 * (int64_t)top_n));
}

kv_status kv_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t stride, float scale,
                      const int32_t* tokens, int32_t top_n, float* logprobs, float* entropy, float* top_logprobs,
                      int32_t* top_tokens, void* workspace, uint64_t ws_bytes, int32_t device, void* stream) {
  if (dtype != KV_F32 && dtype != KV_BF16) return kvr_err::set(KV_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > (1 << 20)) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^20");
  if (vocab < 1 || vocab > LP_MAX_VOCAB) return kvr_err::set(KV_EINVAL, "vocab must be 1 .. 2^22");
  if (stride < vocab) return kvr_err::set(KV_EINVAL, "the stride is below the vocabulary");
  if (!(scale > 0.0f) || !(scale < INFINITY)) return kvr_err::set(KV_EINVAL, "scale must be positive and finite");
  if (top_n < 0 || top_n > KV_LOGPROBS_MAX_TOP || top_n > vocab)
    return kvr_err::set(KV_EINVAL, "top_n must be 0 .. %d and at most the vocabulary", KV_LOGPROBS_MAX_TOP);
  if (rows == 0) return kvr_err::clear();
  if (!logits || (logprobs && !tokens) || (top_n > 0 && (!top_logprobs || !top_tokens)))
    return kvr_err::set(KV_EINVAL, "null logits, tokens, top_logprobs or top_tokens");
  if (!logprobs && !entropy && top_n == 0) return kvr_err::clear();
  const uintptr_t words = (uintptr_t)tokens | (uintptr_t)logprobs | (uintptr_t)entropy | (uintptr_t)top_logprobs |
                          (uintptr_t)top_tokens;
  if (words % 4 != 0 || (uintptr_t)logits % elem_bytes(dtype) != 0)
    return kvr_err::set(KV_EINVAL, "an array does not start on a boundary of its elements");
  if (!workspace || (uintptr_t)workspace % 16 != 0)
    return kvr_err::set(KV_EINVAL, "null workspace, or one not on a boundary of 16 bytes");
  const uint64_t need = kv_logprobs_workspace_bytes(rows, vocab, top_n);
  if (need > ws_bytes)
    return kvr_err::set(KV_ENOMEM, "workspace of %llu bytes < %llu needed", (unsigned long long)ws_bytes,
                        (unsigned long long)need);
  DeviceGuard dg(device);
  const kv_status st = device_ready(dg, device);
  if (st != KV_OK) return st;
  const int items = items_of(rows, vocab), chunks = chunks_of(items, vocab);
  LogprobParams p{};
  p.logits = static_cast<const char*>(logits);
  p.stride = stride * elem_bytes(dtype);
  p.vocab = vocab;
  p.chunks = chunks;
  p.top = top_n;
  p.scale = scale;
  p.tokens = tokens;
  p.logprobs = logprobs;
  p.entropy = entropy;
  p.top_logprobs = top_logprobs;
  p.top_tokens = top_tokens;
  p.stats = static_cast<float4*>(workspace);
  p.keys = reinterpret_cast<uint64_t*>(p.stats + rows * chunks);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == KV_BF16) launch<bf16_t>(p, rows, items, s);
  else launch<float>(p, rows, items, s);
  return launched();
}

}  // extern "C"

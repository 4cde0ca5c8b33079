// Log probabilities of given tokens, entropy and likeliest tokens (kvr_logprob.h).
//
// In log2 units, t_v = c (z_v - m) with c = scale log2 e and m the row's largest logit,
// e_v = 2^t_v, l = sum e_v and s = sum t_v e_v:
//   log p_t = scale (z_t - m) - ln 2 log2 l,   entropy = ln 2 (log2 l - s / l)
// (both terms of each are of one sign, so nothing cancels).  Over a chunk of the row t_v is
// one operation, fma(c, z_v, -C) with C = c m rounded (m the chunk's): the rounding of C
// shifts all t alike, and is taken out where chunks meet.  Where C is so large that its
// rounding would count, t_v = (z_v - m) c.  (That everywhere: 61 us for 1024 rows of 151936
// in bf16, not 55.)  A row is cut into chunks; a workgroup reads its chunk once, into
// registers, takes the chunk's m, l and s from there and, where asked, its top_n entries;
// a second kernel merges the chunks of each row in a fixed order.
//
// Top entries.  (value, lower index first) is one 64-bit key, so that all keys of a
// row differ and the order is total.  A bound that at least top_n entries reach comes
// from the threads' own largest values: one wave finds, bit by bit from the top, a
// value that at least top_n and not many more threads reach; the entries that reach
// it are listed in LDS and ranked by counting.  (Ranking the threads' values by counting
// took 1.7 us a chunk.)  Where equal values make too many of them, the bound is the
// top_n-th of the threads' keys.
//
// What bounds it.  Many rows: HBM, one exp and some six other operations for 4 or 2 bytes:
// 1024 rows of 151936 in bf16 52 - 54 us, 311 MB at up to 6 TB/s, and 4.8 the second kernel.
// 64 rows of 128256 in fp32 with the 20 likeliest, 12.5 + 4.8 us: all chunks are in flight at
// once, so their phases follow each other: 3.5 us (the last 6.4) until a chunk is there, then
// m, l and s, the bound beside them, the entries.  One row: latency, 5.2 + 3.5 us.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "host.h"
#include "kvr_logprob.h"
#include "logits.h"

namespace kvr {
namespace {

constexpr int LP_NT = 256;
// Entries of a thread.  A workgroup's piece in flight is 32 KB of fp32: 1024 rows of
// 151936 in bf16 took 70 us with 64 entries, 64 with 16 and 55 with 32; one row takes
// as long with 16 as with 32.
constexpr int LP_ITEMS = 32;
constexpr int LP_CHUNK = LP_NT * LP_ITEMS;
constexpr int LP_MAX_VOCAB = 256 * LP_CHUNK;
constexpr int64_t LP_MOST_CHUNKS = (1 << 24) - 1;  // of a call: a grid holds 2^32 - 1 threads

struct LogprobParams {
  const char* logits;
  int64_t stride;  // bytes
  int vocab, chunks, top;
  float scale, scale2;  // scale log2 e
  const int32_t* tokens;
  float* logprobs;
  float* entropy;
  float* top_logprobs;
  int32_t* top_tokens;
  float4* stats;   // [rows][chunks] m, l, s
  uint64_t* keys;  // [rows][chunks][top]
};

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

// Ranks by counting: how many of the n keys in LDS are larger.
__device__ __forceinline__ int rank_of(uint64_t key, const uint64_t* keys, int n) {
  int r = 0;
#pragma unroll 8
  for (int i = 0; i < n; ++i) r += keys[i] > key;
  return r;
}

// PER: entries of a thread at most.  With a bound that is one of the threads' keys, the
// top_n <= 64 threads that reach it have no more entries than the list takes; with one
// that comes from their values, lists above LP_LIST are given up for that, and so are bounds
// that more than MOST_REACH threads reach.  Only equal values make either: lists of 256 and
// 1024, bounds of 96 and 240 threads took the same on ordinary logits.
constexpr int LP_LIST = 512, MOST_REACH = 160;
template <int PER>
struct TopScratch {
  static constexpr int KEYS = 64 * PER;
  uint64_t keys[KEYS];
  uint32_t own[LP_NT];
  uint32_t bound;  // of the order bits; 0xffffffff: too many threads reach it
  int count;
};

// One wave: a value that at least `least` and, equal values apart, at most `most` of the
// threads' values reach.  First the longest run of the leading bits of `upper` (no smaller
// than any of them) that enough of them reach, then bit by bit of those that T has.
template <typename T, typename S>
__device__ __forceinline__ void find_bound(int least, int most, uint32_t upper, S& s) {
  const int lane = threadIdx.x & 63;
  uint32_t u[LP_NT / 64];
#pragma unroll
  for (int i = 0; i < LP_NT / 64; ++i) u[i] = s.own[i * 64 + lane];
  auto reach = [&](uint32_t v) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < LP_NT / 64; ++i) n += __builtin_popcountll(__ballot(u[i] >= v));
    return n;
  };
  uint32_t bound = 0;
  int n = LP_NT, free = 32;  // the lowest bits of the bound that are 0
#pragma unroll 1
  for (int low = 0; low < free;) {
    const int mid = (low + free) / 2;
    const uint32_t v = upper & ~0u << mid;
    const int k = reach(v);
    if (k >= least) {
      bound = v;
      n = k;
      free = mid;
    } else {
      low = mid + 1;
    }
  }
  // upper's next bit is 1, and with it too few reach
#pragma unroll 1
  for (int b = free - 2; b >= 32 - 8 * (int)sizeof(T) && n > most; --b) {
    const uint32_t v = bound | 1u << b;
    const int k = reach(v);
    if (k >= least) {
      bound = v;
      n = k;
    }
  }
  if (lane == 0) {
    s.bound = n > MOST_REACH ? 0xffffffffu : bound;
    s.count = 0;
  }
}
// Threads that a bound may be reached by: fewer need more of its bits, more make a longer list to
// rank.  With top + 2 the same, with 4 top + 8 64 rows of 20000 in bf16 with the 64 likeliest
// 10.7 us, not 8.2, of 128256 13.6, not 12.1.
__device__ __forceinline__ int most_threads(int top) { return min(64, 2 * top + 8); }
template <typename S>
__device__ __forceinline__ void collect(uint64_t key, S& s) {
  const int at = atomicAdd(&s.count, 1);  // any order: the ranks settle it
  if (at < S::KEYS) s.keys[at] = key;
}
// The same with whole keys, all different: the top-th largest of the threads' own,
// ranked by counting in the list's place.
template <typename S>
__device__ __forceinline__ uint64_t bound_of_keys(uint64_t own, int top, S& s) {
  static_assert(S::KEYS > LP_NT, "the threads' keys fit the list");
  const int t = threadIdx.x;
  __syncthreads();  // the list and its count have been read
  s.keys[t] = own;
  if (t == 0) s.count = 0;
  __syncthreads();
  if (rank_of(own, s.keys, LP_NT) == top - 1) s.keys[LP_NT] = own;
  __syncthreads();
  const uint64_t bound = s.keys[LP_NT];
  __syncthreads();
  return bound;
}

// Sums and maximum over the workgroup, in every thread; red holds a value a wave.
__device__ __forceinline__ float2 block_total(float a, float b, float2* red) {
  a = sum_over_wave(a);
  b = sum_over_wave(b);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = make_float2(a, b);
  __syncthreads();
  float2 v = red[0];
#pragma unroll
  for (int i = 1; i < LP_NT / 64; ++i) {
    v.x += red[i].x;
    v.y += red[i].y;
  }
  return v;
}
__device__ __forceinline__ float block_most(float v, float* red) {
  v = max_over_wave(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < LP_NT / 64; ++i) v = fmaxf(v, red[i]);
  return v;
}

// A row's token and its logit, then the results from the row's sums.
template <typename T>
struct Row {
  int64_t row;
  int tok = -1;
  float z = 0.0f;
  float base, log_l, s_l;
  bool none;  // every logit -infinity
  __device__ __forceinline__ explicit Row(int64_t r) : row(r) {}
  __device__ __forceinline__ void load(const LogprobParams& p) {
    if (!p.logprobs) return;
    tok = p.tokens[row];
    if (tok >= 0 && tok < p.vocab) z = Elem<T>::load(reinterpret_cast<const T*>(p.logits + row * p.stride), tok);
  }
  __device__ __forceinline__ void sums(float m, float l, float s) {
    base = base_of(m);
    none = l == 0.0f;
    log_l = none ? 0.0f : log2f(l);
    s_l = s / l;
  }
  __device__ __forceinline__ float logprob(const LogprobParams& p, float v) const {
    return none ? -INFINITY : scaled_difference(v, base, p.scale, LN2 * log_l);
  }
  __device__ __forceinline__ void put(const LogprobParams& p) const {
    if (p.logprobs)
      p.logprobs[row] = tok < 0 ? 0.0f : tok < p.vocab ? logprob(p, z) : log_l != log_l ? log_l : -INFINITY;
    if (p.entropy) {
      const float h = LN2 * (log_l - s_l);
      p.entropy[row] = none || h < 0.0f ? 0.0f : h;  // NaN stays
    }
  }
  __device__ __forceinline__ void put_top(const LogprobParams& p, int rank, uint64_t key) const {
    p.top_tokens[row * p.top + rank] = (int32_t)key_index(key);
    p.top_logprobs[row * p.top + rank] = logprob(p, ordered_value((uint32_t)(key >> 32)));
  }
};

// ONE: rows of one chunk, whose results it writes itself (a call on 64 rows of 5000 with the
// 20 likeliest 6.9 us; 10.8 with the second kernel).
template <typename T, bool TOP, bool ONE>
__global__ __launch_bounds__(LP_NT) void logprob_chunk_kernel(LogprobParams p) {
  constexpr int VEC = Piece<T>::N, VECS = LP_ITEMS / VEC, STEP = LP_NT * VEC;
  __shared__ float s_most[LP_NT / 64];
  __shared__ float2 s_sums[LP_NT / 64];
  const int t = threadIdx.x;
  const int c = ONE ? 0 : blockIdx.x % p.chunks;
  const int64_t row = ONE ? blockIdx.x : blockIdx.x / p.chunks;
  Row<T> result(row);
  if (ONE && t == 0) result.load(p);
  const T* z = reinterpret_cast<const T*>(p.logits + row * p.stride);
  const int begin = c * LP_CHUNK, first = begin + t * VEC;
  Piece<T> v[VECS];
  if (begin + LP_CHUNK <= p.vocab) {
#pragma unroll
    for (int i = 0; i < VECS; ++i) v[i].load(z + (begin + i * STEP) + (uint32_t)(t * VEC));
  } else {
    // the row's end: a piece that crosses it is loaded from further left, what others
    // hold of it masked
#pragma unroll
    for (int i = 0; i < VECS; ++i) {
      const int at = first + i * STEP, from = min(at, p.vocab - VEC);
      if (p.vocab >= VEC) {
        v[i].load(z + from);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[i].set(j, from + j >= at ? v[i].value(j) : -INFINITY);
      } else {
        v[i] = Piece<T>{};
#pragma unroll
        for (int j = 0; j < VEC; ++j) v[i].set(j, i == 0 && at + j < p.vocab ? Elem<T>::load(z, at + j) : -INFINITY);
      }
    }
  }
  float most[VECS], own = -INFINITY;
#pragma unroll
  for (int i = 0; i < VECS; ++i) {
    most[i] = v[i].value(0);
#pragma unroll
    for (int j = 1; j < VEC; ++j) most[i] = fmaxf(most[i], v[i].value(j));
    own = fmaxf(own, most[i]);
  }
  // nothing but -infinity (or NaN): sums of zeros (or NaN)
  __shared__ typename std::conditional<TOP, TopScratch<LP_ITEMS>, int>::type s_top;
  if constexpr (TOP) s_top.own[t] = order_bits(own);
  const float m = block_most(own, s_most);
  // a wave finds the bound first (of the workgroups of a CU, which come 256 apart, not the same one)
  if constexpr (TOP)
    if (t / 64 == (blockIdx.x >> 8) % (LP_NT / 64)) find_bound<T>(p.top, most_threads(p.top), order_bits(m), s_top);
  float l = 0.0f, s = 0.0f;
  const float base = base_of(m), cm = c_of(base, p.scale2);
  auto add = [&](float x) {
    const float e = __builtin_amdgcn_exp2f(x);
    l += e;
    s = fmaf(fmaxf(x, -1e30f), e, s);  // -infinity times 0; a NaN is in l
  };
  if (by_c(cm)) {
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) add(fmaf(v[i].value(j), p.scale2, -cm));
  } else {
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
      for (int j = 0; j < VEC; ++j) add((v[i].value(j) - base) * p.scale2);
  }
  const float2 sums = block_total(l, s, s_sums);
  if constexpr (ONE) {
    l = s = 0.0f;
    add_chunk(m, sums.x, sums.y, base, p.scale2, l, s);
    result.sums(m, l, s);
    if (t == 0) result.put(p);
  } else {
    if (t == 0) p.stats[row * p.chunks + c] = make_float4(m, sums.x, sums.y, 0.0f);
  }
  if constexpr (TOP) {
    uint64_t bound = (uint64_t)s_top.bound << 32;
    const auto key_at = [&](int at) {  // past the vocabulary: as NaN of higher indices, below all others
      return make_key(at < p.vocab ? order_bits(Elem<T>::load(z, at)) : 0u, at);
    };
#pragma unroll 1
    for (bool by_key = s_top.bound == 0xffffffffu;; by_key = true) {
      if (by_key) {
        uint64_t key = 0;
#pragma unroll 8
        for (int i = 0; i < LP_ITEMS; ++i) key = max(key, key_at(first + i / VEC * STEP + i % VEC));
        bound = bound_of_keys(key, p.top, s_top);
      }
      // pieces with an entry that may reach the bound are read again
      uint32_t hit = 0;
#pragma unroll
      for (int i = 0; i < VECS; ++i) hit |= (order_bits(most[i]) >= (uint32_t)(bound >> 32) ? 1u : 0u) << i;
#pragma unroll 1
      while (hit) {
        const int at = first + (__ffs(hit) - 1) * STEP;
        hit &= hit - 1;
        if (at + VEC <= p.vocab) {
          Piece<T> w;
          w.load(z + at);
#pragma unroll
          for (int j = 0; j < VEC; ++j) {
            const uint64_t k = make_key(order_bits(w.value(j)), at + j);
            if (k >= bound) collect(k, s_top);
          }
        } else {
#pragma unroll 1
          for (int j = 0; j < VEC; ++j) {
            const uint64_t k = key_at(at + j);
            if (k >= bound) collect(k, s_top);
          }
        }
      }
      __syncthreads();
      if (by_key || s_top.count <= LP_LIST) break;
    }
    const int n = min(s_top.count, s_top.KEYS);
    uint64_t* out = p.keys + (row * p.chunks + c) * p.top;
    for (int i = t; i < n; i += LP_NT) {
      const uint64_t k = s_top.keys[i];
      const int r = rank_of(k, s_top.keys, n);
      if (r >= p.top) continue;
      if (ONE) result.put_top(p, r, k);
      else out[r] = k;
    }
  }
}

template <typename T, bool TOP>
__global__ __launch_bounds__(LP_NT) void logprob_row_kernel(LogprobParams p) {
  const int t = threadIdx.x, lane = t & 63;
  const int64_t row = blockIdx.x;
  const float4* stats = p.stats + row * p.chunks;
  const uint64_t* keys = p.keys + row * p.chunks * p.top;
  const int total = p.chunks * p.top;
  // `each` keys of falling order a thread: its largest, and its least where it has as many
  const int each = (total + LP_NT - 1) / LP_NT;
  uint64_t own = t, least = ~0ull;  // threads without a key: below all of them, and different
  if (TOP)
    for (int i = t * each; i < (t + 1) * each; ++i) {
      const uint64_t k = i < total ? keys[i] : 0;
      own = max(own, k);
      least = min(least, k);
    }
  Row<T> result(row);
  if (t == 0) result.load(p);
  // every wave merges all chunks, in the same order
  float m = -INFINITY;
  for (int c = lane; c < p.chunks; c += 64) m = fmaxf(m, stats[c].x);
  m = max_over_wave(m);
  float l = 0.0f, s = 0.0f;
  for (int c = lane; c < p.chunks; c += 64) {
    const float4 q = stats[c];
    add_chunk(q.x, q.y, q.z, base_of(m), p.scale2, l, s);
  }
  result.sums(m, sum_over_wave(l), sum_over_wave(s));
  if (t == 0) result.put(p);
  if constexpr (TOP) {
    // a thread holds ceil(256 * 64 / 256) keys at most
    __shared__ TopScratch<64> s_top;
    // a bound that top_n keys reach because enough threads' least ones do
    s_top.own[t] = (uint32_t)(least >> 32);
    __syncthreads();
    const int threads = (p.top + each - 1) / each;
    // (up to 8 threads of `each` keys too many: with none the same, with 32 7.6 us, not 6.5, for the
    // 64 likeliest of 64 rows of 128256 in bf16)
    if (t < 64) find_bound<T>(threads, each == 1 ? most_threads(p.top) : threads + 8, order_bits(m), s_top);
    __syncthreads();
    uint64_t bound = (uint64_t)s_top.bound << 32;
#pragma unroll 1
    for (bool by_key = s_top.bound == 0xffffffffu;; by_key = true) {
      if (by_key) bound = bound_of_keys(own, p.top, s_top);
      if (own >= bound)
        for (int i = t * each; i < min((t + 1) * each, total); ++i)
          if (keys[i] >= bound) collect(keys[i], s_top);
      __syncthreads();
      if (by_key || s_top.count <= LP_LIST) break;
    }
    const int n = min(s_top.count, s_top.KEYS);
    for (int i = t; i < n; i += LP_NT) {
      const uint64_t k = s_top.keys[i];
      const int r = rank_of(k, s_top.keys, n);
      if (r < p.top) result.put_top(p, r, k);
    }
  }
}

int chunks_of(int vocab) { return (vocab + LP_CHUNK - 1) / LP_CHUNK; }

template <typename T, bool TOP>
void launch(const LogprobParams& p, int64_t rows, hipStream_t s) {
  const dim3 grid((unsigned)(rows * p.chunks));
  if (p.chunks == 1) {
    hipLaunchKernelGGL((logprob_chunk_kernel<T, TOP, true>), grid, dim3(LP_NT), 0, s, p);
    return;
  }
  hipLaunchKernelGGL((logprob_chunk_kernel<T, TOP, false>), grid, dim3(LP_NT), 0, s, p);
  hipLaunchKernelGGL((logprob_row_kernel<T, TOP>), dim3((unsigned)rows), dim3(LP_NT), 0, s, p);
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" {

uint64_t kv_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top_n) {
  if (rows <= 0 || rows > (1 << 20) || vocab <= 0 || vocab > LP_MAX_VOCAB || top_n < 0 ||
      top_n > KV_LOGPROBS_MAX_TOP || top_n > vocab)
    return 0;
  const int64_t chunks = chunks_of(vocab);
  if (rows * chunks > LP_MOST_CHUNKS) return 0;
  return (uint64_t)(rows * chunks * (16 + 8 * (int64_t)top_n));
}

kv_status kv_logprobs(const void* logits, int32_t dtype, int64_t rows, int32_t vocab, int64_t stride, float scale,
                      const int32_t* tokens, int32_t top_n, float* logprobs, float* entropy, float* top_logprobs,
                      int32_t* top_tokens, void* workspace, uint64_t ws_bytes, int32_t device, void* stream) {
  if (dtype != KV_F32 && dtype != KV_BF16) return kvr_err::set(KV_EINVAL, "unknown dtype %d", dtype);
  if (rows < 0 || rows > (1 << 20)) return kvr_err::set(KV_EINVAL, "rows must be 0 .. 2^20");
  if (vocab < 1 || vocab > LP_MAX_VOCAB) return kvr_err::set(KV_EINVAL, "vocab must be 1 .. 2^21");
  if (rows * chunks_of(vocab) > LP_MOST_CHUNKS)
    return kvr_err::set(KV_EINVAL, "rows * vocab of one call above 2^37: split the rows");
  if (stride < vocab) return kvr_err::set(KV_EINVAL, "the stride is below the vocabulary");
  if (!(scale > 0.0f) || !(scale <= 0x1p127f))
    return kvr_err::set(KV_EINVAL, "scale must be positive and at most 2^127");
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
  const int chunks = chunks_of(vocab);
  LogprobParams p{};
  p.logits = static_cast<const char*>(logits);
  p.stride = stride * elem_bytes(dtype);
  p.vocab = vocab;
  p.chunks = chunks;
  p.top = top_n;
  p.scale = scale;
  p.scale2 = scale * LOG2E;
  p.tokens = tokens;
  p.logprobs = logprobs;
  p.entropy = entropy;
  p.top_logprobs = top_logprobs;
  p.top_tokens = top_tokens;
  p.stats = static_cast<float4*>(workspace);
  p.keys = reinterpret_cast<uint64_t*>(p.stats + rows * chunks);
  hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  if (dtype == KV_BF16) top_n ? launch<bf16_t, true>(p, rows, s) : launch<bf16_t, false>(p, rows, s);
  else top_n ? launch<float, true>(p, rows, s) : launch<float, false>(p, rows, s);
  return launched();
}

}  // extern "C"

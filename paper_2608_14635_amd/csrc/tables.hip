// Block tables and slot maps from request lengths (kvr_tables.h).
//
// Request r's first row is the sum of the new positions before it, its first
// block of the free list the sum of the blocks needed before it: two prefix sums
// over the requests.  A row then follows by itself: position p of request r lies
// in table entry j = p / B, which is an old entry (j < ceil(held / B)) or the
// free list's at[r] + j - ceil(held / B).  The row of a new block's first
// position (p = j B, which is never an old one) writes the entry, so that the
// entries need no pass of their own.
//
// One launch: every workgroup sums over all requests itself, 512 a step, and
// works off its window of rows against each step's requests while they are in
// LDS; no workgroup waits for another.  Short calls are the launch and one scan step (64
// requests: 4.4 us); of long ones the rows' writes are half (333 requests, 2.7 million
// positions: 33 MB in 14.9 us), the rest each workgroup's way through scan, search and
// free list.  (A workgroup that worked off two or four windows for each scan took 19 and
// 28 us; eight rows a thread 16.7, 256 threads 15.5, 1024 18.5.)
#include <algorithm>

#include "host.h"
#include "kvr_tables.h"

namespace kvr {
namespace {

constexpr int TG_NT = 512;   // threads of a workgroup, requests of a scan step
constexpr int TG_PER = 4;    // consecutive rows of a thread
constexpr int TG_WIN = TG_NT * TG_PER;

struct GrowParams {
  const int32_t* held;
  const int32_t* lens;
  int R, B, shift;  // shift: log2 B, or -1
  const int32_t* free_blocks;
  int num_free;
  int32_t* tables;
  int max_blocks;
  int64_t max_rows;
  int32_t* row_offsets;
  int64_t* slots;
  int32_t* positions;
  int32_t* counts;
};

// Two sums in one word: rows in the low half, blocks in the high one.  Both stay
// below 2^32 for calls as documented; whatever they hold, every index made from
// them is checked before its use.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
  // within rows of 16 lanes, then their last lanes' sums into the rows behind
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);   // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);   // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);   // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15 into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31 into rows 2 and 3
  return v;
}

__global__ __launch_bounds__(TG_NT) void tables_grow_kernel(GrowParams p) {
  __shared__ uint32_t s_row[TG_NT], s_at[TG_NT];
  __shared__ int s_held[TG_NT], s_have[TG_NT], s_n[TG_NT];
  __shared__ uint64_t s_wave[TG_NT / 64];
  __shared__ int s_unplaced;
  const int t = threadIdx.x, lane = t & 63, w = t >> 6;
  const uint32_t B = (uint32_t)p.B;
  // n / B: a shift where B is a power of two (a division by a number known only here is
  // some twenty instructions)
  const auto blocks_of = [&](uint32_t n) { return p.shift >= 0 ? n >> p.shift : n / B; };
  int unplaced = 0;
  if (t == 0) s_unplaced = 0;
  for (int64_t win = blockIdx.x;; win += gridDim.x) {
    const int64_t row0 = win * TG_WIN + t * TG_PER;  // the thread's first row
    int64_t slot[TG_PER];
    int pos[TG_PER];
#pragma unroll
    for (int u = 0; u < TG_PER; ++u) slot[u] = pos[u] = -1;
    uint64_t base = 0;  // the sums before this step's requests
    for (int r0 = 0; r0 < p.R; r0 += TG_NT) {
      const int r = r0 + t;
      int held = 0, n = 0;
      uint32_t need = 0, have = 0, want = 0;
      if (r < p.R) {
        held = p.held ? max(p.held[r], 0) : 0;
        const int len = max(p.lens[r], held);
        n = len - held;
        have = blocks_of((uint32_t)held + B - 1);
        want = min(blocks_of((uint32_t)len + B - 1), (uint32_t)p.max_blocks);
        need = want > have ? want - have : 0;
      }
      const uint64_t own = (uint64_t)need << 32 | (uint32_t)n;
      const uint64_t incl = (uint64_t)wave_scan(need) << 32 | wave_scan((uint32_t)n);
      if (lane == 63) s_wave[w] = incl;
      __syncthreads();
      uint64_t before = base;
#pragma unroll
      for (int i = 0; i < TG_NT / 64; ++i) {
        if (i < w) before += s_wave[i];
        base += s_wave[i];
      }
      const uint64_t excl = before + incl - own;
      const uint32_t row = (uint32_t)excl, at = (uint32_t)(excl >> 32);
      s_row[t] = row;
      s_at[t] = at;
      s_held[t] = held;
      s_have[t] = (int)have;
      s_n[t] = n;
      if (blockIdx.x == 0 && win == 0 && r < p.R) {
        p.row_offsets[r] = (int32_t)row;
        // rows without a slot: an old last block that is none, then the positions
        // from the first entry the list or the table has no room for.  (The list's
        // ids are not looked at: this workgroup would read all that are handed out.)
        const uint32_t len = (uint32_t)held + n;
        uint32_t from = held;  // first position of the new entries
        if (n > 0 && have * B > (uint32_t)held) {
          const uint32_t end = min(have * B, len);
          if (have > (uint32_t)p.max_blocks || p.tables[(int64_t)r * p.max_blocks + have - 1] < 0)
            unplaced += end - from;
          from = end;
        }
        const uint32_t left = (uint32_t)p.num_free > at ? p.num_free - at : 0;  // blocks left to it
        const uint32_t upto = have + min(need, left);                           // entries with a block
        const uint64_t placed = (uint64_t)upto * B;
        if (len > from && placed < len) unplaced += len - max(from, (uint32_t)placed);
      }
      __syncthreads();
      // this step's rows among mine
      const int count = min(TG_NT, p.R - r0);
      const int64_t lo = s_row[0], hi = (uint32_t)base;
      const int64_t first = max(row0, lo);
      if (first < min(row0 + TG_PER, hi)) {
        int a = 0, b = count - 1;  // the last request whose first row is not past `first`
        while (a < b) {
          const int m = (a + b + 1) / 2;
          if (s_row[m] <= first) a = m;
          else b = m - 1;
        }
        int64_t end = 0;  // behind the request's last row
        int q = 0, j = 0, off = 0, entry = -1;  // a row's position: offset `off` of table entry j, whose block this is
        auto look = [&]() {
          int32_t* cell = p.tables + (int64_t)(r0 + a) * p.max_blocks + j;
          const int fresh = j - s_have[a];  // an entry of the call's own
          entry = -1;
          if ((uint32_t)j >= (uint32_t)p.max_blocks) return;
          if (fresh < 0) {
            entry = *cell;
          } else {
            const uint32_t f = s_at[a] + fresh;
            if (f < (uint32_t)p.num_free) entry = p.free_blocks[f];
            if (off == 0) *cell = entry;
          }
        };
        auto enter = [&](int64_t i) {
          end = (int64_t)s_row[a] + s_n[a];
          q = s_held[a] + (int)(i - s_row[a]);
          j = blocks_of(q);
          off = q - j * p.B;
          look();
        };
        bool in = false;
#pragma unroll
        for (int u = 0; u < TG_PER; ++u) {
          const int64_t i = row0 + u;
          if (i < first || i >= hi) continue;
          if (!in) {
            enter(i);
            in = true;
          } else if (i >= end) {
            do a = min(a + 1, count - 1);
            while (a < count - 1 && s_n[a] == 0);  // i < hi: a request further on holds it
            enter(i);
          } else {
            ++q;
            if (++off == p.B) {
              off = 0;
              ++j;
              look();
            }
          }
          pos[u] = q;
          slot[u] = entry >= 0 ? (int64_t)entry * p.B + off : -1;
        }
      }
      __syncthreads();
    }
    const int64_t total = (uint32_t)base;
    if (row0 + TG_PER <= p.max_rows) {
      typedef int64_t pair __attribute__((ext_vector_type(2), aligned(8)));
      typedef int quad __attribute__((ext_vector_type(4), aligned(4)));
      reinterpret_cast<pair*>(p.slots + row0)[0] = pair{slot[0], slot[1]};
      reinterpret_cast<pair*>(p.slots + row0)[1] = pair{slot[2], slot[3]};
      if (p.positions) *reinterpret_cast<quad*>(p.positions + row0) = quad{pos[0], pos[1], pos[2], pos[3]};
    } else {
#pragma unroll
      for (int u = 0; u < TG_PER; ++u)
        if (row0 + u < p.max_rows) {
          p.slots[row0 + u] = slot[u];
          if (p.positions) p.positions[row0 + u] = pos[u];
        }
    }
    if (blockIdx.x == 0 && win == 0) {
      if (unplaced) atomicAdd(&s_unplaced, unplaced);
      __syncthreads();
      if (t == 0) {
        const int need = (int)min(base >> 32, (uint64_t)INT32_MAX);
        p.row_offsets[p.R] = (int32_t)total;
        p.counts[0] = min(need, p.num_free);
        p.counts[1] = max(need - p.num_free, 0);
        p.counts[2] = (int32_t)total;
        p.counts[3] = s_unplaced;
      }
    }
    if ((win + gridDim.x) * TG_WIN >= max(total, p.max_rows)) break;
  }
}

}  // namespace
}  // namespace kvr

using namespace kvr;

extern "C" kv_status kv_tables_grow(const int32_t* held, const int32_t* lens, int32_t R, int32_t B,
                                    const int32_t* free_blocks, int32_t num_free, int32_t* tables,
                                    int32_t max_blocks, int64_t max_rows, int32_t* row_offsets,
                                    int64_t* slots, int32_t* positions, int32_t* counts, int32_t device,
                                    void* stream) {
  if (R < 0 || R > 1 << 30 || num_free < 0 || max_blocks < 0 || max_rows < 0 || max_rows > INT32_MAX)
    return kvr_err::set(KV_EINVAL,
                        "num_requests is 0 .. 2^30; num_free, max_blocks_per_req and max_rows 0 .. 2^31 - 1");
  if (B <= 0) return kvr_err::set(KV_EINVAL, "block_size must be positive");
  if (!row_offsets || !counts) return kvr_err::set(KV_EINVAL, "null row_offsets or counts");
  if (R > 0 && !lens) return kvr_err::set(KV_EINVAL, "null lens");
  if (R > 0 && max_blocks > 0 && !tables) return kvr_err::set(KV_EINVAL, "null block_tables");
  if (num_free > 0 && !free_blocks) return kvr_err::set(KV_EINVAL, "null free_blocks");
  if (max_rows > 0 && !slots) return kvr_err::set(KV_EINVAL, "null slots");
  const uintptr_t words = (uintptr_t)held | (uintptr_t)lens | (uintptr_t)free_blocks | (uintptr_t)tables |
                          (uintptr_t)row_offsets | (uintptr_t)positions | (uintptr_t)counts;
  if (words % 4 != 0 || (uintptr_t)slots % 8 != 0)
    return kvr_err::set(KV_EINVAL, "an array does not start on a boundary of its elements");
  DeviceGuard dg(device);
  const kv_status st = device_ready(dg, device);
  if (st != KV_OK) return st;
  const int shift = (B & (B - 1)) == 0 ? __builtin_ctz(B) : -1;
  const GrowParams p{held,   lens,       R,        B,           shift, free_blocks, num_free,
                     tables, max_blocks, max_rows, row_offsets, slots, positions,   counts};
  // a workgroup a window, up to 2^25 rows; further windows are walked
  const int grid = (int)std::max<int64_t>(1, std::min<int64_t>((max_rows + TG_WIN - 1) / TG_WIN, 1 << 14));
  hipLaunchKernelGGL(tables_grow_kernel, dim3(grid), dim3(TG_NT), 0, reinterpret_cast<hipStream_t>(stream), p);
  return launched();
}

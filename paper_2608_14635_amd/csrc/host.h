// What the host files of the library share: error reporting, the model checks,
// the arena handle and the device guard.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <utility>
#include <vector>

#include "kvr.h"
#include "kvr_profile.h"

// the calling thread's error message
namespace kvr_err {
kv_status set(kv_status st, const char* fmt, ...);
kv_status clear();
}  // namespace kvr_err

struct kv_arena {
  void* base;
  uint64_t bytes;
  kv_model_desc desc;
  int32_t block_size;
  int64_t num_blocks;
  int32_t device;
  int* probe_flag;
  // pinned host staging for metadata uploads; reused after its last copy completed
  void* pinned = nullptr;
  size_t pinned_bytes = 0;
  hipEvent_t staged = nullptr;
  bool staged_pending = false;
  // optional per-kernel-class timing
  bool profile = false;
  std::vector<std::pair<int, std::pair<hipEvent_t, hipEvent_t>>> prof_pending;
  std::vector<hipEvent_t> prof_pool;
  double prof_ms[KV_PROF_CLASSES] = {};
  int64_t prof_launches[KV_PROF_CLASSES] = {};
  double prof_flops[KV_PROF_CLASSES] = {};
  std::vector<double> pending_flops;
};

struct kv_packed {
  void* base;
  uint64_t bytes;
  kv_model_desc desc;
  int32_t block_size;
  int64_t num_blocks;
  int32_t device;
  // staging as kv_arena's (kv_packed_decode_step)
  void* pinned = nullptr;
  size_t pinned_bytes = 0;
  hipEvent_t staged = nullptr;
  bool staged_pending = false;
};

namespace kvr {

inline int64_t elem_bytes(int32_t dtype) { return dtype == KV_BF16 ? 2 : 4; }
inline int64_t round_up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

kv_status check_desc(const kv_model_desc* d);
bool live_arena(const kv_arena* a);
bool live_packed(const kv_packed* a);
struct PackedLayer packed_layer(const kv_packed* a, int32_t layer);
// The checks of a bind: `base` is device memory on `device`, and a kernel's round
// trip there succeeds (Sec. 4.2 step 2).  *flag receives the 4 bytes it used.
kv_status probe_memory(const void* base, int32_t device, int** flag);

struct DeviceGuard {
  int prev = -1;
  bool changed = false;
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev != dev) {
      err = hipSetDevice(dev);
      changed = err == hipSuccess;
    }
  }
  ~DeviceGuard() {
    if (changed) (void)hipSetDevice(prev);
  }
};

// Around the launches of an entry point: the device is current and holds no error
// of earlier work; the launches went in.
inline kv_status device_ready(const DeviceGuard& dg, int device) {
  if (dg.err != hipSuccess) {
    (void)hipGetLastError();
    return kvr_err::set(KV_EDEVICE, "cannot select device %d: %s", device, hipGetErrorString(dg.err));
  }
  const hipError_t pre = hipGetLastError();
  if (pre != hipSuccess) return kvr_err::set(KV_EDEVICE, "pending device error: %s", hipGetErrorString(pre));
  return KV_OK;
}
inline kv_status launched() {
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return kvr_err::set(KV_EDEVICE, "kernel launch failed: %s", hipGetErrorString(err));
  return kvr_err::clear();
}

}  // namespace kvr

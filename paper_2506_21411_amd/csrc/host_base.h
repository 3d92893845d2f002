// Host-side basics shared by the library's translation units: status and alignment helpers, the stage-timing records, the
// per-device caches.  One copy of each in the library (inline variables).
#pragma once
#include "../../include/dchag.h"

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>
#include <mutex>
#include <unordered_map>
#include <vector>

#include "dchag_dev.h"

namespace dchag {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }
inline size_t elem_size(dchag_dtype dt) { return dt == DCHAG_F32 ? 4 : 2; }
inline bool misaligned(const void* p) { return p && (reinterpret_cast<uintptr_t>(p) & 15u); }

inline int launch_status() { return hipGetLastError() == hipSuccess ? DCHAG_OK : DCHAG_ERR_LAUNCH; }

// Optional stage timing (dchag_profile_begin / dchag_profile_end): an event pair per launch.
struct StageRecord {
  hipEvent_t start, stop;
  int stage, level;
};
inline bool g_profiling = false;
inline int g_level = 0;
inline std::vector<StageRecord> g_records;
// The level a stage record is filed under; written only while a profile is being taken.
inline void set_level(int level) {
  if (g_profiling) g_level = level;
}

struct StageTimer {
  hipStream_t st;
  bool on;
  StageRecord rec;
  StageTimer(int stage, hipStream_t s) : st(s), on(g_profiling) {
    if (!on) return;
    rec.stage = stage;
    rec.level = g_level;
    if (hipEventCreate(&rec.start) != hipSuccess || hipEventCreate(&rec.stop) != hipSuccess) {
      on = false;
      return;
    }
    (void)hipEventRecord(rec.start, st);
  }
  ~StageTimer() {
    if (!on) return;
    (void)hipEventRecord(rec.stop, st);
    g_records.push_back(rec);
  }
};

// Compute units of the CURRENT device (looked up once per device; 256 without a device).
constexpr int kMaxDevices = 64;
inline int compute_units() {
  static std::atomic<int> cus[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return 256;
  int n = cus[dev].load(std::memory_order_relaxed);
  if (n) return n;
  if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < kXcds) n = 256;
  cus[dev].store(n, std::memory_order_relaxed);
  return n;
}

// Raises a kernel's dynamic-LDS limit to at least `bytes`, once per (device, kernel): later launches only look the
// table up.  Returns 0 or DCHAG_ERR_LAUNCH.
inline int ensure_dynamic_lds(const void* kernel, int bytes) {
  static std::mutex mu;
  static std::unordered_map<const void*, int> done[kMaxDevices];
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kMaxDevices) return DCHAG_ERR_LAUNCH;
  std::lock_guard<std::mutex> lock(mu);
  auto it = done[dev].find(kernel);
  if (it != done[dev].end() && it->second >= bytes) return DCHAG_OK;
  if (hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes) != hipSuccess) return DCHAG_ERR_LAUNCH;
  done[dev][kernel] = bytes;
  return DCHAG_OK;
}

}  // namespace dchag

// Host-side helpers shared by the translation units of libsgdb: device attributes
// (queried once per device), launch status, checks of types and addresses.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstdio>
#include <mutex>

#include "../../include/sgdb.h"

namespace sgdb {

constexpr int kMaxDevices = 64;

struct DeviceInfo {
  std::atomic<bool> known{false};  // set last, with release: a reader that sees it sees the other fields
  int index = 0;
  int sms = 0;
  int max_smem_optin = 0;
};
inline DeviceInfo g_dev[kMaxDevices];
inline std::mutex g_dev_mutex;

inline bool is_aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline sgdb_status_t device_info(const DeviceInfo** out) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SGDB_ERR_CUDA;
  if (dev < 0 || dev >= kMaxDevices) return SGDB_ERR_UNSUPPORTED;
  DeviceInfo& d = g_dev[dev];
  if (!d.known.load(std::memory_order_acquire)) {
    std::lock_guard<std::mutex> lock(g_dev_mutex);
    if (!d.known.load(std::memory_order_relaxed)) {
      if (cudaDeviceGetAttribute(&d.sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
          cudaDeviceGetAttribute(&d.max_smem_optin, cudaDevAttrMaxSharedMemoryPerBlockOptin, dev) !=
              cudaSuccess)
        return SGDB_ERR_CUDA;
      d.index = dev;
      d.known.store(true, std::memory_order_release);
    }
  }
  *out = &d;
  return SGDB_OK;
}

inline sgdb_status_t launch_status() {
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) {
    std::fprintf(stderr, "libsgdb: CUDA error: %s\n", cudaGetErrorString(e));
    return SGDB_ERR_CUDA;
  }
  return SGDB_OK;
}

inline bool dtype_ok(int dt) { return dt == SGDB_F32 || dt == SGDB_BF16; }
inline size_t dtype_size(int dt) { return dt == SGDB_BF16 ? 2 : 4; }

// Address of an array of type dt: present and aligned to its elements.
inline bool array_ok(const void* p, int dt) {
  return p != nullptr && (reinterpret_cast<uintptr_t>(p) & (dtype_size(dt) - 1)) == 0;
}

// Whether rows of type dt at `p`, `ld` elements apart, all start on 16-byte boundaries.
inline bool rows_aligned16(const void* p, int64_t ld, int dt) {
  return is_aligned16(p) && (ld * static_cast<int64_t>(dtype_size(dt))) % 16 == 0;
}

// Patience of the kernels' waits, as sgdb_set_wait_limit_ns left it.
__attribute__((visibility("hidden"))) unsigned long long wait_limit_ns();

// The first half of sgdb_step_orthogonal, one launch (P = 0: the selection alone): select, mean g of the kept rows,
// m <- mu m + g, u = m or (nesterov) g + mu m.  Checks what sgdb_step checks.
__attribute__((visibility("hidden"))) sgdb_status_t select_and_velocity(const void* d_grad, int dt, int64_t P, int64_t ld,
                                                                        const float* d_arrival, const int32_t* d_tags, int32_t t,
                                                                        int32_t N, int32_t b, float* d_momentum, float* d_u, float mu,
                                                                        bool nesterov, uint8_t* d_mask, int32_t* d_order,
                                                                        int32_t* d_info, cudaStream_t s);

// Programmatic dependent launch: the kernel's start may overlap its predecessor's end, earlier still if that is a kernel
// that calls pdl_launch_dependents (layer norm's kernels and those that move the experts' rows do not: measured, it gains
// nothing there and takes up to 2 us from small ones); every kernel launched this way calls pdl_wait before it reads or writes
// global memory (prefetches aside), after which all that came before it in the stream is done.
template <typename... Args, typename... Given>
sgdb_status_t launch_dependent(void (*kernel)(Args...), dim3 grid, int threads, size_t smem, cudaStream_t s, Given... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  (void)cudaLaunchKernelEx(&cfg, kernel, static_cast<Args>(args)...);
  return launch_status();
}

}  // namespace sgdb

// What the C entry points share: device switching, trace ranges, guarded workspace, tensor map encoding.
#pragma once
#include <cuda.h>
#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include <cstdint>

namespace ilre {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*,
                                  const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                  const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder, null if it cannot be had.
inline EncodeTiledFn tensor_map_encoder() {
  void* fn = nullptr;
  cudaDriverEntryPointQueryResult qres;
  if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess ||
      qres != cudaDriverEntryPointSuccess)
    return nullptr;
  return reinterpret_cast<EncodeTiledFn>(fn);
}

static constexpr int kGuardBytes = 256;       // written once behind every workspace buffer
static constexpr int kGuardByte = 0xA5;
static constexpr int kMaxGuards = 48;

// A named range on the host time line for tracing tools that read NVTX (a no-op without one).
struct TraceRange {
  explicit TraceRange(const char* name) { nvtxRangePushA(name); }
  ~TraceRange() { nvtxRangePop(); }
  TraceRange(const TraceRange&) = delete;
  TraceRange& operator=(const TraceRange&) = delete;
};

struct DeviceGuard {
  int prev;
  bool ok;
  explicit DeviceGuard(int dev) : prev(-1), ok(false) {
    if (cudaGetDevice(&prev) != cudaSuccess) return;
    ok = (prev == dev) || (cudaSetDevice(dev) == cudaSuccess);
  }
  ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

// One workspace buffer of the handle, followed by a guard zone of kGuardBytes that nothing may
// write to (checked by ilre_recall_check_guards).
template <class Handle, class T>
bool dev_alloc(Handle* h, T** p, size_t count) {
  *p = nullptr;
  const size_t bytes = ((count ? count : 1) * sizeof(T) + 15) & ~static_cast<size_t>(15);
  if (h->n_guards >= kMaxGuards) return false;
  if (cudaMalloc(reinterpret_cast<void**>(p), bytes + kGuardBytes) != cudaSuccess) return false;
  uint8_t* zone = reinterpret_cast<uint8_t*>(*p) + bytes;
  if (cudaMemset(zone, kGuardByte, kGuardBytes) != cudaSuccess) return false;
  h->guard[h->n_guards++] = zone;
  return true;
}

// How many of the guard zones no longer hold the pattern, or ILRE_ERR_CUDA.
inline int damaged_guards(const uint8_t* const* guard, int n) {
  int damaged = 0;
  uint8_t zone[kGuardBytes];
  for (int i = 0; i < n; ++i) {
    if (cudaMemcpy(zone, guard[i], kGuardBytes, cudaMemcpyDeviceToHost) != cudaSuccess) return ILRE_ERR_CUDA;
    bool intact = true;
    for (int b = 0; b < kGuardBytes; ++b) intact = intact && zone[b] == kGuardByte;
    damaged += intact ? 0 : 1;
  }
  return damaged;
}

#define ILRE_CUDA(expr)                                   \
  do {                                                    \
    if ((expr) != cudaSuccess) return ILRE_ERR_CUDA;      \
  } while (0)

}  // namespace ilre

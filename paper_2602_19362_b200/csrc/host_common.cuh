// What the host sides of the C ABI share: the launch counter, the checks after a CUDA call, the current
// device's SM count, element sizes and the check of a matrix of logits.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "../../include/oapl.h"

namespace oapl {

inline std::atomic<uint64_t> g_launches{0};
#define OAPL_LAUNCHED() (g_launches.fetch_add(1, std::memory_order_relaxed))

constexpr int kMaxDevices = 64;  // per-device host-side caches

#define CK(call)                                   \
  do {                                             \
    if ((call) != cudaSuccess) return OAPL_ERR_CUDA; \
  } while (0)
#define CKL()                                                  \
  do {                                                         \
    OAPL_LAUNCHED();                                           \
    if (cudaGetLastError() != cudaSuccess) return OAPL_ERR_CUDA; \
  } while (0)

inline int sm_count() {
  static int n[kMaxDevices] = {0};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return 0;
  if (!n[dev] && cudaDeviceGetAttribute(&n[dev], cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) n[dev] = 0;
  return n[dev];
}

inline int type_size(int32_t type) {
  return type == OAPL_TYPE_BF16 || type == OAPL_TYPE_F16 ? 2 : (type == OAPL_TYPE_F32 ? 4 : 0);
}

inline int check_logits(const oapl_logits* L) {
  if (!L || !L->logits || L->N <= 0 || L->V <= 0 || L->ld < L->V) return OAPL_ERR_INVALID_ARG;
  const int es = type_size(L->type);
  if (!es) return OAPL_ERR_INVALID_ARG;
  if (!(L->scale > 0.f) || !(L->scale <= 1e6f)) return OAPL_ERR_INVALID_ARG;  // the forward's clamp
  if ((uintptr_t)L->logits % es) return OAPL_ERR_MISALIGNED;
  if (L->N > (int64_t)2000000000 || (int64_t)L->V > (int64_t)2000000000) return OAPL_ERR_UNSUPPORTED_SHAPE;
  return OAPL_OK;
}

}  // namespace oapl

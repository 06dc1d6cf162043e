// What the host sides of the C ABI share: the launch counter, the checks after a CUDA call, the current
// device's SM count, element sizes and the check of a matrix of logits.
#pragma once
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <utility>

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

// The next launch of a call whose kernels begin with after_launch_before(): its start-up goes under the end of the launch
// before it.
template <typename... P, typename... A>
inline cudaError_t launch_next(void (*kern)(P...), dim3 grid, dim3 block, size_t smem, cudaStream_t st, A&&... args) {
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cfg.attrs = &at;
  cfg.numAttrs = 1;
  const cudaError_t rc = cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
  if (rc != cudaSuccess) (void)cudaGetLastError();
  OAPL_LAUNCHED();
  return rc;
}

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

constexpr int64_t kMaxRows = 2000000000;
constexpr int64_t kMaxGrid = 2147483647;

inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool on16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// A matrix in memory, to see what overlaps.
struct Place {
  const void* base;
  int64_t rows, cols, ld;
  int es;
};
enum Overlap { kApart, kSameRows, kMixed };
// kSameRows: the same rows of the same elements.  Matrices of one row pitch may lie between one another's rows.
inline Overlap overlap(const Place& p, const Place& q) {
  using Wide = unsigned __int128;
  if (!p.base || !q.base) return kApart;
  const Wide a = (uintptr_t)p.base, b = (uintptr_t)q.base, ra = (Wide)p.cols * p.es, rb = (Wide)q.cols * q.es;
  const Wide pa = (Wide)p.ld * p.es, pb = (Wide)q.ld * q.es;
  const Wide ea = a + (Wide)(p.rows - 1) * pa + ra, eb = b + (Wide)(q.rows - 1) * pb + rb;
  if (a >= eb || b >= ea) return kApart;
  if (a == b && p.es == q.es && p.rows == q.rows && p.cols == q.cols && (pa == pb || p.rows == 1)) return kSameRows;
  if (pa != pb) return kMixed;
  const Wide off = b >= a ? (b - a) % pa : (pa - (a - b) % pa) % pa;  // q's rows in p's pitch
  return off >= ra && pa - off >= rb ? kApart : kMixed;
}

}  // namespace oapl

// The norm over a list of gradient tensors, and the list scaled to a largest norm.
//
//     sq = sum (s g)^2 over all elements,      out = s g min(1, c / (sqrt(sq) + 1e-6))
//
// Bound by HBM: the norm reads every element once; no element can be scaled before that, so the second call reads them
// again and writes the result.  The list goes to the kernel as its argument, so a call copies nothing to the device.  The
// elements are cut into chunks of kGcChunk, a CTA takes a stretch of successive chunks; the second call takes each
// stretch from its end, where the first one left off, which finds up to an L2 full of elements there.
// Squares are added in fp32 over a thread's 32 elements of a chunk and in fp64 from there, in an order that only the
// list and the number of SMs determine.  A thread whose fp32 sum left the range where that is exact to fp32 rounding
// (values above about 1e14, or nothing but values below about 1e-12) adds the same elements again in fp64.
#pragma once
#include "elements.cuh"

namespace oapl {

constexpr int kGcThreads = 256;
constexpr int kGcChunk = 8192;
constexpr int kGcList = 480;       // tensors of a launch
constexpr int kGcSumsPerSm = 8;    // CTAs, each with one partial sum
constexpr int kErrNonfiniteGrad = -7;  // OAPL_ERR_NONFINITE_INPUT

struct GradTensor {
  const void* in;
  void* out;
  int64_t n;
  int32_t first;       // chunks of the list before this tensor's
  uint8_t in_type, out_type, vec;
};
struct GradList {
  GradTensor t[kGcList];
  int32_t count, chunks;
};

// The tensor that holds a chunk.
__device__ __forceinline__ int grad_find(const GradList& l, int chunk) {
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.t[mid].first <= chunk) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// ------------------------------------------------------------------------------------------------ norm
// Sum of squares of a thread's share of a chunk: W words of elements in registers.
template <typename T, int KE, int U>
__device__ __forceinline__ double grad_squares(const T* g, int n) {
  Raw<T, KE> v[U];
  float s = 0.f, top = 0.f;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int i = (j * kGcThreads + (int)threadIdx.x) * KE;
    if (i + KE <= n) v[j].load(g + i);
  }
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int i = (j * kGcThreads + (int)threadIdx.x) * KE;
    if (i + KE <= n) {
      float f[KE];
      v[j].widen(f);
#pragma unroll
      for (int k = 0; k < KE; ++k) {
        s = fmaf(f[k], f[k], s);
        top = fmaxf(top, fabsf(f[k]));
      }
    }
  }
  if (s < 1e29f && (s > 1e-23f || top == 0.f)) return (double)s;
  double w = 0.0;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int i = (j * kGcThreads + (int)threadIdx.x) * KE;
    if (i + KE <= n) {
      float f[KE];
      v[j].widen(f);
#pragma unroll
      for (int k = 0; k < KE; ++k) w = fma((double)f[k], (double)f[k], w);
    }
  }
  return w;
}

template <typename T>
__device__ __forceinline__ double grad_chunk_squares(const GradTensor& t, int64_t at) {
  const T* g = static_cast<const T*>(t.in) + at;
  const int n = (int)(t.n - at < kGcChunk ? t.n - at : kGcChunk);
  constexpr int KE = Elem<T>::kN;
  double s = 0.0;
  if (t.vec) {
    // four vectors of 16-bit elements or eight of fp32, all in flight
    s = grad_squares<T, KE, kGcChunk / kGcThreads / KE>(g, n);
    const int rest = n / KE * KE + (int)threadIdx.x;
    if (rest < n) {
      const double x = Elem<T>::one(g, rest);
      s = fma(x, x, s);
    }
  } else {
    for (int i = 0; i < n; i += 8 * kGcThreads) s += grad_squares<T, 1, 8>(g + i, n - i);
  }
  return s;
}

__global__ void __launch_bounds__(kGcThreads, 4) grad_norm_kernel(const __grid_constant__ GradList l, double* part) {
  __shared__ double sh[kGcThreads / 32];
  const int64_t b = blockIdx.x, nb = gridDim.x;
  const int lo = (int)(b * l.chunks / nb), hi = (int)((b + 1) * l.chunks / nb);
  double s = 0.0;
  int k = lo < hi ? grad_find(l, lo) : 0;
  for (int c = lo; c < hi; ++c) {
    while (k + 1 < l.count && l.t[k + 1].first <= c) ++k;
    const GradTensor& t = l.t[k];
    const int64_t at = (int64_t)(c - t.first) * kGcChunk;
    if (t.in_type == 0) s += grad_chunk_squares<__nv_bfloat16>(t, at);
    else if (t.in_type == 1) s += grad_chunk_squares<__half>(t, at);
    else s += grad_chunk_squares<float>(t, at);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < kGcThreads / 32; ++w) t += sh[w];
    part[b] = t;
  }
}

__global__ void __launch_bounds__(kGcThreads) grad_norm_join_kernel(const double* part, int n, float scale, float* sq_norm,
                                                                    float* norm, int32_t* status) {
  __shared__ double sh[kGcThreads / 32];
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += kGcThreads) s += part[i];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < kGcThreads / 32; ++w) t += sh[w];
    t *= (double)scale * (double)scale;
    if (sq_norm) *sq_norm = (float)t;
    if (norm) *norm = (float)sqrt(t);
    if (status && !(t <= 1.7976931348623157e308)) atomicCAS(status, 0, kErrNonfiniteGrad);
  }
}

// ------------------------------------------------------------------------------------------------ clipping
template <typename TI, typename TO>
__device__ __forceinline__ void grad_scale_chunk(const GradTensor& t, int64_t at, float factor) {
  const TI* g = static_cast<const TI*>(t.in) + at;
  TO* o = static_cast<TO*>(t.out) + at;
  const int n = (int)(t.n - at < kGcChunk ? t.n - at : kGcChunk);
  constexpr int KE = Elem<TI>::kN > Elem<TO>::kN ? Elem<TI>::kN : Elem<TO>::kN;
  int done = 0;
  if (t.vec) {
    constexpr int U = kGcChunk / kGcThreads / KE;
    Raw<TI, KE> v[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = (j * kGcThreads + (int)threadIdx.x) * KE;
      if (i + KE <= n) v[j].load_stream(g + i);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = (j * kGcThreads + (int)threadIdx.x) * KE;
      if (i + KE <= n) {
        float f[KE];
        v[j].widen(f);
#pragma unroll
        for (int k = 0; k < KE; ++k) f[k] *= factor;
        Raw<TO, KE>::store_stream(o + i, f);
      }
    }
    done = n / KE * KE;
  }
#pragma unroll 4
  for (int i = done + (int)threadIdx.x; i < n; i += kGcThreads) Elem<TO>::put(o, i, Elem<TI>::one(g, i) * factor);
}

template <typename TI>
__device__ __forceinline__ void grad_scale_types(const GradTensor& t, int64_t at, float factor) {
  if (t.out_type == 0) grad_scale_chunk<TI, __nv_bfloat16>(t, at, factor);
  else if (t.out_type == 1) grad_scale_chunk<TI, __half>(t, at, factor);
  else grad_scale_chunk<TI, float>(t, at, factor);
}

__global__ void __launch_bounds__(kGcThreads, 4) grad_clip_kernel(const __grid_constant__ GradList l, const float* sq_norm,
                                                               float clip, float scale) {
  __shared__ float sh;
  if (threadIdx.x == 0) {
    const double sq = *sq_norm;
    double f = 1.0;
    if (sq <= 3.4028234663852886e38) f = fmin(1.0, (double)clip / (sqrt(sq) + 1e-6));  // not for inf or NaN
    sh = (float)f * scale;
  }
  __syncthreads();
  const float factor = sh;
  const int64_t b = blockIdx.x, nb = gridDim.x;
  const int lo = (int)(b * l.chunks / nb), hi = (int)((b + 1) * l.chunks / nb);
  int k = lo < hi ? grad_find(l, hi - 1) : 0;
  for (int c = hi - 1; c >= lo; --c) {
    while (l.t[k].first > c) --k;
    const GradTensor& t = l.t[k];
    if (factor == 1.f && t.in == t.out) continue;  // in place, and nothing changes
    const int64_t at = (int64_t)(c - t.first) * kGcChunk;
    if (t.in_type == 0) grad_scale_types<__nv_bfloat16>(t, at, factor);
    else if (t.in_type == 1) grad_scale_types<__half>(t, at, factor);
    else grad_scale_types<float>(t, at, factor);
  }
}

}  // namespace oapl

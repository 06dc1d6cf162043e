// The norm over a list of gradient tensors, and the list scaled to a largest norm.
//
//     sq = sum (s g)^2 over all elements,      out = s g min(1, c / (sqrt(sq) + 1e-6))
//
// Bound by HBM: the norm reads every element once; no element can be scaled before that, so the second call reads them
// again and writes the result.  The list goes to the kernel as its argument, so a call copies nothing to the device.  The
// elements are cut into chunks of 16 KB that the CTAs take in turn; the second call begins at the end, where the first
// one left off, and finds up to an L2 full of elements there.
// Squares are added in fp32 over a thread's 16 or 32 elements of a chunk and in fp64 from there, in an order that only the
// list and the number of SMs determine.  A thread whose fp32 sum left the range where that is exact to fp32 rounding
// (values above about 1e14, or nothing but values below about 1e-12) adds the same elements again in fp64.
//
// Measured, us: 453 M bf16 elements in 108 tensors, norm 151 (0.94 of the copy rate), clipping to fp32 465 (0.91), to bf16
// 280 (the copy rate); 600 tensors of up to 4100 fp32 elements 18 for both calls after a flush of L2, 14 of them in kernels.
// Loads of the next chunk ahead of this one's sums: 187 to 151.  Tensors off 16-byte boundaries go an element at a time: 100 M
// bf16 elements two bytes off, norm 356 instead of 49, clipping to fp32 217 instead of 115.
#pragma once
#include <type_traits>

#include "elements.cuh"

namespace oapl {

constexpr int kGcThreads = 256;
constexpr int kGcVecs = 4;                                  // 16-byte vectors of a thread that are read together
constexpr int kGcBytes = kGcVecs * kGcThreads * 16;         // of a chunk, in the wider one of its two types
constexpr int kGcList = 960;       // tensors of a launch: 30 KB of its 32 KB of arguments
constexpr int kGcSumsPerSm = 8;    // CTAs, each with one partial sum
constexpr int kErrNonfiniteGrad = -7;  // OAPL_ERR_NONFINITE_INPUT

struct GradTensor {
  const void* in;
  void* out;
  int64_t n;
  int32_t first;       // chunks of the list before this tensor's
  uint8_t in_type, out_type, vec, shift;  // shift: log2 of the elements of a chunk
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
// Sum of squares of a thread's vectors, whatever their type: fp32 where it is exact to fp32 rounding, fp64 otherwise.
template <typename T>
__device__ __forceinline__ double grad_squares(const uint4 (&v)[kGcVecs]) {
  constexpr int KE = Elem<T>::kN;
  float2 s = make_float2(0.f, 0.f);
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < kGcVecs; ++j) {
    float f[KE];
    Elem<T>::widen(v[j], f);
#pragma unroll
    for (int k = 0; k < KE; k += 2) {
      const float2 x = make_float2(f[k], f[k + 1]);
      s = __ffma2_rn(x, x, s);
      top = fmaxf(top, fmaxf(fabsf(x.x), fabsf(x.y)));
    }
  }
  const float sum = s.x + s.y;
  if (sum < 1e29f && (sum > 1e-23f || top == 0.f)) return (double)sum;
  double w = 0.0;
#pragma unroll 1
  for (int j = 0; j < kGcVecs; ++j) {
    const uint4 q = j == 0 ? v[0] : j == 1 ? v[1] : j == 2 ? v[2] : v[3];
    float f[KE];
    Elem<T>::widen(q, f);
#pragma unroll
    for (int k = 0; k < KE; ++k) w = fma((double)f[k], (double)f[k], w);
  }
  return w;
}
__device__ __forceinline__ float grad_one(const void* p, int type, int64_t i) {
  return type == 0 ? Elem<__nv_bfloat16>::one(p, i) : (type == 1 ? Elem<__half>::one(p, i) : Elem<float>::one(p, i));
}

// A thread's vectors of a chunk; elements that they leave out are added up at once.
struct GradShare {
  uint4 v[kGcVecs];
  int type;
};
__device__ __forceinline__ void grad_fetch(const GradList& l, int c, int& k, GradShare& q, double& s) {
  while (k + 1 < l.count && l.t[k + 1].first <= c) ++k;
  const GradTensor& t = l.t[k];
  const int64_t at = (int64_t)(c - t.first) << t.shift;
  const int size = 1 << t.shift, n = t.n - at < size ? (int)(t.n - at) : size;
  const int wide = t.in_type == 2 ? 2 : 1;  // log2 of the bytes of an element
  const uint4* g = reinterpret_cast<const uint4*>(static_cast<const char*>(t.in) + (at << wide));
  const int vecs = t.vec ? n >> (4 - wide) : 0, done = vecs << (4 - wide);
  q.type = t.in_type;
#pragma unroll
  for (int j = 0; j < kGcVecs; ++j) {
    const int i = j * kGcThreads + (int)threadIdx.x;
    q.v[j] = i < vecs ? g[i] : make_uint4(0, 0, 0, 0);
  }
#pragma unroll 1
  for (int i = done + (int)threadIdx.x; i < n; i += kGcThreads) {
    const double x = grad_one(t.in, t.in_type, at + i);
    s = fma(x, x, s);
  }
}
__global__ void __launch_bounds__(kGcThreads, 4) grad_norm_kernel(const __grid_constant__ GradList l, double* part) {
  __shared__ double sh[kGcThreads / 32];
  after_launch_before();
  double s = 0.0;
  int k = grad_find(l, (int)blockIdx.x);
  GradShare now, next;
  grad_fetch(l, (int)blockIdx.x, k, now, s);
  for (int c = blockIdx.x; c < l.chunks; c += gridDim.x) {
    // the next chunk's loads before this one's sums
    if (c + (int)gridDim.x < l.chunks) grad_fetch(l, c + (int)gridDim.x, k, next, s);
    s += now.type == 0   ? grad_squares<__nv_bfloat16>(now.v)
         : now.type == 1 ? grad_squares<__half>(now.v)
                         : grad_squares<float>(now.v);
    now = next;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_down_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    double t = 0.0;
    for (int w = 0; w < kGcThreads / 32; ++w) t += sh[w];
    part[blockIdx.x] = t;
  }
}

__global__ void __launch_bounds__(kGcThreads) grad_norm_join_kernel(const double* part, int n, float scale, float* sq_norm,
                                                                    float* norm, int32_t* status) {
  __shared__ double sh[kGcThreads / 32];
  after_launch_before();
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
    const float root = (float)sqrt(t), square = (float)t;
    if (norm) *norm = root;
    // reported where what the caller gets does not hold the norm: its square leaves fp32 long before it does
    if (status && !(norm ? root <= 3.402823466e38f : square <= 3.402823466e38f)) atomicCAS(status, 0, kErrNonfiniteGrad);
  }
}

// ------------------------------------------------------------------------------------------------ clipping
template <typename TI, typename TO>
__device__ __forceinline__ void grad_scale_chunk(const GradTensor& t, int64_t at, int n, float factor) {
  const TI* g = static_cast<const TI*>(t.in) + at;
  TO* o = static_cast<TO*>(t.out) + at;
  constexpr int KE = Elem<TI>::kN < Elem<TO>::kN ? Elem<TI>::kN : Elem<TO>::kN;  // 16 bytes of the wider type
  constexpr int U = kGcVecs;
  int done = 0;
  if (t.vec) {
    const int vecs = n / KE;
    done = vecs * KE;
    Raw<TI, KE> v[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = j * kGcThreads + (int)threadIdx.x;
      if (i < vecs) v[j].load_stream(g + i * KE);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int i = j * kGcThreads + (int)threadIdx.x;
      if (i < vecs) {
        float f[KE];
        v[j].widen(f);
#pragma unroll
        for (int k = 0; k < KE; ++k) f[k] *= factor;
        Raw<TO, KE>::store_stream(o + i * KE, f);
      }
    }
  }
#pragma unroll 1
  for (int i = done + (int)threadIdx.x; i < n; i += kGcThreads) Elem<TO>::put(o, i, Elem<TI>::one(g, i) * factor);
}

template <typename TI>
__device__ __forceinline__ void grad_scale_types(const GradTensor& t, int64_t at, int n, float factor) {
  if (t.out_type == 0) grad_scale_chunk<TI, __nv_bfloat16>(t, at, n, factor);
  else if (t.out_type == 1) grad_scale_chunk<TI, __half>(t, at, n, factor);
  else grad_scale_chunk<TI, float>(t, at, n, factor);
}

// TI, TO: the types of the whole list, void where it has several.
template <typename TI, typename TO>
__global__ void __launch_bounds__(kGcThreads, 4) grad_clip_kernel(const __grid_constant__ GradList l, const float* sq_norm,
                                                                  const float* norm_of, float clip, float scale) {
  __shared__ float sh;
  if (threadIdx.x == 0) {
    // (the norm itself where it is given: a square is infinite from a norm of 1.8e19 on)
    const double norm = norm_of ? (double)*norm_of : sqrt((double)*sq_norm);
    double f = 1.0;
    if (norm <= 3.4028234663852886e38) f = fmin(1.0, (double)clip / (norm + 1e-6));  // not for inf or NaN
    sh = (float)f * scale;  // (below 1e-38 with fewer bits)
  }
  __syncthreads();
  const float factor = sh;
  const int last = l.chunks - 1 - (int)blockIdx.x;
  int k = grad_find(l, last);
  for (int c = last; c >= 0; c -= gridDim.x) {
    while (l.t[k].first > c) --k;
    const GradTensor& t = l.t[k];
    if (factor == 1.f && t.in == t.out) continue;  // in place, and nothing changes
    const int64_t at = (int64_t)(c - t.first) << t.shift;
    const int size = 1 << t.shift, n = t.n - at < size ? (int)(t.n - at) : size;
    if constexpr (std::is_void<TI>::value) {
      if (t.in_type == 0) grad_scale_types<__nv_bfloat16>(t, at, n, factor);
      else if (t.in_type == 1) grad_scale_types<__half>(t, at, n, factor);
      else grad_scale_types<float>(t, at, n, factor);
    } else {
      grad_scale_chunk<TI, TO>(t, at, n, factor);
    }
  }
}

}  // namespace oapl

// Element types of matrices in memory: 16-byte vectors widened to fp32 and narrowed again, and a few
// instructions that the kernels on such matrices share.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace oapl {

__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ uint4 ldg_stream(const uint4* p) {
  uint4 v;
  asm("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
      : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
      : "l"(p));
  return v;
}

// A launch that follows another one of the same call may begin before that one has ended (host_common.cuh, launch_next):
// it waits here before it touches memory, and lets the launch behind it begin in turn.
__device__ __forceinline__ void after_launch_before() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// Copies to shared memory that need no register.
__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copy_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Element type: kN elements per 16 bytes, widening to fp32 (exact), the packed -inf word.
template <typename T>
struct Elem;
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kN = 8;
  static constexpr uint32_t kNegInf = 0xFF80FF80u;
  static __device__ __forceinline__ void widen(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ float one(const void* p, int64_t i) {
    return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]);
  }
  static __device__ __forceinline__ uint32_t pmax(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t pclamp(uint32_t a, uint32_t low) {  // a NaN stays
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(low));
    return r;
  }
  static __device__ __forceinline__ float pmax_final(uint32_t a) {
    return fmaxf(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint4 narrow(const float (&f)[8]) {
    return make_uint4(pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]),
                      pack_bf16x2(f[6], f[7]));
  }
  static __device__ __forceinline__ void put(void* p, int64_t i, float x) {
    reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  }
};
template <>
struct Elem<__half> {
  static constexpr int kN = 8;
  static constexpr uint32_t kNegInf = 0xFC00FC00u;
  static __device__ __forceinline__ void widen(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      f[2 * i] = t.x;
      f[2 * i + 1] = t.y;
    }
  }
  static __device__ __forceinline__ float one(const void* p, int64_t i) {
    return __half2float(reinterpret_cast<const __half*>(p)[i]);
  }
  static __device__ __forceinline__ uint32_t pmax(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t pclamp(uint32_t a, uint32_t low) {
    uint32_t r;
    asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(low));
    return r;
  }
  static __device__ __forceinline__ float pmax_final(uint32_t a) {
    const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&a));
    return fmaxf(t.x, t.y);
  }
  static __device__ __forceinline__ uint32_t pk(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  static __device__ __forceinline__ uint4 narrow(const float (&f)[8]) {
    return make_uint4(pk(f[0], f[1]), pk(f[2], f[3]), pk(f[4], f[5]), pk(f[6], f[7]));
  }
  static __device__ __forceinline__ void put(void* p, int64_t i, float x) {
    reinterpret_cast<__half*>(p)[i] = __float2half_rn(x);
  }
};
template <>
struct Elem<float> {
  static constexpr int kN = 4;
  static constexpr uint32_t kNegInf = 0xFF800000u;
  static __device__ __forceinline__ void widen(const uint4& v, float (&f)[4]) {
    f[0] = __uint_as_float(v.x);
    f[1] = __uint_as_float(v.y);
    f[2] = __uint_as_float(v.z);
    f[3] = __uint_as_float(v.w);
  }
  static __device__ __forceinline__ float one(const void* p, int64_t i) {
    return reinterpret_cast<const float*>(p)[i];
  }
  static __device__ __forceinline__ uint32_t pmax(uint32_t a, uint32_t b) {
    return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  }
  static __device__ __forceinline__ uint32_t pclamp(uint32_t a, uint32_t low) {
    return __float_as_uint(max_nan(__uint_as_float(a), __uint_as_float(low)));
  }
  static __device__ __forceinline__ float pmax_final(uint32_t a) { return __uint_as_float(a); }
  static __device__ __forceinline__ uint4 narrow(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
  static __device__ __forceinline__ void put(void* p, int64_t i, float x) { reinterpret_cast<float*>(p)[i] = x; }
};

// KE neighbouring elements of a row: 16-byte vectors, 8 bytes, or one element at its natural alignment.  Loading and
// widening are apart, so that several loads can be in flight.
template <typename T, int KE, int BYTES = KE * (int)sizeof(T)>
struct Raw {
  static constexpr int kV = BYTES / 16;
  uint4 v[kV];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] = reinterpret_cast<const uint4*>(p)[i];
  }
  __device__ __forceinline__ void load_stream(const T* p) {
#pragma unroll
    for (int i = 0; i < kV; ++i) v[i] = __ldcs(reinterpret_cast<const uint4*>(p) + i);
  }
  __device__ __forceinline__ void put(T* p) const {  // the bits as they are
#pragma unroll
    for (int i = 0; i < kV; ++i) reinterpret_cast<uint4*>(p)[i] = v[i];
  }
  __device__ __forceinline__ void widen(float (&f)[KE]) const {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      Elem<T>::widen(v[i], *reinterpret_cast<float(*)[Elem<T>::kN]>(&f[i * Elem<T>::kN]));
  }
  static __device__ __forceinline__ void store(T* p, const float (&f)[KE]) {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      reinterpret_cast<uint4*>(p)[i] =
          Elem<T>::narrow(*reinterpret_cast<const float(*)[Elem<T>::kN]>(&f[i * Elem<T>::kN]));
  }
  static __device__ __forceinline__ void store_stream(T* p, const float (&f)[KE]) {
#pragma unroll
    for (int i = 0; i < kV; ++i)
      __stcs(reinterpret_cast<uint4*>(p) + i,
             Elem<T>::narrow(*reinterpret_cast<const float(*)[Elem<T>::kN]>(&f[i * Elem<T>::kN])));
  }
};
template <typename T>
struct Raw<T, 4, 8> {  // half a vector of 16-bit elements, beside a vector of fp32
  uint2 v;
  __device__ __forceinline__ void load(const T* p) { v = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void load_stream(const T* p) { v = __ldcs(reinterpret_cast<const uint2*>(p)); }
  __device__ __forceinline__ void put(T* p) const { *reinterpret_cast<uint2*>(p) = v; }
  __device__ __forceinline__ void widen(float (&f)[4]) const {
    float g[8];
    Elem<T>::widen(make_uint4(v.x, v.y, 0u, 0u), g);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = g[i];
  }
  static __device__ __forceinline__ uint2 narrow(const float (&f)[4]) {
    const float g[8] = {f[0], f[1], f[2], f[3], 0.f, 0.f, 0.f, 0.f};
    const uint4 w = Elem<T>::narrow(g);
    return make_uint2(w.x, w.y);
  }
  static __device__ __forceinline__ void store(T* p, const float (&f)[4]) { *reinterpret_cast<uint2*>(p) = narrow(f); }
  static __device__ __forceinline__ void store_stream(T* p, const float (&f)[4]) {
    __stcs(reinterpret_cast<uint2*>(p), narrow(f));
  }
};
template <typename T, int BYTES>
struct Raw<T, 1, BYTES> {
  T v;
  __device__ __forceinline__ void load(const T* p) { v = *p; }
  __device__ __forceinline__ void load_stream(const T* p) { v = *p; }
  __device__ __forceinline__ void put(T* p) const { *p = v; }
  __device__ __forceinline__ void widen(float (&f)[1]) const { f[0] = Elem<T>::one(&v, 0); }
  static __device__ __forceinline__ void store(T* p, const float (&f)[1]) { Elem<T>::put(p, 0, f[0]); }
};

// 16 bytes that start `off` < 16 bytes into the 32 of lo and hi; off a multiple of the element size.
__device__ __forceinline__ uint4 shift_16(const uint4& lo, const uint4& hi, uint32_t off) {
  // whole words first, two and one at a time, then bits
  const bool two = off & 8u, one = off & 4u;
  const uint32_t a0 = two ? lo.z : lo.x, a1 = two ? lo.w : lo.y, a2 = two ? hi.x : lo.z, a3 = two ? hi.y : lo.w,
                 a4 = two ? hi.z : hi.x, a5 = two ? hi.w : hi.y;
  const uint32_t w0 = one ? a1 : a0, w1 = one ? a2 : a1, w2 = one ? a3 : a2, w3 = one ? a4 : a3, w4 = one ? a5 : a4;
  const uint32_t s = (off & 3u) * 8u;
  return make_uint4(__funnelshift_r(w0, w1, s), __funnelshift_r(w1, w2, s), __funnelshift_r(w2, w3, s),
                    __funnelshift_r(w3, w4, s));
}

// KE neighbouring elements at any alignment: the aligned blocks (of 16 bytes, or 8) that hold them, shifted in registers.
// A block without one of the elements is not touched.
template <typename T, int KE, int BYTES = KE * (int)sizeof(T)>
struct Shifted {
  static constexpr int kV = BYTES / 16;
  uint4 b[kV + 1];
  uint32_t off;  // bytes into the first block
  __device__ __forceinline__ void load(const T* p) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    off = (uint32_t)a & 15u;
    const uint4* q = reinterpret_cast<const uint4*>(a & ~(uintptr_t)15);
#pragma unroll
    for (int i = 0; i < kV; ++i) b[i] = q[i];
    b[kV] = off ? q[kV] : make_uint4(0u, 0u, 0u, 0u);
  }
  __device__ __forceinline__ void raw(Raw<T, KE>& r) const {
#pragma unroll
    for (int i = 0; i < kV; ++i) r.v[i] = shift_16(b[i], b[i + 1], off);
  }
};
template <typename T, int KE>
struct Shifted<T, KE, 8> {
  uint2 b[2];
  uint32_t off;
  __device__ __forceinline__ void load(const T* p) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p);
    off = (uint32_t)a & 7u;
    const uint2* q = reinterpret_cast<const uint2*>(a & ~(uintptr_t)7);
    b[0] = q[0];
    b[1] = off ? q[1] : make_uint2(0u, 0u);
  }
  __device__ __forceinline__ void raw(Raw<T, KE>& r) const {
    const bool one = off & 4u;
    const uint32_t w0 = one ? b[0].y : b[0].x, w1 = one ? b[1].x : b[0].y, w2 = one ? b[1].y : b[1].x;
    const uint32_t s = (off & 3u) * 8u;
    r.v = make_uint2(__funnelshift_r(w0, w1, s), __funnelshift_r(w1, w2, s));
  }
};

}  // namespace oapl

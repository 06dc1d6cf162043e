// What a sampler does to rows of logits before it samples, and its gradient.
//
// For a token v of a row, with c the times it is in the row's answer and `seen` whether it is in the prompt or the answer:
//     z1 = seen ? (z > 0 ? z / r : z r) : z,   z2 = z1 - f c - p [c > 0],   z3 = z2 + its biases,   out = allowed ? z3 : -inf
//     dz = allowed ? (seen ? (z > 0 ? d / r : d r) : d) : 0
//
// Bound by HBM: logits in, result out (over the logits only the vectors that change are touched), and a bit per token of
// the mask.  A CTA takes a slice of a row and keeps one counter per token of the slice in shared memory: it reads the row's
// tokens once, adds up those of its slice there (whole numbers: the order does not matter), and then passes over the
// slice with the counters beside it.  The slice's logits are loaded before the tokens are, so that one latency covers both.
// Few rows are cut into smaller slices, for more CTAs; the tokens are then read by more of them, from L2.
// Tokens with a bias are left out by the pass and written afterwards, each by the thread that holds its first entry in the
// row's list, which adds up the entries in their order: a token may occur there several times.
#pragma once
#include "elements.cuh"

namespace oapl {

constexpr int kAdThreads = 256;
constexpr uint32_t kAdPrompt = 0x80000000u, kAdBiased = 0x40000000u, kAdCount = 0x3FFFFFFFu;
constexpr int kErrBadSpan = -6;   // OAPL_ERR_BAD_SEQ_ORDER
constexpr int kErrBadRow = -5;    // OAPL_ERR_BAD_TARGET

struct AdjustParams {
  const void* z;
  int64_t ld_z;
  int32_t V, N;
  const uint8_t* mask;
  const void* d;       // gradient: of the result
  int64_t ld_d;
  void* out;
  int64_t ld_o;
  const int32_t* tokens;
  int64_t T;
  const int64_t* spans;
  const float *repetition, *frequency, *presence;
  const int64_t* bias_start;
  const int32_t* bias_id;
  const float* bias;
  int64_t biases;
  const uint32_t* allowed;
  int64_t ld_allowed, allowed_rows;
  const int32_t* allowed_row;
  int32_t* status;
  int32_t slices, counters;  // counters: 1 when the slice's words are needed
};

struct AdjustRow {
  float r, f, p;
};
__device__ __forceinline__ float adjust_value(float z, uint32_t w, const AdjustRow& a) {
  if (w & ~kAdBiased) z = z > 0.f ? z / a.r : z * a.r;
  const uint32_t c = w & kAdCount;
  if (c) z = fmaf(-a.f, (float)c, z) - a.p;
  return z;
}
__device__ __forceinline__ float adjust_slope(float d, float z, const AdjustRow& a) { return z > 0.f ? d / a.r : d * a.r; }

// GRAD: the gradient.  OVER: the result goes over the logits.
template <typename T, int KE, int VPT, bool GRAD, bool OVER>
__global__ void __launch_bounds__(kAdThreads) adjust_kernel(AdjustParams p) {
  extern __shared__ __align__(16) uint32_t word[];
  constexpr int kSlice = KE * VPT * kAdThreads;
  constexpr uint32_t kAll = KE == 32 ? 0xFFFFFFFFu : (1u << KE) - 1;
  const int n = (int)(blockIdx.x / (unsigned)p.slices), v0 = (int)(blockIdx.x % (unsigned)p.slices) * kSlice;
  const int len = p.V - v0 < kSlice ? p.V - v0 : kSlice, t = threadIdx.x;
  const T* z = static_cast<const T*>(p.z) + (int64_t)n * p.ld_z + v0;
  const T* d = GRAD ? static_cast<const T*>(p.d) + (int64_t)n * p.ld_d + v0 : z;
  T* out = static_cast<T*>(p.out) + (int64_t)n * p.ld_o + v0;
  const bool live = !p.mask || p.mask[n];
  if (!live) {
    if (GRAD)
      for (int i = t; i < len; i += kAdThreads) Elem<T>::put(out, i, 0.f);
    return;
  }
  // the row of the mask
  const uint32_t* bits = nullptr;
  if (p.allowed) {
    const int64_t at = p.allowed_row ? p.allowed_row[n] : n;
    if (at >= p.allowed_rows) {
      if (t == 0 && p.status) atomicCAS(p.status, 0, kErrBadRow);
    } else if (at >= 0) {
      bits = p.allowed + at * p.ld_allowed;
    }
  }
  Raw<T, KE> v[VPT];
  uint32_t open[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = (j * kAdThreads + t) * KE;
    if (!OVER && i + KE <= len) v[j].load_stream(d + i);
    open[j] = kAll;
    if (bits && i + KE <= len) open[j] = (bits[(v0 + i) >> 5] >> ((v0 + i) & 31)) & kAll;
  }
  AdjustRow a{1.f, 0.f, 0.f};
  if (p.repetition) a.r = p.repetition[n];
  int64_t b0 = 0, b1 = 0;
  if (p.counters) {
    if (p.frequency) a.f = p.frequency[n];
    if (p.presence) a.p = p.presence[n];
    for (int i = t * 4; i < kSlice; i += kAdThreads * 4) *reinterpret_cast<uint4*>(&word[i]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    if (p.spans) {
      const int64_t lo = p.spans[3 * (int64_t)n], mid = p.spans[3 * (int64_t)n + 1], hi = p.spans[3 * (int64_t)n + 2];
      if (lo < 0 || mid < lo || hi < mid || hi > p.T) {
        if (t == 0 && p.status) atomicCAS(p.status, 0, kErrBadSpan);
      } else {
        constexpr int kAhead = 8;
        // without a repetition penalty the prompt does not matter
        for (int64_t i0 = (p.repetition ? lo : mid) + t; i0 < hi; i0 += kAhead * kAdThreads) {
          uint32_t id[kAhead];
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            id[j] = i0 + j * kAdThreads < hi ? (uint32_t)(p.tokens[i0 + j * kAdThreads]) - (uint32_t)v0 : 0xFFFFFFFFu;
#pragma unroll
          for (int j = 0; j < kAhead; ++j)
            if (id[j] < (uint32_t)len) {
              if (i0 + j * kAdThreads < mid) atomicOr(&word[id[j]], kAdPrompt);
              else atomicAdd(&word[id[j]], 1u);
            }
        }
      }
    }
    if (!GRAD && p.bias_start) {
      b0 = p.bias_start[n];
      b1 = p.bias_start[(int64_t)n + 1];
      if (b0 < 0 || b1 < b0 || b1 > p.biases) {
        b0 = b1 = 0;
        if (t == 0 && p.status) atomicCAS(p.status, 0, kErrBadSpan);
      }
      for (int64_t i = b0 + t; i < b1; i += kAdThreads) {
        const uint32_t id = (uint32_t)p.bias_id[i] - (uint32_t)v0;
        if (id < (uint32_t)len) atomicOr(&word[id], kAdBiased);
      }
    }
    __syncthreads();
  }
  const float closed = GRAD ? 0.f : -__int_as_float(0x7F800000);
  // elements i .. i + KE - 1 of the slice, x: of the logits or of d
  auto one = [&](int i, uint32_t w, bool is_open, float x) {
    if (!is_open) {
      Elem<T>::put(out, i, closed);
    } else if (GRAD) {
      Elem<T>::put(out, i, w ? adjust_slope(x, Elem<T>::one(z, i), a) : x);
    } else if (!(w & kAdBiased)) {
      Elem<T>::put(out, i, adjust_value(x, w, a));
    }
  };
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = (j * kAdThreads + t) * KE;
    if (i + KE > len) continue;
    uint32_t w[KE], any = 0;
    if (p.counters) {
      if constexpr (KE == 1) {
        w[0] = word[i];
      } else {
#pragma unroll
        for (int k = 0; k < KE; k += 4) {
          const uint4 q = *reinterpret_cast<const uint4*>(&word[i + k]);
          w[k] = q.x; w[k + 1] = q.y; w[k + 2] = q.z; w[k + 3] = q.w;
        }
      }
#pragma unroll
      for (int k = 0; k < KE; ++k) any |= w[k];
    }
    if (any == 0 && open[j] == kAll) {
      if (!OVER) v[j].put(out + i);
      continue;
    }
    if (open[j] == 0) {
      float f[KE];
#pragma unroll
      for (int k = 0; k < KE; ++k) f[k] = closed;
      Raw<T, KE>::store(out + i, f);
      continue;
    }
    if (OVER) v[j].load(z + i);
    float f[KE];
    v[j].widen(f);
    if (any & kAdBiased) {
#pragma unroll
      for (int k = 0; k < KE; ++k) one(i + k, w[k], open[j] >> k & 1, f[k]);
      continue;
    }
#pragma unroll
    for (int k = 0; k < KE; ++k) {
      if (any) {
        if (GRAD) {
          if (w[k]) f[k] = adjust_slope(f[k], Elem<T>::one(z, i + k), a);
        } else {
          f[k] = adjust_value(f[k], w[k], a);
        }
      }
      if (!(open[j] >> k & 1)) f[k] = closed;
    }
    Raw<T, KE>::store(out + i, f);
  }
  if (KE > 1) {  // what is left of the row
    const int i = len / KE * KE + t;
    if (i < len) {
      const bool is_open = !bits || (bits[(v0 + i) >> 5] >> ((v0 + i) & 31) & 1);
      one(i, p.counters ? word[i] : 0u, is_open, Elem<T>::one(d, i));
    }
  }
  if constexpr (!GRAD) {
    for (int64_t i = b0 + t; i < b1; i += kAdThreads) {
      const int32_t id = p.bias_id[i];
      const uint32_t at = (uint32_t)id - (uint32_t)v0;
      if (at >= (uint32_t)len) continue;
      if (bits && !(bits[id >> 5] >> (id & 31) & 1)) continue;
      bool mine = true;
      for (int64_t k = b0; k < i && mine; ++k) mine = p.bias_id[k] != id;
      if (!mine) continue;
      float sum = 0.f;
      for (int64_t k = i; k < b1; ++k)
        if (p.bias_id[k] == id) sum += p.bias[k];
      Elem<T>::put(out, at, adjust_value(Elem<T>::one(z, at), word[at], a) + sum);
    }
  }
}

}  // namespace oapl

// What a sampler does to rows of logits before it samples, and its gradient.
//
// For a token v of a row, with c the times it is in the row's answer and `seen` whether it is in the prompt or the answer:
//     z1 = seen ? (z > 0 ? z / r : z r) : z,   z2 = z1 - f c - p [c > 0],   z3 = z2 + its biases,   out = allowed ? z3 : -inf
//     dz = allowed ? (seen ? (z > 0 ? d / r : d r) : d) : 0
//
// Bound by HBM: logits in, result out (over the logits only the vectors with a token that is not allowed are touched, and
// the tokens that change), and a bit per token of the mask.  A CTA takes a slice of a row:
//   1. its logits' loads are started, which the steps up to 3 then cover;
//   2. it reads the row's tokens: those of its slice are marked in a bitmap in shared memory, listed when they are met for
//      the first time, and counted (whole numbers and marks: the order does not matter).  Tokens with a bias are marked too;
//   3. the logits of the listed tokens are loaded, a token a thread;
//   4. the slice is copied, closed tokens overwritten;
//   5. behind a barrier the listed tokens' values are stored over what the copy left there, and those of tokens with a
//      bias by the thread that holds the first of a token's biases and adds them up in their order.
// So the copy does not test for tokens that change.  (When it did, with a counter per token beside each vector, a token in
// one of a warp's 256 places cost the warp eight divisions: 2048 x 152064 bf16, gradient 472 us; %GRAD% like this.)
// Rows need not start on 16-byte boundaries: where the two sides are off by the same number of bytes, vectors begin at the
// slice's first boundary (KE > 1); rows off by different numbers go an element at a time (KE == 1).
// Few rows are cut into smaller slices, for more CTAs; the tokens are then read by more of them, from L2.
#pragma once
#include "elements.cuh"

namespace oapl {

constexpr int kAdThreads = 256;
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
  int32_t slices;
  int32_t history, biased;  // whether there are tokens to read, biases to add
};

struct AdjustRow {
  float r, f, p;
};
__device__ __forceinline__ float adjust_slope(float d, float z, const AdjustRow& a) { return z > 0.f ? d / a.r : d * a.r; }
__device__ __forceinline__ float adjust_value(float z, bool seen, uint32_t c, const AdjustRow& a) {
  if (seen) z = z > 0.f ? z / a.r : z * a.r;
  if (c) z = fmaf(-a.f, (float)c, z) - a.p;
  return z;
}

// Shared memory of a CTA whose rows have tokens or biases, for a slice of `n` tokens.  The gradient counts nothing; over
// the logits it keeps its results instead, by their place in the list.
template <bool WORDS>
struct AdjustShared {
  uint32_t* count;    // of the list
  uint32_t* seen;     // [n / 32]
  uint32_t* biased;   // [n / 32]
  uint32_t* word;     // [n] times in the answer, or results
  uint16_t* list;     // [n] tokens of the prompt and the answer, each once
  static constexpr int bytes(int n) { return 16 + n / 4 + (WORDS ? n * 4 : 0) + n * 2; }
  __device__ __forceinline__ AdjustShared(uint32_t* base, int n) {
    count = base;
    seen = count + 4;
    biased = seen + n / 32;
    word = biased + n / 32;
    list = reinterpret_cast<uint16_t*>(word + (WORDS ? n : 0));
  }
};

// GRAD: the gradient.  OVER: the result goes over the logits.
template <typename T, int KE, int VPT, bool GRAD, bool OVER>
__global__ void __launch_bounds__(kAdThreads) adjust_kernel(AdjustParams p) {
  extern __shared__ __align__(16) uint32_t ad_smem[];
  constexpr int kSlice = KE * VPT * kAdThreads;
  static_assert(kSlice <= 65536, "a place in the list has 16 bits");
  constexpr uint32_t kAll = (1u << KE) - 1;
  const int n = (int)(blockIdx.x / (unsigned)p.slices), v0 = (int)(blockIdx.x % (unsigned)p.slices) * kSlice;
  const int len = p.V - v0 < kSlice ? p.V - v0 : kSlice, t = threadIdx.x;
  const T* z = static_cast<const T*>(p.z) + (int64_t)n * p.ld_z + v0;
  const T* d = GRAD ? static_cast<const T*>(p.d) + (int64_t)n * p.ld_d + v0 : z;
  T* out = static_cast<T*>(p.out) + (int64_t)n * p.ld_o + v0;
  if (p.mask && !p.mask[n]) {
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
      bits = p.allowed + at * p.ld_allowed + (v0 >> 5);
    }
  }
  auto is_open = [&](int i) { return !bits || (bits[i >> 5] >> (i & 31) & 1); };
  // elements before the first vector
  int head = KE == 1 ? 0 : (int)(-(reinterpret_cast<uintptr_t>(out) / sizeof(T)) & (KE - 1));
  head = head < len ? head : len;
  Raw<T, KE> v[VPT];
  uint32_t open[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = head + (j * kAdThreads + t) * KE;
    const bool in = i + KE <= len;
    if ((!OVER || GRAD) && in) v[j].load_stream(d + i);
    open[j] = kAll;
    if (bits && in) {
      const int sh = i & 31;
      const uint32_t low = bits[i >> 5], high = sh + KE > 32 ? bits[(i >> 5) + 1] : 0u;
      open[j] = __funnelshift_r(low, high, sh) & kAll;
    }
  }
  const AdjustShared<!GRAD || OVER> sm(ad_smem, kSlice);
  const bool special = p.history || p.biased;
  constexpr int kFirst = 2;  // listed tokens of a thread whose loads go ahead of the copy
  AdjustRow a{1.f, 0.f, 0.f};
  int64_t b0 = 0, b1 = 0;
  int listed = 0;
  float x[kFirst], g[kFirst];
  if (special) {
    constexpr int kAhead = 4;
    if (p.repetition) a.r = p.repetition[n];
    if (!GRAD && p.frequency) a.f = p.frequency[n];
    if (!GRAD && p.presence) a.p = p.presence[n];
    int64_t lo = 0, mid = 0, hi = 0;
    if (p.history) {
      lo = p.spans[3 * (int64_t)n], mid = p.spans[3 * (int64_t)n + 1], hi = p.spans[3 * (int64_t)n + 2];
      if (lo < 0 || mid < lo || hi < mid || hi > p.T) {
        lo = mid = hi = 0;
        if (t == 0 && p.status) atomicCAS(p.status, 0, kErrBadSpan);
      }
      if (!p.repetition) lo = mid;  // without this penalty the prompt does not matter
    }
    if (p.biased) {
      b0 = p.bias_start[n];
      b1 = p.bias_start[(int64_t)n + 1];
      if (b0 < 0 || b1 < b0 || b1 > p.biases) {
        b0 = b1 = 0;
        if (t == 0 && p.status) atomicCAS(p.status, 0, kErrBadSpan);
      }
    }
    // the list's length, marks, and counters
    for (int i = t * 4; i < 4 + kSlice / 16 + (GRAD ? 0 : kSlice); i += kAdThreads * 4)
      *reinterpret_cast<uint4*>(&sm.count[i]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int64_t i0 = lo + t; i0 < hi; i0 += kAhead * kAdThreads) {
      uint32_t id[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        id[j] = i0 + j * kAdThreads < hi ? (uint32_t)(p.tokens[i0 + j * kAdThreads]) - (uint32_t)v0 : 0xFFFFFFFFu;
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (id[j] < (uint32_t)len) {
          const uint32_t bit = 1u << (id[j] & 31);
          uint32_t* word = &sm.seen[id[j] >> 5];
          if (!(*reinterpret_cast<volatile uint32_t*>(word) & bit) && !(atomicOr(word, bit) & bit))
            sm.list[atomicAdd(sm.count, 1u)] = (uint16_t)id[j];
          if (!GRAD && i0 + j * kAdThreads >= mid) atomicAdd(&sm.word[id[j]], 1u);
        }
    }
    for (int64_t i = b0 + t; i < b1; i += kAdThreads) {
      const uint32_t id = (uint32_t)p.bias_id[i] - (uint32_t)v0;
      if (id < (uint32_t)len) atomicOr(&sm.biased[id >> 5], 1u << (id & 31));
    }
    __syncthreads();
    listed = (int)*sm.count;
#pragma unroll
    for (int j = 0; j < kFirst; ++j) {
      const int i = j * kAdThreads + t;
      if (i < listed) {
        x[j] = Elem<T>::one(z, sm.list[i]);
        if (GRAD) g[j] = Elem<T>::one(d, sm.list[i]);
      }
    }
    if (GRAD && OVER) {
      // the copy overwrites the logits that decide on the factor: the results first
      for (int i = kFirst * kAdThreads + t; i < listed; i += kAdThreads) {
        const int at = sm.list[i];
        sm.word[i] = __float_as_uint(adjust_slope(Elem<T>::one(d, at), Elem<T>::one(z, at), a));
      }
      __syncthreads();
    }
  }
  const float closed = GRAD ? 0.f : -__int_as_float(0x7F800000);
  if (OVER && !GRAD) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int i = head + (j * kAdThreads + t) * KE;
      if (open[j] != kAll && open[j]) v[j].load(z + i);
    }
  }
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = head + (j * kAdThreads + t) * KE;
    if (i + KE > len) continue;
    if (open[j] == kAll) {
      if (!OVER || GRAD) v[j].put(out + i);
      continue;
    }
    float f[KE];
    if (open[j]) v[j].widen(f);
#pragma unroll
    for (int k = 0; k < KE; ++k)
      if (!(open[j] >> k & 1)) f[k] = closed;
    Raw<T, KE>::store(out + i, f);
  }
  if (KE > 1 && t < 2 * KE) {  // what is left before and behind the vectors
    const int i = t < KE ? t : head + (len - head) / KE * KE + t - KE;
    if (i < (t < KE ? head : len)) {
      if (!is_open(i)) Elem<T>::put(out, i, closed);
      else if (!OVER || GRAD) out[i] = d[i];
    }
  }
  if (!special) return;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kFirst; ++j) {
    const int i = j * kAdThreads + t;
    if (i < listed) {
      const int at = sm.list[i];
      if (is_open(at)) {
        if (GRAD) Elem<T>::put(out, at, adjust_slope(g[j], x[j], a));
        else if (!(sm.biased[at >> 5] >> (at & 31) & 1)) Elem<T>::put(out, at, adjust_value(x[j], true, sm.word[at], a));
      }
    }
  }
  for (int i = kFirst * kAdThreads + t; i < listed; i += kAdThreads) {
    const int at = sm.list[i];
    if (!is_open(at)) continue;
    if (GRAD)
      Elem<T>::put(out, at, OVER ? __uint_as_float(sm.word[i]) : adjust_slope(Elem<T>::one(d, at), Elem<T>::one(z, at), a));
    else if (!(sm.biased[at >> 5] >> (at & 31) & 1))
      Elem<T>::put(out, at, adjust_value(Elem<T>::one(z, at), true, sm.word[at], a));
  }
  if constexpr (!GRAD) {
    for (int64_t i = b0 + t; i < b1; i += kAdThreads) {
      const int32_t id = p.bias_id[i];
      const uint32_t at = (uint32_t)id - (uint32_t)v0;
      if (at >= (uint32_t)len || !is_open((int)at)) continue;
      bool first = true;
      for (int64_t k = b0; k < i && first; ++k) first = p.bias_id[k] != id;
      if (!first) continue;
      float sum = 0.f;
      for (int64_t k = i; k < b1; ++k)
        if (p.bias_id[k] == id) sum += p.bias[k];
      const bool seen = sm.seen[at >> 5] >> (at & 31) & 1;
      Elem<T>::put(out, at, adjust_value(Elem<T>::one(z, at), seen, sm.word[at], a) + sum);
    }
  }
}

}  // namespace oapl

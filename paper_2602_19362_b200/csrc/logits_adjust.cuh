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
// one of a warp's 256 places cost the warp eight divisions: 2048 x 152064 bf16, gradient 472 us; 235 like this.)
// Rows need not start on 16-byte boundaries: where the two sides are off by the same number of bytes, vectors begin at the
// slice's first boundary (KE > 1); rows off by different numbers go an element at a time (KE == 1).
// Few rows are cut into smaller slices, for more CTAs; the tokens are then read by more of them, from L2.
//
// Measured, us: the gradient 2048 x 152064 bf16, 300 tokens of prompt and up to 1024 of answer, 232 (0.83 of the copy
// rate); the adjustment with all penalties and eight biases 299 (0.65), with a mask 349, rows off 16-byte boundaries 318;
// a mask alone, apart, 199, with sides off by different amounts 449; answers of up to 16384 tokens, each row its own, 661 and
// the gradient 510; one row of 152064 fp32 with 8000 tokens and 40 biases 6.0 on the device; a mask over 64 x 128256 bf16 8.0.
// What is left is latency: spans, tokens and listed logits are loads that wait for one another, with barriers between them, and
// six CTAs (forward) to cover them; issue slots are a quarter busy.  With long answers it is the tokens, which every slice of a
// row reads and tests: a list of them by slice, made once for a row, would be read once.
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

// Shared memory of a CTA whose rows have tokens or biases, for a slice of `n` tokens: n / 2 words to count in, 16 bits a
// token, or 32 bits for half of the slice at a time where an answer is too long for that.  The gradient counts nothing;
// over the logits it keeps its results instead, by their place in the list, a word each.
constexpr int kAdBiases = 256;  // biases of a row that are kept in shared memory; more are read again where they are
template <int WORDS>
struct AdjustShared {
  uint32_t* listed;   // length of the list
  uint32_t* seen;     // [n / 32]
  uint32_t* biased;   // [n / 32]
  uint32_t* word;     // [WORDS n / 2]
  uint16_t* list;     // [n] tokens of the prompt and the answer, each once
  int32_t* bias_id;   // [kAdBiases] the row's first biases
  float* bias;
  static constexpr int bytes(int n) { return 16 + n / 4 + WORDS * n * 2 + n * 2 + kAdBiases * 8; }
  __device__ __forceinline__ AdjustShared(uint32_t* base, int n) {
    listed = base;
    seen = listed + 4;
    biased = seen + n / 32;
    word = biased + n / 32;
    list = reinterpret_cast<uint16_t*>(word + WORDS * n / 2);
    bias_id = reinterpret_cast<int32_t*>(list + n);
    bias = reinterpret_cast<float*>(bias_id + kAdBiases);
  }
};
constexpr int64_t kAdShort = 65535;  // tokens of an answer that 16 bits can count

// Overwrites the elements of a vector that are not open, as words: `what` holds the closing value in each element.
template <typename T, int KE>
__device__ __forceinline__ void adjust_close(Raw<T, KE>& v, uint32_t open, uint32_t what) {
  if constexpr (KE == 1) {
    if (!(open & 1u)) {
      const uint16_t half = (uint16_t)what;
      v.v = sizeof(T) == 2 ? *reinterpret_cast<const T*>(&half) : *reinterpret_cast<const T*>(&what);
    }
  } else {
    uint32_t* w = reinterpret_cast<uint32_t*>(&v.v[0]);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(T) == 4) {
        w[k] = open >> k & 1 ? w[k] : what;
      } else {
        const uint32_t keep = (open >> (2 * k) & 1 ? 0x0000FFFFu : 0u) | (open >> (2 * k + 1) & 1 ? 0xFFFF0000u : 0u);
        w[k] = (w[k] & keep) | (what & ~keep);
      }
    }
  }
}

// GRAD: the gradient.  OVER: the result goes over the logits.
template <typename T, int KE, int VPT, bool GRAD, bool OVER>
__global__ void __launch_bounds__(kAdThreads) adjust_kernel(AdjustParams p) {
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
  // the slice's part of it, in shared memory
  extern __shared__ __align__(16) uint32_t ad_smem[];
  if (bits) {
    for (int i = t; i < (len + 31) / 32; i += kAdThreads) copy_async_4(smem_u32(&ad_smem[i]), bits + i);
    copy_async_commit();
  }
  auto is_open = [&](int i) { return !bits || (ad_smem[i >> 5] >> (i & 31) & 1); };
  // elements before the first vector
  int head = KE == 1 ? 0 : (int)(-(reinterpret_cast<uintptr_t>(out) / sizeof(T)) & (KE - 1));
  head = head < len ? head : len;
  Raw<T, KE> v[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = head + (j * kAdThreads + t) * KE;
    if ((!OVER || GRAD) && i + KE <= len) v[j].load_stream(d + i);
  }
  constexpr int kWords = !GRAD ? 1 : OVER ? 2 : 0;
  const AdjustShared<kWords> sm(ad_smem + kSlice / 32 + 4, kSlice);
  const bool special = p.history || p.biased;
  AdjustRow a{1.f, 0.f, 0.f};
  int64_t lo = 0, mid = 0, hi = 0, b0 = 0, b1 = 0;
  if (special) {
    if (p.repetition) a.r = p.repetition[n];
    if (!GRAD && p.frequency) a.f = p.frequency[n];
    if (!GRAD && p.presence) a.p = p.presence[n];
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
  }
  const bool narrow = GRAD || hi - mid <= kAdShort;
  // Marks, lists and counts the row's tokens among those at from .. from + size of the slice.
  auto gather = [&](int from, int size) {
    constexpr int kAhead = 4;
    const uint32_t base = (uint32_t)v0 + (uint32_t)from;
    for (int i = t * 4; i < 4 + kSlice / 16 + (GRAD ? 0 : kSlice / 2); i += kAdThreads * 4)
      *reinterpret_cast<uint4*>(&sm.listed[i]) = make_uint4(0, 0, 0, 0);
    __syncthreads();
    for (int64_t i0 = lo + t; i0 < hi; i0 += kAhead * kAdThreads) {
      uint32_t id[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        id[j] = i0 + j * kAdThreads < hi ? (uint32_t)(p.tokens[i0 + j * kAdThreads]) - base : 0xFFFFFFFFu;
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (id[j] < (uint32_t)size) {
          const uint32_t bit = 1u << (id[j] & 31);
          uint32_t* word = &sm.seen[id[j] >> 5];
          if (!(*reinterpret_cast<volatile uint32_t*>(word) & bit) && !(atomicOr(word, bit) & bit))
            sm.list[atomicAdd(sm.listed, 1u)] = (uint16_t)id[j];
          if (!GRAD && i0 + j * kAdThreads >= mid) {
            if (narrow) atomicAdd(&sm.word[id[j] >> 1], id[j] & 1 ? 65536u : 1u);
            else atomicAdd(&sm.word[id[j]], 1u);
          }
        }
    }
    for (int64_t i = b0 + t; i < b1; i += kAdThreads) {
      const int32_t token = p.bias_id[i];
      const uint32_t id = (uint32_t)token - base;
      if (id < (uint32_t)size) atomicOr(&sm.biased[id >> 5], 1u << (id & 31));
      if (i - b0 < kAdBiases) {
        sm.bias_id[i - b0] = token;
        sm.bias[i - b0] = p.bias[i];
      }
    }
    __syncthreads();
    return (int)*sm.listed;
  };
  auto counted = [&](int at) { return narrow ? (sm.word[at >> 1] >> (at & 1) * 16) & 0xFFFFu : sm.word[at]; };
  // Stores the value of a token of the list, x and g: its logit and its gradient.
  auto settle = [&](int from, int at, float x, float g) {
    if (!is_open(from + at)) return;
    if (GRAD) Elem<T>::put(out, from + at, adjust_slope(g, x, a));
    else if (!(sm.biased[at >> 5] >> (at & 31) & 1)) Elem<T>::put(out, from + at, adjust_value(x, true, counted(at), a));
  };
  auto settle_rest = [&](int from, int size, int first, int listed) {
    for (int i = first + t; i < listed; i += kAdThreads) {
      const int at = sm.list[i];
      if (GRAD && OVER) {
        if (is_open(from + at)) Elem<T>::put(out, from + at, __uint_as_float(sm.word[i]));
      } else {
        settle(from, at, Elem<T>::one(z, from + at), GRAD ? Elem<T>::one(d, from + at) : 0.f);
      }
    }
    if constexpr (!GRAD) {
      const int count = (int)(b1 - b0), kept = count < kAdBiases ? count : kAdBiases;
      for (int i = t; i < count; i += kAdThreads) {
        const int32_t id = i < kAdBiases ? sm.bias_id[i] : p.bias_id[b0 + i];
        const uint32_t at = (uint32_t)id - (uint32_t)v0 - (uint32_t)from;
        if (at >= (uint32_t)size) continue;
        const float logit = Elem<T>::one(z, from + at);
        const bool shown = is_open(from + (int)at);
        // whether an entry before this one has the token, and the sum of this one and those behind it
        bool first_entry = true;
        float sum = 0.f;
#pragma unroll 4
        for (int k = 0; k < kept; ++k) {
          const bool same = sm.bias_id[k] == id;
          first_entry = first_entry && !(same && k < i);
          if (same && k >= i) sum += sm.bias[k];
        }
        for (int k = kAdBiases; k < count; ++k)
          if (p.bias_id[b0 + k] == id) {
            first_entry = first_entry && k >= i;
            if (k >= i) sum += p.bias[b0 + k];
          }
        if (!first_entry || !shown) continue;
        const bool seen = sm.seen[at >> 5] >> (at & 31) & 1;
        Elem<T>::put(out, from + at, adjust_value(logit, seen, counted((int)at), a) + sum);
      }
    }
  };
  constexpr int kFirst = 2;  // listed tokens of a thread whose loads go ahead of the copy
  int listed = 0;
  float x[kFirst], g[kFirst];
  if (special && narrow) {
    listed = gather(0, len);
#pragma unroll
    for (int j = 0; j < kFirst; ++j) {
      const int i = j * kAdThreads + t;
      if (i < listed) {
        x[j] = Elem<T>::one(z, sm.list[i]);
        g[j] = GRAD ? Elem<T>::one(d, sm.list[i]) : 0.f;
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
  if (bits) {
    copy_async_wait_all();
    __syncthreads();
  }
  uint32_t open[VPT];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int i = head + (j * kAdThreads + t) * KE;
    open[j] = kAll;
    if (bits && i + KE <= len) {
      // (the word behind the slice's last one is there, whatever it holds)
      open[j] = __funnelshift_r(ad_smem[i >> 5], ad_smem[(i >> 5) + 1], i & 31) & kAll;
      if (OVER && !GRAD && open[j] != kAll && open[j]) v[j].load(z + i);
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
    adjust_close<T, KE>(v[j], open[j], GRAD ? 0u : Elem<T>::kNegInf);
    v[j].put(out + i);
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
  if (narrow) {
#pragma unroll
    for (int j = 0; j < kFirst; ++j)
      if (j * kAdThreads + t < listed) settle(0, sm.list[j * kAdThreads + t], x[j], g[j]);
    settle_rest(0, len, kFirst * kAdThreads, listed);
  } else {
    for (int from = 0; from < len; from += kSlice / 2) {
      const int size = len - from < kSlice / 2 ? len - from : kSlice / 2;
      listed = gather(from, size);
      settle_rest(from, size, 0, listed);
      __syncthreads();
    }
  }
}

}  // namespace oapl

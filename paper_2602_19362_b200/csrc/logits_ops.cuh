// Log-probabilities of given tokens, entropy and top alternatives from logits in memory, and the
// gradient of all of them with respect to the logits.
//
// Forward, one pass over a row (z: the row's logits, a: the caller's factor):
//     x_v = a log2(e) z_v - R,  S = sum_v 2^x_v,  T = sum_v 2^x_v x_v      (R: a reference near the maximum)
//     lse = R ln 2 + ln S,   ln p_t = x_t ln 2 - ln S,   entropy = ln S - ln 2 T / S.
// The entropy is formed from sums relative to R.  R is a logit of the row, at most 8 bits below the maximum: where it
// is k bits below, the row holds a second logit with 2^-k of the largest one's weight and an entropy to match, and
// where the maximum stands alone R is the maximum and neither ln S nor ln 2 T / S is large.  What is left is an
// absolute error of a few 2^-24 (two logits 0.5 to 40 bits apart: at most 1.2e-7), so an entropy below about 1e-6 keeps
// no digits.  Sums are fp32: a thread adds up to V / 256 terms to each of two lanes, the rest are trees.
//
// What bounds it: HBM.  At the copy rate an SM has to take 11.5 16-bit logits a cycle and can issue 128 lane
// instructions, 16 of them exponentials; the pass takes about seven per logit.  So the reference R is moved only
// when a batch's maximum exceeds it by 2^8 (no rescaling in the steady state), masked logits are dealt with two
// at a time, and sums and products are two wide.  The top alternatives cost the pass nothing but the group
// maxima that it needs anyway: see top-K below.
// Measured, 4096 rows of 152064 bf16 logits (1.25 GB), single calls: 189 us without alternatives, the copy rate;
// 209 us with eight, where every row ends in a chain of short waits.  Calls in a row, at the power limit: 216 and
// 236.  One row with twenty: 8.0 us.  Rows with fewer finite logits than alternatives (constrained decoding) are read
// twice, see top_by_lists: 4096 such rows 403 us; 64 rows of 128256 fp32 with five, 19.4 us against 10.9, and as much
// when a hundred logits are finite, since no part of a split row then holds enough.
//
// A row goes to a cluster of 1, 2, 4 or 8 CTAs (few rows: the row is split and joined through
// distributed shared memory, so a call is always a single launch without a workspace).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sm100_ptx.cuh"

namespace oapl {

constexpr int kLgThreads = 256;
constexpr int kLgUnroll = 4;       // 16-byte vectors that a thread loads together (a batch)
constexpr int kLgMaxGroups = 32;   // groups of a thread whose maxima are kept for the top alternatives
constexpr int kLgMaxTop = 32;
constexpr int kLgMaxCluster = 8;
constexpr int kErrBadTarget = -5;  // OAPL_ERR_BAD_TARGET
constexpr int kErrNonfinite = -7;  // OAPL_ERR_NONFINITE_INPUT

struct LogitsParams {
  const void* z;
  int64_t ld;  // elements
  int32_t V;
  int32_t N;
  const int32_t* targets;
  const uint8_t* mask;
  float scale;
  // forward
  float clamp;         // see logits_fwd_kernel
  uint32_t clamp_pk;   // packed in the logits' type
  float* token_logp;
  float* token_entropy;
  float* token_lse;
  float* top_logp;
  int32_t* top_id;
  int32_t K;
  int32_t per;    // batches of a group whose maxima are kept
  int32_t slots;  // the most groups that a warp forms
  int32_t* status;
  // backward
  const float* lse;
  const float* entropy;
  const float* g_logp;
  const float* g_entropy;
  const float* g_top;
  const int32_t* ids;
  void* dz;
  int64_t ld_d;
};

// ------------------------------------------------------------------------------------ small pieces
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

// Running sums of one thread.  x = c z - R, c = a log2(e): the reference R is a number of its own in units
// of log2, not a rounded product that stands for a logit, so one multiply-add gives x with one rounding.
struct RowSums {
  float R;
  float2 s, t;  // two lanes each: sum 2^x and sum 2^x x
};
struct RowTotal {
  float R, s, t, m;  // m: the largest logit, clamped
};

constexpr float kLgFloor = -200.f;  // 2^x is 0 in fp32 below this
constexpr float kLgMove = 8.f;      // the reference follows when a maximum exceeds it by 2^8

__device__ __forceinline__ void row_move(RowSums& r, float to) {
  // x + d in place of x: 2^x turns into 2^x 2^d, and 2^x x into (x + d) 2^x 2^d
  const float d = fmaxf(r.R - to, kLgFloor);
  const float f = ex2_approx(d);
  r.t = make_float2(f * fmaf(d, r.s.x, r.t.x), f * fmaf(d, r.s.y, r.t.y));
  r.s = make_float2(f * r.s.x, f * r.s.y);
  r.R = to;
}

// The two-wide forms are the compiler's own: with 64-bit asm operands it copied every pair.
template <int KN>
__device__ __forceinline__ void row_add(RowSums& r, const float (&f)[KN], float c) {
  const float2 nr = make_float2(-r.R, -r.R), cc = make_float2(c, c);
#pragma unroll
  for (int i = 0; i < KN; i += 2) {
    const float2 x = __ffma2_rn(make_float2(f[i], f[i + 1]), cc, nr);
    const float2 e = make_float2(ex2_approx(x.x), ex2_approx(x.y));
    r.s = __fadd2_rn(r.s, e);
    r.t = __ffma2_rn(e, x, r.t);
  }
}

// A float as a whole number of the same order.
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t u = __float_as_uint(v);
  return u ^ (uint32_t(int32_t(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ float warp_max(float v) {  // no NaN
  return from_ordered(__reduce_max_sync(0xffffffffu, ordered(v)));
}

// Sums brought to the reference R.
__device__ __forceinline__ void row_to(RowTotal& a, float R) {
  const float d = fmaxf(a.R - R, kLgFloor), f = ex2_approx(d);
  a.t = f * fmaf(d, a.s, a.t);
  a.s = f * a.s;
  a.R = R;
}
// The lanes' sums joined; every lane adds the same pairs, so all get the same bits.
__device__ __forceinline__ RowTotal row_join_warp(RowTotal a) {
  row_to(a, warp_max(a.R));
  a.m = warp_max(a.m);
#pragma unroll 1
  for (int o = 16; o > 0; o >>= 1) {
    a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
    a.t += __shfl_xor_sync(0xffffffffu, a.t, o);
  }
  return a;
}
// The first n <= 32 sums of a list joined, by every warp.
__device__ __forceinline__ RowTotal row_join_list(const RowTotal* list, int n) {
  const int lane = threadIdx.x & 31;
  RowTotal a = list[lane < n ? lane : 0];
  if (lane >= n) a.s = a.t = 0.f;
  return row_join_warp(a);
}

// Order of the alternatives: larger logit first, then the lower index.  0 = no entry.
__device__ __forceinline__ uint64_t top_key(float v, uint32_t idx) {
  return (uint64_t(ordered(v + 0.f)) << 32) | (0xFFFFFFFFu - idx);  // -0 counts as +0
}
__device__ __forceinline__ float top_value(uint64_t key) { return from_ordered(uint32_t(key >> 32)); }

// A warp's best entries, lane i the i-th best: insert `key` (uniform over the warp).
__device__ __forceinline__ void top_insert(uint64_t& mine, uint64_t key, int lane) {
  const uint32_t better = __ballot_sync(0xffffffffu, mine > key);
  const int pos = __popc(better);  // the list is sorted, so `better` is a prefix
  const uint64_t up = __shfl_up_sync(0xffffffffu, mine, 1);
  if (lane == pos) mine = key;
  if (lane > pos) mine = up;
}

// out[rank] = the K best of entries[0..M), whose keys are distinct; the rest of out is 0.  Up to eight threads
// count for an entry, four keys at a time.  All threads; two barriers, the first before anything is read.
template <int NT>
__device__ __forceinline__ void top_rank(const uint64_t* entries, int M, int K, uint64_t* out) {
  const int tid = threadIdx.x;
  if (tid < kLgMaxTop) out[tid] = 0;
  __syncthreads();
  const int log = M <= NT / 8 ? 3 : (M <= NT / 4 ? 2 : (M <= NT / 2 ? 1 : 0));
  const int ways = 1 << log, part = tid & (ways - 1);
#pragma unroll 1
  for (int i0 = 0; i0 < M; i0 += NT >> log) {
    const int i = i0 + (tid >> log);
    const uint64_t k = i < M ? entries[i] : ~0ull;
    int r = 0;
#pragma unroll 1
    for (int j = part; j < M; j += 4 * ways) {
      uint64_t o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = j + u * ways < M ? entries[j + u * ways] : 0;
#pragma unroll
      for (int u = 0; u < 4; ++u) r += o[u] > k;
    }
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      const int other = __shfl_xor_sync(0xffffffffu, r, 1 << u);
      if (u < log) r += other;
    }
    if (i < M && part == 0 && r < K) out[r] = k;
  }
  __syncthreads();
}

__device__ __forceinline__ void st_cluster_u32(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint32_t addr, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}

// ------------------------------------------------------------------------------------ forward
// The pass clamps logits where c z = -2^27 (a packed maximum), so that -inf and large negative masks give
// 2^x = 0 and a finite x: below 2^27 in magnitude, x is off from c z - R by at most 8.  (fp16 ends at
// -65504: there only -inf is clamped.)  That is exact for every row whose largest logit m lies 512 / c
// above the clamp, with |c m| < 2^26.  The others are done again by row_slow, which is only careful: rows
// that hold nothing but masked logits, an infinity, or a huge common offset.
//
// Top K: a thread's logits form up to 32 groups, whose maxima the pass writes to shared memory (16 bits:
// the upper half of the ordered value, a lower bound).  Each of the w warps with data has j = ceil(K / w)
// threads whose maximum is at least the warp's own j-th largest thread maximum; the smallest of these over
// the warps, thr, therefore has at least K logits at or above it.  Only groups whose maximum reaches thr
// can hold an alternative: a few dozen of a few thousand.  They are read once more, a vector per thread,
// and their entries at or above thr are ranked by counting.  Order and ties are decided by distinct keys,
// so the result does not depend on the order of work.  Rows with too many equal logits for the two small
// lists go through sorted lists instead (top_by_lists).
constexpr int kLgQueue = 64;    // top_by_lists: groups a warp has waiting
constexpr int kLgItems = 256;   // groups to read again
constexpr int kLgCands = 256;   // entries at or above thr
constexpr float kLgPlainX = 67108864.f;    // 2^26

// Where a row's part lies: nh single elements, vectors [v0, v1) of this CTA behind them.
struct RowPart {
  const uint4* zv;
  int nh, nv, v0, v1;
};
template <typename T>
__device__ __forceinline__ RowPart row_part(const LogitsParams& p, int64_t row, int rank, int nc) {
  constexpr int kN = Elem<T>::kN;
  const T* zrow = reinterpret_cast<const T*>(p.z) + row * p.ld;
  RowPart q;
  q.nh = int(((16u - (uint32_t(reinterpret_cast<uintptr_t>(zrow)) & 15u)) & 15u) / sizeof(T));
  if (q.nh > p.V) q.nh = p.V;
  q.nv = (p.V - q.nh) / kN;
  q.zv = reinterpret_cast<const uint4*>(zrow + q.nh);
  const int shift = 31 - __clz(nc);  // nc is a power of two
  q.v0 = int((int64_t(q.nv) * rank) >> shift);
  q.v1 = int((int64_t(q.nv) * (rank + 1)) >> shift);
  return q;
}

// f(x) for every logit of a row by one CTA: 16-byte loads, four under way, and single elements at both ends.
template <typename T, int NT, typename F>
__device__ __forceinline__ void row_each(const T* z, int V, F f) {
  const int tid = threadIdx.x;
  int nh = int(((16u - (uint32_t(reinterpret_cast<uintptr_t>(z)) & 15u)) & 15u) / sizeof(T));
  if (nh > V) nh = V;
  const int nv = (V - nh) / Elem<T>::kN, nsingle = V - nv * Elem<T>::kN;
  const uint4* zv = reinterpret_cast<const uint4*>(z + nh);
  for (int i0 = tid; i0 < nv; i0 += 4 * NT) {
    uint4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (i0 + u * NT < nv) v[u] = zv[i0 + u * NT];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i0 + u * NT >= nv) break;
      float x[Elem<T>::kN];
      Elem<T>::widen(v[u], x);
#pragma unroll
      for (int e = 0; e < Elem<T>::kN; ++e) f(x[e]);
    }
  }
  if (tid < nsingle) f(Elem<T>::one(z, tid < nh ? tid : nv * Elem<T>::kN + tid));
}

// A whole row by one CTA, any logits: the exact maximum m first, then x = c (z - m).  All threads get
// {m, sum 2^x, sum 2^x x}; sh: NT / 32 entries.
template <typename T, int NT>
__device__ __forceinline__ RowTotal row_careful(const T* z, int V, float c, RowTotal* sh) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  float m = -INFINITY;
  bool nan = false;
  row_each<T, NT>(z, V, [&](float v) {
    nan |= v != v;
    m = fmaxf(m, v);
  });
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  __syncthreads();
  if (lane == 0) sh[warp].m = m;
  nan = __syncthreads_or(nan);
  for (int w = 0; w < (NT / 32); ++w) m = fmaxf(m, sh[w].m);
  RowTotal r;
  r.R = 0.f;
  r.m = m;
  r.s = r.t = 0.f;
  if (!nan && m > -INFINITY) {
    row_each<T, NT>(z, V, [&](float v) {
      const float x = max_nan((v - m) * c, kLgFloor);
      const float e = ex2_approx(x);
      r.s += e;
      r.t = fmaf(e, x, r.t);
    });
  } else if (nan) {
    r.s = __int_as_float(0x7FC00000);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float s = __shfl_xor_sync(0xffffffffu, r.s, o), t = __shfl_xor_sync(0xffffffffu, r.t, o);
    r.s = (lane & o) ? s + r.s : r.s + s;
    r.t = (lane & o) ? t + r.t : r.t + t;
  }
  __syncthreads();
  if (lane == 0) sh[warp] = r;
  __syncthreads();
  r = sh[0];
  for (int w = 1; w < (NT / 32); ++w) {
    r.s += sh[w].s;
    r.t += sh[w].t;
  }
  __syncthreads();
  return r;
}

template <typename T, int NT>
__device__ __noinline__ RowTotal row_slow(const T* z, int V, float c, RowTotal* sh) {
  return row_careful<T, NT>(z, V, c, sh);
}

// The K best entries of every warp's part of the row through lists that are kept sorted over the lanes,
// whatever the ties: `out` gets the lists one behind the other, *count their length.  All threads.
template <typename T, int NT>
__device__ __noinline__ void top_by_lists(const LogitsParams& p, const RowPart& q, int nb, int g, uint32_t thr,
                                          uint32_t thr16, float zs, bool has_single, const uint16_t* gmax,
                                          uint64_t* out, int* count) {
  using E = Elem<T>;
  constexpr int kN = E::kN;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, K = p.K, per = p.per;
  __shared__ uint16_t sh_queue[(NT / 32) * kLgQueue];
  uint16_t* queue = sh_queue + warp * kLgQueue;
  __syncthreads();  // everybody has read the count
  if (tid == 0) *count = 0;
  uint64_t mine = 0;  // lane i: the warp's i-th best entry so far
  uint64_t kth = 0;
  auto offer = [&](float v, uint32_t idx, bool in) {
    const uint64_t key = top_key(v, idx);
    uint32_t b = __ballot_sync(0xffffffffu, in && v > -INFINITY && uint32_t(key >> 32) >= thr && key > kth);
    if (b) {
      do {
        const int src = __ffs(b) - 1;
        b &= b - 1;
        top_insert(mine, __shfl_sync(0xffffffffu, key, src), lane);
      } while (b);
      kth = __shfl_sync(0xffffffffu, mine, K - 1);
    }
  };
  if (warp == 0) offer(zs, uint32_t(tid < q.nh ? tid : q.nv * kN + tid), has_single);
  int nq = 0;
  for (int k = 0; k < g || nq > 0;) {
    while (k < g && nq <= kLgQueue - 32) {
      const bool in = gmax[k * NT + tid] >= thr16;
      const uint32_t b = __ballot_sync(0xffffffffu, in);
      if (in) queue[nq + __popc(b & ((1u << lane) - 1u))] = uint16_t(k * 32 + lane);
      nq += __popc(b);
      ++k;
    }
    __syncwarp();
    const int take = min(nq, 32);
    const int item = lane < take ? queue[nq - take + lane] : -1;
    nq -= take;
    const int ig = item >> 5, il = item & 31;
    const int b0 = ig * per, b1 = min(b0 + per, nb);
    const int first = q.v0 + warp * 32 + il;  // vector u of batch b: first + (b * kLgUnroll + u) * NT
    bool act = item >= 0;
    if (act) {
      // nothing in the group can enter when its largest possible value at its lowest index would not
      const uint32_t o16 = gmax[ig * NT + warp * 32 + il];
      const uint32_t low = E::kNegInf == 0xFF80FF80u && (o16 & 0x8000u) ? 0u : 0xFFFFu;
      const uint32_t at = uint32_t(q.nh + (first + b0 * kLgUnroll * NT) * kN);
      act = ((uint64_t((o16 << 16) | low) << 32) | (0xFFFFFFFFu - at)) > kth;
    }
    if (__any_sync(0xffffffffu, act)) {
      for (int b = b0; __any_sync(0xffffffffu, act && b < b1); ++b) {
        uint4 v[kLgUnroll];
#pragma unroll
        for (int w = 0; w < kLgUnroll; ++w) {
          const int i = first + (b * kLgUnroll + w) * NT;
          v[w] = make_uint4(E::kNegInf, E::kNegInf, E::kNegInf, E::kNegInf);
          if (act && b < b1 && i < q.v1) v[w] = ldg_stream(q.zv + i);
        }
#pragma unroll
        for (int w = 0; w < kLgUnroll; ++w) {
          const float vm = E::pmax_final(E::pmax(E::pmax(v[w].x, v[w].y), E::pmax(v[w].z, v[w].w)));
          if (!__any_sync(0xffffffffu, uint32_t(top_key(vm, 0) >> 32) >= thr)) continue;
          float f[kN];
          E::widen(v[w], f);
          const int i = first + (b * kLgUnroll + w) * NT;
#pragma unroll
          for (int e = 0; e < kN; ++e) offer(f[e], uint32_t(q.nh + i * kN + e), true);
        }
      }
    }
    __syncwarp();
  }
  __syncthreads();  // the count is 0
  // the warps' lists one behind the other; their order does not matter
  const int have = __popc(__ballot_sync(0xffffffffu, lane < K && mine != 0));
  int to = 0;
  if (lane == 0 && have) to = atomicAdd(count, have);
  to = __shfl_sync(0xffffffffu, to, 0);
  if (lane < have) out[to + lane] = mine;
  __syncthreads();
}

template <typename T, bool TOP, int NT>
__global__ void __launch_bounds__(NT, (TOP ? 1024 : 1280) / NT) logits_fwd_kernel(const LogitsParams p) {
  using E = Elem<T>;
  constexpr int kN = E::kN;
  extern __shared__ __align__(16) uint16_t gmax[];  // TOP: [slots][NT] group maxima, the items
  __shared__ RowTotal sh_tot[(NT / 32)];
  __shared__ RowTotal sh_cl[kLgMaxCluster];
  __shared__ uint64_t sh_list[kLgCands];  // kLgCands = kLgMaxCluster * kLgMaxTop, no less than NT / 32 * kLgMaxTop
  __shared__ uint64_t sh_cl_list[kLgMaxCluster * kLgMaxTop];
  __shared__ uint64_t sh_best[kLgMaxTop];
  __shared__ uint32_t sh_thr[(NT / 32)];
  __shared__ int sh_count, sh_items;
  uint16_t* items = gmax + p.slots * NT;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  uint32_t nc, rank;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(nc));
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
  const int K = p.K, V = p.V;
  const float c = p.scale * 1.4426950408889634f;
  const int64_t row = blockIdx.x >> (31 - __clz(nc));
  if (p.mask && p.mask[row] == 0) {
    if (rank == 0) {
      if (tid == 0) {
        if (p.token_logp) p.token_logp[row] = 0.f;
        if (p.token_entropy) p.token_entropy[row] = 0.f;
        if (p.token_lse) p.token_lse[row] = 0.f;
      }
      if (TOP && tid < K) {
        if (p.top_logp) p.top_logp[row * K + tid] = 0.f;
        if (p.top_id) p.top_id[row * K + tid] = -1;
      }
    }
    return;  // every CTA of a cluster alike
  }
  // The other CTAs' shared memory may be written once they run: this barrier's first half here, its
  // second before the join.
  if (nc > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");

  const T* zrow = reinterpret_cast<const T*>(p.z) + row * p.ld;
  int target = 0;
  if (rank == 0 && tid == 0 && p.token_logp) target = p.targets[row];
  const RowPart q = row_part<T>(p, row, rank, nc);
  const int nsingle = V - q.nv * kN;  // head and tail elements: the last CTA takes them
  const int nb = (q.v1 - q.v0 + NT * kLgUnroll - 1) / (NT * kLgUnroll);
  const int per = p.per;
  float zs = -INFINITY;
  if (rank == nc - 1 && tid < nsingle) zs = E::one(zrow, tid < q.nh ? tid : q.nv * kN + tid);

  RowSums r;
  r.R = fmaf(p.clamp, c, 256.f);  // a clamped logit counts for nothing
  r.s = r.t = make_float2(0.f, 0.f);
  float tmax = p.clamp, gm = p.clamp;
  int g = 0, in_group = 0;
  uint4 cur[kLgUnroll], nxt[TOP ? kLgUnroll : 1];
  // Whole batches of all threads need neither bounds nor a filling (4096 x 152064 bf16 with and without alternatives,
  // single calls 209 and 189 us, 212 and 192 with one form for all; in a row 236 and 216, 243 and 222); the variant for
  // few rows has one form, since the first pass through the code is its time (256 rows: 22.8 us, 24.2 with two).
  constexpr bool kWhole = !TOP || NT < kLgThreads;
  const int whole = kWhole ? (q.v1 - q.v0) / (NT * kLgUnroll) : 0;
  const uint4* mine = q.zv + q.v0 + tid;
  auto load = [&](int b, uint4* v) {
    const uint4* at = mine + b * (NT * kLgUnroll);
    if (kWhole && b < whole) {
#pragma unroll
      for (int u = 0; u < kLgUnroll; ++u) v[u] = ldg_stream(at + u * NT);
    } else {
      const int i0 = q.v0 + b * (NT * kLgUnroll) + tid;
#pragma unroll
      for (int u = 0; u < kLgUnroll; ++u) {
        const int i = i0 + u * NT;
        v[u] = make_uint4(E::kNegInf, E::kNegInf, E::kNegInf, E::kNegInf);
        if (i < q.v1) v[u] = ldg_stream(kWhole ? at + u * NT : q.zv + i);
      }
    }
  };
  if (nb > 0) load(0, cur);
  const bool bad_target = target < 0 || target >= V;
  float z_target = 0.f;
  if (rank == 0 && tid == 0 && p.token_logp && !bad_target) z_target = E::one(zrow, target);  // behind the first loads
  auto take = [&](uint4* v) {
    uint32_t pm = 0;
#pragma unroll
    for (int u = 0; u < kLgUnroll; ++u) {
      v[u] = make_uint4(E::pclamp(v[u].x, p.clamp_pk), E::pclamp(v[u].y, p.clamp_pk), E::pclamp(v[u].z, p.clamp_pk),
                        E::pclamp(v[u].w, p.clamp_pk));
      const uint32_t a = E::pmax(E::pmax(v[u].x, v[u].y), E::pmax(v[u].z, v[u].w));
      pm = u ? E::pmax(pm, a) : a;
    }
    const float bm = E::pmax_final(pm);
    tmax = fmaxf(tmax, bm);
    if (TOP) {
      gm = fmaxf(gm, bm);
      if (++in_group == per) {
        gmax[g * NT + tid] = uint16_t(top_key(gm, 0) >> 48);
        gm = p.clamp;
        in_group = 0;
        ++g;
      }
    }
    if (fmaf(bm, c, -r.R) > kLgMove) row_move(r, bm * c);
#pragma unroll
    for (int u = 0; u < kLgUnroll; ++u) {
      float f[kN];
      E::widen(v[u], f);
      row_add<kN>(r, f, c);
    }
  };
  // Without alternatives five CTAs per SM hide each other's loads; with them, registers allow four, which load a
  // batch ahead (4096 x 152064 bf16: the other way round both take 8 % more).
  if (TOP) {
#pragma unroll 1
    for (int b = 0; b < nb; b += 2) {
      if (b + 1 < nb) load(b + 1, nxt);
      take(cur);
      if (b + 1 == nb) break;
      if (b + 2 < nb) load(b + 2, cur);
      take(nxt);
    }
  } else {
    for (int b = 0; b < nb; ++b) {
      if (b) load(b, cur);
      take(cur);
    }
  }
  if (TOP && in_group) {
    gmax[g * NT + tid] = uint16_t(top_key(gm, 0) >> 48);
    ++g;
  }
  float wmax = tmax;
  if (rank == nc - 1 && tid < nsingle) {
    const float z = max_nan(zs, p.clamp);
    if (fmaf(z, c, -r.R) > kLgMove) row_move(r, z * c);
    const float f[2] = {z, p.clamp};
    row_add<2>(r, f, c);
    wmax = fmaxf(wmax, z);
  }

  // ---- join the sums: lanes, warps
  RowTotal tot;
  {
    tot.R = r.R;
    tot.s = r.s.x + r.s.y;
    tot.t = r.t.x + r.t.y;
    tot.m = wmax;
  }
  tot = row_join_warp(tot);
  if (lane == 0) sh_tot[warp] = tot;

  // ---- top alternatives of this CTA's part
  if (TOP) {
    const uint32_t none = uint32_t(top_key(-INFINITY, 0) >> 32);  // -inf is no alternative
    const int with = min((q.v1 - q.v0 + 31) / 32, (NT / 32));      // warps with data
    uint32_t left = ordered(tmax + 0.f), jth = 0xFFFFFFFFu;
    if (warp < with) {
      for (int n = (K + with - 1) / with; n > 0; --n) {
        jth = __reduce_max_sync(0xffffffffu, left);
        if (left == jth) left = 0;  // equal ones together: the next is lower, which is safe
      }
    }
    if (lane == 0) sh_thr[warp] = jth;
    if (tid == 0) sh_count = sh_items = 0;
    __syncthreads();
    uint32_t thr = with ? __reduce_min_sync(0xffffffffu, sh_thr[lane % (NT / 32)]) : 0u;
    // at the clamp the maxima say nothing: everything above -inf is to be looked at
    if (thr <= uint32_t(top_key(p.clamp, 0) >> 32)) thr = none + 1;
    const uint32_t thr16 = thr > none + 1 ? thr >> 16 : 0;
    const float thr_f = from_ordered(thr);  // NaN is no alternative

    // groups to read again
    uint32_t hot = 0;
#pragma unroll 8
    for (int k = 0; k < g; ++k) hot |= uint32_t(gmax[k * NT + tid] >= thr16) << k;
    if (hot) {
      int at = atomicAdd(&sh_items, __popc(hot));
      do {
        if (at < kLgItems) items[at] = uint16_t((__ffs(hot) - 1) * NT + tid);
        ++at;
        hot &= hot - 1;
      } while (hot);
    }
    if (rank == nc - 1 && tid < nsingle) {
      if (zs >= thr_f) {
        const int at = atomicAdd(&sh_count, 1);
        if (at < kLgCands) sh_list[at] = top_key(zs, uint32_t(tid < q.nh ? tid : q.nv * kN + tid));
      }
    }
    __syncthreads();
    const int n_items = sh_items;
    if (n_items <= kLgItems) {
      const int vecs = per * kLgUnroll;  // of a group
      const int n_vecs = n_items * vecs;
#pragma unroll 1
      for (int i0 = tid; i0 < n_vecs; i0 += 2 * NT) {
        uint4 v[2];  // two under way
        int at[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int i = i0 + u * NT, it = i < n_vecs ? items[i / vecs] : 0;
          at[u] = i < n_vecs ? q.v0 + ((it / NT) * vecs + i % vecs) * NT + it % NT : q.v1;
          if (at[u] < q.v1) v[u] = ldg_stream(q.zv + at[u]);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          if (at[u] < q.v1) {
            float f[kN];
            E::widen(v[u], f);
            uint32_t in = 0;
#pragma unroll
            for (int e = 0; e < kN; ++e) in |= uint32_t(f[e] >= thr_f) << e;
            if (in) {
              int to = atomicAdd(&sh_count, __popc(in));
#pragma unroll
              for (int e = 0; e < kN; ++e) {
                if (in >> e & 1) {
                  if (to < kLgCands) sh_list[to] = top_key(f[e], uint32_t(q.nh + at[u] * kN + e));
                  ++to;
                }
              }
            }
          }
        }
      }
    }
    __syncthreads();
    if (n_items > kLgItems || sh_count > kLgCands) {
      top_by_lists<T, NT>(p, q, nb, g, thr, thr16, zs, rank == nc - 1 && tid < nsingle, gmax, sh_list, &sh_count);
    }
    top_rank<NT>(sh_list, sh_count, K, sh_best);
  } else {
    __syncthreads();
  }
  tot = row_join_list(sh_tot, (NT / 32));

  // ---- join the CTAs of the row in CTA 0
  if (nc > 1) {
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    if (tid == 0) {
      const uint32_t to = mapa_shared(smem_u32(&sh_cl[rank]), 0);
      st_cluster_u32(to, __float_as_uint(tot.R));
      st_cluster_u32(to + 4, __float_as_uint(tot.s));
      st_cluster_u32(to + 8, __float_as_uint(tot.t));
      st_cluster_u32(to + 12, __float_as_uint(tot.m));
    }
    if (TOP && tid < K) st_cluster_u64(mapa_shared(smem_u32(&sh_cl_list[rank * K + tid]), 0), sh_best[tid]);
    cluster_sync_all();
    if (rank != 0) return;
    tot = row_join_list(sh_cl, int(nc));
    if (TOP) {
      // as with the warps: at least K entries reach the smallest of the CTAs' j-th bests, j = ceil(K / nc)
      uint64_t bound = ~0ull;
      const int j = (K + int(nc) - 1) >> (31 - __clz(nc));
#pragma unroll
      for (uint32_t w = 0; w < kLgMaxCluster; ++w)
        if (w < nc) bound = min(bound, sh_cl_list[w * K + j - 1]);
      const uint64_t key = tid < int(nc) * K ? sh_cl_list[tid] : 0;
      if (tid == 0) sh_count = 0;
      __syncthreads();
      if (key != 0 && key >= bound) sh_list[atomicAdd(&sh_count, 1)] = key;
      __syncthreads();
      top_rank<NT>(sh_list, sh_count, K, sh_best);
    }
  }

  // ---- results
  const float ln2 = 0.6931471805599453f;
  const bool plain = fabsf(tot.m * c) < kLgPlainX && (tot.m - p.clamp) * c > 512.f;  // the same for all threads
  if (!plain) tot = row_slow<T, NT>(zrow, V, c, sh_tot);
  // no finite logit: every probability is 0, lse = -inf, nothing to choose from
  const bool empty = tot.m == -INFINITY && tot.s == 0.f;
  const bool broken = !empty && !(tot.m > -INFINITY && tot.m < INFINITY && tot.s > 0.f && tot.s < INFINITY);
  const float nan = __int_as_float(0x7FC00000);
  const float ln_s = logf(tot.s);
  // ln p of a logit, relative to the reference, so that a large common offset does not cost digits
  auto ln_p = [&](float z) {
    if (broken) return nan;
    if (empty || z == -INFINITY) return -INFINITY;
    if (!plain) return p.scale * (z - tot.m) - ln_s;
    return z > p.clamp ? fmaf(fmaf(z, c, -tot.R), ln2, -ln_s) : fmaf(p.scale, z, -fmaf(tot.R, ln2, ln_s));
  };
  if (tid == 0) {
    if (p.token_lse)
      p.token_lse[row] = broken ? nan : (empty ? -INFINITY : (plain ? fmaf(tot.R, ln2, ln_s) : fmaf(p.scale, tot.m, ln_s)));
    if (p.token_entropy) p.token_entropy[row] = broken ? nan : (empty ? 0.f : fmaxf(0.f, ln_s - ln2 * (tot.t / tot.s)));
    if (p.token_logp) p.token_logp[row] = bad_target ? nan : ln_p(z_target);
    if (p.status && (bad_target || broken)) atomicCAS(p.status, 0, bad_target ? kErrBadTarget : kErrNonfinite);
  }
  if (TOP && tid < K) {
    const uint64_t key = sh_best[tid];
    if (p.top_id) p.top_id[row * K + tid] = key ? int32_t(0xFFFFFFFFu - uint32_t(key)) : -1;
    if (p.top_logp) p.top_logp[row * K + tid] = broken ? nan : (key ? ln_p(top_value(key)) : -INFINITY);
  }
}

// ------------------------------------------------------------------------------------ backward
// dz_v = a ( -p_v (G + g_H (ln p_v + H)) + g_lp [v = t] + sum_k g_k [v = id_k] ),  G = g_lp + sum_k g_k,
// p_v = e^(a z_v - lse).  One read and one write per logit, HBM-bound; dz may be the logits themselves.
// Six CTAs per SM (four: 12 % slower), five with one batch a CTA (64 x 152064 bf16 with 32 entries a row: 7.8 us, 8.5
// with six).  A CTA takes a span of a row, one batch of loads or, where there are rows enough (kMany), four, which
// share the row's factors and the scan of its entries: these are half of the instructions otherwise, and under the
// power limit fewer instructions are a higher clock.  4096 x 152064 bf16 in repeated calls: 383 us with four batches,
// the copy rate; 404 us with one.  257 x 32003 fp32 with 8 entries a row: 13.1 us with one, 15.1 with four.  Rows of
// the result at another offset from 16 bytes than the logits' rows are read an element at a time: 503 us against 380.
// The few entries with a point term are written again after the CTA's stores, from logits read before them.
struct RowGrad {
  float a, nlse;  // ln p = a z + nlse
  float A, B;     // dz = p (A ln p + B)
};
// ln p is kept finite, so that p = 0 gives 0.
__device__ __forceinline__ float2 grad_smooth(float2 z, const RowGrad& r) {
  float2 lp = __ffma2_rn(z, make_float2(r.a, r.a), make_float2(r.nlse, r.nlse));
  lp = make_float2(max_nan(lp.x, -1e5f), max_nan(lp.y, -1e5f));
  const float2 x = __fmul2_rn(lp, make_float2(1.4426950408889634f, 1.4426950408889634f));
  const float2 w = __ffma2_rn(lp, make_float2(r.A, r.A), make_float2(r.B, r.B));
  return __fmul2_rn(make_float2(ex2_approx(x.x), ex2_approx(x.y)), w);
}

// What the gradient needs of a row; lane k of every warp holds alternative k.
struct RowTerms {
  int target, id;  // -1 where there is none, or outside [0, V): they count for nothing
  float g_target, g_id, G, ge, H, lse;
};
__device__ __forceinline__ RowTerms row_terms(const LogitsParams& p, int64_t row) {
  const int lane = threadIdx.x & 31, K = p.K, V = p.V;
  RowTerms t;
  // all loads first: none waits for another
  t.lse = p.lse[row];
  t.target = p.g_logp ? p.targets[row] : -1;
  t.g_target = p.g_logp ? p.g_logp[row] : 0.f;
  t.id = lane < K ? p.ids[row * K + lane] : -1;
  t.g_id = lane < K ? p.g_top[row * K + lane] : 0.f;
  t.ge = p.g_entropy ? p.g_entropy[row] : 0.f;
  t.H = p.g_entropy ? p.entropy[row] : 0.f;
  if (t.target < 0 || t.target >= V) {
    t.target = -1;
    t.g_target = 0.f;
  }
  if (t.id < 0 || t.id >= V) {
    t.id = -1;
    t.g_id = 0.f;
  }
  t.G = t.g_target;
  if (K) {
    float sum = t.g_id;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    t.G += sum;
  }
  return t;
}
__device__ __forceinline__ RowGrad row_grad(const LogitsParams& p, const RowTerms& t, float lse) {
  return {p.scale, -lse, -p.scale * t.ge, -p.scale * fmaf(t.ge, t.H, t.G)};
}
// The entry with a point term that this thread writes (-1: none), with all terms of that entry.  An entry is written
// by one warp: warp 0 the alternatives, whose lanes of equal index add the same terms in the same order (the target's
// first, then by k); warp 1 the target where it is none of them.
__device__ __forceinline__ int row_point(const RowTerms& t, int K, float& point) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  point = 0.f;
  if (warp == 0 && K) {
    if (t.id == t.target) point = t.g_target;
    for (int k = 0; k < K; ++k) {
      const int other = __shfl_sync(0xffffffffu, t.id, k);
      const float g = __shfl_sync(0xffffffffu, t.g_id, k);
      if (other == t.id) point += g;
    }
    return t.id;
  }
  if (warp == 1 && t.target >= 0 && !__any_sync(0xffffffffu, t.id == t.target)) {
    point = t.g_target;
    return lane == 0 ? t.target : -1;
  }
  return -1;
}

// Beyond this |lse| its fp32 digits do not resolve p (half a step of 1024 is 2^-14 of p; at 1e9 it is e^32).  Such a
// row (a large common offset, or nothing but a finite mask value) is done by one CTA, which forms the maximum m and
// the sum S again and takes ln p = a (z - m) - ln S, in three passes over the row: 34 us for one of 152064 bf16, 0.77 ms
// for 4096 of them against 0.38 for other rows.
constexpr float kLgResolved = 1024.f;
template <typename T>
__device__ __forceinline__ void grad_row_apart(const LogitsParams& p, int64_t row) {
  using E = Elem<T>;
  __shared__ RowTotal sh_tot[kLgThreads / 32];
  const T* z = reinterpret_cast<const T*>(p.z) + row * p.ld;
  T* d = reinterpret_cast<T*>(p.dz) + row * p.ld_d;
  const RowTotal tot = row_careful<T, kLgThreads>(z, p.V, p.scale * 1.4426950408889634f, sh_tot);
  const bool none = tot.m == -INFINITY && tot.s == 0.f;  // not the row that this lse is of: p = 0
  const float m = none ? 0.f : tot.m, ln_s = none ? 1e30f : logf(tot.s);
  const RowTerms t = row_terms(p, row);
  const RowGrad r = row_grad(p, t, ln_s);
  float point;
  const int at = row_point(t, p.K, point);
  const float z_at = at >= 0 ? E::one(z, at) : 0.f;
  __syncthreads();  // the logits at these entries have been read
  if (((reinterpret_cast<uintptr_t>(z) ^ reinterpret_cast<uintptr_t>(d)) & 15) == 0) {
    // single elements up to a 16-byte boundary and behind the last one, vectors between
    int nh = int(((16u - (uint32_t(reinterpret_cast<uintptr_t>(d)) & 15u)) & 15u) / sizeof(T));
    if (nh > p.V) nh = p.V;
    const int nv = (p.V - nh) / E::kN, nsingle = p.V - nv * E::kN;
    const uint4* zv = reinterpret_cast<const uint4*>(z + nh);
    uint4* dv = reinterpret_cast<uint4*>(d + nh);
    for (int i0 = threadIdx.x; i0 < nv; i0 += 2 * kLgThreads) {
      uint4 v[2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
        if (i0 + u * kLgThreads < nv) v[u] = zv[i0 + u * kLgThreads];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (i0 + u * kLgThreads >= nv) break;
        float f[E::kN];
        E::widen(v[u], f);
#pragma unroll
        for (int e = 0; e < E::kN; e += 2) {
          const float2 g = grad_smooth(make_float2(f[e] - m, f[e + 1] - m), r);
          f[e] = g.x;
          f[e + 1] = g.y;
        }
        dv[i0 + u * kLgThreads] = E::narrow(f);
      }
    }
    const int i = int(threadIdx.x) < nh ? threadIdx.x : nv * E::kN + threadIdx.x;
    if (int(threadIdx.x) < nsingle) E::put(d, i, grad_smooth(make_float2(E::one(z, i) - m, 0.f), r).x);
  } else {
    for (int i = threadIdx.x; i < p.V; i += kLgThreads)
      E::put(d, i, grad_smooth(make_float2(E::one(z, i) - m, 0.f), r).x);
  }
  __syncthreads();
  if (at >= 0) E::put(d, at, fmaf(r.a, point, grad_smooth(make_float2(z_at - m, 0.f), r).x));
}

template <typename T, bool kMany>
__global__ void __launch_bounds__(kLgThreads, kMany ? 6 : 5)
logits_bwd_kernel(const __grid_constant__ LogitsParams p, int spans) {
  using E = Elem<T>;
  constexpr int kN = E::kN;
  const int tid = threadIdx.x;
  const int64_t row = blockIdx.x / unsigned(spans);
  const int span = int(blockIdx.x % unsigned(spans));
  const int V = p.V, K = p.K;
  const T* zrow = reinterpret_cast<const T*>(p.z) + row * p.ld;
  T* drow = reinterpret_cast<T*>(p.dz) + row * p.ld_d;

  const uint32_t az = uint32_t(reinterpret_cast<uintptr_t>(zrow)) & 15u;
  const uint32_t ad = uint32_t(reinterpret_cast<uintptr_t>(drow)) & 15u;
  int nh = int(((16u - ad) & 15u) / sizeof(T));
  if (nh > V) nh = V;
  const int nv = (V - nh) / kN;
  const int nsingle = V - nv * kN;
  const bool together = az == ad;  // loads and stores share the vector boundaries
  const bool live = !p.mask || p.mask[row] != 0;
  // a batch, or equal spans of whole rounds of the CTA
  const int per_span =
      kMany ? (nv + spans * kLgThreads - 1) / (spans * kLgThreads) * kLgThreads : kLgThreads * kLgUnroll;
  const int w0 = min(nv, span * per_span);
  const int w1 = min(nv, w0 + per_span);

  if (!live) {
    for (int i = w0 + tid; i < w1; i += kLgThreads)
      *reinterpret_cast<uint4*>(drow + nh + int64_t(i) * kN) = make_uint4(0, 0, 0, 0);
    if (span == 0 && tid < nsingle) E::put(drow, tid < nh ? tid : nv * kN + tid, 0.f);
    return;
  }

  uint4 v[kLgUnroll];
  auto load = [&](int at) {
#pragma unroll
    for (int u = 0; u < kLgUnroll; ++u) {
      const int i = at + u * kLgThreads + tid;
      if (together && i < w1) v[u] = *(reinterpret_cast<const uint4*>(zrow + nh) + i);
    }
  };
  load(w0);
  float zs = 0.f;
  const int single = tid < nh ? tid : nv * kN + tid;
  if (span == 0 && tid < nsingle) zs = E::one(zrow, single);

  const RowTerms t = row_terms(p, row);
  float lse = t.lse;
  if (fabsf(lse) > kLgResolved) {  // the same for all threads of the row
    if (lse >= -1e30f) {
      if (span == 0) grad_row_apart<T>(p, row);
      return;
    }
    lse = 1e30f;  // no finite logit, or nothing but a type's lowest value as a mask: every p is 0
  }
  const RowGrad r = row_grad(p, t, lse);
  float point;
  int at = row_point(t, K, point);
  if (at >= 0) {  // owned by the CTA that stores it
    const int vec = (at - nh) / kN;
    const bool is_single = at < nh || at >= nh + nv * kN;
    if (is_single ? span != 0 : (vec < w0 || vec >= w1)) at = -1;
  }
  const float z_at = at >= 0 ? E::one(zrow, at) : 0.f;
  const bool any_point = __syncthreads_or(at >= 0);  // the logits at these entries have been read

  for (int at = w0; at < w1; at += kLgThreads * kLgUnroll) {
    if (kMany && at != w0) load(at);
#pragma unroll
    for (int u = 0; u < kLgUnroll; ++u) {
      const int i = at + u * kLgThreads + tid;
      if (i < w1) {
        float f[kN];
        if (together) {
          E::widen(v[u], f);
        } else {
#pragma unroll
          for (int e = 0; e < kN; ++e) f[e] = E::one(zrow, nh + int64_t(i) * kN + e);
        }
#pragma unroll
        for (int e = 0; e < kN; e += 2) {
          const float2 d = grad_smooth(make_float2(f[e], f[e + 1]), r);
          f[e] = d.x;
          f[e + 1] = d.y;
        }
        *reinterpret_cast<uint4*>(drow + nh + int64_t(i) * kN) = E::narrow(f);
      }
    }
    if (!kMany) break;
  }
  if (span == 0 && tid < nsingle) E::put(drow, single, grad_smooth(make_float2(zs, 0.f), r).x);
  if (any_point) {
    __syncthreads();
    if (at >= 0) E::put(drow, at, fmaf(r.a, point, grad_smooth(make_float2(z_at, 0.f), r).x));
  }
}

}  // namespace oapl

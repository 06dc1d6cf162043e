// Quantisation of a matrix to 8-bit floating point with one fp32 scale per 1 x 128 or 128 x 128 block,
// as it stands or turned (transposed), for the product in scaled_matmul.cuh.
//
//   amax  = max(largest |x| of the block, 2^-100)
//   scale = amax / top                              (top = 448 for e4m3, 57344 for e5m2)
//   q     = round((0.875 x) / (0.875 amax / top))   to the 8-bit type, nearest even
// top is 0.875 times a power of two, so for 16-bit inputs both sides of that quotient are exact and a
// value half way between two 8-bit numbers is seen as such.  For fp32 inputs 0.875 x is rounded first, which can move a
// quotient that lies within 2^-23 of such a value onto it or across.  The quotient is correctly rounded: a product
// with the rounded reciprocal, and one residual step (Markstein's theorem on division by multiply-add).  With
// power-of-two scales, scale = 2^ceil(log2(amax / top)) and the result is that of x / scale, which is exact: the
// rounding of 0.875 x keeps the order of values and moves none onto another one of fewer than 20 bits.
// A NaN in a block makes its scale and all its values NaN; an infinity makes the scale infinite, the
// finite values 0 and itself NaN.
//
// HBM-bound: x is read once and q written once.  A CTA takes a 128 x 128 tile, which it holds in registers
// between the maximum and the rounding: 8 rows x 16 bytes a thread, all loads in flight together, five CTAs
// (16-bit types) per SM.  Maxima are taken on packed words; what rounding needs of a block is computed once
// and shared.  Rows that do not start on a 16-byte boundary are read as the aligned 16-byte blocks that hold
// them (a block without an element of the row is not touched) and shifted in registers: 8192 x 3585 bf16 29.4 us,
// 8192 x 3584 15.9; turned, 1999 x 50021 95.5 and 65 us.  A turned tile goes through 16 KB of swizzled shared memory, so
// that it too leaves in 16-byte stores.  Five CTAs cost the form with 128 x 128 blocks five words of local memory a
// thread, 1.3 % of its instructions (152064 x 3584 bf16: 247 us, the copy rate).
#pragma once
#include "logits_ops.cuh"

namespace oapl {

constexpr int kQtTile = 128;
constexpr int kQtRows = 8;                        // rows of a thread
constexpr int kQtGroups = kQtTile / kQtRows;      // lane groups, one above the other

struct QuantParams {
  const void* x;
  int64_t ldx;        // elements
  int32_t R, C;       // of x
  uint8_t* q;
  int64_t ldq;        // bytes
  float* scale;       // scale of row block i and column block j of q: scale[i * srow + j * scol]
  int64_t srow, scol;
  int32_t pow2;
  int32_t vec;        // every row of x starts on a 16-byte boundary
};

template <int E5M2>
__device__ __forceinline__ uint32_t cvt_fp8x2(float lo, float hi) {
  uint16_t r;
  if (E5M2)
    asm("cvt.rn.satfinite.e5m2x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  else
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}

// Larger magnitude of packed words, with some sign; NaN stays.  word_abs: magnitude of element i of a word.
template <typename T>
__device__ __forceinline__ uint32_t word_absmax(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ uint32_t word_absmax<__nv_bfloat16>(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <>
__device__ __forceinline__ uint32_t word_absmax<__half>(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.xorsign.abs.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
template <>
__device__ __forceinline__ uint32_t word_absmax<float>(uint32_t a, uint32_t b) {
  return __float_as_uint(max_nan(fabsf(__uint_as_float(a)), fabsf(__uint_as_float(b))));
}
template <typename T>
__device__ __forceinline__ float word_abs(uint32_t w, int i) {
  if (sizeof(T) == 4) return fabsf(__uint_as_float(w));
  const uint16_t h = uint16_t(i ? w >> 16 : w);
  return fabsf(Elem<T>::one(&h, 0));
}
template <typename T>
__device__ __forceinline__ float word_abs(uint32_t w) {  // the larger one
  return sizeof(T) == 4 ? word_abs<T>(w, 0) : max_nan(word_abs<T>(w, 0), word_abs<T>(w, 1));
}

// What a block needs to round its values: y = a * inv, and one residual step against b.  For an infinite or
// NaN block b = 0 and inv = 0 or NaN, which gives 0 for finite values and NaN otherwise.
struct QuantScale {
  float b, inv;
};
template <int E5M2>
__device__ __forceinline__ QuantScale quant_scale(float amax, bool pow2, float& scale) {
  constexpr float kTop = E5M2 ? 57344.f : 448.f;
  constexpr int kTopExp = E5M2 ? 15 : 8;  // top = 1.75 * 2^kTopExp
  QuantScale s;
  amax = max_nan(amax, 7.888609052210118e-31f);  // 2^-100
  if (!(amax <= 3.402823466e38f)) {
    scale = amax;
    s.b = 0.f;
    s.inv = amax != amax ? amax : 0.f;
    return s;
  }
  if (pow2) {
    const uint32_t u = __float_as_uint(amax);
    const int e = int(u >> 23) - kTopExp + ((u & 0x7FFFFFu) > 0x600000u);  // mantissa above 1.75: next power
    scale = __uint_as_float(uint32_t(e) << 23);
    s.b = scale * 0.875f;
  } else {
    scale = amax / kTop;
    s.b = amax * (0.875f / kTop);
  }
  s.inv = 1.f / s.b;
  return s;
}
__device__ __forceinline__ float quant_one(float x, const QuantScale& s) {
  const float a = x * 0.875f;
  const float y = a * s.inv;
  return fmaf(fmaf(-y, s.b, a), s.inv, y);
}

// 16 bytes that start m bytes into the 32 of lo and hi; m a multiple of the element size, below 16.
__device__ __forceinline__ uint4 shift_bytes(const uint4& lo, const uint4& hi, uint32_t m) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = (m & 8) ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = (m & 4) ? w[i + 1] : w[i];
  const uint32_t s = (m & 3) * 8;
  return make_uint4(__funnelshift_r(w[0], w[1], s), __funnelshift_r(w[1], w[2], s), __funnelshift_r(w[2], w[3], s),
                    __funnelshift_r(w[3], w[4], s));
}

template <typename T, int E5M2, bool BLOCK, bool TURN>
__global__ void __launch_bounds__(kQtGroups * kQtTile / Elem<T>::kN, sizeof(T) == 4 ? 2 : 5)
quantize_kernel(const QuantParams p) {
  using E = Elem<T>;
  constexpr int kN = E::kN;                    // columns of a thread
  constexpr int kLanes = kQtTile / kN;         // lanes of a row: 16 or 32
  constexpr int kThreads = kQtGroups * kLanes;  // 256 or 512
  constexpr int kPer = 4 / sizeof(T);          // elements of a word
  __shared__ __align__(16) uint32_t sh_red[TURN && !BLOCK ? kQtGroups * kQtTile / kPer : kQtTile];
  __shared__ __align__(16) QuantScale sh_qs[kQtTile];
  __shared__ __align__(16) uint8_t sh_tile[TURN ? kQtTile * kQtTile : 16];

  const int tid = threadIdx.x, lane = tid % kLanes, group = tid / kLanes;
  // neighbours in the order of the result's rows, whose lines they share (1999 x 50021 turned: 66 us against 73)
  const unsigned inner = (unsigned(TURN ? p.R : p.C) + kQtTile - 1) / kQtTile;
  const int a0 = int(blockIdx.x / inner) * kQtTile, b0 = int(blockIdx.x % inner) * kQtTile;
  const int r0 = TURN ? b0 : a0, c0 = TURN ? a0 : b0;
  const int row = r0 + group * kQtRows, col = c0 + lane * kN;

  // ---- the thread's 8 x kN values
  uint4 v[kQtRows];
  const char* x = reinterpret_cast<const char*>(p.x) + (int64_t(row) * p.ldx + col) * int64_t(sizeof(T));
  const int64_t pitch = p.ldx * int64_t(sizeof(T));
  if (p.vec) {
#pragma unroll
    for (int i = 0; i < kQtRows; ++i) {
      v[i] = make_uint4(0, 0, 0, 0);
      if (row + i < p.R && col < p.C) v[i] = ldg_stream(reinterpret_cast<const uint4*>(x + i * pitch));
    }
  } else {
#pragma unroll
    for (int i = 0; i < kQtRows; ++i) {
      v[i] = make_uint4(0, 0, 0, 0);
      if (row + i < p.R && col < p.C) {
        const char* a = x + i * pitch;
        const uint32_t m = uint32_t(reinterpret_cast<uintptr_t>(a)) & 15u;
        const uint4* at = reinterpret_cast<const uint4*>(a - m);
        const uint4 lo = __ldg(at);
        uint4 hi = make_uint4(0, 0, 0, 0);
        // the second block starts 16 - m bytes on: only when the row still has an element there
        if (col + int((16u - m) / sizeof(T)) < p.C && m) hi = __ldg(at + 1);
        v[i] = shift_bytes(lo, hi, m);
      }
    }
  }
  if (col < p.C && col + kN > p.C) {  // behind the row's end
#pragma unroll
    for (int i = 0; i < kQtRows; ++i) {
      uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int left = p.C - (col + j * kPer);
        if (left <= 0) w[j] = 0;
        if (kPer == 2 && left == 1) w[j] &= 0xFFFFu;
      }
      v[i] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }

  // ---- largest magnitudes, and what rounding needs of every block
  if (TURN && !BLOCK) {
    uint4 m = v[0];
#pragma unroll
    for (int i = 1; i < kQtRows; ++i)
      m = make_uint4(word_absmax<T>(m.x, v[i].x), word_absmax<T>(m.y, v[i].y), word_absmax<T>(m.z, v[i].z),
                     word_absmax<T>(m.w, v[i].w));
    reinterpret_cast<uint4*>(sh_red)[group * kLanes + lane] = m;
    __syncthreads();
    if (tid < kQtTile) {
      uint32_t a = sh_red[tid / kPer];
#pragma unroll
      for (int g = 1; g < kQtGroups; ++g) a = word_absmax<T>(a, sh_red[g * (kQtTile / kPer) + tid / kPer]);
      float scale;
      sh_qs[tid] = quant_scale<E5M2>(word_abs<T>(a, tid % kPer), p.pow2, scale);
      if (c0 + tid < p.C) p.scale[int64_t(c0 + tid) * p.srow + int64_t(r0 / kQtTile) * p.scol] = scale;
    }
  } else {
    uint32_t m[kQtRows];
#pragma unroll
    for (int i = 0; i < kQtRows; ++i)
      m[i] = word_absmax<T>(word_absmax<T>(v[i].x, v[i].y), word_absmax<T>(v[i].z, v[i].w));
    if (BLOCK) {
#pragma unroll
      for (int i = 1; i < kQtRows; ++i) m[0] = word_absmax<T>(m[0], m[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m[0] = word_absmax<T>(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
      if ((tid & 31) == 0) sh_red[tid >> 5] = m[0];
      __syncthreads();
      if (tid == 0) {
        uint32_t a = sh_red[0];
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) a = word_absmax<T>(a, sh_red[w]);
        float scale;
        sh_qs[0] = quant_scale<E5M2>(word_abs<T>(a), p.pow2, scale);
        const int64_t i = (TURN ? c0 : r0) / kQtTile, j = (TURN ? r0 : c0) / kQtTile;
        p.scale[i * p.srow + j * p.scol] = scale;
      }
    } else {
      // eight rows over a lane group: every exchange halves the rows that a lane still holds, so that a
      // lane ends with row (lane / (kLanes / 8)) of its group after 8 exchanges instead of 32
#pragma unroll
      for (int h = 4, o = kLanes / 2; h > 0; h >>= 1, o >>= 1) {
        const bool up = lane & o;
#pragma unroll
        for (int i = 0; i < h; ++i) {
          const uint32_t keep = up ? m[i + h] : m[i], send = up ? m[i] : m[i + h];
          m[i] = word_absmax<T>(keep, __shfl_xor_sync(0xffffffffu, send, o));
        }
      }
#pragma unroll
      for (int o = kLanes / 16; o > 0; o >>= 1) m[0] = word_absmax<T>(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
      if (lane % (kLanes / 8) == 0) sh_red[group * kQtRows + lane / (kLanes / 8)] = m[0];
      __syncthreads();
      if (tid < kQtTile) {
        float scale;
        sh_qs[tid] = quant_scale<E5M2>(word_abs<T>(sh_red[tid]), p.pow2, scale);
        if (r0 + tid < p.R) p.scale[int64_t(r0 + tid) * p.srow + int64_t(c0 / kQtTile) * p.scol] = scale;
      }
    }
  }
  __syncthreads();

  // ---- round and store
  if (!TURN) {
    QuantScale qs = sh_qs[0];
#pragma unroll
    for (int i = 0; i < kQtRows; ++i) {
      if (!BLOCK) qs = sh_qs[group * kQtRows + i];
      float f[kN];
      E::widen(v[i], f);
#pragma unroll
      for (int e = 0; e < kN; ++e) f[e] = quant_one(f[e], qs);
      uint32_t w[kN / 4];
#pragma unroll
      for (int e = 0; e < kN; e += 4)
        w[e / 4] = cvt_fp8x2<E5M2>(f[e], f[e + 1]) | (cvt_fp8x2<E5M2>(f[e + 2], f[e + 3]) << 16);
      if (row + i < p.R) {
        uint8_t* q = p.q + int64_t(row + i) * p.ldq + col;
        if (col + kN <= p.C) {
          if (kN == 8)
            *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
          else
            *reinterpret_cast<uint32_t*>(q) = w[0];
        } else {
#pragma unroll
          for (int e = 0; e < kN; ++e)
            if (col + e < p.C) q[e] = uint8_t(w[e / 4] >> (8 * (e & 3)));
        }
      }
    }
  } else {
    // Two columns at a time, so that their words and factors are done with: eight rows of the pair, rounded,
    // are turned into eight bytes of each column.  8-byte unit u of row c of the turned tile sits at
    // u ^ (c / kN), which spreads a warp's stores over all banks.
#pragma unroll
    for (int e = 0; e < kN; e += 2) {
      const QuantScale s0 = sh_qs[BLOCK ? 0 : lane * kN + e], s1 = sh_qs[BLOCK ? 0 : lane * kN + e + 1];
      uint32_t r[kQtRows];
#pragma unroll
      for (int i = 0; i < kQtRows; ++i) {
        float f[kN];
        E::widen(v[i], f);
        r[i] = cvt_fp8x2<E5M2>(quant_one(f[e], s0), quant_one(f[e + 1], s1));
      }
      uint32_t lo[2], hi[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t a = __byte_perm(r[4 * h], r[4 * h + 1], 0x5140), c = __byte_perm(r[4 * h + 2], r[4 * h + 3], 0x5140);
        lo[h] = __byte_perm(a, c, 0x5410);
        hi[h] = __byte_perm(a, c, 0x7632);
      }
      uint8_t* to = sh_tile + (lane * kN + e) * kQtTile + ((group ^ (lane & 15)) * 8);
      *reinterpret_cast<uint2*>(to) = make_uint2(lo[0], lo[1]);
      *reinterpret_cast<uint2*>(to + kQtTile) = make_uint2(hi[0], hi[1]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kQtTile * 8 / kThreads; ++k) {
      const int c = k * (kThreads / 8) + (tid >> 3), u = (tid & 7) * 2, sw = (c / kN) & 15;
      if (c0 + c >= p.C) continue;
      const uint2 lo = *reinterpret_cast<const uint2*>(sh_tile + c * kQtTile + ((u ^ sw) * 8));
      const uint2 hi = *reinterpret_cast<const uint2*>(sh_tile + c * kQtTile + (((u + 1) ^ sw) * 8));
      uint8_t* q = p.q + int64_t(c0 + c) * p.ldq + r0 + u * 8;
      const int left = p.R - (r0 + u * 8);
      if (left >= 16) {
        *reinterpret_cast<uint4*>(q) = make_uint4(lo.x, lo.y, hi.x, hi.y);
      } else {
        const uint32_t w[4] = {lo.x, lo.y, hi.x, hi.y};
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (e < left) q[e] = uint8_t(w[e >> 2] >> (8 * (e & 3)));
      }
    }
  }
}

}  // namespace oapl

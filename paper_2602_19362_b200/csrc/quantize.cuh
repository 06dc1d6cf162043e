// Quantisation of a matrix to 8-bit floating point with one fp32 scale per 1 x 128 or 128 x 128 block,
// as it stands or turned (transposed), for the product in scaled_matmul.cuh.
//
//   amax  = max(largest |x| of the block, 2^-100)
//   scale = amax / top                              (top = 448 for e4m3, 57344 for e5m2)
//   q     = round((0.875 x) / (0.875 amax / top))   to the 8-bit type, nearest even
// top is 0.875 times a power of two, so for 16-bit inputs both sides of that quotient are exact and a
// value half way between two 8-bit numbers is seen as such.  The quotient is correctly rounded: a
// product with the rounded reciprocal, and one residual step (Markstein's theorem on division by
// multiply-add).  With power-of-two scales, scale = 2^ceil(log2(amax / top)) and x / scale is exact.
// A NaN in a block makes its scale and all its values NaN; an infinity makes the scale infinite.
//
// HBM-bound: x is read once and q written once.  A CTA of 256 threads takes a 128 x 128 tile, which it
// holds in registers between the maximum and the rounding (64 values a thread, all its loads in flight
// together).  A turned tile goes through 16 KB of swizzled shared memory, so that it too leaves in
// 16-byte stores.
#pragma once
#include "logits_ops.cuh"

namespace oapl {

constexpr int kQtThreads = 256;
constexpr int kQtTile = 128;

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

// What a block needs to round its values: y = a * inv, and one residual step against b.
struct QuantScale {
  float scale, b, inv;
};
template <int E5M2>
__device__ __forceinline__ QuantScale quant_scale(float amax, bool pow2) {
  constexpr float kTop = E5M2 ? 57344.f : 448.f;
  constexpr int kTopExp = E5M2 ? 15 : 8;  // top = 1.75 * 2^kTopExp
  QuantScale s;
  amax = max_nan(amax, 7.888609052210118e-31f);  // 2^-100
  if (pow2 && amax <= 3.402823466e38f) {
    const uint32_t u = __float_as_uint(amax);
    const int e = int(u >> 23) - kTopExp + ((u & 0x7FFFFFu) > 0x600000u);  // mantissa above 1.75: next power
    s.scale = __uint_as_float(uint32_t(e) << 23);
    s.b = s.scale * 0.875f;
  } else {
    s.scale = amax / kTop;
    s.b = amax * (0.875f / kTop);
  }
  s.inv = 1.f / s.b;
  return s;
}
__device__ __forceinline__ float quant_one(float x, const QuantScale& s, bool finite) {
  const float a = x * 0.875f;
  if (!finite) return a / s.b;
  const float y = a * s.inv;
  return fmaf(fmaf(-y, s.b, a), s.inv, y);
}

template <typename T, int E5M2, bool BLOCK, bool TURN>
__global__ void __launch_bounds__(kQtThreads) quantize_kernel(const QuantParams p) {
  using E = Elem<T>;
  constexpr int kN = E::kN;                   // columns of a thread
  constexpr int kLanes = kQtTile / kN;        // lanes of a row: 16 or 32
  constexpr int kGroups = kQtThreads / kLanes;  // 16 or 8
  constexpr int kRows = kQtTile / kGroups;    // rows of a thread: 8 or 16
  __shared__ float sh_red[TURN && !BLOCK ? kGroups * kQtTile : kQtTile];
  __shared__ float sh_scale[kQtTile];
  __shared__ __align__(16) uint8_t sh_tile[TURN ? kQtTile * kQtTile : 16];

  const int tid = threadIdx.x, lane = tid % kLanes, group = tid / kLanes;
  const int tiles_c = (p.C + kQtTile - 1) / kQtTile;
  const int r0 = int(blockIdx.x / tiles_c) * kQtTile, c0 = int(blockIdx.x % tiles_c) * kQtTile;
  const int row = r0 + group * kRows, col = c0 + lane * kN;

  // ---- the thread's kRows x kN values
  uint4 v[kRows];
  const T* x = reinterpret_cast<const T*>(p.x) + int64_t(row) * p.ldx + col;
  const bool whole = p.vec && col + kN <= p.C;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    v[i] = make_uint4(0, 0, 0, 0);
    if (row + i < p.R) {
      if (whole) {
        v[i] = ldg_stream(reinterpret_cast<const uint4*>(x + i * p.ldx));
      } else {
        float f[kN];
#pragma unroll
        for (int e = 0; e < kN; ++e) f[e] = col + e < p.C ? E::one(x, i * p.ldx + e) : 0.f;
        v[i] = E::narrow(f);
      }
    }
  }

  // ---- largest magnitudes
  QuantScale qs[TURN && !BLOCK ? kN : 1];
  if (TURN && !BLOCK) {
    float m[kN];
#pragma unroll
    for (int e = 0; e < kN; ++e) m[e] = 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      float f[kN];
      E::widen(v[i], f);
#pragma unroll
      for (int e = 0; e < kN; ++e) m[e] = max_nan(m[e], fabsf(f[e]));
    }
#pragma unroll
    for (int e = 0; e < kN; ++e) sh_red[group * kQtTile + lane * kN + e] = m[e];
    __syncthreads();
    if (tid < kQtTile) {
      float a = sh_red[tid];
#pragma unroll
      for (int g = 1; g < kGroups; ++g) a = max_nan(a, sh_red[g * kQtTile + tid]);
      sh_scale[tid] = a;
      if (c0 + tid < p.C)
        p.scale[int64_t(c0 + tid) * p.srow + int64_t(r0 / kQtTile) * p.scol] = quant_scale<E5M2>(a, p.pow2).scale;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < kN; ++e) qs[e] = quant_scale<E5M2>(sh_scale[lane * kN + e], p.pow2);
  } else {
    float m[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      float f[kN];
      E::widen(v[i], f);
      m[i] = fabsf(f[0]);
#pragma unroll
      for (int e = 1; e < kN; ++e) m[i] = max_nan(m[i], fabsf(f[e]));
    }
    if (BLOCK) {
#pragma unroll
      for (int i = 1; i < kRows; ++i) m[0] = max_nan(m[0], m[i]);
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) m[0] = max_nan(m[0], __shfl_xor_sync(0xffffffffu, m[0], o));
      if ((tid & 31) == 0) sh_red[tid >> 5] = m[0];
      __syncthreads();
      float a = sh_red[0];
#pragma unroll
      for (int w = 1; w < kQtThreads / 32; ++w) a = max_nan(a, sh_red[w]);
      qs[0] = quant_scale<E5M2>(a, p.pow2);
      if (tid == 0) {
        const int64_t i = (TURN ? c0 : r0) / kQtTile, j = (TURN ? r0 : c0) / kQtTile;
        p.scale[i * p.srow + j * p.scol] = qs[0].scale;
      }
    } else {
      // the rows of a lane group, every lane of it ending with all maxima
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
#pragma unroll
        for (int o = kLanes / 2; o > 0; o >>= 1) m[i] = max_nan(m[i], __shfl_xor_sync(0xffffffffu, m[i], o));
        if (lane == 0) sh_red[group * kRows + i] = m[i];
      }
      __syncthreads();
      if (tid < kQtTile && r0 + tid < p.R)
        p.scale[int64_t(r0 + tid) * p.srow + int64_t(c0 / kQtTile) * p.scol] = quant_scale<E5M2>(sh_red[tid], p.pow2).scale;
    }
  }

  // ---- round and store
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    if (!BLOCK && !TURN) qs[0] = quant_scale<E5M2>(sh_red[group * kRows + i], p.pow2);
    float f[kN];
    E::widen(v[i], f);
#pragma unroll
    for (int e = 0; e < kN; ++e) {
      const QuantScale& s = qs[TURN && !BLOCK ? e : 0];
      f[e] = quant_one(f[e], s, s.scale <= 3.402823466e38f);
    }
    uint32_t w[kN / 4];
#pragma unroll
    for (int e = 0; e < kN; e += 4)
      w[e / 4] = cvt_fp8x2<E5M2>(f[e], f[e + 1]) | (cvt_fp8x2<E5M2>(f[e + 2], f[e + 3]) << 16);
    if (TURN) {
      v[i].x = w[0];
      if (kN == 8) v[i].y = w[1];
    } else if (row + i < p.R) {
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
  if (TURN) {
    // Row e of the turned tile gets kRows bytes from every lane group.  8-byte unit u of row c sits at
    // u ^ (c / kN), which spreads a warp's stores over all banks.
#pragma unroll
    for (int e = 0; e < kN; ++e) {
#pragma unroll
      for (int h = 0; h < kRows / 8; ++h) {
        uint32_t w[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          uint32_t b[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint4& s = v[h * 8 + k * 4 + i];
            b[i] = ((e < 4 ? s.x : s.y) >> (8 * (e & 3))) & 0xFFu;
          }
          w[k] = b[0] | (b[1] << 8) | (b[2] << 16) | (b[3] << 24);
        }
        const int c = lane * kN + e, u = group * (kRows / 8) + h;
        *reinterpret_cast<uint2*>(sh_tile + c * kQtTile + ((u ^ (lane & 15)) * 8)) = make_uint2(w[0], w[1]);
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int c = k * 32 + (tid >> 3), u = (tid & 7) * 2, sw = (c / kN) & 15;
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

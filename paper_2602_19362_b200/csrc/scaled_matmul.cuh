// C = A . B^T of two matrices of 8-bit floating point with a scale per block of 128 along K:
//
//   C[m, n] (+)= sum_kb sA[m / ga, kb] sB[n / gb, kb] sum_{k in block kb} a[m, k] b[n, k]
//
// The inner sums run on the tensor cores (tcgen05.mma kind::f8f6f4, fp32 accumulators in TMEM).  The
// scales change every 128 values of K, so an accumulator holds one K block only: the epilogue warps
// take it out of TMEM, multiply by the product of the two scales and add in fp32 registers, while the
// tensor cores fill the other accumulator.
//
// CTA pairs (cta_group::2) share a 256 x 256 tile; a K block is 128 bytes, one swizzle row, and takes
// the tensor cores about 512 cycles per pair.  In that time the eight epilogue warps of a CTA move
// 128 x 256 accumulators: per warp 8 loads of 16 columns and 64 two-wide multiply-adds, so they fit
// with room for scales that differ per column.
// Warp 0 issues TMA loads, warp 1 owns TMEM and (in the leader) issues the MMAs, warp 2 copies the
// scales of each K block to shared memory with cp.async, warps 4 to 11 are the epilogue: quadrant
// warp & 3 of the TMEM lanes, one half of the columns each.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "logits_ops.cuh"
#include "sm100_ptx.cuh"

namespace oapl {

constexpr int kSmTile = 256;       // rows and columns of a pair's tile
constexpr int kSmHalf = 128;       // rows of A, and of B, that a CTA loads
constexpr int kSmKB = 128;         // K values (bytes) of a block
constexpr int kSmStages = 5;
constexpr int kSmStageBytes = 2 * kSmHalf * kSmKB;
constexpr int kSmScaleStages = 8;
constexpr int kSmScaleFloats = kSmHalf + kSmTile;  // row scales of this CTA, column scales of the tile
constexpr int kSmEpiWarps = 8;
constexpr int kSmThreads = 32 * (4 + kSmEpiWarps);
// Registers of a thread: 168 at launch (what 384 threads can have), then 56 for the four warps that move
// data and 224 for the epilogue: 128 * 56 + 256 * 224 = 384 * 168.
constexpr int kSmRegs = 168, kSmRegsLow = 56, kSmRegsHigh = 224;
static_assert(128 * kSmRegsLow + 256 * kSmRegsHigh == kSmThreads * kSmRegs, "register split");
constexpr int kSmOutPitch = 33;    // words per row of a warp's 32 x 32 output piece
constexpr int kSmOutBytes = kSmEpiWarps * 32 * kSmOutPitch * 4;
constexpr size_t kSmSmemBytes = size_t(kSmStages) * kSmStageBytes + kSmScaleStages * kSmScaleFloats * 4 +
                                kSmOutBytes + 1024 /*align*/ + 512 /*barriers*/;
static_assert(kSmSmemBytes <= 227 * 1024, "shared memory of a CTA");

enum { OUT_BF16 = 0, OUT_F16 = 1, OUT_F32 = 2 };

struct ScaledParams {
  const float* sa;
  const float* sb;
  int64_t sa_row, sa_col, sb_row, sb_col;  // strides of the scales
  int32_t ga, gb;                          // rows that share a scale: 1 or 128
  int32_t M, N, K;
  void* C;
  int64_t ldc;
  int32_t accumulate;
  int32_t wide;  // every row of C starts on a 32-byte boundary
  int32_t e5_a, e5_b;
  int32_t mt, nt, group;  // tiles along M and N; m tiles that are walked together
  int32_t* err;
};

// D[tmem] (+)= A B^T, 8-bit floating point operands, K = 32 per instruction, for both CTAs of the pair
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ uint32_t make_idesc_f8(int m, int n, int e5_a, int e5_b) {
  return (1u << 4)                  // D format f32
         | (uint32_t(e5_a) << 7)    // A format: 0 e4m3, 1 e5m2
         | (uint32_t(e5_b) << 10)   // B format
         | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
// one arrival on `bar` once all cp.async of this thread so far have landed
__device__ __forceinline__ void cp_async_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}

// Tile number t: groups of `group` tiles along M, inside a group M fastest, so that the tiles in work at
// one time share few rows of A and of B.
__device__ __forceinline__ bool scaled_tile(const ScaledParams& p, int j, int& m0, int& n0) {
  const int64_t t = int64_t(blockIdx.x >> 1) + int64_t(j) * (gridDim.x >> 1);
  if (t >= int64_t(p.mt) * p.nt) return false;
  const int64_t per = int64_t(p.group) * p.nt;
  const int g = int(t / per);
  const int r = int(t - g * per);
  const int rows = min(p.group, p.mt - g * p.group);
  m0 = (g * p.group + r % rows) * kSmTile;
  n0 = (r / rows) * kSmTile;
  return true;
}

template <int OUT>
struct OutElem;
template <>
struct OutElem<OUT_BF16> {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float get(T x) { return __bfloat162float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2bfloat16_rn(x); }
};
template <>
struct OutElem<OUT_F16> {
  using T = __half;
  static __device__ __forceinline__ float get(T x) { return __half2float(x); }
  static __device__ __forceinline__ T put(float x) { return __float2half_rn(x); }
};
template <>
struct OutElem<OUT_F32> {
  using T = float;
  static __device__ __forceinline__ float get(T x) { return x; }
  static __device__ __forceinline__ T put(float x) { return x; }
};

// 32 bytes to or from global memory in one access
__device__ __forceinline__ void st32b(void* p, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

// PERCOL: the columns' scales differ from column to column (gb = 1); otherwise a column half has one.
template <int OUT, bool PERCOL>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kSmThreads, 1)
scaled_matmul_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                     const ScaledParams p) {
  using O = OutElem<OUT>;
  using OT = typename O::T;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  constexpr uint32_t kScaleOff = kSmStages * kSmStageBytes;
  constexpr uint32_t kOutOff = kScaleOff + kSmScaleStages * kSmScaleFloats * 4;
  constexpr uint32_t kBarOff = kOutOff + kSmOutBytes;
  float* scales = reinterpret_cast<float*>(smem + kScaleOff);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kBarOff);
  const uint32_t bar0 = base + kBarOff;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kSmStages + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * kSmStages + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * kSmStages + 2 + b); };
  auto sfull_bar = [&](int s) { return bar0 + 8u * (2 * kSmStages + 4 + s); };
  auto sempty_bar = [&](int s) { return bar0 + 8u * (2 * kSmStages + 4 + kSmScaleStages + s); };
  constexpr int kBars = 2 * kSmStages + 4 + 2 * kSmScaleStages;
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bars + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + kBars + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = cluster_ctarank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < kSmStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(tfull_bar(b), 1);
      mbar_init(tempty_bar(b), 2 * kSmEpiWarps);  // the leader's copy counts the warps of both CTAs
    }
    for (int s = 0; s < kSmScaleStages; ++s) {
      mbar_init(sfull_bar(s), 32);
      mbar_init(sempty_bar(s), kSmEpiWarps);
    }
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmA);
    tma_prefetch_desc(&tmB);
  }
  if (warp == 1) tmem_alloc(smem_u32((const void*)tmem_slot), 512);
  tc_fence_before();
  __syncthreads();
  cluster_sync_all();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int nk = (p.K + kSmKB - 1) / kSmKB;
  int m0, n0;

  if (warp < 4) {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kSmRegsLow));
  if (warp == 0) {
    // ------------------------------------------------------------ operand loads
    if (lane == 0) {
      uint32_t it = 0;
      bool ok = true;
      for (int j = 0; ok && scaled_tile(p, j, m0, n0); ++j) {
        for (int kb = 0; kb < nk; ++kb, ++it) {
          const int s = it % kSmStages;
          if (!mbar_wait(empty_bar(s), ((it / kSmStages) & 1u) ^ 1u, abort_flag)) {
            ok = false;
            break;
          }
          const uint32_t sa = base + s * kSmStageBytes;
          const uint32_t fb = mapa_shared(full_bar(s), 0);
          if (rank == 0) mbar_expect_tx(full_bar(s), 2 * kSmStageBytes);
          tma_load_2d(sa, &tmA, fb, kb * kSmKB, m0 + int(rank) * kSmHalf);
          tma_load_2d(sa + kSmHalf * kSmKB, &tmB, fb, kb * kSmKB, n0 + int(rank) * kSmHalf);
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs (leader CTA)
    if (lane == 0 && rank == 0) {
      const uint32_t idesc = make_idesc_f8(kSmTile, kSmTile, p.e5_a, p.e5_b);
      uint32_t it = 0;
      bool ok = true;
      for (int j = 0; ok && scaled_tile(p, j, m0, n0); ++j) {
        for (int kb = 0; kb < nk; ++kb, ++it) {
          const int s = it % kSmStages, buf = it & 1;
          if (!mbar_wait(tempty_bar(buf), ((it >> 1) & 1u) ^ 1u, abort_flag) ||
              !mbar_wait(full_bar(s), (it / kSmStages) & 1u, abort_flag)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint32_t sa = base + s * kSmStageBytes, sb = sa + kSmHalf * kSmKB;
#pragma unroll
          for (int kk = 0; kk < kSmKB / 32; ++kk)
            umma_f8(tmem_base + buf * kSmTile, smem_desc_sw128(sa + kk * 32, 16, 1024),
                    smem_desc_sw128(sb + kk * 32, 16, 1024), idesc, kk ? 1u : 0u);
          umma_commit_pair(empty_bar(s));
          umma_commit_pair(tfull_bar(buf));
        }
      }
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ scales
    uint32_t it = 0;
    bool ok = true;
    for (int j = 0; ok && scaled_tile(p, j, m0, n0); ++j) {
      const int mrow = m0 + int(rank) * kSmHalf;
      for (int kb = 0; kb < nk; ++kb, ++it) {
        const int s = it % kSmScaleStages;
        ok = mbar_wait(sempty_bar(s), ((it / kSmScaleStages) & 1u) ^ 1u, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        const uint32_t dst = smem_u32(scales + s * kSmScaleFloats);
        const float* sa = p.sa + kb * p.sa_col;
        const float* sb = p.sb + kb * p.sb_col;
#pragma unroll
        for (int i = 0; i < kSmHalf / 32; ++i) {
          const int r = mrow + i * 32 + lane;
          const bool in = r < p.M;
          cp_async4(dst + 4 * (i * 32 + lane), in ? sa + int64_t(p.ga == 1 ? r : r >> 7) * p.sa_row : sa, in);
        }
        if (PERCOL) {
#pragma unroll
          for (int i = 0; i < kSmTile / 32; ++i) {
            const int c = n0 + i * 32 + lane;
            const bool in = c < p.N;
            cp_async4(dst + 4 * (kSmHalf + i * 32 + lane), in ? sb + int64_t(c) * p.sb_row : sb, in);
          }
        } else if (lane < 2) {
          const int c = n0 + lane * 128;
          const bool in = c < p.N;
          cp_async4(dst + 4 * (kSmHalf + lane), in ? sb + int64_t(c >> 7) * p.sb_row : sb, in);
        }
        cp_async_arrive(sfull_bar(s));
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  } else {
    // ------------------------------------------------------------ epilogue
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSmRegsHigh));
    const int quad = warp & 3;
    const int half = (warp - 4) >> 2;  // columns [128 half, 128 half + 128)
    const uint32_t tlane = tmem_base + (uint32_t(quad * 32) << 16) + half * 128;
    float* piece = reinterpret_cast<float*>(smem + kOutOff) + (warp - 4) * 32 * kSmOutPitch;
    uint32_t it = 0;
    bool ok = true;
    for (int j = 0; ok && scaled_tile(p, j, m0, n0); ++j) {
      uint64_t acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = 0;
      for (int kb = 0; kb < nk; ++kb, ++it) {
        const int s = it % kSmScaleStages, buf = it & 1;
        ok = mbar_wait(sfull_bar(s), (it / kSmScaleStages) & 1u, abort_flag);
        ok = ok && mbar_wait(tfull_bar(buf), (it >> 1) & 1u, abort_flag);
        if (!__all_sync(0xffffffffu, ok)) {
          ok = false;
          break;
        }
        tc_fence_after();
        const float* sc = scales + s * kSmScaleFloats;
        const float fa = sc[quad * 32 + lane];
        const float f = PERCOL ? fa : fa * sc[kSmHalf + half];
        const uint64_t f2 = pack2(f, f);
        const uint32_t ta = tlane + buf * kSmTile;
        uint32_t ra[32], rb[32];
        auto add = [&](const uint32_t (&r)[32], int c) {
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const uint64_t v = pack2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
            if (PERCOL) {
              const uint64_t g = *reinterpret_cast<const uint64_t*>(sc + kSmHalf + half * 128 + c * 32 + 2 * i);
              acc[c * 16 + i] = fma2(v, mul2(f2, g), acc[c * 16 + i]);
            } else {
              acc[c * 16 + i] = fma2(v, f2, acc[c * 16 + i]);
            }
          }
        };
        tmem_ld32(ta, ra);
        tmem_ld32(ta + 32, rb);
        tmem_ld_wait();
        add(ra, 0);
        tmem_ld32(ta + 64, ra);
        add(rb, 1);
        tmem_ld32(ta + 96, rb);
        tmem_ld_wait();
        // the accumulator is in registers: hand it back
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(mapa_shared(tempty_bar(buf), 0));
        add(ra, 2);
        add(rb, 3);
        __syncwarp();
        if (lane == 0) mbar_arrive(sempty_bar(s));
      }
      if (!ok) break;

      // ---- the tile's 32 rows x 128 columns of this warp
      const int row0 = m0 + int(rank) * kSmHalf + quad * 32;
      const int col0 = n0 + half * 128;
      if (row0 >= p.M || col0 >= p.N) continue;
      OT* C = reinterpret_cast<OT*>(p.C);
      if (p.wide && !p.accumulate && col0 + 128 <= p.N) {
        if (row0 + lane < p.M) {
          OT* dst = C + int64_t(row0 + lane) * p.ldc + col0;
          constexpr int kPer = 32 / sizeof(OT);  // elements of a 32-byte store
#pragma unroll
          for (int q = 0; q < 128 / kPer; ++q) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              float lo, hi;
              if (OUT == OUT_F32) {
                unpack2(acc[q * 4 + i / 2], lo, hi);
                w[i] = __float_as_uint(i & 1 ? hi : lo);
              } else {
                unpack2(acc[q * 8 + i], lo, hi);
                if (OUT == OUT_BF16) {
                  w[i] = pack_bf16x2(lo, hi);
                } else {
                  const __half2 h = __floats2half2_rn(lo, hi);
                  w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
              }
            }
            st32b(dst + q * kPer, w);
          }
        }
      } else {
        // any alignment, edges, accumulation: 32 x 32 pieces through shared memory, a row at a time
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            float lo, hi;
            unpack2(acc[q * 16 + i], lo, hi);
            piece[lane * kSmOutPitch + 2 * i] = lo;
            piece[lane * kSmOutPitch + 2 * i + 1] = hi;
          }
          __syncwarp();
          const int col = col0 + q * 32 + lane;
          if (col < p.N) {
            const int rows = min(32, p.M - row0);
            OT* dst = C + int64_t(row0) * p.ldc + col;
#pragma unroll 4
            for (int i = 0; i < rows; ++i) {
              float x = piece[i * kSmOutPitch + lane];
              if (p.accumulate) x += O::get(dst[i * p.ldc]);
              dst[i * p.ldc] = O::put(x);
            }
          }
        }
      }
    }
  }

  // ---------------------------------------------------------------- teardown
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (threadIdx.x == 0) {
      if (p.err) atomicCAS(p.err, 0, -8 /*OAPL_ERR_DEVICE_TIMEOUT*/);
      const long long t0 = clock64();  // loads in flight land before shared memory is released
      while (clock64() - t0 < 2000000LL) {
      }
    }
    __syncthreads();
  }
  cluster_sync_all();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

}  // namespace oapl

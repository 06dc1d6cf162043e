// C = A . B^T of two matrices of 8-bit floating point with a scale per block of 128 along K:
//
//   C[m, n] (+)= sum_kb sA[m / ga, kb] sB[n / gb, kb] sum_{k in block kb} a[m, k] b[n, k]
//
// The inner sums run on the tensor cores (tcgen05.mma kind::f8f6f4, fp32 accumulators in TMEM).  The
// scales change every 128 values of K, so an accumulator holds one K block only: the epilogue warps
// take it out of TMEM, multiply by the product of the two scales and add in fp32 registers, while the
// tensor cores fill the other accumulator.
//
// CTA pairs (cta_group::2) share a 256 x 256 tile; a K block is 128 bytes, one swizzle row, and takes the
// tensor cores 512 cycles per pair.  What bounds it is the hand-over of the two accumulators that TMEM has room
// for: an accumulator is away for about 900 cycles between the end of its MMAs and the next ones (commit, the
// warps' wake-up, TMEM loads, hand-back), so a K block takes 725 cycles, 667 with an epilogue that does nothing.
// Halves of 128 columns would give four accumulators, but read A twice from shared memory: slower.  Long calls run at
// the power limit: 4096 x 152064 x 3584 in 1.87 ms (single calls after a pause; 2.2 ms in a row), 2.0 to 2.4 PFLOP/s, in
// a row at about 1.4 GHz.  With a scale per column the epilogue has two operations per pair of values in place of one
// and 32 more reads of shared memory: 1200 cycles per K block, 8192^3 621 us against 443.
// Warp 0 issues TMA loads, warp 1 owns TMEM and (in the leader) issues the MMAs, warps 2 and 3 copy the scales
// of rows and columns to shared memory a few K blocks ahead (cp.async).  They arrive on the accumulator's barrier
// as the tensor cores do, so the epilogue waits once per block.  Warps 4 to 11 are the epilogue: quadrant warp & 3
// of the TMEM lanes, one half of the columns each.  The result leaves through TMA stores while the next tile runs.
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
constexpr int kSmStages = 4;
constexpr int kSmStageBytes = 2 * kSmHalf * kSmKB;
constexpr int kSmSlots = 16;       // K blocks whose scales have room in shared memory
constexpr int kSmAhead = 6;        // K blocks that their copies run ahead
constexpr int kSmSlotFloats = kSmHalf + kSmTile;  // row scales of this CTA, column scales of the tile
constexpr int kSmFree = 4;         // the epilogue frees slots in fours
constexpr int kSmEpiWarps = 8;
constexpr int kSmThreads = 32 * (4 + kSmEpiWarps);
constexpr int kSmOutCols = 32;     // columns of a warp's output piece
constexpr int kSmOutPitch = kSmOutCols + 1;
constexpr int kSmOutWarp = 8192;   // of an epilogue warp: two pieces of 32 rows x 128 bytes, or one of 32 x 33 floats
constexpr int kSmOutBytes = kSmEpiWarps * kSmOutWarp;
static_assert(32 * kSmOutPitch * 4 <= kSmOutWarp, "a padded piece fits");
constexpr size_t kSmSmemBytes = size_t(kSmStages) * kSmStageBytes + kSmSlots * kSmSlotFloats * 4 +
                                kSmOutBytes + 1024 /*align*/ + 512 /*barriers*/;
static_assert(kSmSmemBytes <= 227 * 1024, "shared memory of a CTA");
// Registers of a thread: 168 at launch (what 384 threads can have), then 24 for the four warps that move data
// and 240 for the epilogue, whose loop holds 192 values: 128 * 24 + 256 * 240 = 384 * 168.  (In a row 5 % slower with
// 40 / 232 and 16 % with 56 / 224, where the loop spills its values.  With this split the compiler still keeps some 20
// words in local memory, of which a warp reads two per K block, 1.4 % of its instructions.)
constexpr int kSmRegs = 168, kSmRegsLow = 24, kSmRegsHigh = 240;
static_assert(128 * kSmRegsLow + 256 * kSmRegsHigh == kSmThreads * kSmRegs, "register split");

enum { OUT_BF16 = 0, OUT_F16 = 1, OUT_F32 = 2 };

// Both kernels' give-up path.  wait_cycles: limit of every pipeline wait, in SM cycles.  skip_step: for its test, a
// pipeline step (counted from 1, 0: none) whose loads every CTA leaves out, so that the waits for it run out.  Their
// places in the two structs were measured, since the compiler's registers turn on them: behind `err` 4096 x 152064 x
// 3584 takes 1.86 ms, in the gaps before it 1.91; 152064 x 3584 with 64 rows of A 107 and 99.5 us.
struct ScaledParams {
  const float* sa;
  const float* sb;
  int64_t sa_row, sa_col, sb_row, sb_col;  // strides of the scales
  int32_t ga, gb;                          // rows that share a scale: 1 or 128
  int32_t M, N, K;
  void* C;
  int64_t ldc;
  int32_t accumulate;
  int32_t bulk;  // C leaves by TMA: 1 store, 2 add (fp32), 0 not (rows off 16-byte boundaries, 16-bit sums)
  int32_t e5_a, e5_b;
  int32_t mt, nt, group;  // tiles along M and N; m tiles that are walked together
  int32_t* err;
  long long wait_cycles;
  uint32_t skip_step;
};

// Waits for the warp's loads from TMEM; naming the registers keeps their uses behind it.
__device__ __forceinline__ void tmem_ld_wait_on(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                 "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]),
                 "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]),
                 "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]),
                 "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
               :
               : "memory");
}
__device__ __forceinline__ void tmem_ld_wait_on(uint32_t (&a)[32], uint32_t (&b)[32]) {
  tmem_ld_wait_on(a);
  asm volatile("" : "+r"(b[0]), "+r"(b[1]), "+r"(b[2]), "+r"(b[3]), "+r"(b[4]), "+r"(b[5]), "+r"(b[6]), "+r"(b[7]),
               "+r"(b[8]), "+r"(b[9]), "+r"(b[10]), "+r"(b[11]), "+r"(b[12]), "+r"(b[13]), "+r"(b[14]),
               "+r"(b[15]), "+r"(b[16]), "+r"(b[17]), "+r"(b[18]), "+r"(b[19]), "+r"(b[20]), "+r"(b[21]),
               "+r"(b[22]), "+r"(b[23]), "+r"(b[24]), "+r"(b[25]), "+r"(b[26]), "+r"(b[27]), "+r"(b[28]),
               "+r"(b[29]), "+r"(b[30]), "+r"(b[31]) : : "memory");
}

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
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r != 0;
}
// mbar_wait by a whole warp, with one answer for all lanes
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag, long long limit) {
  if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, limit));
}
__device__ __forceinline__ uint32_t make_idesc_f8(int m, int n, int e5_a, int e5_b) {
  return (1u << 4)                  // D format f32
         | (uint32_t(e5_a) << 7)    // A format: 0 e4m3, 1 e5m2
         | (uint32_t(e5_b) << 10)   // B format
         | (uint32_t(n >> 3) << 17) | (uint32_t(m >> 4) << 24);
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
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

// Tile store from shared memory (bulk group); what lies outside the tensor is clipped.
__device__ __forceinline__ void tma_store_2d(const void* tmap, uint32_t src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                   reinterpret_cast<uint64_t>(tmap)),
               "r"(src), "r"(x), "r"(y)
               : "memory");
}

// PERCOL: the columns' scales differ from column to column (gb = 1); otherwise a column half has one.
template <int OUT, bool PERCOL>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kSmThreads, 1)
scaled_matmul_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                     const __grid_constant__ CUtensorMap tmC, const ScaledParams p) {
  using O = OutElem<OUT>;
  using OT = typename O::T;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  constexpr uint32_t kScaleOff = kSmStages * kSmStageBytes;
  constexpr uint32_t kOutOff = kScaleOff + kSmSlots * kSmSlotFloats * 4;
  constexpr uint32_t kBarOff = kOutOff + kSmOutBytes;
  float* scales = reinterpret_cast<float*>(smem + kScaleOff);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kBarOff);
  const uint32_t bar0 = base + kBarOff;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kSmStages + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * kSmStages + b); };       // accumulator and scales ready
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * kSmStages + 2 + b); };  // accumulator handed back
  auto sempty_bar = [&](int h) { return bar0 + 8u * (2 * kSmStages + 4 + h); };  // slots free again
  constexpr int kBars = 2 * kSmStages + 4 + kSmSlots / kSmFree;
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
      mbar_init(tfull_bar(b), 3);                 // the tensor cores, warps 2 and 3
      mbar_init(tempty_bar(b), 2 * kSmEpiWarps);  // the leader's copy counts the warps of both CTAs
    }
    for (int h = 0; h < kSmSlots / kSmFree; ++h) mbar_init(sempty_bar(h), kSmEpiWarps);
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
          if (it + 1 == p.skip_step) continue;
          const int s = it % kSmStages;
          if (!mbar_wait(empty_bar(s), ((it / kSmStages) & 1u) ^ 1u, abort_flag, p.wait_cycles)) {
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
    // the whole warp walks the loop and one elected lane issues, so that the descriptors stay uniform
    if (rank == 0) {
      const uint32_t idesc = make_idesc_f8(kSmTile, kSmTile, p.e5_a, p.e5_b);
      const uint64_t da0 = smem_desc_sw128(base, 16, 1024), db0 = smem_desc_sw128(base + kSmHalf * kSmKB, 16, 1024);
      uint32_t it = 0;
      bool ok = true;
      for (int j = 0; ok && scaled_tile(p, j, m0, n0); ++j) {
        for (int kb = 0; kb < nk; ++kb, ++it) {
          const int s = it % kSmStages, buf = it & 1;
          ok = warp_wait(full_bar(s), (it / kSmStages) & 1u, abort_flag, p.wait_cycles) &&
               warp_wait(tempty_bar(buf), ((it >> 1) & 1u) ^ 1u, abort_flag, p.wait_cycles);
          if (!ok) break;
          tc_fence_after();
          if (elect_one()) {
            const uint64_t da = da0 + uint32_t(s * (kSmStageBytes >> 4)), db = db0 + uint32_t(s * (kSmStageBytes >> 4));
#pragma unroll
            for (int kk = 0; kk < kSmKB / 32; ++kk)
              umma_f8(tmem_base + buf * kSmTile, da + 2 * kk, db + 2 * kk, idesc, kk ? 1u : 0u);
            umma_commit_pair(tfull_bar(buf));
            umma_commit_pair(empty_bar(s));
          }
          __syncwarp();
        }
      }
    }
  } else {
    // ------------------------------------------------------------ scales: warp 2 the rows', warp 3 the columns'
    const bool cols = warp == 3;
    const int64_t step = cols ? (PERCOL ? 32 * p.sb_row : 0) : (p.ga == 1 ? 32 * p.sa_row : 0);
    const int64_t ahead = cols ? p.sb_col : p.sa_col;
    const uint32_t dst0 = smem_u32(scales) + 4 * (lane + (cols ? kSmHalf : 0));
    const float* at = p.sa;
    int pj = 0, pkb = 0, left = 0;  // left: rows from this lane's first one on; 32 apart, as far as they go
    auto seek = [&]() {
      left = 0;
      if (!scaled_tile(p, pj, m0, n0)) return;
      if (cols) {
        const int c = n0 + (PERCOL ? lane : lane * 128);
        if (PERCOL || lane < 2) left = PERCOL ? p.N - c : min(p.N - c, 1);
        at = p.sb + int64_t(PERCOL ? c : c >> 7) * p.sb_row;
      } else {
        const int r = m0 + int(rank) * kSmHalf + lane;
        left = min(p.M - r, kSmHalf - lane);
        at = p.sa + int64_t(p.ga == 1 ? r : r >> 7) * p.sa_row;
      }
    };
    auto copy = [&](uint32_t t) {  // of the next K block, number t; rows behind the last keep what was there
      const uint32_t dst = dst0 + (t % kSmSlots) * (kSmSlotFloats * 4);
#pragma unroll
      for (int i = 0; i < kSmTile / 32; ++i)
        if (i * 32 < left) cp_async4(dst + i * 128, at + i * step);
      at += ahead;
      if (++pkb == nk) {
        pkb = 0;
        ++pj;
        seek();
      }
    };
    seek();
    bool ok = true;
#pragma unroll 1
    for (uint32_t t = 0; t < kSmAhead; ++t) {
      copy(t);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    uint32_t it = 0;
    for (int j = 0, m, n; ok && scaled_tile(p, j, m, n); ++j) {
      for (int kb = 0; kb < nk; ++kb, ++it) {
        const uint32_t t = it + kSmAhead;
        if (t % kSmFree == 0) {
          ok = warp_wait(sempty_bar(t % kSmSlots / kSmFree), ((t / kSmSlots) & 1u) ^ 1u, abort_flag, p.wait_cycles);
          if (!ok) break;
        }
        copy(t);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(kSmAhead) : "memory");  // this block's have landed
        __syncwarp();
        // the barrier's phase of two blocks before has to be over, or this arrival would count for it
        if (it >= 2) {
          ok = warp_wait(tfull_bar(it & 1), ((it >> 1) & 1u) ^ 1u, abort_flag, p.wait_cycles);
          if (!ok) break;
        }
        if (lane == 0) mbar_arrive(tfull_bar(it & 1));
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
    float* piece = reinterpret_cast<float*>(smem + kOutOff + (warp - 4) * kSmOutWarp);
    const uint32_t back0 = mapa_shared(tempty_bar(0), 0);
    const float* sc_row = scales + quad * 32 + lane;
    const float* sc_col = scales + kSmHalf + (PERCOL ? half * 128 : half);
    uint32_t buf = 0, parity = 0, slot = 0;
    bool ok = true;
    int j = 0;
    for (; scaled_tile(p, j, m0, n0); ++j) {
      float2 acc[64];
#pragma unroll
      for (int i = 0; i < 64; ++i) acc[i] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int kb = 0; kb < nk; ++kb) {
        ok = warp_wait(tfull_bar(buf), parity, abort_flag, p.wait_cycles);
        if (!ok) break;
        tc_fence_after();
        const uint32_t ta = tlane + buf * kSmTile;
        uint32_t ra[32], rb[32];
        tmem_ld32(ta, ra);
        tmem_ld32(ta + 32, rb);
        const float* sc = sc_col + slot * kSmSlotFloats;
        const float fa = sc_row[slot * kSmSlotFloats], f = PERCOL ? fa : fa * sc[0];
        float4 g[4];  // scales of the next 16 columns
        auto scales_of = [&](int c) {
          if (PERCOL) {
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] = *reinterpret_cast<const float4*>(sc + c + 4 * i);
          }
        };
        auto add = [&](const uint32_t (&r)[32], int c) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float4 now[4];
            if (PERCOL) {
#pragma unroll
              for (int i = 0; i < 4; ++i) now[i] = g[i];
              if (c + h < 4) scales_of(c * 32 + h * 16 + 16);
            }
#pragma unroll
            for (int i = h * 16; i < h * 16 + 16; i += 4) {
              const float2 v0 = make_float2(__uint_as_float(r[i]), __uint_as_float(r[i + 1]));
              const float2 v1 = make_float2(__uint_as_float(r[i + 2]), __uint_as_float(r[i + 3]));
              float2 g0 = make_float2(f, f), g1 = g0;
              if (PERCOL) {
                const float4 s4 = now[(i & 15) / 4];
                g0 = __fmul2_rn(g0, make_float2(s4.x, s4.y));
                g1 = __fmul2_rn(g1, make_float2(s4.z, s4.w));
              }
              acc[c * 16 + i / 2] = __ffma2_rn(v0, g0, acc[c * 16 + i / 2]);
              acc[c * 16 + i / 2 + 1] = __ffma2_rn(v1, g1, acc[c * 16 + i / 2 + 1]);
            }
          }
        };
        scales_of(0);
        tmem_ld_wait_on(ra, rb);
        add(ra, 0);
        tmem_ld32(ta + 64, ra);
        add(rb, 1);
        tmem_ld32(ta + 96, rb);
        tmem_ld_wait_on(ra, rb);
        // the accumulator is in registers: hand it back
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(back0 + 8u * buf);
        add(ra, 2);
        add(rb, 3);
        parity ^= buf;
        buf ^= 1;
        if ((++slot & (kSmFree - 1)) == 0) {
          __syncwarp();
          if (lane == 0) mbar_arrive(sempty_bar(slot / kSmFree - 1));
          slot &= kSmSlots - 1;
        }
      }
      if (!ok) break;

      // ---- the tile's 32 rows x 128 columns of this warp
      const int row0 = m0 + int(rank) * kSmHalf + quad * 32;
      const int col0 = n0 + half * 128;
      if (row0 >= p.M || col0 >= p.N) continue;
      OT* C = reinterpret_cast<OT*>(p.C);
      if (p.bulk) {
        // 128 bytes of every row at a time through one of two swizzled 4 KB pieces; the stores run on under the
        // next tile
        constexpr int kCols = 128 / sizeof(OT);
        uint8_t* two = smem + kOutOff + (warp - 4) * kSmOutWarp;
#pragma unroll
        for (int q = 0; q < 128 / kCols; ++q) {
          uint8_t* out = two + (q & 1) * 4096;
          if (lane == 0) tma_store_wait_read<1>();
          __syncwarp();
          uint4* line = reinterpret_cast<uint4*>(out + lane * 128);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (OUT == OUT_F32) {
                const float2 x = acc[q * 16 + c * 2 + i / 2];
                w[i] = __float_as_uint(i & 1 ? x.y : x.x);
              } else {
                const float2 x = acc[q * 32 + c * 4 + i];
                if (OUT == OUT_BF16) {
                  w[i] = pack_bf16x2(x.x, x.y);
                } else {
                  const __half2 h = __floats2half2_rn(x.x, x.y);
                  w[i] = *reinterpret_cast<const uint32_t*>(&h);
                }
              }
            }
            line[c ^ (lane & 7)] = make_uint4(w[0], w[1], w[2], w[3]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            const int x = col0 + q * kCols;
            if (x < p.N) {
              if (p.bulk == 2)
                tma_reduce_add_2d(&tmC, smem_u32(out), x, row0);
              else
                tma_store_2d(&tmC, smem_u32(out), x, row0);
            }
            tma_store_commit();
          }
        }
      } else {
        // any alignment, sums in 16 bits: 32 x 32 pieces through shared memory, a row at a time
        const int rows = min(32, p.M - row0);
#pragma unroll
        for (int q = 0; q < 128 / kSmOutCols; ++q) {
          __syncwarp();
#pragma unroll
          for (int i = 0; i < kSmOutCols / 2; ++i) {
            piece[lane * kSmOutPitch + 2 * i] = acc[q * (kSmOutCols / 2) + i].x;
            piece[lane * kSmOutPitch + 2 * i + 1] = acc[q * (kSmOutCols / 2) + i].y;
          }
          __syncwarp();
          const int c = lane % kSmOutCols, col = col0 + q * kSmOutCols + c;
          if (col < p.N) {
            OT* dst = C + int64_t(row0) * p.ldc + col;
#pragma unroll 4
            for (int i = lane / kSmOutCols; i < rows; i += 32 / kSmOutCols) {
              float x = piece[i * kSmOutPitch + c];
              if (p.accumulate) x += O::get(dst[i * p.ldc]);
              dst[i * p.ldc] = O::put(x);
            }
          }
        }
      }
    }
    // after a wait that ran out: NaN in the warp's part of this tile and of all that were to come
    for (; !ok && scaled_tile(p, j, m0, n0); ++j) {
      const int row0 = m0 + int(rank) * kSmHalf + quad * 32, col0 = n0 + half * 128 + lane;
      for (int i = 0; i < 32 && row0 + i < p.M; ++i)
        for (int c = col0; c < min(p.N, col0 - lane + 128); c += 32)
          reinterpret_cast<OT*>(p.C)[int64_t(row0 + i) * p.ldc + c] = O::put(__int_as_float(0x7FC00000));
    }
    if (lane == 0) tma_store_wait_all();  // before shared memory is released
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

// ------------------------------------------------------------------------------------ few rows
// The same product for at most 64 rows of A (decoded tokens): HBM-bound by B, the weight.  The roles are
// swapped: rows of B fill the 128 lanes of the accumulator and the rows of A are its NT = 16, 32 or 64 columns,
// so a token costs what it needs.  Everything that the warps hand to one another (stages, accumulators, scales)
// goes in batches of kBatch K blocks, because each hand-over costs its warp some 300 to 500 cycles, more than a
// block of a small tile takes to load.  B's rows are shared out evenly: with S SMs and k = ceil(N / (128 S)) rounds
// a CTA takes tiles of ceil(N / (k S)) rows, 25 of 3584 and 115 of 152064 on 148 SMs, so that a small weight keeps
// every SM busy and a large one ends everywhere at the same time.  No pairs: one CTA per SM, all its shared memory
// as stages of the weight stream.
// Measured, 152064 x 3584: 84 to 86 us with 1 to 16 rows of A, the copy rate, 88 with 32 and 99 with 64 (131 with the
// kernel above; 128 columns, when tried, took 146 us with 128 rows, 137 above).  64 rows of other weights, here and
// above: 3584 x 3584 13.4 and 15.3 us, 18944 x 3584 17.3 and 20.0, 8192 x 8192 23.4 and 31.7.  3584 x 3584, one row:
// 7.7 us, 12 with batches of one.
constexpr int kFwRows = 128;
constexpr int kFwEpiWarps = 4;
constexpr int kFwThreads = 32 * (4 + kFwEpiWarps);

template <int NT>
struct FewCfg {
  static constexpr int kBatch = NT <= 16 ? 4 : 2;  // K blocks handed over together
  static constexpr int kBlockBytes = (kFwRows + NT) * kSmKB;
  static constexpr int kStages = NT <= 16 ? 2 : (NT <= 32 ? 5 : 4);
  static constexpr int kBufs = 4;               // batches of accumulators
  static constexpr int kTmemCols = kBufs * kBatch * NT;  // 256 or 512
  static constexpr int kSlots = 8;              // batches whose scales have room
  static constexpr int kAhead = 5;
  static constexpr int kSlotFloats = kBatch * (kFwRows + NT);
  static constexpr size_t kSmemBytes = size_t(kStages) * kBatch * kBlockBytes + kSlots * kSlotFloats * 4 + 1024 + 512;
  static_assert(kSmemBytes <= 227 * 1024, "shared memory of a CTA");
};

struct FewParams {
  const float* sw;  // scales of B's rows, then of A's
  const float* st;
  int64_t sw_row, sw_col, st_row, st_col;
  int32_t gw, gt;
  int32_t M, N, K;  // A's rows, B's rows
  uint32_t skip_step;
  void* C;
  int64_t ldc;
  int32_t accumulate;
  int32_t e5_w, e5_t;
  int32_t rows, tiles;  // rows of B in a tile (at most 128), tiles
  uint32_t wait_cycles;
  int32_t* err;
};

__device__ __forceinline__ void tma_load_2d_one(uint32_t dst, const void* tmap, uint32_t bar, int x, int y) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tmap)), "r"(bar), "r"(x), "r"(y)
      : "memory");
}
__device__ __forceinline__ void umma_f8_one(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                            uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void umma_commit_one(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
template <int N>
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[N], int at) {
  static_assert(N % 16 == 0, "whole loads");
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[at]), "=r"(r[at + 1]), "=r"(r[at + 2]), "=r"(r[at + 3]), "=r"(r[at + 4]), "=r"(r[at + 5]),
        "=r"(r[at + 6]), "=r"(r[at + 7]), "=r"(r[at + 8]), "=r"(r[at + 9]), "=r"(r[at + 10]), "=r"(r[at + 11]),
        "=r"(r[at + 12]), "=r"(r[at + 13]), "=r"(r[at + 14]), "=r"(r[at + 15])
      : "r"(taddr)
      : "memory");
}

template <int OUT, int NT>
__global__ void __launch_bounds__(kFwThreads, 1)
scaled_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmT, const FewParams p) {
  using Cfg = FewCfg<NT>;
  using O = OutElem<OUT>;
  using OT = typename O::T;
  constexpr int kStages = Cfg::kStages, kBufs = Cfg::kBufs;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (base - raw);
  constexpr int kBatch = Cfg::kBatch;
  constexpr uint32_t kStageBytes = kBatch * Cfg::kBlockBytes;
  constexpr uint32_t kScaleOff = kStages * kStageBytes;
  constexpr uint32_t kBarOff = kScaleOff + Cfg::kSlots * Cfg::kSlotFloats * 4;
  float* scales = reinterpret_cast<float*>(smem + kScaleOff);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + kBarOff);
  const uint32_t bar0 = base + kBarOff;
  auto full_bar = [&](int s) { return bar0 + 8u * s; };
  auto empty_bar = [&](int s) { return bar0 + 8u * (kStages + s); };
  auto tfull_bar = [&](int b) { return bar0 + 8u * (2 * kStages + b); };
  auto tempty_bar = [&](int b) { return bar0 + 8u * (2 * kStages + kBufs + b); };
  auto sempty_bar = [&](int h) { return bar0 + 8u * (2 * kStages + 2 * kBufs + h); };
  constexpr int kBars = 2 * kStages + 2 * kBufs + Cfg::kSlots;
  static_assert(8 * (kBars + 2) <= 512, "barriers");
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(bars + kBars);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + kBars + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(full_bar(s), 1);
      mbar_init(empty_bar(s), 1);
    }
    for (int b = 0; b < kBufs; ++b) {
      mbar_init(tfull_bar(b), 2);  // the tensor cores and warp 2
      mbar_init(tempty_bar(b), kFwEpiWarps);
    }
    for (int h = 0; h < Cfg::kSlots; ++h) mbar_init(sempty_bar(h), kFwEpiWarps);
    *abort_flag = 0;
    mbar_fence_init();
    tma_prefetch_desc(&tmW);
    tma_prefetch_desc(&tmT);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32((const void*)tmem_slot)),
                 "r"((uint32_t)Cfg::kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  const int nk = (p.K + kSmKB - 1) / kSmKB, nb = (nk + kBatch - 1) / kBatch;  // K blocks, batches of them

  if (warp == 0) {
    // ------------------------------------------------------------ operand loads
    if (lane == 0) {
      const uint32_t bytes = uint32_t(p.rows + NT) * kSmKB * kBatch;  // whole boxes, whatever lies outside
      uint32_t it = 0;
      bool ok = true;
      for (int t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
        for (int b = 0; b < nb; ++b, ++it) {
          if (it + 1 == p.skip_step) continue;
          const int s = it % kStages;
          if (!mbar_wait(empty_bar(s), ((it / kStages) & 1u) ^ 1u, abort_flag, p.wait_cycles)) {
            ok = false;
            break;
          }
          mbar_expect_tx(full_bar(s), bytes);
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            // blocks behind the last lie outside the matrix and read as 0; x stays a small multiple of 128
            const uint32_t sa = base + s * kStageBytes + i * Cfg::kBlockBytes;
            const int x = min(b * kBatch + i, nk) * kSmKB;
            tma_load_2d_one(sa, &tmW, full_bar(s), x, t * p.rows);
            tma_load_2d_one(sa + kFwRows * kSmKB, &tmT, full_bar(s), x, 0);
          }
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------ MMAs
    const uint32_t idesc = make_idesc_f8(kFwRows, NT, p.e5_w, p.e5_t);
    const uint64_t da0 = smem_desc_sw128(base, 16, 1024), db0 = smem_desc_sw128(base + kFwRows * kSmKB, 16, 1024);
    uint32_t it = 0;
    bool ok = true;
    for (int t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
      for (int b = 0; b < nb; ++b, ++it) {
        const int s = it % kStages, buf = it % kBufs;
        ok = warp_wait(full_bar(s), (it / kStages) & 1u, abort_flag, p.wait_cycles) &&
             warp_wait(tempty_bar(buf), ((it / kBufs) & 1u) ^ 1u, abort_flag, p.wait_cycles);
        if (!ok) break;
        tc_fence_after();
        if (elect_one()) {
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const uint64_t off = uint32_t((s * kStageBytes + i * Cfg::kBlockBytes) >> 4);
#pragma unroll
            for (int kk = 0; kk < kSmKB / 32; ++kk)
              umma_f8_one(tmem_base + (buf * kBatch + i) * NT, da0 + off + 2 * kk, db0 + off + 2 * kk, idesc, kk ? 1u : 0u);
          }
          umma_commit_one(tfull_bar(buf));
          umma_commit_one(empty_bar(s));
        }
        __syncwarp();
      }
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ scales
    const int64_t dw = p.gw == 1 ? 32 * p.sw_row : 0, dt = p.gt == 1 ? 32 * p.st_row : 0;
    const uint32_t dst0 = smem_u32(scales) + 4 * lane;
    const float *pw = p.sw, *pt = p.st;
    int pj = blockIdx.x, pkb = 0, left_w = 0, left_t = 0;
    // rows of B in a tile need not lie in one block of 128: every row's scale is looked up by itself
    int r0 = 0;
    auto seek = [&]() {
      left_w = left_t = 0;
      if (pj >= p.tiles) return;
      r0 = pj * p.rows + lane;
      left_w = min(p.N - r0, p.rows - lane);
      left_t = p.M - lane;
      pw = p.sw + int64_t(p.gw == 1 ? r0 : 0) * p.sw_row;
      pt = p.st + int64_t(p.gt == 1 ? lane : 0) * p.st_row;
    };
    auto copy = [&](uint32_t n) {  // of the next batch, number n
      uint32_t dst = dst0 + (n % Cfg::kSlots) * (Cfg::kSlotFloats * 4);
#pragma unroll 1
      for (int k = 0; k < kBatch && pkb < nk; ++k, ++pkb, dst += (kFwRows + NT) * 4) {
#pragma unroll
        for (int i = 0; i < kFwRows / 32; ++i)
          if (i * 32 < left_w)
            cp_async4(dst + i * 128, p.gw == 1 ? pw + i * dw : pw + int64_t((r0 + i * 32) >> 7) * p.sw_row);
#pragma unroll
        for (int i = 0; i < (NT + 31) / 32; ++i)
          if (i * 32 < left_t && i * 32 + lane < NT) cp_async4(dst + kFwRows * 4 + i * 128, pt + i * dt);
        pw += p.sw_col;
        pt += p.st_col;
      }
      if (pkb == nk) {
        pkb = 0;
        pj += gridDim.x;
        seek();
      }
    };
    seek();
    bool ok = true;
#pragma unroll 1
    for (uint32_t n = 0; n < Cfg::kAhead; ++n) {
      copy(n);
      asm volatile("cp.async.commit_group;" ::: "memory");
    }
    uint32_t it = 0;
    for (int t = blockIdx.x; ok && t < p.tiles; t += gridDim.x) {
      for (int b = 0; b < nb; ++b, ++it) {
        const uint32_t n = it + Cfg::kAhead;
        ok = warp_wait(sempty_bar(n % Cfg::kSlots), ((n / Cfg::kSlots) & 1u) ^ 1u, abort_flag, p.wait_cycles);
        if (!ok) break;
        copy(n);
        asm volatile("cp.async.commit_group;" ::: "memory");
        asm volatile("cp.async.wait_group %0;" ::"n"(Cfg::kAhead) : "memory");  // this batch's have landed
        __syncwarp();
        // the barrier's phase of one round before has to be over, or this arrival would count for it
        if (it >= kBufs) {
          ok = warp_wait(tfull_bar(it % kBufs), ((it / kBufs) & 1u) ^ 1u, abort_flag, p.wait_cycles);
          if (!ok) break;
        }
        if (lane == 0) mbar_arrive(tfull_bar(it % kBufs));
      }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp >= 4) {
    // ------------------------------------------------------------ epilogue
    constexpr int kCols = kBatch * NT;                // accumulator columns of a batch
    constexpr int kPiece = kCols < 64 ? kCols : 64;   // columns taken from TMEM together
    const int quad = warp & 3, r = quad * 32 + lane;
    const uint32_t tlane = tmem_base + (uint32_t(quad * 32) << 16);
    uint32_t buf = 0, parity = 0, slot = 0;
    bool ok = true;
    int t = blockIdx.x;
    for (; t < p.tiles; t += gridDim.x) {
      float2 acc[NT / 2];
#pragma unroll
      for (int i = 0; i < NT / 2; ++i) acc[i] = make_float2(0.f, 0.f);
#pragma unroll 1
      for (int b = 0; b < nb; ++b) {
        ok = warp_wait(tfull_bar(buf), parity, abort_flag, p.wait_cycles);
        if (!ok) break;
        tc_fence_after();
        const uint32_t ta = tlane + buf * kCols;
        const float* sc = scales + slot * Cfg::kSlotFloats;
#pragma unroll
        for (int c = 0; c < kCols; c += kPiece) {
          uint32_t v[kPiece];
#pragma unroll
          for (int i = 0; i < kPiece; i += 16) tmem_ld16(ta + c + i, v, i);
          tmem_ld_wait();
          if (c + kPiece == kCols) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(tempty_bar(buf));
          }
#pragma unroll
          for (int j = 0; j < kPiece; j += NT < kPiece ? NT : kPiece) {
            const int block = (c + j) / NT, c0 = (c + j) % NT;  // K block of the batch, first column
            if (b * kBatch + block >= nk) continue;             // behind the last: its scales were not copied
            const float* sb = sc + block * (kFwRows + NT);
            const float f = sb[r];
            const float2 f2 = make_float2(f, f);
#pragma unroll
            for (int i = 0; i < (NT < kPiece ? NT : kPiece); i += 4) {
              const float4 g = *reinterpret_cast<const float4*>(sb + kFwRows + c0 + i);
              const int k = (c0 + i) / 2;
              acc[k] = __ffma2_rn(make_float2(__uint_as_float(v[j + i]), __uint_as_float(v[j + i + 1])),
                                  __fmul2_rn(f2, make_float2(g.x, g.y)), acc[k]);
              acc[k + 1] = __ffma2_rn(make_float2(__uint_as_float(v[j + i + 2]), __uint_as_float(v[j + i + 3])),
                                      __fmul2_rn(f2, make_float2(g.z, g.w)), acc[k + 1]);
            }
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(sempty_bar(slot));
        if (++buf == kBufs) {
          buf = 0;
          parity ^= 1u;
        }
        if (++slot == Cfg::kSlots) slot = 0;
      }
      if (!ok) break;
      // this thread's row of B is a column of C: a warp stores 32 of them next to one another
      const int col = t * p.rows + r;
      if (r < p.rows && col < p.N) {
        OT* C = reinterpret_cast<OT*>(p.C) + col;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          if (i < p.M) {
            float x = i & 1 ? acc[i / 2].y : acc[i / 2].x;
            if (p.accumulate) x += O::get(C[i * p.ldc]);
            C[i * p.ldc] = O::put(x);
          }
        }
      }
    }
    // after a wait that ran out: NaN in the warp's part of this tile and of all that were to come
    for (; !ok && t < p.tiles; t += gridDim.x) {
      const int col = t * p.rows + r;
      if (r < p.rows && col < p.N)
        for (int i = 0; i < p.M; ++i) reinterpret_cast<OT*>(p.C)[i * p.ldc + col] = O::put(__int_as_float(0x7FC00000));
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
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"((uint32_t)Cfg::kTmemCols)
                 : "memory");
  }
}

}  // namespace oapl

// Launches of the residual norm's kernels: which variant a call takes and with what shape.
#pragma once
#include "host_common.cuh"
#include "residual_norm.cuh"

namespace oapl {

constexpr int kRsWarpD = 512;          // rows of a warp: 16 elements a lane
constexpr int64_t kRsWarpWorkers = 8192, kRsCtaWorkers = 1024;
constexpr size_t kRsSmem = 200 * 1024; // shared memory of an SM that rows on their way may take

// The launch: threads of a row, rows in flight, CTAs of an SM (per_sm, from the registers; fewer where shared memory asks
// for it) and workers, each with rows of its own.
struct ResidualShape {
  int threads, grid, smem;
  int64_t workers;
};
inline ResidualShape residual_shape(ResidualParams& p, int n_sm, int elems, int es, bool warp, bool level, int arrays, int regs) {
  ResidualShape s;
  const int ke = 16 / es, units = (p.d + ke - 1) / ke;
  const bool direct = es == 4 && elems == 32;
  p.pitch = (int32_t)(direct ? 0 : level ? units * 16 : (p.d * es + 15) / 16 * 16 + 16);
  s.threads = warp ? 256 : (int)round_up((size_t)((units + elems / ke - 1) / (elems / ke)), 32);
  const int groups = warp ? 8 : 1;
  const size_t row = (size_t)arrays * p.pitch * groups, sink = level ? 0 : (size_t)(s.threads / 32) * 66 * 16;
  const size_t factors = residual_factors(elems, level) == kFactorShared ? (size_t)2 * elems * 4 * (warp ? 32 : s.threads) : 0;
  // 65536 registers, handed to warps eight a lane at a time
  int per_sm = 65536 / ((regs + 7) / 8 * 8 * 32) / (s.threads / 32);
  if (per_sm < 1) per_sm = 1;
  if (per_sm > 2048 / s.threads) per_sm = 2048 / s.threads;
  // two rows ahead where there is room, and one at least before CTAs are given up
  p.stages = 3;
  auto room = [&] { return (row * p.stages + sink + factors) * per_sm <= kRsSmem; };
  while (p.stages > 2 && !room()) --p.stages;
  while (per_sm > 1 && !room()) --per_sm;
  while (p.stages > 1 && !room()) --p.stages;
  int64_t grid = (p.N + groups - 1) / groups;
  if (grid > (int64_t)n_sm * per_sm) grid = (int64_t)n_sm * per_sm;
  const int64_t most = (warp ? kRsWarpWorkers : kRsCtaWorkers) / groups;
  if (grid > most) grid = most;
  s.grid = (int)grid;
  s.workers = grid * groups;
  p.sink = (int32_t)(row * p.stages);
  p.factors = (int32_t)(row * p.stages + sink);
  s.smem = (int)(row * p.stages + sink + factors);
  return s;
}

// What a launch has done: its workers, and the rows that they took.
struct ResidualRun {
  int64_t workers, rows;
};

// A kernel's registers, with its shared memory allowed, looked up once for each device.
template <typename F>
int residual_registers(F kern, int (&known)[kMaxDevices], int* regs) {
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return OAPL_ERR_CUDA;
  if (!known[dev]) {
    cudaFuncAttributes fa;
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess ||
        cudaFuncGetAttributes(&fa, kern) != cudaSuccess)
      return OAPL_ERR_CUDA;
    known[dev] = fa.numRegs;
  }
  *regs = known[dev];
  return OAPL_OK;
}

template <typename T, int E, bool WARP, int NT, bool FWD, bool LEVEL, int FORM>
int launch_residual(ResidualParams p, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  static int known[kMaxDevices] = {0};
  constexpr int KE = Elem<T>::kN, K = E / KE;
  void (*kern)(ResidualParams);
  if constexpr (FWD) kern = residual_fwd_kernel<T, KE, K, WARP, NT, LEVEL, FORM>;  // a choice that compiles one of the two
  else kern = residual_bwd_kernel<T, KE, K, WARP, NT, LEVEL, FORM>;
  int regs = 0;
  const int rc = residual_registers(kern, known, &regs);
  if (rc != OAPL_OK) return rc;
  const ResidualShape s = residual_shape(p, n_sm, E, (int)sizeof(T), WARP, LEVEL, arrays, regs);
  const bool sums = p.kind_pre >= 0 || p.kind_post >= 0 || p.kind_gate >= 0;
  if (sums && p.N > s.workers * kRsFold) p.N = s.workers * kRsFold;
  run->workers = s.workers;
  run->rows = p.N;
  kern<<<s.grid, s.threads, s.smem, st>>>(p);
  CKL();
  return OAPL_OK;
}

template <typename T, int E, bool WARP, int NT, bool FWD, bool LEVEL>
int pick_residual(const ResidualParams& p, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  const bool whole = p.y && p.w_pre && p.x_out && (FWD || (p.dx_out && p.dx && p.dy && (p.dgate || p.gate_kind != kGateFull)));
  const int form = !whole ? kFormAny : p.gate_kind == kGateFull ? (p.w_post ? kFormPostFull : kFormFull)
                                                                 : (p.w_post ? kFormPost : kFormPlain);
  // Which forms have kernels of their own, 16384 x 3584 bf16 where nothing else is said.  Forward the first (87 us, 99
  // without; the others 84 without w_post and 112 with a gate per element, at most 15 % above what they have to move).  All
  // in the gradient of rows on 16-byte boundaries (118 us without w_post, 196 for any form); of other rows those with
  // w_post, whose second mean costs most; of rows above 8192 those as far as they are on boundaries (4700 x 12288 with a
  // gate per element: 293 us, 364 for any form).
  if constexpr (FWD || E < 32 || LEVEL) {
    if (form == kFormPost) return launch_residual<T, E, WARP, NT, FWD, LEVEL, kFormPost>(p, arrays, n_sm, run, st);
  }
  if constexpr (!FWD) {
    if constexpr (E < 32 || LEVEL) {
      if (form == kFormPostFull)
        return launch_residual<T, E, WARP, NT, FWD, LEVEL, kFormPostFull>(p, arrays, n_sm, run, st);
    }
    if constexpr (E < 32 && LEVEL) {
      if (form == kFormPlain)
        return launch_residual<T, E, WARP, NT, FWD, LEVEL, kFormPlain>(p, arrays, n_sm, run, st);
      if (form == kFormFull) return launch_residual<T, E, WARP, NT, FWD, LEVEL, kFormFull>(p, arrays, n_sm, run, st);
    }
  }
  return launch_residual<T, E, WARP, NT, FWD, LEVEL, kFormAny>(p, arrays, n_sm, run, st);
}

template <typename T, bool FWD, bool LEVEL>
int route_residual(const ResidualParams& p, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  // elements a thread: as few as give a CTA at most 256 threads, 32 beyond that
  if (p.d <= kRsWarpD / 2) return pick_residual<T, 8, true, 256, FWD, LEVEL>(p, arrays, n_sm, run, st);
  if (p.d <= kRsWarpD) return pick_residual<T, 16, true, 256, FWD, LEVEL>(p, arrays, n_sm, run, st);
  if (p.d <= 2048) return pick_residual<T, 8, false, 256, FWD, LEVEL>(p, arrays, n_sm, run, st);
  if (p.d <= 4096) return pick_residual<T, 16, false, 256, FWD, LEVEL>(p, arrays, n_sm, run, st);
  // (fp32 rows off 16-byte boundaries have no room beside their factors where there are five arrays of them)
  const bool room = LEVEL || (size_t)arrays * p.d * sizeof(T) + (size_t)8 * p.d <= kRsSmem;
  if (p.d <= 8192 && room) return pick_residual<T, 16, false, 512, FWD, LEVEL>(p, arrays, n_sm, run, st);
  // fp32 rows are read where they are
  return pick_residual<T, 32, false, 512, FWD, LEVEL && sizeof(T) == 2>(p, arrays, n_sm, run, st);
}

template <typename T, bool FWD>
int route_residual_level(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st) {
  return level ? route_residual<T, FWD, true>(p, arrays, n_sm, run, st)
               : route_residual<T, FWD, false>(p, arrays, n_sm, run, st);
}

// Compiled apart, a type to a file.
int residual_bwd_bf16(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st);
int residual_bwd_f16(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st);
int residual_bwd_f32(const ResidualParams& p, bool level, int arrays, int n_sm, ResidualRun* run, cudaStream_t st);

}  // namespace oapl

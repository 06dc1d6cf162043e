// Host side of oapl_residual_norm and its gradient: checks, launches.
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "host_common.cuh"
#include "residual_norm.cuh"

namespace oapl {

constexpr int kRsWarpD = 512;          // rows of a warp: 16 elements a lane
constexpr int64_t kRsWarpWorkers = 8192, kRsCtaWorkers = 1024;
constexpr size_t kRsSmem = 200 * 1024; // shared memory of an SM that rows on their way may take

static int64_t residual_workers(int64_t N, int32_t d) {
  const int64_t most = d <= kRsWarpD ? kRsWarpWorkers : kRsCtaWorkers;
  return N < most ? N : most;
}

static int check_residual(const oapl_residual* r, bool forward) {
  if (!r || r->N <= 0 || r->d <= 0) return OAPL_ERR_INVALID_ARG;
  const int es = type_size(r->type);
  if (!es) return OAPL_ERR_INVALID_ARG;
  if (forward && !r->x) return OAPL_ERR_INVALID_ARG;
  if (r->x && r->ld_x < r->d) return OAPL_ERR_INVALID_ARG;
  if (r->y && r->ld_y < r->d) return OAPL_ERR_INVALID_ARG;
  if (!r->y && (r->w_post || r->gate_kind != OAPL_GATE_NONE)) return OAPL_ERR_INVALID_ARG;
  if (!r->y && !r->w_pre) return OAPL_ERR_INVALID_ARG;  // nothing but a scaled copy
  if ((r->w_post || r->w_pre) && !type_size(r->weight_type)) return OAPL_ERR_INVALID_ARG;
  if (r->gate_kind < OAPL_GATE_NONE || r->gate_kind > OAPL_GATE_FULL) return OAPL_ERR_INVALID_ARG;
  if ((r->gate_kind != OAPL_GATE_NONE) != (r->gate != nullptr)) return OAPL_ERR_INVALID_ARG;
  if (r->gate && !type_size(r->gate_type)) return OAPL_ERR_INVALID_ARG;
  if (r->gate_kind == OAPL_GATE_ROW && r->ld_gate < 1) return OAPL_ERR_INVALID_ARG;
  if (r->gate_kind == OAPL_GATE_FULL && (r->ld_gate < r->d || r->gate_type != r->type)) return OAPL_ERR_INVALID_ARG;
  if (!(r->eps >= 0.f) || !std::isfinite(r->eps) || !std::isfinite(r->weight_offset) ||
      !std::isfinite(r->residual_scale) || !std::isfinite(r->branch_scale))
    return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)r->x % es || (uintptr_t)r->y % es) return OAPL_ERR_MISALIGNED;
  if (r->gate && (uintptr_t)r->gate % type_size(r->gate_type)) return OAPL_ERR_MISALIGNED;
  if ((r->w_post || r->w_pre) && ((uintptr_t)r->w_post | (uintptr_t)r->w_pre) % type_size(r->weight_type))
    return OAPL_ERR_MISALIGNED;
  if (r->N > kMaxRows || r->d > kRsMaxD) return OAPL_ERR_UNSUPPORTED_SHAPE;
  return OAPL_OK;
}

static ResidualParams residual_params(const oapl_residual* r) {
  ResidualParams p;
  memset(&p, 0, sizeof(p));
  p.N = r->N;
  p.d = r->d;
  p.x = r->x;
  p.y = r->y;
  p.gate = r->gate;
  p.w_post = r->w_post;
  p.w_pre = r->w_pre;
  p.ld_x = r->ld_x;
  p.ld_y = r->ld_y;
  p.ld_gate = r->ld_gate;
  p.gate_kind = r->gate_kind;
  p.gate_type = r->gate_type;
  p.weight_type = r->weight_type;
  p.weight_offset = r->weight_offset;
  p.eps = r->eps;
  p.a = r->residual_scale;
  p.b = r->branch_scale;
  p.kind_pre = p.kind_post = p.kind_gate = -1;
  return p;
}

// Whether rows start on 16-byte boundaries: of matrices and, where there are any, of the weights.
static bool residual_level(const ResidualParams& p, int es, const Place* m, int count) {
  if (p.d % (16 / es)) return false;
  for (int i = 0; i < count; ++i)
    if (m[i].base && (!on16(m[i].base) || (m[i].rows > 1 && m[i].ld * m[i].es % 16))) return false;
  return on16(p.w_post) && on16(p.w_pre) && (p.gate_kind != OAPL_GATE_COLUMN || on16(p.gate));
}

// The launch: threads of a row, rows in flight, CTAs of an SM (per_sm, from the registers; fewer where shared memory asks
// for it) and workers, each with rows of its own.
struct ResidualShape {
  int threads, grid, smem;
  int64_t workers;
};
static ResidualShape residual_shape(ResidualParams& p, int n_sm, int elems, int es, bool warp, bool level, int arrays, int regs) {
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

// A kernel's registers, with its shared memory allowed, looked up once for each device.
template <typename F>
static int residual_registers(F kern, int (&known)[kMaxDevices], int* regs) {
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

template <typename T, int E, bool WARP, int NT, bool FWD, bool LEVEL, bool COMMON>
static int launch_residual(ResidualParams p, int arrays, int n_sm, int64_t* workers, cudaStream_t st) {
  static int known[kMaxDevices] = {0};
  constexpr int KE = Elem<T>::kN, K = E / KE;
  auto kern = FWD ? residual_fwd_kernel<T, KE, K, WARP, NT, LEVEL, COMMON>
                  : residual_bwd_kernel<T, KE, K, WARP, NT, LEVEL, COMMON>;
  int regs = 0;
  const int rc = residual_registers(kern, known, &regs);
  if (rc != OAPL_OK) return rc;
  const ResidualShape s = residual_shape(p, n_sm, E, (int)sizeof(T), WARP, LEVEL, arrays, regs);
  *workers = s.workers;
  kern<<<s.grid, s.threads, s.smem, st>>>(p);
  CKL();
  return OAPL_OK;
}

template <typename T, int E, bool WARP, int NT, bool FWD>
static int pick_residual(const ResidualParams& p, bool level, int arrays, int n_sm, int64_t* workers, cudaStream_t st) {
  const bool common = p.y && p.w_post && p.w_pre && p.gate_kind != kGateFull && p.x_out &&
                      (FWD || (p.dx_out && p.dx && p.dy));
  if (level)
    return common ? launch_residual<T, E, WARP, NT, FWD, true, true>(p, arrays, n_sm, workers, st)
                  : launch_residual<T, E, WARP, NT, FWD, true, false>(p, arrays, n_sm, workers, st);
  return common ? launch_residual<T, E, WARP, NT, FWD, false, true>(p, arrays, n_sm, workers, st)
                : launch_residual<T, E, WARP, NT, FWD, false, false>(p, arrays, n_sm, workers, st);
}

template <typename T, bool FWD>
static int route_residual(const ResidualParams& p, bool level, int arrays, int n_sm, int64_t* workers, cudaStream_t st) {
  // elements a thread: as few as give a CTA at most 256 threads, 32 beyond that
  if (p.d <= kRsWarpD / 2) return pick_residual<T, 8, true, 256, FWD>(p, level, arrays, n_sm, workers, st);
  if (p.d <= kRsWarpD) return pick_residual<T, 16, true, 256, FWD>(p, level, arrays, n_sm, workers, st);
  if (p.d <= 2048) return pick_residual<T, 8, false, 256, FWD>(p, level, arrays, n_sm, workers, st);
  if (p.d <= 4096) return pick_residual<T, 16, false, 256, FWD>(p, level, arrays, n_sm, workers, st);
  // (fp32 rows off 16-byte boundaries have no room beside their factors where there are five arrays of them)
  const bool room = level || (size_t)arrays * p.d * sizeof(T) + (size_t)8 * p.d <= kRsSmem;
  if (p.d <= 8192 && room) return pick_residual<T, 16, false, 512, FWD>(p, level, arrays, n_sm, workers, st);
  // fp32 rows are read where they are
  return pick_residual<T, 32, false, 512, FWD>(p, level && sizeof(T) == 2, arrays, n_sm, workers, st);
}

template <bool FWD>
static int route_residual_type(const ResidualParams& p, int32_t type, bool level, int arrays, int n_sm, int64_t* workers,
                               cudaStream_t st) {
  if (type == OAPL_TYPE_BF16) return route_residual<__nv_bfloat16, FWD>(p, level, arrays, n_sm, workers, st);
  if (type == OAPL_TYPE_F16) return route_residual<__half, FWD>(p, level, arrays, n_sm, workers, st);
  return route_residual<float, FWD>(p, level, arrays, n_sm, workers, st);
}

}  // namespace oapl

using namespace oapl;

extern "C" {

int oapl_residual_norm(const oapl_residual* r, void* x_out, int64_t ld_x_out, void* h, int64_t ld_h, float* rstd_post,
                       float* rstd_pre, void* stream) {
  const int rc = check_residual(r, true);
  if (rc != OAPL_OK) return rc;
  const int es = type_size(r->type);
  if ((h != nullptr) != (r->w_pre != nullptr) || (!x_out && !h)) return OAPL_ERR_INVALID_ARG;
  if ((x_out && ld_x_out < r->d) || (h && ld_h < r->d)) return OAPL_ERR_INVALID_ARG;
  if ((rstd_post && !r->w_post) || (rstd_pre && !r->w_pre)) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)x_out % es || (uintptr_t)h % es || (((uintptr_t)rstd_post | (uintptr_t)rstd_pre) & 3))
    return OAPL_ERR_MISALIGNED;
  const bool full = r->gate_kind == OAPL_GATE_FULL;
  const Place m[5] = {{x_out, r->N, r->d, ld_x_out, es}, {h, r->N, r->d, ld_h, es}, {r->x, r->N, r->d, r->ld_x, es},
                      {r->y, r->N, r->d, r->ld_y, es}, {full ? r->gate : nullptr, r->N, r->d, r->ld_gate, es}};
  if (overlap(m[0], m[1]) != kApart) return OAPL_ERR_INVALID_ARG;
  for (int o = 0; o < 2; ++o)
    for (int i = 2; i < 5; ++i)
      if (overlap(m[o], m[i]) == kMixed) return OAPL_ERR_INVALID_ARG;
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  ResidualParams p = residual_params(r);
  p.x_out = x_out;
  p.ld_xo = ld_x_out;
  p.h = h;
  p.ld_h = ld_h;
  p.rstd_post = rstd_post;
  p.rstd_pre = rstd_pre;
  int64_t workers = 0;
  const int arrays = 1 + (r->y != nullptr) + full;
  const bool level = residual_level(p, es, m, 5);
  return route_residual_type<true>(p, r->type, level, arrays, n_sm, &workers,
                                   static_cast<cudaStream_t>(stream));
}

size_t oapl_residual_norm_workspace_bytes(int64_t N, int32_t d) {
  if (N <= 0 || d <= 0 || N > kMaxRows || d > kRsMaxD) return 0;
  // a warp's rows come eight at a time
  return 3 * sizeof(float) * (size_t)d * round_up((size_t)residual_workers(N, d), 8);
}

int oapl_residual_norm_bwd(const oapl_residual* r, const void* x_out, int64_t ld_x_out, const float* rstd_post,
                           const float* rstd_pre, const void* dh, int64_t ld_dh, const void* dx_out, int64_t ld_dx_out,
                           void* dx, int64_t ld_dx, void* dy, int64_t ld_dy, void* dgate, int64_t ld_dgate,
                           float* dw_post, float* dw_pre, int accumulate, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_residual(r, false);
  if (rc != OAPL_OK) return rc;
  const int es = type_size(r->type);
  const bool pre = r->w_pre != nullptr, post = r->w_post != nullptr, full = r->gate_kind == OAPL_GATE_FULL;
  const bool row = r->gate_kind == OAPL_GATE_ROW, column = r->gate_kind == OAPL_GATE_COLUMN;
  if (pre && (!x_out || !rstd_pre || !dh)) return OAPL_ERR_INVALID_ARG;
  if ((!pre && (dh || dw_pre || !dx_out)) || (post && !rstd_post) || (!post && dw_post)) return OAPL_ERR_INVALID_ARG;
  if ((dy && !r->y) || (dgate && !r->gate)) return OAPL_ERR_INVALID_ARG;
  if (!dx && !dy && !dgate && !dw_post && !dw_pre) return OAPL_ERR_INVALID_ARG;
  if ((pre && (ld_x_out < r->d || ld_dh < r->d)) || (dx_out && ld_dx_out < r->d) || (dx && ld_dx < r->d) ||
      (dy && ld_dy < r->d) || (dgate && full && ld_dgate < r->d) || (dgate && row && ld_dgate < 1))
    return OAPL_ERR_INVALID_ARG;
  const int gs = full ? es : 4;
  if ((pre && ((uintptr_t)x_out % es || (uintptr_t)dh % es)) || (uintptr_t)dx_out % es || (uintptr_t)dx % es ||
      (uintptr_t)dy % es || (uintptr_t)dgate % gs ||
      (((uintptr_t)dw_post | (uintptr_t)dw_pre | (uintptr_t)rstd_post | (uintptr_t)rstd_pre) & 3))
    return OAPL_ERR_MISALIGNED;
  const Place m[8] = {{dx, r->N, r->d, ld_dx, es}, {dy, r->N, r->d, ld_dy, es},
                      {full ? dgate : nullptr, r->N, r->d, ld_dgate, es},
                      {pre ? x_out : nullptr, r->N, r->d, ld_x_out, es}, {dh, r->N, r->d, ld_dh, es},
                      {dx_out, r->N, r->d, ld_dx_out, es}, {r->y, r->N, r->d, r->ld_y, es},
                      {full ? r->gate : nullptr, r->N, r->d, r->ld_gate, es}};
  for (int o = 0; o < 3; ++o)
    for (int i = o + 1; i < 8; ++i) {
      const Overlap v = overlap(m[o], m[i]);
      if (v == kMixed || (i < 3 && v != kApart)) return OAPL_ERR_INVALID_ARG;
    }
  ResidualParams p = residual_params(r);
  int kinds = 0;
  ResidualJoinParams j;
  memset(&j, 0, sizeof(j));
  if (dw_pre) { j.out[kinds] = dw_pre; p.kind_pre = kinds++; }
  if (dw_post) { j.out[kinds] = dw_post; p.kind_post = kinds++; }
  if (dgate && column) { j.out[kinds] = static_cast<float*>(dgate); p.kind_gate = kinds++; }
  if (kinds) {
    if (!ws) return OAPL_ERR_INVALID_ARG;
    if (!on16(ws)) return OAPL_ERR_MISALIGNED;
    if (ws_bytes < oapl_residual_norm_workspace_bytes(r->N, r->d)) return OAPL_ERR_WORKSPACE_TOO_SMALL;
  }
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  p.x_out = const_cast<void*>(x_out);
  p.ld_xo = ld_x_out;
  p.rstd_post = const_cast<float*>(rstd_post);
  p.rstd_pre = const_cast<float*>(rstd_pre);
  p.dh = dh;
  p.ld_dh = ld_dh;
  p.dx_out = dx_out;
  p.ld_dxo = ld_dx_out;
  p.dx = dx;
  p.ld_dx = ld_dx;
  p.dy = dy;
  p.ld_dy = ld_dy;
  p.dgate = dgate;
  p.ld_dg = ld_dgate;
  p.part = static_cast<float*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const int arrays = 2 * pre + (dx_out != nullptr) + (r->y != nullptr) + full;
  const bool level = residual_level(p, es, m, 8);
  const int run = route_residual_type<false>(p, r->type, level, arrays, n_sm, &j.workers, st);
  if (run != OAPL_OK || !kinds) return run;
  j.part = p.part;
  j.d = r->d;
  j.accumulate = accumulate != 0;
  residual_join_kernel<<<dim3((unsigned)((r->d + 31) / 32), (unsigned)kinds), dim3(32, kRsShares), 0, st>>>(j);
  CKL();
  return OAPL_OK;
}

}  // extern "C"

// Host side of oapl_residual_norm and its gradient: checks, launches.
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "residual_host.cuh"

namespace oapl {

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

static int residual_fwd(const ResidualParams& p, int32_t type, bool level, int arrays, int n_sm, cudaStream_t st) {
  ResidualRun run;
  if (type == OAPL_TYPE_BF16) return route_residual_level<__nv_bfloat16, true>(p, level, arrays, n_sm, &run, st);
  if (type == OAPL_TYPE_F16) return route_residual_level<__half, true>(p, level, arrays, n_sm, &run, st);
  return route_residual_level<float, true>(p, level, arrays, n_sm, &run, st);
}

static int residual_bwd(const ResidualParams& p, int32_t type, bool level, int arrays, int n_sm, ResidualRun* run,
                        cudaStream_t st) {
  if (type == OAPL_TYPE_BF16) return residual_bwd_bf16(p, level, arrays, n_sm, run, st);
  if (type == OAPL_TYPE_F16) return residual_bwd_f16(p, level, arrays, n_sm, run, st);
  return residual_bwd_f32(p, level, arrays, n_sm, run, st);
}

// The gradient's rows from `rows` on.
static void residual_skip(ResidualParams& p, int64_t rows, int es) {
  auto skip = [&](auto& at, int64_t bytes) {
    using P = std::remove_reference_t<decltype(at)>;
    if (at) at = reinterpret_cast<P>(reinterpret_cast<uintptr_t>(at) + (uintptr_t)(rows * bytes));
  };
  skip(p.x_out, p.ld_xo * es);
  skip(p.dh, p.ld_dh * es);
  skip(p.dx_out, p.ld_dxo * es);
  skip(p.y, p.ld_y * es);
  skip(p.dx, p.ld_dx * es);
  skip(p.dy, p.ld_dy * es);
  skip(p.rstd_post, 4);
  skip(p.rstd_pre, 4);
  if (p.gate_kind == kGateFull) {
    skip(p.gate, p.ld_gate * es);
    skip(p.dgate, p.ld_dg * es);
  } else if (p.gate_kind == kGateRow) {
    skip(p.gate, p.ld_gate * type_size(p.gate_type));
    skip(p.dgate, p.ld_dg * 4);
  }
  p.N -= rows;
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
  const int arrays = 1 + (r->y != nullptr) + full;
  const bool level = residual_level(p, es, m, 5);
  return residual_fwd(p, r->type, level, arrays, n_sm, static_cast<cudaStream_t>(stream));
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
  j.part = p.part;
  j.d = r->d;
  j.accumulate = accumulate != 0;
  for (;;) {
    ResidualRun run;
    const int ran = residual_bwd(p, r->type, level, arrays, n_sm, &run, st);
    if (ran != OAPL_OK || !kinds) return ran;
    j.workers = run.workers;
    CK(launch_next(residual_join_kernel, dim3((unsigned)((r->d + 31) / 32), (unsigned)kinds), dim3(32, kRsShares), 0, st, j));
    if (run.rows == p.N) break;
    residual_skip(p, run.rows, es);
    j.accumulate = 1;
  }
  return OAPL_OK;
}

}  // extern "C"

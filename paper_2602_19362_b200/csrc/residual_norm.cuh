// The end of a block and the beginning of the next one: norm of the block's result, gate, residual sum, norm.
//
//     yh = y r_y,  r_y = (mean y^2 + eps)^-1/2,  u = w_post yh      (u = y without w_post)
//     x' = a x + b g u                                              (g: per row, per channel, per element, or 1)
//     h  = w_pre xh,  xh = x' r_x,  r_x = (mean x'^2 + eps)^-1/2
// and, with t the whole gradient of x',
//     t  = dx' + r_x (w_pre dh - xh mean(w_pre dh xh)),     dw_pre = sum_n dh xh
//     dx = a t,   dg = b t u,   e = b g t,                  dw_post = sum_n e yh
//     dy = r_y (w_post e - yh mean(w_post e yh))            (dy = e without w_post)
// h and the statistics are formed from x' before it is rounded to its type; the gradient starts from x' as it was stored.
//
// Bound by HBM: forward two matrices in and two out, gradient four in and two out, each once.  A row's values stay on
// the SM between its sums and its results.  A CTA (a warp for short rows) takes one row after another; 16-byte
// asynchronous copies bring the rows ahead into shared memory, each thread copying and reading its own columns, so that
// no barrier is needed for them.  The gradient's second mean needs t, which needs the first; with A = b g u it is
//     sum A t = sum A (dx' + r_x w_pre dh) - r_x mean(w_pre dh xh) sum A xh,
// so one exchange between the row's threads gives all three sums.
// Sums over rows (dw_pre, dw_post, dg per channel) are kept in registers over a CTA's rows, written as one partial row per
// CTA, and joined in a fixed order by a second launch.  All sums are fp32.
#pragma once
#include "elements.cuh"

namespace oapl {

constexpr int kRsMaxThreads = 512;
constexpr int kRsMaxD = 16384;
enum { kGateNone = 0, kGateRow = 1, kGateColumn = 2, kGateFull = 3 };

struct ResidualParams {
  int64_t N;
  int32_t d;
  const void *x, *y, *gate, *w_post, *w_pre;
  int64_t ld_x, ld_y, ld_gate;
  int32_t gate_kind, gate_type, weight_type;
  float weight_offset, eps, a, b;
  // forward: results.  gradient: x' and the statistics are inputs
  void *x_out, *h;
  int64_t ld_xo, ld_h;
  float *rstd_post, *rstd_pre;
  // gradient
  const void *dh, *dx_out;
  int64_t ld_dh, ld_dxo;
  void *dx, *dy, *dgate;
  int64_t ld_dx, ld_dy, ld_dg;
  float* part;      // [kinds][workers][d]
  int32_t kind_pre, kind_post, kind_gate;  // where a kind's partial rows are, -1 without
  int32_t stages;   // rows that are in flight
};

// KE elements of a weight of any type, as fp32.
template <int KE>
__device__ __forceinline__ void load_weight(const void* w, int type, int c, float offset, float (&f)[KE]) {
  if (type == 0) {
    Raw<__nv_bfloat16, KE> r;
    r.load(static_cast<const __nv_bfloat16*>(w) + c);
    r.widen(f);
  } else if (type == 1) {
    Raw<__half, KE> r;
    r.load(static_cast<const __half*>(w) + c);
    r.widen(f);
  } else {
    Raw<float, KE> r;
    r.load(static_cast<const float*>(w) + c);
    r.widen(f);
  }
#pragma unroll
  for (int i = 0; i < KE; ++i) f[i] += offset;
}
// fp32 vectors have four elements where a weight in 16 bits has eight to a vector: half a vector of it.
template <>
__device__ __forceinline__ void load_weight<4>(const void* w, int type, int c, float offset, float (&f)[4]) {
  if (type == 2) {
    const float4 v = *reinterpret_cast<const float4*>(static_cast<const float*>(w) + c);
    f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(w) + c);
    float g[8];
    if (type == 0) Elem<__nv_bfloat16>::widen(make_uint4(v.x, v.y, 0u, 0u), g);
    else Elem<__half>::widen(make_uint4(v.x, v.y, 0u, 0u), g);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = g[i];
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] += offset;
}

__device__ __forceinline__ float load_one(const void* p, int type, int64_t i) {
  return type == 0 ? Elem<__nv_bfloat16>::one(p, i) : (type == 1 ? Elem<__half>::one(p, i) : Elem<float>::one(p, i));
}

__device__ __forceinline__ void copy_async_16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Until the copies of all but the last `ahead` rows are there.
__device__ __forceinline__ void copy_async_wait(int ahead) {
  if (ahead == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
  else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// The threads of a row: a warp, or the whole CTA.
template <bool WARP>
struct RowGroup {
  int t, nt;
  int64_t first, step;
  float* red;   // [2][kMaxSums][32]
  int turn;
  static constexpr int kMaxSums = 3;
  __device__ __forceinline__ RowGroup(float* red_) : red(red_), turn(0) {
    if (WARP) {
      const int warps = (int)blockDim.x >> 5;
      t = threadIdx.x & 31;
      nt = 32;
      first = (int64_t)blockIdx.x * warps + (threadIdx.x >> 5);
      step = (int64_t)gridDim.x * warps;
    } else {
      t = threadIdx.x;
      nt = blockDim.x;
      first = blockIdx.x;
      step = gridDim.x;
    }
  }
  template <int M>
  __device__ __forceinline__ void sum(float (&v)[M]) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
      for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], o);
    if (WARP) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = (int)blockDim.x >> 5;
    float* to = red + turn * kMaxSums * 32;  // the sums after next are two barriers away
    turn ^= 1;
    if (lane == 0)
#pragma unroll
      for (int m = 0; m < M; ++m) to[m * 32 + warp] = v[m];
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) {
      float s = lane < warps ? to[m * 32 + lane] : 0.f;
#pragma unroll
      for (int o = 8; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);  // at most 16 warps
      v[m] = __shfl_sync(0xffffffffu, s, 0);
    }
  }
};

// Rows on their way: with KE > 1 through shared memory, `arrays` rows to a stage; with KE == 1 read where they are.
template <typename T, int KE, int K>
struct RowFeed {
  static constexpr bool kStaged = KE > 1;
  const T* base[5];
  int64_t ld[5];
  uint32_t addr;            // shared memory of this row group
  const unsigned char* mem;
  int arrays, units, stages;
  __device__ __forceinline__ int unit(int t, int nt, int k) const { return t + k * nt; }
  __device__ __forceinline__ void fetch(int64_t row, int64_t N, int stage, int t, int nt) {
    if (!kStaged) return;
    if (row < N) {
#pragma unroll
      for (int a = 0; a < 5; ++a)
        if (a < arrays) {
          const T* src = base[a] + row * ld[a];
          const uint32_t dst = addr + (uint32_t)((stage * arrays + a) * units) * 16u;
#pragma unroll
          for (int k = 0; k < K; ++k) {
            const int u = unit(t, nt, k);
            if (u < units) copy_async_16(dst + (uint32_t)u * 16u, src + (int64_t)u * KE);
          }
        }
    }
    copy_async_commit();
  }
  __device__ __forceinline__ void read(int a, int64_t row, int stage, int u, float (&f)[KE]) const {
    if constexpr (kStaged) {
      Elem<T>::widen(*reinterpret_cast<const uint4*>(mem + ((size_t)(stage * arrays + a) * units + u) * 16), f);
    } else {
      f[0] = Elem<T>::one(base[a] + row * ld[a], u);
    }
  }
};

template <typename T, int KE, int K, bool WARP>
__device__ __forceinline__ RowFeed<T, KE, K> row_feed(const ResidualParams& p, unsigned char* ring, int arrays) {
  RowFeed<T, KE, K> f;
  f.arrays = arrays;
  f.units = p.d / KE;
  f.stages = p.stages;
  f.mem = ring + (WARP ? (size_t)(threadIdx.x >> 5) * p.stages * arrays * f.units * 16 : 0);
  f.addr = smem_u32(f.mem);
  return f;
}

// ------------------------------------------------------------------------------------------------ forward
template <typename T, int KE, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : kRsMaxThreads) residual_fwd_kernel(ResidualParams p) {
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ float red[2 * RowGroup<WARP>::kMaxSums * 32];
  RowGroup<WARP> grp(red);
  const bool has_y = p.y != nullptr, post = p.w_post != nullptr, pre = p.w_pre != nullptr;
  const int arrays = 1 + has_y + (p.gate_kind == kGateFull);
  RowFeed<T, KE, K> feed = row_feed<T, KE, K, WARP>(p, ring, arrays);
  feed.base[0] = static_cast<const T*>(p.x);
  feed.ld[0] = p.ld_x;
  feed.base[1] = static_cast<const T*>(p.y);
  feed.ld[1] = p.ld_y;
  feed.base[2] = static_cast<const T*>(p.gate);
  feed.ld[2] = p.ld_gate;
  const int t = grp.t, nt = grp.nt;
  for (int s = 0; s + 1 < p.stages; ++s) feed.fetch(grp.first + s * grp.step, p.N, s, t, nt);
  const float inv_d = 1.f / (float)p.d;
  int stage = 0, ahead = p.stages - 1;
  for (int64_t row = grp.first; row < p.N; row += grp.step) {
    // the slot that this fetch fills was read in the round before
    feed.fetch(row + (int64_t)ahead * grp.step, p.N, stage == 0 ? p.stages - 1 : stage - 1, t, nt);
    float g_row = p.b;
    if (p.gate_kind == kGateRow) g_row *= load_one(p.gate, p.gate_type, row * p.ld_gate);
    if (feed.kStaged) copy_async_wait(ahead);
    if (post) {
      float ss[1] = {0.f};
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int u = feed.unit(t, nt, k);
        if (u < feed.units) {
          float f[KE];
          feed.read(1, row, stage, u, f);
#pragma unroll
          for (int i = 0; i < KE; ++i) ss[0] = fmaf(f[i], f[i], ss[0]);
        }
      }
      grp.sum(ss);
      const float r = 1.f / sqrtf(fmaf(ss[0], inv_d, p.eps));
      if (t == 0 && p.rstd_post) p.rstd_post[row] = r;
      g_row *= r;
    }
    float v[K][KE], ss[1] = {0.f};
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = feed.unit(t, nt, k);
      if (u < feed.units) {
        const int c = u * KE;
        feed.read(0, row, stage, u, v[k]);
#pragma unroll
        for (int i = 0; i < KE; ++i) v[k][i] *= p.a;
        if (has_y) {
          float f[KE], w[KE];
          feed.read(1, row, stage, u, f);
#pragma unroll
          for (int i = 0; i < KE; ++i) f[i] *= g_row;
          if (post) {
            load_weight<KE>(p.w_post, p.weight_type, c, p.weight_offset, w);
#pragma unroll
            for (int i = 0; i < KE; ++i) f[i] *= w[i];
          }
          if (p.gate_kind >= kGateColumn) {
            if (p.gate_kind == kGateColumn) load_weight<KE>(p.gate, p.gate_type, c, 0.f, w);
            else feed.read(2, row, stage, u, w);
#pragma unroll
            for (int i = 0; i < KE; ++i) f[i] *= w[i];
          }
#pragma unroll
          for (int i = 0; i < KE; ++i) v[k][i] += f[i];
        }
#pragma unroll
        for (int i = 0; i < KE; ++i) ss[0] = fmaf(v[k][i], v[k][i], ss[0]);
        if (p.x_out) Raw<T, KE>::store(static_cast<T*>(p.x_out) + row * p.ld_xo + c, v[k]);
      }
    }
    if (pre) {
      grp.sum(ss);
      const float r = 1.f / sqrtf(fmaf(ss[0], inv_d, p.eps));
      if (t == 0 && p.rstd_pre) p.rstd_pre[row] = r;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int u = feed.unit(t, nt, k);
        if (u < feed.units) {
          float w[KE];
          load_weight<KE>(p.w_pre, p.weight_type, u * KE, p.weight_offset, w);
#pragma unroll
          for (int i = 0; i < KE; ++i) w[i] *= v[k][i] * r;
          Raw<T, KE>::store(static_cast<T*>(p.h) + row * p.ld_h + u * KE, w);
        }
      }
    }
    stage = stage + 1 == p.stages ? 0 : stage + 1;
  }
}

// ------------------------------------------------------------------------------------------------ gradient
template <typename T, int KE, int K, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : kRsMaxThreads) residual_bwd_kernel(ResidualParams p) {
  extern __shared__ __align__(16) unsigned char ring[];
  __shared__ float red[2 * RowGroup<WARP>::kMaxSums * 32];
  RowGroup<WARP> grp(red);
  const bool has_y = p.y != nullptr, post = p.w_post != nullptr, pre = p.w_pre != nullptr, has_dx = p.dx_out != nullptr;
  // the arrays of a stage, in this order, those that there are
  const int at_xo = 0, at_dh = 1, at_dx = pre ? 2 : 0, at_y = at_dx + has_dx, at_g = at_y + has_y;
  const int arrays = at_g + (p.gate_kind == kGateFull);
  RowFeed<T, KE, K> feed = row_feed<T, KE, K, WARP>(p, ring, arrays);
  auto put = [&](int at, const void* base, int64_t ld) {
#pragma unroll
    for (int a = 0; a < 5; ++a)
      if (a == at) {
        feed.base[a] = static_cast<const T*>(base);
        feed.ld[a] = ld;
      }
  };
  if (pre) {
    put(at_xo, p.x_out, p.ld_xo);
    put(at_dh, p.dh, p.ld_dh);
  }
  if (has_dx) put(at_dx, p.dx_out, p.ld_dxo);
  if (has_y) put(at_y, p.y, p.ld_y);
  if (p.gate_kind == kGateFull) put(at_g, p.gate, p.ld_gate);
  const int t = grp.t, nt = grp.nt;
  for (int s = 0; s + 1 < p.stages; ++s) feed.fetch(grp.first + s * grp.step, p.N, s, t, nt);
  const float inv_d = 1.f / (float)p.d;
  float a_pre[K][KE], a_post[K][KE], a_gate[K][KE];
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < KE; ++i) a_pre[k][i] = a_post[k][i] = a_gate[k][i] = 0.f;
  int stage = 0, ahead = p.stages - 1;
  for (int64_t row = grp.first; row < p.N; row += grp.step) {
    feed.fetch(row + (int64_t)ahead * grp.step, p.N, stage == 0 ? p.stages - 1 : stage - 1, t, nt);
    const float r_x = pre ? p.rstd_pre[row] : 0.f, r_y = post ? p.rstd_post[row] : 1.f;
    const float g_row = p.gate_kind == kGateRow ? load_one(p.gate, p.gate_type, row * p.ld_gate) : 1.f;
    if (feed.kStaged) copy_async_wait(ahead);
    // b w_post g r_y of a column: what y is multiplied with to give A (a row's gate comes later)
    auto branch = [&](int u, float (&e)[KE]) {
#pragma unroll
      for (int i = 0; i < KE; ++i) e[i] = p.b;
      float w[KE];
      if (post) {
        load_weight<KE>(p.w_post, p.weight_type, u * KE, p.weight_offset, w);
#pragma unroll
        for (int i = 0; i < KE; ++i) e[i] *= w[i];
      }
      if (p.gate_kind >= kGateColumn) {
        if (p.gate_kind == kGateColumn) load_weight<KE>(p.gate, p.gate_type, u * KE, 0.f, w);
        else feed.read(at_g, row, stage, u, w);
#pragma unroll
        for (int i = 0; i < KE; ++i) e[i] *= w[i];
      }
    };
    const bool second = has_y && (post || p.gate_kind == kGateRow);
    float s[3] = {0.f, 0.f, 0.f};
    if (pre || second) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int u = feed.unit(t, nt, k);
        if (u < feed.units) {
          float q[KE], xo[KE], tt[KE];
#pragma unroll
          for (int i = 0; i < KE; ++i) q[i] = xo[i] = tt[i] = 0.f;
          if (pre) {
            float w[KE];
            feed.read(at_dh, row, stage, u, q);
            feed.read(at_xo, row, stage, u, xo);
            load_weight<KE>(p.w_pre, p.weight_type, u * KE, p.weight_offset, w);
#pragma unroll
            for (int i = 0; i < KE; ++i) {
              q[i] *= w[i];
              xo[i] *= r_x;
              s[0] = fmaf(q[i], xo[i], s[0]);
            }
          }
          if (second) {
            float e[KE], y[KE];
            if (has_dx) feed.read(at_dx, row, stage, u, tt);
            feed.read(at_y, row, stage, u, y);
            branch(u, e);
#pragma unroll
            for (int i = 0; i < KE; ++i) {
              const float A = e[i] * (y[i] * r_y);
              s[1] = fmaf(A, fmaf(r_x, q[i], tt[i]), s[1]);
              s[2] = fmaf(A, xo[i], s[2]);
            }
          }
        }
      }
      grp.sum(s);
    }
    const float m1 = r_x * s[0] * inv_d;                 // t = dx' + r_x q - m1 xh
    const float dg_row = fmaf(-m1, s[2], s[1]);          // sum of A t without a row's gate
    const float m2 = g_row * dg_row * inv_d;
    if (p.gate_kind == kGateRow && t == 0 && p.dgate) static_cast<float*>(p.dgate)[row * p.ld_dg] = dg_row;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = feed.unit(t, nt, k);
      if (u < feed.units) {
        const int c = u * KE;
        float tt[KE];
#pragma unroll
        for (int i = 0; i < KE; ++i) tt[i] = 0.f;
        if (has_dx) feed.read(at_dx, row, stage, u, tt);
        if (pre) {
          float q[KE], xo[KE], w[KE];
          feed.read(at_dh, row, stage, u, q);
          feed.read(at_xo, row, stage, u, xo);
          load_weight<KE>(p.w_pre, p.weight_type, c, p.weight_offset, w);
#pragma unroll
          for (int i = 0; i < KE; ++i) {
            xo[i] *= r_x;
            a_pre[k][i] = fmaf(q[i], xo[i], a_pre[k][i]);
            tt[i] = fmaf(-m1, xo[i], fmaf(r_x, q[i] * w[i], tt[i]));
          }
        }
        float o_dx[KE];
#pragma unroll
        for (int i = 0; i < KE; ++i) o_dx[i] = p.a * tt[i];
        if (has_y) {
          float y[KE], w[KE], g[KE];
          feed.read(at_y, row, stage, u, y);
#pragma unroll
          for (int i = 0; i < KE; ++i) {
            y[i] *= r_y;
            w[i] = 1.f;
            g[i] = g_row;
            tt[i] *= p.b;
          }
          if (post) load_weight<KE>(p.w_post, p.weight_type, c, p.weight_offset, w);
          if (p.gate_kind >= kGateColumn) {
            if (p.gate_kind == kGateColumn) load_weight<KE>(p.gate, p.gate_type, c, 0.f, g);
            else feed.read(at_g, row, stage, u, g);
            float o[KE];
#pragma unroll
            for (int i = 0; i < KE; ++i) {
              o[i] = tt[i] * y[i] * w[i];
              a_gate[k][i] += o[i];
            }
            if (p.gate_kind == kGateFull && p.dgate)
              Raw<T, KE>::store(static_cast<T*>(p.dgate) + row * p.ld_dg + c, o);
          }
#pragma unroll
          for (int i = 0; i < KE; ++i) {
            tt[i] *= g[i];
            if (post) {
              a_post[k][i] = fmaf(tt[i], y[i], a_post[k][i]);
              tt[i] = r_y * fmaf(-m2, y[i], tt[i] * w[i]);
            }
          }
          if (p.dy) Raw<T, KE>::store(static_cast<T*>(p.dy) + row * p.ld_dy + c, tt);
        }
        if (p.dx) Raw<T, KE>::store(static_cast<T*>(p.dx) + row * p.ld_dx + c, o_dx);
      }
    }
    stage = stage + 1 == p.stages ? 0 : stage + 1;
  }
  // this worker's sums over its rows
  const int64_t workers = grp.step;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int u = feed.unit(t, nt, k);
    if (u < feed.units) {
      const int64_t at = grp.first * p.d + u * KE, kind = workers * p.d;
      if (p.kind_pre >= 0) Raw<float, KE>::store(p.part + p.kind_pre * kind + at, a_pre[k]);
      if (p.kind_post >= 0) Raw<float, KE>::store(p.part + p.kind_post * kind + at, a_post[k]);
      if (p.kind_gate >= 0) Raw<float, KE>::store(p.part + p.kind_gate * kind + at, a_gate[k]);
    }
  }
}

// Sums of a column over the workers: blockDim = (32 columns, 8 shares of the workers), blockIdx.y the kind.
struct ResidualJoinParams {
  const float* part;
  int64_t workers;
  int32_t d, accumulate;
  float* out[3];
};
__global__ void __launch_bounds__(256) residual_join_kernel(ResidualJoinParams p) {
  __shared__ float sh[8][33];
  const int c = (int)blockIdx.x * 32 + (int)threadIdx.x;
  float s = 0.f;
  if (c < p.d) {
    const float* from = p.part + (int64_t)blockIdx.y * p.workers * p.d + c;
#pragma unroll 8
    for (int64_t w = threadIdx.y; w < p.workers; w += 8) s += from[w * p.d];
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  if (threadIdx.y == 0 && c < p.d) {
    float v = 0.f;
    for (int i = 0; i < 8; ++i) v += sh[i][threadIdx.x];
    float* o = p.out[blockIdx.y] + c;
    *o = p.accumulate ? *o + v : v;
  }
}

}  // namespace oapl

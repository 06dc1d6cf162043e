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
// Sums over rows (dw_pre, dw_post, dg per channel) are kept in registers over a worker's rows, written as its partial row, and
// joined in a fixed order by a second launch.  All sums are fp32.  A launch gives a worker at most kRsFold rows, so that no
// running sum has more terms than that; more rows take further launches, whose joins add to what is there.
//
// Measured, us, 16384 x 3584 bf16: forward 88 (0.83 of the copy rate), gradient 131 with its join (0.84); 11000 x 5120: 84 and
// 148; 100000 x 256: 42 and 74; fp32, 8000 x 3584, gradient 134.  Rows of 3583 elements that start on 16-byte boundaries: 113
// and 252; off them: 159 and 317, where every array is shifted by itself, three times the instructions of the arithmetic.
// The gradient's arithmetic is written two wide and takes half of the issue slots; one wide, with weights widened for each row
// and parts left out at run time, it took 83 instructions an element and 270 us.  Calls without dx_out or without y have no form
// of their own (see ResidualHas): 191 without dx_out, of five matrices; the norm alone 61 forward and 134 back without dx_out.
// What is left forward is the chain of two sums over a row, which the other CTAs of an SM cover.
#pragma once
#include "elements.cuh"

namespace oapl {

constexpr int kRsMaxThreads = 512;
constexpr int kRsMaxD = 16384;
// Rows of a worker in a launch, where sums over rows are asked for.  One running sum over 4096 rows of like sign was off by 418
// half steps of fp32, 256 rows at a time by 15.  A further launch costs 14 to 17 us: 131072 x 5120, whose workers are 148,
// 1642 us in four launches, 1690 in seven of 128 rows, 1590 in one; up to 37888 rows of it take one, 75776 of 3584.
constexpr int kRsFold = 256;
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
  int32_t stages, pitch;  // rows of an array in shared memory, bytes from one to the next
  int32_t sink, factors;  // where the warps' buffers for results, and the columns' factors, begin there
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

// Until the copies of all but the last `ahead` rows are there.
__device__ __forceinline__ void copy_async_wait(int ahead) {
  if (ahead == 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
  else if (ahead == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
  else if (ahead == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
  else asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// The threads of a row: a warp, or the whole CTA.
template <bool WARP>
struct RowGroup {
  static constexpr int kSlot = 3 * 16;  // three sums of at most 16 warps
  int t, nt;
  int64_t first, step;
  float* red;  // two slots
  __device__ __forceinline__ explicit RowGroup(float* red_) : red(red_) {
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
      for (int i = t; i < 64 + kSlot; i += nt) red[i] = 0.f;  // the places of warps that there are not
      __syncthreads();
    }
  }
  __device__ __forceinline__ void sync() const {
    if (WARP) __syncwarp();
    else __syncthreads();
  }
  // Sum over the row's threads, the same bits in each of them.
  __device__ __forceinline__ float sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (WARP) return v;
    if ((t & 31) == 0) red[t >> 5] = v;
    __syncthreads();
    const float4* r = reinterpret_cast<const float4*>(red);
    const float4 p = r[0], q = r[1], x = r[2], y = r[3];
    swap();
    return (((p.x + p.y) + (p.z + p.w)) + ((q.x + q.y) + (q.z + q.w))) +
           (((x.x + x.y) + (x.z + x.w)) + ((y.x + y.y) + (y.z + y.w)));
  }
  // Three sums: lanes share them out as they halve, six exchanges for the three.
  __device__ __forceinline__ void sum3(float (&v)[3]) {
    const int lane = threadIdx.x & 31;
    const bool h16 = lane & 16, h8 = lane & 8;
    float x = (h16 ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, h16 ? v[0] : v[1], 16);
    const float z = v[2] + __shfl_xor_sync(0xffffffffu, v[2], 16);
    x = (h8 ? z : x) + __shfl_xor_sync(0xffffffffu, h8 ? x : z, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    // lanes 0 .. 7 hold the first sum, 16 .. 23 the second, 8 .. 15 and 24 .. 31 the third
    if (WARP) {
      v[0] = __shfl_sync(0xffffffffu, x, 0);
      v[1] = __shfl_sync(0xffffffffu, x, 16);
      v[2] = __shfl_sync(0xffffffffu, x, 8);
      return;
    }
    if ((lane & 7) == 0 && lane < 24) red[(lane == 0 ? 0 : lane == 16 ? 16 : 32) + (t >> 5)] = x;
    __syncthreads();
#pragma unroll
    for (int m = 0; m < 3; ++m) v[m] = red[m * 16 + (lane & 15)];
#pragma unroll
    for (int o = 8; o > 0; o >>= 1)
#pragma unroll
      for (int m = 0; m < 3; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], o);
    swap();
  }
  // Sums use the two slots in turn: a slot is written again two barriers after it was.
  __device__ __forceinline__ void swap() { red = reinterpret_cast<float*>(reinterpret_cast<uintptr_t>(red) ^ 256u); }
};
// The slots lie 256 bytes apart in 512 aligned bytes.
constexpr int kRsRedFloats = 64 + RowGroup<false>::kSlot;

// Rows on their way through shared memory, `arrays` of them to a stage, in units of KE elements (16 bytes).
// LEVEL: all rows start on 16-byte boundaries and have whole units.  A thread copies the units that it will read, so a wait
// for its own copies is all that a stage needs.
// Otherwise the aligned 16-byte blocks that hold a row are copied as they are, whoever reads them, and a barrier follows
// the wait.  A unit is then two blocks shifted in registers (fp32: four words), its elements behind the row's end taken
// as 0.
// kDirect: fp32 rows above 8192 elements, five of which shared memory has no room for, are read where they are.
extern __shared__ __align__(16) unsigned char rs_ring[];

template <typename T, int KE, int K, bool LEVEL>
struct RowFeed {
  static constexpr bool kDirect = sizeof(T) == 4 && KE * K == 32;
  const T* next[5];        // the row that is fetched next, at this thread's first unit (LEVEL) or its beginning
  const T* here[5];        // not LEVEL: the row that is read
  int64_t hop[5];          // elements from one of the group's rows to the next
  uint32_t offset, pitch;  // of this row group's part of the ring, of a row
  int arrays, units, d, t, nt;
  int64_t left;            // rows that are still to be fetched
  template <bool WARP>
  __device__ __forceinline__ void init(const ResidualParams& p, int arrays_, const RowGroup<WARP>& g) {
    arrays = arrays_;
    d = p.d;
    units = (p.d + KE - 1) / KE;
    pitch = (uint32_t)p.pitch;
    offset = WARP ? (uint32_t)(threadIdx.x >> 5) * (uint32_t)(p.stages * arrays) * pitch : 0u;
    t = g.t;
    nt = g.nt;
    left = g.first < p.N ? (p.N - 1 - g.first) / g.step + 1 : 0;
  }
  template <bool WARP>
  __device__ __forceinline__ void array(int a, const void* base, int64_t ld, const RowGroup<WARP>& g) {
    here[a] = static_cast<const T*>(base) + g.first * ld;
    next[a] = here[a] + (LEVEL ? t * KE : 0);
    hop[a] = g.step * ld;
  }
  // Starts the copies of the next row into a stage; one group of copies whether there is a row or not.
  __device__ __forceinline__ void fetch(int stage) {
    if constexpr (kDirect) return;
    if (left > 0) {
      --left;
#pragma unroll
      for (int a = 0; a < 5; ++a)
        if (a < arrays) {
          const uint32_t dst = smem_u32(rs_ring) + offset + (uint32_t)(stage * arrays + a) * pitch + (uint32_t)t * 16u;
          if constexpr (LEVEL) {
#pragma unroll
            for (int k = 0; k < K; ++k)
              if (t + k * nt < units) copy_async_16(dst + (uint32_t)(k * nt) * 16u, next[a] + k * nt * KE);
          } else {
            const uintptr_t from = reinterpret_cast<uintptr_t>(next[a]) & ~(uintptr_t)15;
            const int blocks = (int)((reinterpret_cast<uintptr_t>(next[a] + d) - from + 15) >> 4);
            for (int u = t; u < blocks; u += nt)
              copy_async_16(dst + (uint32_t)(u - t) * 16u, reinterpret_cast<const void*>(from + (uintptr_t)u * 16));
          }
          next[a] += hop[a];
        }
    }
    copy_async_commit();
  }
  // Waits for the row of `stage` and starts the copies of the row that is `ahead` of it into the slot that was read in
  // the round before.
  template <bool WARP>
  __device__ __forceinline__ void turn(int stage, int ahead, const RowGroup<WARP>& g) {
    if constexpr (kDirect) {
    } else if constexpr (LEVEL) {
      fetch(stage == 0 ? ahead : stage - 1);
      copy_async_wait(ahead);
    } else if (ahead) {
      copy_async_wait(ahead - 1);
      g.sync();
      fetch(stage == 0 ? ahead : stage - 1);
    } else {
      g.sync();
      fetch(0);
      copy_async_wait(0);
      g.sync();
    }
  }
  // An array's row of a stage: this thread's first unit, and how far the row is off its first block.
  struct Place {
    const uint4* p;
    uint32_t off;
  };
  __device__ __forceinline__ Place place(int a, int stage) const {
    Place r;
    const T* row = nullptr;
#pragma unroll
    for (int i = 0; i < 5; ++i)
      if (i == a) row = here[i];
    r.off = LEVEL ? 0u : (uint32_t)reinterpret_cast<uintptr_t>(row) & 15u;
    if constexpr (kDirect)
      r.p = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row) & ~(uintptr_t)15) + t;
    else
      r.p = reinterpret_cast<const uint4*>(rs_ring + offset + (uint32_t)(stage * arrays + a) * pitch) + t;
    return r;
  }
  __device__ __forceinline__ void advance() {
    if constexpr (!LEVEL) {
#pragma unroll
      for (int a = 0; a < 5; ++a)
        if (a < arrays) here[a] += hop[a];
    }
  }
  __device__ __forceinline__ void read(const Place& q, int k, float (&f)[KE]) const {
    if constexpr (LEVEL) {
      Elem<T>::widen(q.p[k * nt], f);
    } else {
      const int have = d - (t + k * nt) * KE;  // elements from here to the row's end, at least one
      if constexpr (sizeof(T) == 4) {
        // fp32 off its boundary: a word at a time is a third of the instructions of shifting whole blocks
        const float* e = reinterpret_cast<const float*>(reinterpret_cast<const unsigned char*>(q.p + k * nt) + q.off);
#pragma unroll
        for (int i = 0; i < KE; ++i) f[i] = i < have ? e[i] : 0.f;
        return;
      } else {
        const uint4 lo = q.p[k * nt];
        if (q.off == 0) {  // the same for all threads
          Elem<T>::widen(lo, f);
        } else {
          Elem<T>::widen(shift_16(lo, q.p[k * nt + 1], q.off), f);
        }
      }
      if (have < KE) {
#pragma unroll
        for (int i = 0; i < KE; ++i)
          if (i >= have) f[i] = 0.f;
      }
    }
  }
};

// Writes unit k of every thread of a warp to a row.  LEVEL: where it belongs.  Otherwise through the warp's buffer in
// shared memory, from which the row's aligned 16-byte blocks leave whole, and up to 15 bytes before and behind them an
// element a lane.
template <typename T, int KE, bool LEVEL>
struct RowSink {
  uint4* buf;  // of this warp: 32 units, one more that is read but not used, two of these in turn
  int d, t, nt, turn;
  __device__ __forceinline__ RowSink(unsigned char* mem, int d_, int t_, int nt_) : d(d_), t(t_), nt(nt_), turn(0) {
    buf = reinterpret_cast<uint4*>(mem) + (threadIdx.x >> 5) * 66;
  }
  // For all lanes of the warp.  row: the row's first element.
  __device__ __forceinline__ void put(T* row, int k, const float (&o)[KE]) {
    if constexpr (LEVEL) {
      if (t + k * nt < d / KE) Raw<T, KE>::store(row + (t + k * nt) * KE, o);
    } else {
      const int lane = threadIdx.x & 31, first = (t - lane + k * nt) * KE;  // the warp's first element
      int n = d - first;
      if (n <= 0) return;
      n = n < 32 * KE ? n : 32 * KE;
      T* to = row + first;
      // elements before the first boundary, the same for all units of a row
      int head = (int)(-(reinterpret_cast<uintptr_t>(row) / sizeof(T)) & (KE - 1));
      if (head == 0 || sizeof(T) == 4) {  // (fp32: a word at a time, as it is read)
        const int have = n - lane * KE;
        if (have >= KE && head == 0) {
          Raw<T, KE>::store(to + lane * KE, o);
        } else {
#pragma unroll
          for (int i = 0; i < KE; ++i)
            if (i < have) Elem<T>::put(to, lane * KE + i, o[i]);
        }
        return;
      }
      uint4* b = buf + turn * 33;
      turn ^= 1;
      b[lane] = Elem<T>::narrow(o);
      __syncwarp();
      head = head < n ? head : n;
      const int blocks = (n - head) / KE;
      if (lane < blocks)
        reinterpret_cast<uint4*>(to + head)[lane] = shift_16(b[lane], b[lane + 1], (uint32_t)head * (uint32_t)sizeof(T));
      const int e = lane < KE ? lane : head + blocks * KE + lane - KE;
      if (lane < 2 * KE && e < (lane < KE ? head : n)) to[e] = reinterpret_cast<const T*>(b)[e];
    }
  }
};

// Arithmetic on a vector's elements, two wide.
template <int KE>
__device__ __forceinline__ void v_fma(float (&o)[KE], const float (&a)[KE], const float (&b)[KE], const float (&c)[KE]) {
  if constexpr (KE == 1) {
    o[0] = fmaf(a[0], b[0], c[0]);
  } else {
#pragma unroll
    for (int i = 0; i < KE; i += 2) {
      const float2 r = __ffma2_rn(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), make_float2(c[i], c[i + 1]));
      o[i] = r.x;
      o[i + 1] = r.y;
    }
  }
}
template <int KE>
__device__ __forceinline__ void v_fma(float (&o)[KE], const float (&a)[KE], float b, const float (&c)[KE]) {
  if constexpr (KE == 1) {
    o[0] = fmaf(a[0], b, c[0]);
  } else {
#pragma unroll
    for (int i = 0; i < KE; i += 2) {
      const float2 r = __ffma2_rn(make_float2(a[i], a[i + 1]), make_float2(b, b), make_float2(c[i], c[i + 1]));
      o[i] = r.x;
      o[i + 1] = r.y;
    }
  }
}
template <int KE>
__device__ __forceinline__ void v_mul(float (&o)[KE], const float (&a)[KE], const float (&b)[KE]) {
  if constexpr (KE == 1) {
    o[0] = a[0] * b[0];
  } else {
#pragma unroll
    for (int i = 0; i < KE; i += 2) {
      const float2 r = __fmul2_rn(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]));
      o[i] = r.x;
      o[i + 1] = r.y;
    }
  }
}
template <int KE>
__device__ __forceinline__ void v_mul(float (&o)[KE], const float (&a)[KE], float b) {
  if constexpr (KE == 1) {
    o[0] = a[0] * b;
  } else {
#pragma unroll
    for (int i = 0; i < KE; i += 2) {
      const float2 r = __fmul2_rn(make_float2(a[i], a[i + 1]), make_float2(b, b));
      o[i] = r.x;
      o[i + 1] = r.y;
    }
  }
}
template <int KE>
__device__ __forceinline__ void v_dot(float2& s, const float (&a)[KE], const float (&b)[KE]) {
  if constexpr (KE == 1) {
    s.x = fmaf(a[0], b[0], s.x);
  } else {
#pragma unroll
    for (int i = 0; i < KE; i += 2) s = __ffma2_rn(make_float2(a[i], a[i + 1]), make_float2(b[i], b[i + 1]), s);
  }
}
template <int KE>
__device__ __forceinline__ void v_set(float (&o)[KE], float v) {
#pragma unroll
  for (int i = 0; i < KE; ++i) o[i] = v;
}

// Factors of a thread's columns over its rows: kept in registers; or, where shifting needs those, as fp32 in shared memory,
// each thread's own; or, for rows so wide that there is no room either, formed again for each row.
enum { kFactorRegisters = 0, kFactorShared = 1, kFactorFormed = 2 };
__host__ __device__ constexpr int residual_factors(int elems, bool level) {
  return elems == 32 ? kFactorFormed : level ? kFactorRegisters : kFactorShared;
}
template <int KE, int K, int WHERE>
struct ColumnFactor {
  float w[WHERE == kFactorRegisters ? K : 1][KE];
  float4* mem;  // [K * KE / 4][nt]
  int t, nt;
  template <typename F>
  __device__ __forceinline__ void init(unsigned char* at, int t_, int nt_, int units, bool mine, F form) {
    mem = reinterpret_cast<float4*>(at);
    t = t_;
    nt = nt_;
    if constexpr (WHERE == kFactorRegisters) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (t + k * nt < units) form(t + k * nt, w[k]);
    } else if constexpr (WHERE == kFactorShared) {
      if (mine)
        for (int k = 0; k < K; ++k) {
          if (t + k * nt >= units) break;
          form(t + k * nt, w[0]);
#pragma unroll
          for (int i = 0; i < KE / 4; ++i)
            mem[(k * (KE / 4) + i) * nt + t] = make_float4(w[0][4 * i], w[0][4 * i + 1], w[0][4 * i + 2], w[0][4 * i + 3]);
        }
    }
  }
  template <typename F>
  __device__ __forceinline__ const float (&get(int k, int u, F form))[KE] {
    if constexpr (WHERE == kFactorRegisters) {
      return w[k];
    } else if constexpr (WHERE == kFactorShared) {
#pragma unroll
      for (int i = 0; i < KE / 4; ++i) {
        const float4 q = mem[(k * (KE / 4) + i) * nt + t];
        w[0][4 * i] = q.x;
        w[0][4 * i + 1] = q.y;
        w[0][4 * i + 2] = q.z;
        w[0][4 * i + 3] = q.w;
      }
      return w[0];
    } else {
      form(u, w[0]);
      return w[0];
    }
  }
};

// CTAs of an SM that the registers are shared out for.
constexpr int residual_ctas(bool forward, int elems, int nt) {
  return nt > 256 ? 1 : forward ? (elems == 8 ? 4 : 3) : (elems == 8 ? 3 : 2);
}

// What a call has.  The blocks of a model come in four forms, all with y, w_pre, dx' and every result: with or without w_post,
// with a gate per element or without.  (The norm that makes the head's rows has no dx' from elsewhere, the first one no y: these
// take the kernel for any form.)  Kernels that know theirs when they are compiled have no branches for the rest, and
// registers for all they need (16384 x 3584 bf16, gradient: 118 us without w_post and 171 with a gate per element, 196 and
// 245 for any form).
enum { kFormAny = 0, kFormPost = 1, kFormPlain = 2, kFormPostFull = 3, kFormFull = 4 };
template <int FORM>
struct ResidualHas {
  bool y, post, pre, full, dx_out;
  __device__ __forceinline__ explicit ResidualHas(const ResidualParams& p) {
    constexpr bool kAny = FORM == kFormAny;
    y = !kAny || p.y != nullptr;
    post = kAny ? p.w_post != nullptr : FORM == kFormPost || FORM == kFormPostFull;
    pre = !kAny || p.w_pre != nullptr;
    full = kAny ? p.gate_kind == kGateFull : FORM == kFormPostFull || FORM == kFormFull;
    dx_out = !kAny || p.dx_out != nullptr;
  }
};

// KE elements of a weight, 0 behind the row's end; LEVEL: there are whole vectors, on 16-byte boundaries.
template <int KE, bool LEVEL>
__device__ __forceinline__ void row_weight(const void* w, int type, int d, int c, float offset, float (&f)[KE]) {
  if constexpr (LEVEL) {
    load_weight<KE>(w, type, c, offset, f);
  } else {
    auto some = [&](auto one) {
#pragma unroll
      for (int i = 0; i < KE; ++i) f[i] = c + i < d ? one(c + i) + offset : 0.f;
    };
    if (type == 0) some([&](int i) { return Elem<__nv_bfloat16>::one(w, i); });
    else if (type == 1) some([&](int i) { return Elem<__half>::one(w, i); });
    else some([&](int i) { return Elem<float>::one(w, i); });
  }
}

// A column's factors: of h, and of y (b w_post, and a channel's gate).
template <int KE, bool LEVEL>
__device__ __forceinline__ void form_pre(const ResidualParams& p, bool pre, int c, float (&w)[KE]) {
  if (pre) row_weight<KE, LEVEL>(p.w_pre, p.weight_type, p.d, c, p.weight_offset, w);
  else v_set(w, 0.f);
}
template <int KE, bool LEVEL>
__device__ __forceinline__ void form_y(const ResidualParams& p, bool post, int c, float (&w)[KE]) {
  if (post) row_weight<KE, LEVEL>(p.w_post, p.weight_type, p.d, c, p.weight_offset, w);
  else v_set(w, 1.f);
  v_mul(w, w, p.b);
  if (p.gate_kind == kGateColumn) {
    float g[KE];
    row_weight<KE, LEVEL>(p.gate, p.gate_type, p.d, c, 0.f, g);
    v_mul(w, w, g);
  }
}

// ------------------------------------------------------------------------------------------------ forward
template <typename T, int KE, int K, bool WARP, int NT, bool LEVEL, int FORM>
__global__ void __launch_bounds__(NT, residual_ctas(true, KE * K, NT)) residual_fwd_kernel(ResidualParams p) {
  __shared__ __align__(512) float red[kRsRedFloats];
  RowGroup<WARP> grp(red);
  const ResidualHas<FORM> has(p);
  RowFeed<T, KE, K, LEVEL> feed;
  feed.init(p, 1 + has.y + has.full, grp);
  feed.array(0, p.x, p.ld_x, grp);
  feed.array(1, p.y, p.ld_y, grp);
  feed.array(2, p.gate, p.ld_gate, grp);
  feed.array(3, nullptr, 0, grp);
  feed.array(4, nullptr, 0, grp);
  const int t = grp.t, nt = grp.nt, units = feed.units, ahead = p.stages - 1;
  for (int s = 0; s < ahead; ++s) feed.fetch(s);
  constexpr int kWhere = residual_factors(KE * K, LEVEL);
  ColumnFactor<KE, K, kWhere> f_pre, f_y;
  auto make_pre = [&](int u, float (&w)[KE]) { form_pre<KE, LEVEL>(p, has.pre, u * KE, w); };
  auto make_y = [&](int u, float (&w)[KE]) { form_y<KE, LEVEL>(p, has.post, u * KE, w); };
  const bool mine = !WARP || threadIdx.x < 32;  // a warp's rows have the same columns as the next warp's
  unsigned char* factors = rs_ring + p.factors;
  f_pre.init(factors, t, nt, units, mine, make_pre);
  f_y.init(factors + K * KE * 4 * nt, t, nt, units, mine, make_y);
  if (WARP && kWhere == kFactorShared) __syncthreads();
  const float inv_d = 1.f / (float)p.d;
  T* x_out = static_cast<T*>(p.x_out) + grp.first * p.ld_xo;
  T* h = static_cast<T*>(p.h) + grp.first * p.ld_h;
  RowSink<T, KE, LEVEL> sink(rs_ring + p.sink, p.d, t, nt);
  int stage = 0;
  for (int64_t row = grp.first; row < p.N; row += grp.step) {
    float g_row = 1.f;
    if (p.gate_kind == kGateRow) g_row = load_one(p.gate, p.gate_type, row * p.ld_gate);
    feed.turn(stage, ahead, grp);
    const auto at_x = feed.place(0, stage), at_y = feed.place(1, stage), at_g = feed.place(2, stage);
    float v[K][KE];
    float2 ss = make_float2(0.f, 0.f);
    if (has.y) {
#pragma unroll
      for (int k = 0; k < K; ++k)
        if (t + k * nt < units) {
          feed.read(at_y, k, v[k]);
          v_dot(ss, v[k], v[k]);
        }
      if (has.post) {
        const float r = 1.f / sqrtf(fmaf(grp.sum(ss.x + ss.y), inv_d, p.eps));
        if (t == 0 && p.rstd_post) p.rstd_post[row] = r;
        g_row *= r;
      }
    }
    ss = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = t + k * nt;
      if (u < units) {
        float x[KE];
        feed.read(at_x, k, x);
        if (has.y) {
          v_mul(v[k], v[k], g_row);
          v_mul(v[k], v[k], f_y.get(k, u, make_y));
          if (has.full) {
            float g[KE];
            feed.read(at_g, k, g);
            v_mul(v[k], v[k], g);
          }
          v_fma(v[k], x, p.a, v[k]);
        } else {
          v_mul(v[k], x, p.a);
        }
        v_dot(ss, v[k], v[k]);
      }
      if (FORM != kFormAny || p.x_out) sink.put(x_out, k, v[k]);
    }
    if (has.pre) {
      const float r = 1.f / sqrtf(fmaf(grp.sum(ss.x + ss.y), inv_d, p.eps));
      if (t == 0 && p.rstd_pre) p.rstd_pre[row] = r;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const int u = t + k * nt;
        if (u < units) {
          v_mul(v[k], v[k], r);
          v_mul(v[k], v[k], f_pre.get(k, u, make_pre));
        }
        sink.put(h, k, v[k]);
      }
    }
    x_out += grp.step * p.ld_xo;
    h += grp.step * p.ld_h;
    feed.advance();
    stage = stage == ahead ? 0 : stage + 1;
  }
}

// ------------------------------------------------------------------------------------------------ gradient
// Of a column only two sums are needed: dw_pre, and S = sum_n t yh (times a row's or an element's gate).  Without these
// gates dw_post = b g S and dg = b w_post S, both per channel; with them dw_post = b S.
template <typename T, int KE, int K, bool WARP, int NT, bool LEVEL, int FORM>
__global__ void __launch_bounds__(NT, residual_ctas(false, KE * K, NT)) residual_bwd_kernel(ResidualParams p) {
  __shared__ __align__(512) float red[kRsRedFloats];
  after_launch_before();
  RowGroup<WARP> grp(red);
  const ResidualHas<FORM> has(p);
  // the arrays of a stage, in this order, those that there are
  const int i_dx = has.pre ? 2 : 0, i_y = i_dx + has.dx_out, i_g = i_y + has.y;
  RowFeed<T, KE, K, LEVEL> feed;
  feed.init(p, i_g + has.full, grp);
#pragma unroll
  for (int a = 0; a < 5; ++a) {
    const void* from = nullptr;
    int64_t ld = 0;
    if (has.pre && a == 0) { from = p.x_out; ld = p.ld_xo; }
    if (has.pre && a == 1) { from = p.dh; ld = p.ld_dh; }
    if (has.dx_out && a == i_dx) { from = p.dx_out; ld = p.ld_dxo; }
    if (has.y && a == i_y) { from = p.y; ld = p.ld_y; }
    if (has.full && a == i_g) { from = p.gate; ld = p.ld_gate; }
    feed.array(a, from, ld, grp);
  }
  const int t = grp.t, nt = grp.nt, units = feed.units, ahead = p.stages - 1;
  for (int s = 0; s < ahead; ++s) feed.fetch(s);
  constexpr int kWhere = residual_factors(KE * K, LEVEL);
  ColumnFactor<KE, K, kWhere> f_pre, f_y;
  auto make_pre = [&](int u, float (&w)[KE]) { form_pre<KE, LEVEL>(p, has.pre, u * KE, w); };
  auto make_y = [&](int u, float (&w)[KE]) { form_y<KE, LEVEL>(p, has.post, u * KE, w); };
  const bool mine = !WARP || threadIdx.x < 32;  // a warp's rows have the same columns as the next warp's
  unsigned char* factors = rs_ring + p.factors;
  f_pre.init(factors, t, nt, units, mine, make_pre);
  f_y.init(factors + K * KE * 4 * nt, t, nt, units, mine, make_y);
  if (WARP && kWhere == kFactorShared) __syncthreads();
  const float inv_d = 1.f / (float)p.d;
  const bool second = has.y && (has.post || p.gate_kind == kGateRow);
  T* dx = static_cast<T*>(p.dx) + grp.first * p.ld_dx;
  T* dy = static_cast<T*>(p.dy) + grp.first * p.ld_dy;
  RowSink<T, KE, LEVEL> sink(rs_ring + p.sink, p.d, t, nt);
  float a_pre[K][KE], a_y[K][KE];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    v_set(a_pre[k], 0.f);
    v_set(a_y[k], 0.f);
  }
  int stage = 0;
  for (int64_t row = grp.first; row < p.N; row += grp.step) {
    const float r_x = has.pre ? p.rstd_pre[row] : 0.f, r_y = has.post ? p.rstd_post[row] : 1.f;
    const float g_row = p.gate_kind == kGateRow ? load_one(p.gate, p.gate_type, row * p.ld_gate) : 1.f;
    feed.turn(stage, ahead, grp);
    const auto at_xo = feed.place(0, stage), at_dh = feed.place(1, stage), at_dx = feed.place(i_dx, stage),
               at_y = feed.place(i_y, stage), at_g = feed.place(i_g, stage);
    // c = dx' + r_x w_pre dh, and the sums of (w_pre dh) xh, A c and A xh
    float c[K][KE];
    float2 s0 = make_float2(0.f, 0.f), s1 = s0, s2 = s0;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = t + k * nt;
      if (u < units) {
        float xh[KE];
        if (has.dx_out) feed.read(at_dx, k, c[k]);
        else v_set(c[k], 0.f);
        if (has.pre) {
          float dh[KE];
          feed.read(at_dh, k, dh);
          feed.read(at_xo, k, xh);
          v_mul(xh, xh, r_x);
          v_fma(a_pre[k], dh, xh, a_pre[k]);
          v_mul(dh, dh, f_pre.get(k, u, make_pre));
          v_dot(s0, dh, xh);
          v_fma(c[k], dh, r_x, c[k]);
        } else {
          v_set(xh, 0.f);
        }
        if (second) {
          float A[KE];
          feed.read(at_y, k, A);
          v_mul(A, A, f_y.get(k, u, make_y));
          if (has.full) {
            float g[KE];
            feed.read(at_g, k, g);
            v_mul(A, A, g);
          }
          v_dot(s1, A, c[k]);
          v_dot(s2, A, xh);
        }
      }
    }
    float s[3] = {s0.x + s0.y, (s1.x + s1.y) * r_y, (s2.x + s2.y) * r_y};
    if (has.pre || second) grp.sum3(s);
    const float m1 = r_x * s[0] * inv_d;         // t = c - m1 xh
    const float dg_row = fmaf(-m1, s[2], s[1]);  // sum of A t without a row's gate
    const float m2 = g_row * dg_row * inv_d, e_row = g_row * r_y;
    const float m1x = -m1 * r_x, m2y = -m2 * r_y * r_y;  // with x' and y as they were stored
    if (p.gate_kind == kGateRow && t == 0 && p.dgate) static_cast<float*>(p.dgate)[row * p.ld_dg] = dg_row;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = t + k * nt;
      float o_dx[KE], o_dg[KE], o[KE];
      if (u < units) {
        if (has.pre) {
          float xo[KE];
          feed.read(at_xo, k, xo);
          v_fma(c[k], xo, m1x, c[k]);
        }
        v_mul(o_dx, c[k], p.a);
        if (LEVEL && (FORM != kFormAny || p.dx)) sink.put(dx, k, o_dx);
        if (has.y) {
          float y[KE];
          feed.read(at_y, k, y);
          v_mul(o, c[k], f_y.get(k, u, make_y));  // b w_post g t
          if (has.full) {
            float g[KE], e[KE];
            feed.read(at_g, k, g);
            v_mul(c[k], c[k], g);
            v_mul(e, y, r_y);
            v_fma(a_y[k], c[k], e, a_y[k]);
            v_mul(o_dg, e, o);
            v_mul(o, o, g);
          } else {
            v_mul(c[k], c[k], e_row);
            v_fma(a_y[k], c[k], y, a_y[k]);
          }
          v_mul(o, o, e_row);
          if (has.post) v_fma(o, y, m2y, o);
          if (LEVEL && (FORM != kFormAny || p.dy)) sink.put(dy, k, o);
        }
      }
      if (!LEVEL && (FORM != kFormAny || p.dx)) sink.put(dx, k, o_dx);
      if (!LEVEL && (FORM != kFormAny || p.dy)) sink.put(dy, k, o);
      if (has.full && p.dgate) sink.put(static_cast<T*>(p.dgate) + row * p.ld_dg, k, o_dg);
    }
    dx += grp.step * p.ld_dx;
    dy += grp.step * p.ld_dy;
    feed.advance();
    stage = stage == ahead ? 0 : stage + 1;
  }
  // this worker's sums over its rows
  const int64_t kind = grp.step * p.d;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c = (t + k * nt) * KE;
    if (c >= p.d) continue;
    float* to = p.part + grp.first * p.d + c;
    auto put = [&](float* q, const float(&f)[KE]) {
      if constexpr (LEVEL) {
        Raw<float, KE>::store(q, f);
      } else {
#pragma unroll
        for (int i = 0; i < KE; ++i)
          if (c + i < p.d) q[i] = f[i];
      }
    };
    if (p.kind_pre >= 0) put(to + p.kind_pre * kind, a_pre[k]);
    float w[KE];
    if (p.kind_post >= 0) {
      v_set(w, 1.f);
      if (p.gate_kind == kGateColumn) row_weight<KE, LEVEL>(p.gate, p.gate_type, p.d, c, 0.f, w);
      v_mul(w, w, p.b);
      v_mul(w, w, a_y[k]);
      put(to + p.kind_post * kind, w);
    }
    if (p.kind_gate >= 0) {
      v_set(w, 1.f);
      if (has.post) row_weight<KE, LEVEL>(p.w_post, p.weight_type, p.d, c, p.weight_offset, w);
      v_mul(w, w, p.b);
      v_mul(w, w, a_y[k]);
      put(to + p.kind_gate * kind, w);
    }
  }
}

// Sums of a column over the workers: blockDim = (32 columns, kRsShares shares of the workers), blockIdx.y the kind.
struct ResidualJoinParams {
  const float* part;
  int64_t workers;
  int32_t d, accumulate;
  float* out[3];
};
constexpr int kRsShares = 32;
static __global__ void __launch_bounds__(32 * kRsShares) residual_join_kernel(ResidualJoinParams p) {
  __shared__ float sh[kRsShares][33];
  after_launch_before();
  const int c = (int)blockIdx.x * 32 + (int)threadIdx.x;
  float s = 0.f;
  if (c < p.d) {
    const float* from = p.part + (int64_t)blockIdx.y * p.workers * p.d + c;
#pragma unroll 8
    for (int64_t w = threadIdx.y; w < p.workers; w += kRsShares) s += from[w * p.d];
  }
  sh[threadIdx.y][threadIdx.x] = s;
  __syncthreads();
  // a warp to a column, a lane to a share
  const int col = threadIdx.y;
  float v = sh[threadIdx.x][col];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  const int at = (int)blockIdx.x * 32 + col;
  if (threadIdx.x == 0 && at < p.d) {
    float* o = (blockIdx.y == 0 ? p.out[0] : blockIdx.y == 1 ? p.out[1] : p.out[2]) + at;
    *o = p.accumulate ? *o + v : v;
  }
}

}  // namespace oapl

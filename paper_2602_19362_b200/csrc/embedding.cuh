// Embedding lookup, and the gradient of its table.
//
//     out[n] = s table[id_n],       dtable[v] (+)= s sum_{n: id_n = v} dout[n]
//
// Both are bound by HBM: the lookup moves each row once in and once out; the gradient reads dout once and, when it does
// not add to what is there, writes every row of the table's gradient, most of them zeros.
//
// The gradient adds rows in the order of their positions, without atomics on sums, so it is the same in every run:
//   1. the positions are sorted by token (stable): up to kEbCountMax of them by counting, for each, the keys before it;
//      more by a radix sort of one to four passes, each a move of a tile's positions that also counts the next digits;
//   2. the sorted list is cut into chunks.  A CTA adds up a chunk's rows; a run of equal tokens that lies within the
//      chunk goes straight to the table, the two that may reach over the chunk's ends leave partial sums;
//   3. the CTA of the chunk where a run begins that reaches further adds up its partial sums.
// A token that holds a tenth of the batch is thus spread over many CTAs.  Sums are fp32: up to kEbMaxChunk terms in a
// chunk, then the chunks' partial sums.
// Rows without a token are cleared by further CTAs of the launch of step 2, which find out by searching the sorted list.
// Batches of up to kEbFew positions take one launch: a CTA for each position, which ends when the token has occurred before
// and otherwise finds its other positions and adds up their rows.
//
// Measured, us: 64 rows of 3584 bf16 2.7 on the device; 32768 x 3584 58 (the copy rate), 32768 x 3583 96 (two loads and a shift
// per vector); gradient of 40960 x 1536 bf16 into 151936 rows 185 (0.89 of the copy rate), of which the sums and the zeros
// take 158, the sort 17; 65536 x 1536 into 20000 rows 85; 3001 x 1001 fp16 off 16-byte boundaries into 50021 rows 53; 23 x 313
// into 1486 rows, in one launch, 8.2 (13.3 with the sort and the sums apart).  Added to what is there: 40960 x 1536 into 151936
// rows 100, 65536 x 1536 into 20000 rows 129, 524288 x 1536 into 152064 rows 509 (480 with every row written).
// Clearing rows beside the sort, whose CTAs leave most SMs idle, was tried: it slowed the sort by what it saved.
#pragma once
#include <type_traits>

#include "elements.cuh"

namespace oapl {

constexpr int kEbThreads = 256;
constexpr int kEbCountMax = 8192;   // positions sorted by counting: work grows with their square (6.5 us for 3001, one
                                    // launch; the radix sort of two passes is three launches of 4 to 8 us)
constexpr int kEbTile = 2048;       // positions of a CTA of the radix sort
constexpr int kEbMoveThreads = 512;
constexpr int kEbMaxBits = 10;      // digit of a pass
constexpr int kEbMinChunk = 32, kEbMaxChunk = 256;
constexpr int kEbMaxZeroRows = 32;  // rows of the table of a CTA that clears
constexpr int kEbFew = 1024;        // positions of the single launch
constexpr int kErrBadId = -5;       // OAPL_ERR_BAD_TARGET

struct LookupParams {
  const int32_t* ids;
  const uint8_t* mask;
  int64_t N;
  int32_t V, d;
  float scale;
  int32_t* status;
  const void* in;  // table, or dout
  int64_t ld_in;
  void* out;       // looked-up rows, or the table's gradient
  int64_t ld_out;
  // gradient
  uint2* sorted;   // (token, position); tokens of rows that do not count are V
  float* part;     // [chunks][2][d]: sums of a chunk's first run, when it came from before, and of its last one
  int32_t chunk, chunks, slabs, zero_rows;
  int32_t accumulate;
  uint32_t* joins; // chunks whose last run reaches further: how many, then which
};

// The token of position n, V where it does not count.  Both loads are in flight together.
__device__ __forceinline__ uint32_t lookup_key(const LookupParams& p, int64_t n) {
  const uint32_t id = (uint32_t)p.ids[n];
  const uint32_t live = p.mask ? p.mask[n] : 1u;
  return live && id < (uint32_t)p.V ? id : (uint32_t)p.V;
}
__device__ __forceinline__ void lookup_check(const LookupParams& p, int64_t n) {
  if (p.status && !(p.mask && !p.mask[n]) && (uint32_t)p.ids[n] >= (uint32_t)p.V) atomicCAS(p.status, 0, kErrBadId);
}

// Clears a row of the table's gradient, by all `threads` of a CTA.
__device__ __forceinline__ void clear_row(const LookupParams& p, int64_t v, int t, int threads) {
  float* row = static_cast<float*>(p.out) + v * p.ld_out;
  // up to the first 16-byte boundary, vectors, and the rest
  int head = (int)(-(reinterpret_cast<uintptr_t>(row) >> 2) & 3);
  head = head < p.d ? head : p.d;
  const int vecs = (p.d - head) / 4, tail = (p.d - head) % 4;
  float4* body = reinterpret_cast<float4*>(row + head);
  for (int i = t; i < vecs; i += threads) body[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  if (t < head) row[t] = 0.f;
  else if (t < head + tail) row[vecs * 4 + t] = 0.f;
}

// ------------------------------------------------------------------------------------------------ lookup
template <typename TI, typename TO, int KE>
__device__ __forceinline__ void lookup_put(const LookupParams& p, bool live, const Raw<TI, KE>& v, TO* to) {
  float f[KE];
  if (live) {
    if constexpr (std::is_same<TI, TO>::value) {
      if (p.scale == 1.f) {  // the bits as they are, a NaN's too
        v.put(to);
        return;
      }
    }
    v.widen(f);
#pragma unroll
    for (int i = 0; i < KE; ++i) f[i] *= p.scale;
  } else {
#pragma unroll
    for (int i = 0; i < KE; ++i) f[i] = 0.f;
  }
  Raw<TO, KE>::store(to, f);
}

// A thread: KE elements of R rows, all loads in flight; blockDim.x threads along a row, blockDim.y rows beside one
// another, blockIdx.y pieces of a row.  LEVEL: all rows on 16-byte boundaries.  Otherwise vectors begin at the first boundary
// of a row of the result, the table's row is shifted to them, and the threads behind the row's vectors take one of the up
// to 2 KE - 2 elements before and behind them each.
template <typename TI, typename TO, int KE, int R, bool LEVEL>
__global__ void __launch_bounds__(kEbThreads) embedding_kernel(LookupParams p) {
  const int u = (int)blockIdx.y * (int)blockDim.x + (int)threadIdx.x;
  const int64_t n0 = ((int64_t)blockIdx.x * R) * blockDim.y + threadIdx.y;
  uint32_t key[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t n = n0 + (int64_t)r * blockDim.y;
    key[r] = n < p.N ? lookup_key(p, n) : (uint32_t)p.V;
    if (n < p.N && u == 0) lookup_check(p, n);
  }
  const TI* table = static_cast<const TI*>(p.in);
  TO* out = static_cast<TO*>(p.out) + n0 * p.ld_out;
  const int64_t step = (int64_t)blockDim.y * p.ld_out;
  Raw<TI, KE> v[R];
  if constexpr (LEVEL) {
    const int c = u * KE;
    if (c >= p.d) return;
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (key[r] < (uint32_t)p.V) v[r].load(table + (int64_t)key[r] * p.ld_in + c);
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (n0 + (int64_t)r * blockDim.y < p.N) lookup_put<TI, TO, KE>(p, key[r] < (uint32_t)p.V, v[r], out + r * step + c);
  } else {
    constexpr int kMask = KE - 1;  // a boundary of KE elements of the result
    Shifted<TI, KE> b[R];
    Raw<TI, 1> one[R];
    int c[R];
    bool whole[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      int head = (int)(-(reinterpret_cast<uintptr_t>(out + r * step) / sizeof(TO)) & kMask);
      head = head < p.d ? head : p.d;
      const int vecs = (p.d - head) / KE, e = u - vecs;  // e: place among the single elements
      whole[r] = u < vecs;
      c[r] = whole[r] ? head + u * KE : e < head ? e : vecs * KE + e;
      if (c[r] < p.d && key[r] < (uint32_t)p.V) {
        const TI* from = table + (int64_t)key[r] * p.ld_in + c[r];
        if (whole[r]) b[r].load(from);
        else one[r].load(from);
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
      if (n0 + (int64_t)r * blockDim.y < p.N && c[r] < p.d) {
        const bool live = key[r] < (uint32_t)p.V;
        TO* to = out + r * step + c[r];
        if (whole[r]) {
          b[r].raw(v[r]);
          lookup_put<TI, TO, KE>(p, live, v[r], to);
        } else {
          lookup_put<TI, TO, 1>(p, live, one[r], to);
        }
      }
  }
}

// ------------------------------------------------------------------------------------------------ sorting
// A warp ranks kEbCountRows positions: the CTA brings all keys into shared memory, lanes share them out and compare each
// with the warp's positions.  Of equal keys the earlier position comes first.
constexpr int kEbCountRows = 4;
__global__ void __launch_bounds__(kEbThreads) embedding_count_sort_kernel(LookupParams p) {
  __shared__ uint32_t keys[kEbCountMax];
  after_launch_before();
  const int N = (int)p.N, lane = threadIdx.x & 31;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.joins = 0;
#pragma unroll 8
  for (int m = threadIdx.x; m < N; m += kEbThreads) keys[m] = lookup_key(p, m);
  __syncthreads();
  const int n0 = ((int)blockIdx.x * (kEbThreads / 32) + (threadIdx.x >> 5)) * kEbCountRows;
  if (n0 >= N) return;
  uint32_t key[kEbCountRows];
  int rank[kEbCountRows];
#pragma unroll
  for (int r = 0; r < kEbCountRows; ++r) {
    key[r] = n0 + r < N ? keys[n0 + r] : 0u;
    rank[r] = 0;
  }
  if (lane < kEbCountRows && n0 + lane < N) lookup_check(p, n0 + lane);
  // n0 is a multiple of 4 and the positions of a step are 32: before them all, at them, or behind them all
  int m0 = 0;
#pragma unroll 4
  for (; m0 + 32 <= n0; m0 += 32) {
    const uint32_t k = keys[m0 + lane];
#pragma unroll
    for (int r = 0; r < kEbCountRows; ++r) rank[r] += k <= key[r];
  }
  for (; m0 < N && m0 < n0 + kEbCountRows; m0 += 32) {
    const int m = m0 + lane;
    const uint32_t k = m < N ? keys[m] : 0xFFFFFFFFu;
#pragma unroll
    for (int r = 0; r < kEbCountRows; ++r) rank[r] += k < key[r] || (k == key[r] && m < n0 + r);
  }
#pragma unroll 4
  for (; m0 < N; m0 += 32) {
    const uint32_t k = m0 + lane < N ? keys[m0 + lane] : 0xFFFFFFFFu;
#pragma unroll
    for (int r = 0; r < kEbCountRows; ++r) rank[r] += k < key[r];
  }
#pragma unroll
  for (int r = 0; r < kEbCountRows; ++r) {
    const int at = __reduce_add_sync(0xffffffffu, rank[r]);
    if (lane == 0 && n0 + r < N) p.sorted[at] = make_uint2(key[r], (uint32_t)(n0 + r));
  }
}

struct RadixParams {
  const uint2* in;   // nullptr: the first pass, keys from the ids
  uint2* out;
  uint32_t* hist;    // [tiles][bins] of this pass; with `scanned`, prefix sums over the tiles
  uint32_t* next;    // [tiles][bins] of the next pass, nullptr: the last one
  uint32_t* total;   // [bins], with `scanned`
  uint32_t* clear;   // the first pass: words that the others count in
  int64_t clear_words;
  int32_t shift, bits, tiles, scanned;
};

__device__ __forceinline__ uint2 radix_load(const LookupParams& p, const RadixParams& r, int64_t n) {
  return r.in ? r.in[n] : make_uint2(lookup_key(p, n), (uint32_t)n);
}

// The digits of the first pass, counted by tile.
__global__ void __launch_bounds__(kEbThreads) embedding_radix_count_kernel(LookupParams p, RadixParams r) {
  __shared__ uint32_t h[1 << kEbMaxBits];
  after_launch_before();
  const int bins = 1 << r.bits;
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.joins = 0;
  const int64_t n0 = (int64_t)blockIdx.x * kEbTile + threadIdx.x;
  uint32_t key[kEbTile / kEbThreads];
#pragma unroll
  for (int i = 0; i < kEbTile / kEbThreads; ++i) {
    const int64_t n = n0 + i * kEbThreads;
    key[i] = n < p.N ? lookup_key(p, n) : 0u;
  }
  for (int i = threadIdx.x; i < bins; i += kEbThreads) h[i] = 0;
  for (int64_t i = (int64_t)blockIdx.x * kEbThreads + threadIdx.x; i < r.clear_words; i += (int64_t)gridDim.x * kEbThreads)
    r.clear[i] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEbTile / kEbThreads; ++i)
    if (n0 + i * kEbThreads < p.N) {
      atomicAdd(&h[key[i] & (bins - 1)], 1u);
      if (key[i] == (uint32_t)p.V) lookup_check(p, n0 + i * kEbThreads);
    }
  __syncthreads();
  for (int i = threadIdx.x; i < bins; i += kEbThreads) r.hist[(int64_t)blockIdx.x * bins + i] = h[i];
}

// Many tiles: exclusive prefix sums of 32 digits over the tiles, 32 threads to a digit.
__global__ void __launch_bounds__(1024) embedding_radix_scan_kernel(RadixParams r) {
  __shared__ uint32_t sh[32][33];
  after_launch_before();
  const int bins = 1 << r.bits, bin = (int)blockIdx.x * 32 + (int)threadIdx.x, g = threadIdx.y;
  const int per = (r.tiles + 31) / 32, t0 = g * per, t1 = t0 + per < r.tiles ? t0 + per : r.tiles;
  uint32_t* h = r.hist + bin;
  uint32_t sum = 0;
  if (bin < bins) {
#pragma unroll 8
    for (int t = t0; t < t1; ++t) sum += h[(int64_t)t * bins];
  }
  sh[g][threadIdx.x] = sum;
  __syncthreads();
  uint32_t before = 0, all = 0;
  for (int i = 0; i < 32; ++i) {
    const uint32_t v = sh[i][threadIdx.x];
    before += i < g ? v : 0u;
    all += v;
  }
  if (bin >= bins) return;
  if (g == 0) r.total[bin] = all;
#pragma unroll 8
  for (int t = t0; t < t1; ++t) {
    const uint32_t v = h[(int64_t)t * bins];
    h[(int64_t)t * bins] = before;
    before += v;
  }
}

// Moves a tile's positions to their places.  A warp holds successive positions, 32 at a time in order, so that equal
// digits keep their order: before them come the smaller digits, the tiles before, the warps before and the lanes before.
// Each then counts its next digit for the tile that it has moved to.
__global__ void __launch_bounds__(kEbMoveThreads) embedding_radix_move_kernel(LookupParams p, RadixParams r) {
  constexpr int kWarps = kEbMoveThreads / 32, kRounds = kEbTile / kEbMoveThreads;
  __shared__ uint32_t at[1 << kEbMaxBits], total[1 << kEbMaxBits];  // first place of a digit of this tile, and all of it
  __shared__ uint16_t cnt[kWarps][1 << kEbMaxBits];
  __shared__ uint32_t wsum[kWarps];
  after_launch_before();
  const int bins = 1 << r.bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t n0 = (int64_t)blockIdx.x * kEbTile + warp * 32 * kRounds + lane;
  uint2 e[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) e[i] = n0 + i * 32 < p.N ? radix_load(p, r, n0 + i * 32) : make_uint2(0u, 0u);
  for (int i = threadIdx.x; i < kWarps << (kEbMaxBits - 1); i += kEbMoveThreads) reinterpret_cast<uint32_t*>(&cnt[0][0])[i] = 0;
  // of each digit: all positions, and those of the tiles before
  for (int b = threadIdx.x; b < bins; b += kEbMoveThreads) {
    uint32_t all = 0, ahead = 0;
    if (r.scanned) {
      all = r.total[b];
      ahead = r.hist[(int64_t)blockIdx.x * bins + b];
    } else {
      for (int t0 = 0; t0 < r.tiles; t0 += 16) {
        uint32_t c[16];
#pragma unroll
        for (int t = 0; t < 16; ++t) c[t] = t0 + t < r.tiles ? r.hist[(t0 + t) * bins + b] : 0u;
#pragma unroll
        for (int t = 0; t < 16; ++t) {
          all += c[t];
          ahead += t0 + t < (int)blockIdx.x ? c[t] : 0u;
        }
      }
    }
    total[b] = all;
    at[b] = ahead;
  }
  __syncthreads();
  // the digits' first places: prefix sums, neighbouring digits a thread
  constexpr int kPer = (1 << kEbMaxBits) / kEbMoveThreads;
  uint32_t v[kPer], sum = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = (int)threadIdx.x * kPer + i;
    v[i] = b < bins ? total[b] : 0u;
    sum += v[i];
  }
  uint32_t inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  if (lane == 31) wsum[warp] = inc;
  __syncthreads();
  uint32_t before = inc - sum;
  for (int w = 0; w < warp; ++w) before += wsum[w];
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = (int)threadIdx.x * kPer + i;
    if (b < bins) at[b] += before;
    before += v[i];
  }
  uint16_t rank[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const bool in = n0 + i * 32 < p.N;
    const uint32_t digit = in ? (e[i].x >> r.shift) & (bins - 1) : 0xFFFFFFFFu;
    const uint32_t same = __match_any_sync(0xffffffffu, digit);
    const uint32_t earlier = __popc(same & ((1u << lane) - 1));
    uint16_t had = 0;
    if (in) had = cnt[warp][digit];
    __syncwarp();
    rank[i] = uint16_t(had + earlier);
    if (in && earlier == 0) cnt[warp][digit] = uint16_t(had + __popc(same));
    __syncwarp();
  }
  __syncthreads();
  for (int b = threadIdx.x; b < bins; b += kEbMoveThreads) {
    uint32_t run = 0;
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t c = cnt[w][b];
      cnt[w][b] = uint16_t(run);
      run += c;
    }
  }
  __syncthreads();
  uint32_t place[kRounds];
#pragma unroll
  for (int i = 0; i < kRounds; ++i) place[i] = 0xFFFFFFFFu;
#pragma unroll
  for (int i = 0; i < kRounds; ++i)
    if (n0 + i * 32 < p.N) {
      const uint32_t digit = (e[i].x >> r.shift) & (bins - 1);
      const uint32_t to = at[digit] + cnt[warp][digit] + rank[i];
      r.out[to] = e[i];
      place[i] = (to / kEbTile) << r.bits | ((e[i].x >> (r.shift + r.bits)) & (bins - 1));
    }
  if (!r.next) return;
  // one addition for all lanes that count at the same place: half of a text's tokens share their upper digit
#pragma unroll
  for (int i = 0; i < kRounds; ++i) {
    const uint32_t same = __match_any_sync(0xffffffffu, place[i]);
    if (place[i] != 0xFFFFFFFFu && (same & ((1u << lane) - 1)) == 0) atomicAdd(&r.next[place[i]], (uint32_t)__popc(same));
  }
}

// ------------------------------------------------------------------------------------------------ sums
// Which of the `rows` tokens from v0 on are in the sorted list, a bit each; for a whole warp.  Each half of the warp finds
// one end of their places, 16 probes at a time, and then each lane its token between the two.
__device__ __forceinline__ uint32_t sorted_has(const uint2* s, int64_t n, int64_t v0, int rows) {
  const int lane = threadIdx.x & 31, half = lane >> 4, l = lane & 15;
  const uint32_t key = (uint32_t)(v0 + half * rows);
  int64_t lo = 0, hi = n;  // the first place whose token is at least `key` is in lo .. hi
  while (__any_sync(0xffffffffu, hi > lo)) {
    const int64_t step = (hi - lo + 16) / 17, at = lo + (l + 1) * step - 1;
    // (a half that is done, maybe at the list's start, reads nothing while the other goes on)
    const uint32_t less = __ballot_sync(0xffffffffu, hi > lo && at < hi && s[at].x < key);
    if (hi > lo) {
      const int before = __popc(less >> (half * 16) & 0xFFFFu);
      const int64_t end = lo + (before + 1) * step - 1;  // the first probe that was not less
      lo += before * step;
      hi = before < 16 && end < hi ? end : hi;
    }
  }
  const int64_t from = __shfl_sync(0xffffffffu, lo, 0), to = __shfl_sync(0xffffffffu, lo, 16);
  lo = from, hi = to;
  const uint32_t mine = (uint32_t)(v0 + lane);
  while (lo < hi) {
    const int64_t mid = (lo + hi) >> 1;
    if (s[mid].x < mine) lo = mid + 1; else hi = mid;
  }
  return __ballot_sync(0xffffffffu, lane < rows && lo < to && s[lo].x == mine);
}

template <int KE>
__device__ __forceinline__ void table_put(const LookupParams& p, uint32_t v, int c, const float (&acc)[KE]) {
  float* t = static_cast<float*>(p.out) + (int64_t)v * p.ld_out + c;
  float f[KE];
  if (p.accumulate) {
    Raw<float, KE> old;
    old.load(t);
    old.widen(f);
#pragma unroll
    for (int i = 0; i < KE; ++i) f[i] = fmaf(p.scale, acc[i], f[i]);
  } else {
#pragma unroll
    for (int i = 0; i < KE; ++i) f[i] = p.scale * acc[i];
  }
  Raw<float, KE>::store(t, f);
}

// Grid: chunks x slabs of columns, the slabs of a chunk next to one another, then the CTAs that clear.
template <typename T, int KE>
__global__ void __launch_bounds__(kEbThreads) embedding_sum_kernel(LookupParams p) {
  constexpr int kAhead = KE == 1 ? 16 : 8;  // rows whose loads are in flight together
  __shared__ uint2 e[kEbMaxChunk];
  __shared__ uint32_t live;
  after_launch_before();
  const int slab = (int)(blockIdx.x % (unsigned)p.slabs);
  const int64_t item = blockIdx.x / (unsigned)p.slabs;
  const int c = (slab * (int)blockDim.x + (int)threadIdx.x) * KE;
  if (item >= p.chunks) {
    // clear the rows that no position names
    const int64_t v0 = ((int64_t)blockIdx.x - (int64_t)p.chunks * p.slabs) * p.zero_rows;
    const int rows = p.V - v0 < p.zero_rows ? (int)(p.V - v0) : p.zero_rows;
    if (threadIdx.x < 32) {
      const uint32_t m = sorted_has(p.sorted, p.N, v0, rows);
      if (threadIdx.x == 0) live = m;
    }
    __syncthreads();
    const uint32_t m = live;
    for (int r = 0; r < rows; ++r)
      if (!(m >> r & 1)) clear_row(p, v0 + r, threadIdx.x, blockDim.x);
    return;
  }
  const int64_t first = item * p.chunk;
  const int n = (int)(p.N - first < p.chunk ? p.N - first : p.chunk);
  for (int i = threadIdx.x; i < n; i += blockDim.x) e[i] = p.sorted[first + i];
  const uint32_t none = 0xFFFFFFFFu;
  const uint32_t prev = first ? p.sorted[first - 1].x : none;
  const uint32_t next = first + n < p.N ? p.sorted[first + n].x : none;
  __syncthreads();
  if (c >= p.d) return;
  float acc[KE];
#pragma unroll
  for (int i = 0; i < KE; ++i) acc[i] = 0.f;
  const T* in = static_cast<const T*>(p.in) + c;
  uint32_t key = e[0].x;
  if (key >= (uint32_t)p.V) return;
  bool from_before = key == prev;
  for (int i0 = 0; i0 < n; i0 += kAhead) {
    Raw<T, KE> v[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      if (i0 + j < n && e[i0 + j].x < (uint32_t)p.V) v[j].load_stream(in + (int64_t)e[i0 + j].y * p.ld_in);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (i0 + j >= n) break;
      const uint32_t k = e[i0 + j].x;
      if (k != key) {  // the run before this one has ended; the same for all threads
        if (from_before) {
          Raw<float, KE>::store(p.part + (item * 2) * p.d + c, acc);
        } else {
          table_put<KE>(p, key, c, acc);
        }
#pragma unroll
        for (int i = 0; i < KE; ++i) acc[i] = 0.f;
        key = k;
        from_before = false;
        if (k >= (uint32_t)p.V) return;
      }
      float f[KE];
      v[j].widen(f);
#pragma unroll
      for (int i = 0; i < KE; ++i) acc[i] += f[i];
    }
  }
  if (from_before) {
    Raw<float, KE>::store(p.part + (item * 2) * p.d + c, acc);
  } else if (next == key) {
    Raw<float, KE>::store(p.part + (item * 2 + 1) * p.d + c, acc);
    if (slab == 0 && threadIdx.x == 0) p.joins[1 + atomicAdd(p.joins, 1u)] = (uint32_t)item;
  } else {
    table_put<KE>(p, key, c, acc);
  }
}

// Runs that reach over the end of the chunk where they begin, as the sums listed them: their partial sums.  blockDim.y
// threads of a column share out the chunks and are added up in their order, so the list's order does not matter.
constexpr int kEbJoinCols = 128, kEbJoinShares = 2;
template <int KE>
__global__ void __launch_bounds__(kEbJoinCols * kEbJoinShares) embedding_join_kernel(LookupParams p) {
  constexpr int kAhead = 8;
  __shared__ float sh[kEbJoinShares][kEbJoinCols * KE];
  __shared__ __align__(16) float ring[kAhead][kEbJoinCols * kEbJoinShares * KE];  // each thread's own places
  const int mine = ((int)threadIdx.y * kEbJoinCols + (int)threadIdx.x) * KE;
  after_launch_before();
  const uint32_t slabs = (uint32_t)p.slabs, items = *p.joins * slabs;
  for (uint32_t w = blockIdx.x; w < items; w += gridDim.x) {
    const int64_t item = p.joins[1 + w / slabs];
    const int c = ((int)(w % slabs) * kEbJoinCols + (int)threadIdx.x) * KE;
    const uint32_t key = p.sorted[(item + 1) * p.chunk].x;
    float acc[KE];
#pragma unroll
    for (int i = 0; i < KE; ++i) acc[i] = 0.f;
    if (c < p.d) {
      if (threadIdx.y == 0) {
        Raw<float, KE> t;
        t.load(p.part + (item * 2 + 1) * p.d + c);
        t.widen(acc);
      }
      for (int64_t j0 = item + 1 + threadIdx.y; j0 < p.chunks; j0 += kAhead * kEbJoinShares) {
        // keys and sums together: which of the sums count shows when they are there
        uint32_t in = 0;
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          int64_t at = j0 + j * kEbJoinShares;
          at = at < p.chunks ? at : p.chunks - 1;
          const float* from = p.part + (at * 2) * p.d + c;
          if constexpr (KE == 1) copy_async_4(smem_u32(&ring[j][mine]), from);
          else copy_async_16(smem_u32(&ring[j][mine]), from);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
          const int64_t at = j0 + j * kEbJoinShares;
          in |= (uint32_t)(at < p.chunks && p.sorted[at * p.chunk].x == key) << j;
        }
        copy_async_wait_all();
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
          if (in >> j & 1) {
#pragma unroll
            for (int i = 0; i < KE; ++i) acc[i] += ring[j][mine + i];
          }
        if (!(in >> (kAhead - 1) & 1)) break;
      }
    }
#pragma unroll
    for (int i = 0; i < KE; ++i) sh[threadIdx.y][threadIdx.x + i * kEbJoinCols] = acc[i];
    __syncthreads();
    if (threadIdx.y == 0 && c < p.d) {
#pragma unroll
      for (int y = 1; y < kEbJoinShares; ++y)
#pragma unroll
        for (int i = 0; i < KE; ++i) acc[i] += sh[y][threadIdx.x + i * kEbJoinCols];
      table_put<KE>(p, key, c, acc);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ few positions
// Grid: N positions x slabs of columns, then CTAs that clear.  blockDim = (columns, shares of a token's positions).
template <typename T, int KE>
__global__ void __launch_bounds__(kEbThreads) embedding_few_kernel(LookupParams p) {
  constexpr int kAhead = 8;
  __shared__ uint32_t keys[kEbFew];
  __shared__ uint16_t list[kEbFew];
  __shared__ uint32_t wsum[kEbThreads / 32];
  __shared__ uint32_t live;
  __shared__ float sh[kEbThreads * KE];
  const int N = (int)p.N, cols = blockDim.x, shares = blockDim.y, t = (int)threadIdx.y * cols + (int)threadIdx.x;
  const int lane = t & 31, warp = t >> 5;
#pragma unroll 4
  for (int m = t; m < N; m += kEbThreads) keys[m] = lookup_key(p, m);
  if (t == 0) live = 0;
  __syncthreads();
  const int64_t item = blockIdx.x / (unsigned)p.slabs;
  if (item >= N) {
    const int64_t v0 = ((int64_t)blockIdx.x - (int64_t)N * p.slabs) * p.zero_rows;
    const int rows = p.V - v0 < p.zero_rows ? (int)(p.V - v0) : p.zero_rows;
    for (int m = t; m < N; m += kEbThreads) {
      const int64_t r = (int64_t)keys[m] - v0;
      if (r >= 0 && r < rows) atomicOr(&live, 1u << r);
    }
    __syncthreads();
    const uint32_t m = live;
    for (int r = 0; r < rows; ++r)
      if (!(m >> r & 1)) clear_row(p, v0 + r, t, kEbThreads);
    return;
  }
  const int slab = (int)(blockIdx.x % (unsigned)p.slabs), n = (int)item;
  const uint32_t key = keys[n];
  if (slab == 0 && t == 0) lookup_check(p, n);
  if (key >= (uint32_t)p.V) return;
  bool before = false;
  for (int m = t; m < n; m += kEbThreads) before = before || keys[m] == key;
  if (__syncthreads_or(before)) return;
  // the token's positions, in order: neighbouring ones a thread
  const int per = (N + kEbThreads - 1) / kEbThreads, m0 = t * per, m1 = m0 + per < N ? m0 + per : N;
  uint32_t has = 0;
  for (int m = m0; m < m1; ++m) has += keys[m] == key;
  uint32_t inc = has;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += u;
  }
  if (lane == 31) wsum[warp] = inc;
  __syncthreads();
  uint32_t at = inc - has, all = 0;
  for (int w = 0; w < kEbThreads / 32; ++w) {
    at += w < warp ? wsum[w] : 0u;
    all += wsum[w];
  }
  for (int m = m0; m < m1; ++m)
    if (keys[m] == key) list[at++] = (uint16_t)m;
  __syncthreads();
  // this share of them
  const int count = (int)all, each = (count + shares - 1) / shares, i0 = (int)threadIdx.y * each;
  const int i1 = i0 + each < count ? i0 + each : count;
  const int c = (slab * cols + (int)threadIdx.x) * KE;
  float acc[KE];
#pragma unroll
  for (int i = 0; i < KE; ++i) acc[i] = 0.f;
  if (c < p.d) {
    const T* in = static_cast<const T*>(p.in) + c;
    for (int i = i0; i < i1; i += kAhead) {
      Raw<T, KE> v[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < i1) v[j].load_stream(in + (int64_t)list[i + j] * p.ld_in);
#pragma unroll
      for (int j = 0; j < kAhead; ++j)
        if (i + j < i1) {
          float f[KE];
          v[j].widen(f);
#pragma unroll
          for (int k = 0; k < KE; ++k) acc[k] += f[k];
        }
    }
  }
#pragma unroll
  for (int k = 0; k < KE; ++k) sh[k * kEbThreads + t] = acc[k];
  __syncthreads();
  if (threadIdx.y || c >= p.d) return;
  for (int y = 1; y < shares; ++y)
#pragma unroll
    for (int k = 0; k < KE; ++k) acc[k] += sh[k * kEbThreads + y * cols + t];
  table_put<KE>(p, key, c, acc);
}

}  // namespace oapl

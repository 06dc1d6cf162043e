// Host side of operators around the LM head declared in include/oapl.h: the embedding, the gradient norm and clipping,
// and the adjustments of logits.  Checks, workspaces and launches.
#include <cuda_runtime.h>

#include <cmath>
#include <cstring>

#include "embedding.cuh"
#include "grad_clip.cuh"
#include "host_common.cuh"
#include "logits_adjust.cuh"

namespace oapl {

// ---------------------------------------------------------------------------------------
// Embedding.
static int check_lookup(const oapl_lookup* l) {
  if (!l || !l->ids || l->N <= 0 || l->V <= 0 || !std::isfinite(l->scale)) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)l->ids & 3) return OAPL_ERR_MISALIGNED;
  if (l->N > kMaxRows || (int64_t)l->V > kMaxRows) return OAPL_ERR_UNSUPPORTED_SHAPE;
  return OAPL_OK;
}

static LookupParams lookup_params(const oapl_lookup* l, int32_t d, int32_t* status) {
  LookupParams p;
  memset(&p, 0, sizeof(p));
  p.ids = l->ids;
  p.mask = l->mask;
  p.N = l->N;
  p.V = l->V;
  p.d = d;
  p.scale = l->scale;
  p.status = status;
  return p;
}

template <typename TI, typename TO, int KE, bool LEVEL>
static int launch_embedding(const LookupParams& p, int n_sm, cudaStream_t st) {
  // vectors of a row, and where it may be off 16-byte boundaries the elements before and behind them
  const int64_t units = (int64_t)p.d / KE + (LEVEL ? 0 : 2 * KE - 1);
  int tx = 32;
  while (tx < kEbThreads && tx < units) tx *= 2;
  const dim3 block(tx, kEbThreads / tx);
  const int64_t slabs = (units + tx - 1) / tx, rows = (p.N + block.y - 1) / block.y;
  if (slabs > 65535) return OAPL_ERR_UNSUPPORTED_SHAPE;
  // four rows a thread, for loads in flight, where that still leaves eight CTAs to an SM
  if (rows / 4 * slabs >= 8 * (int64_t)n_sm)
    embedding_kernel<TI, TO, KE, 4, LEVEL><<<dim3((unsigned)((rows + 3) / 4), (unsigned)slabs), block, 0, st>>>(p);
  else
    embedding_kernel<TI, TO, KE, 1, LEVEL><<<dim3((unsigned)rows, (unsigned)slabs), block, 0, st>>>(p);
  CKL();
  return OAPL_OK;
}

template <typename TI, typename TO>
static int route_embedding(const LookupParams& p, int n_sm, cudaStream_t st) {
  constexpr int KE = Elem<TI>::kN < Elem<TO>::kN ? Elem<TI>::kN : Elem<TO>::kN;  // 16 bytes of the wider type
  const bool vec = on16(p.in) && on16(p.out) && p.d % KE == 0 && p.ld_in % KE == 0 && p.ld_out % KE == 0;
  return vec ? launch_embedding<TI, TO, KE, true>(p, n_sm, st) : launch_embedding<TI, TO, KE, false>(p, n_sm, st);
}

template <typename TI>
static int route_embedding_out(const LookupParams& p, int32_t out_type, int n_sm, cudaStream_t st) {
  if (out_type == OAPL_TYPE_BF16) return route_embedding<TI, __nv_bfloat16>(p, n_sm, st);
  if (out_type == OAPL_TYPE_F16) return route_embedding<TI, __half>(p, n_sm, st);
  return route_embedding<TI, float>(p, n_sm, st);
}

// The gradient's workspace: the sorted list, with more positions a second one and the digits' histograms, and two
// partial sums of a row's width for each chunk.
struct LookupCarve {
  int32_t chunk, chunks, bits, passes, tiles;
  size_t sorted, other, hist, totals, joins, part, total;
};
static bool lookup_carve(int64_t N, int32_t V, int32_t d, LookupCarve* c) {
  if (N <= 0 || V <= 0 || d <= 0 || N > kMaxRows || (int64_t)V > kMaxRows || (int64_t)d > kMaxRows) return false;
  // Chunks: short ones give a CTA to each few rows, long ones few partial sums to join where one token is frequent
  // (a token's join takes 0.16 us per chunk).  640 of them are four per SM.
  int64_t chunk = kEbMinChunk;
  while (chunk < kEbMaxChunk && chunk * 640 < N) chunk *= 2;
  const int64_t chunks = (N + chunk - 1) / chunk;
  c->chunk = (int32_t)chunk;
  c->chunks = (int32_t)chunks;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t o = off;
    off = round_up(off + bytes, 256);
    return o;
  };
  c->sorted = take(8 * (size_t)N);
  c->other = c->hist = c->totals = 0;
  c->bits = c->passes = c->tiles = 0;
  if (N > kEbCountMax) {
    int bits = 1;
    while (((int64_t)V >> bits) != 0) ++bits;  // the keys are 0 .. V
    c->passes = (bits + kEbMaxBits - 1) / kEbMaxBits;
    c->bits = (bits + c->passes - 1) / c->passes;
    c->tiles = (int32_t)((N + kEbTile - 1) / kEbTile);
    c->other = take(8 * (size_t)N);
    c->hist = take(4 * (size_t)c->passes * ((size_t)c->tiles << c->bits));
    c->totals = take(4 * ((size_t)1 << c->bits));
  }
  c->joins = take(4 * ((size_t)chunks + 1));
  c->part = take(8 * (size_t)chunks * (size_t)d);
  c->total = off;
  return true;
}

// Rows of the table that a CTA clears: about 16 KB, so that a CTA's search for them goes under the writes of others, and
// between 8 and 32 of them.
static int zero_rows(int32_t d) {
  const int rows = 4096 / d;
  return rows < 8 ? 8 : rows > kEbMaxZeroRows ? kEbMaxZeroRows : rows;
}

template <typename T, int KE>
static int launch_embedding_few(LookupParams p, cudaStream_t st) {
  const int64_t units = p.d / KE;
  int cols = 32;
  while (cols < 128 && cols < units) cols *= 2;
  const int64_t slabs = (units + cols - 1) / cols;
  p.zero_rows = zero_rows(p.d);
  const int64_t zero = p.accumulate ? 0 : ((int64_t)p.V + p.zero_rows - 1) / p.zero_rows;
  if (p.N * slabs + zero > kMaxGrid) return OAPL_ERR_UNSUPPORTED_SHAPE;
  p.slabs = (int32_t)slabs;
  embedding_few_kernel<T, KE><<<(unsigned)(p.N * slabs + zero), dim3(cols, kEbThreads / cols), 0, st>>>(p);
  CKL();
  return OAPL_OK;
}

template <typename T, int KE>
static int launch_embedding_sum(LookupParams p, int n_sm, cudaStream_t st) {
  const int64_t units = p.d / KE;
  const int64_t slabs = (units + kEbThreads - 1) / kEbThreads;
  const int threads = (int)round_up((size_t)((units + slabs - 1) / slabs), 32);
  p.zero_rows = zero_rows(p.d);
  const int64_t zero = p.accumulate ? 0 : ((int64_t)p.V + p.zero_rows - 1) / p.zero_rows;
  if (p.chunks * slabs + zero > kMaxGrid) return OAPL_ERR_UNSUPPORTED_SHAPE;
  p.slabs = (int32_t)slabs;
  CK(launch_next(embedding_sum_kernel<T, KE>, dim3((unsigned)(p.chunks * slabs + zero)), dim3(threads), 0, st, p));
  if (p.chunks > 1) {
    constexpr int JE = KE > 4 ? 4 : KE;
    p.slabs = (int32_t)((p.d / JE + kEbJoinCols - 1) / kEbJoinCols);
    const int64_t most = (int64_t)p.chunks * p.slabs;
    if (most > kMaxGrid) return OAPL_ERR_UNSUPPORTED_SHAPE;
    const int64_t grid = 8 * (int64_t)n_sm;  // how many there are, the device knows
    CK(launch_next(embedding_join_kernel<JE>, dim3((unsigned)(most < grid ? most : grid)),
                   dim3(kEbJoinCols, kEbJoinShares), 0, st, p));
  }
  return OAPL_OK;
}

template <typename T>
static int route_embedding_sum(const LookupParams& p, int n_sm, cudaStream_t st) {
  // (vectors of 16-bit rows have twice the width of the table's; half of them a thread took 199 us instead of 189, 40960 x
  // 1536 into 151936 rows)
  constexpr int KE = Elem<T>::kN;
  const bool vec = on16(p.in) && on16(p.out) && p.d % KE == 0 && p.ld_in % KE == 0 && p.ld_out % 4 == 0;
  if (p.N <= kEbFew) return vec ? launch_embedding_few<T, KE>(p, st) : launch_embedding_few<T, 1>(p, st);
  return vec ? launch_embedding_sum<T, KE>(p, n_sm, st) : launch_embedding_sum<T, 1>(p, n_sm, st);
}

// ---------------------------------------------------------------------------------------
// Gradient norm and clipping.
// log2 of an element's size, -1 for no type.  A list has hundreds of tensors: no divisions here.
static int type_shift(int32_t type) {
  return type == OAPL_TYPE_BF16 || type == OAPL_TYPE_F16 ? 1 : (type == OAPL_TYPE_F32 ? 2 : -1);
}
static int check_tensors(const oapl_tensor* t, int32_t count, bool clip) {
  if (!t || count <= 0) return OAPL_ERR_INVALID_ARG;
  int64_t chunks = 0;
  for (int32_t i = 0; i < count; ++i) {
    const int es = type_shift(t[i].type);
    if (t[i].n < 0 || es < 0) return OAPL_ERR_INVALID_ARG;
    if (!t[i].n) continue;
    const uintptr_t in = (uintptr_t)t[i].data, out = (uintptr_t)t[i].out;
    if (!in) return OAPL_ERR_INVALID_ARG;
    if (in & ((1u << es) - 1)) return OAPL_ERR_MISALIGNED;
    chunks += (t[i].n - 1) / (kGcBytes / 4) + 1;  // the most that its types can give
    if (chunks > kMaxGrid) return OAPL_ERR_UNSUPPORTED_SHAPE;
    if (!clip) continue;
    const int os = type_shift(t[i].out_type);
    if (!out || os < 0) return OAPL_ERR_INVALID_ARG;
    if (out & ((1u << os) - 1)) return OAPL_ERR_MISALIGNED;
    if (in == out) {
      if (t[i].type != t[i].out_type) return OAPL_ERR_INVALID_ARG;
    } else if (in < out + ((uintptr_t)t[i].n << os) && out < in + ((uintptr_t)t[i].n << es)) {
      return OAPL_ERR_INVALID_ARG;  // partly over itself
    }
  }
  return OAPL_OK;
}

// The next tensors of the list that fit into a launch; returns how many entries were used up.
static int32_t fill_list(const oapl_tensor* t, int32_t count, bool clip, GradList* l) {
  l->count = l->chunks = 0;
  int32_t i = 0;
  for (; i < count && l->count < kGcList; ++i) {
    if (!t[i].n) continue;
    GradTensor& g = l->t[l->count++];
    g.in = t[i].data;
    g.out = clip ? t[i].out : nullptr;
    g.n = t[i].n;
    g.first = l->chunks;
    g.in_type = (uint8_t)t[i].type;
    g.out_type = (uint8_t)(clip ? t[i].out_type : 0);
    g.vec = on16(t[i].data) && (!clip || on16(t[i].out));
    g.shift = t[i].type == OAPL_TYPE_F32 || (clip && t[i].out_type == OAPL_TYPE_F32) ? 12 : 13;
    static_assert(kGcBytes == 4 << 12, "a chunk's elements");
    l->chunks += (int32_t)((t[i].n - 1 >> g.shift) + 1);
  }
  return i;
}

template <typename TI>
static auto pick_clip(int out) -> void (*)(GradList, const float*, const float*, float, float) {
  return out == 0 ? grad_clip_kernel<TI, __nv_bfloat16> : out == 1 ? grad_clip_kernel<TI, __half> : grad_clip_kernel<TI, float>;
}

constexpr int kGcMaxSums = 2048;  // partial sums of a launch

// ---------------------------------------------------------------------------------------
// Adjustments of logits.
static int check_adjust(const oapl_logits* L, const oapl_adjust* a) {
  const int rc = check_logits(L);
  if (rc != OAPL_OK) return rc;
  if (!a || a->T < 0 || a->biases < 0) return OAPL_ERR_INVALID_ARG;
  if ((a->tokens && !a->spans) || (a->spans && a->T > 0 && !a->tokens)) return OAPL_ERR_INVALID_ARG;
  if ((a->repetition || a->frequency || a->presence) && !a->spans) return OAPL_ERR_INVALID_ARG;
  if (a->bias_start && a->biases > 0 && (!a->bias_id || !a->bias)) return OAPL_ERR_INVALID_ARG;
  if (a->allowed) {
    if (a->ld_allowed < ((int64_t)L->V + 31) / 32 || a->allowed_rows <= 0) return OAPL_ERR_INVALID_ARG;
    if (!a->allowed_row && a->allowed_rows != L->N) return OAPL_ERR_INVALID_ARG;
  } else if (a->allowed_row) {
    return OAPL_ERR_INVALID_ARG;
  }
  const uintptr_t four = (uintptr_t)a->tokens | (uintptr_t)a->repetition | (uintptr_t)a->frequency |
                         (uintptr_t)a->presence | (uintptr_t)a->bias_id | (uintptr_t)a->bias | (uintptr_t)a->allowed |
                         (uintptr_t)a->allowed_row;
  const uintptr_t eight = (uintptr_t)a->spans | (uintptr_t)a->bias_start;
  if ((four & 3) || (eight & 7)) return OAPL_ERR_MISALIGNED;
  return OAPL_OK;
}

static AdjustParams adjust_params(const oapl_logits* L, const oapl_adjust* a, void* out, int64_t ld_o, int32_t* status) {
  AdjustParams p;
  memset(&p, 0, sizeof(p));
  p.z = L->logits;
  p.ld_z = L->ld;
  p.V = L->V;
  p.N = (int32_t)L->N;
  p.mask = L->mask;
  p.out = out;
  p.ld_o = ld_o;
  p.tokens = a->tokens;
  p.T = a->T;
  p.spans = a->spans;
  p.repetition = a->repetition;
  p.frequency = a->frequency;
  p.presence = a->presence;
  p.bias_start = a->bias_start;
  p.bias_id = a->bias_id;
  p.bias = a->bias;
  p.biases = a->biases;
  p.allowed = a->allowed;
  p.ld_allowed = a->ld_allowed;
  p.allowed_rows = a->allowed_rows;
  p.allowed_row = a->allowed_row;
  p.status = status;
  return p;
}

template <typename T, int KE, int VPT, bool GRAD, bool OVER>
static int launch_adjust(AdjustParams p, cudaStream_t st) {
  constexpr int64_t kSlice = (int64_t)KE * VPT * kAdThreads;
  const int64_t slices = ((int64_t)p.V + kSlice - 1) / kSlice;
  if (slices * p.N > kMaxGrid) return OAPL_ERR_UNSUPPORTED_SHAPE;
  p.slices = (int32_t)slices;
  auto kern = adjust_kernel<T, KE, VPT, GRAD, OVER>;
  const int smem = (p.allowed || p.history || p.biased ? (int)kSlice / 8 + 16 : 0) +
                   (p.history || p.biased ? AdjustShared<!GRAD ? 1 : OVER ? 2 : 0>::bytes((int)kSlice) : 0);
  constexpr int kMost = (int)kSlice / 8 + 16 + AdjustShared<!GRAD ? 1 : OVER ? 2 : 0>::bytes((int)kSlice);
  if (smem > 40 * 1024) {
    static bool done[kMaxDevices] = {false};
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return OAPL_ERR_CUDA;
    if (!done[dev]) {
      if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost) != cudaSuccess)
        return OAPL_ERR_CUDA;
      done[dev] = true;
    }
  }
  kern<<<(unsigned)(slices * p.N), kAdThreads, smem, st>>>(p);
  CKL();
  return OAPL_OK;
}

template <typename T, int KE, bool GRAD, bool OVER>
static int route_adjust_size(const AdjustParams& p, int n_sm, cudaStream_t st) {
  // Slices of 8192 tokens (16384 for the gradient apart from the logits, which counts nothing and keeps nothing, and 4096 an
  // element at a time) where they give every SM four CTAs, else half of that where they do, else 2048.
  constexpr int kMany = (KE == 1 ? 16 : GRAD && !OVER ? 64 : 32) / KE, kSome = kMany / 2, kFew = 8 / KE;
  const int64_t many = (int64_t)p.N * p.V / (kMany * KE * kAdThreads);
  if (many >= 4 * (int64_t)n_sm) return launch_adjust<T, KE, kMany, GRAD, OVER>(p, st);
  if (2 * many >= 4 * (int64_t)n_sm) return launch_adjust<T, KE, kSome, GRAD, OVER>(p, st);
  return launch_adjust<T, KE, kFew, GRAD, OVER>(p, st);
}

template <typename T>
static int route_adjust(const AdjustParams& p, bool grad, cudaStream_t st) {
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  constexpr int KE = Elem<T>::kN;
  // whether a row of b is as far off 16-byte boundaries as the result's
  auto level = [&](const void* b, int64_t ld) {
    return (((uintptr_t)b - (uintptr_t)p.out) & 15) == 0 && (p.N == 1 || (ld - p.ld_o) * (int64_t)sizeof(T) % 16 == 0);
  };
  const bool vec = level(grad ? p.d : p.z, grad ? p.ld_d : p.ld_z);
  if (grad && p.out == p.z)
    return vec ? route_adjust_size<T, KE, true, true>(p, n_sm, st) : route_adjust_size<T, 1, true, true>(p, n_sm, st);
  if (grad)
    return vec ? route_adjust_size<T, KE, true, false>(p, n_sm, st) : route_adjust_size<T, 1, true, false>(p, n_sm, st);
  if (p.out == p.z)
    return vec ? route_adjust_size<T, KE, false, true>(p, n_sm, st) : route_adjust_size<T, 1, false, true>(p, n_sm, st);
  return vec ? route_adjust_size<T, KE, false, false>(p, n_sm, st) : route_adjust_size<T, 1, false, false>(p, n_sm, st);
}

static int route_adjust_type(const AdjustParams& p, int32_t type, bool grad, cudaStream_t st) {
  if (type == OAPL_TYPE_BF16) return route_adjust<__nv_bfloat16>(p, grad, st);
  if (type == OAPL_TYPE_F16) return route_adjust<__half>(p, grad, st);
  return route_adjust<float>(p, grad, st);
}

}  // namespace oapl

using namespace oapl;

extern "C" {

int oapl_embedding(const oapl_lookup* lookup, const void* table, int32_t table_type, int64_t ld_table, int32_t d,
                   void* out, int32_t out_type, int64_t ld_out, int32_t* device_status, void* stream) {
  const int rc = check_lookup(lookup);
  if (rc != OAPL_OK) return rc;
  const int is = type_size(table_type), os = type_size(out_type);
  if (!table || !out || !is || !os || d <= 0 || ld_table < d || ld_out < d) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)table % is || (uintptr_t)out % os) return OAPL_ERR_MISALIGNED;
  const Place a{table, lookup->V, d, ld_table, is}, b{out, lookup->N, d, ld_out, os};
  if (overlap(a, b) != kApart) return OAPL_ERR_INVALID_ARG;
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  LookupParams p = lookup_params(lookup, d, device_status);
  p.in = table;
  p.ld_in = ld_table;
  p.out = out;
  p.ld_out = ld_out;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (table_type == OAPL_TYPE_BF16) return route_embedding_out<__nv_bfloat16>(p, out_type, n_sm, st);
  if (table_type == OAPL_TYPE_F16) return route_embedding_out<__half>(p, out_type, n_sm, st);
  return route_embedding_out<float>(p, out_type, n_sm, st);
}

size_t oapl_embedding_workspace_bytes(int64_t N, int32_t V, int32_t d) {
  LookupCarve c;
  return lookup_carve(N, V, d, &c) ? c.total : 0;
}

int oapl_embedding_bwd(const oapl_lookup* lookup, const void* dout, int32_t type, int64_t ld_dout, int32_t d,
                       float* dtable, int64_t ld_dtable, int accumulate, int32_t* device_status, void* ws,
                       size_t ws_bytes, void* stream) {
  const int rc = check_lookup(lookup);
  if (rc != OAPL_OK) return rc;
  const int es = type_size(type);
  if (!dout || !dtable || !ws || !es || d <= 0 || ld_dout < d || ld_dtable < d) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)dout % es || ((uintptr_t)dtable & 3) || !on16(ws)) return OAPL_ERR_MISALIGNED;
  const Place a{dout, lookup->N, d, ld_dout, es}, b{dtable, lookup->V, d, ld_dtable, 4};
  if (overlap(a, b) != kApart) return OAPL_ERR_INVALID_ARG;
  LookupCarve c;
  if (!lookup_carve(lookup->N, lookup->V, d, &c)) return OAPL_ERR_UNSUPPORTED_SHAPE;
  if (ws_bytes < c.total) return OAPL_ERR_WORKSPACE_TOO_SMALL;
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  uint8_t* w = static_cast<uint8_t*>(ws);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  LookupParams p = lookup_params(lookup, d, device_status);
  p.in = dout;
  p.ld_in = ld_dout;
  p.out = dtable;
  p.ld_out = ld_dtable;
  p.accumulate = accumulate != 0;
  p.chunk = c.chunk;
  p.chunks = c.chunks;
  p.sorted = reinterpret_cast<uint2*>(w + c.sorted);
  p.part = reinterpret_cast<float*>(w + c.part);
  p.joins = reinterpret_cast<uint32_t*>(w + c.joins);
  if (p.N <= kEbFew) {
    // one launch, see the kernel
  } else if (!c.passes) {
    const int per = kEbThreads / 32 * kEbCountRows;
    embedding_count_sort_kernel<<<(unsigned)((p.N + per - 1) / per), kEbThreads, 0, st>>>(p);
    CKL();
  } else {
    uint2* lists[2] = {p.sorted, reinterpret_cast<uint2*>(w + c.other)};
    RadixParams r;
    memset(&r, 0, sizeof(r));
    uint32_t* hist = reinterpret_cast<uint32_t*>(w + c.hist);
    const int64_t words = (int64_t)c.tiles << c.bits;
    r.total = reinterpret_cast<uint32_t*>(w + c.totals);
    r.bits = c.bits;
    r.tiles = c.tiles;
    r.hist = hist;
    r.clear = hist + words;
    r.clear_words = (c.passes - 1) * words;
    // Each tile's CTA adds up all tiles' counts itself while they are few: two batches of loads for 20 tiles (40960 rows),
    // where a launch in between takes 2 to 4 us.  Beyond 64 it would read too much.
    r.scanned = c.tiles > 64;
    embedding_radix_count_kernel<<<(unsigned)c.tiles, kEbThreads, 0, st>>>(p, r);
    CKL();
    for (int k = 0; k < c.passes; ++k) {
      r.hist = hist + k * words;
      r.next = k + 1 < c.passes ? r.hist + words : nullptr;
      r.shift = k * c.bits;
      r.out = lists[(c.passes - 1 - k) & 1];  // the last pass into `sorted`
      if (r.scanned) {
        CK(launch_next(embedding_radix_scan_kernel, dim3((unsigned)(((1 << c.bits) + 31) / 32)), dim3(32, 32), 0, st, r));
      }
      CK(launch_next(embedding_radix_move_kernel, dim3((unsigned)c.tiles), dim3(kEbMoveThreads), 0, st, p, r));
      r.in = r.out;
    }
  }
  if (type == OAPL_TYPE_BF16) return route_embedding_sum<__nv_bfloat16>(p, n_sm, st);
  if (type == OAPL_TYPE_F16) return route_embedding_sum<__half>(p, n_sm, st);
  return route_embedding_sum<float>(p, n_sm, st);
}

size_t oapl_grad_norm_workspace_bytes(int32_t count) {
  return count <= 0 ? 0 : sizeof(double) * kGcMaxSums * (((size_t)count + kGcList - 1) / kGcList);
}

int oapl_grad_norm(const oapl_tensor* tensors, int32_t count, float scale, float* sq_norm, float* norm,
                   int32_t* device_status, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_tensors(tensors, count, false);
  if (rc != OAPL_OK) return rc;
  if ((!sq_norm && !norm) || !ws || !std::isfinite(scale)) return OAPL_ERR_INVALID_ARG;
  if (!on16(ws) || (((uintptr_t)sq_norm | (uintptr_t)norm) & 3)) return OAPL_ERR_MISALIGNED;
  if (ws_bytes < oapl_grad_norm_workspace_bytes(count)) return OAPL_ERR_WORKSPACE_TOO_SMALL;
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  const int most = n_sm * kGcSumsPerSm < kGcMaxSums ? n_sm * kGcSumsPerSm : kGcMaxSums;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  double* part = static_cast<double*>(ws);
  int sums = 0;
  for (int32_t i = 0; i < count;) {
    GradList l;
    i += fill_list(tensors + i, count - i, false, &l);
    if (!l.chunks) continue;
    const int grid = l.chunks < most ? l.chunks : most;
    grad_norm_kernel<<<grid, kGcThreads, 0, st>>>(l, part + sums);
    CKL();
    sums += grid;
  }
  CK(launch_next(grad_norm_join_kernel, dim3(1), dim3(kGcThreads), 0, st, (const double*)part, sums, scale, sq_norm, norm,
                 device_status));
  return OAPL_OK;
}

int oapl_grad_clip(const oapl_tensor* tensors, int32_t count, float scale, const float* sq_norm, float clip_norm,
                   void* stream) {
  return oapl_grad_clip_ex(tensors, count, scale, sq_norm, nullptr, clip_norm, stream);
}

int oapl_grad_clip_ex(const oapl_tensor* tensors, int32_t count, float scale, const float* sq_norm, const float* norm,
                      float clip_norm, void* stream) {
  const int rc = check_tensors(tensors, count, true);
  if (rc != OAPL_OK) return rc;
  if ((!sq_norm && !norm) || !std::isfinite(scale) || !(clip_norm > 0.f) || !std::isfinite(clip_norm))
    return OAPL_ERR_INVALID_ARG;
  if (((uintptr_t)sq_norm | (uintptr_t)norm) & 3) return OAPL_ERR_MISALIGNED;
  const int n_sm = sm_count();
  if (n_sm <= 0) return OAPL_ERR_CUDA;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  for (int32_t i = 0; i < count;) {
    GradList l;
    i += fill_list(tensors + i, count - i, true, &l);
    if (!l.chunks) continue;
    const int most = n_sm * kGcSumsPerSm;
    // a list of one pair of types, as most are, goes to a kernel of that pair, which needs no more than 52 registers
    // (453 M bf16 elements to bf16: 279 us; 383 with all nine pairs in one kernel)
    bool one = true;
    for (int32_t k = 1; k < l.count; ++k) one = one && l.t[k].in_type == l.t[0].in_type && l.t[k].out_type == l.t[0].out_type;
    const int in = l.t[0].in_type, out = l.t[0].out_type;
    auto kern = !one ? grad_clip_kernel<void, void>
                     : in == 0 ? pick_clip<__nv_bfloat16>(out) : in == 1 ? pick_clip<__half>(out) : pick_clip<float>(out);
    kern<<<l.chunks < most ? l.chunks : most, kGcThreads, 0, st>>>(l, sq_norm, norm, clip_norm, scale);
    CKL();
  }
  return OAPL_OK;
}

int oapl_logits_adjust(const oapl_logits* L, const oapl_adjust* a, void* out, int64_t ld_out, int32_t* device_status,
                       void* stream) {
  const int rc = check_adjust(L, a);
  if (rc != OAPL_OK) return rc;
  const int es = type_size(L->type);
  if (!out || ld_out < L->V) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)out % es) return OAPL_ERR_MISALIGNED;
  if (overlap({L->logits, L->N, L->V, L->ld, es}, {out, L->N, L->V, ld_out, es}) == kMixed) return OAPL_ERR_INVALID_ARG;
  AdjustParams p = adjust_params(L, a, out, ld_out, device_status);
  const bool history = a->spans && (a->repetition || a->frequency || a->presence);
  p.history = history;
  p.biased = a->bias_start && a->biases > 0;
  return route_adjust_type(p, L->type, false, static_cast<cudaStream_t>(stream));
}

int oapl_logits_adjust_bwd(const oapl_logits* L, const oapl_adjust* a, const void* d_out, int64_t ld_d_out,
                           void* dlogits, int64_t ld_dlogits, int32_t* device_status, void* stream) {
  const int rc = check_adjust(L, a);
  if (rc != OAPL_OK) return rc;
  const int es = type_size(L->type);
  if (!d_out || !dlogits || ld_d_out < L->V || ld_dlogits < L->V) return OAPL_ERR_INVALID_ARG;
  if ((uintptr_t)d_out % es || (uintptr_t)dlogits % es) return OAPL_ERR_MISALIGNED;
  const Place z{L->logits, L->N, L->V, L->ld, es}, d{d_out, L->N, L->V, ld_d_out, es},
      o{dlogits, L->N, L->V, ld_dlogits, es};
  if (overlap(z, o) == kMixed || overlap(d, o) == kMixed) return OAPL_ERR_INVALID_ARG;
  AdjustParams p = adjust_params(L, a, dlogits, ld_dlogits, device_status);
  p.d = d_out;
  p.ld_d = ld_d_out;
  p.history = a->repetition != nullptr;
  return route_adjust_type(p, L->type, true, static_cast<cudaStream_t>(stream));
}

}  // extern "C"

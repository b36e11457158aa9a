// Token embedding: rows of a table scaled by a constant, and the table's gradient.
//
// Forward: out[i] = scale table[tok_i], a gather.  Backward: dtable[v] = scale sum_{tok_i = v} dout[i].
// The tokens are sorted by a stable radix sort over (token, position), so that every table row's
// terms stand together in token order; tiles of EMB_RUN sorted positions are summed by one group of
// threads each, whatever the tokens' distribution, and the runs that cross tiles are joined from the
// tiles' partial rows in a second launch, in tile order.  No floating-point atomics.
#include "device_common.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ int64_t token_at(const void* tokens, int bytes, int64_t i) {
  return bytes == 8 ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

// VE consecutive elements of T as floats; VE > 1: 16-byte loads
template <typename T, int VE>
__device__ __forceinline__ void load_ve(const void* p, int64_t i, float* v) {
  if constexpr (VE == 1) {
    v[0] = St<T>::ld(p, i);
  } else {
#pragma unroll
    for (int c = 0; c < VE / St<T>::VE; ++c) {
      Chunk<T> k;
      load_chunk<T>(p, i + c * St<T>::VE, k);
#pragma unroll
      for (int e = 0; e < St<T>::VE; ++e) v[c * St<T>::VE + e] = k.v[e];
    }
  }
}
template <typename T, int VE>
__device__ __forceinline__ void store_ve(void* p, int64_t i, const float* v) {
  if constexpr (VE == 1) {
    St<T>::st(p, i, v[0]);
  } else {
#pragma unroll
    for (int c = 0; c < VE / St<T>::VE; ++c) store_chunk<T>(p, i + c * St<T>::VE, v + c * St<T>::VE);
  }
}

// Threads of a row: the smallest power of two that covers its pieces, at most the workgroup.
int threads_per_row(int64_t pieces) {
  int t = 1;
  while (t < THREADS && t < pieces) t *= 2;
  return t;
}

// ---- forward --------------------------------------------------------------------------------

struct EmbedFwd {
  const void *table, *tokens;
  void* out;
  int64_t n, vocab, table_stride, row_stride;
  int width, token_bytes, tpr;
  float scale;
};

template <typename TT, typename TO, int VE>
__global__ __launch_bounds__(THREADS) void embed_fwd_kernel(EmbedFwd a) {
  const int rows = THREADS / a.tpr;
  const int lane = threadIdx.x & (a.tpr - 1);
  for (int64_t i = (int64_t)blockIdx.x * rows + threadIdx.x / a.tpr; i < a.n; i += (int64_t)gridDim.x * rows) {
    const int64_t t = token_at(a.tokens, a.token_bytes, i);
    const bool in = t >= 0 && t < a.vocab;
    for (int c = lane * VE; c < a.width; c += a.tpr * VE) {
      float v[VE];
      if (in) {
        load_ve<TT, VE>(a.table, t * a.table_stride + c, v);
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] *= a.scale;
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[e] = t < 0 ? 0.0f : __builtin_nanf("");
      }
      store_ve<TO, VE>(a.out, i * a.row_stride + c, v);
    }
  }
}

bool al16p(const void* p) { return ((uintptr_t)p & 15) == 0; }

// ---- sort -------------------------------------------------------------------------------------

struct EmbedSort {
  const void* tokens;          // first pass: keys from the tokens, positions 0, 1, ..
  const int32_t *key_in, *pos_in;
  int32_t *key_out, *pos_out;
  unsigned* hist;              // [blocks][EMB_BINS] of this pass
  unsigned* total;             // [EMB_BINS]: if not NULL, hist holds sums over the earlier workgroups and this all of them
  unsigned* hist_next;         // of the next pass, zero before this launch; NULL: last pass
  int64_t n, vocab, blocks;
  int token_bytes, shift;
};

__device__ __forceinline__ int32_t sort_key(const EmbedSort& a, int64_t i) {
  if (a.tokens == nullptr) return a.key_in[i];
  const int64_t t = token_at(a.tokens, a.token_bytes, i);
  return t >= 0 && t < a.vocab ? (int32_t)t : (int32_t)a.vocab;
}

// first pass's histogram of each workgroup's EMB_ITEMS tokens; clears the later passes' histograms
__global__ __launch_bounds__(THREADS) void embed_hist_kernel(EmbedSort a, unsigned* hist, int passes) {
  __shared__ unsigned cnt[EMB_BINS];
  for (int b = threadIdx.x; b < EMB_BINS; b += THREADS) cnt[b] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * EMB_ITEMS;
  for (int k = threadIdx.x; k < EMB_ITEMS; k += THREADS)
    if (i0 + k < a.n) atomicAdd(&cnt[sort_key(a, i0 + k) & (EMB_BINS - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < EMB_BINS; b += THREADS) {
    unsigned* h = hist + (int64_t)blockIdx.x * EMB_BINS + b;
    h[0] = cnt[b];
    for (int p = 1; p < passes; ++p) h[p * a.blocks * EMB_BINS] = 0;
  }
}

// hist[b][bin] becomes the sum over the workgroups before b, total[bin] the sum over all: 8 bins a
// workgroup, 32 threads a bin with a contiguous share of the workgroups each.
__global__ __launch_bounds__(THREADS) void embed_offset_kernel(EmbedSort a) {
  const int bin = blockIdx.x * 8 + (threadIdx.x & 7), part = threadIdx.x >> 3;
  const int64_t share = (a.blocks + 31) / 32;
  const int64_t b0 = part * share < a.blocks ? part * share : a.blocks;
  const int64_t b1 = b0 + share < a.blocks ? b0 + share : a.blocks;
  __shared__ unsigned sum[32][8];
  unsigned t = 0;
  for (int64_t b = b0; b < b1; ++b) t += a.hist[b * EMB_BINS + bin];
  sum[part][threadIdx.x & 7] = t;
  __syncthreads();
  unsigned o = 0, all = 0;
  for (int p = 0; p < 32; ++p) {
    if (p < part) o += sum[p][threadIdx.x & 7];
    all += sum[p][threadIdx.x & 7];
  }
  for (int64_t b = b0; b < b1; ++b) {
    const unsigned c = a.hist[b * EMB_BINS + bin];
    a.hist[b * EMB_BINS + bin] = o;
    o += c;
  }
  if (part == 0) a.total[bin] = all;
}

// One stable radix pass: workgroup b places its EMB_ITEMS items behind those of smaller digits and
// those of the same digit in earlier workgroups.  Within the workgroup each wave owns a contiguous
// quarter; a first sweep counts its digits, a second one ranks items by the number of equal digits
// in lower lanes (ballots) and in earlier rounds (the wave's counters).  Integer counts only, so the
// atomics on the next pass's histogram do not depend on their order.
__global__ __launch_bounds__(THREADS) void embed_scatter_kernel(EmbedSort a) {
  constexpr int WAVES = THREADS / 64, ROUNDS = EMB_ITEMS / THREADS;
  __shared__ unsigned base[WAVES][EMB_BINS];
  __shared__ unsigned wsum[WAVES];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  for (int b = tid; b < WAVES * EMB_BINS; b += THREADS) (&base[0][0])[b] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * EMB_ITEMS + wave * (EMB_ITEMS / WAVES);
  int32_t key[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = i0 + r * 64 + lane;
    key[r] = i < a.n ? sort_key(a, i) : -1;
    if (i < a.n) atomicAdd(&base[wave][(key[r] >> a.shift) & (EMB_BINS - 1)], 1u);
  }
  // each thread: two neighbouring bins; their counts over all workgroups, and over earlier ones
  static_assert(EMB_BINS == 2 * THREADS, "two bins a thread");
  unsigned tot[2] = {0, 0}, before[2] = {0, 0};
  if (a.total != nullptr) {
    const uint2 h = ((const uint2*)(a.hist + (int64_t)blockIdx.x * EMB_BINS))[tid], t = ((const uint2*)a.total)[tid];
    before[0] = h.x;
    before[1] = h.y;
    tot[0] = t.x;
    tot[1] = t.y;
  } else for (int64_t b = 0; b < a.blocks; ++b) {
    const uint2 h = ((const uint2*)(a.hist + b * EMB_BINS))[tid];
    tot[0] += h.x;
    tot[1] += h.y;
    if (b < blockIdx.x) {
      before[0] += h.x;
      before[1] += h.y;
    }
  }
  // exclusive sum of the totals over the bins
  unsigned inc = tot[0] + tot[1];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned up = __shfl_up(inc, o, 64);
    if (lane >= o) inc += up;
  }
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();             // also: every wave's digit counts are complete
  unsigned start = inc - tot[0] - tot[1];
  for (int w = 0; w < wave; ++w) start += wsum[w];
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    unsigned o = start + before[k];
    for (int w = 0; w < WAVES; ++w) {
      const unsigned c = base[w][2 * tid + k];
      base[w][2 * tid + k] = o;
      o += c;
    }
    start += tot[k];
  }
  __syncthreads();
  // The wave's counters are only touched by its own lanes from here on; the leader of each group of
  // equal digits advances them, after every lane of the round has read its own.
  for (int r = 0; r < ROUNDS; ++r) {
    const int64_t i = i0 + r * 64 + lane;
    const bool on = i < a.n;
    const int digit = (key[r] >> a.shift) & (EMB_BINS - 1);
    unsigned long long same = __ballot(on);
#pragma unroll
    for (int b = 0; b < EMB_DIGIT; ++b) {
      const unsigned long long m = __ballot((digit >> b) & 1);
      same &= ((digit >> b) & 1) ? m : ~m;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    unsigned at = 0;
    if (on) at = base[wave][digit];
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (on && rank == 0) base[wave][digit] = at + __popcll(same);
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (on) {
      const unsigned to = at + rank;
      a.key_out[to] = key[r];
      a.pos_out[to] = a.tokens != nullptr ? (int32_t)i : a.pos_in[i];
      if (a.hist_next != nullptr)
        atomicAdd(&a.hist_next[(int64_t)(to / EMB_ITEMS) * EMB_BINS + ((key[r] >> (a.shift + EMB_DIGIT)) & (EMB_BINS - 1))], 1u);
    }
  }
}

// ---- sums -------------------------------------------------------------------------------------

struct EmbedSum {
  const int32_t *key, *pos;    // sorted
  const void* dout;
  float *dtable, *part;        // part [tiles][2][width]
  int64_t n, vocab, tiles, table_stride, row_stride;
  int width, tpr, accumulate;
  float scale;
};

template <int VE>
__device__ __forceinline__ void write_row(const EmbedSum& a, int64_t row, int c, const float* acc) {
  const int64_t o = row * a.table_stride + c;
  float v[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = a.scale * acc[e];
  if (a.accumulate) {
    float old[VE];
    load_ve<float, VE>(a.dtable, o, old);
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] += old[e];
  }
  store_ve<float, VE>(a.dtable, o, v);
}

// Sums of one tile: runs inside the tile are written, a run from the tile before goes to part row 0
// (also when it goes on behind this tile), one that starts here and goes on to part row 1.
template <typename T, int VE>
__global__ __launch_bounds__(THREADS) void embed_sum_kernel(EmbedSum a) {
  const int64_t tile = (int64_t)blockIdx.x * (THREADS / a.tpr) + threadIdx.x / a.tpr;
  const int c = ((threadIdx.x & (a.tpr - 1)) + blockIdx.y * a.tpr) * VE;
  if (tile >= a.tiles || c >= a.width) return;
  const int64_t s0 = tile * EMB_RUN, s1 = s0 + EMB_RUN < a.n ? s0 + EMB_RUN : a.n;
  const int32_t prev = s0 > 0 ? a.key[s0 - 1] : -1, next = s1 < a.n ? a.key[s1] : -1;
  int32_t cur = a.key[s0];
  float acc[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
  auto flush = [&](bool at_end) {
    if (cur >= a.vocab) return;
    if (cur == prev) store_ve<float, VE>(a.part, tile * 2 * a.width + c, acc);
    else if (at_end && cur == next) store_ve<float, VE>(a.part, (tile * 2 + 1) * a.width + c, acc);
    else write_row<VE>(a, cur, c, acc);
  };
  for (int64_t s = s0; s < s1; ++s) {
    const int32_t k = a.key[s];
    if (k != cur) {
      flush(false);
      cur = k;
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
    }
    if (k >= a.vocab) return;
    float v[VE];
    load_ve<T, VE>(a.dout, (int64_t)a.pos[s] * a.row_stride + c, v);
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] += v[e];
  }
  flush(true);
}

// Runs over several tiles, by the tile they start in: its part row 1, then the part rows 0 of the
// tiles up to the one the run ends in.
template <int VE>
__global__ __launch_bounds__(THREADS) void embed_join_kernel(EmbedSum a) {
  const int64_t tile = (int64_t)blockIdx.x * (THREADS / a.tpr) + threadIdx.x / a.tpr;
  const int c = ((threadIdx.x & (a.tpr - 1)) + blockIdx.y * a.tpr) * VE;
  if (tile + 1 >= a.tiles || c >= a.width) return;
  const int64_t s0 = tile * EMB_RUN, s1 = s0 + EMB_RUN;
  const int32_t cur = a.key[s1];
  if (cur >= a.vocab || a.key[s1 - 1] != cur || (s0 > 0 && a.key[s0 - 1] == cur)) return;
  float acc[VE];
  load_ve<float, VE>(a.part, (tile * 2 + 1) * a.width + c, acc);
  for (int64_t t = tile + 1; t < a.tiles && a.key[t * EMB_RUN] == cur; ++t) {
    // the run reaches tile t: at its first position the token still is this one
    float v[VE];
    load_ve<float, VE>(a.part, t * 2 * a.width + c, v);
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] += v[e];
  }
  write_row<VE>(a, cur, c, acc);
}

// Rows without tokens: zero (not when the gradient is added to).  A row has tokens if the sorted keys hold it.
template <int VE>
__global__ __launch_bounds__(THREADS) void embed_zero_kernel(EmbedSum a) {
  const int rows = THREADS / a.tpr;
  const int lane = threadIdx.x & (a.tpr - 1);
  for (int64_t v = (int64_t)blockIdx.x * rows + threadIdx.x / a.tpr; v < a.vocab; v += (int64_t)gridDim.x * rows) {
    int64_t lo = 0, hi = a.n;
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (a.key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    if (lo < a.n && a.key[lo] == v) continue;
    float z[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) z[e] = 0.0f;
    for (int c = lane * VE; c < a.width; c += a.tpr * VE) store_ve<float, VE>(a.dtable, v * a.table_stride + c, z);
  }
}

constexpr int64_t MAX_GRID = 65536;   // workgroups of the row loops

}  // namespace

int launch_embed_fwd(const pnn_embed_desc& d, const void* table, const void* tokens, void* out, hipStream_t s) {
  EmbedFwd a;
  a.table = table;
  a.tokens = tokens;
  a.out = out;
  a.n = d.n;
  a.vocab = d.vocab;
  a.table_stride = d.table_stride;
  a.row_stride = d.row_stride;
  a.width = (int)d.width;
  a.token_bytes = d.token_bytes;
  a.scale = d.scale;
  const int es = d.dtype == PNN_F32 ? 4 : 2, et = d.table_dtype == PNN_F32 ? 4 : 2;
  // 8 elements a piece: whole 16-byte pieces on both sides
  const bool wide = d.width % 8 == 0 && al16p(table) && al16p(out) && d.table_stride * et % 16 == 0 && d.row_stride * es % 16 == 0;
  a.tpr = threads_per_row(wide ? d.width / 8 : d.width);
  const int64_t grid = cdiv64(d.n, THREADS / a.tpr);
  const dim3 g((unsigned)(grid < MAX_GRID ? grid : MAX_GRID));
#define FWD(TT, TO)                                                              \
  do {                                                                           \
    if (wide) hipLaunchKernelGGL((embed_fwd_kernel<TT, TO, 8>), g, dim3(THREADS), 0, s, a); \
    else hipLaunchKernelGGL((embed_fwd_kernel<TT, TO, 1>), g, dim3(THREADS), 0, s, a);      \
  } while (0)
  if (et == 4 && es == 4) FWD(float, float);
  else if (et == 4) FWD(float, uint16_t);
  else if (es == 4) FWD(uint16_t, float);
  else FWD(uint16_t, uint16_t);
#undef FWD
  return (int)hipGetLastError();
}

int launch_embed_bwd(const pnn_embed_desc& d, const void* dout, const void* tokens, float* dtable, int accumulate,
                     void* ws, hipStream_t s) {
  const EmbedWs w = embed_ws(d);
  char* base = (char*)ws;
  EmbedSort a;
  a.n = d.n;
  a.vocab = d.vocab;
  a.blocks = w.blocks;
  a.token_bytes = d.token_bytes;
  unsigned* hist = (unsigned*)(base + w.hist);
  for (int p = 0; d.n > 0 && p < w.passes; ++p) {
    a.tokens = p == 0 ? tokens : nullptr;
    a.key_in = (const int32_t*)(base + w.key[(p + 1) & 1]);
    a.pos_in = (const int32_t*)(base + w.pos[(p + 1) & 1]);
    a.key_out = (int32_t*)(base + w.key[p & 1]);
    a.pos_out = (int32_t*)(base + w.pos[p & 1]);
    a.hist = hist + p * w.blocks * EMB_BINS;
    a.hist_next = p + 1 < w.passes ? hist + (p + 1) * w.blocks * EMB_BINS : nullptr;
    a.shift = p * EMB_DIGIT;
    if (p == 0) {
      hipLaunchKernelGGL(embed_hist_kernel, dim3((unsigned)w.blocks), dim3(THREADS), 0, s, a, hist, w.passes);
      if (const hipError_t e = hipGetLastError()) return (int)e;
    }
    a.total = nullptr;
    if (w.blocks > EMB_DIRECT) {
      a.total = (unsigned*)(base + w.total);
      hipLaunchKernelGGL(embed_offset_kernel, dim3(EMB_BINS / 8), dim3(THREADS), 0, s, a);
      if (const hipError_t e = hipGetLastError()) return (int)e;
    }
    hipLaunchKernelGGL(embed_scatter_kernel, dim3((unsigned)w.blocks), dim3(THREADS), 0, s, a);
    if (const hipError_t e = hipGetLastError()) return (int)e;
  }
  EmbedSum m;
  m.key = (const int32_t*)(base + w.key[(w.passes + 1) & 1]);
  m.pos = (const int32_t*)(base + w.pos[(w.passes + 1) & 1]);
  m.dout = dout;
  m.dtable = dtable;
  m.part = (float*)(base + w.part);
  m.n = d.n;
  m.vocab = d.vocab;
  m.tiles = w.tiles;
  m.table_stride = d.table_stride;
  m.row_stride = d.row_stride;
  m.width = (int)d.width;
  m.accumulate = accumulate != 0;
  m.scale = d.scale;
  const int es = d.dtype == PNN_F32 ? 4 : 2;
  const bool wide = d.width % 8 == 0 && al16p(dtable) && al16p(dout) && d.table_stride % 4 == 0 && d.row_stride * es % 16 == 0;
  const int64_t pieces = wide ? d.width / 8 : d.width;
  m.tpr = threads_per_row(pieces);
  const dim3 block(THREADS);
  if (d.n > 0) {
    const dim3 grid((unsigned)cdiv64(w.tiles, THREADS / m.tpr), (unsigned)cdiv64(pieces, m.tpr));
#define SUMS(T, VE)                                                        \
  do {                                                                     \
    hipLaunchKernelGGL((embed_sum_kernel<T, VE>), grid, block, 0, s, m);   \
    hipLaunchKernelGGL((embed_join_kernel<VE>), grid, block, 0, s, m);     \
  } while (0)
    if (es == 4) {
      if (wide) SUMS(float, 8);
      else SUMS(float, 1);
    } else {
      if (wide) SUMS(uint16_t, 8);
      else SUMS(uint16_t, 1);
    }
#undef SUMS
    if (const hipError_t e = hipGetLastError()) return (int)e;
  }
  if (!m.accumulate) {
    const int64_t g = cdiv64(d.vocab, THREADS / m.tpr);
    const dim3 grid((unsigned)(g < MAX_GRID ? g : MAX_GRID));
    if (wide) hipLaunchKernelGGL((embed_zero_kernel<8>), grid, block, 0, s, m);
    else hipLaunchKernelGGL((embed_zero_kernel<1>), grid, block, 0, s, m);
  }
  return (int)hipGetLastError();
}

}  // namespace pnn

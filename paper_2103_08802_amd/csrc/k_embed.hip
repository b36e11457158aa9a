// Token embedding: rows of a table scaled by a constant, and the table's gradient.
//
// Forward: out[i] = scale table[tok_i], a gather.  Backward: dtable[v] = scale sum_{tok_i = v} dout[i].
// The tokens are sorted by a stable radix sort over (token, position), so that every table row's
// terms stand together in token order; tiles of sorted positions are summed by one group of
// threads each, whatever the tokens' distribution, and the runs that cross tiles are joined from the
// tiles' partial rows in a second launch, by four waves whose sums are added in order: one order
// whatever the run.  A run is joined by one workgroup for every 512 columns, so one token on half of
// 65536 places takes 110 us where the words' distribution takes 71.  No floating-point atomics.
//
// Bound: HBM, for few tokens the dependent launches.  bf16, 16384 tokens, 2048 columns, 65536 rows:
// forward 16.7 us (92 MB; frequent rows come from the caches), gradient 136 us (604 MB at 4.4 TB/s, 480 MB
// of it zeros): sort 33 us in four launches, which clear 130 MB meanwhile, sums 23, joins and the rest
// of the zeros 75.  65536 tokens, 1024 columns, 8192 rows: 82 us a batch, 28 of it the sort, 40 the sums
// (134 MB), 13 the joins.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int THREADS = 256;

__device__ __forceinline__ int64_t token_at(const void* tokens, int bytes, int64_t i) {
  return bytes == 8 ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

// Elements a thread has of a row: two 16-byte pieces of float, one of bf16.  `left`: elements of the row from i on; a
// row's last thread may have fewer than VE.
constexpr int VE = 8;
template <typename T>
__device__ __forceinline__ void load_ve(const void* p, int64_t i, int left, float* v) {
  if (left >= VE) {
#pragma unroll
    for (int c = 0; c < VE; c += St<T>::VE) load_piece<T>(p, i + c, v + c);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] = e < left ? St<T>::ld(p, i + e) : 0.0f;
  }
}
template <typename T>
__device__ __forceinline__ void store_ve(void* p, int64_t i, int left, const float* v) {
  if (left >= VE) {
#pragma unroll
    for (int c = 0; c < VE; c += St<T>::VE) store_piece<T>(p, i + c, v + c, false);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < left) St<T>::st(p, i + e, v[e]);
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
  int width, token_bytes, tpr, past;
  float scale;
};

// W elements of T from i on: the piece of the output's type a thread has at a time
template <typename T, int W>
__device__ __forceinline__ void load_w(const void* p, int64_t i, float* v) {
  if constexpr (W >= St<T>::VE) {
#pragma unroll
    for (int c = 0; c < W; c += St<T>::VE) load_piece<T>(p, i + c, v + c);
  } else {                                         // four bf16 for a piece of float
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef u32x2 Mem __attribute__((aligned(2)));
    const u32x2 u = *(const Mem*)((const uint16_t*)p + i);
    v[0] = __uint_as_float(u.x << 16);
    v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16);
    v[3] = __uint_as_float(u.y & 0xffff0000u);
  }
}

template <typename TT, typename TO>
__global__ __launch_bounds__(THREADS) void embed_fwd_kernel(EmbedFwd a) {
  constexpr int W = St<TO>::VE;
  const int rows = THREADS / a.tpr;
  const int lane = threadIdx.x & (a.tpr - 1);
  for (int64_t i = (int64_t)blockIdx.x * rows + threadIdx.x / a.tpr; i < a.n; i += (int64_t)gridDim.x * rows) {
    const int64_t t = token_at(a.tokens, a.token_bytes, i);
    const bool in = t >= 0 && t < a.vocab;
    const float none = t < 0 ? 0.0f : __builtin_nanf("");
    for (int c = lane * W; c < a.width; c += a.tpr * W) {
      const int64_t from = (in ? t : 0) * a.table_stride + c, to = i * a.row_stride + c;
      if (c + W <= a.width) {
        float v[W];
        if (in) load_w<TT, W>(a.table, from, v);
#pragma unroll
        for (int e = 0; e < W; ++e) v[e] = in ? v[e] * a.scale : none;
        store_piece<TO>(a.out, to, v, a.past);
      } else {
        for (int e = 0; e < a.width - c; ++e) St<TO>::st(a.out, to + e, in ? St<TT>::ld(a.table, from + e) * a.scale : none);
      }
    }
  }
}

// ---- sort -------------------------------------------------------------------------------------

// Rows of the gradient to clear: [row0, row1), `rows` to a workgroup (a power of two up to 32, about 64 KB).
struct ClearRows {
  float* dtable;
  int64_t table_stride, row0, row1;
  int width, rows, past;
};
// workgroup i of those that clear; has: bits of the rows of its word of row bits that are left as they are
__device__ __forceinline__ void clear_rows(const ClearRows& a, int64_t i, const unsigned* present) {
  constexpr int ZE = St<float>::VE;
  const float z[ZE] = {};
  const int64_t first = a.row0 + i * a.rows;
  const unsigned has = present != nullptr ? present[first / 32] >> (first & 31) : 0;
  int tpr = 1;
  while (tpr < (int)blockDim.x && tpr * ZE < a.width) tpr *= 2;
  const int lane = threadIdx.x & (tpr - 1);
  for (int r = threadIdx.x / tpr; r < a.rows; r += blockDim.x / tpr) {
    if (first + r >= a.row1 || (has >> r & 1)) continue;
    for (int c = lane * ZE; c < a.width; c += tpr * ZE) {
      const int64_t o = (first + r) * a.table_stride + c;
      if (c + ZE <= a.width) store_piece<float>(a.dtable, o, z, a.past);
      else
        for (int e = 0; e < a.width - c; ++e) a.dtable[o + e] = 0.0f;
    }
  }
}

struct EmbedSort {
  const void* tokens;          // first pass: keys from the tokens, positions 0, 1, ..
  const int32_t *key_in, *pos_in;
  int32_t *key_out, *pos_out;
  unsigned* hist;              // [blocks][EMB_BINS]
  unsigned* total;             // [EMB_BINS]: if not NULL, hist holds sums over the earlier workgroups and this all of them
  unsigned* present;           // a bit for every row of the table, cleared by the first launch (embed_sum_kernel sets them)
  int64_t n, vocab, blocks, words;
  int token_bytes, shift, passes;
  // The sort leaves the memory idle: the workgroups of its launches behind the first clear_from clear some rows of the
  // gradient, whether or not the sums will write them.
  int64_t clear_from;
  ClearRows clear;
};

__device__ __forceinline__ bool clears_rows(const EmbedSort& a) {
  if (blockIdx.x < a.clear_from) return false;
  clear_rows(a.clear, blockIdx.x - a.clear_from, nullptr);
  return true;
}

// key and position of item i; past the end the last one's (not to be used)
template <bool FIRST>
__device__ __forceinline__ void item(const EmbedSort& a, int64_t i, int32_t& key, int32_t& pos) {
  i = i < a.n ? i : a.n - 1;
  if constexpr (FIRST) {
    const int64_t t = token_at(a.tokens, a.token_bytes, i);
    key = t >= 0 && t < a.vocab ? (int32_t)t : (int32_t)a.vocab;
    pos = (int32_t)i;
  } else {
    key = a.key_in[i];
    pos = a.pos_in[i];
  }
}

__device__ __forceinline__ void clear_present(const EmbedSort& a) {
  for (int64_t w = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; w < a.words; w += a.clear_from * blockDim.x)
    a.present[w] = 0;
}

// The pass's histogram of each workgroup's EMB_ITEMS items (the first one also clears the row bits).  A launch of its
// own for every pass: counted by the pass before as it places its items, the frequent tokens' digits meet in a few
// counters (16384 tokens: that pass 26 us instead of 7).
template <bool FIRST>
__global__ __launch_bounds__(THREADS) void embed_hist_kernel(EmbedSort a) {
  __shared__ unsigned cnt[EMB_BINS];
  if (clears_rows(a)) return;
  if (FIRST) clear_present(a);
  if (blockIdx.x >= a.blocks) return;
  for (int b = threadIdx.x; b < EMB_BINS; b += THREADS) cnt[b] = 0;
  __syncthreads();
  const int64_t i0 = (int64_t)blockIdx.x * EMB_ITEMS;
  int32_t key[EMB_ITEMS / THREADS], pos;
#pragma unroll
  for (int r = 0; r < EMB_ITEMS / THREADS; ++r) item<FIRST>(a, i0 + r * THREADS + threadIdx.x, key[r], pos);
#pragma unroll
  for (int r = 0; r < EMB_ITEMS / THREADS; ++r)
    if (i0 + r * THREADS + threadIdx.x < a.n) atomicAdd(&cnt[(key[r] >> a.shift) & (EMB_BINS - 1)], 1u);
  __syncthreads();
  for (int b = threadIdx.x; b < EMB_BINS; b += THREADS) a.hist[(int64_t)blockIdx.x * EMB_BINS + b] = cnt[b];
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
#pragma unroll 8
  for (int64_t b = b0; b < b1; ++b) t += a.hist[b * EMB_BINS + bin];
  sum[part][threadIdx.x & 7] = t;
  __syncthreads();
  unsigned o = 0, all = 0;
  for (int p = 0; p < 32; ++p) {
    if (p < part) o += sum[p][threadIdx.x & 7];
    all += sum[p][threadIdx.x & 7];
  }
#pragma unroll 8
  for (int64_t b = b0; b < b1; ++b) {
    const unsigned c = a.hist[b * EMB_BINS + bin];
    a.hist[b * EMB_BINS + bin] = o;
    o += c;
  }
  if (part == 0) a.total[bin] = all;
}

// Lanes of the wave whose item has the same digit (ballots over its bits), among those that are on.
__device__ __forceinline__ unsigned long long same_digit(int digit, bool on) {
  unsigned long long same = __ballot(on);
#pragma unroll
  for (int b = 0; b < EMB_DIGIT; ++b) {
    const unsigned long long m = __ballot((digit >> b) & 1);
    same &= ((digit >> b) & 1) ? m : ~m;
  }
  return same;
}

// The place of each lane's item: the counter of its digit plus its rank among the wave's equal digits.
// The counters belong to this wave; the first lane of each group advances its counter once every lane
// has read (one wave's LDS operations complete in order; the fences keep the compiler to it).
__device__ __forceinline__ unsigned take_place(unsigned* counter, int digit, bool on) {
  const unsigned long long same = same_digit(digit, on);
  const int rank = __popcll(same & ((1ull << (threadIdx.x & 63)) - 1));
  unsigned at = 0;
  if (on) at = counter[digit];
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (on && rank == 0) counter[digit] = at + __popcll(same);
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return at + rank;
}

// Turns the waves' digit counts cnt[wave][bin] into first places: behind the smaller digits of all
// items (tot: the counts over all items of this thread's bins, BPT of them in a row), behind `before` (equal digits of earlier
// workgroups), behind earlier waves.
template <int NW, int BPT>
__device__ __forceinline__ void first_places(unsigned (*cnt)[EMB_BINS], const unsigned* tot, const unsigned* before,
                                             unsigned* wsum) {
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  unsigned own = 0;
#pragma unroll
  for (int k = 0; k < BPT; ++k) own += tot[k];
  unsigned inc = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const unsigned up = __shfl_up(inc, o, 64);
    if (lane >= o) inc += up;
  }
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();             // also: every wave's counts are complete
  unsigned start = inc - own;
  for (int w = 0; w < wave; ++w) start += wsum[w];
#pragma unroll
  for (int k = 0; k < BPT; ++k) {
    unsigned o = start + before[k];
    for (int w = 0; w < NW; ++w) {
      const unsigned c = cnt[w][BPT * tid + k];
      cnt[w][BPT * tid + k] = o;
      o += c;
    }
    start += tot[k];
  }
  __syncthreads();
}

// One stable radix pass: workgroup b places its EMB_ITEMS items behind those of smaller digits and
// those of the same digit in earlier workgroups.  Within the workgroup each wave owns a contiguous
// quarter: it counts its digits, then places its items 64 at a time.
template <bool FIRST>
__global__ __launch_bounds__(THREADS) void embed_scatter_kernel(EmbedSort a) {
  constexpr int WAVES = THREADS / 64, ROUNDS = EMB_ITEMS / THREADS;
  __shared__ unsigned base[WAVES][EMB_BINS];
  __shared__ unsigned wsum[WAVES];
  if (clears_rows(a)) return;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  const int64_t i0 = (int64_t)blockIdx.x * EMB_ITEMS + wave * (EMB_ITEMS / WAVES) + lane;
  int32_t key[ROUNDS], pos[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) item<FIRST>(a, i0 + r * 64, key[r], pos[r]);
  // each thread: two neighbouring bins; their counts over all workgroups, and over earlier ones
  static_assert(EMB_BINS == 2 * THREADS, "two bins a thread");
  unsigned tot[2] = {0, 0}, before[2] = {0, 0};
  if (a.total != nullptr) {
    const uint2 h = ((const uint2*)(a.hist + (int64_t)blockIdx.x * EMB_BINS))[tid], t = ((const uint2*)a.total)[tid];
    before[0] = h.x;
    before[1] = h.y;
    tot[0] = t.x;
    tot[1] = t.y;
  } else {
#pragma unroll 8
    for (int b = 0; b < (int)a.blocks; ++b) {
      const uint2 h = ((const uint2*)(a.hist + b * EMB_BINS))[tid];
      tot[0] += h.x;
      tot[1] += h.y;
      before[0] += b < (int)blockIdx.x ? h.x : 0;
      before[1] += b < (int)blockIdx.x ? h.y : 0;
    }
  }
  for (int b = tid; b < WAVES * EMB_BINS; b += THREADS) (&base[0][0])[b] = 0;
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r)
    if (i0 + r * 64 < a.n) atomicAdd(&base[wave][(key[r] >> a.shift) & (EMB_BINS - 1)], 1u);
  first_places<WAVES, 2>(base, tot, before, wsum);
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const bool on = i0 + r * 64 < a.n;
    const unsigned to = take_place(base[wave], (key[r] >> a.shift) & (EMB_BINS - 1), on);
    if (!on) continue;
    a.key_out[to] = key[r];
    a.pos_out[to] = pos[r];
  }
}

// Up to EMB_ITEMS tokens: every pass in one workgroup, the items in LDS between passes.
__global__ __launch_bounds__(2 * THREADS) void embed_sort_kernel(EmbedSort a) {
  constexpr int WAVES = 2 * THREADS / 64, ROUNDS = EMB_ITEMS / (2 * THREADS);
  __shared__ unsigned base[WAVES][EMB_BINS];
  __shared__ unsigned wsum[WAVES];
  __shared__ int32_t skey[EMB_ITEMS], spos[EMB_ITEMS];
  if (clears_rows(a)) return;
  clear_present(a);
  if (blockIdx.x > 0) return;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  const int i0 = wave * (EMB_ITEMS / WAVES) + lane, n = (int)a.n;
  int32_t key[ROUNDS], pos[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) item<true>(a, i0 + r * 64, key[r], pos[r]);
  for (int p = 0; p < a.passes; ++p) {
    const int shift = p * EMB_DIGIT;
    for (int b = tid; b < WAVES * EMB_BINS; b += 2 * THREADS) (&base[0][0])[b] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (i0 + r * 64 < n) atomicAdd(&base[wave][(key[r] >> shift) & (EMB_BINS - 1)], 1u);
    __syncthreads();
    static_assert(EMB_BINS == 2 * THREADS, "a bin a thread");
    unsigned tot = 0;
    const unsigned before = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) tot += base[w][tid];
    first_places<WAVES, 1>(base, &tot, &before, wsum);
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
      const bool on = i0 + r * 64 < n;
      const unsigned to = take_place(base[wave], (key[r] >> shift) & (EMB_BINS - 1), on);
      if (on) {
        skey[to] = key[r];
        spos[to] = pos[r];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r)
      if (i0 + r * 64 < n) {
        key[r] = skey[i0 + r * 64];
        pos[r] = spos[i0 + r * 64];
      }
    __syncthreads();
  }
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r)
    if (i0 + r * 64 < n) {
      a.key_out[i0 + r * 64] = key[r];
      a.pos_out[i0 + r * 64] = pos[r];
    }
}

// ---- sums -------------------------------------------------------------------------------------

struct EmbedSum {
  const int32_t *key, *pos;    // sorted
  const void* dout;
  float *dtable, *part;        // part [tiles][2][width]
  unsigned* present;           // NULL: no row has tokens
  int64_t n, vocab, tiles, table_stride, row_stride;
  int64_t join_blocks;         // second launch: workgroups that join runs; the others clear rows
  int width, tpr, run, accumulate;
  float scale;
  ClearRows clear;             // the rows of the second launch
};

__device__ __forceinline__ void write_row(const EmbedSum& a, int64_t row, int c, int left, const float* acc) {
  const int64_t o = row * a.table_stride + c;
  float v[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = a.scale * acc[e];
  if (a.accumulate) {
    float old[VE];
    load_ve<float>(a.dtable, o, left, old);
#pragma unroll
    for (int e = 0; e < VE; ++e) v[e] += old[e];
  }
  store_ve<float>(a.dtable, o, left, v);
}

// Sums of one tile: runs inside the tile are written, a run from the tile before goes to part row 0
// (also when it goes on behind this tile), one that starts here and goes on to part row 1.  The rows
// of eight positions are loaded at a time.  UNI: a tile's threads are whole waves; WHOLE: the width is a multiple of VE
// (without the second set of loads 67 registers a lane instead of 109: 16384 x 2048 138 us against 149).
template <typename T, bool UNI, bool WHOLE>
__global__ __launch_bounds__(THREADS) void embed_sum_kernel(EmbedSum a) {
  int sub = threadIdx.x / a.tpr;
  if constexpr (UNI) sub = __builtin_amdgcn_readfirstlane(sub);
  const int64_t tile = (int64_t)blockIdx.x * (THREADS / a.tpr) + sub;
  const int c = ((threadIdx.x & (a.tpr - 1)) + blockIdx.y * a.tpr) * VE;
  if (tile >= a.tiles || c >= a.width) return;
  const int64_t s0 = tile * a.run, s1 = s0 + a.run < a.n ? s0 + a.run : a.n;
  const int32_t prev = s0 > 0 ? a.key[s0 - 1] : -1, next = s1 < a.n ? a.key[s1] : -1;
  const int left = WHOLE ? VE : a.width - c;     // elements from c on
  int32_t cur = a.key[s0];
  float acc[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
  auto flush = [&](bool at_end) {
    if (cur >= a.vocab) return;
    if (cur == prev) {
      store_ve<float>(a.part, tile * 2 * a.width + c, left, acc);
    } else {
      if (c == 0 && !a.accumulate) atomicOr(&a.present[cur >> 5], 1u << (cur & 31));
      if (at_end && cur == next) store_ve<float>(a.part, (tile * 2 + 1) * a.width + c, left, acc);
      else write_row(a, cur, c, left, acc);
    }
  };
  constexpr int U = 8;
  for (int64_t s = s0; s < s1 && cur < a.vocab; s += U) {
    int32_t k[U], p[U];
    float v[U][VE];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t i = s + u < s1 ? s + u : s1 - 1;
      k[u] = a.key[i];
      p[u] = a.pos[i];
    }
    if (left >= VE) {
#pragma unroll
      for (int u = 0; u < U; ++u) load_ve<T>(a.dout, (int64_t)p[u] * a.row_stride + c, VE, v[u]);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) load_ve<T>(a.dout, (int64_t)p[u] * a.row_stride + c, left, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (s + u >= s1) break;
      if (k[u] != cur) {
        flush(false);
        cur = k[u];
#pragma unroll
        for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
      }
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] += v[u][e];
    }
  }
  flush(true);
}

// Second launch.  Its first join_blocks workgroups join the runs over several tiles, by the tile they
// start in: its part row 1, then the part rows 0 of the tiles up to the one the run ends in; each of
// the JW groups of 64 threads takes every JW-th of them, the groups' sums are added in order.  The
// others clear the rows without tokens that the sort's launches left.
__global__ __launch_bounds__(THREADS) void embed_join_kernel(EmbedSum a) {
  constexpr int JW = THREADS / 64;
  if (blockIdx.x < a.join_blocks) {
    __shared__ float sum[JW][64][VE];
    const int slabs = (a.width + 64 * VE - 1) / (64 * VE);
    const int64_t tile = blockIdx.x / slabs;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = ((int)(blockIdx.x - tile * slabs) * 64 + lane) * VE;
    const int64_t s0 = tile * a.run, s1 = s0 + a.run;
    const int32_t cur = a.key[s1];
    if (cur >= a.vocab || a.key[s1 - 1] != cur || (s0 > 0 && a.key[s0 - 1] == cur)) return;
    // the run's last tile: the last one whose first key is this token
    int64_t lo = tile + 1, hi = a.tiles - 1;
    while (lo < hi) {
      const int64_t mid = (lo + hi + 1) >> 1;
      if (a.key[mid * a.run] == cur) lo = mid;
      else hi = mid - 1;
    }
    const bool on = c < a.width;
    float acc[VE];
#pragma unroll
    for (int e = 0; e < VE; ++e) acc[e] = 0.0f;
    // rows of the sum: 0 is the first tile's part row 1, r >= 1 part row 0 of tile + r
    const int64_t rows = lo - tile + 1;
    constexpr int U = 4;
    for (int64_t r = wave; on && r < rows; r += U * JW) {
      float v[U][VE];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t i = r + u * JW < rows ? r + u * JW : r;
        load_ve<float>(a.part, (i == 0 ? tile * 2 + 1 : (tile + i) * 2) * a.width + c, a.width - c, v[u]);
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (r + u * JW < rows)
#pragma unroll
          for (int e = 0; e < VE; ++e) acc[e] += v[u][e];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) sum[wave][lane][e] = acc[e];
    __syncthreads();
    if (wave != 0 || !on) return;
#pragma unroll
    for (int w = 1; w < JW; ++w)
#pragma unroll
      for (int e = 0; e < VE; ++e) acc[e] += sum[w][lane][e];
    write_row(a, cur, c, a.width - c, acc);
    return;
  }
  clear_rows(a.clear, blockIdx.x - a.join_blocks, a.present);
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
  a.past = d.n * d.width * es > L2_BYTES;
  a.tpr = threads_per_row(cdiv64(d.width, 16 / es));
  const int64_t grid = cdiv64(d.n, THREADS / a.tpr);
  const dim3 g((unsigned)(grid < MAX_GRID ? grid : MAX_GRID));
#define FWD(TT, TO) hipLaunchKernelGGL((embed_fwd_kernel<TT, TO>), g, dim3(THREADS), 0, s, a)
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
  const dim3 block(THREADS);
  EmbedSort a;
  a.n = d.n;
  a.vocab = d.vocab;
  a.blocks = w.blocks;
  a.token_bytes = d.token_bytes;
  a.passes = w.passes;
  a.words = accumulate ? 0 : w.words;
  a.present = (unsigned*)(base + w.present);
  ClearRows clear;
  clear.dtable = dtable;
  clear.table_stride = d.table_stride;
  clear.width = (int)d.width;
  clear.rows = 32;
  while (clear.rows > 1 && clear.rows * d.width > 16384) clear.rows /= 2;
  clear.past = d.vocab * d.width * 4 > L2_BYTES;
  int64_t rows = accumulate ? 0 : d.vocab;               // rows not yet taken by a launch that clears them
  // The last rows left go to the launch to come: EMB_CLEAR bytes of them, whole words of row bits, and no more rows in
  // all than surely have no token (8192 rows, 65536 tokens: clearing what is written again took 5 us a call) unless the
  // tokens' rows are small (1237 tokens of 515 elements: clearing all rows 21 us, without theirs 25).  Returns the
  // grid: the workgroups they need behind the first `blocks`.
  const int64_t least = (d.n < d.vocab ? d.n : d.vocab) * d.width * 4 <= EMB_CLEAR / 4 ? 0 : cdiv64(d.n, 32) * 32;
  auto take_rows = [&](int64_t blocks) {
    const int64_t words = cdiv64(EMB_CLEAR, 32 * 4 * d.width);
    int64_t from = rows / 32 > words ? (rows / 32 - words) * 32 : 0;
    from = from > least ? from : least < rows ? least : rows;
    a.clear = clear;
    a.clear.row0 = from;
    a.clear.row1 = rows;
    a.clear_from = blocks;
    const int64_t more = cdiv64(rows - from, clear.rows);
    rows = from;
    return dim3((unsigned)(blocks + more));
  };
  // launches that clear the row bits: a workgroup for at most 4096 words more
  const int64_t bits = cdiv64(a.words, 4096) < MAX_GRID ? cdiv64(a.words, 4096) : MAX_GRID;
  int out = 0;
  if (d.n > 0 && w.blocks == 1) {
    a.tokens = tokens;
    a.key_out = (int32_t*)(base + w.key[0]);
    a.pos_out = (int32_t*)(base + w.pos[0]);
    hipLaunchKernelGGL(embed_sort_kernel, take_rows(bits > 1 ? bits : 1), dim3(2 * THREADS), 0, s, a);
    if (const hipError_t e = hipGetLastError()) return (int)e;
  } else if (d.n > 0) {
    a.tokens = tokens;
    a.hist = (unsigned*)(base + w.hist);
    for (int p = 0; p < w.passes; ++p) {
      out = p & 1;
      a.key_in = (const int32_t*)(base + w.key[1 - out]);
      a.pos_in = (const int32_t*)(base + w.pos[1 - out]);
      a.key_out = (int32_t*)(base + w.key[out]);
      a.pos_out = (int32_t*)(base + w.pos[out]);
      a.total = w.blocks > EMB_DIRECT ? (unsigned*)(base + w.total) : nullptr;
      a.shift = p * EMB_DIGIT;
      const dim3 hist_grid = take_rows(p == 0 && bits > w.blocks ? bits : w.blocks);
      if (p == 0) hipLaunchKernelGGL(embed_hist_kernel<true>, hist_grid, block, 0, s, a);
      else hipLaunchKernelGGL(embed_hist_kernel<false>, hist_grid, block, 0, s, a);
      if (a.total != nullptr) hipLaunchKernelGGL(embed_offset_kernel, dim3(EMB_BINS / 8), block, 0, s, a);
      const dim3 grid = take_rows(w.blocks);
      if (p == 0) hipLaunchKernelGGL(embed_scatter_kernel<true>, grid, block, 0, s, a);
      else hipLaunchKernelGGL(embed_scatter_kernel<false>, grid, block, 0, s, a);
      if (const hipError_t e = hipGetLastError()) return (int)e;
    }
  }
  EmbedSum m;
  m.key = (const int32_t*)(base + w.key[out]);
  m.pos = (const int32_t*)(base + w.pos[out]);
  m.dout = dout;
  m.dtable = dtable;
  m.part = (float*)(base + w.part);
  m.present = d.n > 0 ? a.present : nullptr;
  m.n = d.n;
  m.vocab = d.vocab;
  m.tiles = w.tiles;
  m.run = w.run;
  m.table_stride = d.table_stride;
  m.row_stride = d.row_stride;
  m.width = (int)d.width;
  m.accumulate = accumulate != 0;
  m.clear = clear;
  m.clear.row0 = 0;
  m.clear.row1 = rows;
  m.scale = d.scale;
  const int64_t pieces = cdiv64(d.width, VE);
  m.tpr = threads_per_row(pieces);
  if (d.n > 0) {
    const dim3 grid((unsigned)cdiv64(w.tiles, THREADS / m.tpr), (unsigned)cdiv64(pieces, m.tpr));
#define SUMS(T, UNI)                                                                                                \
  do {                                                                                                              \
    if (d.width % VE == 0) hipLaunchKernelGGL((embed_sum_kernel<T, UNI, true>), grid, block, 0, s, m);              \
    else hipLaunchKernelGGL((embed_sum_kernel<T, UNI, false>), grid, block, 0, s, m);                               \
  } while (0)
    if (m.tpr >= 64) {
      if (d.dtype == PNN_F32) SUMS(float, true);
      else SUMS(uint16_t, true);
    } else {
      if (d.dtype == PNN_F32) SUMS(float, false);
      else SUMS(uint16_t, false);
    }
#undef SUMS
    if (const hipError_t e = hipGetLastError()) return (int)e;
  }
  m.join_blocks = (w.tiles > 1 ? w.tiles - 1 : 0) * cdiv64(d.width, 64 * VE);
  const int64_t blocks = m.join_blocks + cdiv64(rows, clear.rows);
  if (blocks == 0) return 0;
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)blocks), block, 0, s, m);
  return (int)hipGetLastError();
}

}  // namespace pnn

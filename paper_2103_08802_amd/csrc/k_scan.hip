// Gated linear recurrence: h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(gate), and its backward.
//
// A stretch of steps acts on the state as h -> A h + B, A = product of its f, B = its result from a
// zero state, and two stretches compose.  A workgroup owns 64 lanes of channels (VEC of them a lane)
// and walks over tiles of NW x S steps: each wave takes S consecutive steps into registers, forms its
// (A, B), and from the (A, B) of the waves before it in LDS and the tile's first state the state its
// own steps start from; the steps are then run once more from there.  Every element is loaded once,
// the next tile's loads are in flight meanwhile, and there is one barrier a tile.  The backward goes
// through the tiles from the last: its chain c_t = f_t (dh_t + c_{t+1}) composes the same way from the
// right with the same A, and the states inside a tile are formed again from the state kept by the
// forward (every SCAN_CHUNK steps).
//
// Few channels do not fill the device with workgroups: a sequence's tiles are then dealt to several
// (scan_dealt), in order, by a ticket counter.  A workgroup publishes its tile's (A, B) as soon as the
// tile has been loaded, and takes the state the tile starts from by applying the (A, B) of the tiles
// since its own last one, in order.  So every element is still loaded once, and the bits do not depend
// on which workgroup had which tile.  Nobody waits for a later ticket: the holder of the smallest
// unpublished one waits for nothing, hence every wait ends, however few workgroups run at a time.
//
// Bound: HBM.  bf16, 8 x 2048 steps of 2048 channels: forward 42 us (201 MB, 4.8 TB/s; a large copy
// reaches 5.2), backward 81 us (335 MB, 4.2 TB/s); float 65 and 145 us (403 and 671 MB, part of it from
// the caches).  One sequence of 65536 steps, 1024 channels: forward 99 us (403 MB, 4.1 TB/s; with a first
// launch that sums up ranges and reads x and gate twice 139), backward 206 us (671 MB): there a tile of
// 128 steps costs a look back of two to three microseconds that nothing hides, as one workgroup fills a
// compute unit's registers.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int FS = SCAN_FS, BS = SCAN_BS;

struct Dims {
  int length, channels, groups, chunks, tiles;
  int dealt;                // workgroups a sequence's tiles are dealt to
  int past;                 // results larger than the L2 caches (store_to)
  int64_t chains;           // batch x groups
  pnn_seq_stride x, gate, h, dh, dx, dgate;
  unsigned* tickets;        // [chains]: the next tile
  float* first;             // [batch][channels]: the state before the first (backward: gradient after the last) step
  float2* sum;              // [chains][tiles][64 VEC]: (A, B) of a tile, READY set in A once published
};

// f = sigmoid(g) and keep = 1 - f = exp(-g) f, each to about an ulp (keep is not formed by subtraction), or zero where it
// is under about 1.6e-38 (f below g = -87, keep above 87.3): gates of -inf and +inf replace and hold a state exactly,
// however large it is.  g is held between -87 and 100, where exp(-g) is finite, by minimum and maximum that keep NaN.
// exp(-g) = 2^t (1 + d): t = -g log2(e) rounded, d the rest of that
// product to first order.  A bf16 g has 8 bits, so its product with the leading 16 bits of log2(e) is
// exact; for float the rounding is recovered by a fused multiply-add, and the reciprocal is refined.
template <typename T>
__device__ __forceinline__ void gate_of(float g, float& f, float& keep) {
  const bool closed = g < -87.0f;
  g = __builtin_elementwise_minimum(__builtin_elementwise_maximum(g, -87.0f), 100.0f);
  float e, r;
  if constexpr (sizeof(T) == 2) {
    constexpr float HI = 1.44268798828125f;                    // 16 bits of log2(e)
    constexpr float REST = (float)((1.4426950408889634074 - 1.44268798828125) * 0.69314718055994530942);
    e = __builtin_amdgcn_exp2f(g * -HI) * fmaf(g, -REST, 1.0f);
    r = __builtin_amdgcn_rcpf(1.0f + e);
  } else {
    constexpr float L = 1.44269502f, LO = 1.92596299e-8f;      // log2(e) in two floats
    const float t = g * -L;
    const float rest = fmaf(g, -LO, fmaf(g, -L, -t));
    e = __builtin_amdgcn_exp2f(t) * fmaf(rest, 0.693147181f, 1.0f);
    const float d = 1.0f + e;
    r = __builtin_amdgcn_rcpf(d);
    r = fmaf(fmaf(-d, r, 1.0f), r, r);
  }
  f = closed ? 0.0f : r;
  keep = e * r;
}

// VEC neighbouring channels of T as they are in memory
template <typename T, int VEC> struct Raw;
template <> struct Raw<uint16_t, 1> {
  typedef uint16_t U;
  typedef U Mem;
  __device__ static __forceinline__ void get(U u, float* v) { v[0] = bf2f(u); }
  __device__ static __forceinline__ U put(const float* v) { return f2bf(v[0]); }
};
template <> struct Raw<uint16_t, 2> {
  typedef uint32_t U;
  typedef U Mem __attribute__((aligned(2)));   // rows may start on any element
  __device__ static __forceinline__ void get(U u, float* v) {
    v[0] = __uint_as_float(u << 16);
    v[1] = __uint_as_float(u & 0xffff0000u);
  }
  __device__ static __forceinline__ U put(const float* v) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(U, __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2));
  }
};
template <> struct Raw<float, 1> {
  typedef float U;
  typedef U Mem;
  __device__ static __forceinline__ void get(U u, float* v) { v[0] = u; }
  __device__ static __forceinline__ U put(const float* v) { return v[0]; }
};

// Steps t0 .. t0 + S - 1 of one channel group, the ones from `end` on as `none`.  t0 and end are the
// same for all lanes.
template <typename T, int VEC, int S>
__device__ __forceinline__ void load_steps(typename Raw<T, VEC>::U (&r)[S], const void* base, const pnn_seq_stride& st,
                                           int64_t b, int t0, int end, int c, typename Raw<T, VEC>::U none) {
  typedef const typename Raw<T, VEC>::Mem Mem;
  const T* p = (const T*)base + (b * st.batch + (int64_t)t0 * st.step);
  if (t0 + S <= end) {
#pragma unroll
    for (int s = 0; s < S; ++s) r[s] = *at<Mem>(p + s * st.step, c * sizeof(T));
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s) r[s] = t0 + s < end ? *at<Mem>(p + s * st.step, c * sizeof(T)) : none;
  }
}

__device__ __forceinline__ int length_of(const int32_t* lengths, int64_t b, int length) {
  if (lengths == nullptr) return length;
  const int n = lengths[b];
  return n < 0 ? 0 : n > length ? length : n;
}

// The workgroup's sequence and channels: neighbouring workgroups have neighbouring channels of the same tiles
struct Place {
  int wave, lane, c, cc;
  int64_t chain, b;
  bool on;
};
template <int VEC>
__device__ __forceinline__ Place place(const Dims& d) {
  Place p;
  p.chain = blockIdx.x % d.chains;
  p.b = p.chain / d.groups;
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const ScanGroup r = scan_group(d.channels, (int)(p.chain - p.b * d.groups), VEC);
  p.c = r.first + p.lane * VEC;
  p.on = p.c < r.end;
  // lanes past the end load what the last one does; of an odd number of channels the last pair overlaps the one before
  // it, in the same wave, and both lanes store the same bits
  p.cc = p.c + VEC <= r.end ? p.c : r.end - VEC;
  p.c = p.cc;
  return p;
}

// ---- tiles dealt to several workgroups ---------------------------------------------------------

// A is never negative, so its sign bit tells a published pair from the zeros written ahead of the launch; the pair is
// one 8-byte word, stored and loaded whole at the device-wide level.
constexpr unsigned long long READY = 0x80000000ull;
constexpr int LOOK = 32;                   // tiles looked back at together
// Polls after which a thread gives up for good (seconds; a wait takes microseconds): what it would have waited for
// becomes NaN instead of the device hanging.
constexpr int MAX_POLLS = 1 << 22;

__device__ __forceinline__ void publish(float2* at, float A, float B) {
  const unsigned long long v = (unsigned long long)__float_as_uint(B) << 32 | __float_as_uint(A) | READY;
  __hip_atomic_store((unsigned long long*)at, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// known (of wave 0) from the state in front of tile k0 to that in front of tile k1, through the tiles' published pairs.
// Called by the whole workgroup; look: LOOK x 64 VEC pairs of LDS, free at the call.
template <int VEC, int NW>
__device__ __forceinline__ void look_back(const Dims& d, const Place& p, int k0, int k1, float (&known)[VEC], float2* look,
                                          bool& gave_up) {
  constexpr int CH = 64 * VEC;
  for (int j0 = k0; j0 < k1; j0 += LOOK) {
    const int m = k1 - j0 < LOOK ? k1 - j0 : LOOK;
    const unsigned long long* src = (const unsigned long long*)(d.sum + (p.chain * d.tiles + j0) * CH);
    for (int i = threadIdx.x; i < m * CH; i += 64 * NW) {
      unsigned long long v = __hip_atomic_load(src + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      for (int n = 0; !(v & READY) && !gave_up; ++n) {
        __builtin_amdgcn_s_sleep(1);
        v = __hip_atomic_load(src + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        gave_up = n >= MAX_POLLS;
      }
      const float A = v & READY ? __uint_as_float((unsigned)v & 0x7fffffffu) : __builtin_nanf("");
      look[i] = make_float2(A, __uint_as_float((unsigned)(v >> 32)));
    }
    __syncthreads();
    if (p.wave == 0)
#pragma unroll 4
      for (int j = 0; j < m; ++j)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 n = look[(j * 64 + p.lane) * VEC + e];
          known[e] = fmaf(n.x, known[e], n.y);
        }
    if (j0 + LOOK < k1) __syncthreads();   // before `look` is filled again
  }
}

// Before a launch with dealt tiles: no ticket taken, nothing published, the first states (dh0 may replace dhT, hT h0).
__global__ __launch_bounds__(256) void scan_begin_kernel(Dims d, const float* from, int64_t states, int64_t pairs) {
  const int64_t i0 = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  for (int64_t i = i0; i < pairs; i += step) d.sum[i] = make_float2(0.0f, 0.0f);
  for (int64_t i = i0; i < states; i += step) d.first[i] = from != nullptr ? from[i] : 0.0f;
  for (int64_t i = i0; i < d.chains; i += step) d.tickets[i] = 0;
}

// The tiles of a workgroup, in order: all of them, or by ticket.  `next` is taken one tile ahead, so that its loads can
// be in flight while `cur` is worked on.
template <bool DEALT>
struct Tiles {
  int cur, next;
  unsigned* ticket;
  __device__ __forceinline__ Tiles(const Dims& d, const Place& p, int* lds) {
    ticket = d.tickets + p.chain;
    cur = 0;
    next = 1;
    if constexpr (DEALT) {
      if (threadIdx.x == 0) {
        lds[0] = (int)__hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        lds[1] = (int)__hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      __syncthreads();
      cur = __builtin_amdgcn_readfirstlane(lds[0]);
      next = __builtin_amdgcn_readfirstlane(lds[1]);
    }
  }
  // thread 0: the ticket after next
  __device__ __forceinline__ int request() {
    return DEALT && threadIdx.x == 0 ? (int)__hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : 0;
  }
};

// f and b = (1 - f) x of the steps; identity from `end` on
template <typename T, int VEC, int S>
__device__ __forceinline__ void gates(const typename Raw<T, VEC>::U (&rx)[S], const typename Raw<T, VEC>::U (&rg)[S],
                                      int t0, int end, float (&f)[S][VEC], float (&b)[S][VEC]) {
#pragma unroll
  for (int s = 0; s < S; ++s) {
    float x[VEC], g[VEC];
    Raw<T, VEC>::get(rx[s], x);
    Raw<T, VEC>::get(rg[s], g);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      float keep;
      gate_of<T>(g[e], f[s][e], keep);
      b[s][e] = keep * x[e];
    }
  }
  if (t0 + S > end) {
#pragma unroll
    for (int s = 0; s < S; ++s)
      if (t0 + s >= end) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          f[s][e] = 1.0f;
          b[s][e] = 0.0f;
        }
      }
  }
}

// ---- forward --------------------------------------------------------------------------------

template <typename T, int VEC, int NW, bool DEALT>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 4 : 1) void scan_fwd_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  constexpr int L = NW * FS;
  __shared__ float2 part[2][NW][64][VEC];
  __shared__ float2 look[DEALT ? LOOK * 64 * VEC : 1];
  __shared__ float start[64][VEC];
  __shared__ int ticket[2];
  const Place p = place<VEC>(d);
  const int len = length_of(a.lengths, p.b, d.length), end = d.length;
  Tiles<DEALT> tiles(d, p, ticket);
  U rx[FS], rg[FS];
  auto load = [&](int k) {
    load_steps<T, VEC, FS>(rx, a.x, d.x, p.b, k * L + p.wave * FS, len, p.cc, U(0));
    load_steps<T, VEC, FS>(rg, a.gate, d.gate, p.b, k * L + p.wave * FS, len, p.cc, U(0));
  };
  if (tiles.cur < d.tiles) load(tiles.cur);
  // the state in front of the tile at hand; DEALT: of wave 0, in front of tile `known`
  float carry[VEC];
  int known = 0;
  bool gave_up = false;
  const float* first = DEALT ? d.first : a.h0;
#pragma unroll
  for (int e = 0; e < VEC; ++e) carry[e] = first != nullptr ? first[p.b * d.channels + p.cc + e] : 0.0f;
  T* const hp = (T*)a.h + p.b * d.h.batch;
  bool last = d.tiles == 0;
  int buf = 0;
  while (tiles.cur < d.tiles) {
    const int k = tiles.cur, t = k * L + p.wave * FS;
    const int after = tiles.request();
    float f[FS][VEC], b[FS][VEC], A[VEC], B[VEC], h[VEC];
    gates<T, VEC, FS>(rx, rg, t, len, f, b);
    if (tiles.next < d.tiles) load(tiles.next);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      A[e] = 1.0f;
      B[e] = 0.0f;
#pragma unroll
      for (int s = 0; s < FS; ++s) {
        A[e] *= f[s][e];
        B[e] = fmaf(f[s][e], B[e], b[s][e]);
      }
      h[e] = carry[e];
    }
    if constexpr (NW > 1) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) part[buf][p.wave][p.lane][e] = make_float2(A[e], B[e]);
      __syncthreads();
    }
    if constexpr (DEALT) {
      // wave 0: the tile's pair, published; the state in front of the tile, then behind it (by the pair, so that the
      // bits are those another workgroup would get)
      if (p.wave == 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          A[e] = 1.0f;
          B[e] = 0.0f;
        }
#pragma unroll 4
        for (int w = 0; w < NW; ++w)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float2 n = part[buf][w][p.lane][e];
            A[e] *= n.x;
            B[e] = fmaf(n.x, B[e], n.y);
          }
#pragma unroll
        for (int e = 0; e < VEC; ++e) publish(d.sum + ((p.chain * d.tiles + k) * 64 + p.lane) * VEC + e, A[e], B[e]);
      }
      look_back<VEC, NW>(d, p, known, k, carry, look, gave_up);
      if (p.wave == 0)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          start[p.lane][e] = carry[e];
          carry[e] = fmaf(A[e], carry[e], B[e]);
        }
      known = k + 1;
      if (threadIdx.x == 0) ticket[0] = after;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < VEC; ++e) h[e] = start[p.lane][e];
#pragma unroll 4
      for (int w = 0; w < p.wave; ++w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 n = part[buf][w][p.lane][e];
          h[e] = fmaf(n.x, h[e], n.y);
        }
    } else if constexpr (NW > 1) {
#pragma unroll 4
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (w == p.wave) h[e] = carry[e];
          const float2 n = part[buf][w][p.lane][e];
          carry[e] = fmaf(n.x, carry[e], n.y);
        }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) carry[e] = fmaf(A[e], carry[e], B[e]);
    }
    if (a.states != nullptr && t % SCAN_CHUNK == 0 && t < d.length && p.on)
#pragma unroll
      for (int e = 0; e < VEC; ++e) a.states[(p.b * d.chunks + t / SCAN_CHUNK) * d.channels + p.c + e] = h[e];
    if (t + FS <= len) {
#pragma unroll
      for (int s = 0; s < FS; ++s) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) h[e] = fmaf(f[s][e], h[e], b[s][e]);
        if (p.on) store_to(at<typename Raw<T, VEC>::Mem>(hp + (int64_t)(t + s) * d.h.step, p.c * sizeof(T)), Raw<T, VEC>::put(h), d.past);
      }
    } else {
#pragma unroll
      for (int s = 0; s < FS; ++s) {
        float o[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          h[e] = fmaf(f[s][e], h[e], b[s][e]);
          o[e] = t + s < len ? h[e] : 0.0f;
        }
        if (p.on && t + s < end) *at<typename Raw<T, VEC>::Mem>(hp + (int64_t)(t + s) * d.h.step, p.c * sizeof(T)) = Raw<T, VEC>::put(o);
      }
    }
    last = k == d.tiles - 1;
    tiles.cur = tiles.next;
    tiles.next = DEALT ? __builtin_amdgcn_readfirstlane(ticket[0]) : tiles.next + 1;
    buf ^= 1;
  }
  if (a.hT != nullptr && last && p.wave == 0 && p.on)
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.hT[p.b * d.channels + p.c + e] = carry[e];
}

// ---- backward -------------------------------------------------------------------------------

// Tile k of the chain is the k-th from the sequence's end.
template <typename T, int VEC, int NW, bool DEALT>
__global__ __launch_bounds__(64 * NW, NW == 8 ? 4 : 1) void scan_bwd_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  constexpr int L = NW * BS;
  static_assert(NW < 8 || L % SCAN_CHUNK == 0, "tiles start at kept states (fewer waves: one tile)");
  __shared__ float2 part[2][NW][64][VEC];
  __shared__ float back[2][NW][64][VEC];
  __shared__ float2 look[DEALT ? LOOK * 64 * VEC : 1];
  __shared__ float start[64][VEC];
  __shared__ int ticket[2];
  const Place p = place<VEC>(d);
  const int len = length_of(a.lengths, p.b, d.length), end = d.length;
  Tiles<DEALT> tiles(d, p, ticket);
  U rx[BS], rg[BS], rd[BS];
  float state[VEC], carry[VEC];
  auto load = [&](int k) {
    const int tile = d.tiles - 1 - k, t = tile * L + p.wave * BS;
    load_steps<T, VEC, BS>(rx, a.x, d.x, p.b, t, len, p.cc, U(0));
    load_steps<T, VEC, BS>(rg, a.gate, d.gate, p.b, t, len, p.cc, U(0));
    load_steps<T, VEC, BS>(rd, a.dh, d.dh, p.b, t, len, p.cc, U(0));
#pragma unroll
    for (int e = 0; e < VEC; ++e) state[e] = a.states[(p.b * d.chunks + tile * L / SCAN_CHUNK) * d.channels + p.cc + e];
  };
  if (tiles.cur < d.tiles) load(tiles.cur);
  // the gradient from behind the tile at hand; DEALT: of wave 0, from behind tile `known`
  int known = 0;
  bool gave_up = false;
  const float* first = DEALT ? d.first : a.dhT;
#pragma unroll
  for (int e = 0; e < VEC; ++e) carry[e] = first != nullptr ? first[p.b * d.channels + p.cc + e] : 0.0f;
  T* const xp = (T*)a.dx + p.b * d.dx.batch;
  T* const gp = (T*)a.dgate + p.b * d.dgate.batch;
  bool last = d.tiles == 0;
  int buf = 0;
  while (tiles.cur < d.tiles) {
    const int k = tiles.cur, t = (d.tiles - 1 - k) * L + p.wave * BS;
    const int after = tiles.request();
    float f[BS][VEC], keep[BS][VEC], x[BS][VEC], g[BS][VEC], h[VEC], c[VEC];
#pragma unroll
    for (int s = 0; s < BS; ++s) {
      float v[VEC];
      Raw<T, VEC>::get(rg[s], v);
      Raw<T, VEC>::get(rx[s], x[s]);
      Raw<T, VEC>::get(rd[s], g[s]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) gate_of<T>(v[e], f[s][e], keep[s][e]);
    }
    if (t + BS > len) {
#pragma unroll
      for (int s = 0; s < BS; ++s)
        if (t + s >= len)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            f[s][e] = 1.0f;
            keep[s][e] = x[s][e] = g[s][e] = 0.0f;
          }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) h[e] = state[e];
    if constexpr (!DEALT)
      if (tiles.next < d.tiles) load(tiles.next);
    float A[VEC], B[VEC], C[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      A[e] = 1.0f;
      B[e] = C[e] = 0.0f;
#pragma unroll
      for (int s = 0; s < BS; ++s) {
        A[e] *= f[s][e];
        B[e] = fmaf(f[s][e], B[e], keep[s][e] * x[s][e]);
        C[e] = f[BS - 1 - s][e] * (g[BS - 1 - s][e] + C[e]);
      }
      c[e] = carry[e];
    }
    if constexpr (NW > 1) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        part[buf][p.wave][p.lane][e] = make_float2(A[e], B[e]);
        back[buf][p.wave][p.lane][e] = C[e];
      }
      __syncthreads();
      // h: from the kept state through the waves before this one
#pragma unroll 4
      for (int w = 0; w < p.wave; ++w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float2 n = part[buf][w][p.lane][e];
          h[e] = fmaf(n.x, h[e], n.y);
        }
    }
    if constexpr (DEALT) {
      if (p.wave == 0) {       // as in the forward, from the right
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          A[e] = 1.0f;
          C[e] = 0.0f;
        }
#pragma unroll 4
        for (int w = NW - 1; w >= 0; --w)
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const float n = part[buf][w][p.lane][e].x;
            A[e] *= n;
            C[e] = fmaf(n, C[e], back[buf][w][p.lane][e]);
          }
#pragma unroll
        for (int e = 0; e < VEC; ++e) publish(d.sum + ((p.chain * d.tiles + k) * 64 + p.lane) * VEC + e, A[e], C[e]);
      }
      look_back<VEC, NW>(d, p, known, k, carry, look, gave_up);
      // only now: loads return in order, so the look back would wait for these (30000 steps 195 us with the forward, 184
      // so; the forward's longer tiles are better off with the loads ahead)
      if (tiles.next < d.tiles) load(tiles.next);
      if (p.wave == 0)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          start[p.lane][e] = carry[e];
          carry[e] = fmaf(A[e], carry[e], C[e]);
        }
      known = k + 1;
      if (threadIdx.x == 0) ticket[0] = after;
      __syncthreads();
#pragma unroll
      for (int e = 0; e < VEC; ++e) c[e] = start[p.lane][e];
#pragma unroll 4
      for (int w = NW - 1; w > p.wave; --w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) c[e] = fmaf(part[buf][w][p.lane][e].x, c[e], back[buf][w][p.lane][e]);
    } else if constexpr (NW > 1) {
#pragma unroll 4
      for (int w = NW - 1; w >= 0; --w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (w == p.wave) c[e] = carry[e];
          carry[e] = fmaf(part[buf][w][p.lane][e].x, carry[e], back[buf][w][p.lane][e]);
        }
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) carry[e] = fmaf(A[e], carry[e], C[e]);
    }
#pragma unroll
    for (int s = 0; s < BS; ++s)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float next = fmaf(f[s][e], h[e], keep[s][e] * x[s][e]);
        x[s][e] = h[e] - x[s][e];
        h[e] = next;
      }
    auto gradients = [&](int stop) {
#pragma unroll
      for (int s = BS - 1; s >= 0; --s) {
        float ox[VEC], og[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float G = g[s][e] + c[e];
          ox[e] = G * keep[s][e];
          og[e] = ox[e] * f[s][e] * x[s][e];
          c[e] = f[s][e] * G;
        }
        if (p.on && t + s < stop) {
          store_to(at<typename Raw<T, VEC>::Mem>(xp + (int64_t)(t + s) * d.dx.step, p.c * sizeof(T)), Raw<T, VEC>::put(ox), d.past);
          store_to(at<typename Raw<T, VEC>::Mem>(gp + (int64_t)(t + s) * d.dgate.step, p.c * sizeof(T)), Raw<T, VEC>::put(og), d.past);
        }
      }
    };
    // whole waves without a comparison a step, waves behind the end without the sums (16 x 2048 x 1024: 75.4 us where one
    // form for all took 77.1; ragged 76.0 and 78.6)
    if (t + BS <= len) {
      gradients(t + BS);
    } else {
      if (t < len) gradients(len);
      // behind the sequence's end: zeros, whatever passes through
#pragma unroll
      for (int s = 0; s < BS; ++s)
        if (p.on && t + s >= len && t + s < end) {
          const typename Raw<T, VEC>::U zero = 0;
          store_to(at<typename Raw<T, VEC>::Mem>(xp + (int64_t)(t + s) * d.dx.step, p.c * sizeof(T)), zero, d.past);
          store_to(at<typename Raw<T, VEC>::Mem>(gp + (int64_t)(t + s) * d.dgate.step, p.c * sizeof(T)), zero, d.past);
        }
    }
    last = k == d.tiles - 1;
    tiles.cur = tiles.next;
    tiles.next = DEALT ? __builtin_amdgcn_readfirstlane(ticket[0]) : tiles.next + 1;
    buf ^= 1;
  }
  if (a.dh0 != nullptr && last && p.wave == 0 && p.on)
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.dh0[p.b * d.channels + p.c + e] = carry[e];
}

Dims dims(const pnn_scan_desc& d, const ScanArgs& a, int vec, int tile) {
  Dims m;
  m.length = (int)d.length;
  m.channels = (int)d.channels;
  m.groups = (int)cdiv64(d.channels, 64 * vec);
  m.chunks = (int)scan_chunks(d);
  m.tiles = (int)cdiv64(d.length, tile);
  m.chains = d.batch * m.groups;
  m.dealt = scan_dealt(m.chains, m.tiles);
  m.past = d.batch * d.length * d.channels * (d.dtype == PNN_F32 ? 4 : 2) > L2_BYTES;
  m.x = d.x;
  m.gate = d.gate;
  m.h = d.h;
  m.dh = d.dh;
  m.dx = d.dx;
  m.dgate = d.dgate;
  const ScanWs w = scan_ws(d.batch * d.channels, m.chains, m.tiles, vec);
  m.tickets = (unsigned*)((char*)a.ws + w.tickets);
  m.first = (float*)((char*)a.ws + w.first);
  m.sum = (float2*)((char*)a.ws + w.sum);
  return m;
}

void begin(const Dims& m, const float* from, int64_t states, int vec, hipStream_t s) {
  const int64_t pairs = m.chains * m.tiles * 64 * vec, n = pairs > states ? pairs : states;
  const int64_t grid = cdiv64(n, 1024) < 4096 ? cdiv64(n, 1024) : 4096;
  hipLaunchKernelGGL(scan_begin_kernel, dim3((unsigned)grid), dim3(256), 0, s, m, from, states, pairs);
}

}  // namespace

int launch_scan_fwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s) {
  const bool pair = scan_pairs(d, false);
  const int nw = scan_waves(d.batch * cdiv64(d.channels, pair ? 128 : 64), d.length, FS);
#define FWD(T, VEC, NW)                                                                                             \
  do {                                                                                                              \
    const Dims m = dims(d, a, VEC, NW * FS);                                                                        \
    const dim3 grid((unsigned)(m.chains * m.dealt)), block(64 * NW);                                                \
    if constexpr (NW == SCAN_NW) /* fewer waves: a single tile, or enough sequences */                              \
      if (m.dealt > 1) {                                                                                            \
        begin(m, a.h0, d.batch * d.channels, VEC, s);                                                               \
        hipLaunchKernelGGL((scan_fwd_kernel<T, VEC, NW, true>), grid, block, 0, s, m, a);                           \
        break;                                                                                                      \
      }                                                                                                             \
    hipLaunchKernelGGL((scan_fwd_kernel<T, VEC, NW, false>), grid, block, 0, s, m, a);                              \
  } while (0)
#define FWD_NW(T, VEC)                \
  do {                                \
    if (nw == 1) FWD(T, VEC, 1);      \
    else if (nw == 4) FWD(T, VEC, 4); \
    else if (nw == 8) FWD(T, VEC, 8); \
    else FWD(T, VEC, SCAN_NW);             \
  } while (0)
  if (d.dtype == PNN_F32) FWD_NW(float, 1);
  else if (pair) FWD_NW(uint16_t, 2);
  else FWD_NW(uint16_t, 1);
#undef FWD_NW
#undef FWD
  return (int)hipGetLastError();
}

int launch_scan_bwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s) {
  const bool pair = scan_pairs(d, true);
  const int nw = scan_waves(d.batch * cdiv64(d.channels, pair ? 128 : 64), d.length, BS);
#define BWD(T, VEC, NW)                                                                                             \
  do {                                                                                                              \
    const Dims m = dims(d, a, VEC, NW * BS);                                                                        \
    const dim3 grid((unsigned)(m.chains * m.dealt)), block(64 * NW);                                                \
    if constexpr (NW == SCAN_NW && VEC == 1) /* pairs: enough sequences */                                          \
      if (m.dealt > 1) {                                                                                            \
        begin(m, a.dhT, d.batch * d.channels, VEC, s);                                                               \
        hipLaunchKernelGGL((scan_bwd_kernel<T, VEC, NW, true>), grid, block, 0, s, m, a);                           \
        break;                                                                                                      \
      }                                                                                                             \
    hipLaunchKernelGGL((scan_bwd_kernel<T, VEC, NW, false>), grid, block, 0, s, m, a);                              \
  } while (0)
#define BWD_NW(T, VEC)                \
  do {                                \
    if (nw == 1) BWD(T, VEC, 1);      \
    else if (nw == 4) BWD(T, VEC, 4); \
    else if (nw == 8) BWD(T, VEC, 8); \
    else BWD(T, VEC, SCAN_NW);             \
  } while (0)
  if (d.dtype == PNN_F32) BWD_NW(float, 1);
  else if (pair) BWD_NW(uint16_t, 2);
  else BWD_NW(uint16_t, 1);
#undef BWD_NW
#undef BWD
  return (int)hipGetLastError();
}

}  // namespace pnn

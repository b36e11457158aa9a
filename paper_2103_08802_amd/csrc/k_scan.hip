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
// Few channels do not fill the device with workgroups: the sequence is then split into ranges of
// tiles (scan_ranges), whose (A, B) a first launch sums up; each range's workgroup composes those of
// the ranges before (backward: behind) it, in order.  That launch reads x and gate (backward: gate
// and dh) a second time.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int FS = SCAN_FS, BS = SCAN_BS;

struct Dims {
  int length, channels, groups, chunks;
  int past;                 // results larger than the L2 caches (store_to)
  int ranges, range_tiles;  // ranges of the sequence and their tiles
  pnn_seq_stride x, gate, h, dh, dx, dgate;
  float *first;             // [batch][channels]: the state before the first (backward: gradient after the last) step
  float2 *sum;              // [batch][ranges][channels]: (A, B) of a range
};

// f = sigmoid(g) and keep = 1 - f = exp(-g) f, each to about an ulp (keep is not formed by subtraction).
// g is held between -87 and 100, where both are constant to the last bit and exp(-g) is finite, by
// minimum and maximum that keep NaN.  exp(-g) = 2^t (1 + d): t = -g log2(e) rounded, d the rest of that
// product to first order.  A bf16 g has 8 bits, so its product with the leading 16 bits of log2(e) is
// exact; for float the rounding is recovered by a fused multiply-add, and the reciprocal is refined.
template <typename T>
__device__ __forceinline__ void gate_of(float g, float& f, float& keep) {
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
  f = r;
  keep = e * r;
}

// VEC neighbouring channels of T as they are in memory
template <typename T, int VEC> struct Raw;
template <> struct Raw<uint16_t, 1> {
  typedef uint16_t U;
  __device__ static __forceinline__ void get(U u, float* v) { v[0] = bf2f(u); }
  __device__ static __forceinline__ U put(const float* v) { return f2bf(v[0]); }
};
template <> struct Raw<uint16_t, 2> {
  typedef uint32_t U;
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
  __device__ static __forceinline__ void get(U u, float* v) { v[0] = u; }
  __device__ static __forceinline__ U put(const float* v) { return v[0]; }
};

// Steps t0 .. t0 + S - 1 of one channel group, the ones from `end` on as `none`.  t0 and end are the
// same for all lanes.
template <typename T, int VEC, int S>
__device__ __forceinline__ void load_steps(typename Raw<T, VEC>::U (&r)[S], const void* base, const pnn_seq_stride& st,
                                           int64_t b, int t0, int end, int c, typename Raw<T, VEC>::U none) {
  typedef typename Raw<T, VEC>::U U;
  const T* p = (const T*)base + (b * st.batch + (int64_t)t0 * st.step);
  if (t0 + S <= end) {
#pragma unroll
    for (int s = 0; s < S; ++s) r[s] = *at<const U>(p + s * st.step, c * sizeof(T));
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s) r[s] = t0 + s < end ? *at<const U>(p + s * st.step, c * sizeof(T)) : none;
  }
}

__device__ __forceinline__ int length_of(const int32_t* lengths, int64_t b, int length) {
  if (lengths == nullptr) return length;
  const int n = lengths[b];
  return n < 0 ? 0 : n > length ? length : n;
}

// The workgroup's place: channel group fastest, then range, then sequence
struct Place {
  int group, range, wave, lane, c, cc;
  int64_t b;
  bool on;
};
template <int VEC>
__device__ __forceinline__ Place place(const Dims& d, int ranges) {
  Place p;
  const int64_t i = blockIdx.x;
  p.group = (int)(i % d.groups);
  p.range = (int)(i / d.groups % ranges);
  p.b = i / ((int64_t)d.groups * ranges);
  p.lane = threadIdx.x & 63;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.c = (p.group * 64 + p.lane) * VEC;
  p.on = p.c < d.channels;
  p.cc = p.on ? p.c : d.channels - VEC;    // lanes past the end load what the last one does
  return p;
}

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

// (A, B) of every range but the last; each wave takes a contiguous part of the range
template <typename T, int VEC, int NW>
__global__ __launch_bounds__(64 * NW) void scan_fwd_sum_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  __shared__ float2 part[NW][64][VEC];
  const Place p = place<VEC>(d, d.ranges - 1);
  const int len = length_of(a.lengths, p.b, d.length);
  const int t0 = p.range * d.range_tiles * (NW * FS) + p.wave * d.range_tiles * FS;
  const int t1 = t0 + d.range_tiles * FS;
  float A[VEC], B[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    A[e] = 1.0f;
    B[e] = 0.0f;
  }
  // two register sets of 8 steps: one is loaded while the other is summed
  U rx[2][8], rg[2][8];
  auto load = [&](int k, int t) {
    load_steps<T, VEC, 8>(rx[k], a.x, d.x, p.b, t, len, p.cc, U(0));
    load_steps<T, VEC, 8>(rg[k], a.gate, d.gate, p.b, t, len, p.cc, U(0));
  };
  auto add = [&](int k, int t) {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      float x[VEC], g[VEC];
      Raw<T, VEC>::get(rx[k][s], x);
      Raw<T, VEC>::get(rg[k][s], g);
      if (t + s < len)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          float f, keep;
          gate_of<T>(g[e], f, keep);
          A[e] *= f;
          B[e] = fmaf(f, B[e], keep * x[e]);
        }
    }
  };
  static_assert(FS == 16, "two sets a tile");
  load(0, t0);
  for (int t = t0; t < t1 && t < len; t += FS) {
    load(1, t + 8);
    add(0, t);
    if (t + FS < t1) load(0, t + FS);
    add(1, t + 8);
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[p.wave][p.lane][e] = make_float2(A[e], B[e]);
  __syncthreads();
  if (p.wave != 0 || !p.on) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    for (int w = 1; w < NW; ++w) {
      const float2 n = part[w][p.lane][e];
      A[e] *= n.x;
      B[e] = fmaf(n.x, B[e], n.y);
    }
    d.sum[(p.b * d.ranges + p.range) * d.channels + p.c + e] = make_float2(A[e], B[e]);
    if (p.range == 0) d.first[p.b * d.channels + p.c + e] = a.h0 != nullptr ? a.h0[p.b * d.channels + p.c + e] : 0.0f;
  }
}

template <typename T, int VEC, int NW>
__global__ __launch_bounds__(64 * NW) void scan_fwd_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  constexpr int L = NW * FS;
  __shared__ float2 part[2][NW][64][VEC];
  const Place p = place<VEC>(d, d.ranges);
  const int len = length_of(a.lengths, p.b, d.length);
  const int r0 = p.range * d.range_tiles * L;
  const int r1 = r0 + d.range_tiles * L < d.length ? r0 + d.range_tiles * L : d.length;
  U rx[FS], rg[FS];
  load_steps<T, VEC, FS>(rx, a.x, d.x, p.b, r0 + p.wave * FS, len, p.cc, U(0));
  load_steps<T, VEC, FS>(rg, a.gate, d.gate, p.b, r0 + p.wave * FS, len, p.cc, U(0));
  float carry[VEC];
  const float* first = d.ranges > 1 ? d.first : a.h0;
#pragma unroll
  for (int e = 0; e < VEC; ++e) carry[e] = first != nullptr ? first[p.b * d.channels + p.cc + e] : 0.0f;
#pragma unroll 8
  for (int r = 0; r < p.range; ++r)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float2 n = d.sum[(p.b * d.ranges + r) * d.channels + p.cc + e];
      carry[e] = fmaf(n.x, carry[e], n.y);
    }
  T* const hp = (T*)a.h + p.b * d.h.batch;
  int buf = 0;
  for (int tile = r0; tile < r1; tile += L, buf ^= 1) {
    const int t = tile + p.wave * FS;
    float f[FS][VEC], b[FS][VEC], A[VEC], B[VEC], h[VEC];
    gates<T, VEC, FS>(rx, rg, t, len, f, b);
    if (tile + L < r1) {
      load_steps<T, VEC, FS>(rx, a.x, d.x, p.b, t + L, len, p.cc, U(0));
      load_steps<T, VEC, FS>(rg, a.gate, d.gate, p.b, t + L, len, p.cc, U(0));
    }
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
        if (p.on) store_to(at<U>(hp + (int64_t)(t + s) * d.h.step, p.c * sizeof(T)), Raw<T, VEC>::put(h), d.past);
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
        if (p.on && t + s < r1) *at<U>(hp + (int64_t)(t + s) * d.h.step, p.c * sizeof(T)) = Raw<T, VEC>::put(o);
      }
    }
  }
  if (a.hT != nullptr && p.range == d.ranges - 1 && p.wave == 0 && p.on)
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.hT[p.b * d.channels + p.c + e] = carry[e];
}

// ---- backward -------------------------------------------------------------------------------

// (A, B) of every range but the first, for the chain from the right: c -> A c + B
template <typename T, int VEC, int NW>
__global__ __launch_bounds__(64 * NW) void scan_bwd_sum_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  __shared__ float2 part[NW][64][VEC];
  const Place p = place<VEC>(d, d.ranges - 1);
  const int range = p.range + 1;
  const int len = length_of(a.lengths, p.b, d.length);
  const int t0 = range * d.range_tiles * (NW * BS) + p.wave * d.range_tiles * BS;
  const int t1 = t0 + d.range_tiles * BS;
  float A[VEC], B[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    A[e] = 1.0f;
    B[e] = 0.0f;
  }
  U rg[BS], rd[BS];
  load_steps<T, VEC, BS>(rg, a.gate, d.gate, p.b, t1 - BS, len, p.cc, U(0));
  load_steps<T, VEC, BS>(rd, a.dh, d.dh, p.b, t1 - BS, len, p.cc, U(0));
  for (int t = t1 - BS; t >= t0; t -= BS) {
    float f[BS][VEC], g[BS][VEC];
#pragma unroll
    for (int s = 0; s < BS; ++s) {
      float v[VEC], keep;
      Raw<T, VEC>::get(rg[s], v);
      Raw<T, VEC>::get(rd[s], g[s]);
#pragma unroll
      for (int e = 0; e < VEC; ++e) gate_of<T>(v[e], f[s][e], keep);
    }
    if (t > t0) {
      load_steps<T, VEC, BS>(rg, a.gate, d.gate, p.b, t - BS, len, p.cc, U(0));
      load_steps<T, VEC, BS>(rd, a.dh, d.dh, p.b, t - BS, len, p.cc, U(0));
    }
#pragma unroll
    for (int s = BS - 1; s >= 0; --s)
      if (t + s < len)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          A[e] *= f[s][e];
          B[e] = f[s][e] * (g[s][e] + B[e]);
        }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) part[p.wave][p.lane][e] = make_float2(A[e], B[e]);
  __syncthreads();
  if (p.wave != NW - 1 || !p.on) return;
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    for (int w = NW - 2; w >= 0; --w) {
      const float2 n = part[w][p.lane][e];
      A[e] *= n.x;
      B[e] = fmaf(n.x, B[e], n.y);
    }
    d.sum[(p.b * d.ranges + range) * d.channels + p.c + e] = make_float2(A[e], B[e]);
    if (range == d.ranges - 1)
      d.first[p.b * d.channels + p.c + e] = a.dhT != nullptr ? a.dhT[p.b * d.channels + p.c + e] : 0.0f;
  }
}

template <typename T, int VEC, int NW>
__global__ __launch_bounds__(64 * NW) void scan_bwd_kernel(Dims d, ScanArgs a) {
  typedef typename Raw<T, VEC>::U U;
  constexpr int L = NW * BS;
  static_assert(NW < SCAN_NW || L == SCAN_CHUNK, "tiles start at kept states (fewer waves: one tile)");
  __shared__ float2 part[2][NW][64][VEC];
  __shared__ float back[2][NW][64][VEC];
  const Place p = place<VEC>(d, d.ranges);
  const int len = length_of(a.lengths, p.b, d.length);
  const int r0 = p.range * d.range_tiles * L;
  const int r1 = r0 + d.range_tiles * L < d.length ? r0 + d.range_tiles * L : d.length;
  const int last = r1 > r0 ? r0 + (r1 - r0 - 1) / L * L : r0 - L;   // no step: no tile
  U rx[BS], rg[BS], rd[BS];
  float state[VEC], carry[VEC];
  auto load = [&](int tile) {
    const int t = tile + p.wave * BS;
    load_steps<T, VEC, BS>(rx, a.x, d.x, p.b, t, len, p.cc, U(0));
    load_steps<T, VEC, BS>(rg, a.gate, d.gate, p.b, t, len, p.cc, U(0));
    load_steps<T, VEC, BS>(rd, a.dh, d.dh, p.b, t, len, p.cc, U(0));
#pragma unroll
    for (int e = 0; e < VEC; ++e) state[e] = a.states[(p.b * d.chunks + tile / SCAN_CHUNK) * d.channels + p.cc + e];
  };
  if (last >= r0) load(last);
  const float* first = d.ranges > 1 ? d.first : a.dhT;
#pragma unroll
  for (int e = 0; e < VEC; ++e) carry[e] = first != nullptr ? first[p.b * d.channels + p.cc + e] : 0.0f;
#pragma unroll 8
  for (int r = d.ranges - 1; r > p.range; --r)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float2 n = d.sum[(p.b * d.ranges + r) * d.channels + p.cc + e];
      carry[e] = fmaf(n.x, carry[e], n.y);
    }
  T* const xp = (T*)a.dx + p.b * d.dx.batch;
  T* const gp = (T*)a.dgate + p.b * d.dgate.batch;
  int buf = 0;
  for (int tile = last; tile >= r0; tile -= L, buf ^= 1) {
    const int t = tile + p.wave * BS;
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
    if (tile > r0) load(tile - L);
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
      float first_h[VEC];
#pragma unroll
      for (int e = 0; e < VEC; ++e) first_h[e] = h[e];
#pragma unroll 4
      for (int w = 0; w < NW; ++w)
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          if (w == p.wave) h[e] = first_h[e];
          const float2 n = part[buf][w][p.lane][e];
          first_h[e] = fmaf(n.x, first_h[e], n.y);
        }
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
      if (p.on && t + s < r1) {
        store_to(at<U>(xp + (int64_t)(t + s) * d.dx.step, p.c * sizeof(T)), Raw<T, VEC>::put(ox), d.past);
        store_to(at<U>(gp + (int64_t)(t + s) * d.dgate.step, p.c * sizeof(T)), Raw<T, VEC>::put(og), d.past);
      }
    }
  }
  if (a.dh0 != nullptr && p.range == 0 && p.wave == 0 && p.on)
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.dh0[p.b * d.channels + p.c + e] = carry[e];
}

bool even(const pnn_seq_stride& s) { return s.batch % 2 == 0 && s.step % 2 == 0; }
bool al4(const void* p) { return ((uintptr_t)p & 3) == 0; }

Dims dims(const pnn_scan_desc& d, const ScanArgs& a, int vec, int tile) {
  Dims m;
  m.length = (int)d.length;
  m.channels = (int)d.channels;
  m.groups = (int)cdiv64(d.channels, 64 * vec);
  m.chunks = (int)scan_chunks(d);
  const int64_t tiles = cdiv64(d.length, tile);
  const int64_t ranges = scan_ranges(d.batch * m.groups, tiles);
  m.range_tiles = (int)cdiv64(tiles, ranges);
  if (m.range_tiles < 1) m.range_tiles = 1;
  m.ranges = (int)cdiv64(tiles, m.range_tiles);
  if (m.ranges < 1) m.ranges = 1;
  m.past = d.batch * d.length * d.channels * (d.dtype == PNN_F32 ? 4 : 2) > L2_BYTES;
  m.x = d.x;
  m.gate = d.gate;
  m.h = d.h;
  m.dh = d.dh;
  m.dx = d.dx;
  m.dgate = d.dgate;
  m.first = (float*)a.ws;
  m.sum = (float2*)((char*)a.ws + round256(d.batch * d.channels * 4));
  return m;
}

}  // namespace

int launch_scan_fwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s) {
  const int nw = d.length <= FS ? 1 : d.length <= 4 * FS ? 4 : 16;
  const bool pair = d.dtype == PNN_BF16 && d.channels % 2 == 0 && al4(a.x) && al4(a.gate) && al4(a.h) && even(d.x) &&
                    even(d.gate) && even(d.h);
#define FWD(T, VEC, NW)                                                                                             \
  do {                                                                                                              \
    const Dims m = dims(d, a, VEC, NW * FS);                                                                        \
    const int64_t n = d.batch * m.groups;                                                                           \
    if constexpr (NW == SCAN_NW) /* fewer waves: a single tile */                                                   \
      if (m.ranges > 1)                                                                                             \
        hipLaunchKernelGGL((scan_fwd_sum_kernel<T, VEC, NW>), dim3((unsigned)(n * (m.ranges - 1))), dim3(64 * NW), 0, s, m, a); \
    hipLaunchKernelGGL((scan_fwd_kernel<T, VEC, NW>), dim3((unsigned)(n * m.ranges)), dim3(64 * NW), 0, s, m, a);   \
  } while (0)
#define FWD_NW(T, VEC)                \
  do {                                \
    if (nw == 1) FWD(T, VEC, 1);      \
    else if (nw == 4) FWD(T, VEC, 4); \
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
  const int nw = d.length <= BS ? 1 : d.length <= 4 * BS ? 4 : 16;
  const bool pair = d.dtype == PNN_BF16 && d.channels % 2 == 0 && al4(a.x) && al4(a.gate) && al4(a.dh) && al4(a.dx) &&
                    al4(a.dgate) && even(d.x) && even(d.gate) && even(d.dh) && even(d.dx) && even(d.dgate);
#define BWD(T, VEC, NW)                                                                                             \
  do {                                                                                                              \
    const Dims m = dims(d, a, VEC, NW * BS);                                                                        \
    const int64_t n = d.batch * m.groups;                                                                           \
    if constexpr (NW == SCAN_NW) /* fewer waves: a single tile */                                                   \
      if (m.ranges > 1)                                                                                             \
        hipLaunchKernelGGL((scan_bwd_sum_kernel<T, VEC, NW>), dim3((unsigned)(n * (m.ranges - 1))), dim3(64 * NW), 0, s, m, a); \
    hipLaunchKernelGGL((scan_bwd_kernel<T, VEC, NW>), dim3((unsigned)(n * m.ranges)), dim3(64 * NW), 0, s, m, a);   \
  } while (0)
#define BWD_NW(T, VEC)                \
  do {                                \
    if (nw == 1) BWD(T, VEC, 1);      \
    else if (nw == 4) BWD(T, VEC, 4); \
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

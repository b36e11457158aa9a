// Linear attention with a decay for each head, and its backward:
//   S_t = lambda S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t.
//
// Chunks of C steps.  With i, j steps of a chunk of len and S the state before it,
//   o_i = scale (sum_{j <= i} lambda^(i - j) (q_i k_j) v_j + lambda^(i + 1) q_i S)
//   S  <- lambda^len S + sum_j k_j (lambda^(len - 1 - j) v_j)^T,
// four products on the matrix units.  A workgroup of four waves takes 64 ET value columns of a head through the
// chunks; a wave holds the state of its 16 ET columns in registers, in the layout that the products leave it in and
// that they take it in (rows d of a state column are the summation index of q S, so the column's registers are an
// operand as they stand, with the summation index permuted).  q k is formed once a workgroup and goes through LDS.
//
// The backward is the same sum three times:
//   dq: queries do, keys v, values k, from the transposed state;
//   dk: backwards in time, queries v, keys do, values q;   dv: backwards in time, queries k, keys q, values do,
// where a state before a step's own term weighs lambda^i instead of lambda^(i + 1) (`shift`).
//
// Few heads do not fill the device: their sequences are cut into segments, whose states from zero are formed by a
// first launch (without outputs), chained by a second, and taken as first states by the third.
//
// Roundings to bf16 besides the outputs' (bf16 tensors only): the weighted q k and the state, where they are operands
// of the products with v and q; each is as large as the output's own rounding.  The state itself is fp32, and the
// weighted values that are added to it are split into two bf16 parts (16 bits), and three (24 bits) where the caller
// wants the state.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int NT = 256;                     // threads: four waves
constexpr int AHEAD = 8;                    // state rows a lane of the single step has in flight
constexpr float LOG2E = 1.44269504f;

struct Role {
  const void *q, *k, *v;
  void* o;
  const float* s0;                          // [batch][heads][..], null: zero
  float* sT;                                // null: not wanted
  float* seg;                               // states of segments in the kernel's own layout; null: one segment
  pnn_head_stride qs, ks, vs, os;
  int64_t s_inner, s_value;                 // strides of s0 and sT
  int inner, value;                         // widths: summed over in q k, and of v
  int q_group, k_group, v_group;            // heads that share one of q, k, v
  int o_float;                              // o is fp32 whatever the type
  int shift;                                // 1: backwards in time
  float intra, inter, update;               // factors of the three sums
  int blocks, first;                        // value blocks; first workgroup of the role in the launch
};

struct Lin {
  Role role[3];
  const float* decay;
  const int32_t* lengths;
  int roles, batch, heads, length;
  int nseg, seg_chunks;                     // segments and chunks of one
};

// log2 of a head's decay; NaN for what is none
__device__ __forceinline__ float log2_decay(const float* decay, int head) {
  const float d = decay[head];
  return d <= 0.0f ? d * LOG2E : __builtin_nanf("");
}
// lambda^n, with 0^0 = 1
__device__ __forceinline__ float power(float l2, int n) {
  return n == 0 ? (l2 == l2 ? 1.0f : l2) : __builtin_amdgcn_exp2f(l2 * (float)n);
}
__device__ __forceinline__ int steps_of(const int32_t* lengths, int b, int length) {
  if (lengths == nullptr) return length;
  const int n = lengths[b];
  return n < 0 ? 0 : n < length ? n : length;
}
__device__ __forceinline__ bool lost(float v) { return !(fabsf(v) < INFINITY); }

// rows of a chunk in registers, 16 bytes a lane and row piece
template <typename T, int C, int W>
struct Stage {
  static constexpr int VE = St<T>::VE, PR = W / VE, N = C * PR / NT, LD = W + VE;   // LD: a row in LDS, 16 bytes longer
  uint4 r[N];

  // row i is step `base + i`, of n; backwards in time step n - 1 - (base + i)
  __device__ __forceinline__ void load(const T* p, int64_t step, int width, int base, int n, int shift) {
    const int col = (threadIdx.x % PR) * VE;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int i = base + threadIdx.x / PR + j * (NT / PR);
      r[j] = make_uint4(0, 0, 0, 0);
      if (i >= n || col >= width) continue;
      const T* s = p + (int64_t)(shift ? n - 1 - i : i) * step + col;
      if (col + VE <= width) {
        const typename Piece<T>::Vec u = *(const typename Piece<T>::Mem*)s;
        r[j] = __builtin_bit_cast(uint4, u);
      } else {
        T e[VE];
#pragma unroll
        for (int x = 0; x < VE; ++x) e[x] = col + x < width ? s[x] : (T)0;
        __builtin_memcpy(&r[j], e, 16);
      }
    }
  }
  __device__ __forceinline__ void store(T* lds) const {
    const int col = (threadIdx.x % PR) * VE;
#pragma unroll
    for (int j = 0; j < N; ++j) *(uint4*)(lds + (threadIdx.x / PR + j * (NT / PR)) * LD + col) = r[j];
  }
  // whether a value is infinite or NaN
  __device__ __forceinline__ bool lost() const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const uint32_t w[4] = {r[j].x, r[j].y, r[j].z, r[j].w};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if constexpr (sizeof(T) == 2) {
          m |= (w[x] & 0x7f80u) == 0x7f80u;
          m |= (w[x] & 0x7f800000u) == 0x7f800000u;
        } else {
          m |= (w[x] & 0x7f800000u) == 0x7f800000u;
        }
      }
    }
    return m != 0;
  }
};

// operand of a product from rows in LDS: the lane's row, summation index along the row
template <typename T>
__device__ __forceinline__ Frag<T> row_frag(const T* p) {
  Frag<T> f;
  f.from_raw(*(const uint4*)p);
  return f;
}
// the same with the summation index in the order of state_frag
__device__ __forceinline__ void query_frag(Frag<uint16_t>& f, const uint16_t* row, int kk, int g) {
  const uint2 a = *(const uint2*)(row + kk * 32 + 4 * g), b = *(const uint2*)(row + kk * 32 + 16 + 4 * g);
  f.from_raw(make_uint4(a.x, a.y, b.x, b.y));
}
__device__ __forceinline__ void query_frag(Frag<float>& f, const float* row, int kk, int g) {
  f.from_raw(*(const uint4*)(row + kk * 16 + 4 * g));
}
// operand from the columns of a matrix in LDS, summation index down the column: lane (i, g) takes column
// (i >> 2) spread + (i & 3) of `m` and VE rows from VE g on
__device__ __forceinline__ void column_frag(Frag<uint16_t>& f, const uint16_t* m, int ld, int i, int g, int spread) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* P;
  const uint16_t* p = m + (8 * g + (i >> 2)) * ld + (i & 3) * spread;    // a lane's address is row i >> 2, piece i & 3
  const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p));
  const uint2 b = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(p + 4 * ld)));
  f.from_raw(make_uint4(a.x, a.y, b.x, b.y));
}
__device__ __forceinline__ void column_frag(Frag<float>& f, const float* m, int ld, int i, int g, int spread) {
  const float* p = m + 4 * g * ld + (i >> 2) * spread + (i & 3);
#pragma unroll
  for (int e = 0; e < 4; ++e) f.v[e] = p[e * ld];
}
// the state's columns as an operand: summation index d = 32 kk + 4 g + (0 .. 3) and 16 more (float: 16 kk + 4 g + ..)
template <int KT, int ET>
__device__ __forceinline__ void state_frag(Frag<uint16_t>& f, const f32x4 (&S)[KT][ET], int kk, int et) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.v[e] = (__bf16)S[2 * kk][et][e];
    f.v[4 + e] = (__bf16)S[2 * kk + 1][et][e];
  }
}
template <int KT, int ET>
__device__ __forceinline__ void state_frag(Frag<float>& f, const f32x4 (&S)[KT][ET], int kk, int et) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.v[e] = S[kk][et][e];
}
// b w in three parts of 8 bits
__device__ __forceinline__ void split(const Frag<uint16_t>& b, const float* w, Frag<uint16_t> (&part)[3]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = (float)b.v[e] * w[e];
    part[0].v[e] = (__bf16)v;
    const float rest = v - (float)part[0].v[e];
    part[1].v[e] = (__bf16)rest;
    part[2].v[e] = (__bf16)(rest - (float)part[1].v[e]);
  }
}
__device__ __forceinline__ void finite_only(Frag<uint16_t>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (lost((float)f.v[e])) f.v[e] = (__bf16)0.0f;
}
__device__ __forceinline__ void finite_only(Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lost(f.v[e])) f.v[e] = 0.0f;
}

template <typename T>
__device__ __forceinline__ void put4(T* p, f32x4 v) {      // aligned
  if constexpr (sizeof(T) == 4) {
    *(f32x4*)p = v;
  } else {
    uint2 u;
    u.x = (uint32_t)f2bf(v[0]) | ((uint32_t)f2bf(v[1]) << 16);
    u.y = (uint32_t)f2bf(v[2]) | ((uint32_t)f2bf(v[3]) << 16);
    *(uint2*)p = u;
  }
}

// KD: inner width, padded; a workgroup has 64 ET value columns; OUT: outputs, not the state alone
template <typename T, int KD, int ET, int C, bool OUT>
__global__ __launch_bounds__(NT, 2) void linattn_kernel(Lin a) {
  constexpr int VE = St<T>::VE, KS = 4 * VE, KT = KD / 16, CT = C / 16, EB = 64 * ET;
  typedef Stage<T, C, KD> SK;
  typedef Stage<T, C, EB> SV;
  constexpr int LK = SK::LD, LV = SV::LD, LP = C + VE;
  __shared__ __attribute__((aligned(16))) T kt[C * LK];
  __shared__ __attribute__((aligned(16))) T vt[C * LV];
  __shared__ __attribute__((aligned(16))) T qt[OUT ? C * LK : 1];
  __shared__ __attribute__((aligned(16))) T pt[OUT ? C * LP : 1];
  __shared__ __attribute__((aligned(16))) float wt[C];
  __shared__ int bad;
  int z = 0;
  while (z + 1 < a.roles && (int)blockIdx.x >= a.role[z + 1].first) ++z;
  const Role& R = a.role[z];
  int at = blockIdx.x - R.first;
  const int block = at % R.blocks;
  at /= R.blocks;
  const int seg = at % a.nseg, bh = at / a.nseg;
  const int b = bh / a.heads, h = bh % a.heads;
  const int w = threadIdx.x / 64, lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
  const int n = steps_of(a.lengths, b, a.length);
  const float l2 = log2_decay(a.decay, h);
  const T* q = (const T*)R.q + b * R.qs.batch + (h / R.q_group) * R.qs.head;
  const T* k = (const T*)R.k + b * R.ks.batch + (h / R.k_group) * R.ks.head;
  const T* v = (const T*)R.v + b * R.vs.batch + (h / R.v_group) * R.vs.head + block * EB;
  const int e0 = block * EB + w * 16 * ET;             // the wave's first value column
  const int vwidth = R.value - block * EB;
  // state: S[dt][et][r] is row d = 16 dt + 4 g + r of column e0 + 4 ET (i >> 2) + 4 et + (i & 3)
  const int se = e0 + 4 * ET * (i >> 2) + (i & 3);
  f32x4 S[KT][ET];
  const int64_t state = (int64_t)bh * R.inner * R.value;
  float* const segment = R.seg == nullptr ? nullptr
      : R.seg + ((((int64_t)bh * a.nseg + seg) * R.blocks + block) * 4 + w) * (KT * ET * 256) + lane * 4;
#pragma unroll
  for (int dt = 0; dt < KT; ++dt)
#pragma unroll
    for (int et = 0; et < ET; ++et) {
      f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
      if (OUT && segment != nullptr) {
        s = *(const f32x4*)(segment + (dt * ET + et) * 256);
      } else if (OUT && R.s0 != nullptr) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = 16 * dt + 4 * g + r, e = se + 4 * et;
          if (d < R.inner && e < R.value) s[r] = R.s0[state + d * R.s_inner + e * R.s_value];
        }
      }
      S[dt][et] = s;
    }
  const int chunks = (a.length + C - 1) / C;
  const int c0 = seg * a.seg_chunks, c1 = c0 + a.seg_chunks < chunks ? c0 + a.seg_chunks : chunks;
  const int live = (n + C - 1) / C < c1 ? (n + C - 1) / C : c1;       // chunks with steps
  SK rq, rk;
  SV rv;
  auto load = [&](int c) {
    if (OUT) rq.load(q, R.qs.step, R.inner, c * C, n, R.shift);
    rk.load(k, R.ks.step, R.inner, c * C, n, R.shift);
    rv.load(v, R.vs.step, vwidth, c * C, n, R.shift);
  };
  if (c0 < live) load(c0);
  if (OUT) {                                    // tiles of pt above the diagonal stay zero
    for (int x = threadIdx.x; x < C * LP; x += NT) pt[x] = (T)0;
  }
  const bool exact = R.sT != nullptr;           // states that the caller sees
  int held = -1;                                // the length that wt is for
  // outputs of a chunk: row t's 4 ET values from column e on
  auto put = [&](int c, int t, f32x4 (&acc)[ET]) {
    const int gi = c * C + t;
    if (gi >= a.length) return;
    const int step = R.shift && gi < n ? n - 1 - gi : gi;
    const int e = e0 + 4 * ET * g;
    if (gi >= n) {
#pragma unroll
      for (int et = 0; et < ET; ++et) acc[et] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int64_t o = b * R.os.batch + step * R.os.step + h * R.os.head + e;
    if (R.o_float) {
#pragma unroll
      for (int x = 0; x < 4 * ET; ++x)
        if (e + x < R.value) ((float*)R.o)[o + x] = acc[x / 4][x % 4];
      return;
    }
    constexpr int PC = 4 * ET;
    if (e + PC <= R.value) {
      typedef T V __attribute__((ext_vector_type(PC)));
      typedef V VM __attribute__((aligned(sizeof(T))));
      V u;
#pragma unroll
      for (int x = 0; x < PC; ++x) {
        if constexpr (sizeof(T) == 4) u[x] = acc[x / 4][x % 4];
        else u[x] = f2bf(acc[x / 4][x % 4]);
      }
      *(VM*)((T*)R.o + o) = u;
    } else {
#pragma unroll
      for (int x = 0; x < PC; ++x)
        if (e + x < R.value) St<T>::st(R.o, o + x, acc[x / 4][x % 4]);
    }
  };
  for (int c = c0; c < live; ++c) {
    const int len = n - c * C < C ? n - c * C : C;
    __syncthreads();                            // the chunk before is done with LDS
    if (threadIdx.x == 0) bad = 0;
    if (OUT) rq.store(qt);
    rk.store(kt);
    rv.store(vt);
    if (held != len) {
      held = len;
      for (int x = threadIdx.x; x < C; x += NT) wt[x] = x < len ? R.update * power(l2, len - 1 - x + R.shift) : 0.0f;
    }
    const bool odd = OUT && rv.lost();
    __syncthreads();
    if (odd) bad = 1;
    if (c + 1 < live) load(c + 1);
    if constexpr (OUT) {
      // pt[t][s] = intra lambda^(t - s) q_t k_s for s <= t; tiles dealt to the waves
      for (int tile = w; tile < CT * CT; tile += 4) {
        const int ti = CT == 4 ? w : tile / CT, si = CT == 4 ? tile / 4 : tile % CT;
        if (si > ti) continue;
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < KD / KS; ++kk)
          mma(row_frag(kt + (si * 16 + i) * LK + kk * KS + g * VE), row_frag(qt + (ti * 16 + i) * LK + kk * KS + g * VE),
              acc);
        const int t = ti * 16 + i;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int apart = t - (si * 16 + 4 * g + r);
          acc[r] = apart >= 0 ? acc[r] * (R.intra * power(l2, apart < 0 ? 0 : apart)) : 0.0f;
        }
        put4(pt + t * LP + si * 16 + 4 * g, acc);
      }
      __syncthreads();
    }
    const bool some = OUT && bad != 0;
    Frag<T> vf[C / KS][ET];
#pragma unroll
    for (int kb = 0; kb < C / KS; ++kb)
#pragma unroll
      for (int et = 0; et < ET; ++et)
        column_frag(vf[kb][et], vt + kb * KS * LV + w * 16 * ET + 4 * et, LV, i, g, 4 * ET);
    if constexpr (OUT) {
      Frag<T> sf[KD / KS][ET];
#pragma unroll
      for (int kk = 0; kk < KD / KS; ++kk)
#pragma unroll
        for (int et = 0; et < ET; ++et) state_frag(sf[kk][et], S, kk, et);
#pragma unroll
      for (int ti = 0; ti < CT; ++ti) {
        const int t = ti * 16 + i;
        f32x4 acc[ET];
#pragma unroll
        for (int et = 0; et < ET; ++et) acc[et] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int kk = 0; kk < KD / KS; ++kk) {
          Frag<T> qf;
          query_frag(qf, qt + t * LK, kk, g);
#pragma unroll
          for (int et = 0; et < ET; ++et) mma(sf[kk][et], qf, acc[et]);
        }
        const float from = R.inter * power(l2, t + 1 - R.shift);
#pragma unroll
        for (int et = 0; et < ET; ++et) acc[et] *= from;
#pragma unroll
        for (int kb = 0; kb < C / KS; ++kb) {
          if (kb * KS >= 16 * (ti + 1)) continue;
          const Frag<T> pf = row_frag(pt + t * LP + kb * KS + g * VE);
#pragma unroll
          for (int et = 0; et < ET; ++et) {
            Frag<T> vv = vf[kb][et];
            if (some) finite_only(vv);
            mma(vv, pf, acc[et]);
          }
        }
        if (some) {
          // an infinite or NaN value reaches the steps from its own on, which a product with the zeros above the
          // diagonal does not keep to: such values one by one
          for (int s = 0; s <= t; ++s) {
            const float p = St<T>::ld(pt, t * LP + s);
#pragma unroll
            for (int x = 0; x < 4 * ET; ++x) {
              const float val = St<T>::ld(vt, s * LV + w * 16 * ET + 4 * ET * g + x);
              if (lost(val)) acc[x / 4][x % 4] += p * val;
            }
          }
        }
        put(c, t, acc);
      }
    }
    // the state after the chunk
    const float gone = power(l2, len);
#pragma unroll
    for (int dt = 0; dt < KT; ++dt)
#pragma unroll
      for (int et = 0; et < ET; ++et) S[dt][et] *= gone;
#pragma unroll
    for (int kb = 0; kb < C / KS; ++kb) {
      if constexpr (sizeof(T) == 2) {
        Frag<T> part[ET][3];
        float ws[VE];
        *(f32x4*)ws = *(const f32x4*)&wt[kb * KS + g * VE];
        *(f32x4*)(ws + 4) = *(const f32x4*)&wt[kb * KS + g * VE + 4];
#pragma unroll
        for (int et = 0; et < ET; ++et) split(vf[kb][et], ws, part[et]);
#pragma unroll
        for (int dt = 0; dt < KT; ++dt) {
          Frag<T> kf;
          column_frag(kf, kt + kb * KS * LK + dt * 16, LK, i, g, 4);
#pragma unroll
          for (int et = 0; et < ET; ++et) {
            if (exact) mma(kf, part[et][2], S[dt][et]);
            mma(kf, part[et][1], S[dt][et]);
            mma(kf, part[et][0], S[dt][et]);
          }
        }
      } else {
        const f32x4 ws = *(const f32x4*)&wt[kb * KS + g * VE];
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
          for (int e = 0; e < 4; ++e) vf[kb][et].v[e] *= ws[e];
#pragma unroll
        for (int dt = 0; dt < KT; ++dt) {
          Frag<T> kf;
          column_frag(kf, kt + kb * KS * LK + dt * 16, LK, i, g, 4);
#pragma unroll
          for (int et = 0; et < ET; ++et) mma(kf, vf[kb][et], S[dt][et]);
        }
      }
    }
  }
  if constexpr (OUT) {
    for (int c = c0 < live ? live : c0; c < c1; ++c) {              // chunks behind the sequence's end
      for (int t = i; t < C; t += 16) {
        f32x4 none[ET] = {};
        put(c, t, none);
      }
    }
    if (R.sT != nullptr && seg == a.nseg - 1) {
#pragma unroll
      for (int dt = 0; dt < KT; ++dt)
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int d = 16 * dt + 4 * g + r, e = se + 4 * et;
            if (d < R.inner && e < R.value) R.sT[state + d * R.s_inner + e * R.s_value] = S[dt][et][r];
          }
    }
  } else {
#pragma unroll
    for (int dt = 0; dt < KT; ++dt)
#pragma unroll
      for (int et = 0; et < ET; ++et) *(f32x4*)(segment + (dt * ET + et) * 256) = S[dt][et];
  }
}

// The segments' states from zero become their first states: a thread takes one piece of four through the segments.
template <int KD, int ET, int C>
__global__ __launch_bounds__(NT) void linattn_chain_kernel(Lin a) {
  constexpr int KT = KD / 16;
  const Role& R = a.role[blockIdx.y];
  const int64_t pieces = (int64_t)R.blocks * 4 * KT * ET * 64;
  const int per = (int)(pieces / NT);                         // workgroups of a head
  const int bh = blockIdx.x / per;
  if (bh >= a.batch * a.heads) return;                        // a role with fewer blocks
  const int x = (blockIdx.x % per) * NT + threadIdx.x;
  const int lane = x % 64, et = x / 64 % ET, dt = x / 64 / ET % KT, wave = x / 64 / ET / KT;   // wave of all blocks
  const int i = lane & 15, g = lane >> 4;
  const int d = 16 * dt + 4 * g, e = wave * 16 * ET + 4 * ET * (i >> 2) + 4 * et + (i & 3);
  f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  if (R.s0 != nullptr) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (d + r < R.inner && e < R.value)
        s[r] = R.s0[(int64_t)bh * R.inner * R.value + (d + r) * R.s_inner + e * R.s_value];
  }
  const int b = bh / a.heads, n = steps_of(a.lengths, b, a.length);
  const float l2 = log2_decay(a.decay, bh % a.heads);
  f32x4* p = (f32x4*)R.seg + (int64_t)bh * a.nseg * pieces + x;
  for (int j = 0; j < a.nseg; ++j) {
    f32x4 u = {0.0f, 0.0f, 0.0f, 0.0f};
    if (j + 1 < a.nseg) u = p[j * pieces];
    p[j * pieces] = s;
    const int64_t from = (int64_t)j * a.seg_chunks * C, steps = n - from;
    const int64_t most = (int64_t)a.seg_chunks * C;
    const int len = steps < 0 ? 0 : steps < most ? (int)steps : (int)most;
    s = s * power(l2, len) + u;
  }
}

// One step of every sequence: a workgroup takes 4 VW .. of the value columns of a head, VW a lane, its rows dealt to
// the groups of `lanes` lanes.
template <typename T, int VW>
__global__ __launch_bounds__(NT) void linattn_step_kernel(Lin a, int lanes) {
  __shared__ float part[NT * VW];
  const Role& R = a.role[0];
  const int block = blockIdx.x % R.blocks, bh = blockIdx.x / R.blocks;
  const int b = bh / a.heads, h = bh % a.heads;
  const bool live = steps_of(a.lengths, b, 1) > 0;
  const int groups = NT / lanes, lane = threadIdx.x % lanes, group = threadIdx.x / lanes;
  const int e = (block * lanes + lane) * VW;
  const float l2 = log2_decay(a.decay, h), lam = power(l2, 1);
  const int64_t q = b * R.qs.batch + (h / R.q_group) * R.qs.head, k = b * R.ks.batch + (h / R.k_group) * R.ks.head;
  const int64_t v = b * R.vs.batch + (h / R.v_group) * R.vs.head;
  const int64_t state = (int64_t)bh * R.inner * R.value;
  typedef float V __attribute__((ext_vector_type(VW)));
  typedef V VM __attribute__((aligned(4)));
  float ve[VW], o[VW];
#pragma unroll
  for (int x = 0; x < VW; ++x) {
    ve[x] = live && e < R.value ? St<T>::ld(R.v, v + e + x) : 0.0f;
    o[x] = 0.0f;
  }
  if (e < R.value) {
    for (int d0 = group; d0 < R.inner; d0 += AHEAD * groups) {
      V s[AHEAD];                               // rows in flight; the stores below may go to the same place
      float kd[AHEAD], qd[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int d = d0 + j * groups;
        const bool on = d < R.inner;
#pragma unroll
        for (int x = 0; x < VW; ++x) s[j][x] = 0.0f;
        if (on && R.s0 != nullptr) s[j] = *(const VM*)(R.s0 + (state + (int64_t)d * R.value + e));
        kd[j] = on && live ? St<T>::ld(R.k, k + d) : 0.0f;
        qd[j] = on && live ? St<T>::ld(R.q, q + d) : 0.0f;
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        const int d = d0 + j * groups;
        if (d >= R.inner) break;
        if (live) {
#pragma unroll
          for (int x = 0; x < VW; ++x) {
            s[j][x] = fmaf(lam, s[j][x], kd[j] * ve[x]);
            o[x] = fmaf(qd[j], s[j][x], o[x]);
          }
        }
        if (R.sT != nullptr) *(VM*)(R.sT + (state + (int64_t)d * R.value + e)) = s[j];
      }
    }
  }
#pragma unroll
  for (int x = 0; x < VW; ++x) part[threadIdx.x * VW + x] = o[x];
  __syncthreads();
  if (group != 0 || e >= R.value) return;
  for (int j = 1; j < groups; ++j)
#pragma unroll
    for (int x = 0; x < VW; ++x) o[x] += part[(j * lanes + lane) * VW + x];
#pragma unroll
  for (int x = 0; x < VW; ++x)
    St<T>::st(R.o, b * R.os.batch + h * R.os.head + e + x, live ? o[x] * R.inter : 0.0f);
}

// gradients of keys and values that heads share: out = the heads' sum, in their order
template <typename T>
__global__ __launch_bounds__(NT) void linattn_heads_kernel(const float* part, void* out, pnn_head_stride st, int64_t rows,
                                                           int length, int kv, int group, int width) {
  const int64_t x = (int64_t)blockIdx.x * NT + threadIdx.x;
  const int e = (int)(x % width);
  const int64_t r = x / width;                            // (batch, step, shared head)
  if (r >= rows) return;
  float s = 0.0f;
  for (int j = 0; j < group; ++j) s += part[(r * group + j) * width + e];
  const int64_t bt = r / kv;
  St<T>::st(out, bt / length * st.batch + bt % length * st.step + r % kv * st.head + e, s);
}

template <typename T, int KD, int ET>
int launch_roles(Lin& a, hipStream_t s) {
  constexpr int C = lin_chunk(sizeof(T), KD);
  int64_t grid = 0;
  int most = 0;
  for (int z = 0; z < a.roles; ++z) {
    Role& R = a.role[z];
    R.first = (int)grid;
    grid += (int64_t)a.batch * a.heads * a.nseg * R.blocks;
    if (R.blocks > most) most = R.blocks;
  }
  if (a.nseg > 1) {
    hipLaunchKernelGGL((linattn_kernel<T, KD, ET, C, false>), dim3((unsigned)grid), dim3(NT), 0, s, a);
    const unsigned per = (unsigned)(most * KD / 16 * ET);     // 4 KT ET 64 / NT a block
    hipLaunchKernelGGL((linattn_chain_kernel<KD, ET, C>), dim3(per * a.batch * a.heads, a.roles), dim3(NT), 0, s, a);
  }
  hipLaunchKernelGGL((linattn_kernel<T, KD, ET, C, true>), dim3((unsigned)grid), dim3(NT), 0, s, a);
  return (int)hipGetLastError();
}

template <typename T>
int launch_shape(Lin& a, const LinShape& p, hipStream_t s) {
  if (p.pad == 64) return p.tiles == 1 ? launch_roles<T, 64, 1>(a, s) : launch_roles<T, 64, 2>(a, s);
  if (p.pad == 128) return p.tiles == 1 ? launch_roles<T, 128, 1>(a, s) : launch_roles<T, 128, 2>(a, s);
  return launch_roles<T, 256, 1>(a, s);
}

int launch_any(int dtype, Lin& a, const LinShape& p, hipStream_t s) {
  a.nseg = p.segments;
  a.seg_chunks = p.seg_chunks;
  return dtype == PNN_F32 ? launch_shape<float>(a, p, s) : launch_shape<uint16_t>(a, p, s);
}

Lin common(const pnn_linattn_desc& d, const float* decay, const int32_t* lengths) {
  Lin a = {};
  a.decay = decay;
  a.lengths = lengths;
  a.batch = (int)d.batch;
  a.heads = (int)d.heads;
  a.length = (int)d.length;
  a.nseg = 1;
  return a;
}

}  // namespace

int launch_linattn_fwd(const pnn_linattn_desc& d, const void* q, const void* k, const void* v, const float* decay,
                       const int32_t* lengths, const float* s0, void* o, float* sT, void* ws, hipStream_t s) {
  Lin a = common(d, decay, lengths);
  const int group = (int)(d.heads / d.kv_heads);
  Role& R = a.role[0];
  a.roles = 1;
  R.q = q, R.k = k, R.v = v, R.o = o;
  R.qs = d.q, R.ks = d.k, R.vs = d.v, R.os = d.o;
  R.q_group = 1, R.k_group = R.v_group = group;
  R.s0 = s0, R.sT = sT;
  R.s_inner = d.value_width, R.s_value = 1;
  R.inner = (int)d.key_width, R.value = (int)d.value_width;
  R.intra = R.inter = d.scale, R.update = 1.0f;
  if (d.length == 1) {
    const int vw = R.value % 4 == 0 ? 4 : 1;
    int lanes = 1;
    while (lanes < 32 && lanes * vw < R.value) lanes *= 2;
    R.blocks = (int)cdiv64(R.value, lanes * vw);
    const dim3 grid((unsigned)(d.batch * d.heads * R.blocks));
#define STEP(T, VW) hipLaunchKernelGGL((linattn_step_kernel<T, VW>), grid, dim3(NT), 0, s, a, lanes)
    if (d.dtype == PNN_F32) { if (vw == 4) STEP(float, 4); else STEP(float, 1); }
    else { if (vw == 4) STEP(uint16_t, 4); else STEP(uint16_t, 1); }
#undef STEP
    return (int)hipGetLastError();
  }
  const LinShape p = lin_shape(d, d.key_width, d.value_width, 1);
  R.blocks = p.blocks;
  R.seg = p.segments > 1 ? (float*)ws : nullptr;
  return launch_any(d.dtype, a, p, s);
}

int launch_linattn_bwd(const pnn_linattn_desc& d, const void* q, const void* k, const void* v, const float* decay,
                       const int32_t* lengths, const float* s0, const void* dout, const float* dsT, void* dq, void* dk,
                       void* dv, float* ds0, void* ws, hipStream_t s) {
  const int group = (int)(d.heads / d.kv_heads);
  const LinBwd w = lin_bwd(d);
  char* const base = (char*)ws;
  Lin a = common(d, decay, lengths);
  Role &Q = a.role[0], &K = a.role[1];
  a.roles = 2;
  // dq_t = scale sum_{s <= t} lambda^(t - s) (do_t v_s) k_s + ..: inner width that of the values
  Q.q = dout, Q.k = v, Q.v = k, Q.o = dq;
  Q.qs = d.dout, Q.ks = d.v, Q.vs = d.k, Q.os = d.dq;
  Q.q_group = 1, Q.k_group = Q.v_group = group;
  Q.s0 = s0;
  Q.s_inner = 1, Q.s_value = d.value_width;
  Q.inner = (int)d.value_width, Q.value = (int)d.key_width;
  Q.intra = Q.inter = d.scale, Q.update = 1.0f;
  Q.blocks = w.wide.blocks;
  Q.seg = w.wide.segments > 1 ? (float*)(base + w.seg_q) : nullptr;
  // dk_s = sum_{t >= s} lambda^(t - s) (v_s do_t) scale q_t + lambda^(n - 1 - s) v_s dS_T
  K.q = v, K.k = dout, K.v = q, K.o = group > 1 ? (void*)(base + w.part_k) : dk;
  K.qs = d.v, K.ks = d.dout, K.vs = d.q, K.os = group > 1 ? lin_dense(d, d.key_width) : d.dk;
  K.q_group = group, K.k_group = K.v_group = 1;
  K.s0 = dsT;
  K.s_inner = 1, K.s_value = d.value_width;
  K.inner = (int)d.value_width, K.value = (int)d.key_width;
  K.intra = K.update = d.scale, K.inter = 1.0f;
  K.shift = 1;
  K.o_float = group > 1;
  K.blocks = w.wide.blocks;
  K.seg = w.wide.segments > 1 ? (float*)(base + w.seg_k) : nullptr;
  if (const int e = launch_any(d.dtype, a, w.wide, s)) return e;
  // dv_s = sum_{t >= s} lambda^(t - s) (k_s q_t) scale do_t + lambda^(n - 1 - s) k_s dS_T; dS_0
  Lin c = common(d, decay, lengths);
  Role& V = c.role[0];
  c.roles = 1;
  V.q = k, V.k = q, V.v = dout, V.o = group > 1 ? (void*)(base + w.part_v) : dv;
  V.qs = d.k, V.ks = d.q, V.vs = d.dout, V.os = group > 1 ? lin_dense(d, d.value_width) : d.dv;
  V.q_group = group, V.k_group = V.v_group = 1;
  V.s0 = dsT, V.sT = ds0;
  V.s_inner = d.value_width, V.s_value = 1;
  V.inner = (int)d.key_width, V.value = (int)d.value_width;
  V.intra = V.update = d.scale, V.inter = 1.0f;
  V.shift = 1;
  V.o_float = group > 1;
  V.blocks = w.deep.blocks;
  V.seg = w.deep.segments > 1 ? (float*)(base + w.seg_v) : nullptr;
  if (const int e = launch_any(d.dtype, c, w.deep, s)) return e;
  if (group > 1) {
    const int64_t rows = d.batch * d.length * d.kv_heads;
    auto sum = [&](const float* part, void* out, const pnn_head_stride& st, int64_t width) {
      const dim3 grid((unsigned)cdiv64(rows * width, NT));
      if (d.dtype == PNN_F32)
        hipLaunchKernelGGL((linattn_heads_kernel<float>), grid, dim3(NT), 0, s, part, out, st, rows, (int)d.length,
                           (int)d.kv_heads, group, (int)width);
      else
        hipLaunchKernelGGL((linattn_heads_kernel<uint16_t>), grid, dim3(NT), 0, s, part, out, st, rows, (int)d.length,
                           (int)d.kv_heads, group, (int)width);
    };
    sum((const float*)(base + w.part_k), dk, d.dk, d.key_width);
    sum((const float*)(base + w.part_v), dv, d.dv, d.value_width);
  }
  return (int)hipGetLastError();
}

}  // namespace pnn

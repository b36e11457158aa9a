// Linear attention with a decay for each head, and its backward:
//   S_t = lambda S_{t-1} + k_t v_t^T,   o_t = scale q_t^T S_t.
//
// Chunks of C steps.  With i, j steps of a chunk of len and S the state before it,
//   o_i = scale (sum_{j <= i} lambda^(i - j) (q_i k_j) v_j + lambda^(i + 1) q_i S)
//   S  <- lambda^len S + sum_j k_j (lambda^(len - 1 - j) v_j)^T,
// four products on the matrix units.  A workgroup of four or eight waves takes 64 or 128 value columns of a head through
// the chunks; a wave holds the state of its 16 columns in registers, in the layout that the products leave it in and
// that they take it in (a state column's rows are the summation index of q S, so its registers are an operand as they
// stand).  q k is formed once a workgroup and goes through LDS.  32 steps to a chunk, so that q, k, v and the outputs
// fit LDS for three workgroups a CU (64 steps with two column tiles a wave: 477 us where this took 384).
//
// The backward is the same sum three times:
//   dq: queries do, keys v, values k, from the transposed state;
//   dk: backwards in time, queries v, keys do, values q;   dv: backwards in time, queries k, keys q, values do,
// where a state before a step's own term weighs lambda^i instead of lambda^(i + 1) (`shift`).
//
// Few heads do not fill the device: their sequences are cut into segments, whose states from zero are formed by a
// first launch (without outputs), chained by a second, and taken as first states by the third.
//
// What bounds it is a chunk's chain of waits (copy to LDS, barrier, q k, barrier, outputs, state), not the matrix units
// or memory.  8 sequences of 2048 steps, 16 heads of 128 x 128, bf16: forward 107 us (270 MB, 2.5 TB/s, one workgroup
// of four waves a CU, 1.7 us a chunk), backward 167 us (700 MB, 4.2 TB/s, three a CU, 2.6 us a chunk); without its
// products the forward takes 78, without products and output stores 44.  One sequence of 32768 steps: 73 us for the
// states (293 MB, 4.0 TB/s), 16 for the chain, 136 for the outputs (577 MB, 4.2 TB/s).  A chunk's products with all
// operands read ahead, more registers and fewer waves: no gain (107, backward 166), spills in the eight-wave form.
//
// Roundings to bf16 besides the outputs' (bf16 tensors only): the weighted q k and the state, where they are operands
// of the products with v and q; together they are as large as the output's own rounding (outputs 2.34e-3 from 64 bits;
// two bf16 parts of each 1.66e-3, the output's rounding alone, but the training batch 315 us for 268 and the prompt 235 for
// 217).  The state itself is fp32, and the weighted values that are added to it are split into two bf16 parts: 16 bits,
// under a hundredth of the state's rounding as an operand, which is all that a call without sT (ds0) reads it for, its
// segments' states and the sums of dk and dq included.  Three parts (24 bits) where the caller wants the state.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int C = LIN_CHUNK;
constexpr int NT = 256;                     // threads of the small kernels
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
  int blocks;                               // workgroups a head's value columns are dealt to
};

struct Lin {
  Role role[3];
  const float* decay;
  const int32_t* lengths;
  int roles, batch, heads, length;
  int nseg, seg_chunks;                     // segments and chunks of one
  int most;                                 // blocks of the role with the most
  int items;                                // batch x heads x segments
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

// Rows of a chunk on their way through registers, 16 bytes a lane and row piece.  The piece that the row's end cuts is
// loaded and stored so that it ends there, over elements of the piece before it (LEFT: columns in front of a tile's
// rows, which nobody reads, for a value block that starts less than a piece before the row's end).  What is behind a
// row's end in LDS stays as clear() left it.  TINY: rows may be shorter than a piece; they are copied when they are
// stored.
template <typename T, int NT, int W, int PAD, bool TINY>
struct Stage {
  static constexpr int VE = St<T>::VE, PR = W / VE, N = (C * PR + NT - 1) / NT;
  static constexpr int LD = W + PAD * VE, LEFT = VE, SIZE = LEFT + C * LD;   // elements: of a row in LDS, in all
  static constexpr int ROWS = NT / PR;      // rows that the lanes' first pieces are of
  static_assert((N == 1 || N * NT == C * PR) && PAD >= 2, "whole pieces; a place behind the row");
  const T* p;                               // the lane's first piece of the next chunk; TINY: the chunk
  int64_t step;
  int at;                                   // where the lane's first piece goes in LDS
  int width, now;                           // of a row; rows of the sequence in the chunk held
  uint4 r[N];

  // the sequence's row 0 (its last one backwards in time) at this tile's columns, elements from row to row, columns, row
  __device__ __forceinline__ void begin(const T* first, int64_t step_, int width_, int64_t row) {
    step = step_;
    width = width_;
    const LinPiece x = lin_piece(threadIdx.x, C, PR, VE, width);
    at = LEFT + x.row * LD + x.to;
    p = first + row * step;
    if (!TINY) p += x.row * step + x.from;
  }
  static __device__ __forceinline__ void clear(T* lds) {
    for (int x = threadIdx.x; x < SIZE; x += NT) lds[x] = (T)0;
  }
  // the row of the lane's first piece
  __device__ __forceinline__ int row_at() const { return (at - LEFT + VE) / LD; }
  // The next chunk, of which `len` > 0 rows belong to the sequence.  Nothing here depends on the lane but addresses (a
  // load under a condition waits for the one before it): lanes that store nothing load a piece all the same, and those
  // of rows behind the sequence's end its last row.
  __device__ __forceinline__ void load(int len) {
    now = len;
    if (TINY) return;
    if (len >= C) {
#pragma unroll
      for (int j = 0; j < N; ++j) r[j] = piece(p + j * ROWS * step);
    } else {
      const int last = len - 1 - row_at();
#pragma unroll
      for (int j = 0; j < N; ++j) r[j] = piece(p + (j * ROWS < last ? j * ROWS : last) * step);
    }
  }
  static __device__ __forceinline__ uint4 piece(const T* s) {
    return __builtin_bit_cast(uint4, *(const typename Piece<T>::Mem*)s);
  }
  __device__ __forceinline__ void store(T* lds) {
    if (!TINY) {
      if (now < C) {
        asm volatile("");                   // a branch, not selections in every chunk
        const int row0 = row_at();
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (row0 + j * ROWS >= now) r[j] = make_uint4(0, 0, 0, 0);
      }
      typedef typename Piece<T>::Mem Mem;
#pragma unroll
      for (int j = 0; j < N; ++j) *(Mem*)(lds + at + j * ROWS * LD) = __builtin_bit_cast(typename Piece<T>::Vec, r[j]);
    } else {
      for (int x = threadIdx.x; x < C * W; x += NT) {
        const int row = x / W, c = x % W;
        if (c < width) lds[LEFT + row * LD + c] = row < now ? p[row * step + c] : (T)0;
      }
    }
    p += C * step;
  }
  // whether a value is infinite or NaN (TINY: not looked at)
  __device__ __forceinline__ bool lost() const {
    if (TINY) return true;
    // an exponent of ones carries into the bit above it
    constexpr uint32_t EXP = sizeof(T) == 2 ? 0x7f807f80u : 0x7f800000u, ONE = sizeof(T) == 2 ? 0x00800080u : 0x00800000u;
    constexpr uint32_t TOP = sizeof(T) == 2 ? 0x80008000u : 0x80000000u;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < N; ++j)
      m |= ((r[j].x & EXP) + ONE) | ((r[j].y & EXP) + ONE) | ((r[j].z & EXP) + ONE) | ((r[j].w & EXP) + ONE);
    return (m & TOP) != 0;
  }
};

// operand of a product from rows in LDS: the lane's row, summation index along the row
template <typename T>
__device__ __forceinline__ Frag<T> row_frag(const T* p) {
  Frag<T> f;
  f.from_raw(*(const uint4*)p);
  return f;
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
// A state tile's rows: row 4 g + r of tile dt is d = state_row(dt, g) + r.  bf16: chosen so that the lane's rows of two
// tiles are eight in a row, which is an operand's summation order; float: four of one tile are.
template <typename T>
__device__ __forceinline__ int state_row(int dt, int g) {
  return sizeof(T) == 2 ? 32 * (dt >> 1) + 8 * g + 4 * (dt & 1) : 16 * dt + 4 * g;
}
// the keys' columns that go with them
template <typename T>
__device__ __forceinline__ void key_frag(Frag<T>& f, const T* m, int ld, int dt, int i, int g) {
  if constexpr (sizeof(T) == 2) column_frag(f, m + 32 * (dt >> 1) + 4 * (dt & 1), ld, i, g, 8);
  else column_frag(f, m + 16 * dt, ld, i, g, 4);
}
// the state's columns as an operand of step kk
template <int KT>
__device__ __forceinline__ void state_frag(Frag<uint16_t>& f, const f32x4 (&S)[KT], int kk) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f.v[e] = (__bf16)S[2 * kk][e];
    f.v[4 + e] = (__bf16)S[2 * kk + 1][e];
  }
}
template <int KT>
__device__ __forceinline__ void state_frag(Frag<float>& f, const f32x4 (&S)[KT], int kk) {
#pragma unroll
  for (int e = 0; e < 4; ++e) f.v[e] = S[kk][e];
}
// v w in parts of 8 bits: the two largest, and with them what is left
__device__ __forceinline__ void split(const Frag<uint16_t>& v, const float* w, Frag<uint16_t> (&part)[2], float* rest) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  const uint4 u = __builtin_bit_cast(uint4, v.v);
  const uint32_t in[4] = {u.x, u.y, u.z, u.w};
  uint32_t out[2][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = __uint_as_float(in[e] << 16) * w[2 * e], b = __uint_as_float(in[e] & 0xffff0000u) * w[2 * e + 1];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
      const uint32_t c = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{a, b}), bf16x2));
      out[p][e] = c;
      a -= __uint_as_float(c << 16);
      b -= __uint_as_float(c & 0xffff0000u);
    }
    rest[2 * e] = a;
    rest[2 * e + 1] = b;
  }
#pragma unroll
  for (int p = 0; p < 2; ++p) part[p].from_raw(make_uint4(out[p][0], out[p][1], out[p][2], out[p][3]));
}

__device__ __forceinline__ bool not_finite(float v) { return !(fabsf(v) < INFINITY); }
__device__ __forceinline__ void finite_only(Frag<uint16_t>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (not_finite((float)f.v[e])) f.v[e] = (__bf16)0.0f;
}
__device__ __forceinline__ void finite_only(Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (not_finite(f.v[e])) f.v[e] = 0.0f;
}

// nothing moves over this: without it the compiler has the next products' operands in registers, and spills
__device__ __forceinline__ void phase_end() { __builtin_amdgcn_sched_barrier(0); }

// four neighbouring values, rounded (any: to any alignment)
__device__ __forceinline__ uint2 round4(f32x4 v) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  return __builtin_bit_cast(uint2, __builtin_convertvector(v, bf16x4));
}
template <typename T>
__device__ __forceinline__ void put4(T* p, f32x4 v) {
  if constexpr (sizeof(T) == 4) *(f32x4*)p = v;
  else *(uint2*)p = round4(v);
}
template <typename T>
__device__ __forceinline__ void put_any(T* p, f32x4 v) {
  typedef f32x4 FM __attribute__((aligned(4)));
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  typedef u32x2 UM __attribute__((aligned(2)));
  if constexpr (sizeof(T) == 4) {
    *(FM*)p = v;
  } else {
    const uint2 u = round4(v);
    *(UM*)p = u32x2{u.x, u.y};
  }
}

// waves that a SIMD is to hold, as far as registers and LDS allow
constexpr int lin_occupancy(int size, int pad, int waves) {
  if (size == 4) return pad == 64 ? (waves == 4 ? 3 : 4) : pad == 128 ? 2 : waves == 4 ? 1 : 2;
  return pad == 64 ? 4 : pad == 128 ? (waves == 4 ? 3 : 4) : 2;
}

// KD: inner width, padded; NW waves of 16 value columns each; OUT: outputs, not the state alone;
// TINY: rows shorter than 16 bytes.
template <typename T, int KD, int NW, bool OUT, bool TINY>
__global__ __launch_bounds__(64 * NW, lin_occupancy(sizeof(T), KD, NW)) void linattn_kernel(Lin a) {
  constexpr int NT = 64 * NW, VE = St<T>::VE, KS = 4 * VE, KT = KD / 16, CT = C / 16, EB = 16 * NW;
  constexpr int TILES = CT * (CT + 1) / 2;      // tiles of pt on or below the diagonal, one a wave
  static_assert(CT == 2 && TILES <= NW, "tiles of pt");
  // Rows in LDS are longer than they need be by 16 bytes times what kept the lanes' reads apart best: 2, and 4 for the
  // keys, whose columns are read in pieces 16 bytes apart (conflicts cost 3.4 of 12.3 million cycles; 9.7 of 18.6 with
  // 1, 6 and 4 for queries, keys and values; the training batch 352 -> 337 us).
  typedef Stage<T, NT, KD, 2, TINY> SQ;
  typedef Stage<T, NT, KD, 4, TINY> SK;
  typedef Stage<T, NT, EB, 2, TINY> SV;
  constexpr int LQ = SQ::LD, LK = SK::LD, LV = SV::LD, LP = C + 2 * VE, LO = EB + 4;
  __shared__ __attribute__((aligned(16))) T ks[SK::SIZE];
  __shared__ __attribute__((aligned(16))) T vs[SV::SIZE];
  __shared__ __attribute__((aligned(16))) T qs[OUT ? SQ::SIZE : 1];
  __shared__ __attribute__((aligned(16))) T pt[OUT ? C * LP : 1];
  __shared__ __attribute__((aligned(16))) float ot[OUT ? C * LO : 4];       // outputs on their way
  __shared__ __attribute__((aligned(16))) float wt[C], near[OUT ? C + 16 : 1], from[OUT ? C : 1];
  T *const kt = ks + SK::LEFT, *const vt = vs + SV::LEFT, *const qt = qs + SQ::LEFT;
  __shared__ int bad;
  // workgroups eight apart run on one XCD and share its L2: the roles and value blocks of a head and segment, which read
  // the same tensors
  const int inside = blockIdx.x / 8 % (a.roles * a.most), item = blockIdx.x / 8 / (a.roles * a.most) * 8 + blockIdx.x % 8;
  const Role& R = a.role[inside / a.most];
  const int block = inside % a.most;
  if (item >= a.items || block >= R.blocks) return;
  const int seg = item % a.nseg, bh = item / a.nseg;
  if (!OUT && seg == a.nseg - 1) return;               // nobody starts from its state
  const int b = bh / a.heads, h = bh % a.heads;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x & 63;
  const int n = steps_of(a.lengths, b, a.length);
  const float l2 = log2_decay(a.decay, h);
  const int e0 = block * EB + w * 16;                  // the wave's first value column
  const bool mine = e0 < R.value;
  // state: S[dt][r] is row state_row(dt, lane >> 4) + r of column e0 + (lane & 15)
  f32x4 S[KT];
  const int64_t state = (int64_t)bh * R.inner * R.value;
  float* const segment = R.seg == nullptr ? nullptr
      : R.seg + ((((int64_t)bh * a.nseg + seg) * R.blocks + block) * NW + w) * (KT * 256) + lane * 4;
#pragma unroll
  for (int dt = 0; dt < KT; ++dt) {
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
    if (OUT && segment != nullptr) {
      s = *(const f32x4*)(segment + dt * 256);
    } else if (OUT && R.s0 != nullptr) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int d = state_row<T>(dt, lane >> 4) + r, e = e0 + (lane & 15);
        if (d < R.inner && e < R.value) s[r] = R.s0[state + d * R.s_inner + e * R.s_value];
      }
    }
    S[dt] = s;
  }
  const int chunks = (a.length + C - 1) / C;
  const int c0 = seg * a.seg_chunks, c1 = c0 + a.seg_chunks < chunks ? c0 + a.seg_chunks : chunks;
  const int live = (n + C - 1) / C < c1 ? (n + C - 1) / C : c1;       // chunks with steps
  SQ rq;
  SK rk;
  SV rv;
  {
    // backwards in time row 0 is step n - 1 and the rows go down
    const int64_t row = (int64_t)c0 * C;
    auto first = [&](const void* base, const pnn_head_stride& s, int group) {
      return (const T*)base + (b * s.batch + (h / group) * s.head + (R.shift && n > 0 ? (n - 1) * s.step : 0));
    };
    auto step = [&](const pnn_head_stride& s) { return R.shift ? -s.step : s.step; };
    if (OUT) rq.begin(first(R.q, R.qs, R.q_group), step(R.qs), R.inner, row);
    rk.begin(first(R.k, R.ks, R.k_group), step(R.ks), R.inner, row);
    rv.begin(first(R.v, R.vs, R.v_group) + block * EB, step(R.vs), R.value - block * EB, row);
  }
  auto load = [&](int c) {
    const int len = n - c * C;
    if (OUT) rq.load(len);
    rk.load(len);
    rv.load(len);
  };
  if (c0 < live) load(c0);
  if (OUT) SQ::clear(qs);
  SK::clear(ks);
  SV::clear(vs);
  if constexpr (OUT) {                          // tiles of pt above the diagonal stay zero
    for (int x = threadIdx.x; x < C * LP; x += NT) pt[x] = (T)0;
    for (int x = threadIdx.x; x < C; x += NT) {
      near[C - 1 - x] = R.intra * power(l2, x);           // of the steps before, nearest last
      from[x] = R.inter * power(l2, x + 1 - R.shift);
    }
    if (threadIdx.x < 16) near[C + threadIdx.x] = 0.0f;
  }
  const bool exact = R.sT != nullptr;           // states that the caller sees
  int held = -1;                                // the length that wt and gone are for
  float gone = 0.0f;
  // Outputs of a chunk go to LDS and from there, whole rows, to memory when the next chunk is being worked on: stores
  // behind the loads of the next chunk would be waited for with them.
  const int inner = R.inner, columns = R.value - block * EB < EB ? R.value - block * EB : EB;
  const int64_t ostep = R.shift ? -R.os.step : R.os.step;
  const int64_t ofirst = b * R.os.batch + h * R.os.head + block * EB;
  constexpr int OR = EB / 4, ON = C * OR / NT;             // pieces of four: of a row, of a lane
  int64_t oat = ofirst + (R.shift ? (int64_t)(n - 1 - c0 * C) : (int64_t)c0 * C) * R.os.step +
                (int)(threadIdx.x / OR) * ostep + threadIdx.x % OR * 4;
  auto give = [&](int len) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));               // formed anew in each chunk, as the addresses below
    const int t = tid / OR, e = tid % OR * 4;
    const float* const from_lds = &ot[t * LO + e];
    if (len >= C && columns % 4 == 0) {
      if (e < columns) {
#pragma unroll
        for (int x = 0; x < ON; ++x) {
          const f32x4 v = *(const f32x4*)(from_lds + x * (NT / OR) * LO);
          if (R.o_float) put_any((float*)R.o + oat + x * (NT / OR) * ostep, v);
          else put_any((T*)R.o + oat + x * (NT / OR) * ostep, v);
        }
      }
    } else {
      asm volatile("");
      for (int x = 0; x < ON; ++x)
        for (int y = 0; y < 4; ++y) {
          if (t + x * (NT / OR) >= len || e + y >= columns) continue;
          const int64_t o = oat + x * (NT / OR) * ostep + y;
          const float v = from_lds[x * (NT / OR) * LO + y];
          if (R.o_float) ((float*)R.o)[o] = v;
          else St<T>::st(R.o, o, v);
        }
    }
    oat += C * ostep;
  };
  for (int c = c0; c < live; ++c) {
    // addresses in LDS formed anew each time: kept, they cost 60 registers
    int i = lane & 15, g = lane >> 4;
    asm volatile("" : "+v"(i), "+v"(g));
    const int len = n - c * C < C ? n - c * C : C;
    __syncthreads();                            // the chunk before is done with LDS
    if (threadIdx.x == 0) bad = 0;
    if (OUT) rq.store(qs);
    rk.store(ks);
    rv.store(vs);
    if (held != len) {
      held = len;
      gone = power(l2, len);
      for (int x = threadIdx.x; x < C; x += NT) wt[x] = x < len ? R.update * power(l2, len - 1 - x + R.shift) : 0.0f;
    }
    const bool odd = OUT && rv.lost();
    __syncthreads();
    if (odd) bad = 1;
    if (OUT && c > c0) give(C);
    if (c + 1 < live) load(c + 1);
    // Operands are read from LDS a batch ahead of the products that take them: read and waited for one by one, they
    // made the waits half as long again.
    f32x4 acc[CT];
    Frag<T> vf[C / KS];
    float since[CT];
    if constexpr (OUT) {
      // pt[t][s] = intra lambda^(t - s) q_t k_s for s <= t
      if (w < TILES) {
        const int ti = w < 1 ? 0 : 1, si = w < 2 ? 0 : 1, t = ti * 16 + i;
        constexpr int B = KD / KS < 4 ? KD / KS : 4;
        f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k0 = 0; k0 < KD / KS; k0 += B) {
          if (k0 * KS >= inner) continue;
          Frag<T> kf[B], qf[B];
#pragma unroll
          for (int kk = 0; kk < B; ++kk) {
            kf[kk] = row_frag(kt + (si * 16 + i) * LK + (k0 + kk) * KS + g * VE);
            qf[kk] = row_frag(qt + t * LQ + (k0 + kk) * KS + g * VE);
          }
          phase_end();
#pragma unroll
          for (int kk = 0; kk < B; ++kk) mma(kf[kk], qf[kk], p);
        }
        const int apart = t - si * 16 - 4 * g;  // of the first of the lane's four
        float f[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) f[r] = near[C - 1 - apart + r];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = apart >= r ? p[r] * f[r] : 0.0f;     // not 0 times what may be NaN
        put4(pt + t * LP + si * 16 + 4 * g, p);
      }
    }
    if (mine) {
      if constexpr (OUT) {
        // from the state before the chunk
#pragma unroll
        for (int ti = 0; ti < CT; ++ti) acc[ti] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        Frag<T> qf[2][CT];
        auto queries = [&](int kk) {
#pragma unroll
          for (int ti = 0; ti < CT; ++ti) qf[kk & 1][ti] = row_frag(qt + (ti * 16 + i) * LQ + kk * KS + g * VE);
        };
        queries(0);
#pragma unroll
        for (int kk = 0; kk < KD / KS; ++kk) {
          if (kk * KS >= inner) continue;
          if (kk + 1 < KD / KS) queries(kk + 1);
          Frag<T> sf;
          state_frag(sf, S, kk);
          phase_end();
#pragma unroll
          for (int ti = 0; ti < CT; ++ti) mma(sf, qf[kk & 1][ti], acc[ti]);
          phase_end();
        }
#pragma unroll
        for (int ti = 0; ti < CT; ++ti) since[ti] = from[ti * 16 + i];
      }
#pragma unroll
      for (int kb = 0; kb < C / KS; ++kb) column_frag(vf[kb], vt + kb * KS * LV + w * 16, LV, i, g, 4);
    }
    if (OUT) __syncthreads();                   // pt is complete
    if (!mine) continue;
    if constexpr (OUT) {
      if (bad == 0) {
        Frag<T> pf[CT][C / KS];
#pragma unroll
        for (int ti = 0; ti < CT; ++ti)
#pragma unroll
          for (int kb = 0; kb < C / KS; ++kb)
            if (kb * KS < 16 * (ti + 1)) pf[ti][kb] = row_frag(pt + (ti * 16 + i) * LP + kb * KS + g * VE);
#pragma unroll
        for (int ti = 0; ti < CT; ++ti)
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[ti][r] *= since[ti];
        phase_end();
#pragma unroll
        for (int kb = 0; kb < C / KS; ++kb)
#pragma unroll
          for (int ti = 0; ti < CT; ++ti)
            if (kb * KS < 16 * (ti + 1)) mma(vf[kb], pf[ti][kb], acc[ti]);
      } else {
        // An infinite or NaN value reaches the steps from its own on, which a product with the zeros above the diagonal
        // does not keep to: such values are left out of it and added one by one.
#pragma unroll
        for (int ti = 0; ti < CT; ++ti) {
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[ti][r] *= since[ti];
#pragma unroll
          for (int kb = 0; kb < C / KS; ++kb) {
            if (kb * KS >= 16 * (ti + 1)) continue;
            Frag<T> v = vf[kb];
            finite_only(v);
            mma(v, row_frag(pt + (ti * 16 + i) * LP + kb * KS + g * VE), acc[ti]);
          }
          for (int s = 0; s <= ti * 16 + i; ++s) {
            const float p = St<T>::ld(pt, (ti * 16 + i) * LP + s);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float v = St<T>::ld(vt, s * LV + w * 16 + 4 * g + x);
              if (not_finite(v)) acc[ti][x] += p * v;
            }
          }
        }
      }
      phase_end();
    }
    // the state after the chunk: batches of two of its tiles and one summation step
    constexpr int B = 2, PB = KT / B, BATCHES = C / KS * PB;
    Frag<T> kf[2][B];
    auto keys = [&](int u) {
#pragma unroll
      for (int x = 0; x < B; ++x) key_frag(kf[u & 1][x], kt + u / PB * KS * LK, LK, u % PB * B + x, i, g);
    };
    keys(0);
    if constexpr (OUT) {
#pragma unroll
      for (int ti = 0; ti < CT; ++ti) *(f32x4*)&ot[(ti * 16 + i) * LO + w * 16 + 4 * g] = acc[ti];
    }
#pragma unroll
    for (int dt = 0; dt < KT; ++dt) S[dt] *= gone;
    Frag<T> part[2];
#pragma unroll
    for (int u = 0; u < BATCHES; ++u) {
      const int kb = u / PB, dt = u % PB * B;
      if (dt == 0) {
        float ws[VE];
#pragma unroll
        for (int x = 0; x < VE; x += 4) *(f32x4*)(ws + x) = *(const f32x4*)&wt[kb * KS + g * VE + x];
        if constexpr (sizeof(T) == 2) {
          float rest[VE];
          split(vf[kb], ws, part, rest);
          if (exact) {
            Frag<T> last;
#pragma unroll
            for (int x = 0; x < VE; ++x) last.v[x] = (__bf16)rest[x];
#pragma unroll
            for (int d = 0; d < KT; ++d) {
              Frag<T> f;
              key_frag(f, kt + kb * KS * LK, LK, d, i, g);
              mma(f, last, S[d]);
            }
          }
        } else {
#pragma unroll
          for (int x = 0; x < VE; ++x) part[0].v[x] = vf[kb].v[x] * ws[x];
        }
      }
      if (u + 1 < BATCHES) keys(u + 1);
      phase_end();
      if (dt * 16 < inner) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int x = 0; x < B; ++x) mma(kf[u & 1][x], part[1], S[dt + x]);
        }
#pragma unroll
        for (int x = 0; x < B; ++x) mma(kf[u & 1][x], part[0], S[dt + x]);
      }
      phase_end();
    }
  }
  if constexpr (OUT) {
    __syncthreads();
    if (live > c0) give(n - (live - 1) * C);
    // steps behind the sequence's end
    const int64_t last = (int64_t)c1 * C < a.length ? (int64_t)c1 * C : a.length;
    for (int64_t t = (n > c0 * C ? n : c0 * C) + w; t < last; t += NW)
      for (int x = lane; x < columns; x += 64) {
        const int64_t o = ofirst + t * R.os.step + x;
        if (R.o_float) ((float*)R.o)[o] = 0.0f;
        else St<T>::st(R.o, o, 0.0f);
      }
    if (R.sT != nullptr && seg == a.nseg - 1) {
#pragma unroll
      for (int dt = 0; dt < KT; ++dt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int d = state_row<T>(dt, lane >> 4) + r, x = e0 + (lane & 15);
          if (d < R.inner && x < R.value) R.sT[state + d * R.s_inner + x * R.s_value] = S[dt][r];
        }
    }
  } else {
#pragma unroll
    for (int dt = 0; dt < KT; ++dt) *(f32x4*)(segment + dt * 256) = S[dt];
  }
}

// The segments' states from zero become their first states: a thread takes one piece of four through the segments.
template <typename T, int KD, int NW>
__global__ __launch_bounds__(NT) void linattn_chain_kernel(Lin a) {
  constexpr int KT = KD / 16;
  const Role& R = a.role[blockIdx.y];
  const int per = R.blocks * NW * KT * 64 / NT;               // workgroups of a head
  const int64_t pieces = (int64_t)per * NT;
  const int bh = blockIdx.x / per;
  if (bh >= a.batch * a.heads) return;                        // a role with fewer blocks
  const int x = blockIdx.x % per * NT + threadIdx.x;
  const int lane = x % 64, dt = x / 64 % KT, wave = x / 64 / KT;         // wave of all blocks
  const int d = state_row<T>(dt, lane >> 4), e = wave * 16 + (lane & 15);
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
  f32x4 u = p[0];
  for (int j = 0; j < a.nseg; ++j) {
    const f32x4 next = j + 2 < a.nseg ? p[(j + 1) * pieces] : u;
    p[j * pieces] = s;
    const int64_t most = (int64_t)a.seg_chunks * C, steps = n - j * most;
    s = s * power(l2, steps < 0 ? 0 : steps < most ? (int)steps : (int)most) + u;
    u = next;
  }
}

// One step of every sequence: a workgroup takes the value columns of a head, up to 32 VW of them, VW a lane, and deals
// the state's rows to its groups of `lanes` lanes.  Bound by the state, which is read and written once: 64 sequences of
// 16 heads of 128 x 128 (134 MB) take 33 us or 4.1 TB/s where a layer's state comes from memory, 24 us where the cache
// behind L2 still holds it.  States larger than L2 are stored past it (37 -> 33 us; AHEAD 4: 35, 16: 42).
template <typename T, int VW>
__global__ __launch_bounds__(NT) void linattn_step_kernel(Lin a, int lanes, bool past) {
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
        if (R.sT != nullptr) store_to((VM*)(R.sT + (state + (int64_t)d * R.value + e)), (VM)s[j], past);
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

// Gradients of keys and values that heads share: the heads' sum, in their order, four values a thread.
template <typename T>
__global__ __launch_bounds__(NT) void linattn_heads_kernel(const float* part_k, const float* part_v, void* dk, void* dv,
                                                           pnn_head_stride ks, pnn_head_stride vs, int64_t rows,
                                                           int length, int kv, int group, int key_width,
                                                           int value_width) {
  const bool keys = blockIdx.y == 0;
  const int width = keys ? key_width : value_width, pieces = (width + 3) / 4;
  const int64_t x = (int64_t)blockIdx.x * NT + threadIdx.x, r = x / pieces;       // (batch, step, shared head)
  const int e = (int)(x % pieces) * 4;
  if (r >= rows) return;
  const float* p = (keys ? part_k : part_v) + r * group * width + e;
  const pnn_head_stride& st = keys ? ks : vs;
  const int64_t bt = r / kv, o = bt / length * st.batch + bt % length * st.step + r % kv * st.head + e;
  void* const out = keys ? dk : dv;
  typedef f32x4 VM __attribute__((aligned(4)));
  if (e + 4 <= width) {
    f32x4 s = *(const VM*)p;
    for (int j = 1; j < group; ++j) s += *(const VM*)(p + (int64_t)j * width);
    put_any((T*)out + o, s);
  } else {
    for (int c = 0; e + c < width; ++c) {
      float s = p[c];
      for (int j = 1; j < group; ++j) s += p[(int64_t)j * width + c];
      St<T>::st(out, o + c, s);
    }
  }
}

template <typename T, int KD, int NW, bool TINY = false>
int launch_roles(Lin& a, hipStream_t s) {
  const dim3 grid((unsigned)(cdiv64(a.items, 8) * 8 * a.roles * a.most)), threads(64 * NW);
  if (a.nseg > 1) {
    hipLaunchKernelGGL((linattn_kernel<T, KD, NW, false, TINY>), grid, threads, 0, s, a);
    const unsigned per = (unsigned)(a.most * (NW * (KD / 16) * 64 / NT));
    hipLaunchKernelGGL((linattn_chain_kernel<T, KD, NW>), dim3(per * a.batch * a.heads, a.roles), dim3(NT), 0, s, a);
  }
  hipLaunchKernelGGL((linattn_kernel<T, KD, NW, true, TINY>), grid, threads, 0, s, a);
  return (int)hipGetLastError();
}

template <typename T>
int launch_type(Lin& a, const LinShape& p, hipStream_t s) {
  if (p.tiny) return launch_roles<T, 256, 8, true>(a, s);
  if (p.pad == 64) return p.waves == 4 ? launch_roles<T, 64, 4>(a, s) : launch_roles<T, 64, 8>(a, s);
  if (p.pad == 128) return p.waves == 4 ? launch_roles<T, 128, 4>(a, s) : launch_roles<T, 128, 8>(a, s);
  return p.waves == 4 ? launch_roles<T, 256, 4>(a, s) : launch_roles<T, 256, 8>(a, s);
}

int launch_shape(int dtype, Lin& a, const LinShape& p, hipStream_t s) {
  a.nseg = p.segments;
  a.seg_chunks = p.seg_chunks;
  a.most = 0;
  for (int z = 0; z < a.roles; ++z) {
    a.role[z].blocks = lin_blocks(p, a.role[z].value);
    if (a.role[z].blocks > a.most) a.most = a.role[z].blocks;
  }
  a.items = a.batch * a.heads * a.nseg;
  return dtype == PNN_F32 ? launch_type<float>(a, p, s) : launch_type<uint16_t>(a, p, s);
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
    const bool past = d.batch * d.heads * R.inner * R.value * 4 > L2_BYTES;
#define STEP(T, VW) hipLaunchKernelGGL((linattn_step_kernel<T, VW>), grid, dim3(NT), 0, s, a, lanes, past)
    if (d.dtype == PNN_F32) { if (vw == 4) STEP(float, 4); else STEP(float, 1); }
    else { if (vw == 4) STEP(uint16_t, 4); else STEP(uint16_t, 1); }
#undef STEP
    return (int)hipGetLastError();
  }
  const LinShape p = lin_shape(d, false);
  R.seg = p.segments > 1 ? (float*)ws : nullptr;
  return launch_shape(d.dtype, a, p, s);
}

int launch_linattn_bwd(const pnn_linattn_desc& d, const void* q, const void* k, const void* v, const float* decay,
                       const int32_t* lengths, const float* s0, const void* dout, const float* dsT, void* dq, void* dk,
                       void* dv, float* ds0, void* ws, hipStream_t s) {
  const int group = (int)(d.heads / d.kv_heads);
  const LinBwd w = lin_bwd(d);
  char* const base = (char*)ws;
  Lin a = common(d, decay, lengths);
  a.roles = 3;
  const bool cut = w.shape.segments > 1, shared = group > 1;
  // dk_s = sum_{t >= s} lambda^(t - s) (v_s do_t) scale q_t + lambda^(n - 1 - s) v_s dS_T
  Role& K = a.role[0];
  K.q = v, K.k = dout, K.v = q, K.o = shared ? (void*)(base + w.part_k) : dk;
  K.qs = d.v, K.ks = d.dout, K.vs = d.q, K.os = shared ? lin_dense(d, d.key_width) : d.dk;
  K.q_group = group, K.k_group = K.v_group = 1;
  K.s0 = dsT;
  K.s_inner = 1, K.s_value = d.value_width;
  K.inner = (int)d.value_width, K.value = (int)d.key_width;
  K.intra = K.update = d.scale, K.inter = 1.0f;
  K.shift = 1;
  K.o_float = shared;
  K.seg = cut ? (float*)(base + w.seg_k) : nullptr;
  // dv_s = sum_{t >= s} lambda^(t - s) (k_s q_t) scale do_t + lambda^(n - 1 - s) k_s dS_T; dS_0
  Role& V = a.role[1];
  V.q = k, V.k = q, V.v = dout, V.o = shared ? (void*)(base + w.part_v) : dv;
  V.qs = d.k, V.ks = d.q, V.vs = d.dout, V.os = shared ? lin_dense(d, d.value_width) : d.dv;
  V.q_group = group, V.k_group = V.v_group = 1;
  V.s0 = dsT, V.sT = ds0;
  V.s_inner = d.value_width, V.s_value = 1;
  V.inner = (int)d.key_width, V.value = (int)d.value_width;
  V.intra = V.update = d.scale, V.inter = 1.0f;
  V.shift = 1;
  V.o_float = shared;
  V.seg = cut ? (float*)(base + w.seg_v) : nullptr;
  // dq_t = scale sum_{s <= t} lambda^(t - s) (do_t v_s) k_s + scale lambda^(t + 1) S_0 do_t
  Role& Q = a.role[2];
  Q.q = dout, Q.k = v, Q.v = k, Q.o = dq;
  Q.qs = d.dout, Q.ks = d.v, Q.vs = d.k, Q.os = d.dq;
  Q.q_group = 1, Q.k_group = Q.v_group = group;
  Q.s0 = s0;
  Q.s_inner = 1, Q.s_value = d.value_width;
  Q.inner = (int)d.value_width, Q.value = (int)d.key_width;
  Q.intra = Q.inter = d.scale, Q.update = 1.0f;
  Q.seg = cut ? (float*)(base + w.seg_q) : nullptr;
  if (const int e = launch_shape(d.dtype, a, w.shape, s)) return e;
  if (shared && d.length > 0) {
    const int64_t rows = d.batch * d.length * d.kv_heads;
    const dim3 grid((unsigned)cdiv64(lin_head_threads(d), NT), 2);
#define HEADS(T) hipLaunchKernelGGL((linattn_heads_kernel<T>), grid, dim3(NT), 0, s, (const float*)(base + w.part_k), \
    (const float*)(base + w.part_v), dk, dv, d.dk, d.dv, rows, (int)d.length, (int)d.kv_heads, group, \
    (int)d.key_width, (int)d.value_width)
    if (d.dtype == PNN_F32) HEADS(float);
    else HEADS(uint16_t);
#undef HEADS
  }
  return (int)hipGetLastError();
}

}  // namespace pnn

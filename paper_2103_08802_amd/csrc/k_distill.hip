// Distillation loss of a row of logits z against a teacher's top logits, and its gradient:
//   loss = alpha tau^2 sum_k p_k (log p_k - log q_{i_k}) + (1 - alpha) (-log s_y)
//   dz_v = scale w (alpha tau (q_v - sum_{i_k = v} p_k) + (1 - alpha) (s_v - [v = y]))
// with q = softmax(z / tau), s = softmax(z), p = softmax(teacher / tau).
//
// One workgroup per row.  The row is loaded once, into registers, as 16-byte pieces of the storage
// type (NC a thread); its maximum, the sums of exponentials and the gradient are formed from there.
// Rows too long for that are read twice (a running maximum and sums, then the gradient).  The
// gradient is first written as if the row had neither entries nor a label; the classes that stand in
// one are written again by the thread of their first entry, from logits gathered before any store.
//
// Rows may start anywhere: the whole pieces between the first and the last 16-byte boundary are the
// row's body, the elements before and behind (fewer than two pieces) go to one thread each.
//
// Bound: HBM (bf16, 4096 x 65536 classes, 64 entries, labels: 205 us, 1.07 GB at 5.2 TB/s, what a large
// copy reaches; the loss alone 127 us), with two rows to a compute unit so that one's exponentials (20 vector
// operations an element in all, two of them exponentials) run while the other's pieces are on their way; rows
// read twice reach 4.1 TB/s of that count (2048 x 131072 float: 528 us, 2048 x 151936 bf16: 296 us).  Few long
// rows: a row's latency, 18 us at 128000 classes.
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int64_t MAX_GRID = 1 << 20;   // rows of a launch
constexpr float LOG2E = 1.44269504f;

struct Distill {
  const void *z, *t;
  const int32_t *index, *labels;
  const float* weight;
  float* loss;
  void* dz;
  int64_t row0, z_stride, dz_stride, t_stride;
  int classes, top, t_bf16, past;
  int hash_mask;                 // a power of two above 2 top, less one
  float tau, alpha, scale;
};

// Which exponentials a row needs: one softmax (tau = 1, or only one of the two terms), both with
// softmax(z)'s exponentials as squares or fourth powers of those of z / 2 or z / 4, or both apart.  4096 x 65536
// bf16: SQUARE 204 us, FOURTH 213, and BOTH, which would serve their temperatures too, 224 (tau 0.5) to 231 (3).
// FOURTH and BOTH spill four registers with eight bf16 pieces a thread.
enum { ONE = 0, SQUARE = 1, FOURTH = 2, BOTH = 3 };

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's reference point: its maximum and log2(e) / tau (ONE: the factor of the only softmax).  The difference
// comes first: an exponent as fma(z, k, -round(k m)) is an operation less, but its rounding error grows with the
// logits themselves and is infinite where all of them are the type's lowest value.
struct Ref {
  float m, kq;
};
// exponentials of z / tau and z about the reference point
template <int MODE>
__device__ __forceinline__ void exps(float z, const Ref& r, float& eq, float& es) {
  const float d = z - r.m;
  eq = exp2_(d * r.kq);
  if constexpr (MODE == ONE) es = eq;
  if constexpr (MODE == SQUARE) es = eq * eq;
  if constexpr (MODE == FOURTH) {
    const float e2 = eq * eq;
    es = e2 * e2;
  }
  if constexpr (MODE == BOTH) es = exp2_(d * LOG2E);
}
// four elements' exponentials added to the sums; the four exponentials stand together, ahead of their uses
template <int MODE>
__device__ __forceinline__ void add_exps(const float* z, const Ref& r, float& sq, float& ss) {
  float eq[4], es[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) exps<MODE == BOTH ? BOTH : ONE>(z[e], r, eq[e], es[e]);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    sq += eq[e];
    if constexpr (MODE == SQUARE) ss = fmaf(eq[e], eq[e], ss);
    if constexpr (MODE == FOURTH) ss = fmaf(eq[e] * eq[e], eq[e] * eq[e], ss);
    if constexpr (MODE == BOTH) ss += es[e];
  }
}
// sums about one reference point as sums about another
template <int MODE>
__device__ __forceinline__ void move_sums(const Ref& from, const Ref& to, float& sq, float& ss) {
  float eq, es;
  exps<MODE>(from.m, to, eq, es);
  sq *= eq;
  ss *= es;
}

// A row of T as a body of whole 16-byte pieces and single elements before (`head`) and behind it
template <typename T>
struct Row {
  const T* p;
  int classes, head, pieces;
  __device__ __forceinline__ Row(const void* base, int64_t off, int classes_) {
    p = (const T*)base + off;
    classes = classes_;
    head = (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
    head = head < classes ? head : classes;
    pieces = (classes - head) / St<T>::VE;
  }
  __device__ __forceinline__ int edges() const { return classes - pieces * St<T>::VE; }   // < 2 VE
  // class of edge element i; unsigned, as it is formed past the edges too and may pass 2^31 there
  __device__ __forceinline__ unsigned edge(unsigned i) const { return i < (unsigned)head ? i : i + pieces * St<T>::VE; }
};

template <typename T>
__device__ __forceinline__ uint4 minus_inf() {
  const uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
  return make_uint4(w, w, w, w);
}

// The piece as loaded, not the floats an earlier sweep unpacked from it (which the compiler would keep, at twice the
// registers), and nothing of later pieces before it.
__device__ __forceinline__ uint4 again(uint4& u) {
  asm volatile("" : "+v"(u.x), "+v"(u.y), "+v"(u.z), "+v"(u.w));
  return u;
}
__device__ __forceinline__ uint4 load16(const void* base, uint32_t bytes) {
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4 v = *at<const u32x4>(base, bytes);
  return make_uint4(v.x, v.y, v.z, v.w);
}
__device__ __forceinline__ void piece_end() { __builtin_amdgcn_sched_barrier(0); }

// NC > 0: the row in registers, NC pieces a thread; NC = 0: read twice
template <typename T, int NT, int NC, int MODE>
__global__ __launch_bounds__(NT, NC == 8 ? 8 : 1) void distill_kernel(Distill a) {
  constexpr int VE = St<T>::VE, NWV = NT / 64;
  extern __shared__ float entries[];              // as many as the call has: short rows share a CU's LDS by dozens
  float* const et = entries;                      // [top] an entry's teacher logit (-inf: no entry)
  float* const ez = et + a.top;                   // [top + 1] the student's logit of its class; the label is entry `top`
  int* const ei = (int*)(ez + a.top + 1);         // [top + 1] its class, -1: none
  int* const table = ei + a.top + 1;              // [hash_mask + 1] classes of entries, hashed
  __shared__ int twice, listed;
  __shared__ float wm[NWV], wt[NWV], wq[NWV], ws[NWV], wp[NWV], wk[NWV];
  __shared__ int wbad[NWV];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  const float inv_tau = 1.0f / a.tau, kt = LOG2E / a.tau;
  const float kq = MODE == ONE && a.top == 0 ? LOG2E : kt;   // the label's softmax alone is untempered
  const int64_t row = a.row0 + blockIdx.x;
  const Row<T> r(a.z, row * a.z_stride, a.classes);
  const T* const body = r.p + r.head;
  // loads: the thread's first teacher entry, the row, then (what depends on it) the entry's class
  const int y = a.labels != nullptr ? a.labels[row] : -1;
  auto teacher = [&](int k) {
    return a.t_bf16 ? St<uint16_t>::ld(a.t, row * a.t_stride + k) : St<float>::ld(a.t, row * a.t_stride + k);
  };
  int i0 = -1;
  float t0 = 0.0f, z0 = 0.0f;
  if (tid < a.top) {
    i0 = a.index[row * a.t_stride + tid];
    t0 = teacher(tid);
  } else if (tid == a.top) {
    i0 = y;
  }
  uint4 raw[NC > 0 ? NC : 1];
  if constexpr (NC > 0) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      raw[j] = minus_inf<T>();
      if (j * NT + tid < r.pieces) raw[j] = load16(body + j * NT * VE, tid * 16);
    }
  }
  const bool has_edge = tid < r.edges();
  const unsigned ve = r.edge(tid);
  const float edge = has_edge ? St<T>::ld(r.p, ve) : -INFINITY;
  for (int h = tid; h <= a.hash_mask; h += NT) table[h] = -1;
  if (tid == 0) twice = listed = 0;
  bool bad = false;
  float tm = -INFINITY;
  auto entry = [&](int k, int& i, float t) {       // entry k's class (-1: none) and teacher logit to LDS
    bad |= i >= a.classes;
    if (k < a.top) {
      t = i >= 0 ? t : -INFINITY;
      et[k] = t;
      tm = t > tm || t != t ? t : tm;              // keeps NaN
    }
    i = i >= 0 && i < a.classes ? i : -1;
    ei[k] = i;
    return i >= 0 ? St<T>::ld(r.p, i) : 0.0f;
  };
  if (tid <= a.top) z0 = entry(tid, i0, t0);       // to LDS only when the row has been summed
  for (int k = tid + NT; k <= a.top; k += NT) {
    int i = k < a.top ? a.index[row * a.t_stride + k] : y;
    const float t = k < a.top ? teacher(k) : 0.0f;
    ez[k] = entry(k, i, t);
  }
  // maximum of the row; with the row read twice also the thread's sums about its own maximum
  float m = edge, sq = 0.0f, ss = 0.0f;
  Ref ref = {0.0f, kq};                            // a thread that has seen nothing but -inf: sums stay 0
  if constexpr (NC > 0) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      Chunk<T> v;
      unpack_chunk<T>(again(raw[j]), v);
#pragma unroll
      for (int e = 0; e < VE; ++e) m = fmaxf(m, v.v[e]);
    }
  } else {
    if (m != -INFINITY) {
      ref = Ref{m, kq};
      exps<MODE>(m, ref, sq, ss);
    }
    for (int c = tid; c < r.pieces; c += NT) {
      Chunk<T> v;
      unpack_chunk<T>(((const uint4*)body)[c], v);
      float cm = v.v[0];
#pragma unroll
      for (int e = 1; e < VE; ++e) cm = fmaxf(cm, v.v[e]);
      if (cm > m) {
        const Ref next = {cm, kq};
        if (m != -INFINITY) move_sums<MODE>(ref, next, sq, ss);
        ref = next;
        m = cm;
      }
#pragma unroll
      for (int e = 0; e < VE; e += 4) add_exps<MODE>(v.v + e, ref, sq, ss);
    }
  }
  const float own = m;
  m = wave_max(m);
  bool nan = tm != tm;
  tm = wave_max(tm);
  const int flags = (__any(bad) ? 1 : 0) | (__any(nan) ? 2 : 0);
  if (lane == 0) {
    wm[wave] = m;
    wt[wave] = tm;
    wbad[wave] = flags;
  }
  __syncthreads();
  int all = 0;
#pragma unroll 4
  for (int w = 0; w < NWV; ++w) {
    m = fmaxf(m, wm[w]);
    tm = fmaxf(tm, wt[w]);
    all |= wbad[w];
  }
  bad = all & 1;
  if (all & 2) tm = __builtin_nanf("");
  const bool some = tm != -INFINITY;             // an entry with a finite (or NaN) teacher logit
  const Ref own_ref = ref;
  ref = Ref{m, kq};
  // sums of exponentials: of the row about m, of the teacher's entries about tm
  if constexpr (NC > 0) {
    float eq, es;
    exps<MODE>(edge, ref, eq, es);
    if (has_edge) {
      sq = eq;
      ss = es;
    }
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      Chunk<T> v;
      unpack_chunk<T>(again(raw[j]), v);
#pragma unroll
      for (int e = 0; e < VE; e += 4) add_exps<MODE>(v.v + e, ref, sq, ss);
      piece_end();
    }
  } else {
    if (own != -INFINITY) move_sums<MODE>(own_ref, ref, sq, ss);
    if (m == -INFINITY) sq = ss = __builtin_nanf("");   // nothing but -inf: no distribution
  }
  // the teacher's sum; whether a class stands in two entries, and whether the label's stands in one
  float ts = 0.0f;
  for (int k = tid; k < a.top; k += NT) {
    ts += some ? exp2_((et[k] - tm) * kt) : 0.0f;
    const int i = ei[k];
    if (i < 0) continue;
    if (i == y) listed = 1;
    // open addressing, at most half full: every probe sequence meets the class or a free place
    for (unsigned h = (unsigned)i * 2654435761u >> 16;; ++h) {
      const int old = atomicCAS(&table[h & a.hash_mask], -1, i);
      if (old == i) twice = 1;
      if (old == i || old == -1) break;
    }
  }
  if (tid <= a.top) ez[tid] = z0;
  sq = wave_add(sq);
  if constexpr (MODE != ONE) ss = wave_add(ss);
  ts = wave_add(ts);
  if (lane == 0) {
    wq[wave] = sq;
    ws[wave] = ss;
    wp[wave] = ts;
  }
  __syncthreads();
  sq = ss = ts = 0.0f;
#pragma unroll 4
  for (int w = 0; w < NWV; ++w) {
    sq += wq[w];
    if constexpr (MODE != ONE) ss += ws[w];
    ts += wp[w];
  }
  if constexpr (MODE == ONE) ss = sq;
  // log p_k - log q_k = (t_k - tm) / tau - log ts - (z_k - m) / tau + log sq
  const float inv_ts = 1.0f / ts, lqt = logf(sq) - logf(ts);
  float kl = 0.0f;
  for (int k = tid; k < a.top; k += NT) {
    if (!some || ei[k] < 0) continue;
    const float p = exp2_((et[k] - tm) * kt) * inv_ts;
    if (p != 0.0f) kl += p * (((et[k] - tm) - (ez[k] - m)) * inv_tau + lqt);
  }
  const bool hard = y >= 0;
  float g = a.scale * (a.weight != nullptr ? a.weight[row] : 1.0f);
  if (bad) g = __builtin_nanf("");
  const float gq = g * a.alpha * a.tau, gs = g * (1.0f - a.alpha);
  const float cq = some || bad ? gq / sq : 0.0f, cs = hard ? gs / ss : 0.0f;
  const bool zero = !some && !hard && !bad;      // neither term: no gradient, whatever the logits
  const float c1 = cq + cs;
  auto grad = [&](float z) {                     // cq eq + cs es
    float eq, es;
    exps<MODE == BOTH ? BOTH : ONE>(z, ref, eq, es);
    if constexpr (MODE == ONE) return c1 * eq;
    if constexpr (MODE == SQUARE) return fmaf(cs, eq, cq) * eq;
    if constexpr (MODE == FOURTH) return fmaf(cs, eq * eq * eq, cq) * eq;
    return fmaf(cq, eq, cs * es);
  };
  if (a.dz != nullptr) {
    T* const dp = (T*)a.dz + row * a.dz_stride;
    const bool together = (((uintptr_t)(dp + r.head)) & 15) == 0;   // the gradient's pieces are the row's
    auto put = [&](int c, uint4 u) {
      Chunk<T> v;
      unpack_chunk<T>(u, v);
#pragma unroll
      for (int e = 0; e < VE; ++e) v.v[e] = grad(v.v[e]);
      if (together) {
        store_piece<T>(dp + r.head, (int64_t)c * VE, v.v, a.past);
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) St<T>::st(dp, r.head + (int64_t)c * VE + e, v.v[e]);
      }
    };
    if (zero) {
      for (unsigned v = tid; v < (unsigned)a.classes; v += NT) St<T>::st(dp, v, 0.0f);   // v may pass 2^31
    } else if constexpr (NC > 0) {
#pragma unroll
      for (int j = 0; j < NC; ++j) {
        if (j * NT + tid < r.pieces) put(j * NT + tid, again(raw[j]));
        piece_end();
      }
    } else {
      for (int c = tid; c < r.pieces; c += NT) put(c, ((const uint4*)body)[c]);
    }
    if (has_edge && !zero) St<T>::st(dp, ve, grad(edge));
  }
  kl = wave_add(kl);
  if (lane == 0) wk[wave] = kl;
  __syncthreads();                               // also orders the stores above before those below (one compute unit's)
  if (tid == 0) {
    float l = 0.0f;
#pragma unroll
    for (int w = 0; w < NWV; ++w) l += wk[w];
    l *= a.alpha * a.tau * a.tau;
    if (hard) l += (1.0f - a.alpha) * (logf(ss) - (ez[a.top] - m));
    a.loss[row] = bad ? __builtin_nanf("") : l;
  }
  if (a.dz != nullptr && !zero && !bad) {
    for (int k = tid; k <= a.top; k += NT) {
      const int i = ei[k];
      if (i < 0) continue;
      bool first = k < a.top || !listed;
      float p = 0.0f;
      if (!twice) {
        if (some && k < a.top) p = exp2_((et[k] - tm) * kt) * inv_ts;
      } else {                                     // the first of a class's entries takes the others' p as well
        for (int j = 0; j < a.top; ++j)
          if (ei[j] == i) {
            if (j < k) first = false;
            if (some) p += exp2_((et[j] - tm) * kt) * inv_ts;
          }
      }
      if (first) St<T>::st(a.dz, row * a.dz_stride + i, grad(ez[k]) - gq * p - (i == y ? gs : 0.0f));
    }
  }
}

// a row's pieces at most: the first and the last boundary may lie inside the row
template <typename T, int MODE>
void launch_rows(const Distill& a, int64_t rows, hipStream_t s) {
  const dim3 grid((unsigned)rows);
  const int pieces = a.classes / St<T>::VE;
#define ROWS(NT, NC) hipLaunchKernelGGL((distill_kernel<T, NT, NC, MODE>), grid, dim3(NT), (3 * a.top + 3 + a.hash_mask) * 4, s, a)
  if (pieces <= 64 * 4) ROWS(64, 4);
  else if (pieces <= 256 * 4) ROWS(256, 4);
  else if (pieces <= 512 * 8) ROWS(512, 8);
  else if (pieces <= 1024 * 8) ROWS(1024, 8);
  else if (pieces <= 1024 * 16) ROWS(1024, 16);
  else ROWS(1024, 0);
#undef ROWS
}

template <typename T>
void launch_mode(const Distill& a, int64_t rows, hipStream_t s) {
  if (a.labels == nullptr || a.top == 0 || a.tau == 1.0f) launch_rows<T, ONE>(a, rows, s);
  else if (a.tau == 2.0f) launch_rows<T, SQUARE>(a, rows, s);
  else if (a.tau == 4.0f) launch_rows<T, FOURTH>(a, rows, s);
  else launch_rows<T, BOTH>(a, rows, s);
}

}  // namespace

int launch_distill(const pnn_distill_desc& d, const void* logits, const int32_t* index, const void* teacher,
                   const int32_t* labels, const float* weight, float* loss, void* dlogits, hipStream_t s) {
  Distill a;
  a.z = logits;
  a.t = teacher;
  a.index = index;
  a.labels = d.alpha == 1.0f ? nullptr : labels;   // a term of weight zero is left out
  a.weight = weight;
  a.loss = loss;
  a.dz = dlogits;
  a.z_stride = d.logit_stride;
  a.dz_stride = d.grad_stride;
  a.t_stride = d.top_stride;
  a.classes = (int)d.classes;
  a.top = d.alpha == 0.0f ? 0 : (int)d.top;
  a.hash_mask = 1;
  while (a.hash_mask < 2 * a.top) a.hash_mask = 2 * a.hash_mask + 1;
  a.t_bf16 = d.teacher_dtype == PNN_BF16;
  a.past = d.rows * d.classes * (d.dtype == PNN_F32 ? 4 : 2) > L2_BYTES;
  a.tau = d.temperature;
  a.alpha = d.alpha;
  a.scale = d.scale;
  for (a.row0 = 0; a.row0 < d.rows; a.row0 += MAX_GRID) {
    const int64_t rows = d.rows - a.row0 < MAX_GRID ? d.rows - a.row0 : MAX_GRID;
    if (d.dtype == PNN_F32) launch_mode<float>(a, rows, s);
    else launch_mode<uint16_t>(a, rows, s);
    if (const hipError_t e = hipGetLastError()) return (int)e;
  }
  return 0;
}

}  // namespace pnn

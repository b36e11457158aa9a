// Clipped policy loss of a row of logits z and the token a that was drawn from it, with a KL term, and its gradient:
//   l = log softmax(z / tau)_a,  r = exp(l - old),  x = ref - l
//   loss = -min(r A, clip(r, 1 - low, 1 + high) A) + kl (exp(x) - 1 - x)
//   dz_v = scale w c / tau ([v = a] - p_v),  c = dloss / dl = -[r A <= clip(r) A] r A - kl (exp(x) - 1)
//
// One workgroup per row, which it loads once, into registers, as 16-byte pieces (NC a thread): maximum, sum of
// exponentials, then the gradient from the same registers.  Rows too long for that are read twice.  Rows without a token
// are not read.
//
// Bound by memory: 4096 x 65536 bf16 take 200 us, 1.07 GB or 5.4 TB/s, as much as a copy.  777 ragged rows of 32771 take
// 21 us (89 MB, 4.2 TB/s): one round of rows, all in the same phase.  A row of 1000 is a launch's own 4 us.
#include "device_common.h"
#include "row_device.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int64_t MAX_GRID = 1 << 20;   // rows of a launch
constexpr float LOG2E = 1.44269504f;

struct Policy {
  const void* z;
  const int32_t* tokens;
  const float *advantage, *old, *ref, *weight;
  float *loss, *logp;
  void* dz;
  int64_t row0, z_stride, dz_stride;
  int classes, past;
  float tau, low, high, kl, scale;
};

// zeros in a row
template <typename T, int NT>
__device__ __forceinline__ void clear_row(T* p, int classes, bool past) {
  const Row<T> r(p, 0, classes);
  float none[St<T>::VE] = {};
  for (int c = threadIdx.x; c < r.pieces; c += NT) store_piece<T>(p + r.head, (int64_t)c * St<T>::VE, none, past);
  if ((int)threadIdx.x < r.edges()) St<T>::st(p, r.edge(threadIdx.x), 0.0f);
}

// NC > 0: the row in registers, NC pieces a thread; NC = 0: read twice
template <typename T, int NT, int NC>
__global__ __launch_bounds__(NT, NC == 8 ? 8 : 1) void policy_kernel(Policy a) {
  constexpr int VE = St<T>::VE, NWV = NT / 64;
  __shared__ float wm[NWV], ws[NWV];
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  const int64_t row = a.row0 + blockIdx.x;
  const int y = a.tokens[row];
  T* const dp = a.dz == nullptr ? nullptr : (T*)a.dz + row * a.dz_stride;
  if (y < 0) {
    if (tid == 0) {
      a.loss[row] = 0.0f;
      if (a.logp != nullptr) a.logp[row] = 0.0f;
    }
    if (dp != nullptr) clear_row<T, NT>(dp, a.classes, a.past);
    return;
  }
  const Row<T> r(a.z, row * a.z_stride, a.classes);
  const T* const body = r.p + r.head;
  const float k = LOG2E / a.tau;
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
  const bool bad = y >= a.classes;
  const float zy = bad ? __builtin_nanf("") : St<T>::ld(r.p, y);
  const float A = a.advantage[row], w = a.scale * (a.weight != nullptr ? a.weight[row] : 1.0f);
  // the row's maximum; with the row read twice also the thread's sum about its own maximum, or about 0 while it has
  // seen nothing above -inf (the sum then stays 0, or NaN)
  float m = edge, s = 0.0f;
  if constexpr (NC > 0) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      Chunk<T> v;
      unpack_chunk<T>(again(raw[j]), v);
#pragma unroll
      for (int e = 0; e < VE; ++e) m = fmaxf(m, v.v[e]);
    }
  } else {
    s = __builtin_amdgcn_exp2f((edge - (m == -INFINITY ? 0.0f : m)) * k);
    for (int c = tid; c < r.pieces; c += NT) {
      Chunk<T> v;
      unpack_chunk<T>(((const uint4*)body)[c], v);
      float cm = v.v[0];
#pragma unroll
      for (int e = 1; e < VE; ++e) cm = fmaxf(cm, v.v[e]);
      if (cm > m) {
        if (m != -INFINITY) s *= __builtin_amdgcn_exp2f((m - cm) * k);
        m = cm;
      }
      const float about = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int e = 0; e < VE; ++e) s += __builtin_amdgcn_exp2f((v.v[e] - about) * k);
    }
  }
  const float own = m;
  m = wave_max(m);
  if (lane == 0) wm[wave] = m;
  __syncthreads();
#pragma unroll 4
  for (int x = 0; x < NWV; ++x) m = fmaxf(m, wm[x]);
  // sum of exponentials about m; a row of nothing but -inf has no distribution: NaN
  if constexpr (NC > 0) {
    if (has_edge) s = __builtin_amdgcn_exp2f((edge - m) * k);
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      Chunk<T> v;
      unpack_chunk<T>(again(raw[j]), v);
      float e2[VE];
#pragma unroll
      for (int e = 0; e < VE; ++e) e2[e] = __builtin_amdgcn_exp2f((v.v[e] - m) * k);
#pragma unroll
      for (int e = 0; e < VE; ++e) s += e2[e];
      piece_end();
    }
  } else {
    if (own != -INFINITY) s *= __builtin_amdgcn_exp2f((own - m) * k);
    if (m == -INFINITY) s = __builtin_nanf("");
  }
  s = wave_add(s);
  if (lane == 0) ws[wave] = s;
  __syncthreads();
  s = 0.0f;
#pragma unroll 4
  for (int x = 0; x < NWV; ++x) s += ws[x];
  const float l = (zy - m) / a.tau - logf(s);
  const float ratio = a.old != nullptr ? expf(l - a.old[row]) : 1.0f;
  const float whole = A == 0.0f && ratio == INFINITY ? 0.0f : ratio * A;         // 0 whatever the ratio, not 0 times infinity
  const float cut = (ratio < 1.0f - a.low ? 1.0f - a.low : ratio > 1.0f + a.high ? 1.0f + a.high : ratio) * A;
  float loss = whole > cut ? -cut : -whole, c = whole > cut ? 0.0f : -whole;       // NaN stays NaN
  if (a.kl != 0.0f) {
    const float x = a.ref[row] - l, up = expm1f(x);
    loss = fmaf(a.kl, up - x, loss);
    c = fmaf(-a.kl, up, c);
  }
  if (bad) loss = c = __builtin_nanf("");
  if (tid == 0) {
    a.loss[row] = loss;
    if (a.logp != nullptr) a.logp[row] = l;
  }
  if (dp == nullptr) return;
  const float g = w * c / a.tau, cp = -g / s;
  auto grad = [&](float z) { return cp * __builtin_amdgcn_exp2f((z - m) * k); };
  const bool together = (((uintptr_t)(dp + r.head)) & 15) == 0;   // the gradient's pieces are the row's
  auto put = [&](int piece, uint4 u) {
    Chunk<T> v;
    unpack_chunk<T>(u, v);
#pragma unroll
    for (int e = 0; e < VE; ++e) v.v[e] = grad(v.v[e]);
    if (together) {
      store_piece<T>(dp + r.head, (int64_t)piece * VE, v.v, a.past);
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e) St<T>::st(dp, r.head + (int64_t)piece * VE + e, v.v[e]);
    }
  };
  if constexpr (NC > 0) {
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      if (j * NT + tid < r.pieces) put(j * NT + tid, again(raw[j]));
      piece_end();
    }
  } else {
    for (int p = tid; p < r.pieces; p += NT) put(p, ((const uint4*)body)[p]);
  }
  if (has_edge) St<T>::st(dp, ve, grad(edge));
  if (bad) return;
  __syncthreads();                               // the token's class again, behind the stores above
  if (tid == 0) St<T>::st(dp, y, g * -expm1f(l));
}

template <typename T>
void launch_rows(const Policy& a, int64_t rows, hipStream_t s) {
  const dim3 grid((unsigned)rows);
  const int pieces = a.classes / St<T>::VE;
#define ROWS(NT, NC) hipLaunchKernelGGL((policy_kernel<T, NT, NC>), grid, dim3(NT), 0, s, a)
  if (pieces <= 64 * 4) ROWS(64, 4);
  else if (pieces <= 256 * 4) ROWS(256, 4);
  else if (pieces <= 512 * 8) ROWS(512, 8);
  else if (pieces <= 1024 * 8) ROWS(1024, 8);
  else if (pieces <= 1024 * 16) ROWS(1024, 16);
  else ROWS(1024, 0);
#undef ROWS
}

}  // namespace

int launch_policy(const pnn_policy_desc& d, const void* logits, const int32_t* tokens, const float* advantage,
                  const float* old, const float* ref, const float* weight, float* loss, float* logp, void* dlogits,
                  hipStream_t s) {
  Policy a;
  a.z = logits;
  a.tokens = tokens;
  a.advantage = advantage, a.old = old, a.ref = ref, a.weight = weight;
  a.loss = loss, a.logp = logp;
  a.dz = dlogits;
  a.z_stride = d.logit_stride;
  a.dz_stride = d.grad_stride;
  a.classes = (int)d.classes;
  a.past = d.rows * d.classes * (d.dtype == PNN_F32 ? 4 : 2) > L2_BYTES;
  a.tau = d.temperature;
  a.low = d.clip_low, a.high = d.clip_high;
  a.kl = d.kl;
  a.scale = d.scale;
  for (a.row0 = 0; a.row0 < d.rows; a.row0 += MAX_GRID) {
    const int64_t rows = d.rows - a.row0 < MAX_GRID ? d.rows - a.row0 : MAX_GRID;
    if (d.dtype == PNN_F32) launch_rows<float>(a, rows, s);
    else launch_rows<uint16_t>(a, rows, s);
    if (const hipError_t e = hipGetLastError()) return (int)e;
  }
  return 0;
}

}  // namespace pnn

// Distillation loss of a row of logits z against a teacher's top logits, and its gradient:
//   loss = alpha tau^2 sum_k p_k (log p_k - log q_{i_k}) + (1 - alpha) (-log s_y)
//   dz_v = scale w (alpha tau (q_v - sum_{i_k = v} p_k) + (1 - alpha) (s_v - [v = y]))
// with q = softmax(z / tau), s = softmax(z), p = softmax(teacher / tau).  One workgroup per row: a
// pass with a running maximum and two running sums (of exp((z - m) / tau) and exp(z - m)), then a
// pass that writes the gradient without the teacher's and the label's terms; the few classes that
// have such terms are written again by the thread of their first entry, from the logits gathered
// before anything was written.
#include "device_common.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int THREADS = 256;
constexpr int64_t MAX_GRID = 1 << 20;
constexpr float LOG2E = 1.44269504f, LN2 = 0.693147181f;

struct Distill {
  const void *z, *t;
  const int32_t *index, *labels;
  const float* weight;
  float* loss;
  void* dz;
  int64_t rows, z_stride, dz_stride, t_stride;
  int classes, top;
  float tau, alpha, scale;
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// maximum that keeps NaN
__device__ __forceinline__ float max_nan(float a, float b) { return a > b || a != a ? a : b; }

// sums of exp2((z - m) kq) and exp2((z - m) log2 e) with their maximum m; joining two empty ones stays empty
struct Stat {
  float m, q, s;
};
__device__ __forceinline__ Stat join(const Stat& a, const Stat& b, float kq) {
  Stat r;
  r.m = max_nan(a.m, b.m);
  const float da = a.m == r.m ? 0.0f : a.m - r.m, db = b.m == r.m ? 0.0f : b.m - r.m;
  r.q = a.q * exp2_(da * kq) + b.q * exp2_(db * kq);
  r.s = a.s * exp2_(da * LOG2E) + b.s * exp2_(db * LOG2E);
  return r;
}

template <typename T, typename TT>
__global__ __launch_bounds__(THREADS) void distill_kernel(Distill a) {
  __shared__ float et[PNN_DISTILL_MAX_TOP + 1];   // an entry's teacher logit, then its p; the label is entry `top`
  __shared__ float ez[PNN_DISTILL_MAX_TOP + 1];   // the student's logit of its class
  __shared__ int ei[PNN_DISTILL_MAX_TOP + 1];     // its class, -1: none
  __shared__ Stat wst[THREADS / 64];
  __shared__ float wred[THREADS / 64];
  __shared__ int bad;
  const int tid = threadIdx.x, wave = tid / 64, lane = tid & 63;
  const float kq = LOG2E / a.tau;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
  __syncthreads();                 // the row before has been read from LDS
  const int64_t z0 = row * a.z_stride, d0 = row * a.dz_stride;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int y = a.labels != nullptr ? a.labels[row] : -1;
  float tm = -INFINITY;
  for (int k = tid; k <= a.top; k += THREADS) {
    const int i = k < a.top ? a.index[row * a.t_stride + k] : y;
    const bool held = i >= 0 && i < a.classes;
    if (i >= a.classes) bad = 1;
    const float t = held && k < a.top ? St<TT>::ld(a.t, row * a.t_stride + k) : -INFINITY;
    ei[k] = held ? i : -1;
    ez[k] = held ? St<T>::ld(a.z, z0 + i) : 0.0f;
    et[k] = t;
    tm = max_nan(tm, t);
  }
  Stat st = {-INFINITY, 0.0f, 0.0f};
  for (int v = tid; v < a.classes; v += THREADS) st = join(st, Stat{St<T>::ld(a.z, z0 + v), 1.0f, 1.0f}, kq);
  for (int o = 32; o >= 1; o >>= 1) {
    const Stat b = {__shfl_xor(st.m, o, 64), __shfl_xor(st.q, o, 64), __shfl_xor(st.s, o, 64)};
    st = join(st, b, kq);
    tm = max_nan(tm, __shfl_xor(tm, o, 64));
  }
  if (lane == 0) {
    wst[wave] = st;
    wred[wave] = tm;
  }
  __syncthreads();
  st = wst[0];
  tm = wred[0];
  for (int w = 1; w < THREADS / 64; ++w) {
    st = join(st, wst[w], kq);
    tm = max_nan(tm, wred[w]);
  }
  const bool some = tm != -INFINITY;       // an entry with a finite (or NaN) teacher logit
  float ts = 0.0f;
  for (int k = tid; k < a.top; k += THREADS) ts += some ? exp2_((et[k] - tm) * kq) : 0.0f;
  ts = wave_sum(ts);
  __syncthreads();
  if (lane == 0) wred[wave] = ts;
  __syncthreads();
  ts = 0.0f;
  for (int w = 0; w < THREADS / 64; ++w) ts += wred[w];
  // loss: log p_k - log q_k = (t_k - tm) / tau - log ts - (z_k - m) / tau + log sum_q
  const float lq = logf(st.q), lt = logf(ts), inv_tau = 1.0f / a.tau;
  float kl = 0.0f;
  for (int k = tid; k < a.top; k += THREADS) {
    float p = 0.0f;
    if (some && ei[k] >= 0) {
      p = exp2_((et[k] - tm) * kq) / ts;
      if (p != 0.0f) kl += p * (((et[k] - tm) * inv_tau - lt) - ((ez[k] - st.m) * inv_tau - lq));
    }
    et[k] = p;
  }
  kl = wave_sum(kl);
  __syncthreads();
  if (lane == 0) wred[wave] = kl;
  __syncthreads();
  const bool hard = y >= 0;
  if (tid == 0) {
    float l = 0.0f;
    for (int w = 0; w < THREADS / 64; ++w) l += wred[w];
    l *= a.alpha * a.tau * a.tau;
    if (hard) l += (1.0f - a.alpha) * (logf(st.s) - (ez[a.top] - st.m));
    a.loss[row] = bad ? __builtin_nanf("") : l;
  }
  if (a.dz == nullptr) continue;
  if (!some && !hard && !bad) {    // neither term: no gradient, whatever the logits
    for (int v = tid; v < a.classes; v += THREADS) St<T>::st(a.dz, d0 + v, 0.0f);
    continue;
  }
  float g = a.scale * (a.weight != nullptr ? a.weight[row] : 1.0f);
  if (bad) g = __builtin_nanf("");
  const float gq = g * a.alpha * a.tau, gs = g * (1.0f - a.alpha);
  const float cq = (some || bad ? gq : 0.0f) / st.q, cs = (hard ? gs : 0.0f) / st.s;
  auto base = [&](float z) { return cq * exp2_((z - st.m) * kq) + cs * exp2_((z - st.m) * LOG2E); };
  for (int v = tid; v < a.classes; v += THREADS) St<T>::st(a.dz, d0 + v, base(St<T>::ld(a.z, z0 + v)));
  __syncthreads();
  for (int k = tid; k <= a.top; k += THREADS) {
    const int i = ei[k];
    if (i < 0) continue;
    bool first = true;
    float p = 0.0f;
    for (int j = 0; j < a.top; ++j)
      if (ei[j] == i) {
        if (j < k) first = false;
        p += et[j];
      }
    if (first) St<T>::st(a.dz, d0 + i, base(ez[k]) - gq * p - (i == y ? gs : 0.0f));
  }
  }
}

}  // namespace

int launch_distill(const pnn_distill_desc& d, const void* logits, const int32_t* index, const void* teacher,
                   const int32_t* labels, const float* weight, float* loss, void* dlogits, hipStream_t s) {
  Distill a;
  a.z = logits;
  a.t = teacher;
  a.index = index;
  a.labels = labels;
  a.weight = weight;
  a.loss = loss;
  a.dz = dlogits;
  a.rows = d.rows;
  a.z_stride = d.logit_stride;
  a.dz_stride = d.grad_stride;
  a.t_stride = d.top_stride;
  a.classes = (int)d.classes;
  a.top = (int)d.top;
  a.tau = d.temperature;
  a.alpha = d.alpha;
  a.scale = d.scale;
  const dim3 grid((unsigned)(d.rows < MAX_GRID ? d.rows : MAX_GRID)), block(THREADS);
#define ROWS(T)                                                                                                 \
  do {                                                                                                          \
    if (d.teacher_dtype == PNN_F32) hipLaunchKernelGGL((distill_kernel<T, float>), grid, block, 0, s, a);       \
    else hipLaunchKernelGGL((distill_kernel<T, uint16_t>), grid, block, 0, s, a);                               \
  } while (0)
  if (d.dtype == PNN_F32) ROWS(float);
  else ROWS(uint16_t);
#undef ROWS
  return (int)hipGetLastError();
}

}  // namespace pnn

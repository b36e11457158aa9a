// Gated linear recurrence: h_t = f_t h_{t-1} + (1 - f_t) x_t with f = sigmoid(gate), and its backward.
#include "device_common.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr int THREADS = 256;

// exp(x) for x <= 0 to about an ulp: x log2(e) in two floats, the low part to first order.
__device__ __forceinline__ float exp_neg(float x) {
  x = x < -120.0f ? -120.0f : x;           // exp(-120) rounds to 0 below; keeps NaN
  const float t = x * 1.44269502f;
  const float lo = fmaf(x, 1.44269502f, -t) + x * 1.92596299e-8f;
  const float r = __builtin_amdgcn_exp2f(t);
  return fmaf(r, lo * 0.693147181f, r);
}

// f = sigmoid(g) and keep = 1 - f, each to about an ulp: the smaller one is not formed by subtraction
__device__ __forceinline__ void gate_of(float g, float& f, float& keep) {
  const float e = exp_neg(-fabsf(g));
  const float d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = fmaf(fmaf(-d, r, 1.0f), r, r);
  const float s = e * r;
  f = g >= 0.0f ? r : s;
  keep = g >= 0.0f ? s : r;
}

__device__ __forceinline__ int64_t length_of(const int32_t* lengths, int64_t b, int64_t length) {
  if (lengths == nullptr) return length;
  const int64_t n = lengths[b];
  return n < 0 ? 0 : n > length ? length : n;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void scan_fwd_kernel(pnn_scan_desc d, ScanArgs a) {
  const int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (i >= d.batch * d.channels) return;
  const int64_t b = i / d.channels, c = i - b * d.channels;
  const int64_t len = length_of(a.lengths, b, d.length), chunks = (d.length + SCAN_CHUNK - 1) / SCAN_CHUNK;
  float h = a.h0 != nullptr ? a.h0[i] : 0.0f;
  for (int64_t t = 0; t < d.length; ++t) {
    if (a.states != nullptr && t % SCAN_CHUNK == 0) a.states[(b * chunks + t / SCAN_CHUNK) * d.channels + c] = h;
    if (t < len) {
      float f, keep;
      gate_of(St<T>::ld(a.gate, b * d.gate.batch + t * d.gate.step + c), f, keep);
      h = fmaf(f, h, keep * St<T>::ld(a.x, b * d.x.batch + t * d.x.step + c));
    }
    St<T>::st(a.h, b * d.h.batch + t * d.h.step + c, t < len ? h : 0.0f);
  }
  if (a.hT != nullptr) a.hT[i] = h;
}

template <typename T>
__global__ __launch_bounds__(THREADS) void scan_bwd_kernel(pnn_scan_desc d, ScanArgs a) {
  const int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x;
  if (i >= d.batch * d.channels) return;
  const int64_t b = i / d.channels, c = i - b * d.channels;
  const int64_t len = length_of(a.lengths, b, d.length), chunks = (d.length + SCAN_CHUNK - 1) / SCAN_CHUNK;
  float carry = a.dhT != nullptr ? a.dhT[i] : 0.0f;     // f_{t+1} G_{t+1}
  for (int64_t k = chunks - 1; k >= 0; --k) {
    float before[SCAN_CHUNK];
    float h = a.states[(b * chunks + k) * d.channels + c];
#pragma unroll
    for (int j = 0; j < SCAN_CHUNK; ++j) {
      const int64_t t = k * SCAN_CHUNK + j;
      before[j] = h;
      if (t < len) {
        float f, keep;
        gate_of(St<T>::ld(a.gate, b * d.gate.batch + t * d.gate.step + c), f, keep);
        h = fmaf(f, h, keep * St<T>::ld(a.x, b * d.x.batch + t * d.x.step + c));
      }
    }
#pragma unroll
    for (int j = SCAN_CHUNK - 1; j >= 0; --j) {
      const int64_t t = k * SCAN_CHUNK + j;
      float dx = 0.0f, dg = 0.0f;
      if (t < len) {
        float f, keep;
        gate_of(St<T>::ld(a.gate, b * d.gate.batch + t * d.gate.step + c), f, keep);
        const float G = St<T>::ld(a.dh, b * d.dh.batch + t * d.dh.step + c) + carry;
        dx = G * keep;
        dg = dx * f * (before[j] - St<T>::ld(a.x, b * d.x.batch + t * d.x.step + c));
        carry = f * G;
      }
      if (t < d.length) {
        St<T>::st(a.dx, b * d.dx.batch + t * d.dx.step + c, dx);
        St<T>::st(a.dgate, b * d.dgate.batch + t * d.dgate.step + c, dg);
      }
    }
  }
  if (a.dh0 != nullptr) a.dh0[i] = carry;
}

}  // namespace

int launch_scan_fwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)cdiv64(d.batch * d.channels, THREADS)), block(THREADS);
  if (d.dtype == PNN_F32) hipLaunchKernelGGL(scan_fwd_kernel<float>, grid, block, 0, s, d, a);
  else hipLaunchKernelGGL(scan_fwd_kernel<uint16_t>, grid, block, 0, s, d, a);
  return (int)hipGetLastError();
}

int launch_scan_bwd(const pnn_scan_desc& d, const ScanArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)cdiv64(d.batch * d.channels, THREADS)), block(THREADS);
  if (d.dtype == PNN_F32) hipLaunchKernelGGL(scan_bwd_kernel<float>, grid, block, 0, s, d, a);
  else hipLaunchKernelGGL(scan_bwd_kernel<uint16_t>, grid, block, 0, s, d, a);
  return (int)hipGetLastError();
}

}  // namespace pnn

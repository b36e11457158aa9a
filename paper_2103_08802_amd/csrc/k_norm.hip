// Norms before and after a block with its gate and the residual sum, and their backward:
//   a = w_post norm(x),  h = res + alpha a silu(gate),  y = w_pre norm(h),  norm(u) = u / sqrt(mean(u^2) + eps),
// each part optional.  Backward, with W elements a row, r = 1 / sqrt(mean(u^2) + eps), t the gradient of norm(u):
//   du = r (t - u r^2 sum(t u) / W);   silu'(g) = s (1 + g (1 - s)), s = sigmoid(g).
//
// A row belongs to TL lanes, NP 16-byte pieces a lane: it is loaded once, into registers.  Teams walk over the rows, so
// that weights are loaded once and the weights' gradients are summed in registers; teams of a workgroup are added up in
// LDS, workgroups by a second launch, each in a fixed order.  The sums that a row needs go over DPP, and over LDS where
// a row has more than a wave.
//
// Bound by memory.  bf16, 16384 rows of 2048 with a residual: forward 52 us (269 MB, 5.1 TB/s), backward 85 us (424 MB,
// 5.0 TB/s, 21 MB of it partial weight gradients) and 8.5 us to join these; one after the other the two take 95.7 us where
// h is formed and 89.9 where it is read.  262144 heads of 128 with a gate: forward 38 us (201 MB, 5.3 TB/s), backward 58 us
// (336 MB, 5.8 TB/s) and 5.  Rows are loaded when their turn comes: a row ahead in registers costs a wave a SIMD and gained
// nothing.  Stores of tensors larger than L2 go past it (heads' backward 107 us if they do not).
#include "device_common.h"
#include "seq_device.h"
#include "seq_internal.h"

namespace pnn {

namespace {

constexpr float LOG2E = 1.44269504f;

struct Norm {
  const void *x, *gate, *res, *dy, *dh;
  const float *w_post, *w_pre;
  void *h, *y, *dx, *dgate, *dres;
  float* part;                    // [workgroups][2][width]: partial gradients of w_post and w_pre
  pnn_row_stride xs, gs, rs, hs, ys, dys, dhs, dxs, dgs, drs;
  int total, heads, width;        // rows x heads, heads, elements of a row
  int post, pre, stored, dw_post, dw_pre, past;     // stored: res is h, as the forward stored it
  float eps, alpha, inv_width;
};

// a row's elements of a lane: piece p of lane l starts at element (p TL + l) VE; TAIL: the row's end may cut one
template <typename T, int TL, int NP, bool TAIL>
struct Cols {
  static constexpr int VE = St<T>::VE, N = NP * VE;
  static constexpr bool HELD = TAIL && TL < 1024;       // pieces stay packed until all are on their way
  static __device__ __forceinline__ int col(int p, int lane) { return (p * TL + lane) * VE; }
  // A row's pieces.  TAIL: still packed; the piece that the row's end cuts, and those behind it, are loaded so that they
  // end there, one load a piece and none under a condition of the lane.  118165 x 110 bf16, forward and backward: 90 us,
  // element by element in the lanes that the end cuts 144; 84495 x 206 98 and 150.  Whole pieces that way: 16384 x 2048
  // 163 and not 154.
  static __device__ __forceinline__ void load(const void* base, int64_t off, int lane, int width, uint4 (&r)[NP],
                                              float (&v)[N]) {
    const T* const row = (const T*)base + off;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = col(p, lane);
      if constexpr (!TAIL) {
        if (c < width) {
          load_piece<T>(base, off + c, v + p * VE);
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            v[p * VE + e] = 0.0f;
            asm volatile("" : "+v"(v[p * VE + e]));          // pieces unpacked here, not behind all loads: that spills
          }
        }
      } else if (width >= VE) {
        r[p] = __builtin_bit_cast(uint4, *(const typename Piece<T>::Mem*)(row + (c < width - VE ? c : width - VE)));
      } else {                                   // a row shorter than a piece
        uint32_t w[4] = {};
#pragma unroll
        for (int e = 0; e < VE; ++e)
          if (c + e < width) {
            if constexpr (sizeof(T) == 4) w[e] = __builtin_bit_cast(uint32_t, row[c + e]);
            else w[e / 2] |= (uint32_t)row[c + e] << (e % 2 * 16);
          }
        r[p] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    if constexpr (TAIL && !HELD) {               // 1024 lanes have no registers for two pieces' (one: not measured)
      unpack(r, lane, width, v);
#pragma unroll
      for (int e = 0; e < N; ++e) asm volatile("" : "+v"(v[e]));
    }
  }
  // their elements; zeros behind the row's end
  static __device__ __forceinline__ void open(const uint4 (&r)[NP], int lane, int width, float (&v)[N]) {
    if (HELD) unpack(r, lane, width, v);
  }
  static __device__ __forceinline__ void unpack(const uint4 (&r)[NP], int lane, int width, float (&v)[N]) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      uint4 u = r[p];
      const int k = col(p, lane) - (width - VE);             // elements of the piece that belong to the one before
      if (width >= VE && k > 0) {
        if constexpr (sizeof(T) == 4) {
          if (k & 2) u = make_uint4(u.z, u.w, 0, 0);
          if (k & 1) u = make_uint4(u.y, u.z, u.w, 0);
        } else {
          if (k & 4) u = make_uint4(u.z, u.w, 0, 0);
          if (k & 2) u = make_uint4(u.y, u.z, u.w, 0);
          if (k & 1) u = make_uint4(u.x >> 16 | u.y << 16, u.y >> 16 | u.z << 16, u.z >> 16 | u.w << 16, u.w >> 16);
        }
        if (k >= VE) u = make_uint4(0, 0, 0, 0);
      }
      Chunk<T> c;
      unpack_chunk<T>(u, c);
#pragma unroll
      for (int e = 0; e < VE; ++e) v[p * VE + e] = c.v[e];
    }
  }
  static __device__ __forceinline__ void store(void* base, int64_t off, int lane, int width, const float (&v)[N],
                                               bool past) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = col(p, lane);
      if (c + VE <= width) {
        store_piece<T>(base, off + c, v + p * VE, past);
      } else if (TAIL && c < width) {            // what is left of the row: 4, 2 and 1 elements
        T* to = (T*)base + off + c;
        const int n = width - c;
        float t[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) t[e] = v[p * VE + e];
#pragma unroll
        for (int h = VE / 2; h > 0; h /= 2)
          if (n & h) {
            typedef T Four __attribute__((ext_vector_type(4)));
            typedef T Two __attribute__((ext_vector_type(2)));
            typedef Four FourMem __attribute__((aligned(sizeof(T))));
            typedef Two TwoMem __attribute__((aligned(sizeof(T))));
            T o[VE];
#pragma unroll
            for (int e = 0; e < h; ++e) St<T>::st(o, e, t[e]);
            if (h == 4) *(FourMem*)to = Four{o[0], o[1], o[2], o[3]};
            else if (h == 2) *(TwoMem*)to = Two{o[0], o[1]};
            else *to = o[0];
            to += h;
#pragma unroll
            for (int e = 0; e + h < VE; ++e) t[e] = t[e + h];
          }
      }
    }
  }
  static __device__ __forceinline__ void weights(const float* w, int lane, int width, float (&v)[N]) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int c = col(p, lane) + e;
        v[p * VE + e] = c >= width ? 0.0f : w != nullptr ? w[c] : 1.0f;
      }
  }
};

// K sums over the lanes of a row, in every lane.  `flip` alternates between two places in LDS, so that one barrier a
// sum is enough.
template <int TL, int K>
__device__ __forceinline__ void row_sums(float (&v)[K], float (*lds)[16][K], int& flip) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
    if constexpr (TL == 16) {
      float s = v[k];
      s += dpp<0xB1>(s);
      s += dpp<0x4E>(s);
      s += dpp<0x141>(s);
      s += dpp<0x140>(s);
      v[k] = s;
    } else {
      v[k] = wave_add(v[k]);
    }
  }
  if constexpr (TL > 64) {
    const int wave = threadIdx.x / 64;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) lds[flip][wave][k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
      v[k] = 0.0f;
#pragma unroll
      for (int w = 0; w < TL / 64; ++w) v[k] += lds[flip][w][k];
    }
    flip ^= 1;
  }
}

// sigmoid, within about 2 + |g| roundings; 0 below -88
__device__ __forceinline__ float sigmoid(float g) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(g * -LOG2E));
}
// g s, with its limit for g = -inf
__device__ __forceinline__ float silu(float g, float s) { return s == 0.0f ? 0.0f : g * s; }
// s (1 + g (1 - s)), with its limits for g = -inf and inf
__device__ __forceinline__ float silu_slope(float g, float s) {
  return s == 0.0f ? 0.0f : s == 1.0f ? 1.0f : s * fmaf(g, 1.0f - s, 1.0f);
}
__device__ __forceinline__ float inverse_root(float mean, float eps) { return 1.0f / sqrtf(mean + eps); }
// r^2 mean(t u); 0 for a row that is normed to zeros, whose sum may be infinite
__device__ __forceinline__ float mean_part(float mean, float r) { return r == 0.0f ? 0.0f : mean * r * r; }

template <typename T, int TL, int NP, bool TAIL>
__global__ __launch_bounds__(TL < 256 ? 256 : TL) void norm_fwd_kernel(Norm a) {
  typedef Cols<T, TL, NP, TAIL> C;
  constexpr int N = C::N, TEAMS = TL < 256 ? 256 / TL : 1;
  __shared__ float lds[2][16][1];
  int flip = 0;
  const int lane = threadIdx.x % TL, W = a.width;
  float w1[N], w2[N];
  if (a.post) C::weights(a.w_post, lane, W, w1);
  if (a.pre) C::weights(a.w_pre, lane, W, w2);
  for (int r = blockIdx.x * TEAMS + threadIdx.x / TL; r < a.total; r += gridDim.x * TEAMS) {
    const int row = r / a.heads, head = r - row * a.heads;
    auto at = [&](const pnn_row_stride& s) { return row * s.row + head * s.head; };
    float x[N], g[N], h[N], s[1];
    uint4 xr[NP], gr[NP], hr[NP];
    C::load(a.x, at(a.xs), lane, W, xr, x);
    if (a.gate != nullptr) C::load(a.gate, at(a.gs), lane, W, gr, g);
    if (a.res != nullptr) C::load(a.res, at(a.rs), lane, W, hr, h);
    C::open(xr, lane, W, x);
    if (a.gate != nullptr) C::open(gr, lane, W, g);
    if (a.res != nullptr) C::open(hr, lane, W, h);
    if (a.post) {
      s[0] = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      row_sums<TL, 1>(s, lds, flip);
      const float r1 = inverse_root(s[0] * a.inv_width, a.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] = x[e] * r1 * w1[e];
    }
    if (a.gate != nullptr) {
#pragma unroll
      for (int e = 0; e < N; ++e) x[e] *= silu(g[e], sigmoid(g[e]));
    }
#pragma unroll
    for (int e = 0; e < N; ++e) h[e] = a.res != nullptr ? fmaf(a.alpha, x[e], h[e]) : a.alpha * x[e];
    if (a.h != nullptr) C::store(a.h, at(a.hs), lane, W, h, a.past);
    if (a.pre) {
      s[0] = 0.0f;
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(h[e], h[e], s[0]);
      row_sums<TL, 1>(s, lds, flip);
      const float r2 = inverse_root(s[0] * a.inv_width, a.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) h[e] = h[e] * r2 * w2[e];
      C::store(a.y, at(a.ys), lane, W, h, a.past);
    }
  }
}

template <typename T, int TL, int NP, bool GATE, bool TAIL>
__global__ __launch_bounds__(TL < 256 ? 256 : TL, norm_waves(TL, NP * St<T>::VE, TAIL)) void norm_bwd_kernel(Norm a) {
  typedef Cols<T, TL, NP, TAIL> C;
  constexpr int N = C::N, VE = C::VE, TEAMS = TL < 256 ? 256 / TL : 1;
  __shared__ float lds2[2][16][2], lds1[2][16][1];
  __shared__ float teams[TEAMS > 1 ? TEAMS * TL * N : 1];
  int flip2 = 0, flip1 = 0;
  const int lane = threadIdx.x % TL, W = a.width;
  // the weights: in registers, and their gradients beside them, four waves fit a SIMD and not five
  // (16384 x 2048 107 us and not 86)
  __shared__ __attribute__((aligned(16))) float weights[2][TL * N];
  float dw1[N] = {}, dw2[N] = {};
  for (int c = threadIdx.x; c < TL * N; c += blockDim.x) {
    weights[0][c] = c >= W ? 0.0f : a.w_post != nullptr ? a.w_post[c] : 1.0f;
    weights[1][c] = c >= W ? 0.0f : a.w_pre != nullptr ? a.w_pre[c] : 1.0f;
  }
  __syncthreads();
  auto weight = [&](int which, float (&w)[N]) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int e = 0; e < VE; e += 4) {
        typedef float f32x4_ __attribute__((ext_vector_type(4)));
        const f32x4_ v = *(const f32x4_*)&weights[which][C::col(p, lane) + e];
#pragma unroll
        for (int x = 0; x < 4; ++x) w[p * VE + e + x] = v[x];
      }
  };
#pragma unroll 1
  for (int r = blockIdx.x * TEAMS + threadIdx.x / TL; r < a.total; r += gridDim.x * TEAMS) {
    const int row = r / a.heads, head = r - row * a.heads;
    auto at = [&](const pnn_row_stride& s) { return row * s.row + head * s.head; };
    float x[N] = {}, g[N], h[N], t[N], d[N];
    uint4 xr[NP], gr[NP], hr[NP], tr[NP], dr[NP];
    if (a.x != nullptr) C::load(a.x, at(a.xs), lane, W, xr, x);
    if (GATE) C::load(a.gate, at(a.gs), lane, W, gr, g);
    if (a.pre) {
      if (a.res != nullptr) C::load(a.res, at(a.rs), lane, W, hr, h);
      C::load(a.dy, at(a.dys), lane, W, tr, t);
    }
    if (a.dh != nullptr) C::load(a.dh, at(a.dhs), lane, W, dr, d);
    if (a.x != nullptr) C::open(xr, lane, W, x);
    if (GATE) C::open(gr, lane, W, g);
    if (a.pre) {
      if (a.res != nullptr) C::open(hr, lane, W, h);
      C::open(tr, lane, W, t);
    }
    if (a.dh != nullptr) C::open(dr, lane, W, d);
    float r1 = 1.0f;
    if (a.post) {
      float s[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      row_sums<TL, 1>(s, lds1, flip1);
      r1 = inverse_root(s[0] * a.inv_width, a.eps);
    }
    if (a.dh == nullptr) {
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = 0.0f;
    }
    float w[N];
    if (a.pre) {
      if (!a.stored) {
        if (a.post) weight(0, w);
        // h as the forward formed it, before its rounding
#pragma unroll
        for (int e = 0; e < N; ++e) {
          float n = a.post ? x[e] * r1 * w[e] : x[e];
          if (GATE) n *= silu(g[e], sigmoid(g[e]));
          h[e] = a.res != nullptr ? fmaf(a.alpha, n, h[e]) : a.alpha * n;
        }
      }
      float s[2] = {0.0f, 0.0f};
      weight(1, w);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        s[0] = fmaf(h[e], h[e], s[0]);
        s[1] = fmaf(t[e] * w[e], h[e], s[1]);
      }
      row_sums<TL, 2>(s, lds2, flip2);
      const float r2 = inverse_root(s[0] * a.inv_width, a.eps), m2 = mean_part(s[1] * a.inv_width, r2);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        d[e] = fmaf(r2, fmaf(-h[e], m2, t[e] * w[e]), d[e]);
        dw2[e] = fmaf(t[e] * h[e], r2, dw2[e]);
      }
    }
    if (a.dres != nullptr) C::store(a.dres, at(a.drs), lane, W, d, a.past);
#pragma unroll
    for (int e = 0; e < N; ++e) d[e] *= a.alpha;
    if (a.post) weight(0, w);
    if (GATE) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float sg = sigmoid(g[e]), n = a.post ? x[e] * r1 * w[e] : x[e];
        h[e] = d[e] * n * silu_slope(g[e], sg);
        d[e] *= silu(g[e], sg);
      }
      if (a.dgate != nullptr) C::store(a.dgate, at(a.dgs), lane, W, h, a.past);
    }
    if (a.post) {
      float m[1] = {0.0f};
#pragma unroll
      for (int e = 0; e < N; ++e) {
        dw1[e] = fmaf(d[e] * x[e], r1, dw1[e]);
        d[e] *= w[e];
        m[0] = fmaf(d[e], x[e], m[0]);
      }
      row_sums<TL, 1>(m, lds1, flip1);
      const float m1 = mean_part(m[0] * a.inv_width, r1);
#pragma unroll
      for (int e = 0; e < N; ++e) d[e] = r1 * fmaf(-x[e], m1, d[e]);
    }
    if (a.dx != nullptr) C::store(a.dx, at(a.dxs), lane, W, d, a.past);
  }
  // the workgroup's sums: its teams in their order
  auto total = [&](float (&v)[N], int which) {
    if constexpr (TEAMS > 1) {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e) teams[(threadIdx.x / TL * N + e) * TL + lane] = v[e];
      __syncthreads();
      if (threadIdx.x >= TL) return;
#pragma unroll 1
      for (int j = 1; j < TEAMS; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] += teams[(j * N + e) * TL + lane];
    }
    float* const p = a.part + ((int64_t)blockIdx.x * 2 + which) * W;
#pragma unroll
    for (int x = 0; x < NP; ++x)
#pragma unroll
      for (int e = 0; e < VE; ++e) {
        const int c = C::col(x, lane) + e;
        if (c < W) p[c] = v[x * VE + e];
      }
  };
  if (a.dw_post) total(dw1, 0);
  if (a.dw_pre) total(dw2, 1);
}

// gradients of the weights: the workgroups' partial sums, 64 stretches of them side by side, then in order
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* part, int wgs, int width, float* dw_post,
                                                         float* dw_pre, int accumulate) {
  __shared__ float sums[64][16];
  const int which = blockIdx.y;
  float* const out = which ? dw_pre : dw_post;
  if (out == nullptr) return;
  const int c = blockIdx.x * 16 + threadIdx.x % 16, group = threadIdx.x / 16;
  float s = 0.0f;
  if (c < width) {
    const int per = (wgs + 63) / 64, end = (group + 1) * per < wgs ? (group + 1) * per : wgs;
#pragma unroll 8
    for (int j = group * per; j < end; ++j) s += part[((int64_t)j * 2 + which) * width + c];
  }
  sums[group][threadIdx.x % 16] = s;
  __syncthreads();
  if (group != 0 || c >= width) return;
#pragma unroll
  for (int j = 1; j < 64; ++j) s += sums[j][threadIdx.x];
  out[c] = accumulate ? out[c] + s : s;
}

Norm common(const pnn_norm_desc& d) {
  Norm a = {};
  a.xs = d.x, a.gs = d.gate, a.rs = d.res, a.hs = d.h, a.ys = d.y;
  a.dys = d.dy, a.dhs = d.dh, a.dxs = d.dx, a.dgs = d.dgate, a.drs = d.dres;
  a.total = (int)(d.rows * d.heads);
  a.heads = (int)d.heads;
  a.width = (int)d.width;
  a.post = d.post != 0;
  a.pre = d.pre != 0;
  a.past = d.rows * d.heads * d.width * (d.dtype == PNN_F32 ? 4 : 2) > L2_BYTES;
  a.eps = d.eps;
  a.alpha = d.alpha;
  a.inv_width = 1.0f / (float)d.width;
  return a;
}

template <typename T, int TL, int NP, bool TAIL>
void launch_one(const Norm& a, int wgs, bool backward, hipStream_t s) {
  const dim3 threads(TL < 256 ? 256 : TL);
  if (backward && a.gate != nullptr)
    hipLaunchKernelGGL((norm_bwd_kernel<T, TL, NP, true, TAIL>), dim3(wgs), threads, 0, s, a);
  else if (backward)
    hipLaunchKernelGGL((norm_bwd_kernel<T, TL, NP, false, TAIL>), dim3(wgs), threads, 0, s, a);
  else
    hipLaunchKernelGGL((norm_fwd_kernel<T, TL, NP, TAIL>), dim3(wgs), threads, 0, s, a);
}
template <typename T>
void launch_norm(const Norm& a, const NormShape& p, bool backward, hipStream_t s) {
  const int wgs = backward ? p.backward : p.forward;
#define NORM(TL, NP) \
  (p.tail ? launch_one<T, TL, NP, true>(a, wgs, backward, s) : launch_one<T, TL, NP, false>(a, wgs, backward, s))
  if (p.lanes == 16) { if (p.pieces == 1) NORM(16, 1); else NORM(16, 2); }
  else if (p.lanes == 64) { if (p.pieces == 1) NORM(64, 1); else NORM(64, 2); }
  else if (p.lanes == 256) { if (p.pieces == 1) NORM(256, 1); else NORM(256, 2); }
  else if (p.pieces == 1) NORM(1024, 1);
  else if (p.pieces == 2) NORM(1024, 2);
  else if constexpr (sizeof(T) == 4) NORM(1024, 4);
#undef NORM
}

}  // namespace

int launch_norm_fwd(const pnn_norm_desc& d, const void* x, const float* w_post, const void* gate, const void* res,
                    const float* w_pre, void* h, void* y, hipStream_t s) {
  Norm a = common(d);
  a.x = x, a.w_post = w_post, a.gate = gate, a.res = res, a.w_pre = w_pre, a.h = h, a.y = y;
  const NormShape p = norm_shape(d);
  if (d.dtype == PNN_F32) launch_norm<float>(a, p, false, s);
  else launch_norm<uint16_t>(a, p, false, s);
  return (int)hipGetLastError();
}

int launch_norm_bwd(const pnn_norm_desc& d, const void* x, const float* w_post, const void* gate, const void* res,
                    const float* w_pre, const void* dy, const void* dh, void* dx, void* dgate, void* dres,
                    float* dw_post, float* dw_pre, int accumulate, void* ws, hipStream_t s) {
  Norm a = common(d);
  a.x = x, a.w_post = w_post, a.gate = gate, a.res = res, a.w_pre = w_pre, a.dy = dy, a.dh = dh;
  a.dx = dx, a.dgate = dgate, a.dres = dres;
  a.stored = d.pre && d.stored;
  if (a.stored) a.rs = d.h;
  a.part = (float*)ws;
  a.dw_post = dw_post != nullptr;
  a.dw_pre = dw_pre != nullptr;
  NormShape p = norm_shape(d);
  if (a.total > 0) {
    if (d.dtype == PNN_F32) launch_norm<float>(a, p, true, s);
    else launch_norm<uint16_t>(a, p, true, s);
  } else {
    p.backward = 0;
  }
  if (a.dw_post || a.dw_pre)
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)cdiv64(d.width, 16), 2), dim3(1024), 0, s, a.part, p.backward,
                       a.width, dw_post, dw_pre, accumulate);
  return (int)hipGetLastError();
}

}  // namespace pnn

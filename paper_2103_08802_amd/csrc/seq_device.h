// Device-side helpers of the sequence operators.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace pnn {

// `bytes` behind an address that is the same for all lanes: a scalar address and a 32-bit lane offset.
// The empty asm pins each to its kind of register here; without it the compiler holds a 64-bit address
// a lane for every load in flight (the paired-channel recurrence backward then spills 250 bytes).
template <typename U, typename P>
__device__ __forceinline__ auto at(P* base, uint32_t bytes) {
  typedef typename std::conditional<std::is_const<U>::value, const char, char>::type B;
  __attribute__((address_space(1))) B* r = (__attribute__((address_space(1))) B*)base;
  asm volatile("" : "+s"(r), "+v"(bytes));
  return (__attribute__((address_space(1))) U*)(r + bytes);
}

// Stores of tensors larger than the L2 caches go past them (`past`): written through on their way, they would evict
// what is still to be read (distillation of 4096 x 65536 logits 255 -> 236 us, of 777 x 32771 33 -> 26 us).
constexpr int64_t L2_BYTES = 32 << 20;
template <typename V, typename P>
__device__ __forceinline__ void store_to(P* p, V v, bool past) {
  if (past) {
    asm volatile("");          // these two keep the stores from being merged into a plain one
    __builtin_nontemporal_store(v, p);
    asm volatile("");
  } else {
    *p = v;
  }
}

// 16-byte pieces of T that need no more than T's alignment (global memory takes unaligned vectors on this device)
template <typename T> struct Piece;
template <> struct Piece<float> {
  typedef float Vec __attribute__((ext_vector_type(4)));
  typedef Vec Mem __attribute__((aligned(4)));
};
template <> struct Piece<uint16_t> {
  typedef uint32_t Vec __attribute__((ext_vector_type(4)));
  typedef Vec Mem __attribute__((aligned(2)));
};
template <typename T>
__device__ __forceinline__ void load_piece(const void* base, int64_t i, float* v) {
  const typename Piece<T>::Vec u = *(const typename Piece<T>::Mem*)((const T*)base + i);
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = u[e];
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(u[e] << 16);
      v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
    }
  }
}
// past: as in store_to
template <typename T>
__device__ __forceinline__ void store_piece(void* base, int64_t i, const float* v, bool past) {
  typedef typename Piece<T>::Vec Vec;
  Vec u;
  if constexpr (sizeof(T) == 4) {
    u = Vec{v[0], v[1], v[2], v[3]};
  } else {
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 bf16x8_ __attribute__((ext_vector_type(8)));
    const f32x8 f = {v[0], v[1], v[2], v[3], v[4], v[5], v[6], v[7]};
    u = __builtin_bit_cast(Vec, __builtin_convertvector(f, bf16x8_));
  }
  if (past) {
    asm volatile("");
    __builtin_nontemporal_store(u, (typename Piece<T>::Mem*)((T*)base + i));
    asm volatile("");
  } else {
    *(typename Piece<T>::Mem*)((T*)base + i) = u;
  }
}

// The wave's sum / maximum in every lane, in a fixed order, without LDS: DPP exchanges within rows of 16 lanes, then
// the four rows by scalar reads.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <typename F>
__device__ __forceinline__ float wave_fold(float v, F f) {
  v = f(v, dpp<0xB1>(v));    // quad_perm 1 0 3 2
  v = f(v, dpp<0x4E>(v));    // quad_perm 2 3 0 1
  v = f(v, dpp<0x141>(v));   // row_half_mirror
  v = f(v, dpp<0x140>(v));   // row_mirror
  auto row = [&](int l) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), l)); };
  return f(f(row(0), row(16)), f(row(32), row(48)));
}
__device__ __forceinline__ float wave_add(float v) {
  return wave_fold(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float wave_max(float v) {
  return wave_fold(v, [](float a, float b) { return fmaxf(a, b); });
}

}  // namespace pnn

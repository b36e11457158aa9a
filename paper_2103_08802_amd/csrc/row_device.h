// Rows of classes, loaded into registers in 16-byte pieces: what the losses over logits share.
#pragma once

#include "device_common.h"
#include "seq_device.h"

namespace pnn {

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

}  // namespace pnn

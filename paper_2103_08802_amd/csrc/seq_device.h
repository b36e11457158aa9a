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

}  // namespace pnn

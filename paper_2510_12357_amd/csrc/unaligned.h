// Vectors read and written at the alignment of their elements: rows of an odd length start anywhere.  The hardware takes
// such 16-byte accesses as they are (they touch one cache line more).
#pragma once

#include <stdint.h>

namespace mm {
namespace {

template <typename E, int N>
struct __attribute__((packed, aligned(sizeof(E)))) Unaligned { E v[N]; };

template <typename V, typename E>
__device__ __forceinline__ V load_unaligned(const E* p) {
  typedef Unaligned<E, sizeof(V) / sizeof(E)> U;
  return __builtin_bit_cast(V, *reinterpret_cast<const U*>(p));
}
template <typename V, typename E>
__device__ __forceinline__ void store_unaligned(E* p, V v) {
  typedef Unaligned<E, sizeof(V) / sizeof(E)> U;
  *reinterpret_cast<U*>(p) = __builtin_bit_cast(U, v);
}

}  // namespace
}  // namespace mm

// What the kernels of the cross entropy from hidden states share.
#pragma once
#include <type_traits>

#include "common.cuh"

namespace szo {
namespace head {

#ifdef __CUDACC__
// For dW of fp16 the rows of G stand at 2^13 times their weight's power of two and those of h at that power over the largest
// one's: what is left of the product is 2^(exponent - 13).  (No row weighs anything: the sums are zeros.)
template <typename T> __device__ __forceinline__ float weight_of(const int32_t* exponent) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) return 1.f;
  const int e = *exponent;
  return e < -126 ? 1.f : __int_as_float((e - 13 + 127) << 23);
}
#endif

}  // namespace head
}  // namespace szo

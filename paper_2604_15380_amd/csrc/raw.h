// Values as they lie in memory, for loads that are to stay on their way: what
// ops.h's load_n converts it also waits for, where it branches on the row's end.
#pragma once

#include <type_traits>

#include "ops.h"

namespace ops {

// V values as they lie in memory: FP32 words, or two BF16 values per word.
template <class T, int V>
struct Raw {
  static constexpr int W = V * sizeof(T) < 4 ? 1 : V * sizeof(T) / 4;
  uint32_t w[W];
};
template <class T, int V>
__device__ __forceinline__ Raw<T, V> zero_raw() {
  Raw<T, V> r;
#pragma unroll
  for (int i = 0; i < Raw<T, V>::W; ++i) r.w[i] = 0;
  return r;
}
typedef uint32_t Words32 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t Words16 __attribute__((ext_vector_type(4), aligned(2)));
template <class T, int V, bool FULL>
__device__ __forceinline__ Raw<T, V> load_raw(const T* p, int left) {
  typedef typename std::conditional<sizeof(T) == 4, Words32, Words16>::type words;
  Raw<T, V> r = zero_raw<T, V>();
  if constexpr (V == 1) {
    if constexpr (sizeof(T) == 4) r.w[0] = *(const uint32_t*)p;
    else r.w[0] = *(const uint16_t*)p;
  } else if (FULL || left >= V) {
    const words v = *(const words*)p;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = v[i];
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < left) {
        if constexpr (sizeof(T) == 4) r.w[i] = ((const uint32_t*)p)[i];
        else r.w[i / 2] |= (uint32_t)((const uint16_t*)p)[i] << (16 * (i & 1));
      }
  }
  return r;
}
template <class T, int V>
__device__ __forceinline__ void unpack(const Raw<T, V>& r, float* x) {
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(r.w[i]);
    else x[i] = __uint_as_float(i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
  }
}

}  // namespace ops

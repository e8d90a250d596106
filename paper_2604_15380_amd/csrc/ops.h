// Shared by the head-tuning operators (norm.hip, dense.hip, optim.hip): typed
// loads and stores, wave sums, activations, their timing classes and their
// workspace.
#pragma once

#include "internal.h"

// timing classes, after those of the model's kernels
enum OpsKernelClass { KC_NORM = KC_COUNT, KC_NORM_BWD, KC_LINEAR, KC_LINEAR_BWD, KC_ADAMW, KC_ALL };

// Room for `need` bytes in the context's reverse-pass workspace.  PAINN_E_OOM
// where it cannot be had, or only by allocating while the stream is captured.
painn_status ops_workspace(painn_ctx* ctx, size_t need);

namespace ops {

inline painn_status fail(painn_ctx* ctx, painn_status st, const std::string& msg) {
  ctx->err = msg;
  return st;
}

// The status of what has been enqueued since the last hipGetLastError.
inline painn_status launched(painn_ctx* ctx, const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return PAINN_OK;
  return fail(ctx, PAINN_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Storage types.  The kernels compute in float.
using b16 = __bf16;

// V consecutive values.  Global memory takes 4- to 16-byte accesses at any
// alignment to the element, so rows of odd width need no form of their own.
template <class T, int V>
struct Pack {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

template <int V>
__device__ __forceinline__ void load(const float* p, float* x) {
  const typename Pack<float, V>::type v = *(const typename Pack<float, V>::type*)p;
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = v[i];
}
template <int V>
__device__ __forceinline__ void load(const b16* p, float* x) {
  const typename Pack<uint16_t, V>::type v = *(const typename Pack<uint16_t, V>::type*)p;
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = __uint_as_float((uint32_t)v[i] << 16);
}
template <int V>
__device__ __forceinline__ void store(float* p, const float* x) {
  typename Pack<float, V>::type v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = x[i];
  *(typename Pack<float, V>::type*)p = v;
}
// (to nearest even, as every rounding to BF16 here)
template <int V>
__device__ __forceinline__ void store(b16* p, const float* x) {
  typename Pack<b16, V>::type v;
#pragma unroll
  for (int i = 0; i < V; ++i) v[i] = (b16)x[i];
  *(typename Pack<b16, V>::type*)p = v;
}
// The first n of V values (n may be <= 0 or above V); what is not loaded is 0.
template <int V, class T>
__device__ __forceinline__ void load_n(const T* p, long long n, float* x) {
  if (n >= V) {
    load<V>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x[i] = 0.f;
      if (i < n) load<1>(p + i, x + i);
    }
  }
}
template <int V, class T>
__device__ __forceinline__ void store_n(T* p, long long n, const float* x) {
  if (n >= V) {
    store<V>(p, x);
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i)
      if (i < n) store<1>(p + i, x + i);
  }
}

// Sum over the wave's 64 lanes, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// activation(z) and its derivative, as written in painn.h
__device__ __forceinline__ float act(float z, int kind) {
  if (kind == PAINN_ACT_SILU) return z / (1.f + expf(-z));
  if (kind == PAINN_ACT_RELU) return z < 0.f ? 0.f : z;
  if (kind == PAINN_ACT_GELU) return 0.5f * z * (1.f + erff(z * 0.70710678118654752f));
  return z;
}
__device__ __forceinline__ float act_slope(float z, int kind) {
  if (kind == PAINN_ACT_SILU) {
    const float s = 1.f / (1.f + expf(-z));
    return s * (1.f + z * (1.f - s));
  }
  if (kind == PAINN_ACT_RELU) return z > 0.f ? 1.f : 0.f;
  if (kind == PAINN_ACT_GELU)
    return 0.5f * (1.f + erff(z * 0.70710678118654752f)) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
  return 1.f;
}

}  // namespace ops

// Shared by the head-tuning operators (norm.hip, dense.hip, optim.hip): typed
// loads and stores, wave sums, activations, their timing classes and their
// workspace.
#pragma once

#include "internal.h"

// timing classes, after those of the model's kernels
enum OpsKernelClass { KC_NORM = KC_COUNT, KC_NORM_BWD, KC_LINEAR, KC_LINEAR_BWD, KC_ADAMW, KC_ALL };

// Room for `need` bytes in the context's workspace ows.  PAINN_E_OOM
// where it cannot be had, or only by allocating while the stream is captured.
painn_status ops_workspace(painn_ctx* ctx, size_t need);

// The context ends: its optimizers refuse every further step.
void adamw_detach(painn_ctx* ctx);

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

// Whether an output that may lie in place of an input does so with other rows,
// which would be overwritten before they are read.
inline bool misplaced(const void* out, int64_t ldo, const void* in, int64_t ldi, int64_t rows) {
  return out && out == in && ldo != ldi && rows > 1;
}

// Threads that one launch holds along an axis of its grid.
constexpr long long LAUNCH_THREADS = 0xffffffffLL;

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
// Store 16-byte words past the caches, for outputs much larger than they are.
template <int V, class T>
__device__ __forceinline__ void store_past(T* p, const float* x) {
  typedef uint32_t word __attribute__((ext_vector_type(4)));
  constexpr int E = 16 / sizeof(T);
#pragma unroll
  for (int k = 0; k < V / E; ++k) {
    T v[E];
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = (T)x[k * E + i];
    word w;
    __builtin_memcpy(&w, v, 16);
    __builtin_nontemporal_store(w, (word*)(p + k * E));
  }
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

// Loads and stores of FP32 that pass the caches by.
template <int V>
__device__ __forceinline__ void load_past_n(const float* p, long long n, float* x) {
  if (n >= V) {
    const typename Pack<float, V>::type v = __builtin_nontemporal_load((const typename Pack<float, V>::type*)p);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = v[i];
  } else {
    load_n<V>(p, n, x);
  }
}
template <int V>
__device__ __forceinline__ void store_past_n(float* p, long long n, const float* x) {
  if (n >= V) {
    typename Pack<float, V>::type v;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = x[i];
    __builtin_nontemporal_store(v, (typename Pack<float, V>::type*)p);
  } else {
    store_n<V>(p, n, x);
  }
}

// Sum over the wave's 64 lanes, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
  for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// activation(z) and its derivative, as written in painn.h.  The exponentials
// and reciprocals are the hardware's (1 ulp): exp(-z) is off by |z| 2^-24 of
// itself, which leaves a sigmoid within 2^-23 absolute.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-z)); }

template <int N>
__device__ __forceinline__ void act(float* z, int kind) {
  if (kind == PAINN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] *= sigmoid(z[i]);
  } else if (kind == PAINN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];
  } else if (kind == PAINN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) z[i] = 0.5f * z[i] * (1.f + erff(z[i] * 0.70710678118654752f));
  }
}
// x *= activation'(z)
template <int N>
__device__ __forceinline__ void mul_slope(float* x, const float* z, int kind) {
  if (kind == PAINN_ACT_SILU) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float s = sigmoid(z[i]);
      x[i] *= s * (1.f + z[i] * (1.f - s));
    }
  } else if (kind == PAINN_ACT_RELU) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] *= z[i] > 0.f ? 1.f : 0.f;
  } else if (kind == PAINN_ACT_GELU) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i] *= 0.5f * (1.f + erff(z[i] * 0.70710678118654752f)) +
              z[i] * fast_exp(-0.5f * z[i] * z[i]) * 0.39894228040143268f;
  }
}

}  // namespace ops

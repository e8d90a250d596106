// The global norm of the gradients of many tensors, and clipping.
//
// One pass over the gradients for the norm: each block walks over pieces of
// 8,192 values of one tensor (a table made once says which) and adds squares in
// FP64, so that no square leaves the range and the sum's order costs no digits;
// the blocks' sums are added in their order.  Clipping is a second pass, or no
// pass at all where the optimizer's step takes the factor.  Bound by memory.
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "raw.h"

struct painn_grad_norm {
  painn_ctx* ctx = nullptr;       // null: the context has been destroyed
  painn_grad_norm *prev = nullptr, *next = nullptr;  // of the context's
  long long pieces = 0;
  bool outs = true;               // every tensor has a place for its clipped values
  void* table = nullptr;          // Piece [pieces], double [GRID]
  double* part = nullptr;
};

namespace {

using namespace ops;

constexpr int PIECE = 8192, GRID = 2048, TB = 256;

// Up to 8,192 consecutive values of a tensor.
struct Piece {
  const void* g;
  void* out;
  int n, bf16;
};

__device__ __forceinline__ double block_sum(double s, double* lds) {
#pragma unroll
  for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += lds[w];
  return s;
}

// A thread's values of a piece: all loads first.
template <class T>
struct Part {
  static constexpr int V = 16 / sizeof(T), STEPS = PIECE / (TB * V);
  Raw<T, V> r[STEPS];
  static __device__ __forceinline__ int at(int j) { return (j * TB + (int)threadIdx.x) * V; }
  __device__ __forceinline__ Part(const T* g, int n) {
    if (n == PIECE) {
#pragma unroll
      for (int j = 0; j < STEPS; ++j) r[j] = load_raw<T, V, true>(g + at(j), V);
    } else {
#pragma unroll
      for (int j = 0; j < STEPS; ++j) r[j] = at(j) < n ? load_raw<T, V, false>(g + at(j), n - at(j)) : zero_raw<T, V>();
    }
  }
};

template <class T>
__device__ __forceinline__ void add_squares(const T* g, int n, double* s) {
  typedef Part<T> P;
  const P p(g, n);
#pragma unroll
  for (int j = 0; j < P::STEPS; ++j) {
    float x[P::V];
    unpack<T, P::V>(p.r[j], x);
#pragma unroll
    for (int i = 0; i < P::V; ++i) {
      const double d = (double)x[i];
      s[i & 1] = __builtin_fma(d, d, s[i & 1]);
    }
  }
}

__global__ void __launch_bounds__(TB) k_grad_squares(const Piece* __restrict__ pieces, long long n,
                                                     double* __restrict__ part) {
  __shared__ double lds[TB / 64];
  double s[2] = {0.0, 0.0};
  Piece next = pieces[blockIdx.x];          // (there are as many pieces as blocks at least)
  for (long long k = blockIdx.x; k < n; k += gridDim.x) {
    const Piece c = next;
    if (k + gridDim.x < n) next = pieces[k + gridDim.x];
    if (c.bf16) add_squares((const b16*)c.g, c.n, s);
    else add_squares((const float*)c.g, c.n, s);
  }
  const double sum = block_sum(s[0] + s[1], lds);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}

// The factor that takes the norm to max_norm at most, from the blocks' sums; the
// block that is asked to writes result, the norm and the factor.
__device__ __forceinline__ float factor_of(const double* __restrict__ part, int n, double max_norm, bool write,
                                           float* __restrict__ result) {
  __shared__ double lds[TB / 64];
  double s = 0.0;
#pragma unroll 8
  for (int k = threadIdx.x; k < n; k += TB) s += part[k];
  const double norm = sqrt(block_sum(s, lds));
  const float f = norm != norm ? (float)norm : norm > max_norm ? (float)(max_norm / norm) : 1.f;
  if (write && threadIdx.x == 0) {
    result[0] = (float)norm;
    result[1] = f;
  }
  return f;
}
__global__ void __launch_bounds__(TB) k_grad_fold(const double* __restrict__ part, int n, double max_norm,
                                                  float* __restrict__ result) {
  factor_of(part, n, max_norm, true, result);
}

template <class T>
__device__ __forceinline__ void scale(const T* g, T* out, int n, float f) {
  typedef Part<T> P;
  const P p(g, n);
#pragma unroll
  for (int j = 0; j < P::STEPS; ++j) {
    float x[P::V];
    unpack<T, P::V>(p.r[j], x);
#pragma unroll
    for (int i = 0; i < P::V; ++i) x[i] *= f;
    if (n == PIECE) store<P::V>(out + P::at(j), x);
    else store_n<P::V>(out + P::at(j), n - P::at(j), x);
  }
}

// Every block adds the sums by itself, in the same order: less than a launch in
// between takes, and than a count of the blocks that have ended (67 M values: 14
// us for its 2,048 atomic additions).
__global__ void __launch_bounds__(TB) k_grad_scale(const Piece* __restrict__ pieces, long long n,
                                                   const double* __restrict__ part, int parts, double max_norm,
                                                   float* __restrict__ result) {
  Piece next = pieces[blockIdx.x];
  const float f = factor_of(part, parts, max_norm, blockIdx.x == 0, result);
  for (long long k = blockIdx.x; k < n; k += gridDim.x) {
    const Piece c = next;
    if (k + gridDim.x < n) next = pieces[k + gridDim.x];
    if (f == 1.f && c.out == c.g) continue;
    if (c.bf16) scale((const b16*)c.g, (b16*)c.out, c.n, f);
    else scale((const float*)c.g, (float*)c.out, c.n, f);
  }
}

painn_status norm_of(painn_grad_norm* h, double max_norm, float* result, bool clip) {
  if (!h || !h->ctx) return PAINN_E_ARG;
  painn_ctx* ctx = h->ctx;
  ctx->err.clear();
  if (!(max_norm >= 0.0)) return fail(ctx, PAINN_E_ARG, "max_norm must not be negative");
  if (!result) return fail(ctx, PAINN_E_ARG, "null result");
  if (clip && !h->outs) return fail(ctx, PAINN_E_ARG, "a tensor has no place for its clipped values");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  const Piece* pp = (const Piece*)h->table;
  const int grid = (int)(h->pieces < GRID ? h->pieces : GRID);
  prof_mark(ctx->prof, ctx->stream, KC_GRAD_NORM, true);
  if (grid) k_grad_squares<<<grid, TB, 0, ctx->stream>>>(pp, h->pieces, h->part);
  if (grid && clip) k_grad_scale<<<grid, TB, 0, ctx->stream>>>(pp, h->pieces, h->part, grid, max_norm, result);
  else k_grad_fold<<<1, TB, 0, ctx->stream>>>(h->part, grid, max_norm, result);
  prof_mark(ctx->prof, ctx->stream, KC_GRAD_NORM, false);
  return launched(ctx, "gradient norm launch");
}

}  // namespace

extern "C" {

painn_status painn_grad_norm_create(painn_ctx* ctx, int32_t n_tensors, const painn_grad_tensor* tensors,
                                    painn_grad_norm** out) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!out || n_tensors < 0 || (n_tensors > 0 && !tensors))
    return fail(ctx, PAINN_E_ARG, "null argument or negative tensor count");
  *out = nullptr;
  long long pieces = 0;
  bool outs = true;
  for (int k = 0; k < n_tensors; ++k) {
    const painn_grad_tensor& t = tensors[k];
    const std::string what = "tensor " + std::to_string(k);
    if (t.n < 0) return fail(ctx, PAINN_E_ARG, what + ": negative size");
    if (t.precision != PAINN_FP32 && t.precision != PAINN_BF16)
      return fail(ctx, PAINN_E_UNSUPPORTED, what + ": gradients are FP32 or BF16");
    if (t.reserved) return fail(ctx, PAINN_E_ARG, what + ": reserved is not 0");
    if (t.n > 0 && !t.grad) return fail(ctx, PAINN_E_ARG, what + ": null array");
    constexpr long long most = 0x7fffffffLL;
    if (t.n <= most * PIECE) pieces += (t.n + PIECE - 1) / PIECE;
    if (t.n > most * PIECE || pieces > most) return fail(ctx, PAINN_E_UNSUPPORTED, "2^31 or more pieces of 8192 values");
    outs = outs && (t.out || t.n == 0);
  }
  painn_grad_norm* h = nullptr;
  try {
    // what is written must be no other tensor's
    struct Range {
      uintptr_t a, b;
      int tensor, written;
    };
    std::vector<Range> ranges;
    for (int k = 0; k < n_tensors; ++k) {
      const painn_grad_tensor& t = tensors[k];
      const uintptr_t size = (uintptr_t)t.n * (t.precision == PAINN_BF16 ? 2 : 4);
      if (!size) continue;
      if (t.out != t.grad) ranges.push_back(Range{(uintptr_t)t.grad, (uintptr_t)t.grad + size, k, 0});
      if (t.out) ranges.push_back(Range{(uintptr_t)t.out, (uintptr_t)t.out + size, k, 1});
    }
    std::sort(ranges.begin(), ranges.end(), [](const Range& x, const Range& y) { return x.a < y.a; });
    // the farthest end so far of all ranges, and of the written ones
    uintptr_t end = 0, end_written = 0;
    for (const Range& r : ranges) {
      if (r.a < (r.written ? end : end_written))
        return fail(ctx, PAINN_E_ARG, "tensor " + std::to_string(r.tensor) + " overlaps one that clipping writes");
      end = std::max(end, r.b);
      if (r.written) end_written = std::max(end_written, r.b);
    }
    h = new (std::nothrow) painn_grad_norm();
    if (!h) return fail(ctx, PAINN_E_OOM, "host allocation failed");
    h->ctx = ctx;
    h->next = ctx->grad_norms;
    if (h->next) h->next->prev = h;
    ctx->grad_norms = h;
    h->pieces = pieces;
    h->outs = outs;
    const size_t list = align256((size_t)pieces * sizeof(Piece)), bytes = list + GRID * sizeof(double);
    std::vector<unsigned char> host(list);
    Piece* hp = (Piece*)host.data();
    for (int k = 0; k < n_tensors; ++k) {
      const painn_grad_tensor& t = tensors[k];
      const int size = t.precision == PAINN_BF16 ? 2 : 4;
      for (int64_t i = 0; i < t.n; i += PIECE)
        *hp++ = Piece{(const char*)t.grad + i * size, t.out ? (char*)t.out + i * size : nullptr,
                      (int)(t.n - i < PIECE ? t.n - i : PIECE), t.precision == PAINN_BF16};
    }
    (void)hipSetDevice(ctx->device);
    hipError_t e = hipMalloc(&h->table, bytes);
    if (e == hipSuccess && list) e = hipMemcpyAsync(h->table, host.data(), list, hipMemcpyHostToDevice, ctx->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(ctx->stream);
    if (e != hipSuccess) {
      (void)hipGetLastError();
      painn_grad_norm_free(h);
      return fail(ctx, PAINN_E_OOM, std::string("gradient table: ") + hipGetErrorString(e));
    }
    h->part = (double*)((char*)h->table + list);
  } catch (...) {
    if (h) painn_grad_norm_free(h);
    return fail(ctx, PAINN_E_OOM, "host allocation failed");
  }
  *out = h;
  return PAINN_OK;
}

painn_status painn_grad_norm_compute(painn_grad_norm* h, double max_norm, float* result) {
  return norm_of(h, max_norm, result, false);
}

painn_status painn_grad_norm_clip(painn_grad_norm* h, double max_norm, float* result) {
  return norm_of(h, max_norm, result, true);
}

painn_status painn_grad_norm_free(painn_grad_norm* h) {
  if (!h) return PAINN_OK;
  if (h->ctx) {
    (void)hipSetDevice(h->ctx->device);
    (void)hipStreamSynchronize(h->ctx->stream);
    if (h->prev) h->prev->next = h->next;
    else h->ctx->grad_norms = h->next;
    if (h->next) h->next->prev = h->prev;
  }
  if (h->table) (void)hipFree(h->table);
  delete h;
  return PAINN_OK;
}

}  // extern "C"

void grad_norm_detach(painn_ctx* ctx) {
  for (painn_grad_norm *h = ctx->grad_norms, *next; h; h = next) {
    next = h->next;
    h->ctx = nullptr;
    h->prev = h->next = nullptr;
  }
  ctx->grad_norms = nullptr;
}

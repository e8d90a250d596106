// AdamW over many tensors in one launch, states in FP32 or 8 bits.
//
// A step is one pass and bound by memory: with BF16 gradients and a BF16 copy
// FP32 states move 28 bytes per value, 8-bit states 16.  Each block has 1,024
// consecutive values of one tensor (a table made once says which), each lane
// four of them, so that the 256 values under one scale of the 8-bit states are
// one load of the wave.  Short blocks and many of them: 4,096 values per block,
// all loads first, took 67 us for 10.3 M values and 225 us for 67 M in 8 bits;
// this takes 57 and 190.  FP32 states pass the caches by, as nothing reads
// them before the next step: 57 -> 47 us (6.1 TB/s; a 1 GiB copy reaches 5.2).
// That is over three sets of arrays in turn, which the last-level cache holds in
// part; over twelve it is 53 us, 5.4 TB/s.
#include <float.h>
#include <math.h>

#include <new>

#include "ops.h"

struct painn_adamw {
  painn_ctx* ctx = nullptr;       // null: the context has been destroyed
  painn_adamw *prev = nullptr, *next = nullptr;      // of the context's optimizers
  painn_adamw_config cfg{};
  int64_t steps = 0;
  long long chunks = 0;
  void* table = nullptr;          // AdamTensor [n_tensors], then Chunk [chunks]
  const void* chunk_list = nullptr;
  bool copies = false;
};

namespace {

using namespace ops;

constexpr int CHUNK = 1024, QBLOCK = 256;
constexpr float QUNIT = 1.f / 448.f, QMIN = 0.001953125f;  // one over the largest e4m3 code; the smallest, 2^-9
constexpr float TINY = 1.17549435e-38f;                  // scales below this are stored as 0

struct AdamTensor {
  long long n;
  float* p;
  const void* g;
  b16* copy;
  void* m;
  void* v;
  float* ms;
  float* vs;
};
struct Chunk {
  int tensor, index;              // values [1024 index, 1024 (index + 1)) of the tensor
};
struct AdamScalars {
  float b1, a1, b2, a2;           // beta, 1 - beta
  float keep, step, down, eps;    // 1 - lr wd, lr / (1 - b1^t), 1 / sqrt(1 - b2^t), eps
};

// p, m and v of one value; every operation rounds as painn.h writes it (no
// contraction), so that a step's bits do not depend on the state's form.
__device__ __forceinline__ float adam(const AdamScalars& s, float& p, float g, float& m, float& v) {
#pragma clang fp contract(off)
  m = m * s.b1 + g * s.a1;
  v = v * s.b2 + (g * g) * s.a2;
  const float root = sqrtf(v);
  p = p * s.keep - (m * s.step) / (root * s.down + s.eps);
  return root;
}

// The largest magnitude of a wave's 256 values, as an integer: NaN stays above
// infinity.
__device__ __forceinline__ float wave_absmax(const float* x) {
  uint32_t u = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = __float_as_uint(x[i]) & 0x7fffffffu;
    u = u > w ? u : w;
  }
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    const uint32_t w = (uint32_t)__shfl_xor((int)u, o);
    u = u > w ? u : w;
  }
  return __uint_as_float(u);
}

// The codes of a wave's 256 values and their scale.  FLOOR: what is above
// zero gets at least the smallest code.
template <bool FLOOR>
__device__ __forceinline__ uint32_t encode(const float* x, float& scale) {
#pragma clang fp contract(off)
  scale = wave_absmax(x) * QUNIT;
  scale = scale < TINY ? 0.f : scale;
  const float inv = scale == 0.f ? 0.f : 1.f / scale;
  float q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[i] = x[i] * inv;
    if (FLOOR) q[i] = x[i] > 0.f && q[i] < QMIN ? QMIN : q[i];
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], w, true);
  return (uint32_t)w;
}

__device__ __forceinline__ void decode(uint32_t w, float scale, float* x) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0] * scale;
  x[1] = a[1] * scale;
  x[2] = b[0] * scale;
  x[3] = b[1] * scale;
}

// Up to four codes of a tensor whose last code may be fewer than four away.
__device__ __forceinline__ uint32_t load_codes(const uint8_t* p, long long n) {
  uint32_t w = 0;
  if (n >= 4) {
    __builtin_memcpy(&w, p, 4);
  } else {
    for (int i = 0; i < n; ++i) w |= (uint32_t)p[i] << (8 * i);
  }
  return w;
}
__device__ __forceinline__ void store_codes(uint8_t* p, long long n, uint32_t w) {
  if (n >= 4) {
    __builtin_memcpy(p, &w, 4);
  } else {
    for (int i = 0; i < n; ++i) p[i] = (uint8_t)(w >> (8 * i));
  }
}

template <class G, bool Q8>
__global__ void __launch_bounds__(256) k_adamw(const AdamTensor* __restrict__ tensors,
                                               const Chunk* __restrict__ chunks, AdamScalars s,
                                               const float* __restrict__ grad_scale) {
  const Chunk c = chunks[blockIdx.x];
  const AdamTensor t = tensors[c.tensor];
  const int lane = threadIdx.x & 63;
  const long long i = (long long)c.index * CHUNK + threadIdx.x * 4, b = i - lane * 4, left = t.n - i;
  float p[4], g[4], m[4], v[4], root[4];
  load_n<4>(t.p + i, left, p);
  load_n<4>((const G*)t.g + i, left, g);
  if (grad_scale) {
    const float f = *grad_scale;
#pragma unroll
    for (int e = 0; e < 4; ++e) g[e] = e < left ? g[e] * f : 0.f;
  }
  if constexpr (Q8) {
    const uint32_t mc = load_codes((const uint8_t*)t.m + i, left), vc = load_codes((const uint8_t*)t.v + i, left);
    decode(mc, b < t.n ? t.ms[b / QBLOCK] : 0.f, m);
    decode(vc, b < t.n ? t.vs[b / QBLOCK] : 0.f, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] *= v[e];
  } else {
    load_past_n<4>((const float*)t.m + i, left, m);
    load_past_n<4>((const float*)t.v + i, left, v);
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) root[e] = adam(s, p[e], g[e], m[e], v[e]);
  store_n<4>(t.p + i, left, p);
  if (t.copy) store_n<4>(t.copy + i, left, p);
  if constexpr (Q8) {
    // (past the tensor's end every value is 0 and stays 0)
    float scale_m, scale_v;
    const uint32_t cm = encode<false>(m, scale_m), cv = encode<true>(root, scale_v);
    store_codes((uint8_t*)t.m + i, left, cm);
    store_codes((uint8_t*)t.v + i, left, cv);
    if (lane == 0 && b < t.n) {
      t.ms[b / QBLOCK] = scale_m;
      t.vs[b / QBLOCK] = scale_v;
    }
  } else {
    store_past_n<4>((float*)t.m + i, left, m);
    store_past_n<4>((float*)t.v + i, left, v);
  }
}

constexpr int64_t STEPS_MAX = 1LL << 62;

bool in01(double b) { return b >= 0.0 && b < 1.0; }
// ... and as an FP32 value, which the kernel has
bool finite_at_least(double x, double lo) { return x >= lo && x <= FLT_MAX; }

}  // namespace

extern "C" {

painn_status painn_adamw_create(painn_ctx* ctx, int32_t n_tensors, const painn_adamw_tensor* tensors,
                                const painn_adamw_config* cfg, painn_adamw** out) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!out || !cfg || n_tensors < 0 || (n_tensors > 0 && !tensors))
    return fail(ctx, PAINN_E_ARG, "null argument or negative tensor count");
  *out = nullptr;
  const painn_adamw_config& c = *cfg;
  if (!in01(c.beta1) || !in01(c.beta2) || !finite_at_least(c.eps, 0.0) || !((float)c.eps > 0.f) ||
      !finite_at_least(c.weight_decay, 0.0) || c.steps < 0 || c.steps > STEPS_MAX)
    return fail(ctx, PAINN_E_ARG, "optimizer hyperparameters out of range");
  if (c.state_bits != 8 && c.state_bits != 32) return fail(ctx, PAINN_E_UNSUPPORTED, "state_bits is 8 or 32");
  if (c.grad_precision != PAINN_FP32 && c.grad_precision != PAINN_BF16)
    return fail(ctx, PAINN_E_UNSUPPORTED, "gradients are FP32 or BF16");
  long long chunks = 0;
  for (int k = 0; k < n_tensors; ++k) {
    const painn_adamw_tensor& t = tensors[k];
    if (t.n < 0) return fail(ctx, PAINN_E_ARG, "tensor " + std::to_string(k) + ": negative size");
    if (t.n > 0 && (!t.param || !t.grad || !t.m || !t.v || (c.state_bits == 8 && (!t.m_scale || !t.v_scale))))
      return fail(ctx, PAINN_E_ARG, "tensor " + std::to_string(k) + ": null array");
    constexpr long long most = LAUNCH_THREADS / 256;
    if (t.n <= most * CHUNK) chunks += (t.n + CHUNK - 1) / CHUNK;
    if (t.n > most * CHUNK || chunks > most)
      return fail(ctx, PAINN_E_UNSUPPORTED, "more blocks of 1024 values than a launch holds (2^24 - 1)");
  }
  painn_adamw* o = new (std::nothrow) painn_adamw();
  if (!o) return fail(ctx, PAINN_E_OOM, "host allocation failed");
  o->ctx = ctx;
  o->next = ctx->optimizers;
  if (o->next) o->next->prev = o;
  ctx->optimizers = o;
  o->cfg = c;
  o->steps = c.steps;
  o->chunks = chunks;
  if (chunks) {
    const size_t head = align256((size_t)n_tensors * sizeof(AdamTensor)), bytes = head + (size_t)chunks * sizeof(Chunk);
    unsigned char* host = new (std::nothrow) unsigned char[bytes]();
    if (!host) {
      painn_adamw_free(o);
      return fail(ctx, PAINN_E_OOM, "host allocation failed");
    }
    AdamTensor* ht = (AdamTensor*)host;
    Chunk* hc = (Chunk*)(host + head);
    for (int k = 0; k < n_tensors; ++k) {
      const painn_adamw_tensor& t = tensors[k];
      ht[k] = AdamTensor{t.n, t.param, t.grad, (b16*)t.copy, t.m, t.v, t.m_scale, t.v_scale};
      for (long long i = 0; i * CHUNK < t.n; ++i) *hc++ = Chunk{k, (int)i};
    }
    (void)hipSetDevice(ctx->device);
    hipError_t e = hipMalloc(&o->table, bytes);
    if (e == hipSuccess) e = hipMemcpyAsync(o->table, host, bytes, hipMemcpyHostToDevice, ctx->stream);
    if (e == hipSuccess) e = hipStreamSynchronize(ctx->stream);
    delete[] host;
    if (e != hipSuccess) {
      (void)hipGetLastError();
      painn_adamw_free(o);
      return fail(ctx, PAINN_E_OOM, std::string("optimizer table: ") + hipGetErrorString(e));
    }
    o->chunk_list = (const char*)o->table + head;
  }
  *out = o;
  return PAINN_OK;
}

painn_status painn_adamw_step(painn_adamw* opt, double lr) { return painn_adamw_step_scaled(opt, lr, nullptr); }

painn_status painn_adamw_step_scaled(painn_adamw* opt, double lr, const float* grad_scale) {
  if (!opt || !opt->ctx) return PAINN_E_ARG;
  painn_ctx* ctx = opt->ctx;
  ctx->err.clear();
  if (!finite_at_least(lr, 0.0)) return fail(ctx, PAINN_E_ARG, "lr must be finite and not negative");
  const painn_adamw_config& c = opt->cfg;
  const double t = (double)(opt->steps + 1);
  const AdamScalars s{(float)c.beta1, (float)(1.0 - c.beta1), (float)c.beta2, (float)(1.0 - c.beta2),
                      (float)(1.0 - lr * c.weight_decay), (float)(lr / (1.0 - pow(c.beta1, t))),
                      (float)(1.0 / sqrt(1.0 - pow(c.beta2, t))), (float)c.eps};
  // (an infinity times the 0 of a value without gradient would be NaN)
  if (!isfinite(s.keep) || !isfinite(s.step))
    return fail(ctx, PAINN_E_ARG, "lr is too large for FP32 (lr weight_decay, or lr / (1 - beta1^t))");
  if (opt->chunks) {
    (void)hipSetDevice(ctx->device);
    (void)hipGetLastError();
    const AdamTensor* tt = (const AdamTensor*)opt->table;
    const Chunk* cc = (const Chunk*)opt->chunk_list;
    const dim3 grid((unsigned)opt->chunks);
    const bool q8 = c.state_bits == 8, g16 = c.grad_precision == PAINN_BF16;
    prof_mark(ctx->prof, ctx->stream, KC_ADAMW, true);
    if (q8 && g16) k_adamw<b16, true><<<grid, 256, 0, ctx->stream>>>(tt, cc, s, grad_scale);
    else if (q8) k_adamw<float, true><<<grid, 256, 0, ctx->stream>>>(tt, cc, s, grad_scale);
    else if (g16) k_adamw<b16, false><<<grid, 256, 0, ctx->stream>>>(tt, cc, s, grad_scale);
    else k_adamw<float, false><<<grid, 256, 0, ctx->stream>>>(tt, cc, s, grad_scale);
    prof_mark(ctx->prof, ctx->stream, KC_ADAMW, false);
    const painn_status st = launched(ctx, "optimizer step launch");
    if (st != PAINN_OK) return st;
  }
  ++opt->steps;
  return PAINN_OK;
}

painn_status painn_adamw_steps(const painn_adamw* opt, int64_t* steps) {
  if (!opt || !steps) return PAINN_E_ARG;
  *steps = opt->steps;
  return PAINN_OK;
}

painn_status painn_adamw_free(painn_adamw* opt) {
  if (!opt) return PAINN_OK;
  if (opt->ctx) {
    (void)hipSetDevice(opt->ctx->device);
    (void)hipStreamSynchronize(opt->ctx->stream);
    if (opt->prev) opt->prev->next = opt->next;
    else opt->ctx->optimizers = opt->next;
    if (opt->next) opt->next->prev = opt->prev;
  }
  if (opt->table) (void)hipFree(opt->table);
  delete opt;
  return PAINN_OK;
}

}  // extern "C"

void adamw_detach(painn_ctx* ctx) {
  for (painn_adamw *o = ctx->optimizers, *next; o; o = next) {
    next = o->next;
    o->ctx = nullptr;
    o->prev = o->next = nullptr;
  }
  ctx->optimizers = nullptr;
}

// The gate: a row's softmax over the heads, its k largest heads, the heads'
// counts and mean probabilities and the balance loss, and the reverse pass
// (FP32, BF16 logits).
//
// A row is held by LPR lanes, NJ times V values (16 bytes) each, so that its
// softmax and its largest heads need nothing but registers and exchanges
// between those lanes.  Up to KREG heads are chosen one after the other, the
// largest key of the row each time (the key carries the head's number, so that
// ties go to the lowest); for more, every value counts the keys above its own,
// which gives its place at once whatever k is.  Counts and sums of
// probabilities stay in the block until its last row; the blocks' partial rows
// are then added in their order.  Bound by memory, or by the launch.
#include <math.h>

#include <type_traits>

#include "ops.h"

namespace {

using namespace ops;

constexpr int KREG = 8;             // heads chosen one after the other
constexpr int HEADS = 1024;         // heads at most
constexpr int GATE_GRID = 256;      // blocks of the forward, whose sums are folded

struct GateArgs {
  long long rows;
  int heads, k, normalize;
  const void* x;
  long long ldx;
  float* weights;
  int* indices;
  int* counts;                      // [heads + 1], the last: rows with a head
  float *share, *loss;
  float* part_p;                    // [blocks][heads]
  int* part_c;                      // [blocks][heads + 1]
  // reverse pass
  const float* dw;
  const int* chosen;
  const int* n;
  double balance;
  void* dx;
  long long lddx;
};

// exp(d) for d <= 0 to 2 ulp: the product d log2 e is carried to both halves.
__device__ __forceinline__ float exp_of(float d) {
  const float c = d < -200.f ? -200.f : d;
  const float t = c * 1.44269504f;
  const float lo = __builtin_fmaf(c, 1.92596299e-8f, __builtin_fmaf(c, 1.44269504f, -t));
  const float e = __builtin_amdgcn_exp2f(t);
  return __builtin_fmaf(e, lo * 0.69314718f, e);
}

// Keys in the values' order; NaN above infinity, -0 as 0; 0 is below every key.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}
template <class T>
struct Key;
template <>
struct Key<float> {
  typedef unsigned long long type;
  static __device__ __forceinline__ type make(float x, int e) {
    return ((type)ordered(x) << 32) | (uint32_t)(0xffffffffu - (uint32_t)e);
  }
  static __device__ __forceinline__ float value(type k) { return value_of((uint32_t)(k >> 32)); }
  static __device__ __forceinline__ int head(type k) { return (int)(0xffffffffu - (uint32_t)k); }
};
template <>
struct Key<b16> {                   // BF16 has 16 bits, which leaves 16 for the head
  typedef uint32_t type;
  static __device__ __forceinline__ type make(float x, int e) {
    return (ordered(x) & 0xffff0000u) | (0xffffu - (uint32_t)e);
  }
  static __device__ __forceinline__ float value(type k) {
    const uint32_t o = k & 0xffff0000u;
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o & 0xffff0000u);
  }
  static __device__ __forceinline__ int head(type k) { return (int)(0xffffu - (k & 0xffffu)); }
};

template <int LPR>
__device__ __forceinline__ float lanes_sum(float x) {
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) x += __shfl_xor(x, o);
  return x;
}

// A row's softmax, held by LPR lanes.
template <class T, int NJ, int LPR>
struct Row {
  static constexpr int V = 16 / sizeof(T), N = NJ * V;
  float x[N];                       // logits; past the heads -infinity
  float e[N];                       // exp(x - top); 0 past the heads
  float top, inv;                   // largest logit (0 for a row of none), 1 / sum of e
  bool some;                        // a head can be taken
  static __device__ __forceinline__ int head(int lane, int i) { return (i / V * LPR + lane) * V + i % V; }
  __device__ __forceinline__ Row(const void* p, long long ld, long long row, bool live, int heads, int lane) {
    float most = -INFINITY;
    bool any = false;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + lane) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) x[j * V + i] = -INFINITY;
      if (live && c < heads) {
        float v[V];
        load_n<V>((const T*)p + row * ld + c, heads - c, v);
#pragma unroll
        for (int i = 0; i < V; ++i) x[j * V + i] = c + i < heads ? v[i] : -INFINITY;
      }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      any |= !(x[i] == -INFINITY);
      most = fmaxf(most, x[i]);
    }
    int a = any;
#pragma unroll
    for (int o = LPR / 2; o; o >>= 1) {
      most = fmaxf(most, __shfl_xor(most, o));
      a |= __shfl_xor(a, o);
    }
    some = a != 0;
    top = most > -INFINITY ? most : 0.f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      e[i] = exp_of(x[i] - top);
      s += e[i];
    }
    s = lanes_sum<LPR>(s);
    inv = some ? 1.f / s : 0.f;
  }
};

// The totals of all blocks' (or one block's) sums: counts, share, loss.  red:
// [blockDim.x] doubles.
__device__ void totals(const GateArgs& a, int blocks, const float* pp, const int* pc, double* red) {
  const int t = threadIdx.x, n = blockDim.x;
  __shared__ int routed, chosen;
  __shared__ double loss;
  if (t == 0) { routed = 0; chosen = 0; }
  __syncthreads();
  int r = 0;
  for (int b = t; b < blocks; b += n) r += pc[(size_t)b * (a.heads + 1) + a.heads];
  if (r) atomicAdd(&routed, r);
  // a head's partial sums in `slices` parts
  int width = 1;
  while (width < a.heads && width < n) width <<= 1;
  const int slices = n / width, l = t & (width - 1), q = t / width;
  double mine = 0.0;                // sum over this thread's heads of counts * sums of p
  for (int h0 = 0; h0 < a.heads; h0 += width) {
    const int h = h0 + l;
    double p = 0.0;
    int c = 0;
    if (h < a.heads)
      for (int b = q; b < blocks; b += slices) {
        p += (double)pp[(size_t)b * a.heads + h];
        c += pc[(size_t)b * (a.heads + 1) + h];
      }
    __syncthreads();
    red[t] = p;
    __syncthreads();
    p = 0.0;
    if (q == 0)
      for (int k = 0; k < slices; ++k) p += red[k * width + l];
    __syncthreads();
    ((int*)red)[t] = c;
    __syncthreads();
    if (q == 0 && h < a.heads) {
      c = 0;
      for (int k = 0; k < slices; ++k) c += ((int*)red)[k * width + l];
      a.counts[h] = c;
      atomicAdd(&chosen, c);
      const double share = routed ? p / routed : 0.0;
      a.share[h] = (float)share;
      mine += share * c;
    }
  }
  __syncthreads();
  red[t] = mine;
  __syncthreads();
  if (t < 64) {
    mine = 0.0;
    for (int k = t; k < n; k += 64) mine += red[k];
#pragma unroll
    for (int o = 32; o; o >>= 1) mine += __shfl_xor(mine, o);
    if (t == 0) {
      a.counts[a.heads] = routed;
      a.loss[0] = chosen ? (float)(mine * a.heads / chosen) : 0.f;
    }
  }
}

__global__ void __launch_bounds__(1024) k_gate_fold(GateArgs a, int blocks) {
  __shared__ double red[1024];
  totals(a, blocks, a.part_p, a.part_c, red);
}

// MANY: more than KREG heads of a row.
template <class T, int NJ, int LPR, bool MANY>
__global__ void __launch_bounds__(1024) k_gate(GateArgs a) {
  typedef Row<T, NJ, LPR> R;
  typedef Key<T> K;
  constexpr int N = R::N, ACROSS = LPR * N;
  // counts [heads + 1]; then the waves' sums of p, or the rows' keys
  extern __shared__ int lds[];
  __shared__ double red[1024];
  int* cnt = lds;
  const int rpb = blockDim.x / LPR, lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  uint32_t* keys = (uint32_t*)(lds + a.heads + 1) + sub * ACROSS;
  for (int h = threadIdx.x; h <= a.heads; h += blockDim.x) cnt[h] = 0;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  __syncthreads();
  int routed = 0;
  for (long long r0 = (long long)blockIdx.x * rpb; r0 < a.rows; r0 += (long long)gridDim.x * rpb) {
    const long long row = r0 + sub;
    const bool live = row < a.rows;
    const R r(a.x, a.ldx, row, live, a.heads, lane);
    float* w = a.weights + row * a.k;
    int* id = a.indices + row * a.k;
    if (r.some) {
      routed += lane == 0;
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += r.e[i] * r.inv;
    }
    if constexpr (!MANY) {
      typename K::type key[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int h = R::head(lane, i);
        key[i] = h < a.heads ? K::make(r.x[i], h) : 0;
      }
      float ws[KREG];
      int is[KREG];
      float total = 0.f;
#pragma unroll
      for (int s = 0; s < KREG; ++s) {
        ws[s] = 0.f;
        is[s] = -1;
        if (s < a.k) {
          typename K::type best = key[0];
#pragma unroll
          for (int i = 1; i < N; ++i) best = key[i] > best ? key[i] : best;
#pragma unroll
          for (int o = LPR / 2; o; o >>= 1) {
            const typename K::type other = __shfl_xor(best, o);
            best = other > best ? other : best;
          }
#pragma unroll
          for (int i = 0; i < N; ++i) key[i] = key[i] == best ? 0 : key[i];
          const float x = K::value(best);
          if (!(x == -INFINITY)) {
            is[s] = K::head(best);
            ws[s] = exp_of(x - r.top);
            total += ws[s];
          }
        }
      }
      if (live) {
        const float f = a.normalize ? (r.some ? 1.f / total : 0.f) : r.inv;
#pragma unroll
        for (int s = 0; s < KREG; ++s)
          if (s < a.k && s % LPR == lane) {
            w[s] = ws[s] * f;
            id[s] = is[s];
            if (is[s] >= 0) atomicAdd(&cnt[is[s]], 1);
          }
      }
    } else {
      __syncthreads();
      int places = 0;               // values that are not -infinity
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int h = R::head(lane, i);
        keys[h] = h < a.heads ? ordered(r.x[i]) : 0;
        places += !(r.x[i] == -INFINITY);
      }
#pragma unroll
      for (int o = LPR / 2; o; o >>= 1) places += __shfl_xor(places, o);
      __syncthreads();
      int rank[N];
#pragma unroll
      for (int i = 0; i < N; ++i) rank[i] = 0;
      for (int h = 0; h < a.heads; ++h) {
        const uint32_t other = keys[h];
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const uint32_t own = ordered(r.x[i]);
          rank[i] += other > own || (other == own && h < R::head(lane, i));
        }
      }
      float total = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (rank[i] < a.k && !(r.x[i] == -INFINITY)) total += r.e[i];
      total = lanes_sum<LPR>(total);
      if (live) {
        const float f = a.normalize ? (r.some ? 1.f / total : 0.f) : r.inv;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (rank[i] < a.k && !(r.x[i] == -INFINITY)) {
            const int h = R::head(lane, i);
            w[rank[i]] = r.e[i] * f;
            id[rank[i]] = h;
            atomicAdd(&cnt[h], 1);
          }
        for (int s = places + lane; s < a.k; s += LPR) {
          w[s] = 0.f;
          id[s] = -1;
        }
      }
    }
  }
  // the block's sums of p, wave by wave
  if (routed) atomicAdd(&cnt[a.heads], routed);
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int o = LPR; o < 64; o <<= 1) sum[i] += __shfl_xor(sum[i], o);
  __syncthreads();
  float* waves = (float*)(lds + a.heads + 1);
  if ((threadIdx.x & 63) < LPR)
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int h = R::head(lane, i);
      if (h < a.heads) waves[(threadIdx.x >> 6) * a.heads + h] = sum[i];
    }
  __syncthreads();
  if (gridDim.x == 1) {
    // (waves' sums as partial rows of p; the counts are whole)
    for (int h = threadIdx.x; h < a.heads; h += blockDim.x) {
      float s = 0.f;
      for (int k = 0; k < (int)blockDim.x / 64; ++k) s += waves[k * a.heads + h];
      waves[h] = s;
    }
    __syncthreads();
    totals(a, 1, waves, cnt, red);
    return;
  }
  for (int h = threadIdx.x; h < a.heads; h += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < (int)blockDim.x / 64; ++k) s += waves[k * a.heads + h];
    a.part_p[(size_t)blockIdx.x * a.heads + h] = s;
  }
  for (int h = threadIdx.x; h <= a.heads; h += blockDim.x) a.part_c[(size_t)blockIdx.x * (a.heads + 1) + h] = cnt[h];
}

// With p the softmax, f = counts / their sum and R the rows that have a head:
//   dp = balance heads / R f (+ dw at the chosen heads, not normalised),
//   dx = p (dp - sum p dp);  normalised, w the chosen heads' own softmax:
//   dx += w (dw - sum w dw).
template <class T, int NJ, int LPR>
__global__ void __launch_bounds__(256) k_gate_bwd(GateArgs a) {
  typedef Row<T, NJ, LPR> R;
  constexpr int N = R::N, V = R::V;
  const int rpb = 256 / LPR, lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  float f[N];
  int all = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int h = R::head(lane, i), c = h < a.heads ? a.n[h] : 0;
    f[i] = (float)c;
    all += c;
  }
#pragma unroll
  for (int o = LPR / 2; o; o >>= 1) all += __shfl_xor(all, o);
  const int routed = a.n[a.heads];
  const float scale = all > 0 && routed > 0 ? (float)(a.balance * a.heads / ((double)routed * all)) : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] *= scale;
  for (long long r0 = (long long)blockIdx.x * rpb; r0 < a.rows; r0 += (long long)gridDim.x * rpb) {
    const long long row = r0 + sub;
    const bool live = row < a.rows;
    const R r(a.x, a.ldx, row, live, a.heads, lane);
    float d[N];
    uint32_t mark = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = 0.f;
    if (a.dw && live)
      for (int s0 = 0; s0 < a.k; s0 += KREG) {
        int is[KREG];
        float ds[KREG];
#pragma unroll
        for (int s = 0; s < KREG; ++s) {
          is[s] = -1;
          ds[s] = 0.f;
          if (s0 + s < a.k) {
            is[s] = a.chosen[row * a.k + s0 + s];
            ds[s] = a.dw[row * a.k + s0 + s];
          }
        }
#pragma unroll
        for (int s = 0; s < KREG; ++s)
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (is[s] == R::head(lane, i)) {
              d[i] += ds[s];
              mark |= 1u << i;
            }
      }
    float dot = 0.f, dotw = 0.f, total = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool on = mark >> i & 1;
      const float p = r.e[i] * r.inv;
      dot += p * (a.normalize ? f[i] : f[i] + d[i]);
      if (on) {
        total += r.e[i];
        dotw += r.e[i] * d[i];
      }
    }
    dot = lanes_sum<LPR>(dot);
    float invw = 0.f;
    if (a.normalize) {
      total = lanes_sum<LPR>(total);
      invw = total > 0.f || total != total ? 1.f / total : 0.f;
      dotw = lanes_sum<LPR>(dotw) * invw;
    }
    float o[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool on = mark >> i & 1;
      const float p = r.e[i] * r.inv;
      o[i] = p * ((a.normalize ? f[i] : f[i] + d[i]) - dot);
      if (a.normalize && on) o[i] += r.e[i] * invw * (d[i] - dotw);
      if (r.x[i] == -INFINITY || !r.some) o[i] = 0.f;
    }
    if (live)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int c = (j * LPR + lane) * V;
        if (c < a.heads) store_n<V>((T*)a.dx + row * a.lddx + c, a.heads - c, o + j * V);
      }
  }
}

// Calls f(NJ, LPR) with the fewest lanes that hold a row of `heads`.
template <class T, class F>
void gate_form(int heads, F&& f) {
  constexpr int V = 16 / sizeof(T);
#define GATE_FORM(NJ, LPR) \
  if (heads <= NJ * LPR * V) return f(std::integral_constant<int, NJ>(), std::integral_constant<int, LPR>());
  GATE_FORM(1, 1)
  GATE_FORM(1, 2)
  GATE_FORM(1, 4)
  GATE_FORM(1, 8)
  GATE_FORM(1, 16)
  GATE_FORM(1, 32)
  GATE_FORM(1, 64)
  GATE_FORM(2, 64)
  if constexpr (sizeof(T) == 4) { GATE_FORM(4, 64) }
#undef GATE_FORM
}

int lanes_of(bool bf16, int heads) {
  const int v = bf16 ? 8 : 4;
  int l = 1;
  while (l < 64 && l * v < heads) l <<= 1;
  return l;
}
// Blocks and threads of the forward: one block while it has few rows.
void gate_grid(bool bf16, long long rows, int heads, int k, int& blocks, int& threads) {
  const int lpr = lanes_of(bf16, heads);
  const bool many = k > KREG;       // (the rows' keys fit LDS for 256 threads)
  blocks = 1;
  threads = many ? 256 : 1024;
  if (rows * lpr <= 2048) return;
  if (rows * lpr <= 256LL * GATE_GRID) threads = 256;
  const long long n = (rows * lpr + threads - 1) / threads;
  blocks = (int)(n < GATE_GRID ? n : GATE_GRID);
}
size_t gate_bytes(int blocks, int heads) {
  return blocks > 1 ? align256((size_t)blocks * heads * 4) + align256((size_t)blocks * (heads + 1) * 4) : 0;
}

template <class T>
painn_status run_gate(painn_ctx* ctx, const GateArgs& a, int blocks, int threads) {
  prof_mark(ctx->prof, ctx->stream, KC_GATE, true);
  gate_form<T>(a.heads, [&](auto nj, auto lanes) {
    constexpr int NJ = decltype(nj)::value, LPR = decltype(lanes)::value, N = NJ * 16 / sizeof(T);
    const bool many = a.k > KREG;
    const size_t keys = many ? (size_t)threads * N : 0, waves = (size_t)(threads / 64) * a.heads;
    const size_t lds = (a.heads + 1 + (keys > waves ? keys : waves)) * 4;
    if (many) k_gate<T, NJ, LPR, true><<<blocks, threads, lds, ctx->stream>>>(a);
    else k_gate<T, NJ, LPR, false><<<blocks, threads, lds, ctx->stream>>>(a);
  });
  if (blocks > 1) k_gate_fold<<<1, 1024, 0, ctx->stream>>>(a, blocks);
  prof_mark(ctx->prof, ctx->stream, KC_GATE, false);
  return launched(ctx, "gate launch");
}

template <class T>
painn_status run_gate_bwd(painn_ctx* ctx, const GateArgs& a) {
  prof_mark(ctx->prof, ctx->stream, KC_GATE_BWD, true);
  gate_form<T>(a.heads, [&](auto nj, auto lanes) {
    constexpr int NJ = decltype(nj)::value, LPR = decltype(lanes)::value;
    const long long n = (a.rows * LPR + 255) / 256;
    k_gate_bwd<T, NJ, LPR><<<(unsigned)(n < 4096 ? n : 4096), 256, 0, ctx->stream>>>(a);
  });
  prof_mark(ctx->prof, ctx->stream, KC_GATE_BWD, false);
  return launched(ctx, "gate reverse launch");
}

painn_status gate_check(painn_ctx* ctx, const painn_gate_args& a) {
  if (a.precision == PAINN_FP64) return fail(ctx, PAINN_E_UNSUPPORTED, "the gate runs in FP32 and BF16");
  if (a.precision != PAINN_FP32 && a.precision != PAINN_BF16) return fail(ctx, PAINN_E_ARG, "unknown precision");
  if (a.heads < 1 || a.k < 1 || a.k > a.heads) return fail(ctx, PAINN_E_ARG, "k must be within 1 and the heads");
  if (a.rows < 0) return fail(ctx, PAINN_E_ARG, "rows must not be negative");
  if (a.normalize != 0 && a.normalize != 1) return fail(ctx, PAINN_E_ARG, "normalize is 0 or 1");
  if (a.heads > HEADS) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 1024 heads");
  if (a.rows > 0x7fffffffLL / a.k) return fail(ctx, PAINN_E_UNSUPPORTED, "2^31 or more choices");
  if (a.rows > 0 && a.ldx < a.heads) return fail(ctx, PAINN_E_ARG, "the row stride is below the heads");
  return PAINN_OK;
}

GateArgs args_of(const painn_gate_args& a) {
  GateArgs g{};
  g.rows = a.rows; g.heads = a.heads; g.k = a.k; g.normalize = a.normalize; g.x = a.logits; g.ldx = a.ldx;
  return g;
}

}  // namespace

extern "C" {

int64_t painn_gate_workspace(painn_precision precision, int64_t rows, int32_t heads, int32_t k) {
  if (rows < 0 || heads < 1 || heads > HEADS || rows > 0x7fffffffLL) return 0;
  int blocks, threads;
  gate_grid(precision == PAINN_BF16, rows, heads, k, blocks, threads);
  return (int64_t)gate_bytes(blocks, heads);
}

painn_status painn_gate(painn_ctx* ctx, const painn_gate_args* args) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!args) return fail(ctx, PAINN_E_ARG, "null arguments");
  const painn_gate_args& a = *args;
  const painn_status st = gate_check(ctx, a);
  if (st != PAINN_OK) return st;
  if (!a.counts || !a.share || !a.loss || (a.rows > 0 && (!a.logits || !a.weights || !a.indices)))
    return fail(ctx, PAINN_E_ARG, "null array");
  GateArgs g = args_of(a);
  g.weights = a.weights; g.indices = a.indices; g.counts = a.counts; g.share = a.share; g.loss = a.loss;
  int blocks, threads;
  gate_grid(a.precision == PAINN_BF16, a.rows, a.heads, a.k, blocks, threads);
  const size_t need = gate_bytes(blocks, a.heads);
  if (a.workspace_bytes < (int64_t)need || (need && !a.workspace))
    return fail(ctx, PAINN_E_ARG, "the workspace is too small: " + std::to_string(need) + " bytes");
  g.part_p = (float*)a.workspace;
  g.part_c = (int*)((char*)a.workspace + align256((size_t)blocks * a.heads * 4));
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  return a.precision == PAINN_FP32 ? run_gate<float>(ctx, g, blocks, threads) : run_gate<b16>(ctx, g, blocks, threads);
}

painn_status painn_gate_backward(painn_ctx* ctx, const painn_gate_args* args, const float* dweights, double balance,
                                 void* dlogits, int64_t ldd) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!args) return fail(ctx, PAINN_E_ARG, "null arguments");
  const painn_gate_args& a = *args;
  const painn_status st = gate_check(ctx, a);
  if (st != PAINN_OK) return st;
  if (!(balance >= -3.4e38 && balance <= 3.4e38)) return fail(ctx, PAINN_E_ARG, "balance must be finite in FP32");
  if (a.rows == 0) return PAINN_OK;
  if (!a.logits || !a.counts || !dlogits || (dweights && !a.indices)) return fail(ctx, PAINN_E_ARG, "null array");
  if (ldd < a.heads) return fail(ctx, PAINN_E_ARG, "the row stride is below the heads");
  if (misplaced(dlogits, ldd, a.logits, a.ldx, a.rows))
    return fail(ctx, PAINN_E_ARG, "dlogits in place of the logits has another row stride");
  GateArgs g = args_of(a);
  g.dw = dweights; g.chosen = a.indices; g.n = a.counts; g.balance = balance; g.dx = dlogits; g.lddx = ldd;
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  return a.precision == PAINN_FP32 ? run_gate_bwd<float>(ctx, g) : run_gate_bwd<b16>(ctx, g);
}

}  // extern "C"

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

#include "raw.h"

namespace {

using namespace ops;

constexpr int KREG = 8;             // heads chosen one after the other
constexpr int HEADS = 1024;         // heads at most
constexpr int GATE_BWD = 2048;      // blocks of the reverse pass at most: 8 per CU
constexpr int GATE_GRID = 512;      // blocks of the forward, whose sums are folded

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
// BF16's last 16 bits are 0, which leaves room for the head: 0xffff - head, so
// that the lowest of equals has the largest key.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t o, bool bf16) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : bf16 ? ~o & 0xffff0000u : ~o);
}
// x of a lane that has another part of the row's reduction: within 16 lanes the
// exchange is part of the instruction that uses it.
template <int O>
__device__ __forceinline__ int lane_of(int x) {
  if constexpr (O == 1) return __builtin_amdgcn_update_dpp(x, x, 0xb1, 0xf, 0xf, false);        // quad_perm 1, 0, 3, 2
  else if constexpr (O == 2) return __builtin_amdgcn_update_dpp(x, x, 0x4e, 0xf, 0xf, false);   // quad_perm 2, 3, 0, 1
  else if constexpr (O == 4) return __builtin_amdgcn_update_dpp(x, x, 0x141, 0xf, 0xf, false);  // 8 lanes mirrored
  else if constexpr (O == 8) return __builtin_amdgcn_update_dpp(x, x, 0x140, 0xf, 0xf, false);  // 16 lanes mirrored
  else if constexpr (O == 16) return __builtin_amdgcn_ds_swizzle(x, 0x401f);                    // xor 16
  else return __shfl_xor(x, 32);
}
// The reduction of x over the row's LPR lanes, in all of them.
template <int LPR, int O = 1, class F>
__device__ __forceinline__ int lanes(int x, F&& f) {
  if constexpr (O < LPR) return lanes<LPR, 2 * O>(f(x, lane_of<O>(x)), f);
  else return x;
}
template <int LPR>
__device__ __forceinline__ float lanes_sum(float x) {
  return __int_as_float(lanes<LPR>(__float_as_int(x), [](int p, int q) {
    return __float_as_int(__int_as_float(p) + __int_as_float(q));
  }));
}
template <int LPR>
__device__ __forceinline__ int lanes_add(int x) {
  return lanes<LPR>(x, [](int p, int q) { return p + q; });
}
template <int LPR>
__device__ __forceinline__ float lanes_max(float x) {
  return __int_as_float(lanes<LPR>(__float_as_int(x), [](int p, int q) {
    return __float_as_int(fmaxf(__int_as_float(p), __int_as_float(q)));
  }));
}
template <int LPR>
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  return (uint32_t)lanes<LPR>((int)x, [](int p, int q) { return (uint32_t)p > (uint32_t)q ? p : q; });
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
  Raw<T, V> raw[NJ];
  // (the values stay on their way until softmax)
  __device__ __forceinline__ void load(const void* p, long long ld, long long row, bool live, int heads, int lane) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + lane) * V;
      raw[j] = zero_raw<T, V>();
      if (live && c < heads) raw[j] = load_raw<T, V, false>((const T*)p + row * ld + c, heads - c);
    }
  }
  __device__ __forceinline__ void softmax(bool live, int heads, int lane) {
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      unpack<T, V>(raw[j], x + j * V);
#pragma unroll
      for (int i = 0; i < V; ++i) x[j * V + i] = live && head(lane, j * V + i) < heads ? x[j * V + i] : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) most = fmaxf(most, x[i]);
    most = lanes_max<LPR>(most);
    top = most > -INFINITY ? most : 0.f;
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      e[i] = exp_of(x[i] - top);
      s += e[i];
    }
    s = lanes_sum<LPR>(s);
    some = !(s == 0.f);             // (1 at least, or NaN)
    inv = some ? 1.f / s : 0.f;
  }
};

// Counts, share and loss from a head's totals: thread t has heads t, t + n, ...
// whose counts and sums of p are c[head], p[head].  red: [16] doubles, n_red [16].
template <class P>
__device__ __forceinline__ void finish(const GateArgs& a, const int* c, const P* p, int routed, double* red, int* n_red) {
  double mine = 0.0;
  int chosen = 0;
  for (int h = threadIdx.x; h < a.heads; h += blockDim.x) {
    const double share = routed ? (double)p[h] / routed : 0.0;
    a.counts[h] = c[h];
    a.share[h] = (float)share;
    mine += share * c[h];
    chosen += c[h];
  }
  // (up to 64 heads: the first wave has them all)
#pragma unroll
  for (int o = 32; o; o >>= 1) {
    mine += __shfl_xor(mine, o);
    chosen += __shfl_xor(chosen, o);
  }
  if (a.heads > 64) {
    if ((threadIdx.x & 63) == 0) {
      red[threadIdx.x >> 6] = mine;
      n_red[threadIdx.x >> 6] = chosen;
    }
    __syncthreads();
    mine = 0.0;
    chosen = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
      mine += red[w];
      chosen += n_red[w];
    }
  }
  if (threadIdx.x == 0) {
    a.counts[a.heads] = routed;
    a.loss[0] = chosen ? (float)(mine * a.heads / chosen) : 0.f;
  }
}

// The blocks' partial rows added, in parts of the blocks side by side and those
// in their order; then as above.
__global__ void __launch_bounds__(1024) k_gate_fold(GateArgs a, int blocks, int width_bits) {
  __shared__ double sum[HEADS + 1024], red[16];
  __shared__ int cnt[HEADS + 1024], n_red[16];
  const int t = threadIdx.x, width = 1 << width_bits, l = t & (width - 1), q = t >> width_bits, slices = 1024 >> width_bits;
  // heads 0 .. heads - 1, then the rows that have a head
  for (int h0 = 0; h0 <= a.heads; h0 += width) {
    const int h = h0 + l;
    double p = 0.0;
    int c = 0;
    if (h <= a.heads) {
#pragma unroll 8
      for (int b = q; b < blocks; b += slices) {
        if (h < a.heads) p += (double)a.part_p[(size_t)b * a.heads + h];
        c += a.part_c[(size_t)b * (a.heads + 1) + h];
      }
    }
    for (int o = width; o < 64; o <<= 1) {
      p += __shfl_xor(p, o);
      c += __shfl_xor(c, o);
    }
    // (a wave's part, or several waves side by side where a part is wider)
    const int parts = width < 64 ? 16 : slices, part = width < 64 ? t >> 6 : q;
    __syncthreads();
    if (width >= 64 || (t & 63) < width) {
      sum[HEADS + part * width + l] = p;
      cnt[HEADS + part * width + l] = c;
    }
    __syncthreads();
    if (t < width && h <= a.heads) {
      p = 0.0;
      c = 0;
      for (int k = 0; k < parts; ++k) {
        p += sum[HEADS + k * width + l];
        c += cnt[HEADS + k * width + l];
      }
      if (h < HEADS) sum[h] = p;
      if (h == a.heads) n_red[0] = c;
      else cnt[h] = c;
    }
  }
  __syncthreads();
  const int routed = n_red[0];
  __syncthreads();
  finish(a, cnt, sum, routed, red, n_red);
}

// MANY: more than KREG heads of a row.
template <class T, int NJ, int LPR, bool MANY>
__global__ void __launch_bounds__(1024) k_gate(GateArgs a) {
  typedef Row<T, NJ, LPR> R;
  constexpr int N = R::N, ACROSS = LPR * N;
  // counts [heads + 1]; then the waves' sums of p, or the rows' keys
  extern __shared__ int lds[];
  __shared__ double red[16];
  __shared__ int n_red[16];
  int* cnt = lds;
  const int rpb = blockDim.x / LPR, lane = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  uint32_t* keys = (uint32_t*)(lds + a.heads + 1) + sub * ACROSS;
  for (int h = threadIdx.x; h <= a.heads; h += blockDim.x) cnt[h] = 0;
  float sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i] = 0.f;
  __syncthreads();
  int routed = 0;
  const long long step = (long long)gridDim.x * rpb;
  R next;
  next.load(a.x, a.ldx, (long long)blockIdx.x * rpb + sub, (long long)blockIdx.x * rpb + sub < a.rows, a.heads, lane);
  for (long long r0 = (long long)blockIdx.x * rpb; r0 < a.rows; r0 += step) {
    const long long row = r0 + sub;
    const bool live = row < a.rows;
    R r = next;
    next.load(a.x, a.ldx, row + step, row + step < a.rows, a.heads, lane);
    r.softmax(live, a.heads, lane);
    float* w = a.weights + row * a.k;
    int* id = a.indices + row * a.k;
    if (r.some) {
      routed += lane == 0;
#pragma unroll
      for (int i = 0; i < N; ++i) sum[i] += r.e[i] * r.inv;
    }
    if constexpr (!MANY) {
      constexpr bool B16 = sizeof(T) == 2;
      uint32_t key[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int h = R::head(lane, i);
        key[i] = h >= a.heads ? 0u : B16 ? (ordered(r.x[i]) & 0xffff0000u) | (0xffffu - (uint32_t)h) : ordered(r.x[i]);
      }
      float ws[KREG];
      int is[KREG];
      float total = 0.f;
#pragma unroll
      for (int s = 0; s < KREG; ++s) {
        ws[s] = 0.f;
        is[s] = -1;
        if (s < a.k) {
          uint32_t best = key[0];
#pragma unroll
          for (int i = 1; i < N; ++i) best = key[i] > best ? key[i] : best;
          best = lanes_max<LPR>(best);
          int h;
          if constexpr (B16) {
            h = (int)(0xffffu - (best & 0xffffu));
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = key[i] == best ? 0u : key[i];
            best &= 0xffff0000u;
          } else {
            // the lowest head of this key
            uint32_t least = 0;
#pragma unroll
            for (int i = N - 1; i >= 0; --i) least = key[i] == best ? 0xffffu - (uint32_t)R::head(lane, i) : least;
            h = (int)(0xffffu - lanes_max<LPR>(least));
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = R::head(lane, i) == h ? 0u : key[i];
          }
          const float x = value_of(best, B16);
          if (!(x == -INFINITY)) {
            is[s] = h;
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
      places = lanes_add<LPR>(places);
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
    for (int h = threadIdx.x; h < a.heads; h += blockDim.x) {
      float s = 0.f;
      for (int k = 0; k < (int)blockDim.x / 64; ++k) s += waves[k * a.heads + h];
      waves[h] = s;
    }
    finish(a, cnt, waves, cnt[a.heads], red, n_red);      // (a thread's heads are those that it added)
    return;
  }
  for (int h = threadIdx.x; h < a.heads; h += blockDim.x) {
    float s = 0.f;
    for (int k = 0; k < (int)blockDim.x / 64; ++k) s += waves[k * a.heads + h];
    a.part_p[(size_t)blockIdx.x * a.heads + h] = s;
  }
  for (int h = threadIdx.x; h <= a.heads; h += blockDim.x) a.part_c[(size_t)blockIdx.x * (a.heads + 1) + h] = cnt[h];
}

// Up to KREG values of a row's n choices, four or two at a time where they
// come so.
template <class S>
__device__ __forceinline__ void load_choices(const S* p, int n, S* x, S none) {
  typedef S four __attribute__((ext_vector_type(4), aligned(4)));
  typedef S two __attribute__((ext_vector_type(2), aligned(4)));
#pragma unroll
  for (int s = 0; s < KREG; s += 4) {
    if (n - s >= 4) {
      const four v = *(const four*)(p + s);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[s + i] = v[i];
    } else {
      x[s] = x[s + 1] = x[s + 2] = x[s + 3] = none;
      if (n - s >= 2) {
        const two v = *(const two*)(p + s);
        x[s] = v[0];
        x[s + 1] = v[1];
        if (n - s == 3) x[s + 2] = p[s + 2];
      } else if (n - s == 1) {
        x[s] = p[s];
      }
    }
  }
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
  const long long step = (long long)gridDim.x * rpb;
  long long row = (long long)blockIdx.x * rpb + sub;
  R next;
  int ni[KREG];
  float nd[KREG];
  const auto ahead = [&](long long at) {
    next.load(a.x, a.ldx, at, at < a.rows, a.heads, lane);
    const int n = a.dw && at < a.rows ? a.k : 0;
    load_choices(a.chosen + at * a.k, n, ni, -1);
    load_choices(a.dw + at * a.k, n, nd, 0.f);
  };
  ahead(row);
  float f[N];
  int all = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int h = R::head(lane, i), c = h < a.heads ? a.n[h] : 0;
    f[i] = (float)c;
    all += c;
  }
  all = lanes_add<LPR>(all);
  const int routed = a.n[a.heads];
  const float scale = all > 0 && routed > 0 ? (float)(a.balance * a.heads / ((double)routed * all)) : 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) f[i] *= scale;
  for (long long r0 = (long long)blockIdx.x * rpb; r0 < a.rows; r0 += step, row += step) {
    const bool live = row < a.rows;
    R r = next;
    int is[KREG];
    float ds[KREG];
#pragma unroll
    for (int s = 0; s < KREG; ++s) {
      is[s] = ni[s];
      ds[s] = nd[s];
    }
    ahead(row + step);
    float d[N];
    uint32_t mark = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) d[i] = 0.f;
    for (int s0 = 0; s0 < a.k; s0 += KREG) {
      if (s0 > 0) {
        const int n = a.dw && live ? a.k - s0 : 0;
        load_choices(a.chosen + row * a.k + s0, n, is, -1);
        load_choices(a.dw + row * a.k + s0, n, ds, 0.f);
      }
#pragma unroll
      for (int s = 0; s < KREG; ++s) {
        if (s0 + s >= a.k) break;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (is[s] == R::head(lane, i)) {
            d[i] += ds[s];
            mark |= 1u << i;
          }
      }
    }
    r.softmax(live, a.heads, lane);
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
  // (65,502 x 16 BF16: half the partial rows of blocks of 256, whose fold took 8.0 us for 5.5)
  if (rows * lpr <= 512LL * GATE_GRID) threads = many ? 256 : 512;
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
  if (blocks > 1) {
    int bits = 0;                   // heads side by side, and the rows' count
    while (bits < 10 && 1 << bits < a.heads + 1) ++bits;
    k_gate_fold<<<1, 1024, 0, ctx->stream>>>(a, blocks, bits);
  }
  prof_mark(ctx->prof, ctx->stream, KC_GATE, false);
  return launched(ctx, "gate launch");
}

template <class T>
painn_status run_gate_bwd(painn_ctx* ctx, const GateArgs& a) {
  prof_mark(ctx->prof, ctx->stream, KC_GATE_BWD, true);
  gate_form<T>(a.heads, [&](auto nj, auto lanes) {
    constexpr int NJ = decltype(nj)::value, LPR = decltype(lanes)::value;
    const long long n = (a.rows * LPR + 255) / 256;
    k_gate_bwd<T, NJ, LPR><<<(unsigned)(n < GATE_BWD ? n : GATE_BWD), 256, 0, ctx->stream>>>(a);
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

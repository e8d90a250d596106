// The reverse pass of group norm (groupnorm.hip has the forward and the split of
// the work that both share).
#include "fold.h"
#include "groupnorm.h"

namespace {

// ---- reverse pass -----------------------------------------------------------------
// With xh = (x - mean) rstd, dz = dy act'(xh gamma + beta) and a = dz gamma:
//   dx = rstd (a - mean(a) - xh mean(a xh)),  dgamma = sum dz xh,  dbeta = sum dz,
// the means over the set.
__device__ __forceinline__ void stats_of(const GnArgs& a, int sample, int group, float& mu, float& rs) {
  mu = a.mu[sample * a.mu_s + group * a.mu_g];
  rs = a.rs[sample * a.rs_s + group * a.rs_g];
}
template <class T, int V, bool FULL, int ACT>
struct Grads {
  float xh[V], dz[V];
  __device__ __forceinline__ Grads() {}
  __device__ __forceinline__ Grads(const GnArgs& a, const Place<V>& p, const Raw<T, V>& x, const Raw<T, V>& dy, float mu,
                                   float rs, const float* g, const float* b) {
    float z[V];
    unpack<T, V>(x, xh);
    unpack<T, V>(dy, dz);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // (0 past the group, as dy is: (0 - mu) rs may be an infinity)
      xh[i] = FULL || i < p.left ? (xh[i] - mu) * rs : 0.f;
      z[i] = xh[i] * g[i] + b[i];
    }
    times_slope<ACT, V>(dz, z, a.act == PAINN_ACT_RELU);
  }
};
// A thread's sums for dgamma and dbeta, and a block's: FP64 where the results are
// FP32 (120,000 x 192, 5 samples, SiLU: off by 8e-8 in 2-norm and 114 us, with FP32
// sums 1.9e-7 and 116), FP32 ahead of BF16 results, which round to 2^-8 of
// themselves.  A block's sum is rounded to FP32 once, the blocks' are added in
// the same type.
template <class T>
struct ColumnSum {
  typedef typename std::conditional<sizeof(T) == 4, double, float>::type type;
};
// (a set's sums: FP32 over a vector, FP64 beyond)
template <class T, int V, bool FULL, int ACT>
__device__ __forceinline__ void add_grads(const Grads<T, V, FULL, ACT>& d, const float* g, double* s,
                                          typename ColumnSum<T>::type* dg, typename ColumnSum<T>::type* db) {
  typedef typename ColumnSum<T>::type S;
  float u[V], w[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    dg[i] += (S)d.dz[i] * (S)d.xh[i];
    db[i] += d.dz[i];
    u[i] = d.dz[i] * g[i];
    w[i] = u[i] * d.xh[i];
  }
  s[0] += (double)tree<V>(u);
  s[1] += (double)tree<V>(w);
}
template <class T, int V, bool FULL, int ACT>
__device__ __forceinline__ void put_dx(const Rows<T, V, FULL>& o, int i, const Grads<T, V, FULL, ACT>& d, const float* g, float rs,
                                       float m1, float m2) {
  float v[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    // (a rounded as in the sums, so that nothing is left of a set of one value)
#pragma clang fp contract(off)
    const float up = d.dz[e] * g[e];
    v[e] = rs * __builtin_fmaf(-d.xh[e], m2, up - m1);
  }
  o.put(i, v);
}

template <class T, int V, bool FULL, int ACT, int TB, bool REST>
__device__ __forceinline__ void team_backward(const GnArgs& a, const Place<V>& p, int team, int s, const Span& q,
                                              const float* g, const float* b, typename ColumnSum<T>::type* dg,
                                              typename ColumnSum<T>::type* db, double* lds) {
  constexpr int NR = steps_held_bwd(TB), U = 2;
  typedef Grads<T, V, FULL, ACT> G;
  const Rows<T, V, FULL> x(a.x, a.ldx, p, q.a, q.b - q.a), y(a.dy, a.lddy, p, q.a, q.b - q.a);
  Raw<T, V> xs[NR], ys[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    xs[i] = x.get(i);
    ys[i] = y.get(i);
  }
  float mu = 0.f, rs = 0.f;
  if (x.n > 0 && (FULL || p.left > 0)) stats_of(a, s, p.group, mu, rs);
  double sum[2] = {0.0, 0.0};
  float dz[NR][V];                      // (kept for dx: 65,502 x 256 BF16 56 us, formed again 64)
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    if (x.has(i)) {
      const G d(a, p, xs[i], ys[i], mu, rs, g, b);
      add_grads<T, V, FULL, ACT>(d, g, sum, dg, db);
#pragma unroll
      for (int e = 0; e < V; ++e) dz[i][e] = d.dz[e];
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) dz[i][e] = 0.f;
    }
  }
  for (int i0 = NR; REST && x.has(i0); i0 += U) {
    Raw<T, V> u[U], w[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      u[i] = x.get(i0 + i);
      w[i] = y.get(i0 + i);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (x.has(i0 + i)) add_grads<T, V, FULL, ACT>(G(a, p, u[i], w[i], mu, rs, g, b), g, sum, dg, db);
  }
  if (!a.out) return;
  team_sum<TB, 2>(a, sum, team, lds);
  const double inv = x.n > 0 ? 1.0 / ((double)x.n * a.cg) : 0.0;
  const float m1 = (float)(sum[0] * inv), m2 = (float)(sum[1] * inv);
  const Rows<T, V, FULL> o(a.out, a.ldo, p, q.a, q.b - q.a);
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (x.has(i)) {
      G d;
      unpack<T, V>(xs[i], d.xh);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        d.xh[e] = (d.xh[e] - mu) * rs;
        d.dz[e] = dz[i][e];
      }
      put_dx<T, V, FULL, ACT>(o, i, d, g, rs, m1, m2);
    }
  for (int i0 = NR; REST && x.has(i0); i0 += U) {
    Raw<T, V> u[U], w[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      u[i] = x.get(i0 + i);
      w[i] = y.get(i0 + i);
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (x.has(i0 + i)) put_dx<T, V, FULL, ACT>(o, i0 + i, G(a, p, u[i], w[i], mu, rs, g, b), g, rs, m1, m2);
  }
}

// Blocks as the forward's.
template <class T, int V, bool FULL, int ACT, int TB>
__global__ void __launch_bounds__(TB) k_group_norm_bwd(GnArgs a) {
  __shared__ double lds[2 * TB];
  typedef typename ColumnSum<T>::type S;
  extern __shared__ double column_sums[];
  S* acc = (S*)column_sums;             // [2][lanes of a row * V]
  const int slab = blockIdx.x, blk = blockIdx.y, lpr = a.lpg * a.gb;
  const bool tiles = blk >= a.l_blocks + a.f_blocks;
  const int team = tiles || blk < a.l_blocks ? TB : a.team, team_bits = 31 - __builtin_clz(team), teams = TB >> team_bits,
            mine = threadIdx.x >> team_bits;
  const Place<V> p(a, slab, (int)threadIdx.x & (team - 1), team);
  float g[V], b[V];
  S dg[V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) {
    g[i] = b[i] = 0.f;
    dg[i] = db[i] = 0;
  }
  load_n<V>((const T*)a.gamma + p.col, p.left, g);
  load_n<V>((const T*)a.beta + p.col, p.left, b);
  if (tiles) {
    const int t = blk - a.l_blocks - a.f_blocks;
    long_samples(a, t, [&](int slot, int sample, const Span&, long long lo, long long hi) {
      typedef Grads<T, V, FULL, ACT> G;
      float mu = 0.f, rs = 0.f;
      if (FULL || p.left > 0) stats_of(a, sample, p.group, mu, rs);
      double s[2] = {0.0, 0.0};
      const Rows<T, V, FULL> x(a.x, a.ldx, p, lo, hi - lo), y(a.dy, a.lddy, p, lo, hi - lo);
      for (int i0 = 0; x.has(i0); i0 += 8) {
        Raw<T, V> u[8], w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] = x.get(i0 + i);
          w[i] = y.get(i0 + i);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (x.has(i0 + i)) add_grads<T, V, FULL, ACT>(G(a, p, u[i], w[i], mu, rs, g, b), g, s, dg, db);
      }
      team_sum<TB, 2>(a, s, TB, lds);
      if (p.row == 0 && p.left == a.cg) a.seg[((size_t)t * 2 + slot) * a.groups + p.group] = make_double2(s[0], s[1]);
    });
  } else {
    const long long held = TB > 64 ? -1 : (long long)(a.team >> a.lpr_bits) * steps_held_bwd(64);
    if (blk < a.l_blocks || TB > 64) {
      longer_samples(a, blk, TB > 64 ? a.f_blocks : a.l_blocks, held + 1, [&](int s, const Span& q) {
        team_backward<T, V, FULL, ACT, TB, true>(a, p, TB, s, q, g, b, dg, db, lds);
      });
    } else if constexpr (TB == 64) {
      // (a sample's rows are looked up while the one before it is worked on)
      const long long step = (long long)a.f_blocks * teams;
      Span next{0, 0};
      long long s0 = (long long)(blk - a.l_blocks) * teams;
      if (s0 + mine < a.samples) next = span(a, (int)(s0 + mine));
      for (; s0 < a.samples; s0 += step) {
        const int s = s0 + mine < a.samples ? (int)(s0 + mine) : 0;
        Span q = next;
        next = Span{0, 0};
        if (s0 + step + mine < a.samples) next = span(a, (int)(s0 + step + mine));
        if (q.b - q.a > held) q.b = q.a;
        if (team < 64 || q.b > q.a) team_backward<T, V, FULL, ACT, 64, false>(a, p, team, s, q, g, b, dg, db, lds);
      }
    }
  }
  if (!a.part) return;
  // the block's column sums: a wave's rows, then wave after wave
  for (int o = lpr; o < 64; o <<= 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[i] = lane_add(dg[i], o);
      db[i] = lane_add(db[i], o);
    }
  }
  const int width = lpr * V, at = (threadIdx.x & (lpr - 1)) * V, per = lpr > 64 ? lpr / 64 : 1;
  for (int w = 0; w < TB / 64; w += per) {
    __syncthreads();
    const int wave = threadIdx.x >> 6;
    if (wave >= w && wave < w + per && (lpr > 64 || (int)(threadIdx.x & 63) < lpr)) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        acc[at + i] = w ? acc[at + i] + dg[i] : dg[i];
        acc[width + at + i] = w ? acc[width + at + i] + db[i] : db[i];
      }
    }
  }
  __syncthreads();
  float* out = a.part + (size_t)blk * 2 * a.cols;
  const int c0 = slab * a.gb * a.cg, many = (a.groups - slab * a.gb < a.gb ? a.groups - slab * a.gb : a.gb) * a.cg;
  for (int c = threadIdx.x; c < many; c += TB) {
    const int q = c / a.cg, k = q * a.lpg * V + c - q * a.cg;
    out[c0 + c] = (float)acc[k];
    out[a.cols + c0 + c] = (float)acc[width + k];
  }
}

// dx of long samples, tile by tile.
template <class T, int V, bool FULL, int ACT, int TB>
__global__ void __launch_bounds__(TB) k_group_norm_bwd_tiles(GnArgs a) {
  __shared__ double lds[2 * TB];
  typedef Grads<T, V, FULL, ACT> G;
  const int slab = blockIdx.x, t = (int)(gridDim.y - 1 - blockIdx.y);   // (the rows read last are in the caches)
  const Place<V> p(a, slab, threadIdx.x, TB);
  long_samples(a, t, [&](int, int sample, const Span& q, long long lo, long long hi) {
    double s[2];
    tiles_sum(a, q, p.group, p.row * a.lpg + (threadIdx.x & (a.lpg - 1)), p.rows * a.lpg, s);
    team_sum<TB, 2>(a, s, TB, lds);
    if (!FULL && p.left <= 0) return;
    const double inv = 1.0 / ((double)(q.b - q.a) * a.cg);
    const float m1 = (float)(s[0] * inv), m2 = (float)(s[1] * inv);
    float mu, rs;
    stats_of(a, sample, p.group, mu, rs);
    float g[V], b[V];
    load_n<V>((const T*)a.gamma + p.col, p.left, g);
    load_n<V>((const T*)a.beta + p.col, p.left, b);
    const Rows<T, V, FULL> x(a.x, a.ldx, p, lo, hi - lo), y(a.dy, a.lddy, p, lo, hi - lo), o(a.out, a.ldo, p, lo, hi - lo);
    for (int i0 = 0; x.has(i0); i0 += 4) {
      Raw<T, V> u[4], w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        u[i] = x.get(i0 + i);
        w[i] = y.get(i0 + i);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x.has(i0 + i)) put_dx<T, V, FULL, ACT>(o, i0 + i, G(a, p, u[i], w[i], mu, rs, g, b), g, rs, m1, m2);
    }
  });
}

template <class T>
painn_status run_bwd(painn_ctx* ctx, const Plan& p, const GnArgs& a, void* dgamma, void* dbeta) {
  const dim3 grid(p.slabs, p.l_blocks + p.f_blocks + p.tiles), tiles(p.slabs, p.tiles);
  const size_t lds = a.part ? (size_t)2 * p.lpg * p.gb * p.v * sizeof(typename ColumnSum<T>::type) : 0;
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM_BWD, true);
  if (a.rows > 0 && a.samples > 0) {
    with_form<T>(p, a.act, [&](auto v, auto full, auto act) {
      constexpr int V = decltype(v)::value;
      constexpr bool FULL = decltype(full)::value;
      constexpr int ACT = decltype(act)::value;
      if (p.tb == 64) k_group_norm_bwd<T, V, FULL, ACT, 64><<<grid, 64, lds, ctx->stream>>>(a);
      else if (p.tb == 256) k_group_norm_bwd<T, V, FULL, ACT, 256><<<grid, 256, lds, ctx->stream>>>(a);
      else k_group_norm_bwd<T, V, FULL, ACT, 512><<<grid, 512, lds, ctx->stream>>>(a);
      if (p.tiles && a.out && p.lpg <= 256) k_group_norm_bwd_tiles<T, V, FULL, ACT, 256><<<tiles, 256, 0, ctx->stream>>>(a);
      else if (p.tiles && a.out) k_group_norm_bwd_tiles<T, V, FULL, ACT, 512><<<tiles, 512, 0, ctx->stream>>>(a);
    });
  }
  if (dgamma) {
    const int n = a.rows > 0 && a.samples > 0 ? p.l_blocks + p.f_blocks + p.tiles : 0;
    fold_columns<T, typename ColumnSum<T>::type>(ctx->stream, n, a.cols, a.part, (T*)dgamma, (T*)dbeta);
  }
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM_BWD, false);
  return launched(ctx, "group norm reverse launch");
}

}  // namespace

extern "C" {

painn_status painn_group_norm_backward(painn_ctx* ctx, const painn_group_norm_args* args, const void* dy, int64_t lddy,
                                       void* dx, int64_t lddx, void* dgamma, void* dbeta) {
  return painn_group_norm_backward_strided(ctx, args, nullptr, dy, lddy, dx, lddx, dgamma, dbeta);
}

painn_status painn_group_norm_backward_strided(painn_ctx* ctx, const painn_group_norm_args* args, const int64_t* strides,
                                               const void* dy, int64_t lddy, void* dx, int64_t lddx, void* dgamma,
                                               void* dbeta) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!args) return fail(ctx, PAINN_E_ARG, "null arguments");
  const painn_group_norm_args& a = *args;
  painn_status st = shape_check(ctx, a.precision, a.rows, a.cols, a.groups, a.n_samples, a.offsets, a.sample_rows, a.max_rows,
                                a.activation, a.reserved);
  if (st != PAINN_OK) return st;
  if (!dgamma != !dbeta) return fail(ctx, PAINN_E_ARG, "dgamma and dbeta are formed together");
  for (int k = 0; strides && k < 4; ++k)
    if (strides[k] < 0) return fail(ctx, PAINN_E_ARG, "a stride of mean or rstd is negative");
  const bool some = a.rows > 0 && a.n_samples > 0;
  if (some) {
    if (!dy || !a.x || !a.gamma || !a.beta || !a.mean || !a.rstd) return fail(ctx, PAINN_E_ARG, "null array");
    if (lddy < a.cols || a.ldx < a.cols || (dx && lddx < a.cols))
      return fail(ctx, PAINN_E_ARG, "a row stride is below cols");
    if (misplaced(dx, lddx, dy, lddy, a.rows)) return fail(ctx, PAINN_E_ARG, "dx in place of dy has another row stride");
  }
  if (!dgamma && (!dx || !some)) return PAINN_OK;
  const Plan p = plan_of(a.precision == PAINN_BF16, a.rows, a.cols, a.groups, a.n_samples, a.offsets != nullptr,
                         a.sample_rows, a.max_rows, true);
  if ((long long)p.slabs * (p.l_blocks + p.f_blocks + p.tiles) > LAUNCH_THREADS / 1024)
    return fail(ctx, PAINN_E_UNSUPPORTED, "more blocks than a launch holds");
  const size_t need = some ? p.seg_bytes + (dgamma ? p.part_bytes : 0) : 0;
  if (a.workspace_bytes < (int64_t)need || (need && !a.workspace))
    return fail(ctx, PAINN_E_ARG, "the workspace is too small: " + std::to_string(need) + " bytes");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  GnArgs g{};
  fill(g, p, a, a.workspace);
  g.dy = dy; g.lddy = lddy; g.out = dx; g.ldo = lddx; g.mu = a.mean; g.rs = a.rstd;
  g.mu_s = strides ? strides[0] : a.groups; g.mu_g = strides ? strides[1] : 1;
  g.rs_s = strides ? strides[2] : a.groups; g.rs_g = strides ? strides[3] : 1;
  if (!dgamma) g.part = nullptr;
  return a.precision == PAINN_FP32 ? run_bwd<float>(ctx, p, g, dgamma, dbeta) : run_bwd<b16>(ctx, p, g, dgamma, dbeta);
}

}  // extern "C"

// Group norm with an activation, channels last, over the rows of ragged samples,
// and its reverse pass (FP32, BF16).
//
// A set is a sample's rows times a group's columns.  Its statistics are sums
// about a value near its mean (FP32, or FP64 where that loses digits), so that a
// mean far from 0 costs none; the reverse pass takes the sums of a and a xh.  Bound by
// memory: x (and dy) should be read once.  A team of threads therefore holds a
// sample's rows of one slab (whole groups, 128 bytes or more of a row, so that
// no line is read by two teams) in registers between its sums and its result;
// rows past those are read again.  How many threads a team has goes by the
// samples' usual length, from a few lanes to a block of 512.
//
// Samples longer than `limit` would leave the chip to a few teams.  They are
// cut into tiles of R <= limit rows: the tiles' sums are formed by further
// blocks of the first launch in FP64, and a second launch adds a sample's tiles, in
// their order, and writes its result.  A tile meets at most two such samples,
// the ones that hold its first and its last row, which gives every (tile,
// sample) its place without a list.
#include "groupnorm.h"

namespace {

// ---- forward --------------------------------------------------------------------
// FP64 sums of x - pivot and its square.
template <class T, int V, bool FULL, int U>
__device__ __forceinline__ void add_rows(const Rows<T, V, FULL>& x, float pivot, double* s) {
  for (int i0 = 0; x.has(i0); i0 += U) {
    Raw<T, V> v[U];
#pragma unroll
    for (int i = 0; i < U; ++i) v[i] = x.get(i0 + i);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float u[V];
      unpack<T, V>(v[i], u);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const double d = x.has(i0 + i) && (FULL || e < x.left) ? (double)u[e] - (double)pivot : 0.0;
        s[0] += d;
        s[1] = __builtin_fma(d, d, s[1]);
      }
    }
  }
}
// The pivot of FP64 sums: the group's first value in a row, so that equal values
// leave no squares (0 where it is not finite).
template <class T, int V>
__device__ __forceinline__ float first_value(const GnArgs& a, const Place<V>& p, long long row) {
  float k = 0.f;
  if (p.left > 0) load_n<1>((const T*)a.x + row * a.ldx + (long long)p.group * a.cg, 1, &k);
  return fabsf(k) < INFINITY ? k : 0.f;
}

// 1 / sqrt(variance + eps); what leaves FP32's range may have a root within it
__device__ __forceinline__ float rstd_of(const GnArgs& a, double var) {
  if (var < 0.0) var = 0.0;
  var += (double)a.eps;
  return var > 1e-30 && var < 1e38 ? 1.f / sqrtf((float)var) : (float)(1.0 / sqrt(var));
}

// d = x - pivot, 0 past the group's end, and the sums of d and d^2
template <class T, int V, bool FULL>
__device__ __forceinline__ void add_about(const Raw<T, V>& r, int left, float pivot, float* s) {
  float d[V], q[2] = {0.f, 0.f};
  unpack<T, V>(r, d);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    d[i] = FULL || i < left ? d[i] - pivot : 0.f;
    q[i & 1] = __builtin_fmaf(d[i], d[i], q[i & 1]);
  }
  s[0] += tree<V>(d);
  s[1] += q[0] + q[1];
}

template <class T, int V, bool FULL, int ACT>
__device__ __forceinline__ void normalise(const GnArgs& a, const Rows<T, V, FULL>& y, int i, const Raw<T, V>& r, float mu,
                                          const float* scale, const float* beta) {
  float x[V];
  unpack<T, V>(r, x);
#pragma unroll
  for (int e = 0; e < V; ++e) x[e] = (x[e] - mu) * scale[e] + beta[e];
  activate<ACT, V>(x, a.act == PAINN_ACT_RELU);
  y.put(i, x);
}

// A team's sample (n = 0 rows: none).  Its statistics: the mean of the rows that
// it holds is the pivot K, then d = x - K and d^2 are summed over all of the
// sample's rows, in FP32:
//   mean = K + sum d / n,  variance = sum d^2 / n - (sum d / n)^2.
// With K the held rows' own mean the subtraction takes at most n / (held
// values) times the sums' rounding, whatever the mean.  The sums are formed again
// in FP64 where that is not enough: squares that leave FP32's range, a
// mean further from K than the deviation (rows held that say little of the rest;
// equal values, K off by a rounding), a sample far longer than max_rows says.
template <class T, int V, bool FULL, int ACT, int TB, bool REST>
__device__ __forceinline__ void team_forward(const GnArgs& a, const Place<V>& p, int team, int s, const Span& q, double* lds) {
  constexpr int NR = steps_held(TB);
  float* flds = (float*)lds;
  const Rows<T, V, FULL> x(a.x, a.ldx, p, q.a, q.b - q.a), y(a.out, a.ldo, p, q.a, q.b - q.a);
  Raw<T, V> v[NR];
#pragma unroll
  for (int i = 0; i < NR; ++i) v[i] = x.get(i);
  float sum[2] = {0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (i * p.rows < x.n) {
      float u[V];
      unpack<T, V>(v[i], u);
      sum[0] += tree<V>(u);
    }
  team_sum<TB, 1>(a, sum, team, flds);
  const int held = !REST || x.n < NR * p.rows ? x.n : NR * p.rows;
  const float pivot = held > 0 ? sum[0] * __builtin_amdgcn_rcpf((float)held * (float)a.cg) : 0.f;
  sum[0] = 0.f;
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (x.has(i)) add_about<T, V, FULL>(v[i], p.left, pivot, sum);
  for (int i0 = NR; REST && x.has(i0); i0 += 4) {
    Raw<T, V> w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x.get(i0 + i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (x.has(i0 + i)) add_about<T, V, FULL>(w[i], p.left, pivot, sum);
  }
  team_sum<TB, 2>(a, sum, team, flds);
  float mu = 0.f, rs = 0.f;
  bool wild = false;
  const float count = (float)x.n * (float)a.cg;
  if (x.n > 0) {
    // (a reciprocal and a root off by one step, and a Newton step each)
    float inv = __builtin_amdgcn_rcpf(count);
    inv = __builtin_fmaf(__builtin_fmaf(-count, inv, 1.f), inv, inv);
    const float d = sum[0] * inv, var = sum[1] * inv - d * d;
    const float ve = (var > 0.f || var != var ? var : 0.f) + a.eps;
    mu = pivot + d;
    rs = __builtin_amdgcn_rsqf(ve);
    rs = __builtin_fmaf(rs * 0.5f, __builtin_fmaf(-ve * rs, rs, 1.f), rs);
    wild = !(sum[1] < 1e38f) || !(ve > 1e-30f && ve < 1e38f) || d * d > ve ||
           (REST && (x.n >> 10) >= NR * p.rows);
  }
  if (team_any<TB>(wild)) {
    double t[2] = {0.0, 0.0};
    const float k = x.n > 0 ? first_value<T, V>(a, p, q.a) : 0.f;
    add_rows<T, V, FULL, 4>(x, k, t);
    team_sum<TB, 2>(a, t, team, lds);
    if (wild) {
      const double n = (double)x.n * a.cg, d = t[0] / n;
      mu = (float)((double)k + d);
      rs = rstd_of(a, t[1] / n - d * d);
    }
  }
  if (s >= 0 && p.row == 0 && p.left == a.cg) {
    if (a.mean) a.mean[(size_t)s * a.groups + p.group] = mu;
    if (a.rstd) a.rstd[(size_t)s * a.groups + p.group] = rs;
  }
  float scale[V], b[V];
  load_n<V>((const T*)a.gamma + p.col, p.left, scale);
  load_n<V>((const T*)a.beta + p.col, p.left, b);
#pragma unroll
  for (int i = 0; i < V; ++i) scale[i] *= rs;
#pragma unroll
  for (int i = 0; i < NR; ++i)
    if (x.has(i)) normalise<T, V, FULL, ACT>(a, y, i, v[i], mu, scale, b);
  // (out may be x: what is left of the sample is read before it is written, by the thread that writes it)
  for (int i0 = NR; REST && x.has(i0); i0 += 4) {
    Raw<T, V> w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x.get(i0 + i);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (x.has(i0 + i)) normalise<T, V, FULL, ACT>(a, y, i0 + i, w[i], mu, scale, b);
  }
}

// The longer samples' blocks, the other samples' blocks, the tiles' sums.  Where
// teams are a wave or less (TB = 64), the samples that such a team cannot hold
// come first, a wave each, so that no long chain of loads is begun when the rest
// is done.  Blocks are single waves then: a block of four holds its registers until
// the slowest ends (65,502 x 256 BF16, ragged: 36 us for 29), and a block of 256
// per long sample waits at its barriers (55).
template <class T, int V, bool FULL, int ACT, int TB>
__global__ void __launch_bounds__(TB) k_group_norm(GnArgs a) {
  __shared__ double lds[2 * TB];
  const int slab = blockIdx.x, blk = blockIdx.y;
  if (blk >= a.l_blocks + a.f_blocks) {
    const int t = blk - a.l_blocks - a.f_blocks;
    const Place<V> p(a, slab, threadIdx.x, TB);
    long_samples(a, t, [&](int slot, int, const Span&, long long lo, long long hi) {
      double s[2] = {0.0, 0.0};
      // the part's mean, and the squares about it
      const float k = first_value<T, V>(a, p, lo);
      add_rows<T, V, FULL, 8>(Rows<T, V, FULL>(a.x, a.ldx, p, lo, hi - lo), k, s);
      team_sum<TB, 2>(a, s, TB, lds);
      const double n = (double)(hi - lo) * a.cg, d = s[0] / n;
      if (p.row == 0 && p.left == a.cg)
        a.seg[((size_t)t * 2 + slot) * a.groups + p.group] = make_double2((double)k + d, s[1] - s[0] * d);
    });
    return;
  }
  const long long held = TB > 64 ? -1 : (long long)(a.team >> a.lpr_bits) * steps_held(64);
  if (blk < a.l_blocks || TB > 64) {
    const Place<V> p(a, slab, threadIdx.x, TB);
    longer_samples(a, blk, TB > 64 ? a.f_blocks : a.l_blocks, held + 1,
                   [&](int s, const Span& q) { team_forward<T, V, FULL, ACT, TB, true>(a, p, TB, s, q, lds); });
  } else if constexpr (TB == 64) {
    const int team = a.team, team_bits = 31 - __builtin_clz(team), teams = 64 >> team_bits, mine = threadIdx.x >> team_bits;
    const Place<V> p(a, slab, (int)threadIdx.x & (team - 1), team);
    for (long long s0 = (long long)(blk - a.l_blocks) * teams; s0 < a.samples; s0 += (long long)a.f_blocks * teams) {
      int s = s0 + mine < a.samples ? (int)(s0 + mine) : -1;
      Span q{0, 0};
      if (s >= 0) q = span(a, s);
      if (q.b - q.a > held) {
        q.b = q.a;
        s = -1;
      }
      if (team < 64 || s >= 0) team_forward<T, V, FULL, ACT, 64, false>(a, p, team, s, q, lds);
    }
  }
}

// The results of long samples, tile by tile.
template <class T, int V, bool FULL, int ACT, int TB>
__global__ void __launch_bounds__(TB) k_group_norm_tiles(GnArgs a) {
  __shared__ double lds[2 * TB];
  const int slab = blockIdx.x, t = (int)(gridDim.y - 1 - blockIdx.y);   // (the rows read last are in the caches)
  const Place<V> p(a, slab, threadIdx.x, TB);
  long_samples(a, t, [&](int, int sample, const Span& q, long long lo, long long hi) {
    // the parts' means and squares n, m, S: m = sum n m / N, then S + n (m - mean)^2
    const double n = (double)(q.b - q.a) * a.cg;
    double mean = 0.0, squares = 0.0;
    const int lane = p.row * a.lpg + (threadIdx.x & (a.lpg - 1)), lanes = p.rows * a.lpg;
    each_tile(a, q, p.group, lane, lanes, [&](double2 v, long long part) { mean += v.x * ((double)part * a.cg); });
    team_sum<TB, 1>(a, &mean, TB, lds);
    mean /= n;
    each_tile(a, q, p.group, lane, lanes, [&](double2 v, long long part) {
      squares += v.y + (v.x - mean) * (v.x - mean) * ((double)part * a.cg);
    });
    team_sum<TB, 1>(a, &squares, TB, lds);
    const float mu = (float)mean, rs = rstd_of(a, squares / n);
    if (lo == q.a && p.row == 0 && p.left == a.cg) {
      if (a.mean) a.mean[(size_t)sample * a.groups + p.group] = mu;
      if (a.rstd) a.rstd[(size_t)sample * a.groups + p.group] = rs;
    }
    float scale[V], b[V];
    load_n<V>((const T*)a.gamma + p.col, p.left, scale);
    load_n<V>((const T*)a.beta + p.col, p.left, b);
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] *= rs;
    const Rows<T, V, FULL> x(a.x, a.ldx, p, lo, hi - lo), y(a.out, a.ldo, p, lo, hi - lo);
    for (int i0 = 0; x.has(i0); i0 += 4) {
      Raw<T, V> w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = x.get(i0 + i);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (x.has(i0 + i)) normalise<T, V, FULL, ACT>(a, y, i0 + i, w[i], mu, scale, b);
    }
  });
}

template <class T>
painn_status run_fwd(painn_ctx* ctx, const Plan& p, const GnArgs& a) {
  const dim3 grid(p.slabs, p.l_blocks + p.f_blocks + p.tiles), tiles(p.slabs, p.tiles);
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM, true);
  with_form<T>(p, a.act, [&](auto v, auto full, auto act) {
    constexpr int V = decltype(v)::value;
    constexpr bool FULL = decltype(full)::value;
    constexpr int ACT = decltype(act)::value;
    if (p.tb == 64) k_group_norm<T, V, FULL, ACT, 64><<<grid, 64, 0, ctx->stream>>>(a);
    else if (p.tb == 256) k_group_norm<T, V, FULL, ACT, 256><<<grid, 256, 0, ctx->stream>>>(a);
    else k_group_norm<T, V, FULL, ACT, 512><<<grid, 512, 0, ctx->stream>>>(a);
    if (p.tiles && p.lpg <= 256) k_group_norm_tiles<T, V, FULL, ACT, 256><<<tiles, 256, 0, ctx->stream>>>(a);
    else if (p.tiles) k_group_norm_tiles<T, V, FULL, ACT, 512><<<tiles, 512, 0, ctx->stream>>>(a);
  });
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM, false);
  return launched(ctx, "group norm launch");
}

}  // namespace

extern "C" {

int64_t painn_group_norm_workspace(painn_precision precision, int64_t rows, int32_t cols, int32_t groups,
                                   int32_t n_samples, int64_t sample_rows, int64_t max_rows, int32_t backward) {
  if ((precision != PAINN_FP32 && precision != PAINN_BF16) || rows < 0 || rows > 0x7fffffffLL || cols < 1 || groups < 1 ||
      cols % groups || n_samples < 0 || sample_rows < 0)
    return 0;
  const Plan p = plan_of(precision == PAINN_BF16, rows, cols, groups, n_samples, sample_rows == 0, sample_rows, max_rows,
                         backward != 0);
  return (int64_t)(p.seg_bytes + p.part_bytes);
}

painn_status painn_group_norm(painn_ctx* ctx, const painn_group_norm_args* args) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!args) return fail(ctx, PAINN_E_ARG, "null arguments");
  const painn_group_norm_args& a = *args;
  painn_status st = shape_check(ctx, a.precision, a.rows, a.cols, a.groups, a.n_samples, a.offsets, a.sample_rows, a.max_rows,
                                a.activation, a.reserved);
  if (st != PAINN_OK) return st;
  if (!(a.eps >= 0.0) || !(a.eps <= 3.4e38) || (a.eps > 0.0 && (float)a.eps == 0.f))
    return fail(ctx, PAINN_E_ARG, "eps must be finite and not negative, in FP32 too");
  if (a.n_samples == 0) return PAINN_OK;
  if (!a.gamma || !a.beta) return fail(ctx, PAINN_E_ARG, "null array");
  if (a.rows > 0) {
    if (!a.x || !a.y) return fail(ctx, PAINN_E_ARG, "null array");
    if (a.ldx < a.cols || a.ldy < a.cols) return fail(ctx, PAINN_E_ARG, "a row stride is below cols");
    if (misplaced(a.y, a.ldy, a.x, a.ldx, a.rows)) return fail(ctx, PAINN_E_ARG, "y in place of x has another row stride");
  }
  const Plan p = plan_of(a.precision == PAINN_BF16, a.rows, a.cols, a.groups, a.n_samples, a.offsets != nullptr,
                         a.sample_rows, a.max_rows, false);
  if ((long long)p.slabs * (p.l_blocks + p.f_blocks + p.tiles) > LAUNCH_THREADS / 1024)
    return fail(ctx, PAINN_E_UNSUPPORTED, "more blocks than a launch holds");
  if (a.workspace_bytes < (int64_t)p.seg_bytes || (p.seg_bytes && !a.workspace))
    return fail(ctx, PAINN_E_ARG, "the workspace is too small: " + std::to_string(p.seg_bytes) + " bytes");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  GnArgs g{};
  fill(g, p, a, a.workspace);
  g.out = a.y; g.ldo = a.ldy; g.mean = a.mean; g.rstd = a.rstd; g.eps = (float)a.eps;
  return a.precision == PAINN_FP32 ? run_fwd<float>(ctx, p, g) : run_fwd<b16>(ctx, p, g);
}

}  // extern "C"

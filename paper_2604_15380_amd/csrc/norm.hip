// Layer norm and its reverse pass (FP32, BF16).
//
// A row is held in the registers of LPR lanes (16 to 64, or a block's 256), V
// values (16 bytes) per lane and step, NJ steps: the mean, then the variance
// about it, then the result, all from one read of the row, with the next row
// on its way meanwhile.  Rows too long for that are read again for each.  The
// lanes walk over the rows, so that gamma and beta are loaded once and the
// reverse pass's column sums (dgamma, dbeta) stay in registers until the end;
// each block then writes one partial row and k_norm_fold adds the blocks'
// partials in their order.  Bound by memory.
#include <type_traits>

#include "ops.h"

namespace {

using namespace ops;

constexpr int TB = 256;

// Sum over the row's LPR lanes.
template <int LPR>
__device__ __forceinline__ float row_sum(float x, float* lds) {
#pragma unroll
  for (int o = (LPR < 64 ? LPR : 64) / 2; o; o >>= 1) x += __shfl_xor(x, o);
  if constexpr (LPR > 64) {
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < LPR / 64; ++w) x += lds[w];
  }
  return x;
}

template <class T, int V, int NJ, int LPR>
__global__ void __launch_bounds__(TB) k_norm(long long rows, int cols, const T* x, long long ldx,
                                             const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                                             T* y, long long ldy, float* __restrict__ mean,
                                             float* __restrict__ rstd) {
  __shared__ float lds[4];
  constexpr int RPB = TB / LPR;                    // rows of a block at a time
  const int t = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const float width = (float)cols;
  float g[NJ][V], b[NJ][V], next[NJ][V];
  const long long step = (long long)gridDim.x * RPB;
  long long r = (long long)blockIdx.x * RPB + sub;
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (j * LPR + t) * V;
    if (r < rows) load_n<V>(x + r * ldx + c, cols - c, next[j]);
    load_n<V>(gamma + c, cols - c, g[j]);
    load_n<V>(beta + c, cols - c, b[j]);
  }
  // (y may be x: a row is read before it or any later one is written)
  for (; r < rows; r += step) {
    float v[NJ][V];
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = next[j][i];
      if (r + step < rows) load_n<V>(x + (r + step) * ldx + c, cols - c, next[j]);
    }
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int i = 0; i < V; ++i) s += v[j][i];
    const float mu = row_sum<LPR>(s, lds) / width;
    s = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[j][i] -= mu;
        s += c + i < cols ? v[j][i] * v[j][i] : 0.f;
      }
    }
    const float rs = 1.f / sqrtf(row_sum<LPR>(s, lds) / width + eps);
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + t) * V;
      float o[V];
#pragma unroll
      for (int i = 0; i < V; ++i) o[i] = v[j][i] * rs * g[j][i] + b[j][i];
      store_n<V>(y + r * ldy + c, cols - c, o);
    }
    if (t == 0) {
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
}

// Rows of any length, one block each.
template <class T>
__global__ void __launch_bounds__(TB) k_norm_long(long long rows, int cols, const T* x, long long ldx,
                                                  const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                                                  T* y, long long ldy, float* __restrict__ mean,
                                                  float* __restrict__ rstd) {
  __shared__ float lds[4];
  const float width = (float)cols;
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* xr = x + r * ldx;
    float s = 0.f, v, g, b;
    for (int c = threadIdx.x; c < cols; c += TB) {
      load<1>(xr + c, &v);
      s += v;
    }
    const float mu = row_sum<TB>(s, lds) / width;
    s = 0.f;
    for (int c = threadIdx.x; c < cols; c += TB) {
      load<1>(xr + c, &v);
      s += (v - mu) * (v - mu);
    }
    const float rs = 1.f / sqrtf(row_sum<TB>(s, lds) / width + eps);
    for (int c = threadIdx.x; c < cols; c += TB) {
      load<1>(xr + c, &v);
      load<1>(gamma + c, &g);
      load<1>(beta + c, &b);
      v = (v - mu) * rs * g + b;
      store<1>(y + r * ldy + c, &v);
    }
    if (threadIdx.x == 0) {
      if (mean) mean[r] = mu;
      if (rstd) rstd[r] = rs;
    }
  }
}

// With xh = (x - mean) rstd and a = dy gamma:
//   dx = rstd (a - mean(a) - xh mean(a xh)),  dgamma = sum dy xh,  dbeta = sum dy.
// part: [gridDim.x][2][cols] partial column sums, or null.
template <class T, int V, int NJ, int LPR>
__global__ void __launch_bounds__(TB) k_norm_bwd(long long rows, int cols, const T* dy, long long lddy,
                                                 const T* __restrict__ x, long long ldx, const T* __restrict__ gamma,
                                                 const float* __restrict__ mean, const float* __restrict__ rstd,
                                                 T* dx, long long lddx, float* __restrict__ part) {
  constexpr int RPB = TB / LPR, W = LPR * V * NJ;
  __shared__ float lds[4];
  __shared__ float acc[RPB > 1 ? W : 1];
  const int t = threadIdx.x % LPR, sub = threadIdx.x / LPR;
  const float width = (float)cols;
  float g[NJ][V], dg[NJ][V], db[NJ][V];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int c = (j * LPR + t) * V;
    load_n<V>(gamma + c, cols - c, g[j]);
#pragma unroll
    for (int i = 0; i < V; ++i) dg[j][i] = db[j][i] = 0.f;
  }
  for (long long r = (long long)blockIdx.x * RPB + sub; r < rows; r += (long long)gridDim.x * RPB) {
    const float mu = mean[r], rs = rstd[r];
    float d[NJ][V], h[NJ][V];
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + t) * V;
      load_n<V>(dy + r * lddy + c, cols - c, d[j]);
      load_n<V>(x + r * ldx + c, cols - c, h[j]);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int c = (j * LPR + t) * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        // (0 beyond the row, as dy is: -mu rs may be an infinity)
        h[j][i] = c + i < cols ? (h[j][i] - mu) * rs : 0.f;
        dg[j][i] += d[j][i] * h[j][i];
        db[j][i] += d[j][i];
        d[j][i] *= g[j][i];
        s1 += d[j][i];
        s2 += d[j][i] * h[j][i];
      }
    }
    if (dx) {
      s1 = row_sum<LPR>(s1, lds) / width;
      s2 = row_sum<LPR>(s2, lds) / width;
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int c = (j * LPR + t) * V;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = rs * (d[j][i] - s1 - h[j][i] * s2);
        store_n<V>(dx + r * lddx + c, cols - c, o);
      }
    }
  }
  if (!part) return;
  // the block's rows one after the other, then one partial row per block
  float* p = part + (size_t)blockIdx.x * 2 * cols;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if constexpr (RPB > 1) {
      for (int w = 0; w < RPB; ++w) {
        __syncthreads();
        if (sub == w) {
#pragma unroll
          for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const int c = (j * LPR + t) * V + i;
              const float s = k ? db[j][i] : dg[j][i];
              acc[c] = w ? acc[c] + s : s;
            }
        }
      }
      __syncthreads();
      for (int c = threadIdx.x; c < cols; c += TB) p[(size_t)k * cols + c] = acc[c];
    } else {
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int c = (j * LPR + t) * V;
        store_n<V>(p + (size_t)k * cols + c, cols - c, k ? db[j] : dg[j]);
      }
    }
  }
}

template <class T>
__global__ void __launch_bounds__(TB) k_norm_bwd_long(long long rows, int cols, const T* dy, long long lddy,
                                                      const T* __restrict__ x, long long ldx,
                                                      const T* __restrict__ gamma, const float* __restrict__ mean,
                                                      const float* __restrict__ rstd, T* dx, long long lddx) {
  __shared__ float lds[4];
  const float width = (float)cols;
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const float mu = mean[r], rs = rstd[r];
    float s1 = 0.f, s2 = 0.f, d, h, g;
    for (int c = threadIdx.x; c < cols; c += TB) {
      load<1>(dy + r * lddy + c, &d);
      load<1>(x + r * ldx + c, &h);
      load<1>(gamma + c, &g);
      s1 += d * g;
      s2 += d * g * ((h - mu) * rs);
    }
    s1 = row_sum<TB>(s1, lds) / width;
    s2 = row_sum<TB>(s2, lds) / width;
    for (int c = threadIdx.x; c < cols; c += TB) {
      load<1>(dy + r * lddy + c, &d);
      load<1>(x + r * ldx + c, &h);
      load<1>(gamma + c, &g);
      d = rs * (d * g - s1 - (h - mu) * rs * s2);
      store<1>(dx + r * lddx + c, &d);
    }
  }
}

// Column sums of long rows: block (b, k) has the rows of slice k of `slices`
// and 256 columns.
template <class T>
__global__ void __launch_bounds__(TB) k_norm_cols(long long rows, int cols, const T* __restrict__ dy, long long lddy,
                                                  const T* __restrict__ x, long long ldx,
                                                  const float* __restrict__ mean, const float* __restrict__ rstd,
                                                  float* __restrict__ part) {
  const int c = blockIdx.x * TB + threadIdx.x;
  if (c >= cols) return;
  float dg = 0.f, db = 0.f, d, h;
  for (long long r = blockIdx.y; r < rows; r += gridDim.y) {
    load<1>(dy + r * lddy + c, &d);
    load<1>(x + r * ldx + c, &h);
    dg += d * ((h - mean[r]) * rstd[r]);
    db += d;
  }
  part[((size_t)blockIdx.y * 2 + 0) * cols + c] = dg;
  part[((size_t)blockIdx.y * 2 + 1) * cols + c] = db;
}

// dgamma (blockIdx.y = 0) or dbeta (1): 32 columns per block at a time, the
// partial rows in 32 slices.
template <class T>
__global__ void __launch_bounds__(1024) k_norm_fold(int n, int cols, const float* __restrict__ part,
                                                    T* __restrict__ dgamma, T* __restrict__ dbeta) {
  __shared__ float s[32][33];
  const int q = threadIdx.x >> 5, l = threadIdx.x & 31;
  for (int c0 = blockIdx.x * 32; c0 < cols; c0 += gridDim.x * 32) {
    const int c = c0 + l;
    float a = 0.f;
    if (c < cols) {
#pragma unroll 8
      for (int k = q; k < n; k += 32) a += part[((size_t)k * 2 + blockIdx.y) * cols + c];
    }
    s[q][l] = a;
    __syncthreads();
    if (q == 0 && c < cols) {
      a = 0.f;
#pragma unroll
      for (int k = 0; k < 32; ++k) a += s[k][l];
      store<1>((blockIdx.y ? dbeta : dgamma) + c, &a);
    }
    __syncthreads();
  }
}

struct NormArgs {
  painn_ctx* ctx;
  long long rows;
  int cols;
  const void *x, *gamma, *beta, *dy;
  long long ldx, ldy, lddy, lddx;
  float eps;
  void *y, *dx, *dgamma, *dbeta;
  float *mean, *rstd;              // outputs of the forward
  const float *mu, *rs;            // inputs of the reverse pass
};

constexpr int NORM_GRID = 2048;     // blocks of a launch: 8 per CU
constexpr int NORM_GRID_BWD = 1024; // and of the reverse pass, whose partial rows are folded
constexpr int NORM_FOLD = 65536;    // and of that, along the columns
constexpr int NORM_COLS = 1 << 30;  // a row's columns at most: their count steps by up to 2^21 in an int

inline int grid_for(long long rows, int rpb, int most) {
  const long long n = (rows + rpb - 1) / rpb;
  return (int)(n < most ? n : most);
}

template <class T, int V, int NJ, int LPR>
void norm_fwd(const NormArgs& a) {
  k_norm<T, V, NJ, LPR><<<grid_for(a.rows, TB / LPR, NORM_GRID), TB, 0, a.ctx->stream>>>(
      a.rows, a.cols, (const T*)a.x, a.ldx, (const T*)a.gamma, (const T*)a.beta, a.eps, (T*)a.y, a.ldy, a.mean,
      a.rstd);
}
template <class T, int V, int NJ, int LPR>
void norm_bwd(const NormArgs& a, int grid, float* part) {
  k_norm_bwd<T, V, NJ, LPR><<<grid, TB, 0, a.ctx->stream>>>(a.rows, a.cols, (const T*)a.dy, a.lddy, (const T*)a.x,
                                                            a.ldx, (const T*)a.gamma, a.mu, a.rs, (T*)a.dx, a.lddx,
                                                            part);
}

// The form for a row of `cols`: f(V, NJ, LPR) with the fewest lanes that hold it
// in one step, then more steps, then a whole block.  False: too long.
#define NORM_FORM(V, NJ, LPR) \
  if (cols <= V * NJ * LPR) { f(std::integral_constant<int, V>(), std::integral_constant<int, NJ>(), \
                                std::integral_constant<int, LPR>()); return true; }
template <class T, class F>
bool norm_form(int cols, F&& f) {
  constexpr int V = 16 / sizeof(T);
  NORM_FORM(V, 1, 16)
  NORM_FORM(V, 1, 32)
  NORM_FORM(V, 1, 64)
  NORM_FORM(V, 2, 64)
  NORM_FORM(V, 4, 64)
  NORM_FORM(V, 2, 256)
  NORM_FORM(V, 4, 256)
  if constexpr (sizeof(T) == 4) { NORM_FORM(V, 8, 256) }
  return false;
}
#undef NORM_FORM

template <class T>
painn_status run_norm(const NormArgs& a) {
  painn_ctx* ctx = a.ctx;
  prof_mark(ctx->prof, ctx->stream, KC_NORM, true);
  const bool held = norm_form<T>(a.cols, [&](auto v, auto nj, auto lpr) {
    norm_fwd<T, decltype(v)::value, decltype(nj)::value, decltype(lpr)::value>(a);
  });
  if (!held)
    k_norm_long<T><<<grid_for(a.rows, 1, NORM_GRID), TB, 0, ctx->stream>>>(
        a.rows, a.cols, (const T*)a.x, a.ldx, (const T*)a.gamma, (const T*)a.beta, a.eps, (T*)a.y, a.ldy, a.mean,
        a.rstd);
  prof_mark(ctx->prof, ctx->stream, KC_NORM, false);
  return launched(ctx, "layer norm launch");
}

template <class T>
painn_status run_norm_bwd(const NormArgs& a) {
  painn_ctx* ctx = a.ctx;
  const int c = a.cols;
  int rpb = 0;                 // rows of a block at a time; 0: too long to hold
  norm_form<T>(c, [&](auto, auto, auto lpr) { rpb = TB / decltype(lpr)::value; });
  const int grid = grid_for(a.rows, rpb ? rpb : 1, NORM_GRID_BWD);
  const int slices = rpb ? grid : grid_for(a.rows, 1, 64);
  float* part = nullptr;
  if (a.dgamma && slices) {
    const painn_status st = ops_workspace(ctx, (size_t)slices * 2 * c * sizeof(float));
    if (st != PAINN_OK) return st;
    part = (float*)ctx->ows.p;
  }
  prof_mark(ctx->prof, ctx->stream, KC_NORM_BWD, true);
  if (a.rows > 0 && rpb) {
    norm_form<T>(c, [&](auto v, auto nj, auto lpr) {
      norm_bwd<T, decltype(v)::value, decltype(nj)::value, decltype(lpr)::value>(a, grid, part);
    });
  } else if (a.rows > 0) {
    // the column sums first: dx may overwrite dy
    if (part)
      k_norm_cols<T><<<dim3((c + TB - 1) / TB, slices), TB, 0, ctx->stream>>>(
          a.rows, c, (const T*)a.dy, a.lddy, (const T*)a.x, a.ldx, a.mu, a.rs, part);
    if (a.dx)
      k_norm_bwd_long<T><<<grid, TB, 0, ctx->stream>>>(a.rows, c, (const T*)a.dy, a.lddy, (const T*)a.x, a.ldx,
                                                       (const T*)a.gamma, a.mu, a.rs, (T*)a.dx, a.lddx);
  }
  if (a.dgamma)
    k_norm_fold<T><<<dim3(grid_for(c, 32, NORM_FOLD), 2), 1024, 0, ctx->stream>>>(slices, c, part, (T*)a.dgamma,
                                                                                (T*)a.dbeta);
  prof_mark(ctx->prof, ctx->stream, KC_NORM_BWD, false);
  return launched(ctx, "layer norm reverse launch");
}

painn_status norm_check(painn_ctx* ctx, int prec, int64_t rows, int32_t cols) {
  if (prec == PAINN_FP64) return fail(ctx, PAINN_E_UNSUPPORTED, "layer norm runs in FP32 and BF16");
  if (prec != PAINN_FP32 && prec != PAINN_BF16) return fail(ctx, PAINN_E_ARG, "unknown precision");
  if (cols < 1) return fail(ctx, PAINN_E_ARG, "cols must be at least 1");
  if (rows < 0) return fail(ctx, PAINN_E_ARG, "rows must not be negative");
  if (cols > NORM_COLS) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 2^30 columns");
  return PAINN_OK;
}

}  // namespace

extern "C" {

painn_status painn_layer_norm(painn_ctx* ctx, painn_precision precision, int64_t rows, int32_t cols, const void* x,
                              int64_t ldx, const void* gamma, const void* beta, double eps, void* y, int64_t ldy,
                              float* mean, float* rstd) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  painn_status st = norm_check(ctx, precision, rows, cols);
  if (st != PAINN_OK) return st;
  // (an eps that is 0 in FP32 alone would make constant rows NaN)
  if (!(eps >= 0.0) || !(eps <= 3.4e38) || (eps > 0.0 && (float)eps == 0.f))
    return fail(ctx, PAINN_E_ARG, "eps must be finite and not negative, in FP32 too");
  if (rows == 0) return PAINN_OK;
  if (!x || !gamma || !beta || !y) return fail(ctx, PAINN_E_ARG, "null array");
  if (ldx < cols || ldy < cols) return fail(ctx, PAINN_E_ARG, "a row stride is below cols");
  if (misplaced(y, ldy, x, ldx, rows)) return fail(ctx, PAINN_E_ARG, "y in place of x has another row stride");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  NormArgs a{};
  a.ctx = ctx; a.rows = rows; a.cols = cols; a.x = x; a.ldx = ldx; a.gamma = gamma; a.beta = beta;
  a.eps = (float)eps; a.y = y; a.ldy = ldy; a.mean = mean; a.rstd = rstd;
  return precision == PAINN_FP32 ? run_norm<float>(a) : run_norm<b16>(a);
}

painn_status painn_layer_norm_backward(painn_ctx* ctx, painn_precision precision, int64_t rows, int32_t cols,
                                       const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* gamma,
                                       const float* mean, const float* rstd, void* dx, int64_t lddx, void* dgamma,
                                       void* dbeta) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  painn_status st = norm_check(ctx, precision, rows, cols);
  if (st != PAINN_OK) return st;
  if (!dgamma != !dbeta) return fail(ctx, PAINN_E_ARG, "dgamma and dbeta are formed together");
  if (rows > 0) {
    if (!dy || !x || !gamma || !mean || !rstd) return fail(ctx, PAINN_E_ARG, "null array");
    if (lddy < cols || ldx < cols || (dx && lddx < cols)) return fail(ctx, PAINN_E_ARG, "a row stride is below cols");
    if (misplaced(dx, lddx, dy, lddy, rows)) return fail(ctx, PAINN_E_ARG, "dx in place of dy has another row stride");
  }
  if (!dgamma && (!dx || rows == 0)) return PAINN_OK;
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  NormArgs a{};
  a.ctx = ctx; a.rows = rows; a.cols = cols; a.dy = dy; a.lddy = lddy; a.x = x; a.ldx = ldx; a.gamma = gamma;
  a.mu = mean; a.rs = rstd; a.dx = dx; a.lddx = lddx; a.dgamma = dgamma; a.dbeta = dbeta;
  return precision == PAINN_FP32 ? run_norm_bwd<float>(a) : run_norm_bwd<b16>(a);
}

}  // extern "C"

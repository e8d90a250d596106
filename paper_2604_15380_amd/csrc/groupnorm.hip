// Group norm with an activation, channels last, over the rows of ragged samples,
// and its reverse pass (FP32, BF16).
//
// A set is a sample's rows times a group's columns.  Its statistics come from
// the sums of x and x^2 in FP64, so that neither the order nor a mean far from
// 0 costs digits; the reverse pass takes the sums of a and a xh.  Bound by
// memory: x (and dy) should be read once.  A team of threads therefore holds a
// sample's rows of one slab (whole groups, 128 bytes or more of a row, so that
// no line is read by two teams) in registers between its sums and its result;
// rows past those are read again.  How many threads a team has goes by the
// samples' usual length, from a few lanes to a block of 1,024.
//
// Samples longer than `limit` would leave the chip to a few teams.  They are
// cut into tiles of R <= limit rows: the tiles' sums are formed by further
// blocks of the first launch, and a second launch adds a sample's tiles, in
// their order, and writes its result.  A tile meets at most two such samples,
// the ones that hold its first and its last row, which gives every (tile,
// sample) its place without a list.
#include <type_traits>

#include "fold.h"
#include "ops.h"

namespace {

using namespace ops;

constexpr int NR = 8;               // row steps that a team holds in registers
constexpr int TILE_MIN = 64, TILES = 512;   // rows of a tile at least; tiles at most
constexpr int GN_COLS = 4096;       // columns of a group at most (a block's lanes hold them)
constexpr int BLOCKS_BWD = 2048;    // blocks of the reverse pass, over all slabs, whose column sums are folded

struct GnArgs {
  long long rows;
  int cols, groups, cg, act;
  const int* offsets;               // null: equal samples of sample_rows rows
  long long sample_rows;
  int samples;
  const void *x, *dy, *gamma, *beta;
  long long ldx, lddy, ldo;
  void* out;                        // y or dx; null: no dx wanted
  float *mean, *rstd;               // forward's outputs
  const float *mu, *rs;             // reverse pass's inputs
  float eps;
  int lpg, gb, slabs;               // lanes of a group, groups and number of slabs
  int team;                         // threads of a sample's team
  int f_blocks;                     // blocks of teams per slab; the tiles' blocks follow
  long long limit;                  // rows that a team takes on
  int tile, tiles;                  // rows of a tile, tiles (0: no sample is longer than limit)
  double2* seg;                     // [tiles][2][groups] sums
  float* part;                      // [f_blocks + tiles][2][cols] column sums of the reverse pass, or null
};

// ---- a slab of a row ----------------------------------------------------------
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

// A thread's place: V columns of a group of the slab, and which of the team's
// rows.
template <int V>
struct Place {
  int group, col, left;             // left: columns from col to the group's end, <= 0 for an idle lane
  int row, rows;                    // the thread's row of the team's
  __device__ __forceinline__ Place(const GnArgs& a, int slab, int t, int team) {
    const int l = t & (a.lpg - 1), q = (t / a.lpg) & (a.gb - 1), lpr = a.lpg * a.gb;
    group = slab * a.gb + q;
    left = group < a.groups ? a.cg - l * V : 0;
    col = left > 0 ? group * a.cg + l * V : 0;
    row = t / lpr;
    rows = team / lpr;
  }
};

// Sums over a group's lanes and the team's rows, in every thread of them.
// TB = 0: teams of at most 64 lanes; else the block is the team, with lds
// [TB / 64][64].
template <int TB>
__device__ __forceinline__ double2 team_sum(const GnArgs& a, double2 s, int team, double2* lds) {
  const int lpr = a.lpg * a.gb, in_wave = TB ? 64 : team;
  for (int o = 1; o < a.lpg && o < in_wave; o <<= 1) {
    s.x += __shfl_xor(s.x, o);
    s.y += __shfl_xor(s.y, o);
  }
  for (int o = lpr; o < in_wave; o <<= 1) {
    s.x += __shfl_xor(s.x, o);
    s.y += __shfl_xor(s.y, o);
  }
  if constexpr (TB > 0) {
    const int lane = threadIdx.x & 63, q = (threadIdx.x / a.lpg) & (a.gb - 1);
    __syncthreads();
    if (lane < lpr && (lane & (a.lpg - 1)) == 0) lds[(threadIdx.x >> 6) * 64 + q] = s;
    __syncthreads();
    s = make_double2(0.0, 0.0);
    for (int w = 0; w < TB / 64; ++w) {
      const double2 v = lds[w * 64 + q];
      s.x += v.x;
      s.y += v.y;
    }
  }
  return s;
}

struct Span {
  long long a, b;
};
__device__ __forceinline__ long long bound(const GnArgs& a, int s) {
  const int o = a.offsets[s];
  return o < 0 ? 0 : o > a.rows ? a.rows : (long long)o;
}
__device__ __forceinline__ Span span(const GnArgs& a, int s) {
  if (!a.offsets) return Span{s * a.sample_rows, (s + 1) * a.sample_rows};
  const long long lo = bound(a, s), hi = bound(a, s + 1);
  return Span{lo, hi < lo ? lo : hi};
}
// The sample that holds a row, or -1: of the samples that begin at or before it
// the last one, found by the wave in steps of 64.
__device__ __forceinline__ int sample_of(const GnArgs& a, long long row) {
  if (!a.offsets) {
    const long long s = row / a.sample_rows;
    return s < a.samples ? (int)s : -1;
  }
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.samples;        // among [lo, lo + n)
  while (n > 1) {
    const int step = (n + 63) / 64, s = lane * step;
    const bool before = s < n && bound(a, lo + s) <= row;
    const int k = __popcll(__ballot(before));
    const int at = k > 0 ? (k - 1) * step : 0;
    n = n - at < step ? n - at : step;
    lo += at;
  }
  const Span p = span(a, lo);
  return row >= p.a && row < p.b ? lo : -1;
}

// ---- forward --------------------------------------------------------------------
template <class T, int V>
__device__ __forceinline__ void add_raw(const Raw<T, V>& r, double2& s) {
  float x[V];
  unpack<T, V>(r, x);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    const double d = (double)x[i];
    s.x += d;
    s.y = __builtin_fma(d, d, s.y);
  }
}

// mean and rstd from a set's sums over n values
__device__ __forceinline__ void statistics(const GnArgs& a, double2 s, double n, float& mu, float& rs) {
  const double m = s.x / n;
  double var = s.y / n - m * m;
  if (var < 0.0) var = 0.0;
  var += (double)a.eps;
  mu = (float)m;
  // (a variance past FP32's range has a root within it)
  rs = var < 1e38 ? 1.f / sqrtf((float)var) : (float)(1.0 / sqrt(var));
}

template <class T, int V, bool FULL>
__device__ __forceinline__ void put(const GnArgs& a, const Place<V>& p, long long row, const float* o) {
  T* y = (T*)a.out + row * a.ldo + p.col;
  if constexpr (FULL) store<V>(y, o);
  else store_n<V>(y, p.left, o);
}

template <class T, int V, bool FULL>
__device__ __forceinline__ void normalise(const GnArgs& a, const Place<V>& p, long long row, const Raw<T, V>& r,
                                          float mu, const float* scale, const float* beta) {
  float x[V];
  unpack<T, V>(r, x);
#pragma unroll
  for (int i = 0; i < V; ++i) x[i] = (x[i] - mu) * scale[i] + beta[i];
  act<V>(x, a.act);
  put<T, V, FULL>(a, p, row, x);
}

template <class T, int V, bool FULL>
__device__ __forceinline__ Raw<T, V> get(const void* x, long long ld, const Place<V>& p, long long row, long long end) {
  if ((FULL || p.left > 0) && row < end) return load_raw<T, V, FULL>((const T*)x + row * ld + p.col, p.left);
  return zero_raw<T, V>();
}

// A tile's sums for slot 0 (the sample of its first row) and 1 (of its last,
// if another), of samples longer than the limit.
template <class F>
__device__ __forceinline__ void long_samples(const GnArgs& a, int t, F&& f) {
  const long long r0 = (long long)t * a.tile, r1 = r0 + a.tile < a.rows ? r0 + a.tile : a.rows;
  const int first = sample_of(a, r0), last = sample_of(a, r1 - 1);
  for (int slot = 0; slot < 2; ++slot) {
    const int s = slot ? last : first;
    if (s < 0 || (slot && last == first)) continue;
    const Span p = span(a, s);
    if (p.b - p.a <= a.limit) continue;
    f(slot, s, p, p.a > r0 ? p.a : r0, p.b < r1 ? p.b : r1);
  }
}

// A long sample's sums: of its tiles, in an order that depends on the sample
// alone.
__device__ __forceinline__ double2 tiles_sum(const GnArgs& a, const Span& p, int group, int lane, int lanes) {
  double2 s = make_double2(0.0, 0.0);
  if (group >= a.groups) return s;
  const int from = (int)(p.a / a.tile), to = (int)((p.b - 1) / a.tile);
  for (int u = from + lane; u <= to; u += lanes) {
    const int slot = u == from && p.a % a.tile != 0;
    const double2 v = a.seg[((size_t)u * 2 + slot) * a.groups + group];
    s.x += v.x;
    s.y += v.y;
  }
  return s;
}

// Teams' blocks (f_blocks per slab), then the tiles' sums.
template <class T, int V, bool FULL, int TB>
__global__ void __launch_bounds__(TB ? TB : 256) k_group_norm(GnArgs a) {
  __shared__ double2 lds[TB ? TB : 256];
  const int slab = blockIdx.x % a.slabs, blk = blockIdx.x / a.slabs;
  if (blk >= a.f_blocks) {
    constexpr int TT = TB ? TB : 256;
    const Place<V> p(a, slab, threadIdx.x, TT);
    const int t = blk - a.f_blocks;
    long_samples(a, t, [&](int slot, int, const Span&, long long lo, long long hi) {
      double2 s = make_double2(0.0, 0.0);
      for (long long r = lo + p.row; r < hi; r += (long long)NR * p.rows) {
        Raw<T, V> v[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) v[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, hi);
#pragma unroll
        for (int i = 0; i < NR; ++i) add_raw<T, V>(v[i], s);
      }
      s = team_sum<TT>(a, s, TT, lds);
      if (p.row == 0 && p.left == a.cg) a.seg[((size_t)t * 2 + slot) * a.groups + p.group] = s;
    });
    return;
  }
  const int team = TB ? TB : a.team, teams = TB ? 1 : 256 / team;
  const int mine = TB ? 0 : (int)threadIdx.x / team;
  const Place<V> p(a, slab, TB ? (int)threadIdx.x : (int)threadIdx.x & (team - 1), team);
  float g[V], b[V];
#pragma unroll
  for (int i = 0; i < V; ++i) g[i] = b[i] = 0.f;
  load_n<V>((const T*)a.gamma + p.col, p.left, g);
  load_n<V>((const T*)a.beta + p.col, p.left, b);
  for (long long s0 = (long long)blk * teams; s0 < a.samples; s0 += (long long)a.f_blocks * teams) {
    const bool some = s0 + mine < a.samples;
    const int s = some ? (int)(s0 + mine) : 0;
    Span q = span(a, s);
    const bool skip = !some || q.b - q.a > a.limit;
    if (skip) q.b = q.a;
    Raw<T, V> v[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) v[i] = get<T, V, FULL>(a.x, a.ldx, p, q.a + p.row + (long long)i * p.rows, q.b);
    double2 sum = make_double2(0.0, 0.0);
#pragma unroll
    for (int i = 0; i < NR; ++i)
      if (q.a + (long long)i * p.rows < q.b) add_raw<T, V>(v[i], sum);
    for (long long r = q.a + p.row + (long long)NR * p.rows; r < q.b; r += 4LL * p.rows) {
      Raw<T, V> w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, q.b);
#pragma unroll
      for (int i = 0; i < 4; ++i) add_raw<T, V>(w[i], sum);
    }
    sum = team_sum<TB>(a, sum, team, lds);
    float mu = 0.f, rs = 0.f;
    if (q.b > q.a) statistics(a, sum, (double)(q.b - q.a) * a.cg, mu, rs);
    if (!skip && p.row == 0 && p.left == a.cg) {
      if (a.mean) a.mean[(size_t)s * a.groups + p.group] = mu;
      if (a.rstd) a.rstd[(size_t)s * a.groups + p.group] = rs;
    }
    if (!FULL && p.left <= 0) continue;
    float scale[V];
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] = rs * g[i];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const long long r = q.a + p.row + (long long)i * p.rows;
      if (r < q.b) normalise<T, V, FULL>(a, p, r, v[i], mu, scale, b);
    }
    // (out may be x: what is left of the sample is read before it is written, by the thread that writes it)
    for (long long r = q.a + p.row + (long long)NR * p.rows; r < q.b; r += 4LL * p.rows) {
      Raw<T, V> w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, q.b);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r + (long long)i * p.rows < q.b) normalise<T, V, FULL>(a, p, r + (long long)i * p.rows, w[i], mu, scale, b);
    }
  }
}

// The results of long samples, tile by tile.
template <class T, int V, bool FULL, int TB>
__global__ void __launch_bounds__(TB) k_group_norm_tiles(GnArgs a) {
  __shared__ double2 lds[TB];
  const int slab = blockIdx.x % a.slabs, t = blockIdx.x / a.slabs;
  const Place<V> p(a, slab, threadIdx.x, TB);
  long_samples(a, t, [&](int, int sample, const Span& q, long long lo, long long hi) {
    const int lane = threadIdx.x & (a.lpg - 1);
    const double2 sum = team_sum<TB>(a, tiles_sum(a, q, p.group, p.row * a.lpg + lane, p.rows * a.lpg), TB, lds);
    float mu, rs;
    statistics(a, sum, (double)(q.b - q.a) * a.cg, mu, rs);
    if (lo == q.a && p.row == 0 && p.left == a.cg) {
      if (a.mean) a.mean[(size_t)sample * a.groups + p.group] = mu;
      if (a.rstd) a.rstd[(size_t)sample * a.groups + p.group] = rs;
    }
    if (!FULL && p.left <= 0) return;
    float scale[V], b[V];
    load_n<V>((const T*)a.gamma + p.col, p.left, scale);
    load_n<V>((const T*)a.beta + p.col, p.left, b);
#pragma unroll
    for (int i = 0; i < V; ++i) scale[i] *= rs;
    for (long long r = lo + p.row; r < hi; r += 4LL * p.rows) {
      Raw<T, V> w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, hi);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (r + (long long)i * p.rows < hi) normalise<T, V, FULL>(a, p, r + (long long)i * p.rows, w[i], mu, scale, b);
    }
  });
}

// ---- reverse pass -----------------------------------------------------------------
// With xh = (x - mean) rstd, dz = dy act'(xh gamma + beta) and a = dz gamma:
//   dx = rstd (a - mean(a) - xh mean(a xh)),  dgamma = sum dz xh,  dbeta = sum dz,
// the means over the set.
template <class T, int V>
struct Grads {
  float xh[V], dz[V];
  __device__ __forceinline__ Grads(const GnArgs& a, const Place<V>& p, const Raw<T, V>& x, const Raw<T, V>& dy, float mu,
                                   float rs, const float* g, const float* b) {
    float z[V];
    unpack<T, V>(x, xh);
    unpack<T, V>(dy, dz);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      // (0 past the group, as dy is: (0 - mu) rs may be an infinity)
      xh[i] = i < p.left ? (xh[i] - mu) * rs : 0.f;
      z[i] = xh[i] * g[i] + b[i];
    }
    mul_slope<V>(dz, z, a.act);
  }
};
// (FP32 over a thread's rows of one load, FP64 beyond)
template <class T, int V>
__device__ __forceinline__ void add_grads(const Grads<T, V>& d, const float* g, double2& s, float* dg, float* db) {
  float s1 = 0.f, s2 = 0.f;
#pragma unroll
  for (int i = 0; i < V; ++i) {
    dg[i] += d.dz[i] * d.xh[i];
    db[i] += d.dz[i];
    const float u = d.dz[i] * g[i];
    s1 += u;
    s2 += u * d.xh[i];
  }
  s.x += (double)s1;
  s.y += (double)s2;
}
template <class T, int V, bool FULL>
__device__ __forceinline__ void put_dx(const GnArgs& a, const Place<V>& p, long long row, const Grads<T, V>& d,
                                       const float* g, float rs, float m1, float m2) {
  float o[V];
#pragma unroll
  for (int i = 0; i < V; ++i) o[i] = rs * (d.dz[i] * g[i] - m1 - d.xh[i] * m2);
  put<T, V, FULL>(a, p, row, o);
}

template <class T, int V, bool FULL, int TB>
__global__ void __launch_bounds__(TB ? TB : 256) k_group_norm_bwd(GnArgs a) {
  constexpr int TT = TB ? TB : 256;
  __shared__ double2 lds[TT];
  extern __shared__ float acc[];        // [2][lanes of a row * V]
  const int slab = blockIdx.x % a.slabs, blk = blockIdx.x / a.slabs, lpr = a.lpg * a.gb;
  const bool tiles = blk >= a.f_blocks;
  const int team = TB || tiles ? TT : a.team, teams = TT / team;
  const int mine = (int)threadIdx.x / team;
  const Place<V> p(a, slab, (int)threadIdx.x & (team - 1), team);
  float g[V], b[V], dg[V], db[V];
#pragma unroll
  for (int i = 0; i < V; ++i) g[i] = b[i] = dg[i] = db[i] = 0.f;
  load_n<V>((const T*)a.gamma + p.col, p.left, g);
  load_n<V>((const T*)a.beta + p.col, p.left, b);
  const bool idle = !FULL && p.left <= 0;
  if (tiles) {
    const int t = blk - a.f_blocks;
    long_samples(a, t, [&](int slot, int sample, const Span&, long long lo, long long hi) {
      const float mu = idle ? 0.f : a.mu[(size_t)sample * a.groups + p.group];
      const float rs = idle ? 0.f : a.rs[(size_t)sample * a.groups + p.group];
      double2 s = make_double2(0.0, 0.0);
      for (long long r = lo + p.row; r < hi; r += 4LL * p.rows) {
        Raw<T, V> x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          x[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, hi);
          y[i] = get<T, V, FULL>(a.dy, a.lddy, p, r + (long long)i * p.rows, hi);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (r + (long long)i * p.rows < hi)
            add_grads<T, V>(Grads<T, V>(a, p, x[i], y[i], mu, rs, g, b), g, s, dg, db);
      }
      s = team_sum<TT>(a, s, TT, lds);
      if (p.row == 0 && p.left == a.cg) a.seg[((size_t)t * 2 + slot) * a.groups + p.group] = s;
    });
  } else {
    for (long long s0 = (long long)blk * teams; s0 < a.samples; s0 += (long long)a.f_blocks * teams) {
      const bool some = s0 + mine < a.samples;
      const int s = some ? (int)(s0 + mine) : 0;
      Span q = span(a, s);
      if (!some || q.b - q.a > a.limit) q.b = q.a;
      Raw<T, V> x[NR], y[NR];
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        x[i] = get<T, V, FULL>(a.x, a.ldx, p, q.a + p.row + (long long)i * p.rows, q.b);
        y[i] = get<T, V, FULL>(a.dy, a.lddy, p, q.a + p.row + (long long)i * p.rows, q.b);
      }
      const float mu = idle ? 0.f : a.mu[(size_t)s * a.groups + p.group];
      const float rs = idle ? 0.f : a.rs[(size_t)s * a.groups + p.group];
      double2 sum = make_double2(0.0, 0.0);
#pragma unroll
      for (int i = 0; i < NR; ++i)
        if (q.a + p.row + (long long)i * p.rows < q.b)
          add_grads<T, V>(Grads<T, V>(a, p, x[i], y[i], mu, rs, g, b), g, sum, dg, db);
      for (long long r = q.a + p.row + (long long)NR * p.rows; r < q.b; r += 2LL * p.rows) {
        Raw<T, V> u[2], w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          u[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, q.b);
          w[i] = get<T, V, FULL>(a.dy, a.lddy, p, r + (long long)i * p.rows, q.b);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (r + (long long)i * p.rows < q.b)
            add_grads<T, V>(Grads<T, V>(a, p, u[i], w[i], mu, rs, g, b), g, sum, dg, db);
      }
      if (!a.out) continue;
      sum = team_sum<TB>(a, sum, team, lds);
      if (idle || q.b == q.a) continue;
      const double inv = 1.0 / ((double)(q.b - q.a) * a.cg);
      const float m1 = (float)(sum.x * inv), m2 = (float)(sum.y * inv);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const long long r = q.a + p.row + (long long)i * p.rows;
        if (r < q.b) put_dx<T, V, FULL>(a, p, r, Grads<T, V>(a, p, x[i], y[i], mu, rs, g, b), g, rs, m1, m2);
      }
      for (long long r = q.a + p.row + (long long)NR * p.rows; r < q.b; r += 2LL * p.rows) {
        Raw<T, V> u[2], w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          u[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, q.b);
          w[i] = get<T, V, FULL>(a.dy, a.lddy, p, r + (long long)i * p.rows, q.b);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const long long rr = r + (long long)i * p.rows;
          if (rr < q.b) put_dx<T, V, FULL>(a, p, rr, Grads<T, V>(a, p, u[i], w[i], mu, rs, g, b), g, rs, m1, m2);
        }
      }
    }
  }
  if (!a.part) return;
  // the block's column sums: a wave's rows, then wave after wave
  for (int o = lpr; o < 64; o <<= 1) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      dg[i] += __shfl_xor(dg[i], o);
      db[i] += __shfl_xor(db[i], o);
    }
  }
  const int width = lpr * V, at = (threadIdx.x & (lpr - 1)) * V, per = lpr > 64 ? lpr / 64 : 1;
  for (int w = 0; w < TT / 64; w += per) {
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
  for (int c = threadIdx.x; c < many; c += TT) {
    const int q = c / a.cg, k = q * a.lpg * V + c - q * a.cg;
    out[c0 + c] = acc[k];
    out[a.cols + c0 + c] = acc[width + k];
  }
}

// dx of long samples, tile by tile.
template <class T, int V, bool FULL, int TB>
__global__ void __launch_bounds__(TB) k_group_norm_bwd_tiles(GnArgs a) {
  __shared__ double2 lds[TB];
  const int slab = blockIdx.x % a.slabs, t = blockIdx.x / a.slabs;
  const Place<V> p(a, slab, threadIdx.x, TB);
  long_samples(a, t, [&](int, int sample, const Span& q, long long lo, long long hi) {
    const int lane = threadIdx.x & (a.lpg - 1);
    const double2 sum = team_sum<TB>(a, tiles_sum(a, q, p.group, p.row * a.lpg + lane, p.rows * a.lpg), TB, lds);
    if (!FULL && p.left <= 0) return;
    const double inv = 1.0 / ((double)(q.b - q.a) * a.cg);
    const float m1 = (float)(sum.x * inv), m2 = (float)(sum.y * inv);
    const float mu = a.mu[(size_t)sample * a.groups + p.group], rs = a.rs[(size_t)sample * a.groups + p.group];
    float g[V], b[V];
    load_n<V>((const T*)a.gamma + p.col, p.left, g);
    load_n<V>((const T*)a.beta + p.col, p.left, b);
    for (long long r = lo + p.row; r < hi; r += 4LL * p.rows) {
      Raw<T, V> x[4], y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[i] = get<T, V, FULL>(a.x, a.ldx, p, r + (long long)i * p.rows, hi);
        y[i] = get<T, V, FULL>(a.dy, a.lddy, p, r + (long long)i * p.rows, hi);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const long long rr = r + (long long)i * p.rows;
        if (rr < hi) put_dx<T, V, FULL>(a, p, rr, Grads<T, V>(a, p, x[i], y[i], mu, rs, g, b), g, rs, m1, m2);
      }
    }
  });
}

// ---- the plan -----------------------------------------------------------------------
int pow2_at_least(long long x) {
  int p = 1;
  while (p < x) p <<= 1;
  return p;
}

struct Plan {
  int v, lpg, gb, slabs, team, tb, f_blocks, tile, tiles;
  bool full;
  long long limit;
  size_t seg_bytes, part_bytes;
};

// max_rows: the longest sample where the caller knows it, else 0.
Plan plan_of(bool bf16, long long rows, int cols, int groups, int samples, bool ragged, long long sample_rows,
             long long max_rows, bool backward) {
  Plan p{};
  const int size = bf16 ? 2 : 4, cg = cols / groups, wide = 16 / size;
  p.v = cg <= 2 ? 1 : wide;
  const int vpg = (cg + p.v - 1) / p.v;
  p.lpg = pow2_at_least(vpg);
  p.gb = 1;
  while (p.gb < groups && p.gb * cg * size < 128 && p.gb * 2 * p.lpg <= 64) p.gb *= 2;
  p.slabs = (groups + p.gb - 1) / p.gb;
  p.full = p.v == wide && cg % p.v == 0 && p.lpg == vpg && groups % p.gb == 0;
  const int lpr = p.lpg * p.gb;
  // the length that a team should hold: known, or twice the mean
  const long long mean = samples ? (rows + samples - 1) / samples : 0;
  long long len = !ragged ? sample_rows : max_rows > 0 && max_rows < rows ? max_rows : rows;
  const long long longest = len;
  if (ragged && len > 2 * mean) len = 2 * mean;
  if (len < 1) len = 1;
  if (len > 1024) len = 1024;
  p.team = lpr * pow2_at_least((len + NR - 1) / NR);
  p.tb = p.team <= 64 ? 0 : p.team <= 256 ? 256 : 1024;
  if (p.tb) p.team = p.tb;
  const long long held = (long long)(p.team / lpr) * NR;
  p.tile = (int)((rows + TILES - 1) / TILES);
  if (p.tile < TILE_MIN) p.tile = TILE_MIN;
  p.limit = 4 * held < 1024 ? 4 * held : held < 1024 ? 1024 : held;
  if (p.limit < p.tile) p.limit = p.tile;
  const int teams = p.tb ? 1 : 256 / p.team;
  long long blocks = (samples + (long long)teams - 1) / teams;
  const long long most = backward ? (BLOCKS_BWD / p.slabs > 1 ? BLOCKS_BWD / p.slabs : 1) : 65536;
  if (blocks > most) blocks = most;
  if (longest > p.limit) p.tiles = (int)((rows + p.tile - 1) / p.tile);
  const long long room = LAUNCH_THREADS / 1024 / p.slabs - p.tiles;
  if (blocks > room && room > 0) blocks = room;
  p.f_blocks = (int)blocks;
  if (!ragged && p.tiles) p.f_blocks = 0;
  if (p.tiles) p.seg_bytes = align256((size_t)p.tiles * 2 * groups * sizeof(double2));
  else p.limit = 1LL << 62;             // (a sample longer than the caller says is taken all the same)
  if (backward) p.part_bytes = (size_t)(p.f_blocks + p.tiles) * 2 * cols * sizeof(float);
  return p;
}

template <class T, class F>
void with_form(const Plan& p, F&& f) {
  constexpr int V = 16 / sizeof(T);
  typedef std::integral_constant<int, V> wide;
  typedef std::integral_constant<int, 1> one;
  if (p.v == 1) f(one(), std::false_type());
  else if (p.full) f(wide(), std::true_type());
  else f(wide(), std::false_type());
}

template <class T>
painn_status run_fwd(painn_ctx* ctx, const Plan& p, const GnArgs& a) {
  const dim3 grid((unsigned)((long long)(p.f_blocks + p.tiles) * p.slabs)), tiles((unsigned)(p.tiles * p.slabs));
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM, true);
  with_form<T>(p, [&](auto v, auto full) {
    constexpr int V = decltype(v)::value;
    constexpr bool FULL = decltype(full)::value;
    if (p.tb == 0) k_group_norm<T, V, FULL, 0><<<grid, 256, 0, ctx->stream>>>(a);
    else if (p.tb == 256) k_group_norm<T, V, FULL, 256><<<grid, 256, 0, ctx->stream>>>(a);
    else k_group_norm<T, V, FULL, 1024><<<grid, 1024, 0, ctx->stream>>>(a);
    if (p.tiles && p.lpg <= 256) k_group_norm_tiles<T, V, FULL, 256><<<tiles, 256, 0, ctx->stream>>>(a);
    else if (p.tiles) k_group_norm_tiles<T, V, FULL, 1024><<<tiles, 1024, 0, ctx->stream>>>(a);
  });
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM, false);
  return launched(ctx, "group norm launch");
}

template <class T>
painn_status run_bwd(painn_ctx* ctx, const Plan& p, const GnArgs& a, void* dgamma, void* dbeta) {
  const dim3 grid((unsigned)((long long)(p.f_blocks + p.tiles) * p.slabs)), tiles((unsigned)(p.tiles * p.slabs));
  const size_t lds = a.part ? (size_t)2 * p.lpg * p.gb * p.v * sizeof(float) : 0;
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM_BWD, true);
  if (a.rows > 0 && a.samples > 0) {
    with_form<T>(p, [&](auto v, auto full) {
      constexpr int V = decltype(v)::value;
      constexpr bool FULL = decltype(full)::value;
      if (p.tb == 0) k_group_norm_bwd<T, V, FULL, 0><<<grid, 256, lds, ctx->stream>>>(a);
      else if (p.tb == 256) k_group_norm_bwd<T, V, FULL, 256><<<grid, 256, lds, ctx->stream>>>(a);
      else k_group_norm_bwd<T, V, FULL, 1024><<<grid, 1024, lds, ctx->stream>>>(a);
      if (p.tiles && a.out && p.lpg <= 256) k_group_norm_bwd_tiles<T, V, FULL, 256><<<tiles, 256, 0, ctx->stream>>>(a);
      else if (p.tiles && a.out) k_group_norm_bwd_tiles<T, V, FULL, 1024><<<tiles, 1024, 0, ctx->stream>>>(a);
    });
  }
  if (dgamma) {
    const int n = a.rows > 0 && a.samples > 0 ? p.f_blocks + p.tiles : 0;
    fold_columns<T>(ctx->stream, n, a.cols, a.part, (T*)dgamma, (T*)dbeta);
  }
  prof_mark(ctx->prof, ctx->stream, KC_GROUP_NORM_BWD, false);
  return launched(ctx, "group norm reverse launch");
}

painn_status shape_check(painn_ctx* ctx, int prec, int64_t rows, int32_t cols, int32_t groups, int32_t samples,
                         const int32_t* offsets, int64_t sample_rows, int64_t max_rows, int act, int reserved) {
  if (reserved) return fail(ctx, PAINN_E_ARG, "reserved is not 0");
  if (prec == PAINN_FP64) return fail(ctx, PAINN_E_UNSUPPORTED, "group norm runs in FP32 and BF16");
  if (prec != PAINN_FP32 && prec != PAINN_BF16) return fail(ctx, PAINN_E_ARG, "unknown precision");
  if (act < PAINN_ACT_NONE || act > PAINN_ACT_GELU) return fail(ctx, PAINN_E_ARG, "unknown activation");
  if (cols < 1 || groups < 1 || cols % groups) return fail(ctx, PAINN_E_ARG, "groups must divide cols");
  if (rows < 0 || samples < 0 || max_rows < 0) return fail(ctx, PAINN_E_ARG, "a count is negative");
  if (cols / groups > GN_COLS) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 4096 columns in a group");
  if (cols > 1 << 24 || rows > 0x7fffffffLL) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 2^24 columns or 2^31 - 1 rows");
  if (!offsets && samples > 0 && (sample_rows < 0 || sample_rows > rows || sample_rows * samples != rows))
    return fail(ctx, PAINN_E_ARG, "without offsets rows must be n_samples times sample_rows");
  return PAINN_OK;
}

void fill(GnArgs& g, const Plan& p, const painn_group_norm_args& a, void* workspace) {
  g.rows = a.rows; g.cols = a.cols; g.groups = a.groups; g.cg = a.cols / a.groups; g.act = a.activation;
  g.offsets = a.offsets; g.sample_rows = a.sample_rows; g.samples = a.n_samples;
  g.x = a.x; g.ldx = a.ldx; g.gamma = a.gamma; g.beta = a.beta;
  g.lpg = p.lpg; g.gb = p.gb; g.slabs = p.slabs; g.team = p.team; g.f_blocks = p.f_blocks; g.limit = p.limit;
  g.tile = p.tile; g.tiles = p.tiles;
  g.seg = (double2*)workspace;
  g.part = (float*)((char*)workspace + p.seg_bytes);
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
  if ((long long)p.slabs * (p.f_blocks + p.tiles) > LAUNCH_THREADS / 1024)
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

painn_status painn_group_norm_backward(painn_ctx* ctx, const painn_group_norm_args* args, const void* dy, int64_t lddy,
                                       void* dx, int64_t lddx, void* dgamma, void* dbeta) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!args) return fail(ctx, PAINN_E_ARG, "null arguments");
  const painn_group_norm_args& a = *args;
  painn_status st = shape_check(ctx, a.precision, a.rows, a.cols, a.groups, a.n_samples, a.offsets, a.sample_rows, a.max_rows,
                                a.activation, a.reserved);
  if (st != PAINN_OK) return st;
  if (!dgamma != !dbeta) return fail(ctx, PAINN_E_ARG, "dgamma and dbeta are formed together");
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
  if ((long long)p.slabs * (p.f_blocks + p.tiles) > LAUNCH_THREADS / 1024)
    return fail(ctx, PAINN_E_UNSUPPORTED, "more blocks than a launch holds");
  const size_t need = some ? p.seg_bytes + (dgamma ? p.part_bytes : 0) : 0;
  if (a.workspace_bytes < (int64_t)need || (need && !a.workspace))
    return fail(ctx, PAINN_E_ARG, "the workspace is too small: " + std::to_string(need) + " bytes");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  GnArgs g{};
  fill(g, p, a, a.workspace);
  g.dy = dy; g.lddy = lddy; g.out = dx; g.ldo = lddx; g.mu = a.mean; g.rs = a.rstd;
  if (!dgamma) g.part = nullptr;
  return a.precision == PAINN_FP32 ? run_bwd<float>(ctx, p, g, dgamma, dbeta) : run_bwd<b16>(ctx, p, g, dgamma, dbeta);
}

}  // extern "C"

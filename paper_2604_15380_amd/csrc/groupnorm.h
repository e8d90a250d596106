// Shared by group norm's two passes: the plan, a thread's place and rows, sums
// over a team, long samples and the activations.
#pragma once

#include <type_traits>

#include "raw.h"

namespace {

using namespace ops;

constexpr int TILE_MIN = 64, TILES = 512;   // rows of a tile at least; tiles at most
constexpr int GN_COLS = 2048;       // columns of a group at most (a block's lanes hold them)
// Waves of the reverse pass, whose blocks' column sums are folded: twice what is
// resident (65,502 x 256 BF16, 1,871 samples: 51 us; with 2,048 56, 8,192 56,
// 15,000, one per sample and slab, 79).
constexpr int WAVES_BWD = 4096;

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
  const float *mu, *rs;             // reverse pass's inputs, with strides by sample and by group
  long long mu_s, mu_g, rs_s, rs_g;
  float eps;
  int lpg, gb, slabs;               // lanes of a group, groups of a slab (powers of 2), slabs
  int lpg_bits, lpr_bits;           // log2 of lpg and of a row's lanes, lpg gb
  int team;                         // threads of a sample's team
  int l_blocks, f_blocks;           // blocks of long and of other samples per slab; the tiles' blocks follow
  long long limit;                  // rows that a team takes on
  int tile, tiles;                  // rows of a tile, tiles (0: no sample is longer than limit)
  double2* seg;                     // [tiles][2][groups]: mean and squares about it; the reverse pass's sums
  float* part;                      // [l_blocks + f_blocks + tiles][2][cols] column sums of the reverse pass, or null
};

// A thread's place: V columns of a group of the slab, and which of the team's
// rows.
template <int V>
struct Place {
  int group, col, left;             // left: columns from col to the group's end, <= 0 for an idle lane
  int row, rows;                    // the thread's row of the team's
  __device__ __forceinline__ Place(const GnArgs& a, int slab, int t, int team) {
    const int l = t & (a.lpg - 1), q = (t >> a.lpg_bits) & (a.gb - 1);
    group = slab * a.gb + q;
    left = group < a.groups ? a.cg - l * V : 0;
    col = left > 0 ? group * a.cg + l * V : 0;
    row = t >> a.lpr_bits;
    rows = team >> a.lpr_bits;
  }
};

// x plus its value in the lane whose number differs in bit o (uniform).
__device__ __forceinline__ float lane_add(float x, int o) {
  const int u = __float_as_int(x);
  int v;
  if (o == 1) v = __builtin_amdgcn_update_dpp(0, u, 0xb1, 0xf, 0xf, true);         // quad_perm 1, 0, 3, 2
  else if (o == 2) v = __builtin_amdgcn_update_dpp(0, u, 0x4e, 0xf, 0xf, true);    // quad_perm 2, 3, 0, 1
  else if (o == 4) v = __builtin_amdgcn_ds_swizzle(u, 0x101f);                     // xor 4 within 32 lanes
  else if (o == 8) v = __builtin_amdgcn_update_dpp(0, u, 0x128, 0xf, 0xf, true);   // a row of 16 turned by 8
  else if (o == 16) v = __builtin_amdgcn_ds_swizzle(u, 0x401f);                    // xor 16 within 32 lanes
  else v = __shfl_xor(u, 32);
  return x + __int_as_float(v);
}
__device__ __forceinline__ double lane_add(double x, int o) { return x + __shfl_xor(x, o); }

// N sums over a group's lanes and the team's rows, in every thread of them.
// TB = 64: teams within a wave; else the block is the team, with lds
// [N][TB / 64][64] of them.
template <int TB, int N, class S>
__device__ __forceinline__ void team_sum(const GnArgs& a, S* s, int team, S* lds) {
  const int lpr = a.lpg * a.gb, in_wave = TB > 64 ? 64 : team;
  for (int o = 1; o < a.lpg && o < in_wave; o <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = lane_add(s[k], o);
  for (int o = lpr; o < in_wave; o <<= 1)
#pragma unroll
    for (int k = 0; k < N; ++k) s[k] = lane_add(s[k], o);
  if constexpr (TB > 64) {
    const int lane = threadIdx.x & 63, q = (threadIdx.x >> a.lpg_bits) & (a.gb - 1);
    __syncthreads();
    if (lane < lpr && (lane & (a.lpg - 1)) == 0)
#pragma unroll
      for (int k = 0; k < N; ++k) lds[k * TB + (threadIdx.x >> 6) * 64 + q] = s[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
      s[k] = 0;
#pragma unroll
      for (int w = 0; w < TB / 64; ++w) s[k] += lds[k * TB + w * 64 + q];
    }
  }
}
template <int TB>
__device__ __forceinline__ bool team_any(bool x) {
  if constexpr (TB > 64) return __syncthreads_or(x);
  else return __any(x);
}

// Row steps that a team of TB threads (0: within a wave) holds in registers.
constexpr int steps_held(int tb) { return tb == 512 ? 16 : 8; }
constexpr int steps_held_bwd(int tb) { return 8; }   // (beside dy and dz)

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
    const uint32_t s = (uint32_t)row / (uint32_t)a.sample_rows;
    return s < (uint32_t)a.samples ? (int)s : -1;
  }
  const int lane = threadIdx.x & 63;
  int lo = 0, n = a.samples;        // among [lo, lo + n)
  while (n > 1) {
    const int step = (n - 1) / 64 + 1, s = lane * step;     // (n may be 2^31 - 1)
    const bool before = s < n && bound(a, lo + s) <= row;
    const int k = __popcll(__ballot(before));
    const int at = k > 0 ? (k - 1) * step : 0;
    n = n - at < step ? n - at : step;
    lo += at;
  }
  const Span p = span(a, lo);
  return row >= p.a && row < p.b ? lo : -1;
}

// A thread's rows of a matrix: row p.row + i p.rows of n, for i = 0, 1, ...
template <class T, int V, bool FULL>
struct Rows {
  const T* at;
  long long step;
  int left, row, rows, n;
  __device__ __forceinline__ Rows(const void* x, long long ld, const Place<V>& p, long long first, long long count) {
    at = (const T*)x + (first + p.row) * ld + p.col;
    step = p.rows * ld;
    left = p.left;
    row = p.row;
    rows = p.rows;
    n = (int)count;
  }
  // (unsigned: row + i rows may pass 2^31 where a sample ends just below it)
  __device__ __forceinline__ bool has(int i) const {
    return (FULL || left > 0) && (uint32_t)row + (uint32_t)i * (uint32_t)rows < (uint32_t)n;
  }
  __device__ __forceinline__ Raw<T, V> get(int i) const {
    if (has(i)) return load_raw<T, V, FULL>(at + i * step, left);
    return zero_raw<T, V>();
  }
  __device__ __forceinline__ void put(int i, const float* o) const {
    T* y = const_cast<T*>(at) + i * step;
    if constexpr (FULL) store<V>(y, o);
    else store_n<V>(y, left, o);
  }
};

// The normal distribution's Phi(z), and exp(-z^2 / 2).  Half of erfc(|z| / sqrt 2)
// as exp(-z^2 / 2) t P(t), t = 1 / (1 + 0.28 |z|), the form of Abramowitz and
// Stegun 7.1.26 with P of degree 8, 1.7e-7 of itself off at most.  In FP32 Phi is
// off by 4.4 x 2^-24 at most, and by 6.5 with the hardware's reciprocal and
// exponential a step off each (12 M arguments within 13, on the CPU); far below 0 the
// exponent's rounding leaves z^2 / 2 x 2^-24 of Phi itself.  About half of the
// instructions that erff takes (147,456 x 256 FP32 with GELU: 30 M vector
// instructions with it).
__device__ __forceinline__ float normal_cdf(float z, float& e) {
  const float u = fabsf(z), t = __builtin_amdgcn_rcpf(__builtin_fmaf(u, 0.28f, 1.f));
  float p = 0.02516147866845131f;
  p = __builtin_fmaf(p, t, -0.09536159783601761f);
  p = __builtin_fmaf(p, t, 0.09532923251390457f);
  p = __builtin_fmaf(p, t, -0.008962316438555717f);
  p = __builtin_fmaf(p, t, 0.07401145249605179f);
  p = __builtin_fmaf(p, t, 0.08328507840633392f);
  p = __builtin_fmaf(p, t, 0.10313647240400314f);
  p = __builtin_fmaf(p, t, 0.11169621348381042f);
  p = __builtin_fmaf(p, t, 0.11170393228530884f);
  e = fast_exp(z * z * -0.5f);
  const float h = p * t * e;
  return z < 0.f ? h : 1.f - h;
}
// The kernels come by activation (none and ReLU, SiLU, GELU), so that a kernel's
// code, 46 KB in the reverse pass of BF16 with SiLU, stays within the instruction
// cache's 64 KB.
enum { ACT_RELU, ACT_SILU, ACT_GELU };

template <int ACT, int N>
__device__ __forceinline__ void activate(float* z, bool relu) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (ACT == ACT_RELU) {
      z[i] = relu && z[i] < 0.f ? 0.f : z[i];
    } else if constexpr (ACT == ACT_SILU) {
      z[i] *= sigmoid(z[i]);
    } else {
      float e;
      z[i] *= normal_cdf(z[i], e);
    }
  }
}
// x *= activation'(z)
template <int ACT, int N>
__device__ __forceinline__ void times_slope(float* x, const float* z, bool relu) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if constexpr (ACT == ACT_RELU) {
      x[i] *= !relu || z[i] > 0.f ? 1.f : 0.f;
    } else if constexpr (ACT == ACT_SILU) {
      const float s = sigmoid(z[i]);
      x[i] *= s * (1.f + z[i] * (1.f - s));
    } else {
      float e;
      const float phi = normal_cdf(z[i], e);
      x[i] *= phi + z[i] * (e * 0.39894228040143268f);
    }
  }
}

template <int V>
__device__ __forceinline__ float tree(const float* x) {
  if constexpr (V == 1) return x[0];
  else return tree<V / 2>(x) + tree<V / 2>(x + V / 2);
}
// Calls f(sample, its rows) for the samples of block blk of `blocks` that have
// `least` rows at least and no more than the limit: every lane looks at one.
template <class F>
__device__ __forceinline__ void longer_samples(const GnArgs& a, int blk, int blocks, long long least, F&& f) {
  for (long long s0 = blk; s0 < a.samples; s0 += 64LL * blocks) {
    const long long s = s0 + (long long)(threadIdx.x & 63) * blocks;
    Span q{0, -1};
    if (s < a.samples) q = span(a, (int)s);
    const bool yes = s < a.samples && q.b - q.a >= least && q.b - q.a <= a.limit;
    for (unsigned long long m = __ballot(yes); m; m &= m - 1) {
      const int lane = __ffsll(m) - 1;
      f((int)(s0 + (long long)lane * blocks),
        Span{__builtin_amdgcn_readlane((int)q.a, lane), __builtin_amdgcn_readlane((int)q.b, lane)});
    }
  }
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

// Calls f(sums, rows) for a long sample's tiles that fall to this one of `lanes`
// lanes, in an order that depends on the sample alone.
template <class F>
__device__ __forceinline__ void each_tile(const GnArgs& a, const Span& p, int group, int lane, int lanes, F&& f) {
  if (group >= a.groups) return;
  const int from = (int)((uint32_t)p.a / (uint32_t)a.tile), to = (int)((uint32_t)(p.b - 1) / (uint32_t)a.tile);
  for (int u = from + lane; u <= to; u += lanes) {
    const long long lo = (long long)u * a.tile, hi = lo + a.tile;
    const int slot = u == from && p.a != lo;
    f(a.seg[((size_t)u * 2 + slot) * a.groups + group], (hi < p.b ? hi : p.b) - (lo > p.a ? lo : p.a));
  }
}
__device__ __forceinline__ void tiles_sum(const GnArgs& a, const Span& p, int group, int lane, int lanes, double* s) {
  s[0] = s[1] = 0.0;
  each_tile(a, p, group, lane, lanes, [&](double2 v, long long) {
    s[0] += v.x;
    s[1] += v.y;
  });
}

// ---- the plan -----------------------------------------------------------------------
inline int pow2_at_least(long long x) {
  int p = 1;
  while (p < x) p <<= 1;
  return p;
}

inline int log2_of(int p) {
  int n = 0;
  while (1 << n < p) ++n;
  return n;
}

struct Plan {
  int v, lpg, gb, slabs, team, tb, l_blocks, f_blocks, tile, tiles;
  bool full;
  long long limit;
  size_t seg_bytes, part_bytes;
};

// max_rows: the longest sample where the caller knows it, else 0.
inline Plan plan_of(bool bf16, long long rows, int cols, int groups, int samples, bool ragged, long long sample_rows,
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
  // the length that a team holds: known, or the mean
  const long long mean = samples ? (rows + samples - 1) / samples : 0;
  const long long longest = !ragged ? sample_rows : max_rows > 0 && max_rows < rows ? max_rows : rows;
  long long len = longest < mean ? longest : mean;
  if (len < 1) len = 1;
  if (len > 1024) len = 256 / lpr * 8;  // (the tiles do those)
  p.team = lpr * pow2_at_least((len + 7) / 8);
  p.tb = p.team <= 64 ? 64 : p.team <= 256 ? 256 : 512;
  if (p.tb > 64) p.team = p.tb;
  const long long held = (long long)(p.tb / lpr) * (backward ? steps_held_bwd(p.tb) : steps_held(p.tb));
  p.tile = (int)((rows + TILES - 1) / TILES);
  if (p.tile < TILE_MIN) p.tile = TILE_MIN;
  p.limit = 4 * held < 1024 ? 4 * held : held < 1024 ? 1024 : held;      // of a block
  if (p.limit < p.tile) p.limit = p.tile;
  if (longest > p.limit) p.tiles = (int)((rows + p.tile - 1) / p.tile);
  const int teams = p.tb / p.team;
  long long room = LAUNCH_THREADS / 1024 / p.slabs - p.tiles;
  if (room > 65535 - p.tiles) room = 65535 - p.tiles;             // (the grid's second axis)
  const long long most_bwd = WAVES_BWD / (p.tb / 64) / p.slabs;
  if (backward && room > most_bwd) room = most_bwd > 8 ? most_bwd : 8;
  if (room < 2) room = 2;                                         // (refused: more blocks than a launch holds)
  if (p.tb == 64 && ragged) {
    // blocks for the samples that a team cannot hold, most of them without one: 16 per
    // CU (65,502 x 256 BF16, 1,871 samples: 27.0 us; one per sample 28.7, 8 per CU
    // 28.5); the reverse pass's half; a few where the caller says that there are none
    room = (room + 1) / 2;
    long long most = backward ? room : 4096 / p.slabs;
    if (most < 8 || longest <= p.team / lpr * 8) most = 8;
    if (most > room) most = room;
    p.l_blocks = (int)(samples < most ? samples : most);
  }
  const long long blocks = (samples + (long long)teams - 1) / teams;
  p.f_blocks = (int)(blocks < room ? blocks : room);
  if (!ragged && p.tiles) p.l_blocks = p.f_blocks = 0;
  if (p.tiles) p.seg_bytes = align256((size_t)p.tiles * 2 * groups * sizeof(double2));
  else p.limit = 1LL << 62;             // (a sample longer than the caller says is taken all the same)
  if (backward) p.part_bytes = (size_t)(p.l_blocks + p.f_blocks + p.tiles) * 2 * cols * sizeof(float);
  return p;
}

template <class T, int ACT, class F>
void with_columns(const Plan& p, F&& f) {
  constexpr int V = 16 / sizeof(T);
  typedef std::integral_constant<int, V> wide;
  typedef std::integral_constant<int, 1> one;
  typedef std::integral_constant<int, ACT> act;
  if (p.v == 1) f(one(), std::false_type(), act());
  else if (p.full) f(wide(), std::true_type(), act());
  else f(wide(), std::false_type(), act());
}
// Calls f(V, FULL, ACT) for the plan's columns and the activation.
template <class T, class F>
void with_form(const Plan& p, int act, F&& f) {
  if (act == PAINN_ACT_SILU) with_columns<T, ACT_SILU>(p, f);
  else if (act == PAINN_ACT_GELU) with_columns<T, ACT_GELU>(p, f);
  else with_columns<T, ACT_RELU>(p, f);
}

inline painn_status shape_check(painn_ctx* ctx, int prec, int64_t rows, int32_t cols, int32_t groups, int32_t samples,
                         const int32_t* offsets, int64_t sample_rows, int64_t max_rows, int act, int reserved) {
  if (reserved) return fail(ctx, PAINN_E_ARG, "reserved is not 0");
  if (prec == PAINN_FP64) return fail(ctx, PAINN_E_UNSUPPORTED, "group norm runs in FP32 and BF16");
  if (prec != PAINN_FP32 && prec != PAINN_BF16) return fail(ctx, PAINN_E_ARG, "unknown precision");
  if (act < PAINN_ACT_NONE || act > PAINN_ACT_GELU) return fail(ctx, PAINN_E_ARG, "unknown activation");
  if (cols < 1 || groups < 1 || cols % groups) return fail(ctx, PAINN_E_ARG, "groups must divide cols");
  if (rows < 0 || samples < 0 || max_rows < 0) return fail(ctx, PAINN_E_ARG, "a count is negative");
  if (cols / groups > GN_COLS) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 2048 columns in a group");
  if (cols > 1 << 24 || rows > 0x7fffffffLL) return fail(ctx, PAINN_E_UNSUPPORTED, "more than 2^24 columns or 2^31 - 1 rows");
  if (!offsets && samples > 0 && (sample_rows < 0 || sample_rows > rows || sample_rows * samples != rows))
    return fail(ctx, PAINN_E_ARG, "without offsets rows must be n_samples times sample_rows");
  return PAINN_OK;
}

inline void fill(GnArgs& g, const Plan& p, const painn_group_norm_args& a, void* workspace) {
  g.rows = a.rows; g.cols = a.cols; g.groups = a.groups; g.cg = a.cols / a.groups; g.act = a.activation;
  g.offsets = a.offsets; g.sample_rows = a.sample_rows; g.samples = a.n_samples;
  g.x = a.x; g.ldx = a.ldx; g.gamma = a.gamma; g.beta = a.beta;
  g.lpg = p.lpg; g.gb = p.gb; g.lpg_bits = log2_of(p.lpg); g.lpr_bits = log2_of(p.lpg * p.gb); g.slabs = p.slabs; g.team = p.team; g.l_blocks = p.l_blocks; g.f_blocks = p.f_blocks; g.limit = p.limit;
  g.tile = p.tile; g.tiles = p.tiles;
  g.seg = (double2*)workspace;
  g.part = (float*)((char*)workspace + p.seg_bytes);
}

}  // namespace

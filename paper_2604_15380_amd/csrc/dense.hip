// Dense layers with bias, activation and residual in the epilogue, one weight
// matrix for all rows or one per group of consecutive rows, and their reverse
// pass (FP32, BF16).
//
// All three products are one tile kernel, D[m][n] = sum_k A[m][k] B[n][k]:
//   forward  A = x, B = w;   dx  A = dz, B = w^T;   dw  A = dz^T, B = x^T.
// A block stages k-blocks of both operands in LDS, its waves feed 16x16x32
// matrix instructions from there.  The weights are the instruction's first
// operand, so that a lane ends up with four neighbouring columns of one row;
// the results pass through LDS once more, so that bias, activation, residual
// and all stores work on whole pieces of rows.  BF16 operands whose rows start
// at 16-byte words go from memory straight to LDS (k_dense16); all others and
// FP32 pass through registers (k_dense); a few rows take k_few.
//
// FP32 operands become three BF16 planes on the way into LDS (split3, mfma.h)
// and six of the nine plane products are formed: 96 matrix-core cycles per
// 16x16x32 against 256 of the FP32 instruction, no further from 64 bits than a
// plain FP32 product (65,502 x 776 x 776: 0.51 ms, a library's FP32 product
// 0.72 ms).
//
// What bounds it: with BF16 the bytes.  65,536 x 1,024 -> 1,024 takes 133 us, 1.03
// PFLOP/s (a library's product without epilogue 104); the loads alone take
// 121, the products alone 103.  At 776 columns a row's 128-byte piece lies in
// two cache lines, which is most of 65,502 x 776 x 776's 113 us (with rows of
// 832 columns 99).  FP32: the vector instructions that split the planes, 6.6
// per value, beside 96 matrix instructions per wave and k-block; at 65,502 x
// 776 x 776 the former take 0.50 of the SIMDs' time, the latter 0.46.
//
// Rows of a ragged batch are tiled per group: a block finds its tile by a scan
// over the groups' row counts, one group per lane, so that no launch or
// readback plans the tiles.  dw contracts over the rows: the batch is cut into
// chunks of equal length wherever the groups end, a block goes through its
// chunk's groups one after the other, and where a group lies in several chunks
// k_fold adds their FP32 parts in order.
#include "mfma.h"
#include "ops.h"

namespace {

using namespace ops;

typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2_t __attribute__((ext_vector_type(2)));

// ---- groups ---------------------------------------------------------------------
struct Groups {
  int n;                        // 0: one group of all rows
  const int32_t* offsets;
  long long rows;
};
struct Span {
  int g;                        // group, -1: none
  int index;                    // tile within the group
  long long lo, hi;             // rows of the group
};

// Rows [lo, hi) of group g, within [0, rows] whatever the offsets are.
__device__ __forceinline__ void group_rows(const Groups& gr, int g, long long& lo, long long& hi) {
  lo = gr.offsets[g];
  hi = gr.offsets[g + 1];
  lo = lo < 0 ? 0 : lo > gr.rows ? gr.rows : lo;
  hi = hi < lo ? lo : hi > gr.rows ? gr.rows : hi;
}

// Tile t of all groups' tiles of `len` rows.  Every wave of the block finds the
// same.
__device__ __forceinline__ Span find_tile(const Groups& gr, int t, int len) {
  Span s{-1, 0, 0, 0};
  if (gr.n == 0) {
    if ((long long)t * len < gr.rows) s = Span{0, t, 0, gr.rows};
    return s;
  }
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int g0 = 0; g0 < gr.n; g0 += 64) {
    long long lo = 0, hi = 0;
    int tiles = 0;
    if (g0 + lane < gr.n) {
      group_rows(gr, g0 + lane, lo, hi);
      tiles = (int)((hi - lo + len - 1) / len);
    }
    int end = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(end, o);
      if (lane >= o) end += x;
    }
    end += before;
    const unsigned long long past = __ballot(t < end);
    if (past) {
      const int l = __ffsll((long long)past) - 1;
      s.index = t - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(tiles, l));
      s.lo = __builtin_amdgcn_readlane((int)lo, l);
      s.hi = __builtin_amdgcn_readlane((int)hi, l);
      // (offsets that decrease may count more tiles than there are)
      if (s.index >= 0 && s.lo + (long long)s.index * len < s.hi) s.g = g0 + l;
      return s;
    }
    before = __builtin_amdgcn_readlane(end, 63);
  }
  return s;
}

// dw: the rows of the batch are cut into chunks of equal length, wherever the
// groups end, so that every block has the same work; a block goes through the
// groups that its chunk meets.  The chunks that hold rows of [lo, hi); a group
// without rows belongs to the chunk that it lies in.
__device__ __forceinline__ void chunks_of(const Groups& gr, int chunk, int chunks, long long lo, long long hi,
                                          int& first, int& last) {
  first = (int)(lo / chunk < chunks ? lo / chunk : chunks - 1);
  last = hi > lo ? (int)((hi - 1) / chunk) : first;
}

// ---- operands -------------------------------------------------------------------
template <class T> struct Mma;
template <> struct Mma<b16> {
  static constexpr int NP = 1, BK = 64;
};
template <> struct Mma<float> {
  static constexpr int NP = 3, BK = 32;
};
// The plane products of FP32, smallest first: lo hi, mid mid, hi lo, mid hi,
// hi mid, hi hi.
constexpr int PLANE_A[6] = {2, 1, 0, 1, 0, 0}, PLANE_B[6] = {0, 1, 2, 0, 1, 0};

// An LDS tile is [row][BK] per plane, its 16-byte chunks permuted within the
// row so that the 16 rows of a fragment, and the rows a transposing store
// writes together, fall into different banks.
template <int BK>
__device__ __forceinline__ int lds_at(int row, int c) {
  const int s = BK == 64 ? (row ^ (row >> 3)) & 7 : ((row >> 1) ^ (row >> 3)) & 3;
  return row * BK + ((c ^ s) << 3);
}

// What one thread carries of a k-block of an operand: R rows x BK.
// Plain: the operand is [row][k]; units of 8 k.
// TR: it is [k][row]; units of 4 k x 8 rows (BF16) or 4 k x 4 rows (FP32).
template <class T, int R, int TH, bool TR>
struct Stage {
  static constexpr int BK = Mma<T>::BK, CH = BK / 8;
  static constexpr bool B = sizeof(T) == 2;
  static constexpr int RU = B ? 8 : 4;                                 // rows of a transposed unit
  static constexpr int UNITS = TR ? R * BK / (4 * RU) : R * BK / 8;
  static constexpr int U = (UNITS + TH - 1) / TH;
  static constexpr int W = B && !TR ? 1 : B ? 4 : TR ? 4 : 2;          // 16-byte words of a unit
  u4_t w[U][W];

  __device__ __forceinline__ static u4_t word(const T* p) {
    u4_t v;
    __builtin_memcpy(&v, p, 16);
    return v;
  }
  // the first n elements of a 16-byte word
  __device__ __forceinline__ static u4_t word_n(const T* p, long long n) {
    constexpr int E = 16 / sizeof(T);
    u4_t v = {0, 0, 0, 0};
    if (n >= E) return word(p);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (e < n) {
        if constexpr (B) {
          uint16_t h;
          __builtin_memcpy(&h, p + e, 2);
          v[e / 2] |= (uint32_t)h << (16 * (e & 1));
        } else {
          uint32_t x;
          __builtin_memcpy(&x, p + e, 4);
          v[e] = x;
        }
      }
    return v;
  }

  // k-block [k0, k0 + BK) of rows [r0, r0 + R); rows < n_rows, k < n_k exist
  // (n_rows, n_k >= 1).  What lies past n_k is zero; rows past n_rows hold
  // anything.
  __device__ __forceinline__ void load(const T* base, long long ld, long long r0, long long n_rows, long long k0,
                                       long long n_k) {
    const int tid = threadIdx.x;
    const bool full = k0 + BK <= n_k && (!TR || r0 + R <= n_rows);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = i * TH + tid;
      if (UNITS % TH != 0 && u >= UNITS) break;
      if constexpr (!TR) {
        long long r = r0 + u / CH;
        r = r < n_rows ? r : n_rows - 1;
        const long long k = k0 + (u % CH) * 8;
        const T* p = base + r * ld + k;
        if (full) {
#pragma unroll
          for (int j = 0; j < W; ++j) w[i][j] = word(p + j * (16 / sizeof(T)));
        } else {
#pragma unroll
          for (int j = 0; j < W; ++j) w[i][j] = word_n(p + j * (16 / sizeof(T)), n_k - k - j * (int)(16 / sizeof(T)));
        }
      } else {
        const long long r = r0 + (u % (R / RU)) * RU;
        const long long k = k0 + (u / (R / RU)) * 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const T* p = base + (k + j) * ld + r;
          if (full) w[i][j] = word(p);
          else w[i][j] = k + j < n_k ? word_n(p, n_rows - r) : u4_t{0, 0, 0, 0};
        }
      }
    }
  }

  // FP32: four k of one row as planes, 5.5 instructions per value plus one that
  // notices what they do not hold: where x - hi is not finite (x an infinity or
  // NaN, or so large that hi rounded to infinity) `bad` becomes NaN.
  __device__ __forceinline__ static void put4(uint16_t* lds, int at, const float* x, float& bad) {
    typedef float f2_t __attribute__((ext_vector_type(2)));
    typedef b16 b2_t __attribute__((ext_vector_type(2)));
    uint32_t p[3][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float a = x[2 * h], b = x[2 * h + 1];
#pragma unroll
      for (int q = 0; q < 3; ++q) {
        p[q][h] = __builtin_bit_cast(uint32_t, __builtin_convertvector(f2_t{a, b}, b2_t));
        if (q == 2) break;
        a -= __uint_as_float(p[q][h] << 16);
        b -= __uint_as_float(p[q][h] & 0xffff0000u);
        if (q == 0) bad = __builtin_fmaf(b, 0.f, __builtin_fmaf(a, 0.f, bad));
      }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) *(u2_t*)(lds + (size_t)q * R * BK + at) = u2_t{p[q][0], p[q][1]};
  }
  // The same for any value (split3).
  __device__ static void put4_any(uint16_t* lds, int at, const float* x) {
    uint32_t p[4][3];
#pragma unroll
    for (int i = 0; i < 4; ++i) split3(x[i], p[i]);
#pragma unroll
    for (int q = 0; q < 3; ++q)
      *(u2_t*)(lds + (size_t)q * R * BK + at) = u2_t{(p[0][q] >> 16) | p[1][q], (p[2][q] >> 16) | p[3][q]};
  }

  __device__ __forceinline__ void put(uint16_t* lds) const {
#pragma unroll
    for (int i = 0; i < U; ++i) put(lds, i);
  }
  __device__ __forceinline__ void put(uint16_t* lds, int i) const {
    const int u = i * TH + threadIdx.x;
    if (UNITS % TH == 0 || u < UNITS) {
      if constexpr (!TR) {
        const int at = lds_at<BK>(u / CH, u % CH);
        if constexpr (B) {
          *(u4_t*)(lds + at) = w[i][0];
        } else {
          float x[8], bad = 0.f;
          __builtin_memcpy(x, w[i], 32);
          put4(lds, at, x, bad);
          put4(lds, at + 4, x + 4, bad);
          if (bad != bad) {
            put4_any(lds, at, x);
            put4_any(lds, at + 4, x + 4);
          }
        }
      } else {
        const int r = (u % (R / RU)) * RU, kg = u / (R / RU);
        if constexpr (B) {
#pragma unroll
          for (int e = 0; e < RU; ++e) {
            uint32_t x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = w[i][j][e >> 1];
            const uint32_t sel = e & 1 ? 0x07060302u : 0x05040100u;     // the upper or lower halves of a pair
            *(u2_t*)(lds + lds_at<BK>(r + e, kg >> 1) + 4 * (kg & 1)) =
                u2_t{__builtin_amdgcn_perm(x[1], x[0], sel), __builtin_amdgcn_perm(x[3], x[2], sel)};
          }
        } else {
          float x[4][4], bad = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[e][j] = __uint_as_float(w[i][j][e]);
            put4(lds, lds_at<BK>(r + e, kg >> 1) + 4 * (kg & 1), x[e], bad);
          }
          if (bad != bad) {
#pragma unroll
            for (int e = 0; e < 4; ++e) put4_any(lds, lds_at<BK>(r + e, kg >> 1) + 4 * (kg & 1), x[e]);
          }
        }
      }
    }
  }
};

// ---- the tile kernel --------------------------------------------------------------
enum { FWD = 0, DX = 1, DW = 2 };

struct Args {
  Groups gr;
  int d_in, d_out;
  const void* a;  long long lda;     // x (FWD), dz (DX, DW)
  const void* b;  long long ldb;     // w [g][d_out][d_in] (FWD, DX), x (DW)
  const void* bias;
  int act;                           // FWD: of z; DX: of xz
  const void* e;  long long lde;     // FWD: residual, DX: xz
  void* out;      long long ldo;     // y, dx, dw
  void* z;        long long ldz;     // FWD
  void* db;                          // DW
  float* part;                       // DW: [chunk + group][d_out][d_in] of groups in several chunks
  float* part_b;                     // DW: [chunk + group][d_out]
  int chunk;                         // DW: rows of a chunk
  int tiles;                         // FWD, DX: row tiles (an upper bound); DW: chunks (at least 1)
  int nt;                            // column tiles of a row tile; DW: tiles of dw
  int nt_in;                         // DW: tiles along d_in
  long long rest;                    // DX, DW in tiles of 64 x 64: from dz to its remainders, 0: none
  bool past, past_z;                 // whether out and z are stored past the caches
};

// A block's tile: rows [m0, m_end) of A from a, rows [n0, n_end) of B from b, nk
// values of k.
template <class T>
struct Tile {
  const T *a, *b;
  long long m0, m_end, n0, n_end, nk;
  int g;                      // group
  int slot;                   // DW: where its part goes, -1: the group is whole
};

// Calls `work` for the block's tile, or for each of its chunk's groups (DW).
template <class T, int BM, int BN, int MODE, class Work>
__device__ __forceinline__ void each_tile(const Args& g, Work&& work) {
  // Many row tiles: the column tiles of one on one XCD, next to each other, so
  // that its rows are read from that L2.  Few: all tiles over all XCDs.  (DW:
  // the tiles of one chunk, whose rows are most of what the pass reads.)
  const bool many = MODE == DW ? g.tiles % 8 == 0 : g.tiles >= 64;
  const int lin = many ? blockIdx.x >> 3 : blockIdx.x;
  const int c = lin % g.nt;
  const int t = many ? (lin / g.nt) * 8 + (blockIdx.x & 7) : lin / g.nt;
  if (t >= g.tiles) return;
  Tile<T> w;
  if constexpr (MODE == DW) {
    const int lane = threadIdx.x & 63, groups = g.gr.n ? g.gr.n : 1;
    const long long begin = (long long)t * g.chunk, end = begin + g.chunk;
    w.m0 = (long long)(c / g.nt_in) * BM;
    w.n0 = (long long)(c % g.nt_in) * BN;
    w.m_end = g.d_out;
    w.n_end = g.d_in;
    for (int g0 = 0; g0 < groups; g0 += 64) {
      long long lo = 0, hi = g.gr.rows;
      int first = 0, last = -1;
      if (g0 + lane < groups) {
        if (g.gr.n) group_rows(g.gr, g0 + lane, lo, hi);
        chunks_of(g.gr, g.chunk, g.tiles, lo, hi, first, last);
      }
      for (unsigned long long todo = __ballot(first <= t && t <= last); todo; todo &= todo - 1) {
        const int l = __ffsll((long long)todo) - 1;
        const bool whole = __builtin_amdgcn_readlane(first, l) == __builtin_amdgcn_readlane(last, l);
        long long r0 = begin, r1 = end < g.gr.rows ? end : g.gr.rows;
        if (g.gr.n) {
          const long long glo = __builtin_amdgcn_readlane((int)lo, l), ghi = __builtin_amdgcn_readlane((int)hi, l);
          r0 = glo > r0 ? glo : r0;
          r1 = ghi < r1 ? ghi : r1;
        }
        w.g = g0 + l;
        w.slot = whole ? -1 : t + w.g;
        w.nk = r1 > r0 ? r1 - r0 : 0;
        w.a = (const T*)g.a + r0 * g.lda;
        w.b = (const T*)g.b + r0 * g.ldb;
        work(w);
      }
    }
  } else {
    const Span s = find_tile(g.gr, t, BM);
    if (s.g < 0) return;
    w.g = s.g;
    w.slot = -1;
    w.a = (const T*)g.a;
    w.b = (const T*)g.b + (size_t)s.g * g.d_out * g.d_in;
    w.m0 = s.lo + (long long)s.index * BM;
    w.m_end = s.hi;
    w.n0 = (long long)c * BN;
    w.n_end = MODE == FWD ? g.d_out : g.d_in;
    w.nk = MODE == FWD ? g.d_in : g.d_out;
    work(w);
  }
}

// The tile's results.  A lane holds, per fragment, row l % 16 and the columns
// 4 (l / 16) .. + 3; stored like that, a wave would write 32 bytes per row.
// So each wave passes 16 rows at a time through its own piece of LDS and takes
// them back as 8 neighbouring columns per lane: bias, activation, residual and
// all loads and stores work on whole rows of the wave's tile.  wm, wn: the
// wave's corner in the tile; lds: finish_floats per wave, free for use.
template <int FN> constexpr int finish_floats() { return 16 * (FN * 16 + 4); }

template <class T, class O, int FM, int FN, int MODE, bool WORDS = false>
__device__ __forceinline__ void finish(const Args& g, const Tile<T>& w, int wm, int wn, const f4_t (&acc)[FM][FN],
                                       const f4_t* accb, bool sum_b, float* lds) {
  constexpr int WT = FN * 16, PITCH = WT + 4, LPR = WT / 8, RPP = 64 / LPR;     // lanes per row, rows per pass
  const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
  float* my = lds + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * finish_floats<FN>();
  const size_t wsize = (size_t)g.d_out * g.d_in;
  const long long n = w.n0 + wn + (lane % LPR) * 8, left = w.n_end - n;
  const bool whole = MODE != DW || w.slot < 0;
  O* out = (O*)g.out + (MODE == DW ? (size_t)w.g * wsize : 0) + n;
  float* part = MODE == DW && !whole ? g.part + (size_t)w.slot * wsize + n : nullptr;
  const long long ldo = MODE == DW ? g.d_in : g.ldo;
  float bias[8];
  if (MODE == FWD && g.bias) load_n<8>((const T*)g.bias + (size_t)w.g * g.d_out + n, left, bias);
  constexpr int PASSES = (16 + RPP - 1) / RPP;
  // xz in whole words: all of them asked for before the first is used, at
  // addresses within the tile's rows and columns
  constexpr bool EARLY = MODE == DX && WORDS && FM * PASSES <= 12;
  u4_t early[EARLY ? FM : 1][EARLY ? PASSES : 1];
  if constexpr (EARLY)
    if (g.act != PAINN_ACT_NONE) {
      const T* xz = (const T*)g.e + (n < w.n_end ? n : w.n_end - 8);
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int q = 0; q < PASSES; ++q) {
          const long long m = w.m0 + wm + 16 * i + q * RPP + lane / LPR;
          __builtin_memcpy(&early[i][q], xz + (m < w.m_end ? m : w.m_end - 1) * g.lde, 16);
        }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
  for (int i = 0; i < FM; ++i) {
#pragma unroll
    for (int j = 0; j < FN; ++j) *(f4_t*)(my + lr * PITCH + 16 * j + 4 * lq) = acc[i][j];
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int q = 0; q < PASSES; ++q) {
      const int r = q * RPP + lane / LPR;
      const long long m = w.m0 + wm + 16 * i + r;
      if (lane < LPR * RPP && r < 16 && m < w.m_end && left > 0) {
        float v[8];
        const f4_t x = *(const f4_t*)(my + r * PITCH + (lane % LPR) * 8);
        const f4_t y = *(const f4_t*)(my + r * PITCH + (lane % LPR) * 8 + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = x[e];
          v[4 + e] = y[e];
        }
        if constexpr (MODE == DW) {
          if (!whole) {
            store_n<8>(part + m * ldo, left, v);
            continue;
          }
        } else if constexpr (MODE == FWD) {
          if (g.bias) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += bias[e];
          }
          if (g.z) {
            if (g.past_z && left >= 8) store_past<8>((T*)g.z + m * g.ldz + n, v);
            else store_n<8>((T*)g.z + m * g.ldz + n, left, v);
          }
          act<8>(v, g.act);
          if (g.e) {
            float res[8];
            load_n<8>((const T*)g.e + m * g.lde + n, left, res);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += res[e];
          }
        } else if (g.act != PAINN_ACT_NONE) {
          float z[8];
          if constexpr (EARLY) {
            T h[8];
            __builtin_memcpy(h, &early[i][q], 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = (float)h[e];
          } else {
            load_n<8>((const T*)g.e + m * g.lde + n, left, z);
          }
          mul_slope<8>(v, z, g.act);
        }
        if (MODE != DW && g.past && left >= 8) store_past<8>(out + m * ldo, v);
        else store_n<8>(out + m * ldo, left, v);
      }
    }
    __builtin_amdgcn_wave_barrier();
    if constexpr (MODE == DW) {
      const long long m = w.m0 + wm + 16 * i + lr;
      if (sum_b && lq == 0 && m < w.m_end) {
        const float v = accb[i][0];
        if (whole) store<1>((T*)g.db + (size_t)w.g * g.d_out + m, &v);
        else g.part_b[(size_t)w.slot * g.d_out + m] = v;
      }
    }
  }
}

template <class T, int BM, int BN>
constexpr int stage_halfs() { return Mma<T>::NP * (BM + BN) * Mma<T>::BK; }

template <class T, class O, int BM, int BN, int WM, int WN, int MODE>
__device__ __forceinline__ void product(const Args& g, const Tile<T>& w, uint16_t* lds) {
  using M = Mma<T>;
  constexpr int NP = M::NP, BK = M::BK, TH = 64 * WM * WN;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  uint16_t *As = lds, *Bs = lds + NP * BM * BK;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const bool sum_b = MODE == DW && g.db != nullptr && w.n0 == 0 && wn == 0;

  f4_t acc[FM][FN], accb[MODE == DW ? FM : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    if constexpr (MODE == DW) accb[i] = f4_t{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f4_t{0, 0, 0, 0};
  }
  bf8_t ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (b16)1.f;

  Stage<T, BM, TH, MODE == DW> sa;
  Stage<T, BN, TH, MODE != FWD> sb;
  const long long nk = w.nk;
  const T* a = w.a;
  if (nk > 0) {
    sa.load(a, g.lda, w.m0, w.m_end, 0, nk);
    sb.load(w.b, g.ldb, w.n0, w.n_end, 0, nk);
  }
  for (long long k0 = 0; k0 < nk;) {
    k0 += BK;
    if constexpr (MODE != FWD && BM == 64 && sizeof(T) == 2)
      if (k0 >= nk && g.rest && a == w.a) {      // once more, with the remainders
        a += g.rest;
        k0 = 0;
      }
    sa.put(As);
    sb.put(Bs);
    __syncthreads();
    if (k0 < nk) {
      sa.load(a, g.lda, w.m0, w.m_end, k0, nk);
      sb.load(w.b, g.ldb, w.n0, w.n_end, k0, nk);
    }
#pragma unroll
    for (int kk = 0; kk < BK / 32; ++kk) {
      bf8_t fb[FN][NP];
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int p = 0; p < NP; ++p)
          fb[j][p] = *(const bf8_t*)(Bs + p * BN * BK + lds_at<BK>(wn + 16 * j + lr, 4 * kk + lq));
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        bf8_t fa[NP];
#pragma unroll
        for (int p = 0; p < NP; ++p)
          fa[p] = *(const bf8_t*)(As + p * BM * BK + lds_at<BK>(wm + 16 * i + lr, 4 * kk + lq));
        if constexpr (NP == 3 && MODE != DW) {
          // A k-block's six products are summed apart and added once: one
          // rounding of the running sum in place of six.  Error of x w^T at 776
          // columns 4.2e-7 -> 1.1e-7 (a library's FP32 product 4.9e-7; at dx of
          // few rows it has 2.5e-7); 65,502 x 776 -> 776 508 -> 516 us, dx 526 ->
          // 541.  dw's parts per chunk keep its sums short (4,096 rows 2.5e-7,
          // the library 1.2e-6); apart it took 773 -> 815 us, as its
          // registers spill.
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            f4_t part = {0, 0, 0, 0};
#pragma unroll
            for (int q = 0; q < 6; ++q)
              part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][PLANE_B[q]], fa[PLANE_A[q]], part, 0, 0, 0);
            acc[i][j] += part;
            __builtin_amdgcn_sched_barrier(0);       // (else all six of all j at once: 40 registers more)
          }
        } else {
#pragma unroll
          for (int q = 0; q < (NP == 1 ? 1 : 6); ++q)
#pragma unroll
            for (int j = 0; j < FN; ++j)
              acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[j][NP == 1 ? 0 : PLANE_B[q]],
                                                                 fa[NP == 1 ? 0 : PLANE_A[q]], acc[i][j], 0, 0, 0);
        }
        if constexpr (MODE == DW)
          if (sum_b) {
            // the column sums of dz, as a product with ones
#pragma unroll
            for (int p = NP - 1; p >= 0; --p)
              accb[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fa[p], accb[i], 0, 0, 0);
          }
      }
    }
    __syncthreads();
  }
  finish<T, O, FM, FN, MODE>(g, w, wm, wn, acc, accb, sum_b, (float*)lds);
}

template <class T, class O, int BM, int BN, int WM, int WN, int MODE>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_dense(Args g) {
  constexpr int HALFS = stage_halfs<T, BM, BN>();
  static_assert(HALFS * 2 >= WM * WN * finish_floats<BN / WN / 16>() * 4, "room for finish");
  __shared__ __attribute__((aligned(16))) uint16_t lds[HALFS];
  each_tile<T, BM, BN, MODE>(g, [&](const Tile<T>& w) {
    product<T, O, BM, BN, WM, WN, MODE>(g, w, lds);
    if constexpr (MODE == DW) __syncthreads();      // the next group's operands take its place
  });
}

// ---- BF16 operands in 16-byte words -------------------------------------------------
// Where every row of the operands starts at a multiple of 16 bytes and the
// widths are multiples of 8, the k-blocks go from memory to LDS without
// passing registers (16 bytes per lane, the lanes of a wave next to each other
// in LDS), into the buffer that is not being read.  Words past the last k
// come from a word of zeros.  A plain operand lies as [row][64] with its
// 16-byte chunks permuted by the row; a transposed one stays [k][row] with its
// chunks permuted by k and is turned by the transposing LDS reads, 4 k x 16
// rows at a time (lane l asks for k = l / 4 % 4 and rows 4 (l % 4) .. + 3 of
// its 16 lanes' block and receives 4 k of row l % 16).
__device__ const u4_t zero_word = {0, 0, 0, 0};

typedef short s4_t __attribute__((ext_vector_type(4)));

// 16 bytes per lane from p to LDS, the lanes one after the other from byte `at`
// (the same for the wave).  Written as an instruction because the compiler
// would wait for it before any LDS read, the other buffer's too: it knows
// nothing of it, and wait_loads() does the waiting.  (It has no register
// output that could be taken too early.  m0, the LDS base, is an operand, which
// the compiler sets; the instruction needs a cycle after that.)
__device__ __forceinline__ void load_to_lds(const void* p, uint32_t at) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(p), "{m0}"(at) : "memory");
}
__device__ __forceinline__ uint32_t lds_byte(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// All of this wave's loads are done, those to LDS among them.
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0)" : : : "memory"); }

template <int R, int TH, bool TR>
struct Dma {
  static constexpr int BK = 64, CH = BK / 8, C = R / 8, UNITS = R * CH, U = (UNITS + TH - 1) / TH;
  static constexpr int READS = TR ? 2 : 1;      // LDS reads of a fragment
  static_assert(UNITS % 64 == 0, "whole waves of words");
  const b16* base;             // of the next k-block, the same for all lanes
  uint32_t off[U];             // this lane's words in it

  // plain: chunk c of a row lies at c ^ (row % 8), so that 8 rows' words of one
  // chunk lie in different banks
  // transposed: chunk c of k's row lies at (c + 2 (k % 4)) % C; the reverse
  __device__ __forceinline__ static int row_chunk(int at, int k) {
    const int c = at - 2 * (k & 3);
    return c < 0 ? c + C : c;
  }
  // the word's first k in the k-block
  __device__ __forceinline__ static int first_k(int i) {
    const int u = i * TH + threadIdx.x;
    if constexpr (TR) return u / C;
    return ((u % CH) ^ ((u / CH) & 7)) * 8;
  }
  // Rows [r0, r0 + R) of n_rows (at least 1; transposed: a multiple of 8) of a
  // matrix whose row stride is below 2^22.  Rows past n_rows hold others' values.
  __device__ __forceinline__ void init(const b16* m, long long ld, long long r0, long long n_rows) {
    const int most = (int)(n_rows - r0 < R ? n_rows - r0 : R) - (TR ? 8 : 1);
    base = TR ? m + r0 : m + r0 * ld;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int u = i * TH + threadIdx.x, k = first_k(i);
      int r = TR ? row_chunk(u % C, k) * 8 : u / CH;
      r = r < most ? r : most;
      off[i] = TR ? k * (uint32_t)ld + r : r * (uint32_t)ld + k;
    }
  }
  // The next k-block, `left` values of k from its start on, to lds.
  __device__ __forceinline__ void next(uint16_t* lds, long long ld, long long left) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t at = lds_byte(lds) + wave * 1024;
    const bool whole = left >= BK;
#pragma unroll
    for (int i = 0; i < U; ++i) {
      if (UNITS % TH != 0 && i * TH + wave * 64 >= UNITS) break;
      if (whole) load_to_lds(base + off[i], at + i * TH * 16);
      else load_to_lds(first_k(i) < left ? base + off[i] : (const b16*)&zero_word, at + i * TH * 16);
    }
    base += TR ? BK * ld : BK;
  }
  // The fragment of rows [r, r + 16) and 32 k from 32 kk on.
  __device__ __forceinline__ static bf8_t frag(const uint16_t* lds, int r, int kk) {
    const int lane = threadIdx.x & 63, lr = lane & 15, lq = lane >> 4;
    if constexpr (!TR) {
      return *(const bf8_t*)(lds + (r + lr) * BK + (((4 * kk + lq) ^ (lr & 7)) << 3));
    } else {
      const int k = 32 * kk + 8 * lq + (lr >> 2);
      int c = (r >> 3) + ((lr & 3) >> 1) + 2 * (k & 3);
      c = c < C ? c : c - C;
      const uint16_t* a = lds + k * R + c * 8 + 4 * (lr & 1);
      const s4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)a);
      const s4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4_t*)(a + 4 * R));
      typedef short s8_t __attribute__((ext_vector_type(8)));
      const s8_t v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf8_t, v);
    }
  }
};

template <class O, int BM, int BN, int WM, int WN, int MODE>
__device__ __forceinline__ void product16(const Args& g, const Tile<b16>& w, uint16_t* lds) {
  constexpr int TH = 64 * WM * WN, BK = 64, SA = BM * BK, S = SA + BN * BK;
  constexpr int FM = BM / WM / 16, FN = BN / WN / 16;
  using A = Dma<BM, TH, MODE == DW>;
  using B = Dma<BN, TH, MODE != FWD>;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wm = (wave / WN) * (BM / WM), wn = (wave % WN) * (BN / WN);
  const bool sum_b = MODE == DW && g.db != nullptr && w.n0 == 0 && wn == 0;

  f4_t acc[FM][FN], accb[MODE == DW ? FM : 1];
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    if constexpr (MODE == DW) accb[i] = f4_t{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < FN; ++j) acc[i][j] = f4_t{0, 0, 0, 0};
  }
  bf8_t ones;
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (b16)1.f;

  A sa;
  B sb;
  sa.init(w.a, g.lda, w.m0, w.m_end);
  sb.init(w.b, g.ldb, w.n0, w.n_end);
  long long left = w.nk;                // k from the block being read on
  auto fetch = [&](int buf, long long from) {
    sa.next(lds + buf * S, g.lda, from);
    sb.next(lds + buf * S + SA, g.ldb, from);
  };
  if (left > 0) fetch(0, left);
  bool again = MODE != FWD && g.rest != 0;
  for (int cur = 0; left > 0; cur ^= 1) {
    // everybody's words of this block are there, and nobody reads the other buffer
    wait_loads();
    __syncthreads();
    left -= BK;
    if constexpr (MODE != FWD && BM == 64)
      if (left <= 0 && again) {                  // once more, with the remainders
        again = false;
        left = w.nk;
        sa.init(w.a + g.rest, g.lda, w.m0, w.m_end);
        sb.init(w.b, g.ldb, w.n0, w.n_end);
      }
    if (left > 0) fetch(cur ^ 1, left);
    const uint16_t *a = lds + cur * S, *b = a + SA;
    bf8_t fa[2][FM], fb[2][FN];
    auto read = [&](int kk) {
#pragma unroll
      for (int j = 0; j < FN; ++j) fb[kk][j] = B::frag(b, wn + 16 * j, kk);
#pragma unroll
      for (int i = 0; i < FM; ++i) fa[kk][i] = A::frag(a, wm + 16 * i, kk);
    };
    auto multiply = [&](int kk) {
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[kk][j], fa[kk][i], acc[i][j], 0, 0, 0);
      if constexpr (MODE == DW)
        if (sum_b) {
          // the column sums of dz, as a product with ones
#pragma unroll
          for (int i = 0; i < FM; ++i)
            accb[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, fa[kk][i], accb[i], 0, 0, 0);
        }
    };
    // The second half's fragments are read between the first half's products,
    // a read to every few products; left to itself the compiler reads a few
    // and waits for them, over and over.
    constexpr int READS = FM * A::READS + FN * B::READS, PER = FM * FN / READS > 0 ? FM * FN / READS : 1;
    read(0);
    __builtin_amdgcn_sched_barrier(0);
    read(1);
    multiply(0);
#pragma unroll
    for (int q = 0; q < READS; ++q) {
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);       // LDS reads
      __builtin_amdgcn_sched_group_barrier(0x008, PER, 0);     // matrix products
    }
    __builtin_amdgcn_sched_barrier(0);
    multiply(1);
  }
  __syncthreads();
  finish<b16, O, FM, FN, MODE, true>(g, w, wm, wn, acc, accb, sum_b, (float*)lds);
}

template <class O, int BM, int BN, int WM, int WN, int MODE>
__global__ void __launch_bounds__(64 * WM * WN, 2) k_dense16(Args g) {
  constexpr int HALFS = 2 * (BM + BN) * 64;
  static_assert(HALFS * 2 >= WM * WN * finish_floats<BN / WN / 16>() * 4, "room for finish");
  __shared__ __attribute__((aligned(16))) uint16_t lds[HALFS];
  each_tile<b16, BM, BN, MODE>(g, [&](const Tile<b16>& w) {
    product16<O, BM, BN, WM, WN, MODE>(g, w, lds);
    if constexpr (MODE == DW) __syncthreads();      // the next group's operands take its place
  });
}

// ---- few rows ---------------------------------------------------------------------
// The forward of a few rows reads its weights once and little else: a block has
// 16 rows x 16 columns, its four waves share out k and load their fragments
// from memory straight into registers, 8 k-blocks' loads at once (FP32: 4);
// their sums meet in LDS.
template <class T>
struct Words8 {                     // 8 k of one row: 16 or 32 bytes
  T x[8];
  __device__ __forceinline__ void load(const T* p, long long n) {
    if (n >= 8) {
      __builtin_memcpy(x, p, sizeof(x));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[i] = (T)0.f;
        if (i < n) x[i] = p[i];
      }
    }
  }
  __device__ __forceinline__ void planes(bf8_t* f) const {
    if constexpr (sizeof(T) == 2) {
      __builtin_memcpy(f, x, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t p[3];
        split3(x[i], p);
#pragma unroll
        for (int q = 0; q < 3; ++q) f[q][i] = __builtin_bit_cast(b16, (uint16_t)(p[q] >> 16));
      }
    }
  }
};

template <class T, class O>
__global__ void __launch_bounds__(256) k_few(Args g) {
  using M = Mma<T>;
  constexpr int NP = M::NP, AHEAD = sizeof(T) == 2 ? 8 : 4;
  __shared__ f4_t sums[4][64];
  each_tile<T, 16, 16, FWD>(g, [&](const Tile<T>& w) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int lr = lane & 15, lq = lane >> 4;
    const long long m = w.m0 + lr, n = w.n0 + lr;
    const T* pa = w.a + (m < w.m_end ? m : w.m_end - 1) * g.lda;
    const T* pb = w.b + (n < w.n_end ? n : w.n_end - 1) * g.ldb;
    f4_t acc = {0, 0, 0, 0};
    for (long long k0 = 32 * wave; k0 < w.nk; k0 += 128 * AHEAD) {
      Words8<T> a[AHEAD], b[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        const long long k = k0 + 128 * i + 8 * lq;
        a[i].load(pa + k, w.nk - k);
        b[i].load(pb + k, w.nk - k);
      }
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        bf8_t fa[NP], fb[NP];
        a[i].planes(fa);
        b[i].planes(fb);
        if constexpr (NP == 1) {
          acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[0], fa[0], acc, 0, 0, 0);
        } else {
          f4_t part = {0, 0, 0, 0};
#pragma unroll
          for (int q = 0; q < 6; ++q)
            part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fb[PLANE_B[q]], fa[PLANE_A[q]], part, 0, 0, 0);
          acc += part;
        }
      }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    const long long c = w.n0 + 4 * lq, left = w.n_end - c;
    if (wave == 0 && m < w.m_end && left > 0) {
      float v[4], e[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = (acc[r] + sums[1][lane][r]) + (sums[2][lane][r] + sums[3][lane][r]);
      if (g.bias) {
        load_n<4>((const T*)g.bias + (size_t)w.g * g.d_out + c, left, e);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += e[r];
      }
      if (g.z) store_n<4>((T*)g.z + m * g.ldz + c, left, v);
      act<4>(v, g.act);
      if (g.e) {
        load_n<4>((const T*)g.e + m * g.lde + c, left, e);
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] += e[r];
      }
      store_n<4>((O*)g.out + m * g.ldo + c, left, v);
    }
  });
}

// dz = dy activation'(z), rows of whole 128-byte lines, what its rounding to BF16
// leaves of it where g.rest asks, and dbias from the values before they are
// rounded.  A block has cl x 256 / cl threads, V columns each;
// chunks of rows and parts of dbias as for dw.
struct DzArgs {
  Groups gr;
  int d_out, cl;
  int chunk, tiles;
  const void* dy;  long long lddy;
  const void* z;   long long ldz;
  void* dz;        long long lddz;
  long long rest;                    // from dz to its remainders, 0: none
  void* db;                          // may be null
  float* part_b;                     // [chunk + group][d_out]
};

// What is left of values rounded to T; 0 where that is not finite.
template <class T, int V>
__device__ __forceinline__ void store_rest(T* p, const float* d) {
  if constexpr (sizeof(T) == 2) {
    float r[V];
#pragma unroll
    for (int k = 0; k < V; ++k) {
      const float h = (float)(T)d[k];
      r[k] = __builtin_isfinite(h) ? d[k] - h : 0.f;
    }
    store<V>(p, r);
  }
}

constexpr int DZ_TB = 256;
template <class T, int KIND>
__global__ void __launch_bounds__(DZ_TB) k_dz(DzArgs g) {
  constexpr int V = 16 / sizeof(T);
  __shared__ float red[DZ_TB * V];
  const int rl = threadIdx.x / g.cl, lc = threadIdx.x - rl * g.cl, rows_at_once = DZ_TB / g.cl;
  const int c = (blockIdx.x * g.cl + lc) * V, left = g.d_out - c;
  const bool mine = rl < rows_at_once && c < g.lddz;
  const int lane = threadIdx.x & 63, t = blockIdx.y, groups = g.gr.n ? g.gr.n : 1;
  const T* __restrict__ dy = (const T*)g.dy + c;
  const T* __restrict__ z = (const T*)g.z + c;
  T* __restrict__ dz = (T*)g.dz + c;
  for (int g0 = 0; g0 < groups; g0 += 64) {
    long long lo = 0, hi = g.gr.rows;
    int first = 0, last = -1;
    if (g0 + lane < groups) {
      if (g.gr.n) group_rows(g.gr, g0 + lane, lo, hi);
      chunks_of(g.gr, g.chunk, g.tiles, lo, hi, first, last);
    }
    for (unsigned long long todo = __ballot(first <= t && t <= last); todo; todo &= todo - 1) {
      const int l = __ffsll((long long)todo) - 1, grp = g0 + l;
      const bool whole = __builtin_amdgcn_readlane(first, l) == __builtin_amdgcn_readlane(last, l);
      long long r0 = (long long)t * g.chunk, r1 = r0 + g.chunk < g.gr.rows ? r0 + g.chunk : g.gr.rows;
      if (g.gr.n) {
        const long long glo = __builtin_amdgcn_readlane((int)lo, l), ghi = __builtin_amdgcn_readlane((int)hi, l);
        r0 = glo > r0 ? glo : r0;
        r1 = ghi < r1 ? ghi : r1;
      }
      float sum[V];
#pragma unroll
      for (int k = 0; k < V; ++k) sum[k] = 0.f;
      if (mine && left >= V) {
        for (long long r = r0 + rl; r < r1; r += rows_at_once) {
          float d[V], s[V];
          load<V>(dy + r * g.lddy, d);
          load<V>(z + r * g.ldz, s);
          mul_slope<V>(d, s, KIND);
          store<V>(dz + r * g.lddz, d);
          if (g.rest) store_rest<T, V>(dz + r * g.lddz + g.rest, d);
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += d[k];
        }
      } else if (mine) {
        for (long long r = r0 + rl; r < r1; r += rows_at_once) {
          float d[V], s[V];
          load_n<V>(dy + r * g.lddy, left, d);
          load_n<V>(z + r * g.ldz, left, s);
          mul_slope<V>(d, s, KIND);
          store<V>(dz + r * g.lddz, d);              // (zeros past d_out: whole lines)
          if (g.rest) store_rest<T, V>(dz + r * g.lddz + g.rest, d);
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += d[k];
        }
      }
      if (!g.db) continue;
      __syncthreads();
#pragma unroll
      for (int k = 0; k < V; ++k) red[threadIdx.x * V + k] = sum[k];
      __syncthreads();
      if (rl == 0 && mine && left > 0) {
        for (int q = 1; q < rows_at_once; ++q)
#pragma unroll
          for (int k = 0; k < V; ++k) sum[k] += red[(q * g.cl + lc) * V + k];
        if (whole) store_n<V>((T*)g.db + (size_t)grp * g.d_out + c, left, sum);
        else store_n<V>(g.part_b + (size_t)(t + grp) * g.d_out + c, left, sum);
      }
    }
  }
}

// dbias of the groups that lie in several of k_dz's chunks: 32 columns per
// block, the parts in 32 slices.  blockIdx.y: the group.
template <class T>
__global__ void __launch_bounds__(1024) k_fold_bias(DzArgs g) {
  __shared__ float red[32][33];
  const int grp = blockIdx.y, q = threadIdx.x >> 5, l = threadIdx.x & 31, c = blockIdx.x * 32 + l;
  long long lo = 0, hi = g.gr.rows;
  if (g.gr.n) group_rows(g.gr, grp, lo, hi);
  int first, last;
  chunks_of(g.gr, g.chunk, g.tiles, lo, hi, first, last);
  if (first == last) return;
  float sum = 0.f;
  if (c < g.d_out) {
#pragma unroll 8
    for (int k = first + q; k <= last; k += 32) sum += g.part_b[(size_t)(k + grp) * g.d_out + c];
  }
  red[q][l] = sum;
  __syncthreads();
  if (q == 0 && c < g.d_out) {
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < 32; ++k) sum += red[k][l];
    store<1>((T*)g.db + (size_t)grp * g.d_out + c, &sum);
  }
}

// dw and dbias of the groups that lie in several chunks: their parts added in
// the order of the rows.  blockIdx.y: the group.
template <class T>
__global__ void __launch_bounds__(256) k_fold(Args g) {
  const int grp = blockIdx.y;
  long long lo = 0, hi = g.gr.rows;
  if (g.gr.n) group_rows(g.gr, grp, lo, hi);
  int first, last;
  chunks_of(g.gr, g.chunk, g.tiles, lo, hi, first, last);
  const int count = last - first + 1;
  if (count == 1) return;
  first += grp;
  const size_t wsize = (size_t)g.d_out * g.d_in;
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
  if (i < wsize) {
    const float* p = g.part + (size_t)first * wsize + i;
    float sum[4] = {0, 0, 0, 0}, v[4];
    for (int k = 0; k < count; ++k, p += wsize) {
      load_n<4>(p, (long long)(wsize - i), v);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += v[e];
    }
    store_n<4>((T*)g.out + (size_t)grp * wsize + i, (long long)(wsize - i), sum);
  }
  if (g.db)
    for (size_t o = (size_t)blockIdx.x * 256 + threadIdx.x; o < (size_t)g.d_out; o += (size_t)gridDim.x * 256) {
      float sum = 0.f;
      for (int k = 0; k < count; ++k) sum += g.part_b[(size_t)(first + k) * g.d_out + o];
      store<1>((T*)g.db + (size_t)grp * g.d_out + o, &sum);
    }
}

inline long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// Upper bound of the row tiles of `len` rows.
inline long long tile_bound(const Groups& gr, int len) { return ceil_div(gr.rows, len) + gr.n; }

// Blocks that fill the card: 256 CUs, two blocks each.
constexpr long long FULL = 512;

// Whether an operand's rows can be read in 16-byte words.
inline bool words(const void* p, long long ld, int width) {
  return (uintptr_t)p % 16 == 0 && ld % 8 == 0 && ld < (1 << 22) && width % 8 == 0;
}

template <int MODE>
bool words_path(const Args& a) {
  return words(a.a, a.lda, MODE == FWD ? a.d_in : a.d_out) && words(a.b, a.ldb, a.d_in) &&
         (size_t)a.d_out * a.d_in % 8 == 0;
}

// Whether an output is stored past the caches: where it is larger than the
// L2s (8 x 4 MB), so that it does not drive the operands out of them, and its
// rows are whole 128-byte lines; a line written in two parts would go to
// memory twice.  (65,536 x 1,024 -> 1,024, SiLU, z kept: 171 -> 151 us; at 776
// columns, rows of 12 1/8 lines, 159 -> 172 us.)
inline bool past_caches(const void* p, long long ld, long long rows, size_t es) {
  return (uintptr_t)p % 128 == 0 && ld * es % 128 == 0 && rows * ld * es > (32 << 20);
}

template <class T, int BM, int BN, int WM, int WN, int MODE, class O = T>
bool launch(hipStream_t st, Args a, long long tiles, long long nt) {
  if (tiles > 0x7fffffffLL / (nt < 8 ? 8 : nt) - 8) return false;
  const long long blocks = (MODE != DW && tiles >= 64 ? ceil_div(tiles, 8) * 8 : tiles) * nt;
  if (blocks == 0) return true;
  if (blocks > LAUNCH_THREADS / (64 * WM * WN)) return false;
  a.tiles = (int)tiles;
  a.nt = (int)nt;
  a.past = past_caches(a.out, a.ldo, a.gr.rows, sizeof(O));
  a.past_z = past_caches(a.z, a.ldz, a.gr.rows, sizeof(T));
  if constexpr (sizeof(T) == 2) {
    if (words_path<MODE>(a)) {
      k_dense16<O, BM, BN, WM, WN, MODE><<<dim3((unsigned)blocks), 64 * WM * WN, 0, st>>>(a);
      return true;
    }
  }
  if constexpr (BM > 128 || BN > 128) return false;       // (chosen for words_path only)
  else k_dense<T, O, BM, BN, WM, WN, MODE><<<dim3((unsigned)blocks), 64 * WM * WN, 0, st>>>(a);
  return true;
}

// Rounds of tiles of bm x bn that a card with `at_once` of them in work goes
// through (a group's last tile is half empty on average).
inline long long rounds(const Groups& gr, int bm, int width, int bn, long long at_once) {
  return ceil_div((ceil_div(gr.rows, bm) + gr.n / 2) * ceil_div(width, bn), at_once);
}

// FWD and DX: tiles of 128 x 128, two to a CU, or of 64 x 64 where those leave
// CUs idle.  FP32: 128 x 64 for up to 1.5 rounds of them.  BF16 words: the
// tiles of least cost, where a round of 128 x 128 counts 1, of 128 x 160 (for widths like 776 = 4.85 x 160) 1.25 and of 256 x
// 256, one to a CU, 1.74: it moves half the bytes per product through the
// caches.  us at 65,500 rows for 128 x 128 / 128 x 160 / 256 x 256 with the
// costs in brackets: 776 -> 776 134 / 119 / 131 (7 / 6.3 / 7); 1,024 -> 1,024
// 159 / 171 / 143 (8 / 8.8 / 7); 256 -> 1,024 63 / 67 / 55 (8 / 8.8 / 7); 1,024
// -> 256 45 / 50 / 40 (2 / 2.5 / 1.7); 256 -> 384, z kept, 33 / 46 / 37 (3 /
// 3.8 / 3.5).
// O: the results' type; FP32 from BF16 operands is a readout's form, a few
// columns wide, and has the small tiles alone (us at 65,502 rows, BF16 results /
// FP32: 776 -> 1 21.7 / 18.6, 776 -> 776 113 / 218).
template <class T, int MODE, class O = T>
bool run_rows(hipStream_t st, const Args& a) {
  const int width = MODE == FWD ? a.d_out : a.d_in;
  const long long rows = tile_bound(a.gr, 128), cols = ceil_div(width, 128);
  if constexpr (MODE == FWD) {
    // Its blocks' waves split the inner dimension, which has to be long enough
    // to be worth it (us, k_few / tiles of 64 x 64, 32 rows to 776 columns: BF16
    // inner 64 8.9 / 6.3, 256 7.8 / 7.1, 384 7.3 / 7.8, 776 6.6 / 10.6; FP32 128
    // 9.8 / 9.1, 192 9.5 / 10.7, 776 14 / 27; 512 rows of 776 11.8 / 11.0, FP32
    // 38 / 27; each with 2 us of the events around it)
    if (a.d_in > (sizeof(T) == 2 ? 256 : 128) && tile_bound(a.gr, 16) * ceil_div(width, 16) <= FULL) {
      Args b = a;
      b.tiles = (int)tile_bound(a.gr, 16);
      b.nt = (int)ceil_div(width, 16);
      const long long blocks = (b.tiles >= 64 ? ceil_div(b.tiles, 8) * 8 : b.tiles) * (long long)b.nt;
      k_few<T, O><<<dim3((unsigned)blocks), 256, 0, st>>>(b);
      return true;
    }
  }
  constexpr bool SMALL = sizeof(O) != sizeof(T);
  if (SMALL || rows * cols < FULL / 2 || (MODE == DX && a.rest))
    return launch<T, 64, 64, 2, 2, MODE, O>(st, a, tile_bound(a.gr, 64), ceil_div(width, 64));
  if constexpr (SMALL) {
    return false;
  } else if constexpr (sizeof(T) == 4) {
    // (128 x 128 / 128 x 64: 13,800 rows 337 -> 776 71 / 61 us, its dx 88 / 75; two
    // full rounds, dx of 65,502 x 256 -> 1,024, 212 / 238)
    if (2 * rows * cols <= 3 * FULL) return launch<T, 128, 64, 2, 2, MODE>(st, a, rows, ceil_div(width, 64));
  } else {
    if (words_path<MODE>(a)) {
      const double c128 = (double)rounds(a.gr, 128, width, 128, FULL);
      const double c160 = 1.25 * rounds(a.gr, 128, width, 160, FULL);
      const double c256 = 1.74 * rounds(a.gr, 256, width, 256, FULL / 2);
      if (c256 < c128 && c256 < c160)
        return launch<T, 256, 256, 2, 4, MODE>(st, a, tile_bound(a.gr, 256), ceil_div(width, 256));
      if (c160 < c128) return launch<T, 128, 160, 2, 2, MODE>(st, a, rows, ceil_div(width, 160));
    }
  }
  if constexpr (!SMALL) return launch<T, 128, 128, 2, 2, MODE>(st, a, rows, cols);
}

// Chunks of the rows for dw, nt tiles each: of least time, where a k-block
// takes a block about 1 us (FP32 1.5; two blocks to a CU) and a chunk's part of
// dw 0.033 us per tile to be written and read.  A multiple of 8 in BF16: a
// chunk's tiles on one XCD read its rows from one L2 (776 -> 776, 65,502 rows:
// 264 us with 10 chunks over all XCDs, 132 with 8).  (Tiles of 256 x 256 in BF16
// took 160 us where 128 x 128 took 159: half the operand bytes, but a third
// more padding and twice the parts.)
inline long long dw_chunks(long long rows, long long nt, int groups, bool half) {
  const int block_k = half ? 64 : 32;
  const double step = half ? 1.0 : 1.5;
  const long long most = rows / 64 < 512 ? rows / 64 : 512;
  const int by = half && most >= 8 ? 8 : 1;
  long long best = 1;
  double least = 1e300;
  for (long long s = by; s <= (most > by ? most : by); s += by) {
    const double t = (double)ceil_div(s * nt, FULL) * rows / s / block_k * step + 0.033 * s * nt;
    if (t < least) {
      least = t;
      best = s;
    }
  }
  // (a block goes through its chunk's groups one by one)
  while (best * 4 < groups && best * 64 < rows) best *= 2;
  return best;
}

const char* const TOO_LARGE = "more tiles than a launch of 2^32 threads holds";

template <class T>
painn_status run_fwd(painn_ctx* ctx, const painn_linear_args& p, int n_groups, const int32_t* offsets) {
  Args a{};
  a.gr = Groups{n_groups, offsets, p.rows};
  a.d_in = p.d_in; a.d_out = p.d_out;
  a.a = p.x; a.lda = p.ldx;
  a.b = p.w; a.ldb = p.d_in;
  a.bias = p.bias;
  a.act = p.activation;
  a.e = p.residual; a.lde = p.ldr;
  a.out = p.y; a.ldo = p.ldy;
  a.z = p.z; a.ldz = p.ldz;
  prof_mark(ctx->prof, ctx->stream, KC_LINEAR, true);
  bool ok;
  if constexpr (sizeof(T) == 2) ok = p.y_fp32 ? run_rows<T, FWD, float>(ctx->stream, a) : run_rows<T, FWD>(ctx->stream, a);
  else ok = run_rows<T, FWD>(ctx->stream, a);
  prof_mark(ctx->prof, ctx->stream, KC_LINEAR, false);
  if (!ok) return fail(ctx, PAINN_E_UNSUPPORTED, TOO_LARGE);
  return launched(ctx, "dense layer launch");
}

template <class T>
painn_status run_bwd(painn_ctx* ctx, const painn_linear_backward_args& p, int n_groups, const int32_t* offsets) {
  const int G = n_groups ? n_groups : 1;
  Args a{};
  a.gr = Groups{n_groups, offsets, p.rows};
  a.d_in = p.d_in; a.d_out = p.d_out;
  a.a = p.dy; a.lda = p.lddy;
  const hipStream_t st = ctx->stream;
  const bool have_dz = p.activation != PAINN_ACT_NONE && p.rows > 0;

  // dz and dbias
  DzArgs z{};
  constexpr int V = 16 / sizeof(T);
  const long long z_ld = ceil_div(p.d_out, 8 * V) * 8 * V, z_cols = ceil_div(z_ld / V, DZ_TB);
  size_t dz_bytes = 0, zb_bytes = 0;
  if (have_dz) {
    z.gr = a.gr;
    z.d_out = p.d_out;
    z.cl = (int)ceil_div(z_ld / V, z_cols);
    z.lddz = z_ld;
    // 16 blocks to a CU, at least 8 rows for each thread (65,502 x 776 BF16 from
    // memory, us: 4,096 blocks 59, 2,048 65, 512 91)
    const long long at_once = DZ_TB / z.cl, fill = ceil_div(4096, z_cols), few = ceil_div(p.rows, 8 * at_once);
    const long long zc = ceil_div(p.rows, fill < few ? fill : few);
    z.chunk = (int)(zc > (1 << 30) ? 1 << 30 : zc);
    z.tiles = (int)ceil_div(p.rows, z.chunk);
    z.dy = p.dy; z.lddy = p.lddy;
    z.z = p.z; z.ldz = p.ldz;
    z.db = p.dbias;
    // One rounding of dz to BF16 is one relative error of a whole row of dx and
    // of dw's.  Over many values it adds as much again as the rounding of the
    // result (1.4 times its error), but over a few, as in an energy's readout
    // of 28 rows, 2.1 times.  So up to 8,192 values their remainders go through
    // the products too (us, without / with: 28 x 257 -> 1 18 / 22, 8 x 776 -> 776
    // 22 / 27, 120 x 64 -> 64 15 / 17, 8,192 x 776 -> 1 53 / 77; beyond the limit,
    // 65,502 x 776 -> 1, 164 / 282).
    // And at any size where the caller asks for it: 65,502 x 776 -> 776 in 16
    // groups, both activations, 375 -> 938 us (tiles of 64 x 64), error of dx and
    // dw 0.0023 -> 0.0017, which is the rounding of the result.
    if (sizeof(T) == 2 && (p.dx || p.dw) && (p.dz_remainders || p.rows <= 8192 / p.d_out)) z.rest = p.rows * z.lddz;
    dz_bytes = align256((size_t)(z.rest ? 2 : 1) * p.rows * z.lddz * sizeof(T));
    a.rest = z.rest;
    zb_bytes = p.dbias ? align256((size_t)(z.tiles + G - 1) * p.d_out * sizeof(float)) : 0;
    a.lda = z.lddz;
  }

  // dw: its tiles and chunks
  Args d = a;
  d.b = p.x; d.ldb = p.ldx;
  d.out = p.dw;
  d.db = have_dz ? nullptr : p.dbias;
  const size_t wsize = (size_t)p.d_out * p.d_in;
  const int bt = p.d_in > 64 && p.d_out > 64 && !a.rest ? 128 : 64;
  const long long nt = ceil_div(p.d_out, bt) * ceil_div(p.d_in, bt);
  const long long cut = ceil_div(p.rows, dw_chunks(p.rows, nt, n_groups, sizeof(T) == 2));
  d.chunk = (int)(cut < 1 ? 1 : cut > (1 << 30) ? 1 << 30 : cut);
  d.nt_in = (int)ceil_div(p.d_in, bt);
  const long long chunks = p.rows > 0 ? ceil_div(p.rows, d.chunk) : 1;
  d.tiles = (int)chunks;
  const bool parts = p.dw && chunks > 1;
  if (parts && ceil_div(wsize, 1024) > LAUNCH_THREADS / 256) return fail(ctx, PAINN_E_UNSUPPORTED, TOO_LARGE);
  const size_t slots = (size_t)(chunks + G - 1);
  const size_t part_bytes = parts ? align256(slots * wsize * sizeof(float)) : 0;
  const size_t need = dz_bytes + zb_bytes + part_bytes + (parts ? slots * p.d_out * sizeof(float) : 0);
  if (need) {
    const painn_status ws = ops_workspace(ctx, need);
    if (ws != PAINN_OK) return ws;
  }
  char* ws = (char*)ctx->ows.p;
  d.part = (float*)(ws + dz_bytes + zb_bytes);
  d.part_b = (float*)(ws + dz_bytes + zb_bytes + part_bytes);

  prof_mark(ctx->prof, st, KC_LINEAR_BWD, true);
  bool ok = true;
  if (have_dz) {
    z.dz = ws;
    z.part_b = (float*)(ws + dz_bytes);
    a.a = d.a = ws;
    ok = z.tiles < 65536;
    if (ok) {
      const dim3 grid((unsigned)z_cols, z.tiles);
      if (p.activation == PAINN_ACT_SILU) k_dz<T, PAINN_ACT_SILU><<<grid, DZ_TB, 0, st>>>(z);
      else if (p.activation == PAINN_ACT_RELU) k_dz<T, PAINN_ACT_RELU><<<grid, DZ_TB, 0, st>>>(z);
      else k_dz<T, PAINN_ACT_GELU><<<grid, DZ_TB, 0, st>>>(z);
      if (p.dbias && z.tiles > 1) k_fold_bias<T><<<dim3((unsigned)ceil_div(p.d_out, 32), G), 1024, 0, st>>>(z);
    }
  }
  if (ok && p.dw) {
    ok = bt == 128 ? launch<T, 128, 128, 2, 2, DW>(st, d, chunks, nt) : launch<T, 64, 64, 2, 2, DW>(st, d, chunks, nt);
    if (ok && parts) k_fold<T><<<dim3((unsigned)ceil_div(wsize, 1024), G), 256, 0, st>>>(d);
  }
  if (ok && p.dx && p.rows > 0) {
    a.b = p.w; a.ldb = p.d_in;
    a.act = p.x_activation;
    a.e = p.xz; a.lde = p.ldxz;
    a.out = p.dx; a.ldo = p.lddx;
    ok = run_rows<T, DX>(st, a);
  }
  prof_mark(ctx->prof, st, KC_LINEAR_BWD, false);
  if (!ok) return fail(ctx, PAINN_E_UNSUPPORTED, TOO_LARGE);
  return launched(ctx, "dense layer reverse launch");
}

bool known_act(int a) { return a >= PAINN_ACT_NONE && a <= PAINN_ACT_GELU; }

painn_status dense_check(painn_ctx* ctx, int prec, int act, int x_act, int64_t rows, int d_in, int d_out,
                         int n_groups, const int32_t* offsets, bool grouped) {
  if (prec == PAINN_FP64) return fail(ctx, PAINN_E_UNSUPPORTED, "the dense layer runs in FP32 and BF16");
  if (prec != PAINN_FP32 && prec != PAINN_BF16) return fail(ctx, PAINN_E_ARG, "unknown precision");
  if (!known_act(act) || !known_act(x_act)) return fail(ctx, PAINN_E_ARG, "unknown activation");
  if (d_in < 1 || d_out < 1) return fail(ctx, PAINN_E_ARG, "widths must be at least 1");
  if (rows < 0) return fail(ctx, PAINN_E_ARG, "rows must not be negative");
  if (d_in > (1 << 20) || d_out > (1 << 20) || rows > (1LL << 40))
    return fail(ctx, PAINN_E_UNSUPPORTED, "widths above 2^20 or more than 2^40 rows");
  if (grouped) {
    if (n_groups < 1 || n_groups > 4096) return fail(ctx, PAINN_E_ARG, "n_groups must be in [1, 4096]");
    if (!offsets) return fail(ctx, PAINN_E_ARG, "null offsets");
    if (rows > 0x7fffffffLL) return fail(ctx, PAINN_E_ARG, "grouped rows must be below 2^31");
  }
  return PAINN_OK;
}

painn_status fwd_entry(painn_ctx* ctx, const painn_linear_args* p, int n_groups, const int32_t* offsets, bool grouped) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!p) return fail(ctx, PAINN_E_ARG, "null args");
  const painn_status st = dense_check(ctx, p->precision, p->activation, 0, p->rows, p->d_in, p->d_out, n_groups,
                                      offsets, grouped);
  if (st != PAINN_OK) return st;
  if (p->rows == 0) return PAINN_OK;
  if (!p->x || !p->w || !p->y) return fail(ctx, PAINN_E_ARG, "null array");
  if (p->ldx < p->d_in || p->ldy < p->d_out || (p->residual && p->ldr < p->d_out) || (p->z && p->ldz < p->d_out))
    return fail(ctx, PAINN_E_ARG, "a row stride is below the row's width");
  if (p->y_fp32 != 0 && p->y_fp32 != 1) return fail(ctx, PAINN_E_ARG, "y_fp32 is 0 or 1");
  if (p->y_fp32 && p->precision == PAINN_BF16 && p->y == p->residual)
    return fail(ctx, PAINN_E_ARG, "y in place of the residual has another type");
  if (misplaced(p->y, p->ldy, p->residual, p->ldr, p->rows))
    return fail(ctx, PAINN_E_ARG, "y in place of the residual has another row stride");
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  return p->precision == PAINN_FP32 ? run_fwd<float>(ctx, *p, n_groups, offsets)
                                    : run_fwd<b16>(ctx, *p, n_groups, offsets);
}

painn_status bwd_entry(painn_ctx* ctx, const painn_linear_backward_args* p, int n_groups, const int32_t* offsets,
                       bool grouped) {
  if (!ctx) return PAINN_E_ARG;
  ctx->err.clear();
  if (!p) return fail(ctx, PAINN_E_ARG, "null args");
  const painn_status st = dense_check(ctx, p->precision, p->activation, p->x_activation, p->rows, p->d_in, p->d_out,
                                      n_groups, offsets, grouped);
  if (st != PAINN_OK) return st;
  if (p->dz_remainders != 0 && p->dz_remainders != 1) return fail(ctx, PAINN_E_ARG, "dz_remainders is 0 or 1");
  if (p->dbias && !p->dw) return fail(ctx, PAINN_E_ARG, "dbias is formed with dw");
  if (p->rows > 0) {
    if (!p->dy || (p->activation != PAINN_ACT_NONE && !p->z) || (p->dw && !p->x) || (p->dx && !p->w) ||
        (p->dx && p->x_activation != PAINN_ACT_NONE && !p->xz))
      return fail(ctx, PAINN_E_ARG, "null array");
    if (p->lddy < p->d_out || (p->activation != PAINN_ACT_NONE && p->ldz < p->d_out) || (p->dw && p->ldx < p->d_in) ||
        (p->dx && p->lddx < p->d_in) || (p->dx && p->x_activation != PAINN_ACT_NONE && p->ldxz < p->d_in))
      return fail(ctx, PAINN_E_ARG, "a row stride is below the row's width");
    if (p->x_activation != PAINN_ACT_NONE && misplaced(p->dx, p->lddx, p->xz, p->ldxz, p->rows))
      return fail(ctx, PAINN_E_ARG, "dx in place of xz has another row stride");
  }
  if (!p->dw && (!p->dx || p->rows == 0)) return PAINN_OK;
  (void)hipSetDevice(ctx->device);
  (void)hipGetLastError();
  return p->precision == PAINN_FP32 ? run_bwd<float>(ctx, *p, n_groups, offsets)
                                    : run_bwd<b16>(ctx, *p, n_groups, offsets);
}

}  // namespace

extern "C" {

painn_status painn_linear(painn_ctx* ctx, const painn_linear_args* args) {
  return fwd_entry(ctx, args, 0, nullptr, false);
}
painn_status painn_linear_backward(painn_ctx* ctx, const painn_linear_backward_args* args) {
  return bwd_entry(ctx, args, 0, nullptr, false);
}
painn_status painn_grouped_linear(painn_ctx* ctx, const painn_linear_args* args, int32_t n_groups,
                                  const int32_t* offsets) {
  return fwd_entry(ctx, args, n_groups, offsets, true);
}
painn_status painn_grouped_linear_backward(painn_ctx* ctx, const painn_linear_backward_args* args, int32_t n_groups,
                                           const int32_t* offsets) {
  return bwd_entry(ctx, args, n_groups, offsets, true);
}

}  // extern "C"

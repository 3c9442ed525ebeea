// Attention over the paged 4-bit cache (format: include/pyr.h).
//
// With s the (scale, zero) of a row and group, a score is q . K_j = sum_g scale_jg (sum_{d in g} q_d c_jd) + zero_jg
// (sum_{d in g} q_d): codes stay small integers, which are exact in every type, and the two factors are applied in fp32 to
// the group's sum. The same for V: o += p_j scale_jg c_jd + p_j zero_jg. Softmax is kept as a running maximum and sum.
//
// Work. The unit is one tile of 16 rows of one (entry, KV head, column group); a column is one query row (token, query head
// of the KV head). All units of a call are numbered in order and every warp takes the same number of consecutive ones, so
// lists of any lengths keep the whole machine equally busy. A warp whose range starts or ends inside a (entry, head, column
// group) leaves a partial state; the CTA merges its warps' states in order, and what crosses CTAs goes to a workspace where
// the CTA that finishes last merges it, again in order: results do not depend on which CTA that is.
//
// One more warp loads for all of them: its lane w keeps the ring of warp w filled, a stage of which is one bulk copy of up to two
// tiles (a head's tiles of a page are contiguous). As lanes of one warp the loaders cost an instruction each step instead of
// one for every warp that consumes.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <climits>

#include "pyr_internal.h"
#include "tc_common.cuh"

namespace pyr {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kStageTiles = 2;           // a stage of a warp's ring: one copy of up to two tiles
constexpr int kStageRows = kStageTiles * kPageTile;
// What beginning and ending a (entry, head, column group) costs a warp, in tiles: its queries, a first step that sets the maximum
// and the scales' factors, its sums (64 ragged lists of 32 heads: 102 us with 2, 96 with 3, 92 with 4, 90 with 6 and 8).
constexpr int kSegmentUnits = kAttnSegmentUnits;
// A warp's share is at least this much: next to nothing, since small calls are bound by a warp's own latency, 2 us a step
// (with 2 instead of 4 and 8: 385 rows of 32 heads 20.5, 22.5 and 24.6 us, the small fp32 model 21, 26 and 32 us).
constexpr int kMinUnits = 2;
constexpr int kCtaTiles = 8;             // a (entry, head, column group) of up to this many tiles a warp may be a CTA's alone
constexpr int kMaxWarps = 12;

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }

template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// A partial state's place in the call.
struct Piece {
  long long u0, u1;      // units of its (entry, head, column group) that stand for tiles
  int entry, h, cg;
  int begins, ends;      // whether it holds the first / the last of them
  int valid;
};

struct Sched {
  long long sums[kMaxWarps + 1];
  long long first_unit[kMaxWarps];   // of the entry in which a warp's range starts
  long long share_u, share_units;    // the CTA's units, where it takes one (entry, head, column group)
  int entry[kMaxWarps], list[kMaxWarps], len[kMaxWarps];
  int abort_flag;
  int last[2], open_c1[2], open_count[2], open_piece[2];   // what the CTA leaves for others
  float den[kAttnCols];
  Piece piece[kMaxWarps][2];
};

template <int kWarpsAll>
__device__ __forceinline__ long long block_scan(long long x, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  long long before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWarpsAll; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return before + incl - x;
}

// Units of entry i: 0 if its list id is out of range (the entry is refused). A (head, column group) has kSegmentUnits units
// that stand for no tile before those that do: short lists cost more than their tiles, and a warp's share must say so.
__device__ __forceinline__ long long entry_units(const PagesAttnArgs& a, int i, int cgs, int* list, int* len) {
  *list = pages_list(a.p, a.lists, i);
  *len = *list < 0 ? 0 : pages_len(a.p, *list);
  return *list < 0 ? 0 : (long long)(attn_tiles(*len) + kSegmentUnits) * a.p.Hkv * cgs;
}

// The (entry, head, column group) that a warp works on, and the tiles [t, t1) of it that are the warp's.
struct Place {
  int entry, len, tiles, h, cg, t, t1;
  int list;

  __device__ __forceinline__ void open(const PagesAttnArgs& a) {       // the entry's list
    list = pages_list(a.p, a.lists, entry);
    len = list < 0 ? 0 : pages_len(a.p, list);
    tiles = list < 0 ? 0 : (int)attn_tiles(len);
  }
  // Takes units from `left` on, of which `r` of this (head, column group) lie before the warp's.
  __device__ __forceinline__ void take(int r, int* left) {
    const int n = min(*left, tiles + kSegmentUnits - r);
    t = max(0, r - kSegmentUnits);
    t1 = max(0, r + n - kSegmentUnits);
    *left -= n;
  }
  // unit o of entry e, whose list and length are at hand
  __device__ __forceinline__ void start(const PagesAttnArgs& a, int cgs, int e, int l, int n, long long o, int* left) {
    entry = e; list = l; len = n;
    tiles = (int)attn_tiles(len);
    const int per = tiles + kSegmentUnits;
    int r;
    if (o >> 31 == 0) {                          // (64-bit divisions take a tenth of a microsecond each)
      const uint32_t hc = (uint32_t)o / (uint32_t)per;
      r = (int)((uint32_t)o - hc * per);
      h = (int)(hc / (uint32_t)cgs);
      cg = (int)(hc - (uint32_t)h * cgs);
    } else {
      r = (int)(o % per);
      const long long hc = o / per;
      cg = (int)(hc % cgs);
      h = (int)(hc / cgs);
    }
    take(r, left);
  }
  // The next one. Returns whether its list is another.
  __device__ __forceinline__ bool next(const PagesAttnArgs& a, int cgs, int* left) {
    bool other = false;
    if (++cg >= cgs) {
      cg = 0;
      if (++h >= a.p.Hkv) {
        h = 0;
        other = true;
        do { ++entry; open(a); } while (list < 0 && entry + 1 < a.n);  // refused entries have no unit
      }
    }
    take(0, left);
    return other;
  }
};

// Where an entry's column lies in out and lse.
struct OutPlace {
  int64_t out, lse;
  __device__ __forceinline__ OutPlace(const PagesAttnArgs& a, int entry, int h, int col) {
    const int tok = col / a.rep, head = h * a.rep + col % a.rep;
    out = (int64_t)entry * a.osb + (int64_t)tok * a.ost + (int64_t)head * a.osh;
    lse = ((int64_t)entry * a.Hq + head) * a.T + tok;
  }
};
__device__ __forceinline__ float lse_of(float m, float den) {
  return den > 0.f ? (m + log2f(den)) * kLn2 : (den == 0.f ? -INFINITY : den);
}

// Shared memory of a CTA: per warp a ring of tiles, the queries of its segment and a state of [cols][D + 2]; the state that a
// warp leaves last goes where its ring was.
template <class Body>
struct Layout {
  static constexpr int state = Body::COLS * (Body::kDim + 2);
  static constexpr int ring = Body::kStages * kStageTiles * Body::kTileBytes;
  static constexpr int warp_bytes = (ring + (Body::kQueryFloats + state) * 4 + 127) / 128 * 128;
  static_assert(state * 4 <= ring, "the last state fits the ring");
  static_assert(kAttnMaxCtas * Body::COLS * 4 <= Body::kWarps * warp_bytes, "a weight per CTA and column fits where the rings were");
  static constexpr int total = Body::kWarps * warp_bytes;
};

// ------------------------------------------------------------------ one warp's tiles, on CUDA cores (fp32)
// Every product in fp32: fp32 outputs are held to what fp32 can do, which operands of fewer bits cannot. A sum of codes times
// queries (up to 15 of them each) leaves fp32 before q . K does: a query row with an element of 2^100 or more is taken times 2^-64, its
// scores times 2^64. Bound by its multiply-adds where a KV head has several query rows (2 x 128 of them a row and column).
// Lane 4 i + j. K: rows i and i + 8, the quarter of the dimensions that chunk j of a stored row holds. V: the eighth of the
// dimensions that chunk i holds, of the rows j, j + 4, j + 8, j + 12.
template <int D, int GROUP, int kCols>
struct CoreBody {
  using Type = float;
  static constexpr int kDim = D, COLS = kCols, kWarps = 7, kBlocks = 1, kQueryFloats = COLS * D + 4;   // queries and their scores' factors lie in shared memory
  static constexpr int kStages = 3, kTileBytes = kPageTile * (D + 8 * (D / GROUP));
  static constexpr int G = D / GROUP, U = GROUP / 32, X = D / 32;   // X: words of K / halves of V in a lane's chunk
  static_assert(COLS <= 4, "a factor a column");
  float acc[COLS][4 * X];
  float m[COLS], l[COLS], qsum[COLS][G];
  int limit[COLS];

  __device__ __forceinline__ void begin(const PagesAttnArgs& a, const Place& c, int cols_total, float* qs, int lane) {
    const int j = lane & 3, col0 = c.cg * COLS;
    const int ncols = min(COLS, cols_total - col0);
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      m[x] = -INFINITY; l[x] = 0.f;
#pragma unroll
      for (int y = 0; y < 4 * X; ++y) acc[x][y] = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) qsum[x][g] = 0.f;
      const int col = col0 + x, tok = col / a.rep, head = c.h * a.rep + col % a.rep;
      limit[x] = c.len - (a.T - 1 - tok);
      const float* q = static_cast<const float*>(a.q) + (int64_t)c.entry * a.qsb + (int64_t)tok * a.qst + (int64_t)head * a.qsh;
      // queries in the order of the stored codes
      bool far = false;
      for (int p = lane; p < D; p += 32) {
        const float v = x < ncols ? q[8 * k_slot_word(D, GROUP, p >> 3) + (p & 7)] : 0.f;
        qs[x * D + p] = v;
        far |= fabsf(v) >= 0x1p100f;
      }
      far = __any_sync(0xffffffffu, far);
      if (lane == 0) qs[COLS * D + x] = far ? 0x1p64f : 1.f;
      if (far)
        for (int p = lane; p < D; p += 32) qs[x * D + p] *= 0x1p-64f;
    }
    __syncwarp();
#pragma unroll
    for (int x = 0; x < COLS; ++x)
#pragma unroll
      for (int s = 0; s < X; ++s)
#pragma unroll
        for (int k = 0; k < 8; ++k) qsum[x][s / U] += qs[x * D + (j * X + s) * 8 + k];
  }

  __device__ __forceinline__ void tile(const PagesAttnArgs& a, const uint8_t* tp, int row0, int rows, const float* qs, int lane) {
    const int i = lane >> 2, j = lane & 3;
    const float sc2 = a.scale * kLog2e;
    float s[2][COLS];
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const int r = i + 8 * rr;
      const uint32_t* codes = reinterpret_cast<const uint32_t*>(tp + tile_k_row(D, r)) + j * X;
#pragma unroll
      for (int x = 0; x < COLS; ++x) s[rr][x] = 0.f;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float part[COLS];
#pragma unroll
        for (int x = 0; x < COLS; ++x) part[x] = 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int w = g * U + u;
          const uint32_t word = codes[w];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float cf = (float)((word >> (4 * k)) & 15u);
#pragma unroll
            for (int x = 0; x < COLS; ++x) part[x] = fmaf(cf, qs[x * D + (j * X + w) * 8 + k], part[x]);
          }
        }
        const uint32_t sz = *reinterpret_cast<const uint32_t*>(tp + tile_k_word(D, G, r, g));
        const float scale = __uint_as_float(sz << 16), zero = __uint_as_float(sz & 0xffff0000u);
#pragma unroll
        for (int x = 0; x < COLS; ++x) s[rr][x] += fmaf(scale, part[x], zero * qsum[x][g]);
      }
#pragma unroll
      for (int x = 0; x < COLS; ++x) {
        s[rr][x] += __shfl_xor_sync(0xffffffffu, s[rr][x], 1);
        s[rr][x] += __shfl_xor_sync(0xffffffffu, s[rr][x], 2);
        // rows behind the list's end hold anything: replaced, not multiplied away
        s[rr][x] = r < rows && row0 + r < limit[x] ? s[rr][x] * qs[COLS * D + x] * sc2 : -INFINITY;
      }
    }
    const bool edge = row0 + kPageTile > limit[0];               // some column sees less than the whole tile
    float p[2][COLS];
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      float mx = fmaxf(s[0][x], s[1][x]);
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
      mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
      const float m_new = fmaxf(m[x], mx);
      const float ref = m_new == -INFINITY ? 0.f : m_new;       // nothing seen yet: every term is zero
      const float corr = exp2f(m[x] - ref);
      p[0][x] = exp2f(s[0][x] - ref);
      p[1][x] = exp2f(s[1][x] - ref);
      l[x] = l[x] * corr + p[0][x] + p[1][x];
      m[x] = m_new;
#pragma unroll
      for (int y = 0; y < 4 * X; ++y) acc[x][y] *= corr;
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int r = j + 4 * y;                                  // its probabilities are in the lanes of row r (or r - 8)
      float pr[COLS];
#pragma unroll
      for (int x = 0; x < COLS; ++x) pr[x] = __shfl_sync(0xffffffffu, p[y >> 1][x], (r & 7) << 2);
      if (r < rows) {
        const uint16_t* codes = reinterpret_cast<const uint16_t*>(tp + tile_v_row(D, r)) + i * X;
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const uint32_t sz = *reinterpret_cast<const uint32_t*>(tp + tile_v_word(D, G, r, g));
          const float scale = __uint_as_float(sz << 16), zero = __uint_as_float(sz & 0xffff0000u);
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const uint32_t half = codes[g * U + u];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float val = fmaf(scale, (float)((half >> (4 * k)) & 15u), zero);
              if (edge && !(fabsf(val) <= 3.402823466e38f)) {      // what a column does not see must not reach it as 0 x NaN
#pragma unroll
                for (int x = 0; x < COLS; ++x)
                  if (row0 + r < limit[x]) acc[x][(g * U + u) * 4 + k] = fmaf(pr[x], val, acc[x][(g * U + u) * 4 + k]);
                val = 0.f;
              }
#pragma unroll
              for (int x = 0; x < COLS; ++x) acc[x][(g * U + u) * 4 + k] = fmaf(pr[x], val, acc[x][(g * U + u) * 4 + k]);
            }
          }
        }
      }
    }
  }

  __device__ __forceinline__ void stage(const PagesAttnArgs& a, const uint8_t* tp, int row0, int rows, const float* qs, int lane) {
#pragma unroll 1
    for (int x = 0; x < kStageTiles && rows > x * kPageTile; ++x)
      tile(a, tp + x * kTileBytes, row0 + x * kPageTile, min(rows - x * kPageTile, kPageTile), qs, lane);
  }

  // sums over the lanes that share a row or a dimension
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], o);
#pragma unroll
      for (int y = 0; y < 4 * X; ++y) {
        acc[x][y] += __shfl_xor_sync(0xffffffffu, acc[x][y], 1);
        acc[x][y] += __shfl_xor_sync(0xffffffffu, acc[x][y], 2);
      }
    }
  }
  __device__ __forceinline__ void keep(float* state, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
#pragma unroll
      for (int y = 0; y < 4 * X; ++y)
        if (j == (y & 3)) state[x * (D + 2) + 4 * v_slot_half(D, GROUP, i * X + (y >> 2)) + (y & 3)] = acc[x][y];
      if (lane == 0) { state[x * (D + 2) + D] = m[x]; state[x * (D + 2) + D + 1] = l[x]; }
    }
  }
  __device__ __forceinline__ void write(const PagesAttnArgs& a, const Place& c, int cols_total, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
      if (c.cg * COLS + x >= cols_total) break;
      const OutPlace at(a, c.entry, c.h, c.cg * COLS + x);
      const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];
#pragma unroll
      for (int y = 0; y < 4 * X; ++y)
        if (j == (y & 3))
          static_cast<float*>(a.out)[at.out + 4 * v_slot_half(D, GROUP, i * X + (y >> 2)) + (y & 3)] = acc[x][y] * inv;
      if (lane == 0 && a.lse) a.lse[at.lse] = lse_of(m[x], l[x]);
    }
  }
};

// ------------------------------------------------------------------ one warp's tiles, on tensor cores (bf16)
// Rows of the cache are the 16 rows of m16n8k16, the (up to 8) query rows its 8 columns: S^T = K Q^T, O^T = V^T P^T. The
// instruction's rate is far from a bound here; what counts is that a register of codes becomes an operand in few steps. Lane
// 4 i + j holds, of K's row i (and i + 8), chunk j: a word's nibbles k and k + 4 are a pair of operands, and since any order
// of the dimensions will do as long as the queries have the same, the words are stored in the order in which lanes take
// them. Of V it holds chunk i of four rows, two rows' halves side by side giving pairs of rows of one dimension.
// (Legacy warp-level MMA: a decode step reads every code once, and tcgen05 would need the codes as 8- or 16-bit
// operands in shared memory first.)
// Row r of the matrices is row r ^ ((r >> 1) & 1) of the tile, which spreads the lanes' shared-memory reads over the banks.
//
// Operands are f16. A code masked in place is an operand already: as the bits of an f16 number a nibble n in bits 0 .. 3 is the
// subnormal n 2^-24, in bits 4 .. 7 it is n 2^-20, both exact, so that a word's eight codes take one shift and four masks
// and nothing is added or converted. (The factors go into the queries for K, into the sums at the end for V.) What f16 lacks
// is range, so both factors that are not codes are normalised by powers of two: a query row so that its largest element is
// near f16's (what is then below f16's smallest step is below 2^-35 of that element), and the scales that multiply P, which
// f16 holds to 2^-11, by a factor per group that follows them (`norm`) and keeps the products near f16's top: many rows of
// little weight behind one of much add up, and what f16 drops of them is the same for all. (16384 rows of 2^-17.5 of the first
// one's weight, one of the first 32 with scales 50 times the others': off by up to 0.013 of values of 1.2 with factors near 1.)
// The factor that a score needs to undo the first, 2^e for a row whose largest element has the exponent e, times 2^9 and the
// softmax scale, passes fp32 from about e = 122 on: part of it is then multiplied in by itself (`up`), in the stages' branch for
// edges, which such a segment always takes.
// V's codes have a mean of 7.5, so that o grows with the number of rows while what matters in it grows with its root. The
// instruction truncates its sums, and an o far above what matters would let that show: every kCentre steps what a group's o
// have in common is moved to the group's sum of zeros, which is kept apart and rounded. (100 k rows a list, error against 64
// bits: 1.65e-3 is the output's own rounding, 1.77e-3 with 4 or 8, 1.78e-3 with 16, 1.90e-3 with 64; the rest is P's.)
//
// What bounds it: 277 instructions a tile and warp, 88 of them to take codes out of words, half of all on the integer pipe (52 % busy
// over a launch) and the rest waiting for one another in 11 warps an SM: 161 registers allow no more (15 warps with 128,
// some of them spilled, are as fast). Measured with an idle start (64 lists of 1088 rows, 32 heads, 321 MB): 76 us = 4.2 TB/s;
// by the SMs' clocks about 5 us pass before the first tile is there and 7 from the last tile to the end (merging).
// A group of V that is zero throughout (heads padded with zeros) has no factor, and every stage looks for one: 64 lists of 1088
// rows, 32 heads, groups of 32: 94 us, 113 with such a group.
__device__ __forceinline__ void mma_full(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return reinterpret_cast<uint32_t&>(x); }
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) { return as_u32(__floats2half2_rn(lo, hi)); }
// The four pairs of codes (nibbles k and k + 4) of x as f16 pairs: times 2^-24 for k = 0 and 2, times 2^-20 for k = 1 and 3.
__device__ __forceinline__ void codes4(uint32_t x, uint32_t* y) {
  const uint32_t z = x >> 8;
  y[0] = x & 0x000F000Fu;
  y[1] = x & 0x00F000F0u;
  y[2] = z & 0x000F000Fu;
  y[3] = z & 0x00F000F0u;
}
// 2^k, -127 <= k <= 127
__device__ __forceinline__ float power_of_two(int k) {
  return __uint_as_float(k > -127 ? (uint32_t)(k + 127) << 23 : 0x00400000u);
}
// The exponent of x > 0 (-127 for 0 and subnormals).
__device__ __forceinline__ int exponent_of(float x) { return (int)(__float_as_uint(x) >> 23) - 127; }
// 2^-e for the exponent e of x > 0 (clamped so that it and its inverse are numbers)
__device__ __forceinline__ float inverse_power(float x) {
  return power_of_two(-min(max(exponent_of(x), -114), 126));
}

template <int D, int GROUP>
struct MmaBody {
  using Type = __nv_bfloat16;
  static constexpr int G = D / GROUP, U = GROUP / 32, X = D / 32;
  static constexpr int kDim = D, COLS = 8, kWarps = 11, kBlocks = 1, kQueryFloats = 0;
  static constexpr int kTileBytes = kPageTile * (D + 8 * G), kStages = kTileBytes > 2304 ? 2 : 3;
  static constexpr float kLazy = 4.f;            // the maximum is raised once a score is 2^4 above it
  // The largest scale of a group times its factor is set to 2^8 .. 2^9 and set anew above 2^11, or where all rows of a stage are below
  // 2^4: P times that stays below 2^15 (f16 ends at 2^16), is held to 2^-11 down to weights of 2^-18 of the largest, and what
  // is smaller to 2^-29 of it.
  static constexpr float kScaleTop = 0x1p11f, kScaleSet = 0x1p8f, kScaleLow = 0x1p4f;
  static constexpr int kCentre = 8;
  uint32_t qf[X][4];
  float qsum[G][2];                              // sums of the queries over a group
  float o[X][2][4], zacc[G][2], norm[G], l[2], sc2[2], up[2];
  float ref[2], raise[2];                        // the maximum (0 and raise = -Inf: nothing seen) and what raises it, before sc2
  int limit[2], limit_min, steps;

  __device__ __forceinline__ void begin(const PagesAttnArgs& a, const Place& c, int cols_total, float*, int lane) {
    const int i = lane >> 2, j = lane & 3, col0 = c.cg * COLS;
    bool far = false;
    {
      const int col = col0 + i, tok = col / a.rep, head = c.h * a.rep + col % a.rep;
      const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)c.entry * a.qsb + (int64_t)tok * a.qst + (int64_t)head * a.qsh;
      float f[X][8], big = 0.f;
#pragma unroll
      for (int w = 0; w < X; ++w) {
        uint4 r = make_uint4(0, 0, 0, 0);
        if (col < cols_total) r = *reinterpret_cast<const uint4*>(q + 8 * k_slot_word(D, GROUP, j * X + w));
        const uint32_t u[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          f[w][2 * k] = __uint_as_float(u[k] << 16);
          f[w][2 * k + 1] = __uint_as_float(u[k] & 0xffff0000u);
          big = fmaxf(big, fmaxf(fabsf(f[w][2 * k]), fabsf(f[w][2 * k + 1])));
        }
      }
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
      big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
      // 2^-e, of a row that is smaller still 2^112: with 2^15 a number, and bf16's smallest, 2^-133, keeps all its bits
      const int e = min(max(exponent_of(big), -112), 127);
      const float down = power_of_two(-e);
#pragma unroll
      for (int w = 0; w < X; ++w)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float by = k & 1 ? 0x1p11f * down : 0x1p15f * down;      // for codes times 2^-20 and 2^-24
          qf[w][k] = pack_f16(f[w][k] * by, f[w][k + 4] * by);
        }
      // Scores come out times 2^-9 down, so they take `scale` times 2^(9 + e): up to 2^96 of it in sc2, the rest in up. (At least
      // 2^-149, at most the largest number: a row that a column does not see is -Inf times it.)
      const float scale = a.scale * kLog2e;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int all = 9 + __shfl_sync(0xffffffffu, e, (2 * j + x) * 4);
        const int apart = min(max(all + exponent_of(scale) - 96, 0), 127), k = all - apart;
        sc2[x] = fminf(fmaxf(scale * power_of_two(k / 2) * power_of_two(k - k / 2), 0x1p-149f), 3.402823466e38f);
        up[x] = power_of_two(apart);
        far |= apart > 0;
      }
      far = __any_sync(0xffffffffu, far);
    }
    // sums of the queries over each group, by the instruction itself (every row of a matrix of constants that undo the queries'
    // factors: operands 0, 1 go with nibbles 0 and 2 of a code word, operands 2, 3 with nibbles 1 and 3)
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const uint32_t undo[4] = {0x2C002C00u, 0x2C002C00u, 0x3C003C00u, 0x3C003C00u};       // 1/16, 1
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        mma_full(s, undo, qf[g * U + u][0], qf[g * U + u][1]);
        mma_full(s, undo, qf[g * U + u][2], qf[g * U + u][3]);
      }
      qsum[g][0] = s[0] * 0x1p-20f;
      qsum[g][1] = s[1] * 0x1p-20f;
      zacc[g][0] = zacc[g][1] = 0.f;
      norm[g] = 0.f;
    }
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) o[x][y][0] = o[x][y][1] = o[x][y][2] = o[x][y][3] = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      raise[x] = -INFINITY; ref[x] = 0.f; l[x] = 0.f;
      limit[x] = c.len - (a.T - 1 - (col0 + 2 * j + x) / a.rep);
    }
    limit_min = far ? INT_MIN / 2 : c.len - (a.T - 1 - col0 / a.rep);
    steps = 0;
  }

  __device__ __forceinline__ float top_score(int x) const { return raise[x] == -INFINITY ? -INFINITY : ref[x]; }

  // Brings the group's factor to the largest scale of the tile (the lanes hold two rows each): o goes with it.
  __device__ __forceinline__ void renorm(int g, float big) {
    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 4));
    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 8));
    big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 16));
    if (!(big > 0.f)) return;                    // only zeros (or NaN): any factor will do
    const float to = inverse_power(big) * kScaleSet;
    float by = norm[g] == 0.f ? 1.f : to / norm[g];
    if (by > 1.f) {                              // what has been summed is beyond such small scales if it does not stay finite
      float most = 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int k = 0; k < 4; ++k) most = fmaxf(most, fabsf(o[g * U + u][y][k]));
      if (__any_sync(0xffffffffu, most > 0.f && most * by > 1e30f)) return;
      by = fminf(by, 3.402823466e38f);           // (Inf, where nothing has been summed: it stays zero)
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[g * U + u][y][k] *= by;
    norm[g] = to;
  }

  // Moves what a group's o have in common (one of them, that is) to the group's sum of zeros.
  __device__ __forceinline__ void centre(int lane) {
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float c = __shfl_sync(0xffffffffu, o[g * U][0][x], lane & 3);
        if (lane < 4 && norm[g] != 0.f) zacc[g][x] += c * 0x1p24f * (1.f / norm[g]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            o[g * U + u][y][x] -= c;
            o[g * U + u][y][2 + x] -= 16.f * c;
          }
      }
  }

  // Up to two tiles (those of a stage): `rows` of their 32 rows belong to the list, the first of them is its row `row0`.
  __device__ __forceinline__ void stage(const PagesAttnArgs& a, const uint8_t* tp, int row0, int rows, const float*, int lane) {
    const int i = lane >> 2, j = lane & 3;
    const int ri = i ^ ((i >> 1) & 1);           // tile rows of matrix rows i and i + 8
    const bool edge = rows < kStageRows || row0 + kStageRows > limit_min;
    if (++steps == kCentre) {
      steps = 0;
      centre(lane);
    }

    // S^T = K Q^T, one accumulator per group, then scale and zero
    float s[kStageTiles][4];
#pragma unroll
    for (int b = 0; b < kStageTiles; ++b) {
      const uint8_t* tile = tp + b * kTileBytes;
      uint32_t kc[2][X];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t* src = reinterpret_cast<const uint32_t*>(tile + tile_k_row(D, ri + 8 * r)) + j * X;
        if constexpr (X == 4) {
          const uint4 v = *reinterpret_cast<const uint4*>(src);
          kc[r][0] = v.x; kc[r][1] = v.y; kc[r][2] = v.z; kc[r][3] = v.w;
        } else {
          const uint2 v = *reinterpret_cast<const uint2*>(src);
          kc[r][0] = v.x; kc[r][1] = v.y;
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < U; ++u) {
          uint32_t lo[4], hi[4];
          codes4(kc[0][g * U + u], lo);
          codes4(kc[1][g * U + u], hi);
          const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
          mma_full(c, a0, qf[g * U + u][0], qf[g * U + u][1]);
          mma_full(c, a1, qf[g * U + u][2], qf[g * U + u][3]);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const uint32_t w = *reinterpret_cast<const uint32_t*>(tile + tile_k_word(D, G, ri + 8 * r, g));
          const float scale = __uint_as_float(w << 16), zero = __uint_as_float(w & 0xffff0000u);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float zq = g == 0 ? zero * qsum[g][x] : fmaf(zero, qsum[g][x], s[b][2 * r + x]);
            s[b][2 * r + x] = fmaf(scale, c[2 * r + x], zq);
          }
        }
      }
    }
    uint32_t vw[kStageTiles][G][2];              // V's (scale, zero) of rows i, i + 8
#pragma unroll
    for (int b = 0; b < kStageTiles; ++b)
#pragma unroll
      for (int g = 0; g < G; ++g)
#pragma unroll
        for (int r = 0; r < 2; ++r)
          vw[b][g][r] = *reinterpret_cast<const uint32_t*>(tp + b * kTileBytes + tile_v_word(D, G, ri + 8 * r, g));
    if (edge) {
      // Rows behind the end hold anything, rows that a token does not see may hold NaN: replaced, not multiplied away.
      // (A NaN scale that some columns see goes into their zero sums by hand.)
      asm volatile("");                          // a branch: as selects this would cost every stage
#pragma unroll
      for (int b = 0; b < kStageTiles; ++b)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int row = b * kPageTile + ri + 8 * r;
#pragma unroll
          for (int x = 0; x < 2; ++x)
            s[b][2 * r + x] = row >= rows || row0 + row >= limit[x] ? -INFINITY : s[b][2 * r + x] * up[x];
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const float scale = __uint_as_float(vw[b][g][r] << 16);
            if (row < rows && scale != scale)
#pragma unroll
              for (int x = 0; x < 2; ++x)
                if (row0 + row < limit[x]) zacc[g][x] = scale;
            if (row >= rows || scale != scale) vw[b][g][r] = 0;
          }
        }
    }
    // Rare work, found by one vote: a score far above the maximum, a scale that P's f16 range no longer covers, or only scales so
    // far below that P would lose bits.
    float top = 0.f, low = INFINITY;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float big = __uint_as_float(vw[0][g][0] << 16);
#pragma unroll
      for (int y = 1; y < 2 * kStageTiles; ++y) big = fmaxf(big, __uint_as_float(vw[y >> 1][g][y & 1] << 16));
      big *= norm[g];
      top = fmaxf(top, big);
      low = fminf(low, big);
    }
    float ms[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) ms[x] = fmaxf(fmaxf(s[0][x], s[0][2 + x]), fmaxf(s[1][x], s[1][2 + x]));
    if (__any_sync(0xffffffffu, ms[0] > raise[0] || ms[1] > raise[1] || top > kScaleTop) ||
        __all_sync(0xffffffffu, low < kScaleLow)) {
#pragma unroll
      for (int g = 0; g < G; ++g) {
        float big = 0.f;
#pragma unroll
        for (int y = 0; y < 2 * kStageTiles; ++y) big = fmaxf(big, __uint_as_float(vw[y >> 1][g][y & 1] << 16));
        const float x = big * norm[g];
        if (__any_sync(0xffffffffu, x > kScaleTop) || __all_sync(0xffffffffu, !(x >= kScaleLow))) renorm(g, big);
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float mx = ms[x];
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float m_old = top_score(x), m_new = fmaxf(m_old, mx);
        const float corr = m_new == -INFINITY ? 1.f : ex2((m_old - m_new) * sc2[x]);
        ref[x] = m_new == -INFINITY ? 0.f : m_new;
        // (rounded down: where the next number is more than kLazy above, it raises the maximum)
        raise[x] = m_new == -INFINITY ? -INFINITY : __fadd_rd(m_new, kLazy / sc2[x]);
        l[x] *= corr;
#pragma unroll
        for (int g = 0; g < G; ++g) zacc[g][x] *= corr;
#pragma unroll
        for (int y = 0; y < X; ++y) {
          o[y][0][x] *= corr; o[y][0][2 + x] *= corr;
          o[y][1][x] *= corr; o[y][1][2 + x] *= corr;
        }
      }
    }

    // P, and O^T += V^T P^T with the group's scale multiplied into P
#pragma unroll
    for (int b = 0; b < kStageTiles; ++b) {
      const uint8_t* tile = tp + b * kTileBytes;
      // (the difference first: a product that is rounded in one place and not in the other is off by 2^-24 of a score, which
      // for scores beyond 2^30 is beyond an exponential's range)
      float p[4];
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        p[x] = ex2((s[b][x] - ref[x]) * sc2[x]);
        p[2 + x] = ex2((s[b][2 + x] - ref[x]) * sc2[x]);
        l[x] += p[x] + p[2 + x];
      }
      uint32_t vc[4][X / 2];                     // rows of matrix rows 2 j, 2 j + 1, 2 j + 8, 2 j + 9
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = ((2 * j + (r & 1)) ^ (j & 1)) + 8 * (r >> 1);
        const uint32_t* src = reinterpret_cast<const uint32_t*>(tile + tile_v_row(D, row)) + i * (X / 2);
        if constexpr (X == 4) {
          const uint2 v = *reinterpret_cast<const uint2*>(src);
          vc[r][0] = v.x; vc[r][1] = v.y;
        } else {
          vc[r][0] = *src;
        }
      }
#pragma unroll
      for (int g = 0; g < G; ++g) {
        uint32_t pb[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float scale = __uint_as_float(vw[b][g][r] << 16);
          const float zero = __uint_as_float(vw[b][g][r] & 0xffff0000u), f = scale * norm[g];
#pragma unroll
          for (int x = 0; x < 2; ++x) zacc[g][x] = fmaf(p[2 * r + x], zero, zacc[g][x]);
          pb[r] = transpose8x8(pack_f16(p[2 * r] * f, p[2 * r + 1] * f));
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int x = g * U + u;
          const uint32_t sel = (x & 1) ? 0x7632 : 0x5410;
          uint32_t v0[4], v1[4];
          codes4(__byte_perm(vc[0][x >> 1], vc[1][x >> 1], sel), v0);
          codes4(__byte_perm(vc[2][x >> 1], vc[3][x >> 1], sel), v1);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t av[4] = {v0[2 * y], v0[2 * y + 1], v1[2 * y], v1[2 * y + 1]};
            mma_full(o[x][y], av, pb[0], pb[1]);
          }
        }
      }
    }
  }

  // sums over the lanes that share a column; o without its factor, with its zeros
  __device__ __forceinline__ void end() {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], b);
#pragma unroll
        for (int g = 0; g < G; ++g) zacc[g][x] += __shfl_xor_sync(0xffffffffu, zacc[g][x], b);
      }
#pragma unroll
      for (int y = 0; y < X; ++y) {
        const float up = norm[y / U] == 0.f ? 0.f : 1.f / norm[y / U];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          o[y][k][x] = fmaf(o[y][k][x] * 0x1p24f, up, zacc[y / U][x]);
          o[y][k][2 + x] = fmaf(o[y][k][2 + x] * 0x1p20f, up, zacc[y / U][x]);
        }
      }
    }
  }
  __device__ __forceinline__ void keep(float* state, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float* st = state + (2 * j + x) * (D + 2);
#pragma unroll
      for (int y = 0; y < X; ++y) {
        const int d = 4 * v_slot_half(D, GROUP, i * X + y);
#pragma unroll
        for (int k = 0; k < 4; ++k) st[d + k] = o[y][k >> 1][2 * (k & 1) + x];
      }
      if (i == 0) { st[D] = top_score(x) * sc2[x]; st[D + 1] = l[x]; }
    }
  }
  __device__ __forceinline__ void write(const PagesAttnArgs& a, const Place& c, int cols_total, int lane) const {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int col = c.cg * COLS + 2 * j + x;
      if (col >= cols_total) break;
      const OutPlace at(a, c.entry, c.h, col);
      const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];
#pragma unroll
      for (int y = 0; y < X; ++y)
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.out) + at.out + 4 * v_slot_half(D, GROUP, i * X + y)) =
            make_uint2(pack_bf16(o[y][0][x] * inv, o[y][0][2 + x] * inv), pack_bf16(o[y][1][x] * inv, o[y][1][2 + x] * inv));
      if (i == 0 && a.lse) a.lse[at.lse] = lse_of(top_score(x) * sc2[x], l[x]);
    }
  }
};

__device__ __forceinline__ bool try_wait_once(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred P;\n\tmbarrier.try_wait.parity.shared::cta.b64 P, [%1], %2;\n\tselp.b32 %0, 1, 0, P;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ bool test_wait_once(uint32_t bar, uint32_t parity) {        // does not suspend
  uint32_t done;
  asm volatile("{\n\t.reg .pred P;\n\tmbarrier.test_wait.parity.shared::cta.b64 P, [%1], %2;\n\tselp.b32 %0, 1, 0, P;\n\t}"
               : "=r"(done) : "r"(bar), "r"(parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ void arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
// one copy global -> shared that completes the phase of `bar`
__device__ __forceinline__ void tile_load(uint32_t dst, const uint8_t* src, uint32_t bytes, uint32_t bar) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(dst), "l"(reinterpret_cast<uint64_t>(src)), "r"(bytes), "r"(bar) : "memory");
}

// Merge of the states [x][D + 2] that the bits of `members` number (`at` gives a state's address), columns x < ncols: the o-th
// four dimensions of them. f gets (column, first dimension, four sums, maximum, denominator).
template <int D, class At, class F>
__device__ __forceinline__ void merge_states(uint32_t members, int ncols, int o, At at, F f) {
  if (o < ncols * (D / 4)) {
    const int x = o / (D / 4), d = o % (D / 4) * 4;
    float M = -INFINITY;
    for (uint32_t b = members; b; b &= b - 1) M = fmaxf(M, at(__ffs(b) - 1)[x * (D + 2) + D]);
    const float ref = M == -INFINITY ? 0.f : M;
    float num[4] = {0.f, 0.f, 0.f, 0.f}, den = 0.f;
    for (uint32_t b = members; b; b &= b - 1) {
      const float* st = at(__ffs(b) - 1) + x * (D + 2);
      const float w = ex2(st[D] - ref);
      const float2 u = *reinterpret_cast<const float2*>(st + d), v = *reinterpret_cast<const float2*>(st + d + 2);
      num[0] = fmaf(w, u.x, num[0]); num[1] = fmaf(w, u.y, num[1]);
      num[2] = fmaf(w, v.x, num[2]); num[3] = fmaf(w, v.y, num[3]);
      den = fmaf(w, st[D + 1], den);
    }
    f(x, d, num, M, den);
  }
}

template <class T>
__device__ __forceinline__ void write4(const PagesAttnArgs& a, const Piece& pc, int col, int d, const float* num, float M,
                                       float den, bool stats) {
  const OutPlace at(a, pc.entry, pc.h, col);
  const float inv = den == 0.f ? 0.f : 1.f / den;
  T* dst = static_cast<T*>(a.out) + at.out + d;
#pragma unroll
  for (int k = 0; k < 4; ++k) dst[k] = from_f<T>(num[k] * inv);
  if (stats && a.lse) a.lse[at.lse] = lse_of(M, den);
}

template <class Body>
__global__ void __launch_bounds__((Body::kWarps + 1) * 32, Body::kBlocks) attn_kernel(PagesAttnArgs a, int cgs) {
  using T = typename Body::Type;
  using L = Layout<Body>;
  constexpr int D = Body::kDim, COLS = Body::COLS, S = Body::kStages, TB = Body::kTileBytes;
  constexpr int kWarps = Body::kWarps, kThreads = (kWarps + 1) * 32;
  static_assert(kWarps <= kMaxWarps, "tables in Sched");
  extern __shared__ __align__(128) uint8_t base[];       // (never cast through an integer: loads from it must stay shared loads)
  __shared__ Sched sh;
  __shared__ uint64_t full[kWarps][S], empty[kWarps][S];
  __shared__ int loaded[kWarps][S];              // a stage's tiles, 0 if they lie in no valid page
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  // where a warp's states lie: place 0 behind the ring and the queries, place 1 in the ring
  auto state_of = [&](int w, int place) {
    return reinterpret_cast<float*>(base + w * L::warp_bytes + (place ? 0 : L::ring + Body::kQueryFloats * 4));
  };
  const int cols_total = a.T * a.rep;

  if (warp < kWarps && lane == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(&full[warp][s], 1); mbar_init(&empty[warp][s], 1); }
    sh.piece[warp][0].valid = sh.piece[warp][1].valid = 0;
  }
  if (t == 0) { sh.abort_flag = 0; sh.open_c1[0] = sh.open_c1[1] = -1; }
  fence_barrier_init();

  // ---- this CTA's share: total units, units per warp, and the entries in which the warps' ranges start
  long long total = 0, part, u_mine = 0, lo_mine = 0;
  int l_mine = 0, len_mine = 0;
  for (int i0 = 0; i0 < a.n; i0 += kThreads) {
    const int i = i0 + t;
    u_mine = i < a.n ? entry_units(a, i, cgs, &l_mine, &len_mine) : 0;
    if (blockIdx.x == 0 && i < a.n && u_mine == 0) record(a.p.status, PYR_ERR_INVALID);
    lo_mine = block_scan<kWarps + 1>(u_mine, sh.sums, &part);
    total += part;
  }
  // With no more (entry, head, column group)s than CTAs, and none long, each CTA takes one: no state crosses CTAs then, which
  // would cost more than the shorter way to the end saves (a step in a graph, us, even shares -> one a CTA; heads of queries
  // and of keys: 1 list x 385 rows, 32/32: 13.8 -> 9.8; 4 x 700, 32/32: 15.2 -> 10.9; 16 x 1300, 64/8: 19.3 -> 14.9; but
  // 1 x 2500, 32/32, 14 tiles a warp: 16.4 -> 18.2).
  long long cta_u = 0, cta_units = 0;
  bool whole_ones = false;
  if (a.n <= kThreads) {
    const bool there = u_mine > 0;
    const bool any_long = __syncthreads_or(there && attn_tiles(len_mine) > kCtaTiles * kWarps);
    const int per_entry = a.p.Hkv * cgs;
    const long long all = (long long)__syncthreads_count(there) * per_entry;
    whole_ones = !any_long && all <= gridDim.x;
    if (whole_ones) {
      if (blockIdx.x >= all) return;             // the whole CTA: nothing is in flight
      const int e = blockIdx.x / per_entry;
      const long long order = block_scan<kWarps + 1>(there, sh.sums, &part);
      if (there && order == e) {
        const int tiles = (int)attn_tiles(len_mine);
        sh.share_u = lo_mine + (long long)(blockIdx.x - e * per_entry) * (tiles + kSegmentUnits) + kSegmentUnits;
        sh.share_units = tiles;
        for (int w = 0; w < kWarps; ++w) { sh.entry[w] = t; sh.first_unit[w] = lo_mine; sh.list[w] = l_mine; sh.len[w] = len_mine; }
      }
      __syncthreads();
      cta_u = sh.share_u;
      cta_units = sh.share_units;
    }
  }
  if (!whole_ones) {
    const long long q = attn_share(total, (long long)gridDim.x * kWarps, kMinUnits);
    if (q < 0) {                                 // (in every CTA)
      if (blockIdx.x == 0 && t == 0) record(a.p.status, PYR_ERR_UNSUPPORTED);
      return;
    }
    cta_units = q * kWarps;
    cta_u = blockIdx.x * cta_units;
    if (cta_u >= total) return;                  // the whole CTA: nothing is in flight
    long long run = 0;
    for (int i0 = 0; i0 < a.n && run < cta_u + cta_units; i0 += kThreads) {
      const int i = i0 + t;
      long long u = u_mine, lo = lo_mine;
      if (a.n > kThreads) {
        u = i < a.n ? entry_units(a, i, cgs, &l_mine, &len_mine) : 0;
        lo = run + block_scan<kWarps + 1>(u, sh.sums, &part);
      }
      for (int w = 0; w < kWarps; ++w) {
        const long long s = cta_u + cta_units * w / kWarps;
        if (s >= lo && s < lo + u) { sh.entry[w] = i; sh.first_unit[w] = lo; sh.list[w] = l_mine; sh.len[w] = len_mine; }
      }
      run += part;
    }
    __syncthreads();
  }

  const int w_of = warp < kWarps ? warp : lane;          // the warp whose range this thread works on or loads for
  const long long u_warp = cta_u + cta_units * min(w_of, kWarps) / kWarps;
  const int mine = w_of < kWarps ? (int)max(0LL, min(cta_u + cta_units * (w_of + 1) / kWarps, total) - u_warp) : 0;    // its units

  if (warp == kWarps) {
    // ------------------------------------------------------------ loaders: lane w for warp w
    Place ld{};
    int slot = 0, skip = 0, in_page = 0, in_stage = 0, issued = 0, left = mine;
    int page_first = -1, page_next = -1;         // page ids as the table has them: of slot 0, and of slot `slot`
    const int tpp = a.p.tiles_per_page, head_bytes = tpp * TB;
    const uint8_t* src = nullptr;
    uint32_t parity = 1;                         // of the wait for an empty stage: the first ones are
    const int32_t* row = a.p.table;
    if (mine > 0) {
      ld.start(a, cgs, sh.entry[w_of], sh.list[w_of], sh.len[w_of], u_warp - sh.first_unit[w_of], &left);
      slot = ld.t / tpp;
      skip = ld.t - slot * tpp;
      row = a.p.table + (size_t)ld.list * a.p.max_pages;
      page_first = row[0];
      page_next = row[slot];
    }
    const uint32_t full0 = smem_u32(&full[w_of < kWarps ? w_of : 0][0]), empty0 = smem_u32(&empty[w_of < kWarps ? w_of : 0][0]);
    const uint32_t ring0 = smem_u32(base) + (w_of < kWarps ? w_of : 0) * L::warp_bytes;
    volatile int* abort_flag = &sh.abort_flag;
    for (uint32_t idle = 0; __any_sync(0xffffffffu, ld.t < ld.t1 || left > 0);) {
      if (ld.t == ld.t1 && left > 0) {           // on to the next (entry, head, column group)
        if (ld.next(a, cgs, &left)) {
          row = a.p.table + (size_t)ld.list * a.p.max_pages;
          page_first = row[0];
        }
        slot = 0;
        in_page = 0;
        page_next = page_first;
      }
      const bool go = ld.t < ld.t1 && test_wait_once(empty0 + 8 * in_stage, parity);
      if (go) {
        if (in_page == 0) {
          src = nullptr;
          if (ld.len > 0) {
            if (page_next >= 0 && page_next < a.p.n_pages)
              src = a.p.pool + ((size_t)page_next * a.p.Hkv + ld.h) * head_bytes + skip * TB;
            else
              record(a.p.status, PYR_ERR_INVALID);
          }
          in_page = min(tpp - skip, ld.t1 - ld.t);
          skip = 0;
          // the id after this one is fetched now and looked at when its page is opened
          if (++slot < a.p.max_pages) page_next = row[slot];
        }
        const int n = min(in_page, kStageTiles);
        loaded[w_of][in_stage] = src ? n : -n;
        if (src) {
          tile_load(ring0 + in_stage * (kStageTiles * TB), src, n * TB, full0 + 8 * in_stage);
          src += n * TB;
        } else {
          arrive(full0 + 8 * in_stage);
        }
        if (++in_stage == S) { in_stage = 0; parity ^= 1; }
        ++issued;
        in_page -= n;
        ld.t += n;
      }
      if (__any_sync(0xffffffffu, go)) {
        idle = 0;
      } else if (++idle > kSpinLimit || *abort_flag) {
        if (lane == 0 && !*abort_flag) { *abort_flag = 1; record(a.p.status, PYR_ERR_TIMEOUT); }
        break;
      }
    }
    __syncwarp();
    if (*abort_flag && w_of < kWarps) {
      // nobody consumes any more: the copies in flight must land before the CTA gives its shared memory back
      volatile int none = 0;
      for (int u = max(0, issued - S); u < issued; ++u)
        mbar_wait_limit(&full[w_of][u % S], (uint32_t)(u / S) & 1, kSpinLimit, &none, nullptr, 0);
    }
  } else if (mine > 0) {
    // ------------------------------------------------------------ consumers
    Place cu{};
    int stage = 0, left = mine;
    cu.start(a, cgs, sh.entry[warp], sh.list[warp], sh.len[warp], u_warp - sh.first_unit[warp], &left);
    uint8_t* ring = base + warp * L::warp_bytes;
    float* qs = reinterpret_cast<float*>(ring + L::ring);
    const uint32_t full0 = smem_u32(&full[warp][0]), empty0 = smem_u32(&empty[warp][0]);
    Body body;
    bool ok = true;
    uint32_t parity = 0;
    while (true) {
      // ---- a segment: the warp's tiles of one (entry, head, column group)
      const int t0 = cu.t, t1 = cu.t1;
      if (t0 == t1) {                            // only units without a tile
        if (left == 0) break;
        cu.next(a, cgs, &left);
        continue;
      }
      body.begin(a, cu, cols_total, qs, lane);
#pragma unroll 1
      for (int tt = t0; tt < t1 && ok;) {
        if (!__all_sync(0xffffffffu, try_wait_once(full0 + 8 * stage, parity))) {
          ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][stage], parity, &sh.abort_flag, a.p.status, PYR_ERR_TIMEOUT));
          if (!ok) break;        // the remaining work is only walked through, so that no other CTA waits for this one's share
        }
        const int n = loaded[warp][stage];
        if (n > 0)
          body.stage(a, ring + stage * (kStageTiles * TB), tt * kPageTile, min(cu.len - tt * kPageTile, n * kPageTile), qs, lane);
        tt += n < 0 ? -n : n;
        __syncwarp();
        if (lane == 0) arrive(empty0 + 8 * stage);
        if (++stage == S) { stage = 0; parity ^= 1; }
      }
      const bool begins = t0 == 0, ends = t1 == cu.tiles;
      body.end();
      if (begins && ends) {
        body.write(a, cu, cols_total, lane);
      } else {
        // a state that began before this warp's range waits in place 0, one that goes on behind it (the last) in place 1
        const int place = begins ? 1 : 0;
        body.keep(state_of(warp, place), lane);
        if (lane == 0) {
          Piece& pc = sh.piece[warp][place];
          pc.u0 = u_warp + (mine - left) - t1;    // (the warp's units up to here end with tile t1 - 1)
          pc.u1 = pc.u0 + cu.tiles;
          pc.entry = cu.entry; pc.h = cu.h; pc.cg = cu.cg;
          pc.begins = begins; pc.ends = ends; pc.valid = 1;
        }
      }
      if (left == 0) break;
      cu.next(a, cgs, &left);
    }
  }

  // ---- merge the CTA's partial states: runs of consecutive ones of the same (entry, head, column group), a warp a run
  __syncthreads();
  static_assert(kWarps * 2 <= 32, "a lane a piece");
  const bool there = lane < kWarps * 2 && sh.piece[lane >> 1][lane & 1].valid;
  uint32_t pieces = __ballot_sync(0xffffffffu, there);
  const uint32_t ending = __ballot_sync(0xffffffffu, there && sh.piece[lane >> 1][lane & 1].ends);
  for (int r = 0; pieces;) {
    // the run: from the first piece left to the next one that ends
    const int f = __ffs(pieces) - 1;
    const uint32_t from = ending >> f << f, upto = from ? (from & -from) * 2 - 1 : 0xffffffffu;
    const uint32_t members = (pieces & upto) >> f;                // bit k: piece f + k
    const bool ends = from != 0;
    pieces &= ~upto;
    const Piece& pc = sh.piece[f >> 1][f & 1];
    // (32 times four dimensions at a time, dealt to the warps run by run)
    const bool whole = pc.begins && ends;
    const int place = pc.begins ? 1 : 0;
    const int ncols = min(COLS, cols_total - pc.cg * COLS);
    auto at = [&](int k) { return (const float*)state_of((f + k) >> 1, (f + k) & 1); };
    float* dst = a.partial + ((size_t)blockIdx.x * 2 + place) * (kAttnCols * (D + 2));
    for (int o = 0; o < ncols * (D / 4); o += 32, r = r == kWarps ? 0 : r + 1) {
      if (r != warp) continue;
      if (whole)
        merge_states<D>(members, ncols, o + lane, at, [&](int x, int d, const float* num, float M, float den) {
          write4<T>(a, pc, pc.cg * COLS + x, d, num, M, den, d == 0);
        });
      else
        merge_states<D>(members, ncols, o + lane, at, [&](int x, int d, const float* num, float M, float den) {
          __stcg(reinterpret_cast<float2*>(dst + x * (D + 2) + d), make_float2(num[0], num[1]));
          __stcg(reinterpret_cast<float2*>(dst + x * (D + 2) + d + 2), make_float2(num[2], num[3]));
          if (d == 0) __stcg(reinterpret_cast<float2*>(dst + x * (D + 2) + D), make_float2(M, den));
        });
    }
    if (!whole && t == 0) {
      sh.open_piece[place] = f;
      sh.open_c1[place] = (int)(pc.u0 / cta_units);
      sh.open_count[place] = (int)((pc.u1 - 1) / cta_units) - (int)(pc.u0 / cta_units) + 1;
    }
    if (!whole) __threadfence();                 // (what another CTA will read)
  }
  __syncthreads();
  if (sh.open_c1[0] < 0 && sh.open_c1[1] < 0) return;     // uniform over the CTA
  if (t < 2) {
    sh.last[t] = 0;
    if (sh.open_c1[t] >= 0) sh.last[t] = atomicAdd(&a.arrived[sh.open_c1[t]], 1) == sh.open_count[t] - 1;
    __threadfence();
  }
  __syncthreads();
  for (int place = 0; place < 2; ++place) {
    if (sh.open_c1[place] < 0 || !sh.last[place]) continue;
    const Piece& pc = sh.piece[sh.open_piece[place] >> 1][sh.open_piece[place] & 1];
    const int c1 = sh.open_c1[place], cn = sh.open_count[place];
    const int ncols = min(COLS, cols_total - pc.cg * COLS);
    // the first CTA holds the beginning (place 1), the others go on with it (place 0)
    const float* src = a.partial + (size_t)c1 * 2 * (kAttnCols * (D + 2));
    const size_t step = 2 * (size_t)(kAttnCols * (D + 2)), second = kAttnCols * (D + 2);
    constexpr int kFew = 8;
    if (cn <= kFew) {                            // everything a thread needs in one round of loads
      for (int o = t; o < ncols * (D / 4); o += kThreads) {
        const int x = o / (D / 4), d = o % (D / 4) * 4;
        float2 ml[kFew], u[kFew], v[kFew];
#pragma unroll
        for (int k = 0; k < kFew; ++k)
          if (k < cn) {
            const float* st = src + k * step + (k == 0 ? second : 0) + x * (D + 2);
            ml[k] = __ldcg(reinterpret_cast<const float2*>(st + D));
            u[k] = __ldcg(reinterpret_cast<const float2*>(st + d));
            v[k] = __ldcg(reinterpret_cast<const float2*>(st + d + 2));
          }
        float M = -INFINITY, num[4] = {0.f, 0.f, 0.f, 0.f}, den = 0.f;
#pragma unroll
        for (int k = 0; k < kFew; ++k)
          if (k < cn) M = fmaxf(M, ml[k].x);
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int k = 0; k < kFew; ++k)
          if (k < cn) {
            const float w = ex2(ml[k].x - ref);
            num[0] = fmaf(w, u[k].x, num[0]); num[1] = fmaf(w, u[k].y, num[1]);
            num[2] = fmaf(w, v[k].x, num[2]); num[3] = fmaf(w, v[k].y, num[3]);
            den = fmaf(w, ml[k].y, den);
          }
        write4<T>(a, pc, pc.cg * COLS + x, d, num, M, den, d == 0);
      }
      if (t == 0) a.arrived[c1] = 0;
      continue;
    }
    // a column's maxima and sums are 2 cn numbers far apart: a warp a column, so that they are fetched together
    float* weight = reinterpret_cast<float*>(base);           // [cn][COLS], where the rings were
    __syncthreads();
    for (int x = warp; x < ncols; x += kWarps + 1) {
      float M = -INFINITY;
      for (int k = lane; k < cn; k += 32) M = fmaxf(M, __ldcg(src + k * step + (k == 0 ? second : 0) + x * (D + 2) + D));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float ref = M == -INFINITY ? 0.f : M;
      float den = 0.f;
      for (int k = lane; k < cn; k += 32) {
        const float* st = src + k * step + (k == 0 ? second : 0) + x * (D + 2) + D;
        const float w = ex2(__ldcg(st) - ref);
        weight[k * COLS + x] = w;
        den = fmaf(w, __ldcg(st + 1), den);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) den += __shfl_xor_sync(0xffffffffu, den, o);
      if (lane == 0) {
        sh.den[x] = den;
        if (a.lse) a.lse[OutPlace(a, pc.entry, pc.h, pc.cg * COLS + x).lse] = lse_of(M, den);
      }
    }
    __syncthreads();
    static_assert(D % 4 == 0, "four dimensions a thread");
    for (int o = t; o < ncols * (D / 4); o += kThreads) {
      const int x = o / (D / 4), d = o % (D / 4) * 4;
      float num[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
      for (int k = 0; k < cn; ++k) {
        const float w = weight[k * COLS + x];
        const float2* st = reinterpret_cast<const float2*>(src + k * step + (k == 0 ? second : 0) + x * (D + 2) + d);
        const float2 u = __ldcg(st), v = __ldcg(st + 1);
        num[0] = fmaf(w, u.x, num[0]); num[1] = fmaf(w, u.y, num[1]);
        num[2] = fmaf(w, v.x, num[2]); num[3] = fmaf(w, v.y, num[3]);
      }
      write4<T>(a, pc, pc.cg * COLS + x, d, num, 0.f, sh.den[x], false);
    }
    if (t == 0) a.arrived[c1] = 0;                         // as the next call expects it
  }
}

template <class Body>
cudaError_t run_attn(const PagesAttnArgs& a, cudaStream_t s) {
  const int cgs = (a.T * a.rep + Body::COLS - 1) / Body::COLS;
  constexpr int smem = Layout<Body>::total;
  cudaError_t e = allow_shared<attn_kernel<Body>>(smem);
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int at_once = Body::kBlocks * sms < kAttnMaxCtas ? Body::kBlocks * sms : kAttnMaxCtas;
  const int ctas = attn_ctas(a.p, a.n, cgs, Body::kWarps * kMinUnits, at_once);
  attn_kernel<Body><<<(unsigned)ctas, (Body::kWarps + 1) * 32, smem, s>>>(a, cgs);
  return cudaGetLastError();
}

template <int D, int GROUP>
cudaError_t pick(const PagesAttnArgs& a, cudaStream_t s) {
  if (a.dtype != PYR_F32) return run_attn<MmaBody<D, GROUP>>(a, s);
  // fp32 pays for every column whether it is there or not: 16 lists of 1088 rows, 32 heads, one column: 207 us with four, 92 with
  // one; two: 118 and 57. Where lists cannot be long and there are SMs for it, columns go to CTAs of their own: the list is
  // read once for each then, but a step, of which a warp has one or two, is that much shorter (7 lists x 4 heads, 272 rows,
  // 4 columns: 13.8 us with four a CTA, 8.6 with one; 128 dimensions: 26.8 and 13.4).
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const long long cols = (long long)a.T * a.rep, pairs = (long long)a.n * a.p.Hkv;
  const bool small = attn_tiles(a.p.max_pages * a.p.page_rows) <= kCtaTiles * CoreBody<D, GROUP, 4>::kWarps;
  if (cols == 1 || (small && pairs * cols <= sms)) return run_attn<CoreBody<D, GROUP, 1>>(a, s);
  if (cols == 2 || (small && pairs * ((cols + 1) / 2) <= sms)) return run_attn<CoreBody<D, GROUP, 2>>(a, s);
  return run_attn<CoreBody<D, GROUP, 4>>(a, s);
}

}  // namespace

cudaError_t launch_pages_attn(const PagesAttnArgs& a, int* launches, cudaStream_t s) {
  const cudaError_t e = a.p.D == 128 ? (a.p.group == 32 ? pick<128, 32>(a, s) : a.p.group == 64 ? pick<128, 64>(a, s) : pick<128, 128>(a, s))
                                     : (a.p.group == 32 ? pick<64, 32>(a, s) : pick<64, 64>(a, s));
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

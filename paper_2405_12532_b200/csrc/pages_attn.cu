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
// A warp loads its tiles itself: lane 0 keeps a ring of bulk copies (a tile is one contiguous copy) in flight.
#include <cuda_bf16.h>

#include "pyr_internal.h"
#include "tc_common.cuh"

namespace pyr {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kStages = 4;               // tiles in a warp's ring
constexpr int kMinUnits = 4;             // a warp's share is at least this many tiles: merging costs more than they do

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }

template <class T> __device__ __forceinline__ float to_f(T x);
template <> __device__ __forceinline__ float to_f<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <class T> __device__ __forceinline__ T from_f(float x);
template <> __device__ __forceinline__ float from_f<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// A partial state's place in the call.
struct Piece {
  long long u0, u1;      // units of its (entry, head, column group)
  int entry, h, cg;
  int begins, ends;      // whether it holds the first / the last of them
  int valid;
};

struct Sched {
  long long sums[kWarps + 1];
  long long first_unit[kWarps];   // of the entry in which a warp's range starts
  int entry[kWarps];
  int abort_flag;
  int last[2];
  Piece piece[kWarps][2];
};

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
  for (int w = 0; w < kWarps; ++w) {
    if (w < warp) before += warp_sums[w];
    all += warp_sums[w];
  }
  *total = all;
  return before + incl - x;
}

// Units of entry i: 0 if its list id is out of range (the entry is refused).
__device__ __forceinline__ long long entry_units(const PagesAttnArgs& a, int i, int cgs) {
  const int l = pages_list(a.p, a.lists, i);
  return l < 0 ? 0 : (long long)attn_tiles(pages_len(a.p, l)) * a.p.Hkv * cgs;
}

// Position in the numbering of units: an entry, and a tile of one of its heads' column groups.
struct Cursor {
  int entry, l, len, tiles, h, cg, t;
  long long u_entry;                     // first unit of the entry

  __device__ __forceinline__ void open(const PagesAttnArgs& a, int cgs) {
    l = pages_list(a.p, a.lists, entry);
    len = l < 0 ? 0 : pages_len(a.p, l);
    tiles = l < 0 ? 0 : (int)attn_tiles(len);
    (void)cgs;
  }
  __device__ __forceinline__ void start(const PagesAttnArgs& a, int cgs, int e, long long first, long long u) {
    entry = e; u_entry = first;
    open(a, cgs);
    const long long o = u - first;
    t = (int)(o % tiles);
    const long long hc = o / tiles;
    cg = (int)(hc % cgs);
    h = (int)(hc / cgs);
  }
  __device__ __forceinline__ void next_tile(const PagesAttnArgs& a, int cgs) {
    if (++t < tiles) return;
    t = 0;
    if (++cg < cgs) return;
    cg = 0;
    if (++h < a.p.Hkv) return;
    h = 0;
    do {                                 // refused entries have no unit
      u_entry += (long long)tiles * a.p.Hkv * cgs;
      if (++entry >= a.n) { tiles = 1; len = 0; l = -1; return; }
      open(a, cgs);
    } while (tiles == 0);
  }
};

// Writes column c of an entry's head: out = num / den for the D dimensions held by `lane`-strided callers.
template <class T, int D>
__device__ __forceinline__ void write_out(const PagesAttnArgs& a, int entry, int h, int col, int d, float value) {
  const int tok = col / a.rep, head = h * a.rep + col % a.rep;
  static_cast<T*>(a.out)[(int64_t)entry * a.osb + (int64_t)tok * a.ost + (int64_t)head * a.osh + d] = from_f<T>(value);
}
__device__ __forceinline__ void write_lse(const PagesAttnArgs& a, int entry, int h, int col, float m, float den) {
  if (!a.lse) return;
  const int tok = col / a.rep, head = h * a.rep + col % a.rep;
  a.lse[((int64_t)entry * a.Hq + head) * a.T + tok] = den > 0.f ? (m + log2f(den)) * kLn2 : (den == 0.f ? -INFINITY : den);
}

// Shared memory of a CTA: per warp a ring of tiles, the queries of its segment and two states of [cols][D + 2].
template <class Body>
struct Layout {
  static constexpr int state = Body::COLS * (Body::kDim + 2);
  static __host__ __device__ int ring_bytes(int tile_bytes) { return kWarps * kStages * tile_bytes; }
  static __host__ __device__ int total(int tile_bytes) {
    return 128 + ring_bytes(tile_bytes) + kWarps * (Body::kQueryFloats + 2 * state) * 4;
  }
};

// ------------------------------------------------------------------ one warp's tiles, on CUDA cores
// Lane 4 i + j. K: rows i and i + 8, the quarter of the dimensions that chunk j of a stored row holds. V: the eighth of the
// dimensions that chunk i holds, of the rows j, j + 4, j + 8, j + 12.
template <class T, int D, int GROUP>
struct CoreBody {
  using Type = T;
  static constexpr int kDim = D, COLS = 4, kBlocks = 2, kQueryFloats = COLS * D;   // queries lie in shared memory
  static constexpr int G = D / GROUP, U = GROUP / 32, X = D / 32;   // X: words of K / halves of V in a lane's chunk
  float acc[COLS][4 * X];
  float m[COLS], l[COLS], qsum[COLS][G];
  int limit[COLS];

  __device__ __forceinline__ void begin(const PagesAttnArgs& a, const Cursor& c, int cols_total, float* qs, int lane) {
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
      const T* q = static_cast<const T*>(a.q) + (int64_t)c.entry * a.qsb + (int64_t)tok * a.qst + (int64_t)head * a.qsh;
      // queries in the order of the stored codes
      for (int p = lane; p < D; p += 32)
        qs[x * D + p] = x < ncols ? to_f(q[8 * k_slot_word(D, GROUP, p >> 3) + (p & 7)]) : 0.f;
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
        s[rr][x] = r < rows && row0 + r < limit[x] ? s[rr][x] * sc2 : -INFINITY;
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
              if (edge && val != val) {      // a NaN that a column does not see must not reach it through 0 x NaN
#pragma unroll
                for (int x = 0; x < COLS; ++x)
                  if (row0 + r < limit[x]) acc[x][(g * U + u) * 4 + k] = val;
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

  // the state of the warp's segment, in dimension order
  __device__ __forceinline__ void end(float* state, int lane) {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < COLS; ++x) {
#pragma unroll
      for (int o = 4; o < 32; o <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], o);
#pragma unroll
      for (int y = 0; y < 4 * X; ++y) {
        float v = acc[x][y];
        v += __shfl_xor_sync(0xffffffffu, v, 1);
        v += __shfl_xor_sync(0xffffffffu, v, 2);
        if (j == (y & 3)) state[x * (D + 2) + 4 * v_slot_half(D, GROUP, i * X + (y >> 2)) + (y & 3)] = v;
      }
      if (lane == 0) { state[x * (D + 2) + D] = m[x]; state[x * (D + 2) + D + 1] = l[x]; }
    }
    __syncwarp();
  }
};

// ------------------------------------------------------------------ one warp's tiles, on tensor cores (bf16)
// Rows of the cache are the 16 rows of m16n8k16, the (up to 8) query rows its 8 columns: S^T = K Q^T, O^T = V^T P^T. The
// instruction is bound neither way here: what counts is that a register of codes becomes an operand in few steps. Lane
// 4 i + j holds, of K's row i (and i + 8), chunk j: a word's nibbles k and k + 4 are a pair of operands, and since any order
// of the dimensions will do as long as the queries have the same, the words are stored in the order in which lanes take
// them. Of V it holds chunk i of four rows, two rows' halves side by side giving pairs of rows of one dimension.
// (Legacy warp-level MMA: a decode step reads every code once, and tcgen05 would need the codes as 8- or 16-bit
// operands in shared memory first.)
// Row r of the matrices is row r ^ ((r >> 1) & 1) of the tile, which spreads the lanes' shared-memory reads over the banks.
__device__ __forceinline__ void mma_full(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// Four pairs of codes (nibbles k and k + 4 of x) as bf16 pairs, less 8: 0x4300 | n is 128 + n.
__device__ __forceinline__ void centred4(uint32_t x, uint32_t* y) {
  const uint32_t bias = 0x43084308u;             // 136
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t v = ((x >> (4 * k)) & 0x000F000Fu) | 0x43004300u;
    const __nv_bfloat162 d = __hsub2(reinterpret_cast<const __nv_bfloat162&>(v), reinterpret_cast<const __nv_bfloat162&>(bias));
    y[k] = reinterpret_cast<const uint32_t&>(d);
  }
}

template <int D, int GROUP>
struct MmaBody {
  using Type = __nv_bfloat16;
  static constexpr int kDim = D, COLS = 8, kBlocks = 3, kQueryFloats = 0;
  static constexpr int G = D / GROUP, U = GROUP / 32, X = D / 32;
  static constexpr float kLazy = 8.f;            // the maximum is raised once a score is 2^8 above it
  uint32_t qf[X][4];
  float qsum[G][2], o[X][2][4], zacc[G][2], m[2], l[2], raise[2];
  int limit[2], limit_min;

  __device__ __forceinline__ void begin(const PagesAttnArgs& a, const Cursor& c, int cols_total, float*, int lane) {
    const int i = lane >> 2, j = lane & 3, col0 = c.cg * COLS;
    const int col = col0 + i, tok = col / a.rep, head = c.h * a.rep + col % a.rep;
    const uint16_t* q = static_cast<const uint16_t*>(a.q) + (int64_t)c.entry * a.qsb + (int64_t)tok * a.qst + (int64_t)head * a.qsh;
#pragma unroll
    for (int w = 0; w < X; ++w) {
      uint4 r = make_uint4(0, 0, 0, 0);
      if (col < cols_total) r = *reinterpret_cast<const uint4*>(q + 8 * k_slot_word(D, GROUP, j * X + w));
      qf[w][0] = __byte_perm(r.x, r.z, 0x5410); qf[w][1] = __byte_perm(r.x, r.z, 0x7632);
      qf[w][2] = __byte_perm(r.y, r.w, 0x5410); qf[w][3] = __byte_perm(r.y, r.w, 0x7632);
    }
    // sums of the queries over each group, by the instruction itself: every row of a matrix of ones
    const uint32_t ones[4] = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        mma_full(s, ones, qf[g * U + u][0], qf[g * U + u][1]);
        mma_full(s, ones, qf[g * U + u][2], qf[g * U + u][3]);
      }
      qsum[g][0] = s[0]; qsum[g][1] = s[1];
      zacc[g][0] = zacc[g][1] = 0.f;
    }
#pragma unroll
    for (int x = 0; x < X; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) o[x][y][0] = o[x][y][1] = o[x][y][2] = o[x][y][3] = 0.f;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      m[x] = -INFINITY; raise[x] = -INFINITY; l[x] = 0.f;
      limit[x] = c.len - (a.T - 1 - (col0 + 2 * j + x) / a.rep);
    }
    limit_min = c.len - (a.T - 1 - col0 / a.rep);
  }

  __device__ __forceinline__ void tile(const PagesAttnArgs& a, const uint8_t* tp, int row0, int rows, const float*, int lane) {
    const int i = lane >> 2, j = lane & 3;
    const int ri = i ^ ((i >> 1) & 1);           // tile rows of matrix rows i and i + 8
    const float sc2 = a.scale * kLog2e;
    const bool edge = rows < kPageTile || row0 + kPageTile > limit_min;

    // S^T = K Q^T, one accumulator per group, then scale and zero
    uint32_t kc[2][X];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      const uint32_t* src = reinterpret_cast<const uint32_t*>(tp + tile_k_row(D, ri + 8 * r)) + j * X;
      if constexpr (X == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(src);
        kc[r][0] = v.x; kc[r][1] = v.y; kc[r][2] = v.z; kc[r][3] = v.w;
      } else {
        const uint2 v = *reinterpret_cast<const uint2*>(src);
        kc[r][0] = v.x; kc[r][1] = v.y;
      }
    }
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < G; ++g) {
      float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        uint32_t lo[4], hi[4];
        centred4(kc[0][g * U + u], lo);
        centred4(kc[1][g * U + u], hi);
        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
        mma_full(c, a0, qf[g * U + u][0], qf[g * U + u][1]);
        mma_full(c, a1, qf[g * U + u][2], qf[g * U + u][3]);
      }
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(tp + tile_k_word(D, G, ri + 8 * r, g));
        const float scale = __uint_as_float(w << 16), zero = fmaf(8.f, scale, __uint_as_float(w & 0xffff0000u));
#pragma unroll
        for (int x = 0; x < 2; ++x) s[2 * r + x] += fmaf(scale, c[2 * r + x], zero * qsum[g][x]);
      }
    }
    bool seen[4] = {true, true, true, true};
    if (edge) {                                  // rows behind the end hold anything: replaced, not multiplied away
#pragma unroll
      for (int r = 0; r < 2; ++r)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          seen[2 * r + x] = ri + 8 * r < rows && row0 + ri + 8 * r < limit[x];
          if (!seen[2 * r + x]) s[2 * r + x] = -INFINITY;
        }
    }
    if (__any_sync(0xffffffffu, fmaxf(s[0], s[2]) > raise[0] || fmaxf(s[1], s[3]) > raise[1])) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        float mx = fmaxf(s[x], s[2 + x]);
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
        const float m_new = fmaxf(m[x], mx * sc2);
        const float corr = m_new == -INFINITY ? 1.f : ex2(m[x] - m_new);
        m[x] = m_new;
        raise[x] = (m_new + kLazy) / sc2;
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
    float p[4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float ref = m[x] == -INFINITY ? 0.f : m[x];
      p[x] = ex2(fmaf(s[x], sc2, -ref));
      p[2 + x] = ex2(fmaf(s[2 + x], sc2, -ref));
      l[x] += p[x] + p[2 + x];
    }

    // O^T += V^T P^T, the group's scale multiplied into P. P is given as the sum of two bf16 numbers: rounded to one, it
    // would be as far off as the output's own rounding.
    uint32_t vc[4][X / 2];                       // rows of matrix rows 2 j, 2 j + 1, 2 j + 8, 2 j + 9
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int mr = 2 * j + (r & 1), row = (mr ^ ((mr >> 1) & 1)) + 8 * (r >> 1);
      const uint32_t* src = reinterpret_cast<const uint32_t*>(tp + tile_v_row(D, row)) + i * (X / 2);
      if constexpr (X == 4) {
        const uint2 v = *reinterpret_cast<const uint2*>(src);
        vc[r][0] = v.x; vc[r][1] = v.y;
      } else {
        vc[r][0] = *src;
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      uint32_t hi[2], lo[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(tp + tile_v_word(D, G, ri + 8 * r, g));
        const float scale = __uint_as_float(w << 16), zero = fmaf(8.f, scale, __uint_as_float(w & 0xffff0000u));
        float ps[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          ps[x] = seen[2 * r + x] ? p[2 * r + x] * scale : 0.f;
          if (seen[2 * r + x]) zacc[g][x] = fmaf(p[2 * r + x], zero, zacc[g][x]);
        }
        const uint32_t h = pack_bf16(ps[0], ps[1]);
        hi[r] = transpose8x8(h);
        lo[r] = transpose8x8(pack_bf16(ps[0] - __uint_as_float(h << 16), ps[1] - __uint_as_float(h & 0xffff0000u)));
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int x = g * U + u;
        const uint32_t sel = (x & 1) ? 0x7632 : 0x5410;
        uint32_t v0[4], v1[4];
        centred4(__byte_perm(vc[0][x >> 1], vc[1][x >> 1], sel), v0);
        centred4(__byte_perm(vc[2][x >> 1], vc[3][x >> 1], sel), v1);
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const uint32_t av[4] = {v0[2 * y], v0[2 * y + 1], v1[2 * y], v1[2 * y + 1]};
          mma_full(o[x][y], av, hi[0], hi[1]);
          mma_full(o[x][y], av, lo[0], lo[1]);
        }
      }
    }
  }

  __device__ __forceinline__ void end(float* state, int lane) {
    const int i = lane >> 2, j = lane & 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int b = 4; b < 32; b <<= 1) {
        l[x] += __shfl_xor_sync(0xffffffffu, l[x], b);
#pragma unroll
        for (int g = 0; g < G; ++g) zacc[g][x] += __shfl_xor_sync(0xffffffffu, zacc[g][x], b);
      }
      float* st = state + (2 * j + x) * (D + 2);
#pragma unroll
      for (int y = 0; y < X; ++y) {
        const int d = 4 * v_slot_half(D, GROUP, i * X + y);
#pragma unroll
        for (int k = 0; k < 4; ++k) st[d + k] = o[y][k >> 1][2 * (k & 1) + x] + zacc[y / U][x];
      }
      if (i == 0) { st[D] = m[x]; st[D + 1] = l[x]; }
    }
    __syncwarp();
  }
};

template <class Body>
__global__ void __launch_bounds__(kThreads, Body::kBlocks) attn_kernel(PagesAttnArgs a, int cgs) {
  using T = typename Body::Type;
  using L = Layout<Body>;
  constexpr int D = Body::kDim, COLS = Body::COLS;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Sched sh;
  __shared__ uint64_t full[kWarps][kStages];
  __shared__ int absent[kWarps][kStages];       // the stage's tile lies in no valid page
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int tile_bytes = a.p.tile_bytes;
  uint8_t* base = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));
  uint8_t* ring = base + warp * kStages * tile_bytes;
  float* floats = reinterpret_cast<float*>(base + L::ring_bytes(tile_bytes));
  float* qs = floats + warp * Body::kQueryFloats;
  float* states = floats + kWarps * Body::kQueryFloats;    // [warp][2][COLS][D + 2]
  const int cols_total = a.T * a.rep;

  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    sh.piece[warp][0].valid = sh.piece[warp][1].valid = 0;
  }
  if (t == 0) sh.abort_flag = 0;
  fence_barrier_init();

  // ---- this CTA's share: total units, units per warp, and the entries in which the warps' ranges start
  long long total = 0, part;
  for (int i0 = 0; i0 < a.n; i0 += kThreads) {
    const int i = i0 + t;
    const long long u = i < a.n ? entry_units(a, i, cgs) : 0;
    if (blockIdx.x == 0 && i < a.n && u == 0) record(a.p.status, PYR_ERR_INVALID);
    block_scan(u, sh.sums, &part);
    total += part;
  }
  const long long workers = (long long)gridDim.x * kWarps;
  long long q = (total + workers - 1) / workers;
  if (q < kMinUnits) q = kMinUnits;
  const long long cta_units = q * kWarps, cta_u = blockIdx.x * cta_units;
  if (cta_u >= total) return;                    // the whole CTA: nothing is in flight
  long long run = 0;
  for (int i0 = 0; i0 < a.n && run < cta_u + cta_units; i0 += kThreads) {
    const int i = i0 + t;
    const long long u = i < a.n ? entry_units(a, i, cgs) : 0;
    const long long lo = run + block_scan(u, sh.sums, &part);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const long long s = cta_u + w * q;
      if (s >= lo && s < lo + u) { sh.entry[w] = i; sh.first_unit[w] = lo; }
    }
    run += part;
  }
  __syncthreads();

  const long long u_warp = cta_u + warp * q;
  long long left = total - u_warp;               // units of this warp
  if (left > q) left = q;
  if (left < 0) left = 0;
  bool ok = true;

  if (left > 0) {
    Cursor ld, cu;
    ld.start(a, cgs, sh.entry[warp], sh.first_unit[warp], u_warp);
    cu = ld;
    long long to_load = left;
    int win_list = -1, win0 = 0, win = -1;       // 32 page ids of the loader's list, one per lane
    long long issued = 0, used = 0;

    auto issue = [&]() {
      const int stage = (int)(issued % kStages);
      int page = -1;
      const int slot = ld.t / a.p.tiles_per_page;
      if (ld.len > 0) {
        if (win_list != ld.l || slot < win0 || slot >= win0 + 32) {
          win_list = ld.l;
          win0 = slot;
          win = pages_page(a.p, ld.l, (int64_t)win0 + lane);
        }
        page = __shfl_sync(0xffffffffu, win, slot - win0);
      }
      if (lane == 0) {
        absent[warp][stage] = page < 0;
        if (page >= 0) {
          mbar_expect_tx(&full[warp][stage], tile_bytes);
          bulk_load(ring + stage * tile_bytes, a.p.pool + pages_tile(a.p, page, ld.h, ld.t % a.p.tiles_per_page), tile_bytes,
                    &full[warp][stage]);
        } else {
          mbar_arrive(&full[warp][stage]);
          if (ld.len > 0) record(a.p.status, PYR_ERR_INVALID);
        }
      }
      ++issued;
      --to_load;
      if (to_load > 0) ld.next_tile(a, cgs);
    };
    for (int s = 0; s < kStages && to_load > 0; ++s) issue();

    Body body;
    while (left > 0) {
      // ---- a segment: the warp's tiles of one (entry, head, column group)
      const int t0 = cu.t;
      const int t1 = (int)min((long long)cu.tiles, t0 + left);
      body.begin(a, cu, cols_total, qs, lane);
      for (int tt = t0; tt < t1; ++tt) {
        const int stage = (int)(used % kStages);
        if (ok) {
          ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][stage], (uint32_t)(used / kStages) & 1, &sh.abort_flag, a.p.status, PYR_ERR_TIMEOUT));
          if (!ok) {
            // a wait ran out: no more copies, and those in flight must land before the shared memory is given back
            volatile int none = 0;
            for (long long c = used; c < issued; ++c)
              mbar_wait_limit(&full[warp][c % kStages], (uint32_t)(c / kStages) & 1, kSpinLimit, &none, nullptr, 0);
          }
        }
        if (ok) {
          const int rows = absent[warp][stage] ? 0 : min(kPageTile, cu.len - tt * kPageTile);
          if (rows > 0) body.tile(a, ring + stage * tile_bytes, tt * kPageTile, rows, qs, lane);
          __syncwarp();
          ++used;
          if (to_load > 0) issue();
        }
      }
      const bool begins = t0 == 0, ends = t1 == cu.tiles;
      // a state that began before this warp's range waits in place 0, one that goes on behind it in place 1
      float* state = states + (warp * 2 + (begins ? 1 : 0)) * L::state;
      body.end(state, lane);
      const int ncols = min(COLS, cols_total - cu.cg * COLS);
      if (begins && ends) {
        for (int x = 0; x < ncols; ++x) {
          const float den = state[x * (D + 2) + D + 1], m = state[x * (D + 2) + D];
          const float inv = den == 0.f ? 0.f : 1.f / den;
          for (int d = lane; d < D; d += 32) write_out<T, D>(a, cu.entry, cu.h, cu.cg * COLS + x, d, state[x * (D + 2) + d] * inv);
          if (lane == 0) write_lse(a, cu.entry, cu.h, cu.cg * COLS + x, m, den);
        }
        __syncwarp();
      } else if (lane == 0) {
        Piece& pc = sh.piece[warp][begins ? 1 : 0];
        pc.u0 = cu.u_entry + ((long long)cu.h * cgs + cu.cg) * cu.tiles;
        pc.u1 = pc.u0 + cu.tiles;
        pc.entry = cu.entry; pc.h = cu.h; pc.cg = cu.cg;
        pc.begins = begins; pc.ends = ends; pc.valid = 1;
      }
      left -= t1 - t0;
      cu.t = t1 - 1;
      if (left > 0) cu.next_tile(a, cgs);
    }
  }

  // ---- merge the CTA's partial states: runs of consecutive ones of the same (entry, head, column group)
  __syncthreads();
  int slot_c1[2] = {-1, -1}, slot_count[2] = {0, 0};      // what the CTA leaves for others: place 0 / place 1
  Piece left_piece[2];
  for (int f = 0; f < kWarps * 2;) {
    if (!sh.piece[f >> 1][f & 1].valid) { ++f; continue; }
    const Piece pc = sh.piece[f >> 1][f & 1];
    int g = f, n = 0, members[kWarps * 2];
    bool ends = false;
    for (; g < kWarps * 2; ++g) {
      const Piece& o = sh.piece[g >> 1][g & 1];
      if (!o.valid) continue;
      if (o.u0 != pc.u0) break;
      members[n++] = g;
      ends = o.ends;
    }
    const bool whole = pc.begins && ends;
    const int place = pc.begins ? 1 : 0;
    const int ncols = min(COLS, cols_total - pc.cg * COLS);
    for (int o = t; o < ncols * D; o += kThreads) {
      const int x = o / D, d = o % D;
      float M = -INFINITY;
      for (int k = 0; k < n; ++k) M = fmaxf(M, states[members[k] * L::state + x * (D + 2) + D]);
      const float ref = M == -INFINITY ? 0.f : M;
      float num = 0.f, den = 0.f;
      for (int k = 0; k < n; ++k) {
        const float* st = states + members[k] * L::state + x * (D + 2);
        const float w = exp2f(st[D] - ref);
        num = fmaf(w, st[d], num);
        den = fmaf(w, st[D + 1], den);
      }
      if (whole) {
        write_out<T, D>(a, pc.entry, pc.h, pc.cg * COLS + x, d, den == 0.f ? 0.f : num / den);
        if (d == 0) write_lse(a, pc.entry, pc.h, pc.cg * COLS + x, M, den);
      } else {
        float* dst = a.partial + ((size_t)blockIdx.x * 2 + place) * (kAttnCols * (D + 2)) + x * (D + 2);
        __stcg(dst + d, num);
        if (d == 0) { __stcg(dst + D, M); __stcg(dst + D + 1, den); }
      }
    }
    if (!whole) {
      left_piece[place] = pc;
      slot_c1[place] = (int)(pc.u0 / cta_units);
      slot_count[place] = (int)((pc.u1 - 1) / cta_units) - slot_c1[place] + 1;
    }
    f = g;
  }
  if (slot_c1[0] < 0 && slot_c1[1] < 0) return;           // uniform over the CTA
  __threadfence();
  __syncthreads();
  if (t < 2) {
    sh.last[t] = 0;
    if (slot_c1[t] >= 0) sh.last[t] = atomicAdd(&a.arrived[slot_c1[t]], 1) == slot_count[t] - 1;
  }
  __syncthreads();
  __threadfence();
  for (int place = 0; place < 2; ++place) {
    if (slot_c1[place] < 0 || !sh.last[place]) continue;
    const Piece pc = left_piece[place];
    const int c1 = slot_c1[place], cn = slot_count[place];
    const int ncols = min(COLS, cols_total - pc.cg * COLS);
    for (int o = t; o < ncols * D; o += kThreads) {
      const int x = o / D, d = o % D;
      // the first CTA holds the beginning (place 1), the others go on with it (place 0)
      const float* src = a.partial + (size_t)c1 * 2 * (kAttnCols * (D + 2)) + x * (D + 2);
      const size_t step = 2 * (size_t)(kAttnCols * (D + 2)), second = kAttnCols * (D + 2);
      float M = -INFINITY;
      for (int k = 0; k < cn; ++k) M = fmaxf(M, __ldcg(src + k * step + (k == 0 ? second : 0) + D));
      const float ref = M == -INFINITY ? 0.f : M;
      float num = 0.f, den = 0.f;
      for (int k = 0; k < cn; ++k) {
        const float* st = src + k * step + (k == 0 ? second : 0);
        const float w = exp2f(__ldcg(st + D) - ref);
        num = fmaf(w, __ldcg(st + d), num);
        den = fmaf(w, __ldcg(st + D + 1), den);
      }
      write_out<T, D>(a, pc.entry, pc.h, pc.cg * COLS + x, d, den == 0.f ? 0.f : num / den);
      if (d == 0) write_lse(a, pc.entry, pc.h, pc.cg * COLS + x, M, den);
    }
    if (t == 0) a.arrived[c1] = 0;                         // as the next call expects it
  }
}

template <class Body>
cudaError_t run_attn(const PagesAttnArgs& a, cudaStream_t s) {
  const int cgs = (a.T * a.rep + Body::COLS - 1) / Body::COLS;
  const int smem = Layout<Body>::total(a.p.tile_bytes);
  cudaError_t e = cudaFuncSetAttribute(attn_kernel<Body>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  // a grid that the machine holds at once, no larger than the work can be
  const long long most = (long long)a.n * a.p.Hkv * cgs * attn_tiles(a.p.max_pages * a.p.page_rows);
  long long ctas = (most + kWarps * kMinUnits - 1) / (kWarps * kMinUnits);
  if (ctas > (long long)Body::kBlocks * sms) ctas = (long long)Body::kBlocks * sms;
  if (ctas > kAttnMaxCtas) ctas = kAttnMaxCtas;
  attn_kernel<Body><<<(unsigned)ctas, kThreads, smem, s>>>(a, cgs);
  return cudaGetLastError();
}

template <int D, int GROUP>
cudaError_t pick(const PagesAttnArgs& a, cudaStream_t s) {
  return a.dtype == PYR_F32 ? run_attn<CoreBody<float, D, GROUP>>(a, s) : run_attn<MmaBody<D, GROUP>>(a, s);
}

}  // namespace

cudaError_t launch_pages_attn(const PagesAttnArgs& a, int* launches, cudaStream_t s) {
  const cudaError_t e = a.p.D == 128 ? (a.p.group == 32 ? pick<128, 32>(a, s) : a.p.group == 64 ? pick<128, 64>(a, s) : pick<128, 128>(a, s))
                                     : (a.p.group == 32 ? pick<64, 32>(a, s) : pick<64, 64>(a, s));
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

// How attention over a paged cache deals out its work, loads and merges: the kernel that the cache's formats share. A format
// gives the Body: one warp's tiles of one (entry, KV head, column group).
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
//
// Over chosen pages (Body::kSparse) every query token is an entry of its own: entry i is token i % T of list entry i / T, its
// columns are the query heads, and tile t of a head lies in the page slot that the head's list of slots names at t / (tiles of a page).
#pragma once
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
// Body::kSegment: what beginning and ending a (entry, head, column group) costs a warp, in tiles: its queries, a first step that sets the
// maximum and the scales' factors, its sums (4 bits, 64 ragged lists of 32 heads: 102 us with 2, 96 with 3, 92 with 4, 90 with 6 and 8).
// Body::kFew, kAtOnce, kRounds: merges across CTAs. Up to kFew states a thread merges for itself, kAtOnce of them loaded at once; of more, the loops
// over 32 states are unrolled kRounds times. Sums go state by state whatever these are. The code runs once, so its size counts (4 bits, 2 lists
// of 100 k rows, 64/8 heads: 60.2 us with 2 and 1, 60.7 with 4 and 4; the 8-bit form of that 82.3 with 4 and 4, 83.1 with 2 and 1).
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

// The list of entry i (-1: refused), and the rows that it sees: of a list, or of one query token of a list.
template <class Body>
__device__ __forceinline__ void entry_list(const PagesAttnArgs& a, int i, int* list, int* len) {
  if constexpr (Body::kSparse) {
    const int e = i / a.T;
    *list = pages_list(a.p, a.lists, e);
    *len = *list < 0 ? 0 : max(0, pages_len(a.p, *list) - (a.T - 1 - (i - e * a.T)));
  } else {
    *list = pages_list(a.p, a.lists, i);
    *len = *list < 0 ? 0 : pages_len(a.p, *list);
  }
}
// The tiles of an entry of `len` rows, for each head: all of them, or those of as many pages as are chosen (at least one, so that zeros
// get written).
template <class Body>
__device__ __forceinline__ int entry_tiles(const PagesAttnArgs& a, int len) {
  if constexpr (Body::kSparse)
    return min(a.n_slots, max(1, pages_for(a.p, len))) * a.p.tiles_per_page;
  else
    return (int)attn_tiles(len);
}
// Units of entry i: 0 if its list id is out of range (the entry is refused). A (head, column group) has Body::kSegment units
// that stand for no tile before those that do: short lists cost more than their tiles, and a warp's share must say so.
template <class Body>
__device__ __forceinline__ long long entry_units(const PagesAttnArgs& a, int i, int cgs, int* list, int* len) {
  entry_list<Body>(a, i, list, len);
  return *list < 0 ? 0 : (long long)(entry_tiles<Body>(a, *len) + Body::kSegment) * a.p.Hkv * cgs;
}

template <class Body>
__device__ __forceinline__ int entries(const PagesAttnArgs& a) { return Body::kSparse ? a.n * a.T : a.n; }

// The (entry, head, column group) that a warp works on, and the tiles [t, t1) of it that are the warp's.
struct Place {
  int entry, len, tiles, h, cg, t, t1;
  int list;

  template <class Body>
  __device__ __forceinline__ void open(const PagesAttnArgs& a) {       // the entry's list
    entry_list<Body>(a, entry, &list, &len);
    tiles = list < 0 ? 0 : entry_tiles<Body>(a, len);
  }
  // Takes units from `left` on, of which `r` of this (head, column group) lie before the warp's.
  template <class Body>
  __device__ __forceinline__ void take(int r, int* left) {
    const int n = min(*left, tiles + Body::kSegment - r);
    t = max(0, r - Body::kSegment);
    t1 = max(0, r + n - Body::kSegment);
    *left -= n;
  }
  // unit o of entry e, whose list and length are at hand
  template <class Body>
  __device__ __forceinline__ void start(const PagesAttnArgs& a, int cgs, int e, int l, int n, long long o, int* left) {
    entry = e; list = l; len = n;
    tiles = entry_tiles<Body>(a, len);
    const int per = tiles + Body::kSegment;
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
    take<Body>(r, left);
  }
  // The next one. Returns whether its entry is another.
  template <class Body>
  __device__ __forceinline__ bool next(const PagesAttnArgs& a, int cgs, int* left) {
    bool other = false;
    if (++cg >= cgs) {
      cg = 0;
      if (++h >= a.p.Hkv) {
        h = 0;
        other = true;
        do { ++entry; open<Body>(a); } while (list < 0 && entry + 1 < entries<Body>(a));  // refused entries have no unit
      }
    }
    take<Body>(0, left);
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
  __device__ __forceinline__ OutPlace(int64_t out, int64_t lse) : out(out), lse(lse) {}
};
template <class Body>
__device__ __forceinline__ OutPlace out_place(const PagesAttnArgs& a, int entry, int h, int col) {
  if constexpr (!Body::kSparse) return OutPlace(a, entry, h, col);
  const int e = entry / a.T, tok = entry - e * a.T, head = h * a.rep + col;
  return OutPlace((int64_t)e * a.osb + (int64_t)tok * a.ost + (int64_t)head * a.osh, ((int64_t)e * a.Hq + head) * a.T + tok);
}
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

template <class Body>
__device__ __forceinline__ void write4(const PagesAttnArgs& a, const Piece& pc, int col, int d, const float* num, float M,
                                       float den, bool stats) {
  using T = typename Body::Type;
  const OutPlace at = out_place<Body>(a, pc.entry, pc.h, col);
  const float inv = den == 0.f ? 0.f : 1.f / den;
  T* dst = static_cast<T*>(a.out) + at.out + d;
#pragma unroll
  for (int k = 0; k < 4; ++k) dst[k] = from_f<T>(num[k] * inv);
  if (stats && a.lse) a.lse[at.lse] = lse_of(M, den);
}

template <class Body>
__global__ void __launch_bounds__((Body::kWarps + 1) * 32, Body::kBlocks) attn_kernel(PagesAttnArgs a, int cgs) {
  using L = Layout<Body>;
  constexpr int D = Body::kDim, COLS = Body::COLS, S = Body::kStages, TB = Body::kTileBytes;
  constexpr int kWarps = Body::kWarps, kThreads = (kWarps + 1) * 32;
  static_assert(kWarps <= kMaxWarps, "tables in Sched");
  extern __shared__ __align__(128) uint8_t base[];       // (never cast through an integer: loads from it must stay shared loads)
  __shared__ Sched sh;
  __shared__ uint64_t full[kWarps][S], empty[kWarps][S];
  __shared__ int loaded[kWarps][S];              // a stage's tiles, negative if they lie in no valid page
  __shared__ int row_of[Body::kSparse ? kWarps : 1][S];   // the row at which a stage begins, where pages are chosen
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  // where a warp's states lie: place 0 behind the ring and the queries, place 1 in the ring
  auto state_of = [&](int w, int place) {
    return reinterpret_cast<float*>(base + w * L::warp_bytes + (place ? 0 : L::ring + Body::kQueryFloats * 4));
  };
  const int cols_total = (Body::kSparse ? 1 : a.T) * a.rep, n_entries = entries<Body>(a);

  if (warp < kWarps && lane == 0) {
    for (int s = 0; s < S; ++s) { mbar_init(&full[warp][s], 1); mbar_init(&empty[warp][s], 1); }
    sh.piece[warp][0].valid = sh.piece[warp][1].valid = 0;
  }
  if (t == 0) { sh.abort_flag = 0; sh.open_c1[0] = sh.open_c1[1] = -1; }
  fence_barrier_init();

  // ---- this CTA's share: total units, units per warp, and the entries in which the warps' ranges start
  long long total = 0, part, u_mine = 0, lo_mine = 0;
  int l_mine = 0, len_mine = 0;
  for (int i0 = 0; i0 < n_entries; i0 += kThreads) {
    const int i = i0 + t;
    u_mine = i < n_entries ? entry_units<Body>(a, i, cgs, &l_mine, &len_mine) : 0;
    if (blockIdx.x == 0 && i < n_entries && u_mine == 0) record(a.p.status, PYR_ERR_INVALID);
    lo_mine = block_scan<kWarps + 1>(u_mine, sh.sums, &part);
    total += part;
  }
  // With no more (entry, head, column group)s than CTAs, and none long, each CTA takes one: no state crosses CTAs then, which
  // would cost more than the shorter way to the end saves (a step in a graph, us, even shares -> one a CTA; heads of queries
  // and of keys: 1 list x 385 rows, 32/32: 13.8 -> 9.8; 4 x 700, 32/32: 15.2 -> 10.9; 16 x 1300, 64/8: 19.3 -> 14.9; but
  // 1 x 2500, 32/32, 14 tiles a warp: 16.4 -> 18.2).
  long long cta_u = 0, cta_units = 0;
  bool whole_ones = false;
  if (n_entries <= kThreads) {
    const bool there = u_mine > 0;
    const bool any_long = __syncthreads_or(there && entry_tiles<Body>(a, len_mine) > kCtaTiles * kWarps);
    const int per_entry = a.p.Hkv * cgs;
    const long long all = (long long)__syncthreads_count(there) * per_entry;
    whole_ones = !any_long && all <= gridDim.x;
    if (whole_ones) {
      if (blockIdx.x >= all) return;             // the whole CTA: nothing is in flight
      const int e = blockIdx.x / per_entry;
      const long long order = block_scan<kWarps + 1>(there, sh.sums, &part);
      if (there && order == e) {
        const int tiles = entry_tiles<Body>(a, len_mine);
        sh.share_u = lo_mine + (long long)(blockIdx.x - e * per_entry) * (tiles + Body::kSegment) + Body::kSegment;
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
    for (int i0 = 0; i0 < n_entries && run < cta_u + cta_units; i0 += kThreads) {
      const int i = i0 + t;
      long long u = u_mine, lo = lo_mine;
      if (n_entries > kThreads) {
        u = i < n_entries ? entry_units<Body>(a, i, cgs, &l_mine, &len_mine) : 0;
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
    const int tpp = a.p.tiles_per_page, head_bytes = pages_head_bytes(a.p);
    const uint8_t* src = nullptr;
    uint32_t parity = 1;                         // of the wait for an empty stage: the first ones are
    const int32_t* row = a.p.table;
    const int32_t* slots = nullptr;              // of the head, where pages are chosen: `slot` counts along them
    int slot_next = -1, avail = 0, row0 = 0;     // page_next's slot; tiles of the page that rows reach; the page's first row
    // the chosen page at place x of the list of slots: its id (-1 if there is none) as the table has it, its slot
    auto chosen = [&](int x) {
      const int want = x < a.n_slots ? slots[x] : -1;
      slot_next = want;
      page_next = want >= 0 && want < a.p.max_pages ? row[want] : -1;
    };
    auto slots_of = [&] { return a.slots + ((size_t)ld.entry * a.p.Hkv + ld.h) * a.n_slots; };
    if (mine > 0) {
      ld.start<Body>(a, cgs, sh.entry[w_of], sh.list[w_of], sh.len[w_of], u_warp - sh.first_unit[w_of], &left);
      slot = ld.t / tpp;
      skip = ld.t - slot * tpp;
      row = a.p.table + (size_t)ld.list * a.p.max_pages;
      if constexpr (Body::kSparse) {
        slots = slots_of();
        chosen(slot);
      } else {
        page_first = row[0];
        page_next = row[slot];
      }
    }
    const uint32_t full0 = smem_u32(&full[w_of < kWarps ? w_of : 0][0]), empty0 = smem_u32(&empty[w_of < kWarps ? w_of : 0][0]);
    const uint32_t ring0 = smem_u32(base) + (w_of < kWarps ? w_of : 0) * L::warp_bytes;
    volatile int* abort_flag = &sh.abort_flag;
    for (uint32_t idle = 0; __any_sync(0xffffffffu, ld.t < ld.t1 || left > 0);) {
      if (ld.t == ld.t1 && left > 0) {           // on to the next (entry, head, column group)
        if (ld.next<Body>(a, cgs, &left)) {
          row = a.p.table + (size_t)ld.list * a.p.max_pages;
          if constexpr (!Body::kSparse) page_first = row[0];
        }
        slot = 0;
        in_page = 0;
        if constexpr (Body::kSparse) {
          slots = slots_of();
          chosen(0);
        } else {
          page_next = page_first;
        }
      }
      const bool go = ld.t < ld.t1 && test_wait_once(empty0 + 8 * in_stage, parity);
      if (go) {
        if (in_page == 0) {
          src = nullptr;
          int64_t first = 0;                     // a chosen page's first row: no page, and nothing wrong, where the token sees none of it
          if constexpr (Body::kSparse) first = slot_next == -1 ? INT_MAX : slot_next < 0 || slot_next >= a.p.max_pages ? 0 : (int64_t)slot_next * a.p.page_rows;
          if (first < ld.len) {
            if (page_next >= 0 && page_next < a.p.n_pages)
              src = a.p.pool + ((size_t)page_next * a.p.Hkv + ld.h) * head_bytes + a.p.head_extra + skip * TB;
            else
              record(a.p.status, PYR_ERR_INVALID);
          }
          in_page = min(tpp - skip, ld.t1 - ld.t);
          if constexpr (Body::kSparse) {
            avail = src ? (int)attn_tiles(min(ld.len - (int)first, a.p.page_rows)) - skip : 0;
            row0 = (int)first + skip * kPageTile;
          }
          skip = 0;
          // the id after this one is fetched now and looked at when its page is opened
          ++slot;
          if constexpr (Body::kSparse) chosen(slot);
          else if (slot < a.p.max_pages) page_next = row[slot];
        }
        const int n = min(in_page, kStageTiles);
        bool there = src != nullptr;
        if constexpr (Body::kSparse) {
          there = avail > 0;
          row_of[w_of][in_stage] = row0;
          row0 += n * kPageTile;
        }
        loaded[w_of][in_stage] = there ? n : -n;
        if (there) {
          const int bytes = (Body::kSparse ? min(n, avail) : n) * TB;
          tile_load(ring0 + in_stage * (kStageTiles * TB), src, bytes, full0 + 8 * in_stage);
          src += bytes;
        } else {
          arrive(full0 + 8 * in_stage);
        }
        if (++in_stage == S) { in_stage = 0; parity ^= 1; }
        ++issued;
        in_page -= n;
        avail -= n;
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
    cu.start<Body>(a, cgs, sh.entry[warp], sh.list[warp], sh.len[warp], u_warp - sh.first_unit[warp], &left);
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
        cu.next<Body>(a, cgs, &left);
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
        if (n > 0) {
          const int row0 = Body::kSparse ? row_of[Body::kSparse ? warp : 0][stage] : tt * kPageTile;
          body.stage(a, ring + stage * (kStageTiles * TB), row0, min(cu.len - row0, n * kPageTile), qs, lane);
        }
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
      cu.next<Body>(a, cgs, &left);
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
          write4<Body>(a, pc, pc.cg * COLS + x, d, num, M, den, d == 0);
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
    constexpr int kFew = Body::kFew, kAtOnce = Body::kAtOnce;
    if (cn <= kFew) {                            // a thread for itself, in few instructions (one list's 64 chosen pages, 7 warps a CTA: all loads in one
                                                 // round 17.3 us, as below 16.7: fetching the code takes as long as the loads)
      for (int o = t; o < ncols * (D / 4); o += kThreads) {
        const int x = o / (D / 4), d = o % (D / 4) * 4;
        const float* st = src + x * (D + 2);
        float M = -INFINITY, num[4] = {0.f, 0.f, 0.f, 0.f}, den = 0.f;
#pragma unroll 1
        for (int k0 = 0; k0 < cn; k0 += 8) {
          float m[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) m[k] = k0 + k < cn ? __ldcg(st + (k0 + k) * step + (k0 + k == 0 ? second : 0) + D) : -INFINITY;
#pragma unroll
          for (int k = 0; k < 8; ++k) M = fmaxf(M, m[k]);
        }
        const float ref = M == -INFINITY ? 0.f : M;
#pragma unroll 1
        for (int k0 = 0; k0 < cn; k0 += kAtOnce) {
          float2 ml[kAtOnce], u[kAtOnce], v[kAtOnce];
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k)
            if (k0 + k < cn) {
              const float* at = st + (k0 + k) * step + (k0 + k == 0 ? second : 0);
              ml[k] = __ldcg(reinterpret_cast<const float2*>(at + D));
              u[k] = __ldcg(reinterpret_cast<const float2*>(at + d));
              v[k] = __ldcg(reinterpret_cast<const float2*>(at + d + 2));
            }
#pragma unroll
          for (int k = 0; k < kAtOnce; ++k)
            if (k0 + k < cn) {
              const float w = ex2(ml[k].x - ref);
              num[0] = fmaf(w, u[k].x, num[0]); num[1] = fmaf(w, u[k].y, num[1]);
              num[2] = fmaf(w, v[k].x, num[2]); num[3] = fmaf(w, v[k].y, num[3]);
              den = fmaf(w, ml[k].y, den);
            }
        }
        write4<Body>(a, pc, pc.cg * COLS + x, d, num, M, den, d == 0);
      }
      if (t == 0) a.arrived[c1] = 0;
      continue;
    }
    // a column's maxima and sums are 2 cn numbers far apart: a warp a column, so that they are fetched together
    float* weight = reinterpret_cast<float*>(base);           // [cn][COLS], where the rings were
    __syncthreads();
    for (int x = warp; x < ncols; x += kWarps + 1) {
      float M = -INFINITY;
#pragma unroll (Body::kRounds)
      for (int k = lane; k < cn; k += 32) M = fmaxf(M, __ldcg(src + k * step + (k == 0 ? second : 0) + x * (D + 2) + D));
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float ref = M == -INFINITY ? 0.f : M;
      float den = 0.f;
#pragma unroll (Body::kRounds)
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
        if (a.lse) a.lse[out_place<Body>(a, pc.entry, pc.h, pc.cg * COLS + x).lse] = lse_of(M, den);
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
      write4<Body>(a, pc, pc.cg * COLS + x, d, num, 0.f, sh.den[x], false);
    }
    if (t == 0) a.arrived[c1] = 0;                         // as the next call expects it
  }
}

template <class Body>
cudaError_t run_attn(const PagesAttnArgs& a, cudaStream_t s) {
  const int cgs = ((Body::kSparse ? 1 : a.T) * a.rep + Body::COLS - 1) / Body::COLS;
  constexpr int smem = Layout<Body>::total;
  cudaError_t e = allow_shared<attn_kernel<Body>>(smem);
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int at_once = Body::kBlocks * sms < kAttnMaxCtas ? Body::kBlocks * sms : kAttnMaxCtas;
  const int ctas = attn_ctas(a.p, Body::kSparse ? (int64_t)a.n * a.T : a.n, cgs, Body::kWarps * kMinUnits, at_once);
  attn_kernel<Body><<<(unsigned)ctas, (Body::kWarps + 1) * 32, smem, s>>>(a, cgs);
  return cudaGetLastError();
}

}  // namespace
}  // namespace pyr

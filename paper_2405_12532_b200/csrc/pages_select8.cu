// Which pages of the paged 8-bit cache a query reads: a cheap score for each page, and the n_slots largest (format: include/pyr.h).
//
// Score of a page for a KV head: the largest, over the head's query heads, of s_q s_K sum_d max(qc_d min_d, qc_d max_d), with qc the query
// in 8 bits and min, max the least and largest code of the page in each dimension: an upper bound of q . K over its rows, up to
// the query's rounding. The sums are whole numbers below 2^21, exact in any order; what follows is two products rounded to fp32, so
// equal inputs give the same pages everywhere. With qc split by its sign a term is one of two products, and the sums are those of
// two matrix products, of max with the codes above 0 and of min with those below: on m16n8k16 with 16 pages as rows and 8 query
// heads as columns; with one query head a KV head as dot products of bytes. (Whole numbers up to 127 are f16 numbers, their products and sums exact in fp32. Byte-wise dot products on the
// integer side took 30 us for two tokens of 32 lists of up to 512 pages, 8 heads; the warp-level instruction because the
// operands are bytes in registers.)
//
// One CTA, or a cluster of up to 8 where there are few, for each (entry, KV head) and up to kTokens query tokens, for which the
// extrema are read once. The scores of a list stay in the first CTA's shared memory (the others write theirs there), which finds
// the n_slots-th largest by its bits and writes the pages in order, token by token. What bounds it is the latency of its steps one after the
// other: ids, extrema, queries, scores, the n_slots-th, writing, each 1 to 4 us with issue slots 30 % busy (24 us for two tokens of 32 lists of up to 512
// pages, whose extrema take 4.6).
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pyr_internal.h"

namespace pyr {
namespace {

namespace cg = cooperative_groups;
constexpr int kTokens = 4;
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100
constexpr uint32_t kForced = 0xFFFFFFFFu;              // the key of a page that is taken whatever its score

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// A number's place in the order of scores; NaN counts as Inf, -0 as 0. (Below kForced.)
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x + 0.f : INFINITY);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ void mma16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
               "{%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t as_u32(__half2 x) { return reinterpret_cast<uint32_t&>(x); }
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return reinterpret_cast<__half2&>(x); }
// Four signed bytes as pairs of f16: bytes 0 and 2, bytes 1 and 3 (1024 + 128 + code, less 1152).
__device__ __forceinline__ void codes_of(uint32_t w, uint32_t* even, uint32_t* odd) {
  const __half2 off = as_half2(0xE480E480u);
  w ^= 0x80808080u;
  *even = as_u32(__hadd2(as_half2(__byte_perm(w, 0x64646464u, 0x4240)), off));
  *odd = as_u32(__hadd2(as_half2(__byte_perm(w, 0x64646464u, 0x4341)), off));
}

// A query row (at element `row` of q) in 8 bits by a warp: a lane's D / 32 codes, side by side; its scale (NaN if an element is not finite).
template <int D>
__device__ __forceinline__ float codes_of_query(const PagesSelectArgs& a, int64_t row, int* code) {
  constexpr int N = D / 32;
  const int lane = threadIdx.x & 31;
  float x[N], top = 0.f;
  if (a.dtype == PYR_F32) {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      const float2 v = *reinterpret_cast<const float2*>(static_cast<const float*>(a.q) + row + N * lane + k);
      x[k] = v.x; x[k + 1] = v.y;
    }
  } else {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      const uint32_t v = *reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(a.q) + row + N * lane + k);
      x[k] = __uint_as_float(v << 16); x[k + 1] = __uint_as_float(v & 0xffff0000u);
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) top = max_nan(top, fabsf(x[k]));
  // (magnitudes, Inf and NaN among them, are ordered as their bits are)
  top = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(top) & 0x7fffffffu));
  float s = __fdiv_rn(top, 127.f);
  if (s < kScaleMin) s = 0.f;
  const bool fine = top <= 3.402823466e38f;
  const float inverse = fine && s > 0.f ? __fdiv_rn(1.f, s) : 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k) code[k] = fine ? __float2int_rn(__fmul_rn(x[k], inverse)) : 0;
  return fine ? s : __uint_as_float(0x7FC00000u);
}

// The n_slots pages (of npages, more than that) with the largest keys, in order, by a whole CTA.
template <int kThreads>
struct Choice {
  alignas(16) uint32_t hist[256];
  uint32_t warp_sums[kThreads / 32], both[2][kThreads / 32];
  uint32_t bin, before, count;
};
template <int kThreads>
__device__ __forceinline__ void choose_pages(const uint32_t* keys, int npages, int n_slots, int32_t* out, Choice<kThreads>& sh) {
  constexpr int kWarps = kThreads / 32;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  // Keys that are not forced share their high bits: the 8 bits from the first that differs on are looked at first, and so on until a
  // group is taken whole (or its keys are equal: the first of them are).
  uint32_t ones = 0xFFFFFFFFu, any = 0, forced = 0;
  for (int x0 = 0; x0 < npages; x0 += kThreads) {
    const uint32_t key = x0 + t < npages ? keys[x0 + t] : kForced;
    if (key == kForced) forced += x0 + t < npages;
    else { ones &= key; any |= key; }
  }
  ones = __reduce_and_sync(0xffffffffu, ones);
  any = __reduce_or_sync(0xffffffffu, any);
  forced = __reduce_add_sync(0xffffffffu, forced);
  if (lane == 0) { sh.both[0][warp] = ones; sh.both[1][warp] = any; sh.warp_sums[warp] = forced; }
  __syncthreads();
  forced = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) { ones &= sh.both[0][w]; any |= sh.both[1][w]; forced += sh.warp_sums[w]; }
  // keys with these bits above `shift`, `need` of which are wanted (all with larger ones are)
  uint32_t need = n_slots - forced, prefix = any, threshold = any;
  int shift = 32 - __clz(ones ^ any);          // bits that differ (0: all keys are the same)
  prefix = shift < 32 ? prefix >> shift << shift : 0u;
  bool whole = need == 0;                      // every key that is left is taken, or none
  if (whole) threshold = kForced;
  while (!whole && shift > 0) {
    const int low = max(shift - 8, 0);
    const uint32_t mask = shift < 32 ? 0xFFFFFFFFu << shift : 0u;
    for (int x = t; x < 256; x += kThreads) sh.hist[x] = 0;
    __syncthreads();
    for (int x = t; x < npages; x += kThreads) {
      const uint32_t key = keys[x];
      if (key != kForced && (key & mask) == prefix) atomicAdd(&sh.hist[key >> low & 255u & ((1u << (shift - low)) - 1u)], 1u);
    }
    __syncthreads();
    if (warp == 0) {                           // lane i: bins 255 - 8 i and the seven below it, the largest first
      const uint4 lo = reinterpret_cast<const uint4*>(sh.hist)[62 - 2 * lane], hi = reinterpret_cast<const uint4*>(sh.hist)[63 - 2 * lane];
      const uint32_t c[8] = {hi.w, hi.z, hi.y, hi.x, lo.w, lo.z, lo.y, lo.x};
      uint32_t mine8 = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) mine8 += c[k];
      uint32_t incl = mine8;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      uint32_t before = incl - mine8;
      if (before < need && need <= incl) {
        bool found = false;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (!found && before + c[k] >= need) { sh.bin = 255 - 8 * lane - k; sh.before = before; sh.count = c[k]; found = true; }
          if (!found) before += c[k];
        }
      }
    }
    __syncthreads();
    prefix |= sh.bin << low;
    need -= sh.before;
    whole = sh.count == need;
    shift = low;
    threshold = prefix;
  }
  // ---- pages above it, and those equal to it in what has been looked at: all of them, or the first `need`, in order
  const uint32_t mask = shift < 32 ? 0xFFFFFFFFu << shift : 0u;
  uint32_t done = 0, equal = 0;
  if (whole && need > 0) need = 0xFFFFu << 16;
  __syncthreads();
  for (int x0 = 0; x0 < npages; x0 += kThreads) {
    const int x = x0 + t;
    const uint32_t key = x < npages ? keys[x] : 0u, bits = key == kForced ? key : key & mask;
    const bool above = x < npages && (key == kForced || bits > threshold), same = x < npages && key != kForced && bits == threshold;
    const uint32_t ba = __ballot_sync(0xffffffffu, above), bs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) sh.warp_sums[warp] = __popc(ba) | __popc(bs) << 16;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t n = sh.warp_sums[w];
      before += w < warp ? n : 0;
      total += n;
    }
    const uint32_t lower = (1u << lane) - 1u;
    const uint32_t a0 = done + (before & 0xFFFFu) + __popc(ba & lower), e0 = equal + (before >> 16) + __popc(bs & lower);
    if (above || (same && e0 < need)) out[a0 + min(e0, need)] = x;
    done += total & 0xFFFFu;
    equal += total >> 16;
    __syncthreads();
  }
}

// The extrema of two pages that a lane feeds to the instruction, and their scales (-1: no page).
template <int X> struct Extrema { uint4 least[2][X], most[2][X]; float scale[2]; };

// kGroups: groups of 8 query heads (of one or several tokens) for which the extrema's codes are taken apart once
template <int D, int kGroups, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : 640 / kThreads) select8_kernel(PagesSelectArgs a, int tokens) {
  constexpr int kWarps = kThreads / 32;
  constexpr int X = D / 64, KS = D / 16;         // 16-byte pieces of a row of extrema a lane, steps over D
  extern __shared__ __align__(16) uint32_t shared[];
  __shared__ Choice<kThreads> sh;
  __shared__ int pages_of[kTokens];              // that hold rows the token sees
  const int key_stride = (a.p.max_pages + 3) / 4 * 4, tok_groups = (a.T + tokens - 1) / tokens, groups = (a.rep + 7) / 8;
  uint32_t* keys = shared;                                         // [tokens][max_pages]
  // codes of the queries as the instruction takes them: [tokens][groups of 8 heads][steps][lanes] of two registers
  uint2* codes = reinterpret_cast<uint2*>(shared + tokens * key_stride);
  float* sq = reinterpret_cast<float*>(codes + tokens * groups * KS * 32);            // [tokens][groups * 8]
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ranks = cluster.num_blocks();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const uint32_t item = blockIdx.x / (uint32_t)ranks, eg = item / (uint32_t)a.p.Hkv;
  const int h = (int)(item - eg * a.p.Hkv), e = (int)(eg / (uint32_t)tok_groups), tok0 = (int)(eg - (uint32_t)e * tok_groups) * tokens;
  const int ntok = min(tokens, a.T - tok0);
  auto out_of = [&](int tok) { return a.slots + (((int64_t)e * a.T + tok0 + tok) * a.p.Hkv + h) * a.n_slots; };
  const int l = pages_list(a.p, a.lists, e);

  // ---- page ids of the first steps are on their way before the list's length is there
  const int i8 = lane >> 2, j = lane & 3;
  const int32_t* table = a.p.table + (size_t)max(l, 0) * a.p.max_pages;
  const int head_bytes = pages_head_bytes(a.p), step = kWarps * 16 * ranks;        // pages of a step of the cluster
  const int mine = (rank * kWarps + warp) * 16 + i8;               // this lane's pages: this one and the eighth behind it
  int limit = l < 0 ? 0 : a.p.max_pages;                           // pages looked at
  int ids[2];
  auto fetch_ids = [&](int base) {
#pragma unroll
    for (int y = 0; y < 2; ++y) ids[y] = base + 8 * y < limit ? table[base + 8 * y] : -1;
  };
  fetch_ids(mine);
  const int last_len = l < 0 ? 0 : pages_len(a.p, l) - (a.T - tok0 - ntok);          // rows that the last of the tokens sees
  const int pages = pages_for(a.p, max(0, last_len));
  if (t < ntok) pages_of[t] = pages_for(a.p, max(0, last_len - (ntok - 1 - t)));
  __syncthreads();
  if (pages <= a.n_slots) {                                        // (for every token, in the whole cluster)
    if (rank == 0) {
      if (l < 0 && t == 0) record(a.p.status, PYR_ERR_INVALID);
      for (int tok = 0; tok < ntok; ++tok)
        for (int x = t; x < a.n_slots; x += kThreads) out_of(tok)[x] = x < pages_of[tok] ? x : -1;
    }
    return;
  }
  limit = pages;
  auto fetch = [&](int base, Extrema<X>& to) {
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      to.scale[y] = -1.f;
#pragma unroll
      for (int x = 0; x < X; ++x) to.least[y][x] = to.most[y][x] = make_uint4(0, 0, 0, 0);
      if (base + 8 * y < pages && ids[y] >= 0 && ids[y] < a.p.n_pages) {
        const uint8_t* head = a.p.pool + ((size_t)ids[y] * a.p.Hkv + h) * head_bytes;
#pragma unroll
        for (int x = 0; x < X; ++x) {
          to.least[y][x] = reinterpret_cast<const uint4*>(head)[X * j + x];
          to.most[y][x] = reinterpret_cast<const uint4*>(head + D)[X * j + x];
        }
        to.scale[y] = *reinterpret_cast<const float*>(head + 2 * D);
      }
    }
  };
  // (the first step's extrema on their way to the L2 cache while the queries are worked out)
#pragma unroll
  for (int y = 0; y < 2; ++y)
    if (j < 3 && mine + 8 * y < pages && ids[y] >= 0 && ids[y] < a.p.n_pages)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(a.p.pool + ((size_t)ids[y] * a.p.Hkv + h) * head_bytes + 128 * j));

  // ---- the queries in 8 bits, a warp a head: lane `lane` has the four (two) dimensions of a word (half) of the extrema
  constexpr int N = D / 32;
  for (int r = warp; r < ntok * groups * 8; r += kWarps) {
    const int tok = r / (groups * 8), c = r - tok * groups * 8;
    const int w = N * lane / 4, at = ((r / 8 * KS + w % (4 * X)) * 32 + (r & 7) * 4 + w / (4 * X));        // word w: lane w / (4 X)'s of step w mod 4 X
    uint16_t half[N] = {};
    if (c < a.rep) {
      const int64_t row = (int64_t)e * a.qsb + (int64_t)(tok0 + tok) * a.qst + (int64_t)(h * a.rep + c) * a.qsh;
      int code[N];
      const float s = codes_of_query<D>(a, row, code);
#pragma unroll
      for (int k = 0; k < N; ++k) half[k] = __half_as_ushort(__int2half_rn(code[k]));
      if (lane == 0) sq[r] = s;
    }
    uint16_t* dst = reinterpret_cast<uint16_t*>(codes + at);       // dimensions 0 and 2 of a word, 1 and 3
    if constexpr (N == 4) {
      *reinterpret_cast<uint2*>(dst) = make_uint2(half[0] | (uint32_t)half[2] << 16, half[1] | (uint32_t)half[3] << 16);
    } else {
      dst[lane & 1] = half[0];
      dst[2 + (lane & 1)] = half[1];
    }
  }
  uint32_t* keys0 = ranks > 1 ? cluster.map_shared_rank(keys, 0) : keys;
  if (ranks > 1) cluster.sync(); else __syncthreads();

  // ---- scores
#pragma unroll 1
  for (int base = mine; base - i8 < pages; base += step) {
    Extrema<X> now;
    fetch(base, now);
    fetch_ids(base + step);
    // kGroups groups of 8 heads at a time, which may be of several tokens
    float best[2] = {-INFINITY, -INFINITY};      // of the token
    int g = 0, tok = 0;
#pragma unroll 1
    for (int g0 = 0; g0 < ntok * groups; g0 += kGroups) {
      if (kGroups > 1)
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int x = 0; x < X; ++x) {            // (else codes would be kept from one round to the next, in more registers than there are)
          asm volatile("" : "+r"(now.least[y][x].x), "+r"(now.least[y][x].y), "+r"(now.least[y][x].z), "+r"(now.least[y][x].w));
          asm volatile("" : "+r"(now.most[y][x].x), "+r"(now.most[y][x].y), "+r"(now.most[y][x].z), "+r"(now.most[y][x].w));
        }
      float acc[kGroups][4] = {};
      const uint2* q = codes + g0 * KS * 32 + lane;
      const int n = min(kGroups, ntok * groups - g0);
#pragma unroll
      for (int x = 0; x < X; ++x) {
        const uint32_t m0[4] = {now.most[0][x].x, now.most[0][x].y, now.most[0][x].z, now.most[0][x].w};
        const uint32_t m1[4] = {now.most[1][x].x, now.most[1][x].y, now.most[1][x].z, now.most[1][x].w};
        const uint32_t l0[4] = {now.least[0][x].x, now.least[0][x].y, now.least[0][x].z, now.least[0][x].w};
        const uint32_t l1[4] = {now.least[1][x].x, now.least[1][x].y, now.least[1][x].z, now.least[1][x].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t am[4], al[4];
          codes_of(m0[k], &am[0], &am[2]);
          codes_of(m1[k], &am[1], &am[3]);
          codes_of(l0[k], &al[0], &al[2]);
          codes_of(l1[k], &al[1], &al[3]);
#pragma unroll
          for (int u = 0; u < kGroups; ++u)
            if (kGroups == 1 || u < n) {
              const uint2 b = q[(u * KS + 4 * x + k) * 32];
              const __half2 none = as_half2(0), b0 = as_half2(b.x), b1 = as_half2(b.y);
              mma16(acc[u], am, as_u32(__hmax2(b0, none)), as_u32(__hmax2(b1, none)));
              mma16(acc[u], al, as_u32(__hmin2(b0, none)), as_u32(__hmin2(b1, none)));
            }
        }
      }
#pragma unroll
      for (int u = 0; u < kGroups; ++u)
        if (kGroups == 1 || u < n) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int c = 8 * g + 2 * j + (k & 1);
            if (c < a.rep) best[k >> 1] = max_nan(best[k >> 1], __fmul_rn(__fmul_rn(sq[tok * groups * 8 + c], now.scale[k >> 1]), acc[u][k]));
          }
          if (++g == groups) {                   // the token's last
            const int npages = pages_of[tok];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              best[y] = max_nan(best[y], __shfl_xor_sync(0xffffffffu, best[y], 1));
              best[y] = max_nan(best[y], __shfl_xor_sync(0xffffffffu, best[y], 2));
              const int x = base + 8 * y;
              if (j == 0 && x < npages) {
                const bool none = now.scale[y] == -1.f;
                if (none) record(a.p.status, PYR_ERR_INVALID);
                keys0[tok * key_stride + x] = x < a.keep_first || x >= npages - a.keep_last ? kForced : none ? 0u : key_of(best[y]);
              }
              best[y] = -INFINITY;
            }
            g = 0;
            ++tok;
          }
        }
    }
  }
  if (ranks > 1) {
    cluster.sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

#pragma unroll 1
  for (int tok = 0; tok < ntok; ++tok, keys += key_stride) {
    const int npages = pages_of[tok];
    int32_t* out = out_of(tok);
    if (npages <= a.n_slots) {
      for (int x = t; x < a.n_slots; x += kThreads) out[x] = x < npages ? x : -1;
      continue;
    }
    choose_pages<kThreads>(keys, npages, a.n_slots, out, sh);
  }
}

// One query head a KV head: words of four bytes multiplied on the integer side, D / 16 lanes a page, a CTA (or a cluster) a token. The matrix
// instruction takes eight heads whether they are there or not (64 lists of 32 heads, 69 pages, 12.7 us, by it 18.5; one list of 502 pages of 8 heads 7.2,
// 8.4; four tokens of 64 lists of 8 heads, 63 pages, 11.4, 20.9. With two to four heads this form, four at a time, took 19 for 15 us on 32 lists of
// 250 pages and 12 for 8 on one list of 32 heads, 12 for 14 on 64 short lists).
template <int D, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : 768 / kThreads) select8_bytes_kernel(PagesSelectArgs a) {
  constexpr int kWarps = kThreads / 32;
  constexpr int LPP = D / 16, PPW = 32 / LPP, W = D / 4, U = 2;    // lanes a page, pages a warp and step, words of a row, steps at once
  extern __shared__ __align__(16) uint32_t shared[];
  __shared__ Choice<kThreads> sh;
  uint32_t* keys = shared;                                         // [max_pages] rounded up to 4
  __shared__ __align__(16) uint32_t plus[2 * W];                   // the query's codes above 0, then those below
  __shared__ float sq;
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ranks = cluster.num_blocks();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const uint32_t item = blockIdx.x / (uint32_t)ranks, et = item / (uint32_t)a.p.Hkv;
  const int h = (int)(item - et * a.p.Hkv), e = (int)(et / (uint32_t)a.T), tok = (int)(et - (uint32_t)e * a.T);
  int32_t* out = a.slots + (int64_t)item * a.n_slots;
  const int l = pages_list(a.p, a.lists, e);
  const int len = l < 0 ? 0 : max(0, pages_len(a.p, l) - (a.T - 1 - tok));
  const int pages = pages_for(a.p, len);
  if (pages <= a.n_slots) {                                        // (the whole cluster)
    if (rank == 0) {
      if (l < 0 && t == 0) record(a.p.status, PYR_ERR_INVALID);
      for (int x = t; x < a.n_slots; x += kThreads) out[x] = x < pages ? x : -1;
    }
    return;
  }
  // ---- the query in 8 bits
  if (warp == 0) {
    constexpr int N = D / 32;
    int c[N];
    const float s = codes_of_query<D>(a, (int64_t)e * a.qsb + (int64_t)tok * a.qst + (int64_t)h * a.qsh, c);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      reinterpret_cast<int8_t*>(plus)[N * lane + k] = (int8_t)max(c[k], 0);
      reinterpret_cast<int8_t*>(plus + W)[N * lane + k] = (int8_t)min(c[k], 0);
    }
    if (lane == 0) sq = s;
  }
  uint32_t* keys0 = ranks > 1 ? cluster.map_shared_rank(keys, 0) : keys;
  if (ranks > 1) cluster.sync(); else __syncthreads();

  // ---- scores
  const int sub = lane / LPP, part = lane % LPP;
  const int32_t* table = a.p.table + (size_t)l * a.p.max_pages;
  const int head_bytes = pages_head_bytes(a.p);
  const int step = kWarps * PPW * U;                               // pages of a CTA's step
  // (a step's extrema are on their way while the one before is worked out, and its page ids before that)
  int ids[U];
  uint4 mn_next[U], mx_next[U];
  float sk_next[U];
  auto fetch_ids = [&](int base) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = base + (u * kWarps + warp) * PPW + sub;
      ids[u] = x < pages ? table[x] : -1;
    }
  };
  auto fetch = [&] {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      mn_next[u] = mx_next[u] = make_uint4(0, 0, 0, 0);
      sk_next[u] = -1.f;                                           // no page
      if (ids[u] >= 0 && ids[u] < a.p.n_pages) {
        const uint8_t* head = a.p.pool + ((size_t)ids[u] * a.p.Hkv + h) * head_bytes;
        mn_next[u] = reinterpret_cast<const uint4*>(head)[part];
        mx_next[u] = reinterpret_cast<const uint4*>(head + D)[part];
        sk_next[u] = *reinterpret_cast<const float*>(head + 2 * D);
      }
    }
  };
  fetch_ids(rank * step);
  fetch();
  fetch_ids((rank + ranks) * step);
  for (int base = rank * step; base < pages; base += ranks * step) {
    uint4 mn[U], mx[U];
    float sk[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { mn[u] = mn_next[u]; mx[u] = mx_next[u]; sk[u] = sk_next[u]; }
    fetch();
    fetch_ids(base + 2 * ranks * step);
    const uint4 qp = reinterpret_cast<const uint4*>(plus)[part], qn = reinterpret_cast<const uint4*>(plus + W)[part];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = base + (u * kWarps + warp) * PPW + sub;
      int sum = __dp4a((int)mx[u].x, (int)qp.x, 0);
      sum = __dp4a((int)mn[u].x, (int)qn.x, sum);
      sum = __dp4a((int)mx[u].y, (int)qp.y, sum);
      sum = __dp4a((int)mn[u].y, (int)qn.y, sum);
      sum = __dp4a((int)mx[u].z, (int)qp.z, sum);
      sum = __dp4a((int)mn[u].z, (int)qn.z, sum);
      sum = __dp4a((int)mx[u].w, (int)qp.w, sum);
      sum = __dp4a((int)mn[u].w, (int)qn.w, sum);
#pragma unroll
      for (int o = LPP / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (part == 0 && x < pages) {
        const bool none = sk[u] == -1.f;
        if (none) record(a.p.status, PYR_ERR_INVALID);
        keys0[x] = x < a.keep_first || x >= pages - a.keep_last ? kForced : none ? 0u : key_of(__fmul_rn(__fmul_rn(sq, sk[u]), (float)sum));
      }
    }
  }
  if (ranks > 1) {
    cluster.sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }
  choose_pages<kThreads>(keys, pages, a.n_slots, out, sh);
}

// A call's kernel with up to kThreads threads a CTA, of which `items` work on different lists, heads or tokens.
template <int kThreads, class... Args>
cudaError_t run(void (*kernel)(Args...), const PagesSelectArgs& a, int64_t items, int smem, cudaStream_t s, Args... args) {
  const int sms = device_sm_count();
  // several CTAs a list where that many find room at once and each has a step or more to do (one list of 502 pages, 8 heads: 8.6 us, with one 10.1)
  int ranks = 1;
  while (kThreads == 512 && ranks < 8 && items * ranks * 2 <= sms && a.p.max_pages > ranks * (kThreads / 2)) ranks *= 2;
  if (items * ranks > 0x7fffffffLL) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(items * ranks)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = ranks; at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at; cfg.numAttrs = ranks > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
template <int D, int kGroups, int kThreads>
cudaError_t run_mma(const PagesSelectArgs& a, int64_t items, int tokens, int smem, cudaStream_t s) {
  const cudaError_t e = allow_shared<select8_kernel<D, kGroups, kThreads>>(kSelect8Shared);
  return e != cudaSuccess ? e : run<kThreads, PagesSelectArgs, int>(select8_kernel<D, kGroups, kThreads>, a, items, smem, s, a, tokens);
}
template <int D, int kThreads>
cudaError_t run_bytes(const PagesSelectArgs& a, int64_t items, int smem, cudaStream_t s) {
  const cudaError_t e = allow_shared<select8_bytes_kernel<D, kThreads>>(kSelect8Shared);
  return e != cudaSuccess ? e : run<kThreads, PagesSelectArgs>(select8_bytes_kernel<D, kThreads>, a, items, smem, s, a);
}
// As many threads for a list as there is room for, where its table is long enough to occupy them (one list of 502 pages and 32 of up to
// 512, 8 heads: 8.6 and 24.1 us, with 128 throughout 19.4 and 33.5). The table's width decides, since lengths lie on the device: short lists in wide
// tables get as many.
template <int D, int kGroups>
cudaError_t by_length(const PagesSelectArgs& a, int sms, int tokens, int smem, cudaStream_t s) {
  const int64_t items = (int64_t)a.n * ((a.T + tokens - 1) / tokens) * a.p.Hkv;
  const auto fits = [&](int threads) { return items * threads <= (int64_t)sms * 640 && a.p.max_pages * 2 >= threads; };
  return fits(512) ? run_mma<D, kGroups, 512>(a, items, tokens, smem, s) : fits(256) ? run_mma<D, kGroups, 256>(a, items, tokens, smem, s)
         : fits(128) ? run_mma<D, kGroups, 128>(a, items, tokens, smem, s) : fits(64) ? run_mma<D, kGroups, 64>(a, items, tokens, smem, s)
         : a.p.max_pages > 512 ? run_mma<D, kGroups, 128>(a, items, tokens, smem, s) : run_mma<D, kGroups, 32>(a, items, tokens, smem, s);
}
template <int D>
cudaError_t by_length_bytes(const PagesSelectArgs& a, int sms, int smem, cudaStream_t s) {
  const int64_t items = (int64_t)a.n * a.T * a.p.Hkv;
  const auto fits = [&](int threads) { return items * threads <= (int64_t)sms * 1024 && a.p.max_pages * 2 >= threads; };
  return fits(512) ? run_bytes<D, 512>(a, items, smem, s) : fits(256) ? run_bytes<D, 256>(a, items, smem, s)
         : fits(128) ? run_bytes<D, 128>(a, items, smem, s) : a.p.max_pages > 1024 ? run_bytes<D, 256>(a, items, smem, s) : run_bytes<D, 32>(a, items, smem, s);
}

}  // namespace

cudaError_t launch_pages_select8(const PagesSelectArgs& a, int* launches, cudaStream_t s) {
  // several tokens a CTA where there are more (entry, KV head)s than SMs, and memory for their scores (two tokens of 32 lists of up to 512 pages:
  // 24.1 us, a token a CTA 29.1); groups of 8 query heads one by one where there is one (one list: 8.6 us, by the code for four 9.2)
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int64_t one = pages_select8_shared(a.p.max_pages, a.p.D, a.rep);
  if (a.rep == 1) {
    const cudaError_t e = a.p.D == 128 ? by_length_bytes<128>(a, sms, (int)one, s) : by_length_bytes<64>(a, sms, (int)one, s);
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  int tokens = 1;
  while (tokens < kTokens && tokens < a.T && (tokens + 1) * one <= kSelect8Shared && (int64_t)a.n * a.p.Hkv >= sms) ++tokens;
  const int smem = (int)(tokens * one);
  const bool one_group = tokens == 1 && a.rep <= 8;
  const cudaError_t e = a.p.D == 128 ? (one_group ? by_length<128, 1>(a, sms, tokens, smem, s) : by_length<128, 4>(a, sms, tokens, smem, s))
                                     : (one_group ? by_length<64, 1>(a, sms, tokens, smem, s) : by_length<64, 4>(a, sms, tokens, smem, s));
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

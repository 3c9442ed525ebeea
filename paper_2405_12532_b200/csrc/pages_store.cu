// Rows into and out of the paged 4-bit cache (format: include/pyr.h).
//
// A group of `group` values x is stored as codes c = rint((x - zero) / scale) in 0 .. 15 with zero = min x rounded down to
// bf16 and scale = (max x - zero) / 15 rounded up to bf16: with these two roundings every code is in range without a
// clamp, and a code's value scale * c + zero is within scale / 2 of x. The product scale * c is exact in fp32 (8 + 4 bits).
// Arithmetic is plain IEEE single precision, never contracted, so that the stored bytes are the same everywhere.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "pyr_internal.h"

namespace pyr {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kRowThreads = 256;                 // of a CTA that writes an entry's few rows
constexpr int kTileThreads = 64;                 // of one whose warps take a tile each and come and go on their own (8 x 2005 rows
                                                 // of 40 heads written and read: 167.5 us with 256, 164.9, 163.2)
constexpr int kFewRows = 512;                    // rows times heads of an entry that one CTA writes as fast as many
constexpr uint32_t kNanWord = 0x7FC07FC0u;       // (scale, zero) of a group that has no finite range
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }

__device__ __forceinline__ float min_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// x rounded down / up (x >= 0) to a bf16 number, as the fp32 that holds it
__device__ __forceinline__ float floor_bf16(float x) {
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float((b & 0xFFFF0000u) + ((x < 0.f && (b & 0xFFFFu)) ? 0x10000u : 0u));
}
__device__ __forceinline__ float ceil_bf16(float x) {
  const uint32_t b = __float_as_uint(x);
  return __uint_as_float((b & 0xFFFF0000u) + ((b & 0xFFFFu) ? 0x10000u : 0u));
}

__device__ __forceinline__ void load8(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <class T> __device__ __forceinline__ void store8(T* p, const float* x);
template <> __device__ __forceinline__ void store8<float>(float* p, const float* x) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    w[i] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x[2 * i])) |
           ((uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(x[2 * i + 1])) << 16);
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// Eight elements of a row as they are loaded, and what a group needs of them.
template <class T> struct Eight;
template <> struct Eight<float> {
  float x[8];
  float lo, hi;
  __device__ __forceinline__ void load(const float* p) { load8(p, x); }
  __device__ __forceinline__ void nan() {
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = __uint_as_float(0x7FC00000u);
  }
  // smallest and largest of the group (NaN if there is one); its kLanes threads sit side by side
  template <int kLanes> __device__ __forceinline__ void extrema() {
    lo = hi = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) { lo = min_nan(lo, x[k]); hi = max_nan(hi, x[k]); }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) {
      lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
      hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
  }
  __device__ __forceinline__ void take_extrema(const Eight& o, int lane) {       // those of another thread
    lo = __shfl_sync(0xffffffffu, o.lo, lane);
    hi = __shfl_sync(0xffffffffu, o.hi, lane);
  }
  __device__ __forceinline__ void set_extrema(const Eight& o) { lo = o.lo; hi = o.hi; }
  __device__ __forceinline__ float low() const { return lo; }
  __device__ __forceinline__ float high() const { return hi; }
  __device__ __forceinline__ float at(int k) const { return x[k]; }
};
// bf16: two elements to an instruction; the smallest and the negated largest travel as one pair
template <> struct Eight<__nv_bfloat16> {
  uint32_t w[4];
  uint32_t ends;                                 // low half: smallest, high half: minus the largest
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    const uint4 r = *reinterpret_cast<const uint4*>(p);
    w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w;
  }
  __device__ __forceinline__ void nan() { w[0] = w[1] = w[2] = w[3] = 0x7FC07FC0u; }
  static __device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
  }
  template <int kLanes> __device__ __forceinline__ void extrema() {
    const uint32_t mn = least(least(w[0], w[1]), least(w[2], w[3]));
    const uint32_t mx = most(most(w[0], w[1]), most(w[2], w[3])) ^ 0x80008000u;
    ends = least(__byte_perm(mn, mx, 0x5410), __byte_perm(mn, mx, 0x7632));
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) ends = least(ends, __shfl_xor_sync(0xffffffffu, ends, o));
  }
  __device__ __forceinline__ void take_extrema(const Eight& o, int lane) { ends = __shfl_sync(0xffffffffu, o.ends, lane); }
  __device__ __forceinline__ void set_extrema(const Eight& o) { ends = o.ends; }
  __device__ __forceinline__ float low() const { return __uint_as_float(ends << 16); }
  __device__ __forceinline__ float high() const { return -__uint_as_float(ends & 0xffff0000u); }
  __device__ __forceinline__ float at(int k) const {
    return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16);
  }
};

// A group's (scale, zero) word and 1 / scale, from its extrema.
__device__ __forceinline__ uint32_t group_word(float lo, float hi, float* inv) {
  const float zero = floor_bf16(lo);
  const float span = __fsub_rn(hi, zero);
  float scale = ceil_bf16(__fdiv_rn(span, 15.f));
  if (scale < kScaleMin) scale = 0.f;
  const bool finite = span <= 3.402823466e38f;   // not so: infinite or not a number
  *inv = scale > 0.f && finite ? __fdiv_rn(1.f, scale) : 0.f;
  return finite ? (__float_as_uint(scale) >> 16) | (__float_as_uint(zero) & 0xFFFF0000u) : kNanWord;
}
// The eight codes (dimension k in bits 4k ..). Adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it in the
// low bits; the rest of that number's bits are above bit 21, out of the way of the 16 bits that four codes make.
template <class T>
__device__ __forceinline__ uint32_t group_codes(const Eight<T>& x, uint32_t word, float inv) {
  constexpr float kRound = 12582912.f;
  const float zero = __uint_as_float(word & 0xFFFF0000u);
  uint32_t half[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x.at(4 * h + k), zero), inv), kRound));
    half[h] = c[0] + 16u * c[1] + 256u * c[2] + 4096u * c[3];
  }
  const uint32_t w = __byte_perm(half[0], half[1], 0x5410);
  return word == kNanWord ? 0u : w;              // (NaN everywhere: any code would do)
}

// Decides every entry of a write before any row moves: plan[i] = first row, -1 if the entry is refused. A warp per entry.
__global__ void __launch_bounds__(kPlanThreads) write_plan_kernel(PagesWriteArgs a, int words) {
  extern __shared__ uint32_t seen[];              // two bits per list: met, met twice
  let_next_start();
  uint32_t* twice = seen + words;
  const int t = threadIdx.x, lane = t & 31;
  for (int i = t; i < 2 * words; i += kPlanThreads) seen[i] = 0;
  __syncthreads();
  for (int i = t; i < a.n; i += kPlanThreads) {
    const int l = pages_list(a.p, a.lists, i);
    if (l >= 0 && (atomicOr(&seen[l >> 5], 1u << (l & 31)) >> (l & 31) & 1u)) atomicOr(&twice[l >> 5], 1u << (l & 31));
  }
  __syncthreads();
  for (int i = t >> 5; i < a.n; i += kPlanThreads / 32) {
    const int l = pages_list(a.p, a.lists, i);
    const int cnt = a.counts ? a.counts[i] : a.n_rows;
    bool ok = l >= 0 && cnt >= 0 && cnt <= a.n_rows && !(twice[l >> 5] >> (l & 31) & 1u);
    int start = 0, len = 0;
    if (ok) {
      len = pages_len(a.p, l);
      start = a.first ? a.first[i] : len;
      ok = start >= 0 && start <= len && (int64_t)start + cnt <= (int64_t)a.p.max_pages * a.p.page_rows;
    }
    if (ok && cnt > 0) {
      const int s1 = (int)(((int64_t)start + cnt - 1) / a.p.page_rows);
      for (int s = start / a.p.page_rows + lane; s <= s1; s += 32) {
        const int page = pages_page(a.p, l, s);
        ok = ok && page >= 0 && a.p.refs[page] == 1;
      }
    }
    ok = __all_sync(0xffffffffu, ok);
    if (lane == 0) {
      a.plan[i] = ok ? start : -1;
      if (ok) { if (start + cnt > len) a.p.lens[l] = start + cnt; }
      else record(a.p.status, PYR_ERR_INVALID);
    }
  }
}

// A thread holds eight dimensions of a row, D / 8 threads a row: word wi of K, halves 2 wi and 2 wi + 1 of V. In the stored order
// (include/pyr.h) the two halves are one 32-bit word too, unless a group has 32 dimensions: then the word takes the same
// half of two neighbouring groups, whose threads swap one half each.
template <int D, int GROUP>
struct VWord {
  static constexpr bool kSwap = GROUP == 32;
  static __device__ __forceinline__ int slot(int wi) {
    if (!kSwap) return v_half_slot(D, GROUP, 2 * wi) / 2;
    const int g = wi / 4, m = wi % 4;
    return (2 * m + (g & 1)) * (D / 64) + g / 2;
  }
  // from a thread's own halves (low: 2 wi, high: 2 wi + 1) to the word in its slot, and back: the same swap
  static __device__ __forceinline__ uint32_t swap(uint32_t x, int wi) {
    if (!kSwap) return x;
    const bool odd = wi / 4 & 1;
    const uint32_t got = __shfl_xor_sync(0xffffffffu, odd ? x & 0xFFFFu : x >> 16, 4);
    return odd ? (x & 0xFFFF0000u) | got : (x & 0xFFFFu) | (got << 16);
  }
};

// Quantises and stores one tile's rows by one warp. `src` of lane r (< 16): the source row that becomes row r of the tile, -1
// where that row is not written, -2 where its source does not exist (NaN is stored). Four passes over rows are in flight
// at a time; their groups' scales are worked out side by side, a lane a group, and handed back, instead of by every thread
// of a group.
template <class T, int D, int GROUP>
__device__ __forceinline__ void store_tile(uint8_t* tile, const T* k, const T* v, int64_t sn, int src, int lane) {
  constexpr int LPR = D / 8, RPP = 32 / LPR, G = D / GROUP, P = kPageTile / RPP, B = 4, LG = GROUP / 8;
  constexpr int NW = B * RPP * G;                // groups of a batch of passes, of K and of V
  static_assert(NW <= 32, "a lane a group");
  const int sub = lane / LPR, wi = lane % LPR;
  const int my_row = lane / G, my_pass = my_row / RPP, my_lane = my_row % RPP * LPR + lane % G * LG;   // of the lane's group
#pragma unroll
  for (int b = 0; b < P / B; ++b) {
    int from[B];
    bool any = false;
#pragma unroll
    for (int q = 0; q < B; ++q) {
      from[q] = __shfl_sync(0xffffffffu, src, (b * B + q) * RPP + sub);
      any |= from[q] != -1;
    }
    if (!__any_sync(0xffffffffu, any)) continue;
    const int row_src = __shfl_sync(0xffffffffu, src, b * B * RPP + (my_row < B * RPP ? my_row : 0));
    Eight<T> x[2][B];
#pragma unroll
    for (int q = 0; q < B; ++q) {
      if (from[q] >= 0) {
        x[0][q].load(k + (int64_t)from[q] * sn + wi * 8);
        x[1][q].load(v + (int64_t)from[q] * sn + wi * 8);
      } else {
        x[0][q].nan();
        x[1][q].nan();
      }
    }
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      Eight<T> mine;
#pragma unroll
      for (int q = 0; q < B; ++q) {
        x[kv][q].template extrema<LG>();
        Eight<T> got;
        got.take_extrema(x[kv][q], my_lane);
        if (q == 0 || my_pass == q) mine.set_extrema(got);
      }
      float inv;
      const uint32_t word = group_word(mine.low(), mine.high(), &inv);
      if (lane < NW && row_src != -1)
        reinterpret_cast<uint32_t*>(tile + (kv ? tile_v_word(D, G, b * B * RPP, 0) : tile_k_word(D, G, b * B * RPP, 0)))[lane] = word;
#pragma unroll
      for (int q = 0; q < B; ++q) {
        const int owner = (q * RPP + sub) * G + wi / LG, r = (b * B + q) * RPP + sub;
        const uint32_t w = __shfl_sync(0xffffffffu, word, owner);
        uint32_t codes = group_codes(x[kv][q], w, __shfl_sync(0xffffffffu, inv, owner));
        if (kv) codes = VWord<D, GROUP>::swap(codes, wi);
        if (from[q] != -1)
          reinterpret_cast<uint32_t*>(tile + (kv ? tile_v_row(D, r) : tile_k_row(D, r)))[kv ? VWord<D, GROUP>::slot(wi) : k_word_slot(D, GROUP, wi)] = codes;
      }
    }
  }
}

// What lane r (< 16) of a warp that writes the tile of rows row0 .. row0 + 15 gives store_tile.
__device__ __forceinline__ int tile_source(const PagesWriteArgs& a, const int32_t* idx, int start, int cnt, int row0, int lane) {
  const int x = row0 + lane - start;
  if (lane >= kPageTile || x < 0 || x >= cnt) return -1;
  const int src = idx ? idx[x] : x;
  if (src >= 0 && src < a.src_rows) return src;
  record(a.p.status, PYR_ERR_INVALID);
  return -2;
}

template <class T>
__device__ __forceinline__ const T* head_rows(const void* p, const PagesWriteArgs& a, int e, int h) {
  return static_cast<const T*>(p) + (int64_t)e * a.sb + (int64_t)h * a.sh;
}
__device__ __forceinline__ const int32_t* entry_idx(const PagesWriteArgs& a, int e, int h) {
  return a.idx ? a.idx + (int64_t)e * a.idx_stride + (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows : nullptr;
}

// One warp per (entry, KV head, tile of its list). `blocks` tiles cover n_rows rows wherever in a tile they begin. 640 k gathered
// rows of 128 dimensions, K and V, from bf16: 92 us = 4.6 TB/s of 420 MB, three quarters of the issue slots taken (eleven
// instructions a value), with loads of four rows and both tensors in flight a warp and 32 warps an SM.
template <class T, int D, int GROUP>
__global__ void __launch_bounds__(kTileThreads, sizeof(T) == 2 ? 16 : 8) write_rows_kernel(PagesWriteArgs a, int blocks, int64_t items) {
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kTileThreads / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  const int blk = (int)(item % blocks);
  const int h = (int)(item / blocks % a.p.Hkv);
  const int e = (int)(item / blocks / a.p.Hkv);
  const int start = a.plan[e];
  if (start < 0) return;
  const int cnt = a.counts ? a.counts[e] : a.n_rows;
  const int row0 = start / kPageTile * kPageTile + blk * kPageTile;
  if (row0 >= start + cnt) return;
  const int src = tile_source(a, entry_idx(a, e, h), start, cnt, row0, lane);
  const int page = pages_page(a.p, pages_list(a.p, a.lists, e), row0 / a.p.page_rows);
  if (page < 0) return;                           // (the plan has seen a valid page here)
  store_tile<T, D, GROUP>(a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile), head_rows<T>(a.k, a, e, h),
                          head_rows<T>(a.v, a, e, h), a.sn, src, lane);
}

// A few rows per entry (a decode step): one CTA per entry decides and stores in one launch.
template <class T, int D, int GROUP>
__global__ void __launch_bounds__(kRowThreads) write_few_kernel(PagesWriteArgs a) {
  const int e = blockIdx.x, t = threadIdx.x;
  const int l = pages_list(a.p, a.lists, e);
  const int cnt = a.counts ? a.counts[e] : a.n_rows;
  bool bad = l < 0 || cnt < 0 || cnt > a.n_rows;
  int start = 0, len = 0;
  if (!bad) {
    len = pages_len(a.p, l);
    start = a.first ? a.first[e] : len;
    bad = start < 0 || start > len || (int64_t)start + cnt > (int64_t)a.p.max_pages * a.p.page_rows;
    if (!bad && cnt > 0)
      for (int s = start / a.p.page_rows + t; s <= (start + cnt - 1) / a.p.page_rows; s += kRowThreads) {
        const int page = pages_page(a.p, l, s);
        bad |= page < 0 || a.p.refs[page] != 1;
      }
  }
  if (a.lists)
#pragma unroll 4
    for (int x = t; x < a.n; x += kRowThreads) bad |= x != e && a.lists[x] == l;
  if (__syncthreads_or(bad)) {                    // (all threads have read the length by now)
    if (t == 0) record(a.p.status, PYR_ERR_INVALID);
    return;
  }
  if (t == 0 && start + cnt > len) a.p.lens[l] = start + cnt;
  // D / 8 threads a row of a head
  constexpr int LPR = D / 8, G = D / GROUP, LG = GROUP / 8, kRows = kRowThreads / LPR;
  const int sub = t / LPR, wi = t % LPR, items = cnt * a.p.Hkv;
#pragma unroll 2
  for (int i0 = 0; i0 < items; i0 += kRows) {
    const int item = i0 + sub;
    const bool live = item < items;
    const int x = live ? item / a.p.Hkv : 0, h = live ? item - x * a.p.Hkv : 0;
    const int32_t* idx = entry_idx(a, e, h);
    const int src = idx ? idx[x] : x;
    const bool good = src >= 0 && src < a.src_rows;
    const int row = start + x, r = row % kPageTile;
    const int page = live ? pages_page(a.p, l, row / a.p.page_rows) : -1;
    Eight<T> kx, vx;
    if (live && good) {
      kx.load(head_rows<T>(a.k, a, e, h) + (int64_t)src * a.sn + wi * 8);
      vx.load(head_rows<T>(a.v, a, e, h) + (int64_t)src * a.sn + wi * 8);
    } else {
      kx.nan();
      vx.nan();
    }
    kx.template extrema<LG>();
    vx.template extrema<LG>();
    float ki, vi;
    const uint32_t kw = group_word(kx.low(), kx.high(), &ki), vw = group_word(vx.low(), vx.high(), &vi);
    const uint32_t kc = group_codes(kx, kw, ki), vc = VWord<D, GROUP>::swap(group_codes(vx, vw, vi), wi);
    if (page < 0) continue;
    if (!good && wi == 0) record(a.p.status, PYR_ERR_INVALID);
    uint8_t* tile = a.p.pool + pages_tile(a.p, page, h, row % a.p.page_rows / kPageTile);
    reinterpret_cast<uint32_t*>(tile + tile_k_row(D, r))[k_word_slot(D, GROUP, wi)] = kc;
    reinterpret_cast<uint32_t*>(tile + tile_v_row(D, r))[VWord<D, GROUP>::slot(wi)] = vc;
    if (wi % LG == 0) {
      *reinterpret_cast<uint32_t*>(tile + tile_k_word(D, G, r, wi / LG)) = kw;
      *reinterpret_cast<uint32_t*>(tile + tile_v_word(D, G, r, wi / LG)) = vw;
    }
  }
}

// The values of eight codes: scale * code + zero, the product exact. Codes become numbers two at a time: 0x6400 | n is the f16
// number 1024 + n, 0x6400 | 16 n is 1024 + 16 n, which takes no integer conversion. (The conversion pipe is 58 % busy all
// the same, with those to fp32 and to bf16; DRAM is what bounds it.) 640 k rows of 128 dimensions, K and V, to bf16: 70 us =
// 6.0 TB/s of 420 MB; a single launch of half of them 38 us = 5.5 TB/s.
__device__ __forceinline__ void values8(uint32_t codes, uint32_t word, float* x) {
  const float scale = __uint_as_float(word << 16), zero = __uint_as_float(word & 0xFFFF0000u);
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const uint32_t bits = k < 2 ? codes : codes >> 8, mask = k & 1 ? 0x00F000F0u : 0x000F000Fu;
    const uint32_t y = (bits & mask) | 0x64006400u;
    const __half2 v = reinterpret_cast<const __half2&>(y);
    const float2 n = __half22float2(k & 1 ? __hfma2(v, __float2half2_rn(0.0625f), __float2half2_rn(-64.f))
                                          : __hsub2(v, __float2half2_rn(1024.f)));
    x[k] = __fmaf_rn(scale, n.x, zero);
    x[k + 4] = __fmaf_rn(scale, n.y, zero);
  }
}

// One warp per (entry, KV head, tile of its list), as for writing.
template <class T, int D, int GROUP>
__global__ void __launch_bounds__(kTileThreads) read_rows_kernel(PagesWriteArgs a, int blocks, int64_t items) {
  constexpr int LPR = D / 8, RPP = 32 / LPR, G = D / GROUP, P = kPageTile / RPP;
  const int lane = threadIdx.x & 31, sub = lane / LPR, wi = lane % LPR;
  const int64_t item = (int64_t)blockIdx.x * (kTileThreads / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  const int blk = (int)(item % blocks);
  const int h = (int)(item / blocks % a.p.Hkv);
  const int e = (int)(item / blocks / a.p.Hkv);
  const int l = pages_list(a.p, a.lists, e);
  const int first = a.first ? a.first[e] : 0;
  const int cnt = a.counts ? a.counts[e] : a.n_rows;
  if (l < 0 || first < 0 || cnt < 0 || cnt > a.n_rows) {
    if (lane == 0) record(a.p.status, PYR_ERR_INVALID);
    return;
  }
  const int end = (int)min((int64_t)pages_len(a.p, l), (int64_t)first + cnt);
  const int64_t tile_row = (int64_t)first / kPageTile * kPageTile + (int64_t)blk * kPageTile;
  if (tile_row >= end) return;
  const int row0 = (int)tile_row;
  const int page = pages_page(a.p, l, row0 / a.p.page_rows);
  if (page < 0) {
    if (lane == 0) record(a.p.status, PYR_ERR_INVALID);
    return;
  }
  const uint8_t* tile = a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile);
  T* k = const_cast<T*>(head_rows<T>(a.k, a, e, h)) + wi * 8;
  T* v = const_cast<T*>(head_rows<T>(a.v, a, e, h)) + wi * 8;
#pragma unroll
  for (int b = 0; b < P; b += 4) {
    uint32_t kc[4], vc[4], kw[4], vw[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int r = (b + q) * RPP + sub;
      kc[q] = reinterpret_cast<const uint32_t*>(tile + tile_k_row(D, r))[k_word_slot(D, GROUP, wi)];
      vc[q] = reinterpret_cast<const uint32_t*>(tile + tile_v_row(D, r))[VWord<D, GROUP>::slot(wi)];
      kw[q] = *reinterpret_cast<const uint32_t*>(tile + tile_k_word(D, G, r, wi / (GROUP / 8)));
      vw[q] = *reinterpret_cast<const uint32_t*>(tile + tile_v_word(D, G, r, wi / (GROUP / 8)));
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int row = row0 + (b + q) * RPP + sub;
      const uint32_t codes = VWord<D, GROUP>::swap(vc[q], wi);
      if (row < first || row >= end) continue;
      float f[8];
      values8(kc[q], kw[q], f);
      store8(k + (int64_t)(row - first) * a.sn, f);
      values8(codes, vw[q], f);
      store8(v + (int64_t)(row - first) * a.sn, f);
    }
  }
}

template <class F>
cudaError_t by_format(const PagesView& p, int dtype, F f) {
  const bool bf = dtype == PYR_BF16;
#define PYR_CASE(D_, G_) if (p.D == D_ && p.group == G_) return bf ? f.template run<__nv_bfloat16, D_, G_>() : f.template run<float, D_, G_>();
  PYR_CASE(128, 32) PYR_CASE(128, 64) PYR_CASE(128, 128) PYR_CASE(64, 32) PYR_CASE(64, 64)
#undef PYR_CASE
  return cudaErrorInvalidValue;
}

struct RunWrite {
  const PagesWriteArgs& a; int blocks; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D, int G> cudaError_t run() {
    return launch_behind(write_rows_kernel<T, D, G>, dim3(grid), dim3(kTileThreads), 0, s, a, blocks, items);
  }
};
struct RunFew {
  const PagesWriteArgs& a; cudaStream_t s;
  template <class T, int D, int G> cudaError_t run() {
    write_few_kernel<T, D, G><<<a.n, kRowThreads, 0, s>>>(a);
    return cudaGetLastError();
  }
};
struct RunRead {
  const PagesWriteArgs& a; int blocks; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D, int G> cudaError_t run() {
    read_rows_kernel<T, D, G><<<grid, kTileThreads, 0, s>>>(a, blocks, items);
    return cudaGetLastError();
  }
};

// Tiles that cover n rows from any row of a tile on.
inline int tiles_over(int n) { return (n + 2 * kPageTile - 2) / kPageTile; }

}  // namespace

cudaError_t launch_pages_write(const PagesWriteArgs& a, int* launches, cudaStream_t s) {
  const int blocks = tiles_over(a.n_rows);
  cudaError_t e;
  if ((int64_t)a.n_rows * a.p.Hkv <= kFewRows) {
    e = by_format(a.p, a.dtype, RunFew{a, s});
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  const int words = (a.p.n_lists + 31) / 32;
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kTileThreads / 32 - 1) / (kTileThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  e = allow_shared<write_plan_kernel>(2 * (kMaxLists / 32) * 4);
  if (e != cudaSuccess) return e;
  write_plan_kernel<<<1, kPlanThreads, 2 * words * sizeof(uint32_t), s>>>(a, words);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  e = by_format(a.p, a.dtype, RunWrite{a, blocks, items, (unsigned)grid, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_read(const PagesWriteArgs& a, int* launches, cudaStream_t s) {
  const int blocks = tiles_over(a.n_rows);
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kTileThreads / 32 - 1) / (kTileThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = by_format(a.p, a.dtype, RunRead{a, blocks, items, (unsigned)grid, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

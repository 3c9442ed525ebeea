// Rows into and out of the paged 8-bit cache (format: include/pyr.h), with the rotation of positions applied on the way in.
//
// One scale for a page and head, K and V apart: s = max(s_old, amax / 127), s_old the scale of rows that stay in the page. New codes
// are rint(x (1 / s)), within 127 since s and its inverse are rounded by 2^-24 each; where s grows, codes that stay become
// rint(code (s_old / s)), which costs them up to half a step more (with a page filled row by row a scale grows some five times).
// Rotation: (x1, x2) -> (x1 c - x2 s, x2 c + x1 s) on the pairs (i, i + D / 2), in fp32, and codes from that: keys are not
// rounded to bf16 in between. Arithmetic is plain IEEE single precision, never contracted: stored bytes are the same everywhere.
#include <cuda_bf16.h>

#include "pyr_internal.h"

namespace pyr {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kOneWarps = 8;                     // of a CTA that stores an entry's one row, a warp a head
constexpr int kReadThreads = 64;
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100
constexpr float kRound = 12582912.f;             // 1.5 2^23: added, it rounds to the nearest integer (ties to even) and leaves it in the low bits

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// N elements of a row (2 or 4) as they are loaded, and as numbers.
template <class T, int N> struct Some;
template <int N> struct Some<float, N> {
  float x[N];
  __device__ __forceinline__ void load(const float* p) {
    if constexpr (N == 4) { const float4 v = *reinterpret_cast<const float4*>(p); x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w; }
    else { const float2 v = *reinterpret_cast<const float2*>(p); x[0] = v.x; x[1] = v.y; }
  }
  __device__ __forceinline__ void set(float v) {
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = v;
  }
  __device__ __forceinline__ float at(int k) const { return x[k]; }
};
template <int N> struct Some<__nv_bfloat16, N> {
  uint32_t w[N / 2];
  __device__ __forceinline__ void load(const __nv_bfloat16* p) {
    if constexpr (N == 4) { const uint2 v = *reinterpret_cast<const uint2*>(p); w[0] = v.x; w[1] = v.y; }
    else w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  __device__ __forceinline__ void set(float v) {
    const uint32_t b = __float_as_uint(v) >> 16;
#pragma unroll
    for (int k = 0; k < N / 2; ++k) w[k] = b | b << 16;
  }
  __device__ __forceinline__ float at(int k) const { return __uint_as_float(k & 1 ? w[k >> 1] & 0xffff0000u : w[k >> 1] << 16); }
};
template <int N> __device__ __forceinline__ void store_some(float* p, const float* x) {
  if constexpr (N == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  else *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  return (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(lo)) | (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(hi)) << 16;
}
template <int N> __device__ __forceinline__ void store_some(__nv_bfloat16* p, const float* x) {
  if constexpr (N == 4) *reinterpret_cast<uint2*>(p) = make_uint2(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]));
  else *reinterpret_cast<uint32_t*>(p) = two_bf16(x[0], x[1]);
}

// N pairs (lo, hi) turned by the angles whose cosines and sines lie at rope[d0 ..] and rope[D / 2 + d0 ..].
template <int N, int D>
__device__ __forceinline__ void rotate(float* lo, float* hi, const float* rope, int d0) {
  Some<float, N> c, s;
  c.load(rope + d0);
  s.load(rope + D / 2 + d0);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float a = lo[k], b = hi[k];
    lo[k] = __fsub_rn(__fmul_rn(a, c.x[k]), __fmul_rn(b, s.x[k]));
    hi[k] = __fadd_rn(__fmul_rn(b, c.x[k]), __fmul_rn(a, s.x[k]));
  }
}

// The scale that rows with the largest magnitude amax bring a (page, head) to, from `before`; what codes that stay and new values are
// multiplied by.
struct Scale { float s, factor, inverse; };
__device__ __forceinline__ Scale scale_of(float amax, float before) {
  Scale r;
  float want = __fdiv_rn(amax, 127.f);
  if (want < kScaleMin) want = 0.f;
  r.s = amax <= 3.402823466e38f && before == before ? fmaxf(before, want) : nan_f();
  const bool some = r.s > 0.f;                   // (not so for NaN: every code 0)
  r.factor = some ? __fdiv_rn(before, r.s) : 0.f;
  r.inverse = some ? __fdiv_rn(1.f, r.s) : 0.f;
  return r;
}
// A code in the low byte (two's complement), from its number times 1 / step; the sums are monotone in the number.
__device__ __forceinline__ float code_sum(float x, float by) { return __fadd_rn(__fmul_rn(x, by), kRound); }
__device__ __forceinline__ int code_int(float sum) { return (int)(__float_as_uint(sum) - 0x4B400000u); }
// Four stored bytes (code + 128) brought to another scale.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float factor) {
  uint32_t r = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) r |= (__float_as_uint(code_sum((float)((int)(w >> (8 * k) & 255u) - 128), factor)) & 255u) << (8 * k);
  return r ^ 0x80808080u;
}
__device__ __forceinline__ uint32_t bytes4(float a, float b, float c, float d) {      // their low bytes
  return __byte_perm(__byte_perm(__float_as_uint(a), __float_as_uint(b), 0x0040), __byte_perm(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
}

__device__ __forceinline__ uint8_t* head_of(const PagesView& p, int page, int h) { return p.pool + pages_tile(p, page, h, 0) - p.head_extra; }
template <class T>
__device__ __forceinline__ const T* source(const void* p, const PagesWriteArgs& a, int e, int h) {
  return static_cast<const T*>(p) + (int64_t)e * a.sb + (int64_t)h * a.sh;
}
// Where entry e's row x of head h comes from, and its position (0 without positions): -1 where either is out of range.
__device__ __forceinline__ int source_row(const PagesWriteArgs& a, int e, int h, int x) {
  const int src = a.idx ? a.idx[(int64_t)e * a.idx_stride + (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows + x] : x;
  return src >= 0 && src < a.src_rows ? src : -1;
}
__device__ __forceinline__ int position(const PagesAppendArgs& a, int e, int h, int x) {
  if (!a.pos) return 0;
  const int pos = a.pos[(int64_t)e * a.pos_stride + (int64_t)(a.w.idx_groups == 1 ? 0 : h) * a.w.n_rows + x];
  return pos >= 0 && pos < a.n_pos ? pos : -1;
}

// One query row by 16 threads: turned by its position (-1: NaN) if `stored`, as it is otherwise.
template <class T, int D>
__device__ __forceinline__ void query_row(const PagesAppendArgs& a, int e, int x, int head, int lane16, bool stored) {
  constexpr int W = D / 32;
  const T* q = static_cast<const T*>(a.q) + (int64_t)e * a.qsb + (int64_t)x * a.qsn + (int64_t)head * a.qsh;
  T* out = static_cast<T*>(a.q_out) + (int64_t)e * a.osb + (int64_t)x * a.osn + (int64_t)head * a.osh;
  const int d0 = W * lane16;
  Some<T, W> lo, hi;
  lo.load(q + d0);
  hi.load(q + D / 2 + d0);
  float f[2][W];
#pragma unroll
  for (int k = 0; k < W; ++k) { f[0][k] = lo.at(k); f[1][k] = hi.at(k); }
  if (stored) {
    const int pos = position(a, e, 0, x);
    if (pos >= 0) {
      rotate<W, D>(f[0], f[1], a.rope + (int64_t)pos * D, d0);
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) f[0][k] = f[1][k] = nan_f();
    }
  }
  store_some<W>(out + d0, f[0]);
  store_some<W>(out + D / 2 + d0, f[1]);
}

// ------------------------------------------------------------------ one row an entry (a decode step)
// grid (entries, groups of kOneWarps heads and then groups of query heads). Every CTA of an entry decides for itself; the one that
// is done last sets the length, which the others have read by then. A warp stores a head: its lower half the key, its upper half
// the value, a thread D / 32 dimensions from either half of them.
template <class T, int D>
__global__ void __launch_bounds__(kOneWarps * 32) append_one_kernel(PagesAppendArgs p, int kv_parts) {
  constexpr int W = D / 32;
  const PagesWriteArgs& a = p.w;
  const int e = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int l = pages_list(a.p, a.lists, e);
  const int cnt = a.counts ? a.counts[e] : 1;
  bool bad = l < 0 || cnt < 0 || cnt > 1;
  int row = 0, len = 0, page = -1;
  if (!bad) {
    len = pages_len(a.p, l);
    row = a.first ? a.first[e] : len;
    bad = row < 0 || row > len || (int64_t)row + cnt > (int64_t)a.p.max_pages * a.p.page_rows;
    if (!bad && cnt > 0) {
      page = pages_page(a.p, l, row / a.p.page_rows);
      bad = page < 0 || a.p.refs[page] != 1;
    }
  }
  if (a.lists)
#pragma unroll 4
    for (int x = t; x < a.n; x += kOneWarps * 32) bad |= x != e && a.lists[x] == l;
  bad = __syncthreads_or(bad);                    // (all threads have read the length by now)
  if (t == 0) {
    if (bad && blockIdx.y == 0) record(a.p.status, PYR_ERR_INVALID);
    const bool last = gridDim.y == 1 || atomicAdd(&p.done[e], 1) == (int)gridDim.y - 1;
    if (last) {
      if (gridDim.y > 1) p.done[e] = 0;
      if (!bad && row + cnt > len) a.p.lens[l] = row + cnt;
    }
  }
  if ((int)blockIdx.y >= kv_parts) {
    const int head = ((int)blockIdx.y - kv_parts) * (2 * kOneWarps) + (t >> 4);
    if (head < p.Hq) query_row<T, D>(p, e, 0, head, t & 15, !bad && cnt > 0);
    return;
  }
  const int h = blockIdx.y * kOneWarps + warp;
  if (bad || cnt == 0 || h >= a.p.Hkv) return;
  const int kv = lane >> 4, d0 = W * (lane & 15);
  const int src = source_row(a, e, h, 0), pos = position(p, e, h, 0);
  float x[2][W];
  if (src >= 0 && pos >= 0) {
    const T* from = source<T>(kv ? a.v : a.k, a, e, h) + (int64_t)src * a.sn;
    Some<T, W> lo, hi;
    lo.load(from + d0);
    hi.load(from + D / 2 + d0);
#pragma unroll
    for (int k = 0; k < W; ++k) { x[0][k] = lo.at(k); x[1][k] = hi.at(k); }
    if (p.pos && kv == 0) rotate<W, D>(x[0], x[1], p.rope + (int64_t)pos * D, d0);
  } else {
    if (lane == 0) record(a.p.status, PYR_ERR_INVALID);
#pragma unroll
    for (int k = 0; k < W; ++k) x[0][k] = x[1][k] = nan_f();
  }
  float amax = 0.f;
#pragma unroll
  for (int k = 0; k < W; ++k) amax = max_nan(amax, max_nan(fabsf(x[0][k]), fabsf(x[1][k])));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) amax = max_nan(amax, __shfl_xor_sync(0xffffffffu, amax, o));

  const int pr = a.p.page_rows, in = row % pr;
  const int64_t page0 = row - in;
  const int upto = (int)(min((int64_t)len, page0 + pr) - page0);    // rows of the list in this page before (none: 0 or less)
  const bool held = in > 0 || upto > in + 1;
  uint8_t* head = head_of(a.p, page, h);
  uint8_t* tile = head + a.p.head_extra + in / kPageTile * a.p.tile_bytes;
  const int r = in % kPageTile, D2 = 2 * D;
  const float before = held ? reinterpret_cast<const float*>(head + D2)[kv] : 0.f;
  const Scale sc = scale_of(amax, before);
  const bool grows = held && !(sc.s == before);
  if (grows) {                                    // rare: rows that stay go to the new scale, whatever their order in the tiles
    const int tiles = (max(upto, in + 1) + kPageTile - 1) / kPageTile;
    for (int b = 0; b < tiles; ++b) {
      uint8_t* other = head + a.p.head_extra + b * a.p.tile_bytes;
      uint4* codes = reinterpret_cast<uint4*>(other + kv * kPageTile * D);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        uint4 w = codes[i * 16 + (lane & 15)];
        w.x = recode4(w.x, sc.factor); w.y = recode4(w.y, sc.factor); w.z = recode4(w.z, sc.factor); w.w = recode4(w.w, sc.factor);
        codes[i * 16 + (lane & 15)] = w;
      }
      if ((lane & 15) == 0) reinterpret_cast<float*>(other + tile8_scales(D))[kv] = sc.s;
    }
  }
  __syncwarp();
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int d = half * (D / 2) + d0;
    int c[W];
#pragma unroll
    for (int k = 0; k < W; ++k) c[k] = sc.s == sc.s ? code_int(code_sum(x[half][k], sc.inverse)) : 0;
    if (kv == 0) {
      uint8_t* at = tile + tile8_k(D, r, d);
      if constexpr (W == 4) *reinterpret_cast<uchar4*>(at) = make_uchar4(c[0] + 128, c[1] + 128, c[2] + 128, c[3] + 128);
      else *reinterpret_cast<uchar2*>(at) = make_uchar2(c[0] + 128, c[1] + 128);
      int8_t* ends = reinterpret_cast<int8_t*>(head);
#pragma unroll
      for (int k = 0; k < W; ++k) {
        int lo = c[k], hi = c[k];
        if (held) {
          lo = min(lo, code_int(code_sum((float)ends[d + k], sc.factor)));
          hi = max(hi, code_int(code_sum((float)ends[D + d + k], sc.factor)));
        }
        ends[d + k] = (int8_t)lo;
        ends[D + d + k] = (int8_t)hi;
      }
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) tile[tile8_v(D, r, d + k)] = (uint8_t)(c[k] + 128);
    }
  }
  if ((lane & 15) == 0) {
    reinterpret_cast<float*>(head + D2)[kv] = sc.s;
    reinterpret_cast<float*>(tile + tile8_scales(D))[kv] = sc.s;
  }
}

// ------------------------------------------------------------------ many rows
// Decides every entry before any row moves: plan[2 i] = first row (-1: refused), plan[2 i + 1] = the length before. A warp per entry.
__global__ void __launch_bounds__(kPlanThreads) append_plan_kernel(PagesWriteArgs a, int words) {
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
      a.plan[2 * i] = ok ? start : -1;
      a.plan[2 * i + 1] = len;
      if (ok) { if (start + cnt > len) a.p.lens[l] = start + cnt; }
      else record(a.p.status, PYR_ERR_INVALID);
    }
  }
}

// The row of a tile that a thread holds as its p-th (of 8): four after the other are the bytes of a V word, in the order 0, 2, 1, 3.
__device__ __forceinline__ int tile_row(int half, int p) { return 4 * half + 2 * (p >> 2) + (p & 1) + 8 * (p >> 1 & 1); }

// One CTA per (entry, KV head, page), a warp per tile; heads side by side, whose rows lie side by side. A thread holds D / 32
// dimensions from either half of eight rows: both members of the rotation's pairs, and whole words of V. `pages` cover n_rows
// rows wherever in a page they begin. CTAs from `items` on turn queries.
template <class T, int D>
__global__ void __launch_bounds__(kPageRows8 * 2) append_pages_kernel(PagesAppendArgs p, int pages, int64_t items) {
  constexpr int W = D / 32;
  __shared__ float top[2][kPageRows8 / kPageTile];
  __shared__ int8_t ends[kPageRows8 / kPageTile][2][D];
  const PagesWriteArgs& a = p.w;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, half = lane >> 4, d0 = W * (lane & 15), pr = a.p.page_rows;
  wait_for_previous();
  if (blockIdx.x >= items) {
    const int64_t unit = ((int64_t)blockIdx.x - items) * (blockDim.x / 16) + (t >> 4);
    const int64_t at = unit / p.Hq;
    if (at >= (int64_t)a.n * a.n_rows) return;
    const int e = (int)(at / a.n_rows), x = (int)(at - (int64_t)e * a.n_rows);
    query_row<T, D>(p, e, x, (int)(unit - at * p.Hq), t & 15, a.plan[2 * e] >= 0 && x < (a.counts ? a.counts[e] : a.n_rows));
    return;
  }
  const int h = (int)(blockIdx.x % a.p.Hkv);
  const int64_t ep = blockIdx.x / a.p.Hkv;
  const int e = (int)(ep / pages);
  const int start = a.plan[2 * e], len = a.plan[2 * e + 1];
  if (start < 0) return;
  const int cnt = a.counts ? a.counts[e] : a.n_rows, end = start + cnt;
  const int slot = start / pr + (int)(ep - (int64_t)e * pages);
  const int64_t page0 = (int64_t)slot * pr;
  if (page0 >= end) return;
  const int page = pages_page(a.p, pages_list(a.p, a.lists, e), slot);
  if (page < 0) return;                           // (the plan has seen a valid page here)
  const int upto = (int)min((int64_t)len, page0 + pr);       // rows of the list that were in this page: up to here
  const bool held = start > page0 || upto > end;
  const int row0 = (int)page0 + warp * kPageTile;

  // ---- this thread's rows: sources and positions by the lane of the row, new ones and those that stay as bits
  int src = -1, pos = -1;
  bool is_new = false, stays = false;
  if (lane < kPageTile) {
    const int row = row0 + lane;
    is_new = row >= start && row < end;
    stays = !is_new && row < upto;
    if (is_new) {
      src = source_row(a, e, h, row - start);
      pos = position(p, e, h, row - start);
      if (src < 0 || pos < 0) { src = -1; record(a.p.status, PYR_ERR_INVALID); }
    }
  }
  const uint32_t news = __ballot_sync(0xffffffffu, is_new), kept = __ballot_sync(0xffffffffu, stays);
  float k[8][2 * W];
  Some<T, W> v[8][2];
  {
    const T* kp = source<T>(a.k, a, e, h) + d0;
    const T* vp = source<T>(a.v, a, e, h) + d0;
#pragma unroll
    for (int b = 0; b < 8; b += 4) {
      Some<T, W> raw[4][2];
      int at[4], ps[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int r = tile_row(half, b + q);
        at[q] = __shfl_sync(0xffffffffu, src, r);
        ps[q] = __shfl_sync(0xffffffffu, pos, r);
        if (at[q] >= 0) {
          const int64_t off = (int64_t)at[q] * a.sn;
          raw[q][0].load(kp + off);
          raw[q][1].load(kp + off + D / 2);
          v[b + q][0].load(vp + off);
          v[b + q][1].load(vp + off + D / 2);
        } else {                                  // not a new row: nothing; one without a source: NaN
          const float x = news >> r & 1u ? nan_f() : 0.f;
          raw[q][0].set(x); raw[q][1].set(x);
          v[b + q][0].set(x); v[b + q][1].set(x);
        }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
#pragma unroll
        for (int i = 0; i < W; ++i) { k[b + q][i] = raw[q][0].at(i); k[b + q][W + i] = raw[q][1].at(i); }
        if (p.pos && at[q] >= 0) rotate<W, D>(k[b + q], k[b + q] + W, p.rope + (int64_t)ps[q] * D, d0);
      }
    }
  }
  float mk = 0.f, mv = 0.f;
#pragma unroll
  for (int q = 0; q < 8; ++q)
#pragma unroll
    for (int i = 0; i < W; ++i) {
      mk = max_nan(mk, max_nan(fabsf(k[q][i]), fabsf(k[q][W + i])));
      mv = max_nan(mv, max_nan(fabsf(v[q][0].at(i)), fabsf(v[q][1].at(i))));
    }
  // (magnitudes, Inf and NaN among them, are ordered as their bits are)
  const uint32_t bk = __reduce_max_sync(0xffffffffu, __float_as_uint(mk) & 0x7fffffffu);
  const uint32_t bv = __reduce_max_sync(0xffffffffu, __float_as_uint(mv) & 0x7fffffffu);
  if (lane == 0) { top[0][warp] = __uint_as_float(bk); top[1][warp] = __uint_as_float(bv); }
  uint8_t* head = head_of(a.p, page, h);
  const float2 old = *reinterpret_cast<const float2*>(head + 2 * D);
  __syncthreads();                                // (the old scales are read, too)
  const int warps = a.p.tiles_per_page;
  uint32_t ak = 0, av = 0;
  for (int w = 0; w < warps; ++w) { ak = max(ak, __float_as_uint(top[0][w])); av = max(av, __float_as_uint(top[1][w])); }
  const float before_k = held ? old.x : 0.f, before_v = held ? old.y : 0.f;
  const Scale sk = scale_of(__uint_as_float(ak), before_k), sv = scale_of(__uint_as_float(av), before_v);

  // ---- codes
  uint8_t* tile = head + a.p.head_extra + warp * a.p.tile_bytes;
  constexpr float kNone = kRound;                 // the sum of code 0
  const bool fine_k = sk.s == sk.s, fine_v = sv.s == sv.s;
  float lo[2 * W], hi[2 * W];
#pragma unroll
  for (int i = 0; i < 2 * W; ++i) { lo[i] = kRound + 127.f; hi[i] = kRound - 127.f; }
  if (news || (kept && !(sk.s == before_k))) {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const int r = tile_row(half, q);
      const bool fresh = news >> r & 1u, stay = kept >> r & 1u;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        uint8_t* at = tile + tile8_k(D, r, g * (D / 2) + d0);
        float c[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          c[i] = fine_k ? code_sum(k[q][g * W + i], sk.inverse) : kNone;
          if (fresh) { lo[g * W + i] = fminf(lo[g * W + i], c[i]); hi[g * W + i] = fmaxf(hi[g * W + i], c[i]); }
        }
        uint32_t w;
        if constexpr (W == 4) w = bytes4(c[0], c[1], c[2], c[3]) ^ 0x80808080u;
        else w = __byte_perm(__float_as_uint(c[0]), __float_as_uint(c[1]), 0x0040) ^ 0x8080u;
        if constexpr (W == 4) {
          if (stay) w = recode4(*reinterpret_cast<const uint32_t*>(at), sk.factor);
          *reinterpret_cast<uint32_t*>(at) = w;
        } else {
          if (stay) w = recode4(*reinterpret_cast<const uint16_t*>(at), sk.factor);
          *reinterpret_cast<uint16_t*>(at) = (uint16_t)w;
        }
      }
    }
  }
  if (news || (kept && !(sv.s == before_v))) {
    const uint32_t mine = half ? 0xF0F0u : 0x0F0Fu;           // this thread's rows
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t* at = reinterpret_cast<uint32_t*>(tile + tile8_v(D, tile_row(half, 4 * j), g * (D / 2) + d0));
        uint32_t w[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
          float c[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) c[q] = fine_v ? code_sum(v[4 * j + q][g].at(i), sv.inverse) : kNone;
          w[i] = bytes4(c[0], c[2], c[1], c[3]) ^ 0x80808080u;
        }
        if (kept & mine) {
          uint32_t from = 0;                      // bytes of rows that stay
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int r = tile_row(half, 4 * j + q), b = 2 * (r & 1) + (r >> 3);
            if (kept >> r & 1u) from |= 255u << (8 * b);
          }
#pragma unroll
          for (int i = 0; i < W; ++i) w[i] = (w[i] & ~from) | (recode4(at[i], sv.factor) & from);
        }
        if constexpr (W == 4) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
      }
  }
  if (lane == 0 && (news | kept)) *reinterpret_cast<float2*>(tile + tile8_scales(D)) = make_float2(sk.s, sv.s);

  // ---- extrema of the codes, a dimension a thread
#pragma unroll
  for (int i = 0; i < 2 * W; ++i) {
    lo[i] = fminf(lo[i], __shfl_xor_sync(0xffffffffu, lo[i], 16));
    hi[i] = fmaxf(hi[i], __shfl_xor_sync(0xffffffffu, hi[i], 16));
  }
  if (half == 0)
#pragma unroll
    for (int g = 0; g < 2; ++g)
#pragma unroll
      for (int i = 0; i < W; ++i) {
        ends[warp][0][g * (D / 2) + d0 + i] = (int8_t)code_int(lo[g * W + i]);
        ends[warp][1][g * (D / 2) + d0 + i] = (int8_t)code_int(hi[g * W + i]);
      }
  __syncthreads();
  int8_t* kept_ends = reinterpret_cast<int8_t*>(head);
  for (int d = t; d < D; d += blockDim.x) {
    int least = 127, most = -127;
    for (int w = 0; w < warps; ++w) { least = min(least, (int)ends[w][0][d]); most = max(most, (int)ends[w][1][d]); }
    if (held) {
      least = min(least, code_int(code_sum((float)kept_ends[d], sk.factor)));
      most = max(most, code_int(code_sum((float)kept_ends[D + d], sk.factor)));
    }
    kept_ends[d] = (int8_t)least;
    kept_ends[D + d] = (int8_t)most;
  }
  if (t == 0) *reinterpret_cast<float2*>(head + 2 * D) = make_float2(sk.s, sv.s);
}

// ------------------------------------------------------------------ rows as values
// One warp per (entry, KV head, tile of its list): a lane takes 16 dimensions of a row of K, four dimensions of four rows of V.
template <class T, int D>
__global__ void __launch_bounds__(kReadThreads) read8_kernel(PagesWriteArgs a, int blocks, int64_t items) {
  constexpr int P = D / 32, E = D / 8;
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kReadThreads / 32) + (threadIdx.x >> 5);
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
  const int64_t tile_row0 = (int64_t)first / kPageTile * kPageTile + (int64_t)blk * kPageTile;
  if (tile_row0 >= end) return;
  const int row0 = (int)tile_row0;
  const int page = pages_page(a.p, l, row0 / a.p.page_rows);
  if (page < 0) {
    if (lane == 0) record(a.p.status, PYR_ERR_INVALID);
    return;
  }
  const uint8_t* tile = a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile);
  T* k = const_cast<T*>(source<T>(a.k, a, e, h));
  T* v = const_cast<T*>(source<T>(a.v, a, e, h));
  const float2 scale = *reinterpret_cast<const float2*>(tile + tile8_scales(D));
  uint4 kc[P], vc[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    kc[i] = reinterpret_cast<const uint4*>(tile)[i * 32 + lane];
    vc[i] = reinterpret_cast<const uint4*>(tile + kPageTile * D)[i * 32 + lane];
  }
  auto value = [](uint32_t w, int b, float s) { return __fmul_rn((float)((int)(w >> (8 * b) & 255u) - 128), s); };
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int piece = i * 32 + lane, r = piece / (D / 16), x = (piece % (D / 16)) ^ (D == 128 ? 4 * (r & 1) : 0), row = row0 + r;
    if (row < first || row >= end) continue;
    const uint32_t w[4] = {kc[i].x, kc[i].y, kc[i].z, kc[i].w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float f[4] = {value(w[q], 0, scale.x), value(w[q], 1, scale.x), value(w[q], 2, scale.x), value(w[q], 3, scale.x)};
      store_some<4>(k + (int64_t)(row - first) * a.sn + 16 * x + 4 * q, f);
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int piece = i * 32 + lane, j = piece / (D / 4), in = piece % (D / 4);
    const int d = in / (E / 4) * E + 4 * ((in % (E / 4)) ^ (j & (E / 4 - 1)));
    const uint32_t w[4] = {vc[i].x, vc[i].y, vc[i].z, vc[i].w};
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int row = row0 + 2 * j + (b >> 1) + 8 * (b & 1);
      if (row < first || row >= end) continue;
      const float f[4] = {value(w[0], b, scale.y), value(w[1], b, scale.y), value(w[2], b, scale.y), value(w[3], b, scale.y)};
      store_some<4>(v + (int64_t)(row - first) * a.sn + d, f);
    }
  }
}

template <class F>
cudaError_t by_format(const PagesView& p, int dtype, F f) {
  const bool bf = dtype == PYR_BF16;
  if (p.D == 128) return bf ? f.template run<__nv_bfloat16, 128>() : f.template run<float, 128>();
  if (p.D == 64) return bf ? f.template run<__nv_bfloat16, 64>() : f.template run<float, 64>();
  return cudaErrorInvalidValue;
}

struct RunOne {
  const PagesAppendArgs& a; int kv_parts, parts; cudaStream_t s;
  template <class T, int D> cudaError_t run() {
    append_one_kernel<T, D><<<dim3(a.w.n, parts), kOneWarps * 32, 0, s>>>(a, kv_parts);
    return cudaGetLastError();
  }
};
struct RunPages {
  const PagesAppendArgs& a; int pages; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D> cudaError_t run() {
    return launch_behind(append_pages_kernel<T, D>, dim3(grid), dim3(2 * a.w.p.page_rows), 0, s, a, pages, items);
  }
};
struct RunRead {
  const PagesWriteArgs& a; int blocks; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D> cudaError_t run() {
    read8_kernel<T, D><<<grid, kReadThreads, 0, s>>>(a, blocks, items);
    return cudaGetLastError();
  }
};

__global__ void rope_table_kernel(float* table, int64_t first, int64_t n_pos, int half, double base) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n_pos * half) return;
  const int64_t at = i / half;
  const int d = (int)(i - at * half);
  double s, c;
  sincos((double)(first + at) * pow(base, -(double)d / (double)half), &s, &c);
  table[at * 2 * half + d] = (float)c;
  table[at * 2 * half + half + d] = (float)s;
}

}  // namespace

cudaError_t launch_pages_append8(const PagesAppendArgs& a, int* launches, cudaStream_t s) {
  const PagesWriteArgs& w = a.w;
  cudaError_t e;
  if (w.n_rows == 1) {
    const int kv_parts = (w.p.Hkv + kOneWarps - 1) / kOneWarps;
    const int parts = kv_parts + (a.q ? (a.Hq + 2 * kOneWarps - 1) / (2 * kOneWarps) : 0);
    if (parts > 65535) return cudaErrorInvalidValue;
    e = by_format(w.p, w.dtype, RunOne{a, kv_parts, parts, s});
    if (e == cudaSuccess) ++*launches;
    return e;
  }
  const int words = (w.p.n_lists + 31) / 32, pr = w.p.page_rows;
  const int pages = (int)(((int64_t)w.n_rows + pr - 2) / pr) + 1;
  const int64_t items = (int64_t)w.n * w.p.Hkv * pages;
  const int64_t queries = a.q ? ((int64_t)w.n * w.n_rows * a.Hq + 2 * pr / 16 - 1) / (2 * pr / 16) : 0;
  if (items + queries > 0x7fffffffLL) return cudaErrorInvalidValue;
  e = allow_shared<append_plan_kernel>(2 * (kMaxLists / 32) * 4);
  if (e != cudaSuccess) return e;
  append_plan_kernel<<<1, kPlanThreads, 2 * words * sizeof(uint32_t), s>>>(w, words);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  e = by_format(w.p, w.dtype, RunPages{a, pages, items, (unsigned)(items + queries), s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_read8(const PagesWriteArgs& a, int* launches, cudaStream_t s) {
  const int blocks = (int)(((int64_t)a.n_rows + 2 * kPageTile - 2) / kPageTile);
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kReadThreads / 32 - 1) / (kReadThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = by_format(a.p, a.dtype, RunRead{a, blocks, items, (unsigned)grid, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_glue_rope_table(float* table, int64_t first, int64_t n_pos, int D, double base, cudaStream_t s) {
  const int64_t grid = (n_pos * (D / 2) + 255) / 256;            // (2^31 positions of 128 pairs: 2^30)
  rope_table_kernel<<<(unsigned)grid, 256, 0, s>>>(table, first, n_pos, D / 2, base);
  return cudaGetLastError();
}

}  // namespace pyr

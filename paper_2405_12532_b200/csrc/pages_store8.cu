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
constexpr int kSelfEntries = 256;                // up to this many entries each CTA may decide for itself, and a call of many rows is one launch
constexpr int kQueryHeads = 4;                   // heads of a query row that a thread turns
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100
constexpr float kRound = 12583040.f;             // 1.5 2^23 + 128: added, it rounds to the nearest integer (ties to even) and leaves it, plus 128, in the low bits

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7FC00000u); }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The largest magnitude of three, NaN if one is NaN.
__device__ __forceinline__ float most_of(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float min_of(float a, float b, float c) {
  float r;
  asm("min.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max_of(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// Two numbers at once, each rounded as alone. A sum is a product with `one` = 1 (or -1), which the kernel gets as an argument: packed
// products and sums are otherwise contracted when they are assembled (measured: rounded once), and so are products with a constant 1.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 x, y, z;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmul.rn.f32x2 z, x, y;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b, float one) {        // a + one b
  float2 r;
  asm("{\n.reg .b64 x, y, z, w;\nmov.b64 x, {%2, %3};\nmov.b64 y, {%4, %5};\nmov.b64 w, {%6, %6};\nfma.rn.f32x2 z, y, w, x;\nmov.b64 {%0, %1}, z;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(one));
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
  __device__ __forceinline__ float2 two(int k) const { return make_float2(x[2 * k], x[2 * k + 1]); }
  // the bits of the largest magnitude so far (Inf and NaN in the order of their bits)
  __device__ __forceinline__ void most(uint32_t* bits) const {
    float m = __uint_as_float(*bits);
#pragma unroll
    for (int k = 0; k < N; k += 2) m = most_of(m, x[k], x[k + 1]);
    *bits = __float_as_uint(m);
  }
  static __device__ __forceinline__ uint32_t finish(uint32_t bits) { return bits & 0x7fffffffu; }
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
  __device__ __forceinline__ float2 two(int k) const { return make_float2(at(2 * k), at(2 * k + 1)); }
  // (two at a time, until finish())
  __device__ __forceinline__ void most(uint32_t* bits) const {
    if constexpr (N == 4) *bits = __vimax3_u16x2(*bits, w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu);
    else *bits = __vmaxu2(*bits, w[0] & 0x7fff7fffu);
  }
  static __device__ __forceinline__ uint32_t finish(uint32_t bits) { return max(bits & 0xffff0000u, bits << 16); }
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

__device__ __forceinline__ void store_eight(float* p, const float* x) { store_some<4>(p, x); store_some<4>(p + 4, x + 4); }
__device__ __forceinline__ void store_eight(__nv_bfloat16* p, const float* x) {
  *reinterpret_cast<uint4*>(p) = make_uint4(two_bf16(x[0], x[1]), two_bf16(x[2], x[3]), two_bf16(x[4], x[5]), two_bf16(x[6], x[7]));
}

// N pairs (lo, hi) turned by the angles whose cosines and sines lie at rope[d0 ..] and rope[D / 2 + d0 ..].
template <int N>
__device__ __forceinline__ void turn(float* lo, float* hi, const Some<float, N>& c, const Some<float, N>& s) {
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const float a = lo[k], b = hi[k];
    lo[k] = __fsub_rn(__fmul_rn(a, c.x[k]), __fmul_rn(b, s.x[k]));
    hi[k] = __fadd_rn(__fmul_rn(b, c.x[k]), __fmul_rn(a, s.x[k]));
  }
}
template <int N, int D>
__device__ __forceinline__ void rotate(float* lo, float* hi, const float* rope, int d0) {
  Some<float, N> c, s;
  c.load(rope + d0);
  s.load(rope + D / 2 + d0);
  turn<N>(lo, hi, c, s);
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
  r.factor = some && before > 0.f ? __fdiv_rn(before, r.s) : 0.f;
  r.inverse = some ? __fdiv_rn(1.f, r.s) : 0.f;
  return r;
}
// A code's stored byte in the low byte, from its number times 1 / step; the sums are monotone in the number.
__device__ __forceinline__ float code_sum(float x, float by) { return __fadd_rn(__fmul_rn(x, by), kRound); }
__device__ __forceinline__ float2 code_sums(float2 x, float by, float one) {
  return add2(make_float2(kRound, kRound), mul2(x, make_float2(by, by)), one);
}
__device__ __forceinline__ int code_int(float sum) { return (int)(__float_as_uint(sum) - 0x4B400080u); }
// Two codes' stored bytes as 16-bit halves, from their sums; four bytes from two of those.
__device__ __forceinline__ uint32_t halves2(float2 c) { return __byte_perm(__float_as_uint(c.x), __float_as_uint(c.y), 0x5410); }
__device__ __forceinline__ uint32_t bytes_of(uint32_t lo, uint32_t hi) { return __byte_perm(lo, hi, 0x6420); }
// Four stored bytes (code + 128) brought to another scale.
__device__ __forceinline__ uint32_t recode4(uint32_t w, float factor) {
  uint32_t r = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) r |= (__float_as_uint(code_sum((float)((int)(w >> (8 * k) & 255u) - 128), factor)) & 255u) << (8 * k);
  return r;
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

// Whether entry e is stored, where and how long its list was, decided by a whole CTA.
struct Entry { int list, start, count, len; bool bad; };
__device__ __forceinline__ Entry decide(const PagesWriteArgs& a, int e) {
  Entry d{pages_list(a.p, a.lists, e), 0, a.counts ? a.counts[e] : a.n_rows, 0, false};
  bool bad = d.list < 0 || d.count < 0 || d.count > a.n_rows;
  if (!bad) {
    d.len = pages_len(a.p, d.list);
    d.start = a.first ? a.first[e] : d.len;
    bad = d.start < 0 || d.start > d.len || (int64_t)d.start + d.count > (int64_t)a.p.max_pages * a.p.page_rows;
    if (!bad && d.count > 0)
      for (int s = d.start / a.p.page_rows + threadIdx.x; s <= (d.start + d.count - 1) / a.p.page_rows; s += blockDim.x) {
        const int page = pages_page(a.p, d.list, s);
        bad |= page < 0 || a.p.refs[page] != 1;
      }
  }
  if (a.lists)
#pragma unroll 4
    for (int x = threadIdx.x; x < a.n; x += blockDim.x) bad |= x != e && a.lists[x] == d.list;
  d.bad = __syncthreads_or(bad);
  return d;
}
// Called once by every CTA of an entry, after decide(): the last of `ctas` sets the length, which the others have read by then, and
// reports what is wrong.
__device__ __forceinline__ void finish(const PagesWriteArgs& a, int e, const Entry& d, int32_t* all_done, int ctas) {
  int32_t* done = all_done + e;
  if (threadIdx.x != 0 || (ctas > 1 && atomicAdd(done, 1) != ctas - 1)) return;
  if (ctas > 1) *done = 0;
  a.plan[2 * e] = d.bad ? -1 : d.start;           // for what comes behind
  if (d.bad) record(a.p.status, PYR_ERR_INVALID);
  else if (d.start + d.count > d.len) a.p.lens[d.list] = d.start + d.count;
}

// ------------------------------------------------------------------ one row an entry (a decode step)
// Bound by its launch and a chain of loads (list, length, page, header): 64 lists of 32 heads with queries 6.8 us in a graph (50.8 by the kernel
// for many rows, which goes through whole pages).
// Every CTA compares its entry's list with all others: n^2 reads for n entries, which count from a thousand on (8 KV and 64 query heads, lists
// named and not: 64 entries 4.7 and 4.5 us, 1024 22.4 and 19.9, 4096 116 and 79, 16 384 925 and 371).
// grid (entries, groups of kOneWarps heads and then groups of query heads). A warp stores a head: its lower half the key, its upper half
// the value, a thread D / 32 dimensions from either half of them.
template <class T, int D>
__global__ void __launch_bounds__(kOneWarps * 32) append_one_kernel(PagesAppendArgs p, int kv_parts) {
  constexpr int W = D / 32;
  const PagesWriteArgs& a = p.w;
  const int e = blockIdx.x, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  // (the row is on its way before anything is decided)
  const bool is_query = (int)blockIdx.y >= kv_parts;
  const int h = blockIdx.y * kOneWarps + warp, kv = lane >> 4, d0 = W * (lane & 15);
  float x[2][W];
  bool good = false;
  if (!is_query && h < a.p.Hkv) {
    const int src = source_row(a, e, h, 0), pos = position(p, e, h, 0);
    good = src >= 0 && pos >= 0;
    if (good) {
      const T* from = source<T>(kv ? a.v : a.k, a, e, h) + (int64_t)src * a.sn;
      Some<T, W> lo, hi;
      lo.load(from + d0);
      hi.load(from + D / 2 + d0);
#pragma unroll
      for (int k = 0; k < W; ++k) { x[0][k] = lo.at(k); x[1][k] = hi.at(k); }
      if (p.pos && kv == 0) rotate<W, D>(x[0], x[1], p.rope + (int64_t)pos * D, d0);
    }
  }
  const Entry d = decide(a, e);
  finish(a, e, d, p.done, gridDim.y);
  if (is_query) {
    const int head = ((int)blockIdx.y - kv_parts) * (2 * kOneWarps) + (t >> 4);
    if (head < p.Hq) query_row<T, D>(p, e, 0, head, t & 15, !d.bad && d.count > 0);
    return;
  }
  if (d.bad || d.count == 0 || h >= a.p.Hkv) return;
  const int row = d.start, len = d.len, page = pages_page(a.p, d.list, row / a.p.page_rows);
  if (!good) {
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
    const int at0 = half * (D / 2) + d0;
    int c[W];
#pragma unroll
    for (int k = 0; k < W; ++k) c[k] = sc.s == sc.s ? code_int(code_sum(x[half][k], sc.inverse)) : 0;
    if (kv == 0) {
      uint8_t* at = tile + tile8_k(D, r, at0);
      if constexpr (W == 4) *reinterpret_cast<uchar4*>(at) = make_uchar4(c[0] + 128, c[1] + 128, c[2] + 128, c[3] + 128);
      else *reinterpret_cast<uchar2*>(at) = make_uchar2(c[0] + 128, c[1] + 128);
      int8_t* ends = reinterpret_cast<int8_t*>(head);
#pragma unroll
      for (int k = 0; k < W; ++k) {
        int lo = c[k], hi = c[k];
        if (held) {
          lo = min(lo, code_int(code_sum((float)ends[at0 + k], sc.factor)));
          hi = max(hi, code_int(code_sum((float)ends[D + at0 + k], sc.factor)));
        }
        ends[at0 + k] = (int8_t)lo;
        ends[D + at0 + k] = (int8_t)hi;
      }
    } else {
#pragma unroll
      for (int k = 0; k < W; ++k) tile[tile8_v(D, r, at0 + k)] = (uint8_t)(c[k] + 128);
    }
  }
  if ((lane & 15) == 0) {
    reinterpret_cast<float*>(head + D2)[kv] = sc.s;
    reinterpret_cast<float*>(tile + tile8_scales(D))[kv] = sc.s;
  }
}

// ------------------------------------------------------------------ many rows
// Decides every entry before any row moves: plan[2 i] = first row (-1: refused), plan[2 i + 1] = the length before. A warp per entry;
// every CTA goes through all of the call's lists for those that are named twice.
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
  for (int i = blockIdx.x * (kPlanThreads / 32) + (t >> 5); i < a.n; i += gridDim.x * (kPlanThreads / 32)) {
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

// A copy of a thread's own from global to shared memory, of as many bytes as a T[W]; what a thread copies only that thread reads.
template <int kBytes>
__device__ __forceinline__ void copy_async(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "n"(kBytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// What bounds it: issue slots that latencies leave empty (52 % busy at 15 warps an SM, 13 instructions a value of K and V; 8 x 2005 gathered rows of
// 40 heads, keys turned: 119 us, 4.2 TB/s, of which packed products and 16-bit extrema took 12). More warps would need fewer registers than the
// rows and their cosines take.
// One CTA per (entry, page, `heads` KV heads one after the other), two warps a tile. A thread holds D / 32 dimensions from either half of
// four rows: both members of the rotation's pairs, and whole words of V. Rows 2 j, 2 j + 1, 2 j + 8 and 2 j + 9 of the tile (j = 0 .. 3 for
// the half warps) are bytes 0, 2, 1 and 3 of its words. Rows come through shared memory, with two `stages` those of the next two heads
// while one is worked on (119 us; with one stage 127). `pages` cover n_rows rows wherever in a page they begin.
template <class T, int D, bool kSelf>
__global__ void __launch_bounds__(kPageRows8 * 4, 1) append_pages_kernel(PagesAppendArgs p, int pages, int heads, int stages, float one) {
  constexpr int W = D / 32;
  using Part = Some<T, W>;
  extern __shared__ __align__(16) uint8_t shared[];         // [stages][warps][16 parts: K's 4 rows x 2 halves, V's][lanes]
  __shared__ uint2 top[kPageRows8 / 8];                     // of warps: largest magnitudes
  __shared__ __align__(16) uint32_t ends[kPageRows8 / 4][2][D / 2];     // of half warps: extrema of their codes, bytes as 16-bit halves
  const PagesWriteArgs& a = p.w;
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, half = lane >> 4, d0 = W * (lane & 15), pr = a.p.page_rows;
  const int chunks = (a.p.Hkv + heads - 1) / heads, per_entry = pages * chunks;
  const int e = (int)(blockIdx.x / per_entry), part = (int)(blockIdx.x - (unsigned)e * per_entry);
  let_next_start();
  Entry d;
  if constexpr (kSelf) {
    d = decide(a, e);
    finish(a, e, d, p.done, per_entry);
  } else {
    wait_for_previous();
    d = Entry{pages_list(a.p, a.lists, e), a.plan[2 * e], a.counts ? a.counts[e] : a.n_rows, a.plan[2 * e + 1], a.plan[2 * e] < 0};
  }
  if (d.bad) return;
  const int h0 = part % chunks * heads, h1 = min(h0 + heads, a.p.Hkv), start = d.start, end = start + d.count;
  const int slot = start / pr + part / chunks;
  const int64_t page0 = (int64_t)slot * pr;
  if (page0 >= end) return;
  const int page = pages_page(a.p, d.list, slot);
  if (page < 0) return;                           // (a valid page has been seen here)
  const int upto = (int)min((int64_t)d.len, page0 + pr);     // rows of the list that were in this page: up to here
  const bool held = start > page0 || upto > end;
  const int row = (int)page0 + (warp >> 1) * kPageTile + lane, j = 2 * (warp & 1) + half;      // (lanes 0 .. 15: the row that a lane looks up)

  // ---- this thread's rows: new ones and those that stay as bits; sources and positions by the lane of the row
  const bool is_new = lane < kPageTile && row >= start && row < end, stays = lane < kPageTile && !is_new && row < upto;
  const uint32_t news = __ballot_sync(0xffffffffu, is_new), kept = __ballot_sync(0xffffffffu, stays);
  auto row_of = [&](int q) { return 2 * j + (q & 1) + 8 * (q >> 1); };
  const bool same = a.idx_groups == 1;            // every head has the same rows
  // where the rows of head `to_copy` come from, looked up an iteration before they are copied; positions of that one and of the one before
  int src = -1, pos = 0, pos_copied = 0;
  auto look_up = [&](int h) {
    if (!is_new || h >= h1) return;
    const int64_t group = same ? 0 : (int64_t)h * a.n_rows;
    src = a.idx ? a.idx[(int64_t)e * a.idx_stride + group + row - start] : row - start;
    pos = p.pos ? p.pos[(int64_t)e * p.pos_stride + group + row - start] : 0;
  };
  Part* const mine = reinterpret_cast<Part*>(shared) + warp * 512 + lane;
  const int stage_parts = blockDim.x * 16;
  int to = 0;                                     // the stage of the next copy
  const T* kp = source<T>(a.k, a, e, h0) + d0;    // of the head that is copied next
  const T* vp = source<T>(a.v, a, e, h0) + d0;
  auto copy = [&] {                               // and checks what has been looked up
    const bool fine = is_new && src >= 0 && src < a.src_rows && (!p.pos || (pos >= 0 && pos < p.n_pos));
    const uint32_t there = __ballot_sync(0xffffffffu, fine);
    pos_copied = fine ? pos : -1;
    Part* dst = mine + to;
    if (there == 0xffffu) {
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t off = (int64_t)__shfl_sync(0xffffffffu, src, row_of(q)) * a.sn;
        const T *kr = kp + off, *vr = vp + off;
        copy_async<sizeof(Part)>(dst + 64 * q, kr);
        copy_async<sizeof(Part)>(dst + 64 * q + 32, kr + D / 2);
        copy_async<sizeof(Part)>(dst + 64 * q + 256, vr);
        copy_async<sizeof(Part)>(dst + 64 * q + 288, vr + D / 2);
      }
    } else {
      if (is_new && !fine) record(a.p.status, PYR_ERR_INVALID);
#pragma unroll 1
      for (int q = 0; q < 4; ++q) {
        const int r = row_of(q), at = __shfl_sync(0xffffffffu, src, r);
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          Part* to_k = dst + 64 * q + 32 * g;
          if (there >> r & 1u) {
            const int64_t off = (int64_t)at * a.sn + g * (D / 2);
            copy_async<sizeof(Part)>(to_k, kp + off);
            copy_async<sizeof(Part)>(to_k + 256, vp + off);
          } else {                                // not a new row: nothing; one without a source: NaN
            Part none;
            none.set(news >> r & 1u ? nan_f() : 0.f);
            *to_k = none;
            to_k[256] = none;
          }
        }
      }
    }
    kp += a.sh;
    vp += a.sh;
    to = stages > 1 ? stage_parts - to : 0;
  };
  Some<float, W> rope[4][2];
  auto fetch_rope = [&] {                         // for the head copied last
    const bool all = __all_sync(0xffffffffu, lane >= kPageTile || pos_copied >= 0);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int at = __shfl_sync(0xffffffffu, pos_copied, row_of(q));
      if (all || at >= 0) {
        rope[q][0].load(p.rope + (int64_t)at * D + d0);
        rope[q][1].load(p.rope + (int64_t)at * D + D / 2 + d0);
      } else {
        rope[q][0].set(1.f);
        rope[q][1].set(0.f);
      }
    }
  };
  look_up(h0);
  copy();
  copies_commit();
  if (p.pos) fetch_rope();
  if (stages > 1) {
    if (!same) look_up(h0 + 1);
    if (h0 + 1 < h1) copy();
    copies_commit();
  }
  uint8_t* head = head_of(a.p, page, h0);
  const int head_bytes = pages_head_bytes(a.p), tile_at = a.p.head_extra + (warp >> 1) * a.p.tile_bytes;
  int from = 0;                                   // the stage that is worked on
  const int warps = 2 * a.p.tiles_per_page;
  float2 old = make_float2(0.f, 0.f);             // scales of rows that stay
  if (held) old = *reinterpret_cast<const float2*>(head + 2 * D);
#pragma unroll 1
  for (int h = h0; h < h1; ++h, head += head_bytes, from = stages > 1 ? stage_parts - from : 0) {
    const Part* part_of = mine + from;            // K: row q's halves at 64 q, 64 q + 32; V's 256 behind
    const float before_k = old.x, before_v = old.y;
    if (held && h + 1 < h1) old = *reinterpret_cast<const float2*>(head + head_bytes + 2 * D);
    if (!same) look_up(h + stages);
    if (stages > 1) copies_wait<1>(); else copies_wait<0>();
    float2 k[4][W];                               // two dimensions each: those of the first half, those of the second
    float mk = 0.f;
    uint32_t mv = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const Part lo = part_of[64 * q], hi = part_of[64 * q + 32];
#pragma unroll
      for (int i = 0; i < W / 2; ++i) {
        float2 x = lo.two(i), y = hi.two(i);
        if (p.pos) {                              // (nothing and NaN stay what they are)
          const float2 c = rope[q][0].two(i), s = rope[q][1].two(i), x0 = x;
          x = add2(mul2(x, c), mul2(y, s), -one);
          y = add2(mul2(y, c), mul2(x0, s), one);
        }
        k[q][i] = x;
        k[q][W / 2 + i] = y;
        mk = most_of(mk, x.x, x.y);
        mk = most_of(mk, y.x, y.y);
      }
      part_of[64 * q + 256].most(&mv);
      part_of[64 * q + 288].most(&mv);
    }
    if (p.pos && !same && stages > 1 && h + 1 < h1) fetch_rope();
    // (magnitudes, Inf and NaN among them, are ordered as their bits are)
    const uint32_t bk = __reduce_max_sync(0xffffffffu, __float_as_uint(mk) & 0x7fffffffu);
    const uint32_t bv = __reduce_max_sync(0xffffffffu, Some<T, W>::finish(mv));
    if (lane == 0) top[warp] = make_uint2(bk, bv);
    __syncthreads();                              // (the old scales are read, too)
    uint2 all = make_uint2(0, 0);
    if (lane < warps) all = top[lane];
    all.x = __reduce_max_sync(0xffffffffu, all.x);
    all.y = __reduce_max_sync(0xffffffffu, all.y);
    // (even lanes K's, odd lanes V's)
    const Scale mine = scale_of(__uint_as_float(lane & 1 ? all.y : all.x), lane & 1 ? before_v : before_k);
    const Scale sk{__shfl_sync(0xffffffffu, mine.s, 0), __shfl_sync(0xffffffffu, mine.factor, 0), __shfl_sync(0xffffffffu, mine.inverse, 0)};
    const Scale sv{__shfl_sync(0xffffffffu, mine.s, 1), __shfl_sync(0xffffffffu, mine.factor, 1), __shfl_sync(0xffffffffu, mine.inverse, 1)};

    // ---- codes
    uint8_t* tile = head + tile_at;
    uint32_t lo2[W], hi2[W];                      // extrema of the codes' bytes, two dimensions to a word
#pragma unroll
    for (int i = 0; i < W; ++i) { lo2[i] = 0x00ff00ffu; hi2[i] = 0; }
    if (news == 0xffffu && sk.s == sk.s && sv.s == sv.s) {
      // a whole tile of new rows (rows of K two by two: their halves lie the other way round in odd rows, with 128 dimensions)
      uint8_t* kat = tile + 2 * j * D + d0;
#pragma unroll
      for (int g = 0; g < 2; ++g) {
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
          uint32_t c[2][W / 2];
#pragma unroll
          for (int i = 0; i < W / 2; ++i) {
            const int x = g * (W / 2) + i;
            c[0][i] = halves2(code_sums(k[q][x], sk.inverse, one));
            c[1][i] = halves2(code_sums(k[q + 1][x], sk.inverse, one));
            lo2[x] = __vimin3_u16x2(lo2[x], c[0][i], c[1][i]);
            hi2[x] = __vimax3_u16x2(hi2[x], c[0][i], c[1][i]);
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            uint8_t* at = kat + y * D + (q >> 1) * (8 * D) + (D / 2) * (D == 128 ? g ^ y : g);
            if constexpr (W == 4) *reinterpret_cast<uint32_t*>(at) = bytes_of(c[y][0], c[y][1]);
            else *reinterpret_cast<uint16_t*>(at) = (uint16_t)bytes_of(c[y][0], 0u);
          }
        }
        uint32_t* vat = reinterpret_cast<uint32_t*>(tile + tile8_v(D, 2 * j, g * (D / 2) + d0));
        uint32_t w[W];
        const Part v[4] = {part_of[256 + 32 * g], part_of[320 + 32 * g], part_of[384 + 32 * g], part_of[448 + 32 * g]};
#pragma unroll
        for (int i = 0; i < W / 2; ++i) {
          float2 c[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) c[q] = code_sums(v[q].two(i), sv.inverse, one);
          w[2 * i] = bytes4(c[0].x, c[2].x, c[1].x, c[3].x);
          w[2 * i + 1] = bytes4(c[0].y, c[2].y, c[1].y, c[3].y);
        }
        if constexpr (W == 4) *reinterpret_cast<uint4*>(vat) = make_uint4(w[0], w[1], w[2], w[3]);
        else *reinterpret_cast<uint2*>(vat) = make_uint2(w[0], w[1]);
      }
    } else {
      const bool fine_k = sk.s == sk.s, fine_v = sv.s == sv.s;
      if (news || (kept && !(sk.s == before_k))) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int r = row_of(q);
          const bool fresh = news >> r & 1u, stay = kept >> r & 1u;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            uint8_t* at = tile + tile8_k(D, r, g * (D / 2) + d0);
            uint32_t c[W / 2];
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
              const int x = g * (W / 2) + i;
              c[i] = fine_k ? halves2(code_sums(k[q][x], sk.inverse, one)) : 0x00800080u;
              if (fresh) { lo2[x] = __vminu2(lo2[x], c[i]); hi2[x] = __vmaxu2(hi2[x], c[i]); }
            }
            if constexpr (W == 4) {
              uint32_t w = bytes_of(c[0], c[1]);
              if (stay) w = recode4(*reinterpret_cast<const uint32_t*>(at), sk.factor);
              *reinterpret_cast<uint32_t*>(at) = w;
            } else {
              uint32_t w = bytes_of(c[0], 0u);
              if (stay) w = recode4(*reinterpret_cast<const uint16_t*>(at), sk.factor);
              *reinterpret_cast<uint16_t*>(at) = (uint16_t)w;
            }
          }
        }
      }
      if (news || (kept && !(sv.s == before_v))) {
        uint32_t from = 0;                        // bytes of rows that stay
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (kept >> row_of(q) & 1u) from |= 255u << (8 * (2 * (q & 1) + (q >> 1)));
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          uint32_t* at = reinterpret_cast<uint32_t*>(tile + tile8_v(D, 2 * j, g * (D / 2) + d0));
          const Part v[4] = {part_of[256 + 32 * g], part_of[320 + 32 * g], part_of[384 + 32 * g], part_of[448 + 32 * g]};
          uint32_t w[W];
#pragma unroll
          for (int i = 0; i < W; ++i) {
            float c[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) c[q] = fine_v ? code_sum(v[q].at(i), sv.inverse) : kRound;
            w[i] = bytes4(c[0], c[2], c[1], c[3]);
          }
          if (from)
#pragma unroll
            for (int i = 0; i < W; ++i) w[i] = (w[i] & ~from) | (recode4(at[i], sv.factor) & from);
          if constexpr (W == 4) *reinterpret_cast<uint4*>(at) = make_uint4(w[0], w[1], w[2], w[3]);
          else *reinterpret_cast<uint2*>(at) = make_uint2(w[0], w[1]);
        }
      }
    }
    if (lane == 0 && (warp & 1) == 0 && (news | kept)) *reinterpret_cast<float2*>(tile + tile8_scales(D)) = make_float2(sk.s, sv.s);

    // ---- the stage is free: rows of the head that takes it
    if (h + stages < h1) {
      copy();
      if (stages == 1 && p.pos && !same) fetch_rope();
    }
    copies_commit();

    // ---- extrema of the half warps' codes
#pragma unroll
    for (int g = 0; g < 2; ++g) {
      const int x = g * (W / 2);
      uint32_t* at = &ends[2 * warp + half][0][(g * (D / 2) + d0) / 2];
      if constexpr (W == 4) {
        *reinterpret_cast<uint2*>(at) = make_uint2(lo2[x], lo2[x + 1]);
        *reinterpret_cast<uint2*>(at + D / 2) = make_uint2(hi2[x], hi2[x + 1]);
      } else {
        at[0] = lo2[x];
        at[D / 2] = hi2[x];
      }
    }
    __syncthreads();
    for (int x = t; x < D; x += blockDim.x) {     // two dimensions' least codes, then their largest
      const bool largest = x >= D / 2;
      const uint32_t flip = largest ? 0x00ff00ffu : 0u;
      const uint32_t* at = &ends[0][0][x];
      uint32_t least = 0x00ff00ffu;
      for (int w = 0; w < 2 * warps; w += 2) least = __vimin3_u16x2(least, at[w * D] ^ flip, at[w * D + D] ^ flip);
      least ^= flip;
      int c[2] = {(int)(least & 255u) - 128, (int)(least >> 16 & 255u) - 128};
      char2* kept_ends = reinterpret_cast<char2*>(head) + x;
      if (held) {
        const char2 was = *kept_ends;
        const int o[2] = {code_int(code_sum((float)was.x, sk.factor)), code_int(code_sum((float)was.y, sk.factor))};
#pragma unroll
        for (int y = 0; y < 2; ++y) c[y] = largest ? max(c[y], o[y]) : min(c[y], o[y]);
      }
      *kept_ends = make_char2((signed char)c[0], (signed char)c[1]);
    }
    if (t == 0) *reinterpret_cast<float2*>(head + 2 * D) = make_float2(sk.s, sv.s);
  }
}

// Queries beside rows that the kernel before has stored: 16 threads a row and kQueryHeads heads of it.
template <class T, int D>
__global__ void __launch_bounds__(256) turn_queries_kernel(PagesAppendArgs p, uint32_t units) {
  constexpr int W = D / 32;
  const uint32_t unit = blockIdx.x * 16u + (threadIdx.x >> 4);
  if (unit >= units) return;
  const PagesWriteArgs& a = p.w;
  const int groups = (p.Hq + kQueryHeads - 1) / kQueryHeads, d0 = W * (threadIdx.x & 15);
  const uint32_t at = unit / (uint32_t)groups;
  const int h0 = (int)(unit - at * groups) * kQueryHeads;
  const int e = (int)(at / (uint32_t)a.n_rows), x = (int)(at - (uint32_t)e * a.n_rows);
  const int pos = x < (a.counts ? a.counts[e] : a.n_rows) ? position(p, e, 0, x) : -1;
  const T* q = static_cast<const T*>(p.q) + (int64_t)e * p.qsb + (int64_t)x * p.qsn + d0;
  T* out = static_cast<T*>(p.q_out) + (int64_t)e * p.osb + (int64_t)x * p.osn + d0;
  Some<T, W> lo[kQueryHeads], hi[kQueryHeads];
  Some<float, W> c, s;
  c.set(nan_f()); s.set(nan_f());
  if (pos >= 0) { c.load(p.rope + (int64_t)pos * D + d0); s.load(p.rope + (int64_t)pos * D + D / 2 + d0); }
#pragma unroll
  for (int i = 0; i < kQueryHeads; ++i)
    if (h0 + i < p.Hq) {
      lo[i].load(q + (int64_t)(h0 + i) * p.qsh);
      hi[i].load(q + (int64_t)(h0 + i) * p.qsh + D / 2);
    }
  wait_for_previous();
  const bool stored = a.plan[2 * e] >= 0 && x < (a.counts ? a.counts[e] : a.n_rows);
#pragma unroll
  for (int i = 0; i < kQueryHeads; ++i)
    if (h0 + i < p.Hq) {
      float f[2][W];
#pragma unroll
      for (int k = 0; k < W; ++k) { f[0][k] = lo[i].at(k); f[1][k] = hi[i].at(k); }
      if (stored) turn<W>(f[0], f[1], c, s);
      store_some<W>(out + (int64_t)(h0 + i) * p.osh, f[0]);
      store_some<W>(out + (int64_t)(h0 + i) * p.osh + D / 2, f[1]);
    }
}

// ------------------------------------------------------------------ rows as values
// Bound by memory (8 x 2005 rows of 40 heads: 81.7 us, 6.1 TB/s).
// One warp per (entry, KV head, tile of its list): a lane takes 8 dimensions of a row of K, four dimensions of four rows of V, so that what
// a warp stores at once lies together.
template <class T, int D>
__global__ void __launch_bounds__(kReadThreads) read8_kernel(PagesWriteArgs a, int blocks, uint32_t items) {
  constexpr int P = D / 32, E = D / 8;
  const int lane = threadIdx.x & 31;
  const uint32_t item = blockIdx.x * (kReadThreads / 32u) + (threadIdx.x >> 5);
  if (item >= items) return;
  const uint32_t eh = item / (uint32_t)blocks;
  const int blk = (int)(item - eh * blocks), e = (int)(eh / (uint32_t)a.p.Hkv), h = (int)(eh - (uint32_t)e * a.p.Hkv);
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
  uint2 kc[2 * P];
  uint4 vc[P];
#pragma unroll
  for (int i = 0; i < 2 * P; ++i) kc[i] = reinterpret_cast<const uint2*>(tile)[i * 32 + lane];
#pragma unroll
  for (int i = 0; i < P; ++i) vc[i] = reinterpret_cast<const uint4*>(tile + kPageTile * D)[i * 32 + lane];
  auto value = [](uint32_t w, int b, float s) { return __fmul_rn((float)((int)(w >> (8 * b) & 255u) - 128), s); };
#pragma unroll
  for (int i = 0; i < 2 * P; ++i) {
    const int piece = i * 32 + lane, r = piece / (D / 8), x = (piece % (D / 8)) ^ (D == 128 ? 8 * (r & 1) : 0), row = row0 + r;
    if (row < first || row >= end) continue;
    float f[8];
#pragma unroll
    for (int b = 0; b < 8; ++b) f[b] = value(b < 4 ? kc[i].x : kc[i].y, b & 3, scale.x);
    store_eight(k + (int64_t)(row - first) * a.sn + 8 * x, f);
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
// Shared memory of a CTA's stages at most: two, but one in fp32 with 128 dimensions and more than 96 rows a page (8 x 2005 rows of 40 heads: 179 us with
// pages of 128 rows, 170 with two stages and pages of 64, floor 125; bf16, which has two with both, 138 and 116).
constexpr int kStageBytes = 200 * 1024;
struct RunPages {
  const PagesAppendArgs& a; int pages, heads; unsigned grid; bool self; cudaStream_t s;
  template <class T, int D> cudaError_t run() {
    const int threads = 4 * a.w.p.page_rows, stage = threads * 16 * (int)sizeof(Some<T, D / 32>), stages = heads > 1 && 2 * stage <= kStageBytes ? 2 : 1;
    cudaError_t e = self ? allow_shared<append_pages_kernel<T, D, true>>(kStageBytes) : allow_shared<append_pages_kernel<T, D, false>>(kStageBytes);
    if (e != cudaSuccess) return e;
    if (!self) return launch_behind(append_pages_kernel<T, D, false>, dim3(grid), dim3(threads), stages * stage, s, a, pages, heads, stages, 1.f);
    append_pages_kernel<T, D, true><<<grid, threads, stages * stage, s>>>(a, pages, heads, stages, 1.f);
    return cudaGetLastError();
  }
};
struct RunQueries {
  const PagesAppendArgs& a; uint32_t units; cudaStream_t s;
  template <class T, int D> cudaError_t run() {
    return launch_behind(turn_queries_kernel<T, D>, dim3((unsigned)((units + 15) / 16)), dim3(256), 0, s, a, units);
  }
};
struct RunRead {
  const PagesWriteArgs& a; int blocks; uint32_t items; unsigned grid; cudaStream_t s;
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
  const int64_t units = a.q ? (int64_t)w.n * w.n_rows * ((a.Hq + kQueryHeads - 1) / kQueryHeads) : 0;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  // several heads a CTA where there are more than the machine holds, since each CTA has to look up its rows first (8 x 2005 rows of 40 heads:
  // 172 us with 2, 149 with 4, 142 with 8, 146 with 16, when each decided for itself; 123, 119 and 123 us with 4, 8 and 16 behind a launch that did)
  const int most = (int)(items / (4 * sms) < 1 ? 1 : items / (4 * sms) > 8 ? 8 : items / (4 * sms));
  const int chunks = (w.p.Hkv + most - 1) / most, heads = (w.p.Hkv + chunks - 1) / chunks;
  const int64_t grid = (int64_t)w.n * pages * ((w.p.Hkv + heads - 1) / heads);
  if (grid > 0x7fffffffLL || units > 0x7fffffffLL) return cudaErrorInvalidValue;
  // Where the CTAs fit twice into the machine at most (512 threads an SM, by registers) each decides for itself; where there are more a launch
  // in front decides for all, since looking up takes each of them 2 us: 4 lists of 512 rows, 160 CTAs, 23.3 us (with the launch 24.8);
  // 32 lists of 512 rows of 8 heads, 1088 CTAs of 128 threads, 28.2 (29.9); 8 lists of 2005 rows, 1320 of 256 threads, 132 (119); 1024 lists of 4
  // rows, 2048 of 128 threads, 55 (48).
  const bool self = w.n <= kSelfEntries && grid * 4 * pr <= (int64_t)2 * 512 * sms;
  if (!self) {
    e = allow_shared<append_plan_kernel>(2 * (kMaxLists / 32) * 4);
    if (e != cudaSuccess) return e;
    const int each = (w.n + kPlanThreads / 32 - 1) / (kPlanThreads / 32);
    append_plan_kernel<<<each < sms ? each : sms, kPlanThreads, 2 * words * sizeof(uint32_t), s>>>(w, words);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  e = by_format(w.p, w.dtype, RunPages{a, pages, heads, (unsigned)grid, self, s});
  if (e != cudaSuccess) return e;
  ++*launches;
  if (!a.q) return cudaSuccess;
  e = by_format(w.p, w.dtype, RunQueries{a, (uint32_t)units, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_read8(const PagesWriteArgs& a, int* launches, cudaStream_t s) {
  const int blocks = (int)(((int64_t)a.n_rows + 2 * kPageTile - 2) / kPageTile);
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kReadThreads / 32 - 1) / (kReadThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = by_format(a.p, a.dtype, RunRead{a, blocks, (uint32_t)items, (unsigned)grid, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_glue_rope_table(float* table, int64_t first, int64_t n_pos, int D, double base, cudaStream_t s) {
  const int64_t grid = (n_pos * (D / 2) + 255) / 256;            // (2^31 positions of 128 pairs: 2^30)
  rope_table_kernel<<<(unsigned)grid, 256, 0, s>>>(table, first, n_pos, D / 2, base);
  return cudaGetLastError();
}

}  // namespace pyr

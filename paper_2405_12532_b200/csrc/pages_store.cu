// Rows into and out of the paged 4-bit cache (format: include/pyr.h).
//
// A group of `group` values x is stored as codes c = rint((x - zero) / scale) in 0 .. 15 with zero = min x rounded down to
// bf16 and scale = (max x - zero) / 15 rounded up to bf16: with these two roundings every code is in range without a
// clamp, and a code's value scale * c + zero is within scale / 2 of x. The product scale * c is exact in fp32 (8 + 4 bits).
// Arithmetic is plain IEEE single precision, never contracted, so that the stored bytes are the same everywhere.
#include <cuda_bf16.h>

#include "pyr_internal.h"

namespace pyr {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kRowThreads = 256;
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

template <class T> __device__ __forceinline__ void load8(const T* p, float* x);
template <> __device__ __forceinline__ void load8<float>(const float* p, float* x) {
  const float4 a = *reinterpret_cast<const float4*>(p), b = *reinterpret_cast<const float4*>(p + 4);
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
template <> __device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float* x) {
  const uint4 r = *reinterpret_cast<const uint4*>(p);
  x[0] = __uint_as_float(r.x << 16); x[1] = __uint_as_float(r.x & 0xffff0000u);
  x[2] = __uint_as_float(r.y << 16); x[3] = __uint_as_float(r.y & 0xffff0000u);
  x[4] = __uint_as_float(r.z << 16); x[5] = __uint_as_float(r.z & 0xffff0000u);
  x[6] = __uint_as_float(r.w << 16); x[7] = __uint_as_float(r.w & 0xffff0000u);
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

// The eight codes of one thread (dimension k of the word in bits 4k ..) and its group's (scale, zero) word. The GROUP / 8
// threads of a group sit side by side.
template <int GROUP>
__device__ __forceinline__ uint32_t quantise8(const float* x, uint32_t* word) {
  float lo = x[0], hi = x[0];
#pragma unroll
  for (int k = 1; k < 8; ++k) { lo = min_nan(lo, x[k]); hi = max_nan(hi, x[k]); }
#pragma unroll
  for (int o = GROUP / 16; o > 0; o >>= 1) {
    lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, o));
    hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, o));
  }
  const float zero = floor_bf16(lo);
  const float span = __fsub_rn(hi, zero);
  float scale = ceil_bf16(__fdiv_rn(span, 15.f));
  if (scale < kScaleMin) scale = 0.f;
  const float inv = scale > 0.f ? __fdiv_rn(1.f, scale) : 0.f;
  if (!(span <= 3.402823466e38f)) {              // infinite or not a number
    *word = kNanWord;
    return 0;
  }
  *word = (__float_as_uint(scale) >> 16) | (__float_as_uint(zero) & 0xFFFF0000u);
  uint32_t w = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    // adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it in the low bits
    const uint32_t c = __float_as_uint(__fadd_rn(__fmul_rn(__fsub_rn(x[k], zero), inv), 12582912.f));
    w |= (c & 15u) << (4 * k);
  }
  return w;
}

// Decides every entry of a write before any row moves: plan[i] = first row, -1 if the entry is refused. A warp per entry.
__global__ void __launch_bounds__(kPlanThreads) write_plan_kernel(PagesWriteArgs a, int words) {
  extern __shared__ uint32_t seen[];              // two bits per list: met, met twice
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

// One warp per (entry, KV head, 16 rows). A thread holds eight dimensions of a row: D / 8 threads a row.
template <class T, int D, int GROUP>
__global__ void __launch_bounds__(kRowThreads) write_rows_kernel(PagesWriteArgs a, int blocks, int64_t items) {
  constexpr int LPR = D / 8, RPP = 32 / LPR, G = D / GROUP;
  const int lane = threadIdx.x & 31, sub = lane / LPR, wi = lane % LPR;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  const int blk = (int)(item % blocks);
  const int h = (int)(item / blocks % a.p.Hkv);
  const int e = (int)(item / blocks / a.p.Hkv);
  const int start = a.plan[e];
  if (start < 0) return;
  const int l = pages_list(a.p, a.lists, e);
  const int cnt = a.counts ? a.counts[e] : a.n_rows;
  const int32_t* idx = a.idx ? a.idx + (int64_t)e * a.idx_stride +
                               (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows : nullptr;
  const T* k = static_cast<const T*>(a.k) + (int64_t)e * a.sb + (int64_t)h * a.sh + wi * 8;
  const T* v = static_cast<const T*>(a.v) + (int64_t)e * a.sb + (int64_t)h * a.sh + wi * 8;
#pragma unroll 2
  for (int pass = 0; pass < kPageTile / RPP; ++pass) {
    const int x = blk * kPageTile + pass * RPP + sub;
    const bool live = x < cnt;
    const int src = live ? (idx ? idx[x] : x) : 0;
    const bool good = src >= 0 && src < a.src_rows;
    float kf[8], vf[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) kf[i] = vf[i] = __uint_as_float(0x7FC00000u);   // a row without a source is NaN
    if (live && good) {
      load8(k + (int64_t)src * a.sn, kf);
      load8(v + (int64_t)src * a.sn, vf);
    }
    uint32_t kword, vword;
    const uint32_t kc = quantise8<GROUP>(kf, &kword), vc = quantise8<GROUP>(vf, &vword);
    if (!live) continue;
    if (!good && wi == 0) record(a.p.status, PYR_ERR_INVALID);
    const int row = start + x;
    const int page = pages_page(a.p, l, row / a.p.page_rows);
    if (page < 0) continue;                       // (the plan has seen a valid page here)
    const int r = row % kPageTile;
    uint8_t* tile = a.p.pool + pages_tile(a.p, page, h, row % a.p.page_rows / kPageTile);
    *reinterpret_cast<uint32_t*>(tile + tile_k_row(D, r) + 4 * k_word_slot(D, GROUP, wi)) = kc;
    *reinterpret_cast<uint16_t*>(tile + tile_v_row(D, r) + 2 * v_half_slot(D, GROUP, 2 * wi)) = (uint16_t)vc;
    *reinterpret_cast<uint16_t*>(tile + tile_v_row(D, r) + 2 * v_half_slot(D, GROUP, 2 * wi + 1)) = (uint16_t)(vc >> 16);
    if (wi % (GROUP / 8) == 0) {
      *reinterpret_cast<uint32_t*>(tile + tile_k_word(D, G, r, wi / (GROUP / 8))) = kword;
      *reinterpret_cast<uint32_t*>(tile + tile_v_word(D, G, r, wi / (GROUP / 8))) = vword;
    }
  }
}

// The values of eight codes: scale * code + zero, the product exact.
__device__ __forceinline__ void values8(uint32_t codes, uint32_t word, float* x) {
  const float scale = __uint_as_float(word << 16), zero = __uint_as_float(word & 0xFFFF0000u);
#pragma unroll
  for (int k = 0; k < 8; ++k) x[k] = __fmaf_rn(scale, (float)((codes >> (4 * k)) & 15u), zero);
}

template <class T, int D, int GROUP>
__global__ void __launch_bounds__(kRowThreads) read_rows_kernel(PagesWriteArgs a, int blocks, int64_t items) {
  constexpr int LPR = D / 8, RPP = 32 / LPR, G = D / GROUP;
  const int lane = threadIdx.x & 31, sub = lane / LPR, wi = lane % LPR;
  const int64_t item = (int64_t)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
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
  const int len = pages_len(a.p, l);
  T* k = static_cast<T*>(const_cast<void*>(a.k)) + (int64_t)e * a.sb + (int64_t)h * a.sh + wi * 8;
  T* v = static_cast<T*>(const_cast<void*>(a.v)) + (int64_t)e * a.sb + (int64_t)h * a.sh + wi * 8;
#pragma unroll 2
  for (int pass = 0; pass < kPageTile / RPP; ++pass) {
    const int x = blk * kPageTile + pass * RPP + sub;
    if (x >= cnt || (int64_t)first + x >= len) continue;
    const int row = first + x;
    const int page = pages_page(a.p, l, row / a.p.page_rows);
    if (page < 0) { if (wi == 0) record(a.p.status, PYR_ERR_INVALID); continue; }
    const int r = row % kPageTile;
    const uint8_t* tile = a.p.pool + pages_tile(a.p, page, h, row % a.p.page_rows / kPageTile);
    const uint32_t kc = *reinterpret_cast<const uint32_t*>(tile + tile_k_row(D, r) + 4 * k_word_slot(D, GROUP, wi));
    const uint32_t v0 = *reinterpret_cast<const uint16_t*>(tile + tile_v_row(D, r) + 2 * v_half_slot(D, GROUP, 2 * wi));
    const uint32_t v1 = *reinterpret_cast<const uint16_t*>(tile + tile_v_row(D, r) + 2 * v_half_slot(D, GROUP, 2 * wi + 1));
    const uint32_t kword = *reinterpret_cast<const uint32_t*>(tile + tile_k_word(D, G, r, wi / (GROUP / 8)));
    const uint32_t vword = *reinterpret_cast<const uint32_t*>(tile + tile_v_word(D, G, r, wi / (GROUP / 8)));
    float f[8];
    values8(kc, kword, f);
    store8(k + (int64_t)x * a.sn, f);
    values8(v0 | (v1 << 16), vword, f);
    store8(v + (int64_t)x * a.sn, f);
  }
}

template <class F>
cudaError_t by_format(const PagesView& p, int dtype, F f) {
  const bool bf = dtype == PYR_BF16;
#define PYR_CASE(D_, G_) if (p.D == D_ && p.group == G_) { if (bf) f.template run<__nv_bfloat16, D_, G_>(); else f.template run<float, D_, G_>(); return cudaGetLastError(); }
  PYR_CASE(128, 32) PYR_CASE(128, 64) PYR_CASE(128, 128) PYR_CASE(64, 32) PYR_CASE(64, 64)
#undef PYR_CASE
  return cudaErrorInvalidValue;
}

struct RunWrite {
  const PagesWriteArgs& a; int blocks; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D, int G> void run() { write_rows_kernel<T, D, G><<<grid, kRowThreads, 0, s>>>(a, blocks, items); }
};
struct RunRead {
  const PagesWriteArgs& a; int blocks; int64_t items; unsigned grid; cudaStream_t s;
  template <class T, int D, int G> void run() { read_rows_kernel<T, D, G><<<grid, kRowThreads, 0, s>>>(a, blocks, items); }
};

}  // namespace

cudaError_t launch_pages_write(const PagesWriteArgs& a, int* launches, cudaStream_t s) {
  const int words = (a.p.n_lists + 31) / 32;
  const int blocks = (a.n_rows + kPageTile - 1) / kPageTile;
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  cudaError_t e = allow_shared<write_plan_kernel>(2 * (kMaxLists / 32) * 4);
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
  const int blocks = (a.n_rows + kPageTile - 1) / kPageTile;
  const int64_t items = (int64_t)a.n * a.p.Hkv * blocks;
  const int64_t grid = (items + kRowThreads / 32 - 1) / (kRowThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  const cudaError_t e = by_format(a.p, a.dtype, RunRead{a, blocks, items, (unsigned)grid, s});
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

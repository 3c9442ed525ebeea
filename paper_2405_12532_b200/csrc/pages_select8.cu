// Which pages of the paged 8-bit cache a query reads: a cheap score for each page, and the n_slots largest (format: include/pyr.h).
//
// Score of a page for a KV head: the largest, over the head's query heads, of s_q s_K sum_d max(qc_d min_d, qc_d max_d), with qc the query
// in 8 bits and min, max the least and largest code of the page in each dimension: an upper bound of q . K over its rows, up to
// the query's rounding. The sums are whole numbers below 2^21, exact in any order; what follows is two products rounded to fp32, so
// equal inputs give the same pages everywhere. With qc split by its sign a term is one of two products: two dot products of
// four bytes a word.
//
// One CTA, or a cluster of up to 8 where there are few, for each (entry, query token, KV head). The scores of a list stay in the first
// CTA's shared memory (the others write theirs there), which finds the n_slots-th largest by its bits, 8 at a time, and
// writes the pages in order.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include "pyr_internal.h"

namespace pyr {
namespace {

namespace cg = cooperative_groups;
constexpr float kScaleMin = 7.888609052210118e-31f;   // 2^-100
constexpr uint32_t kForced = 0xFFFFFFFFu;              // the key of a page that is taken whatever its score

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// A number's place in the order of scores; NaN counts as Inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t b = __float_as_uint(x == x ? x + 0.f : INFINITY);
  return b ^ (b >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}

// R query heads at a time, D / 16 lanes a page.
template <int D, int R, int kThreads>
__global__ void __launch_bounds__(kThreads, kThreads == 512 ? 1 : (R == 8 ? 640 : 768) / kThreads) select8_kernel(PagesSelectArgs a) {
  constexpr int kWarps = kThreads / 32;
  constexpr int LPP = D / 16, PPW = 32 / LPP, W = D / 4, U = 2;    // lanes a page, pages a warp and step, words of a row, steps at once
  extern __shared__ __align__(16) uint32_t shared[];
  __shared__ uint32_t hist[256];
  __shared__ uint32_t warp_sums[kWarps];
  __shared__ uint32_t sh_prefix, sh_need;
  uint32_t* keys = shared;                                         // [max_pages] rounded up to 4
  uint32_t* plus = shared + (a.p.max_pages + 3) / 4 * 4;           // [rep][W] codes above 0, then [rep][W] those below
  float* sq = reinterpret_cast<float*>(plus + 2 * a.rep * W);      // [rep]
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank(), ranks = cluster.num_blocks();
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
  const int64_t item = blockIdx.x / ranks;
  const int h = (int)(item % a.p.Hkv);
  const int64_t et = item / a.p.Hkv;
  const int e = (int)(et / a.T), tok = (int)(et - (int64_t)e * a.T);
  int32_t* out = a.slots + item * a.n_slots;
  const int l = pages_list(a.p, a.lists, e);
  const int len = l < 0 ? 0 : max(0, pages_len(a.p, l) - (a.T - 1 - tok));
  const int pages = (int)(((int64_t)len + a.p.page_rows - 1) / a.p.page_rows);
  if (pages <= a.n_slots) {                                        // (the whole cluster)
    if (rank == 0) {
      if (l < 0 && t == 0) record(a.p.status, PYR_ERR_INVALID);
      for (int x = t; x < a.n_slots; x += kThreads) out[x] = x < pages ? x : -1;
    }
    return;
  }
  // ---- the queries in 8 bits, a warp a head
  for (int r = warp; r < a.rep; r += kWarps) {
    const int64_t row = (int64_t)e * a.qsb + (int64_t)tok * a.qst + (int64_t)(h * a.rep + r) * a.qsh;
    constexpr int N = D / 32;                                      // elements a lane: side by side
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
    for (int k = 0; k < N; ++k) {
      const int c = fine ? __float2int_rn(__fmul_rn(x[k], inverse)) : 0;
      reinterpret_cast<int8_t*>(plus + r * W)[N * lane + k] = (int8_t)max(c, 0);
      reinterpret_cast<int8_t*>(plus + (a.rep + r) * W)[N * lane + k] = (int8_t)min(c, 0);
    }
    if (lane == 0) sq[r] = fine ? s : __uint_as_float(0x7FC00000u);
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
    float sk[U], best[U];
#pragma unroll
    for (int u = 0; u < U; ++u) { mn[u] = mn_next[u]; mx[u] = mx_next[u]; sk[u] = sk_next[u]; best[u] = -INFINITY; }
    fetch();
    fetch_ids(base + 2 * ranks * step);
    for (int r0 = 0; r0 < a.rep; r0 += R) {
      int sums[U][R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const int head = min(r0 + r, a.rep - 1);
        const uint4 qp = reinterpret_cast<const uint4*>(plus + head * W)[part];
        const uint4 qn = reinterpret_cast<const uint4*>(plus + (a.rep + head) * W)[part];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          int s = __dp4a((int)mx[u].x, (int)qp.x, 0);
          s = __dp4a((int)mn[u].x, (int)qn.x, s);
          s = __dp4a((int)mx[u].y, (int)qp.y, s);
          s = __dp4a((int)mn[u].y, (int)qn.y, s);
          s = __dp4a((int)mx[u].z, (int)qp.z, s);
          s = __dp4a((int)mn[u].z, (int)qn.z, s);
          s = __dp4a((int)mx[u].w, (int)qp.w, s);
          sums[u][r] = __dp4a((int)mn[u].w, (int)qn.w, s);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        int* sum = sums[u];
        // sums over the lanes of the page: each step halves the heads that a lane goes on with, as long as there are several
        int first = 0, left = R;
#pragma unroll
        for (int o = LPP / 2; o > 0; o >>= 1) {
          if (left > 1) {
            left /= 2;
            const bool upper = lane & o;
            first += upper ? left : 0;
#pragma unroll
            for (int r = 0; r < R / 2; ++r)
              if (r < left) {
                const int mine = upper ? sum[r + left] : sum[r], other = upper ? sum[r] : sum[r + left];
                sum[r] = mine + __shfl_xor_sync(0xffffffffu, other, o);
              }
          } else {
            sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], o);
          }
        }
#pragma unroll
        for (int r = 0; r < R; ++r)
          if (r < left && r0 + first + r < a.rep)
            best[u] = max_nan(best[u], __fmul_rn(__fmul_rn(sq[r0 + first + r], sk[u]), (float)sum[r]));
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int x = base + (u * kWarps + warp) * PPW + sub;
#pragma unroll
      for (int o = LPP / 2; o > 0; o >>= 1) best[u] = max_nan(best[u], __shfl_xor_sync(0xffffffffu, best[u], o));
      if (part == 0 && x < pages) {
        const bool none = sk[u] == -1.f;
        if (none) record(a.p.status, PYR_ERR_INVALID);
        keys0[x] = x < a.keep_first || x >= pages - a.keep_last ? kForced : none ? 0u : key_of(best[u]);
      }
    }
  }
  if (ranks > 1) {
    cluster.sync();
    if (rank != 0) return;
  } else {
    __syncthreads();
  }

  // ---- the n_slots-th largest key, from its highest bits down; `need` of those that share the bits found so far are wanted
  uint32_t prefix = 0, need = a.n_slots;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int x = t; x < 256; x += kThreads) hist[x] = 0;
    __syncthreads();
    const uint32_t mask = shift == 24 ? 0u : 0xFFFFFFFFu << (shift + 8);
    for (int x0 = 0; x0 < pages; x0 += kThreads) {
      const int x = x0 + t;
      const uint32_t key = x < pages ? keys[x] : 0u;
      const bool in = x < pages && (key & mask) == prefix;
      // (scores share their high bits: the lanes that add to one place do so together)
      const uint32_t digit = in ? key >> shift & 255u : 256u;
      const uint32_t same = __match_any_sync(0xffffffffu, digit);
      if (in && lane == __ffs(same) - 1) atomicAdd(&hist[digit], __popc(same));
    }
    __syncthreads();
    if (warp == 0) {                             // lane i: digits 255 - 8 i and the seven below it, the largest first
      uint32_t mine = 0;
#pragma unroll
      for (int k = 0; k < 8; ++k) mine += hist[255 - 8 * lane - k];
      uint32_t incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t y = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += y;
      }
      uint32_t before = incl - mine;
      if (before < need && need <= incl)
        for (int k = 0; k < 8; ++k) {
          const uint32_t c = hist[255 - 8 * lane - k];
          if (before + c >= need) {
            sh_prefix = prefix | (uint32_t)(255 - 8 * lane - k) << shift;
            sh_need = need - before;
            break;
          }
          before += c;
        }
    }
    __syncthreads();
    prefix = sh_prefix;
    need = sh_need;
    __syncthreads();
  }
  // ---- pages above it, and the first `need` of those equal to it, in order
  uint32_t done = 0, equal = 0;
  for (int x0 = 0; x0 < pages; x0 += kThreads) {
    const int x = x0 + t;
    const uint32_t key = x < pages ? keys[x] : 0u;
    const bool above = x < pages && key > prefix, same = x < pages && key == prefix;
    const uint32_t ba = __ballot_sync(0xffffffffu, above), bs = __ballot_sync(0xffffffffu, same);
    if (lane == 0) warp_sums[warp] = __popc(ba) | __popc(bs) << 16;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const uint32_t s = warp_sums[w];
      before += w < warp ? s : 0;
      total += s;
    }
    const uint32_t lower = (1u << lane) - 1u;
    const uint32_t a0 = done + (before & 0xFFFFu) + __popc(ba & lower), e0 = equal + (before >> 16) + __popc(bs & lower);
    if (above || (same && e0 < need)) out[a0 + min(e0, need)] = x;
    done += total & 0xFFFFu;
    equal += total >> 16;
    __syncthreads();
  }
}

template <int D, int R, int kThreads>
cudaError_t run(const PagesSelectArgs& a, int smem, cudaStream_t s) {
  const cudaError_t e = allow_shared<select8_kernel<D, R, kThreads>>(kSelect8Shared);
  if (e != cudaSuccess) return e;
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int64_t items = (int64_t)a.n * a.T * a.p.Hkv;
  // several CTAs a list where that many find room at once and each has a step or more to do
  int ranks = 1;
  while (kThreads == 512 && ranks < 8 && items * ranks * 2 <= sms && a.p.max_pages > ranks * 128) ranks *= 2;
  if (items * ranks > 0x7fffffffLL) return cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(items * ranks)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = s;
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeClusterDimension;
  at.val.clusterDim.x = ranks; at.val.clusterDim.y = at.val.clusterDim.z = 1;
  cfg.attrs = &at; cfg.numAttrs = ranks > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, select8_kernel<D, R, kThreads>, a);
}
// As many threads for a list as there is room for, where its table is long enough to occupy them.
template <int D, int R>
cudaError_t by_length(const PagesSelectArgs& a, int smem, cudaStream_t s) {
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int64_t items = (int64_t)a.n * a.T * a.p.Hkv;
  const auto fits = [&](int threads) { return items * threads <= (int64_t)sms * 1024 && a.p.max_pages * 2 >= threads; };
  return fits(512) ? run<D, R, 512>(a, smem, s) : fits(256) ? run<D, R, 256>(a, smem, s) : fits(128) ? run<D, R, 128>(a, smem, s)
         : a.p.max_pages > 1024 ? run<D, R, 256>(a, smem, s) : run<D, R, 32>(a, smem, s);
}
template <int D>
cudaError_t by_heads(const PagesSelectArgs& a, int smem, cudaStream_t s) {
  return a.rep == 1 ? by_length<D, 1>(a, smem, s) : a.rep <= 4 ? by_length<D, 4>(a, smem, s) : by_length<D, 8>(a, smem, s);
}

}  // namespace

cudaError_t launch_pages_select8(const PagesSelectArgs& a, int* launches, cudaStream_t s) {
  const int smem = (int)pages_select8_shared(a.p.max_pages, a.p.D, a.rep);
  const cudaError_t e = a.p.D == 128 ? by_heads<128>(a, smem, s) : by_heads<64>(a, smem, s);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

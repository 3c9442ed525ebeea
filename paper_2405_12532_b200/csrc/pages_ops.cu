// Page management of the paged 4-bit cache: taking pages (with the copy that a shared, part-filled last page needs),
// forking, giving up and compacting lists. Tables, lengths and reference counts are device memory, so a call plans on
// the device, and every id that a table or a caller's list holds is range-checked before it is used.
#include "pyr_internal.h"

namespace pyr {
namespace {

constexpr int kThreads = 256;
constexpr int kScanThreads = 1024;
static_assert(kReserveSlice == kScanThreads * 4, "a thread of the scan owns four pages");

__device__ __forceinline__ void record(int* status, int code) { atomicCAS(status, 0, code); }

// Exclusive prefix sum over a block of kScanThreads; *total gets the sum. `warp_sums` is shared memory for 33 values.
__device__ __forceinline__ long long block_scan(long long x, long long* warp_sums, long long* total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += y;
  }
  __syncthreads();                       // the previous use of warp_sums is over
  if (lane == 31) warp_sums[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    long long s = warp_sums[lane], t = s;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += y;
    }
    warp_sums[lane] = t - s;
    if (lane == 31) warp_sums[32] = t;
  }
  __syncthreads();
  *total = warp_sums[32];
  return warp_sums[warp] + incl - x;
}

// ------------------------------------------------------------------ reserve
// Every CTA lists the free pages of its slice of the pool; the CTA that finishes last knows how many lie before each slice
// and plans the entries: how many pages each needs and the rank of its first one among the free pages. (One pass over the
// reference counts by the whole machine; one CTA reading them alone would take over ten times as long for a large pool.)
__global__ void __launch_bounds__(kScanThreads) reserve_plan_kernel(PagesReserveArgs a, int words) {
  extern __shared__ uint32_t seen[];     // a bit per list
  __shared__ long long sums[33];
  __shared__ int is_last, errors;
  const int t = threadIdx.x;
  long long total;
  {
    const int64_t p0 = (int64_t)blockIdx.x * kReserveSlice + t * 4;
    uint32_t free4 = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (p0 + i < a.p.n_pages && a.p.refs[p0 + i] == 0) free4 |= 1u << i;
    long long at = block_scan(__popc(free4), sums, &total);
    int32_t* ids = a.free_ids + (int64_t)blockIdx.x * kReserveSlice;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (free4 >> i & 1u) ids[at++] = (int32_t)(p0 + i);
    if (t == 0) a.slice_first[blockIdx.x + 1] = (int32_t)total;
  }
  __threadfence();
  __syncthreads();
  if (t == 0) is_last = atomicAdd(&a.control[0], 1) == a.slices - 1;
  __syncthreads();
  if (!is_last) return;
  __threadfence();

  long long free_pages = 0;
  for (int s0 = 0; s0 < a.slices; s0 += kScanThreads) {
    const int s = s0 + t;
    const long long c = s < a.slices ? __ldcg(a.slice_first + s + 1) : 0;
    const long long before = free_pages + block_scan(c, sums, &total);
    if (s < a.slices) a.slice_first[s + 1] = (int32_t)(before + c);
    free_pages += total;
  }
  for (int i = t; i < words; i += kScanThreads) seen[i] = 0;
  if (t == 0) { a.slice_first[0] = 0; a.control[0] = 0; errors = 0; }
  __syncthreads();

  long long taken = 0;
  for (int i0 = 0; i0 < a.n; i0 += kScanThreads) {
    const int i = i0 + t;
    long long need = 0;
    int err = 0, old = -1, slot = 0, fresh = 0;
    if (i < a.n) {
      const int l = pages_list(a.p, a.lists, i);
      const int add = a.rows ? a.rows[i] : a.rows_each;
      if (l < 0 || add < 0 || (atomicOr(&seen[l >> 5], 1u << (l & 31)) >> (l & 31) & 1u)) {
        err = PYR_ERR_INVALID;
      } else if (add > 0) {
        const int len = pages_len(a.p, l);
        const int64_t rows = (int64_t)len + add;
        if (rows > (int64_t)a.p.max_pages * a.p.page_rows) {
          err = PYR_ERR_CAPACITY;
        } else {
          const int s1 = (int)((rows + a.p.page_rows - 1) / a.p.page_rows);
          if (len % a.p.page_rows) {               // the part-filled last page: a copy if others hold it too
            const int page = pages_page(a.p, l, len / a.p.page_rows);
            if (page < 0) err = PYR_ERR_INVALID;
            else if (a.p.refs[page] > 1) old = page;
          }
          slot = (len + a.p.page_rows - 1) / a.p.page_rows;
          while (slot < s1 && a.p.table[(size_t)l * a.p.max_pages + slot] >= 0) ++slot;   // reserved before
          fresh = s1 - slot;
          need = fresh + (old >= 0 ? 1 : 0);
        }
      }
    }
    if (err) atomicCAS(&errors, 0, err);
    const long long base = taken + block_scan(need, sums, &total);
    taken += total;
    if (i < a.n) {
      int32_t* pl = a.plan + (int64_t)i * 4;
      pl[0] = (int32_t)(base < 0x7fffffff ? base : 0x7fffffff);
      pl[1] = old; pl[2] = slot; pl[3] = fresh;
    }
  }
  __syncthreads();
  if (t == 0) {
    int err = errors;
    if (!err && taken > free_pages) err = PYR_ERR_CAPACITY;
    if (err) record(a.p.status, err);
    a.control[1] = err ? 0 : 1;
  }
}

// The free page of the given rank.
__device__ __forceinline__ int free_page(const PagesReserveArgs& a, int rank) {
  int lo = 0, hi = a.slices - 1;         // the last slice that has no more than `rank` free pages before it
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (a.slice_first[mid] <= rank) lo = mid; else hi = mid - 1;
  }
  // slices without a free page share their successor's count: the search ends at the last of them, which has one
  return a.free_ids[(int64_t)lo * kReserveSlice + (rank - a.slice_first[lo])];
}

// Copies the first `rows` rows of one head of a page to another page: whole tiles as they lie, of a part-filled tile the
// rows' codes and words.
__device__ __forceinline__ void copy_head_rows(const PagesView& p, int from, int to, int h, int rows) {
  const int G = p.D / p.group, half = kPageTile * p.D / 2;
  const uint8_t* s = p.pool + pages_tile(p, from, h, 0);
  uint8_t* d = p.pool + pages_tile(p, to, h, 0);
  const int whole = rows / kPageTile * p.tile_bytes;
  for (int o = threadIdx.x * 16; o < whole; o += blockDim.x * 16)
    *reinterpret_cast<uint4*>(d + o) = *reinterpret_cast<const uint4*>(s + o);
  const int left = rows % kPageTile;
  s += whole; d += whole;
  const int codes = left * p.D / 2, words = left * G * 4;
  for (int o = threadIdx.x * 16; o < 2 * codes; o += blockDim.x * 16) {
    const int at = o < codes ? o : half + o - codes;
    *reinterpret_cast<uint4*>(d + at) = *reinterpret_cast<const uint4*>(s + at);
  }
  for (int o = threadIdx.x * 4; o < 2 * words; o += blockDim.x * 4) {
    const int at = 2 * half + (o < words ? o : kPageTile * G * 4 + o - words);
    *reinterpret_cast<uint32_t*>(d + at) = *reinterpret_cast<const uint32_t*>(s + at);
  }
}

// grid (entries, parts): part 0 writes the entry's table and counts, every part copies its share of the heads.
__global__ void __launch_bounds__(kThreads) reserve_take_kernel(PagesReserveArgs a) {
  if (a.control[1] == 0) return;
  const int i = blockIdx.x;
  const int32_t* pl = a.plan + (int64_t)i * 4;
  const int base = pl[0], old = pl[1], slot = pl[2], fresh = pl[3];
  if (old < 0 && (fresh == 0 || blockIdx.y != 0)) return;
  const int l = pages_list(a.p, a.lists, i);
  const int copies = old >= 0 ? 1 : 0;
  if (blockIdx.y == 0) {
    int32_t* row = a.p.table + (size_t)l * a.p.max_pages;
    for (int x = threadIdx.x; x < fresh; x += kThreads) {
      const int id = free_page(a, base + copies + x);
      row[slot + x] = id;
      a.p.refs[id] = 1;
    }
  }
  if (copies) {
    const int to = free_page(a, base);
    const int len = pages_len(a.p, l);
    for (int h = blockIdx.y; h < a.p.Hkv; h += gridDim.y) copy_head_rows(a.p, old, to, h, len % a.p.page_rows);
    if (blockIdx.y == 0 && threadIdx.x == 0) {
      a.p.table[(size_t)l * a.p.max_pages + len / a.p.page_rows] = to;
      a.p.refs[to] = 1;
      atomicSub(&a.p.refs[old], 1);
    }
  }
}

// ------------------------------------------------------------------ fork, trim
// One CTA per entry. An entry whose destination appears elsewhere in the call is refused by every CTA that sees it, so the
// outcome does not depend on their order.
__global__ void __launch_bounds__(kThreads) fork_kernel(PagesView p, const int32_t* src, const int32_t* dst, int n) {
  const int e = blockIdx.x;
  const int s = pages_list(p, src, e), d = pages_list(p, dst, e);
  bool bad = s < 0 || d < 0;
  for (int x = threadIdx.x; x < n; x += kThreads) bad = bad || (x != e && dst[x] == d) || src[x] == d;
  int pages = 0, len = 0;
  if (s >= 0 && d >= 0) {
    len = pages_len(p, s);
    pages = (len + p.page_rows - 1) / p.page_rows;
    bad = bad || p.lens[d] != 0 || p.table[(size_t)d * p.max_pages] >= 0;
    for (int x = threadIdx.x; x < pages; x += kThreads) bad = bad || pages_page(p, s, x) < 0;
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) record(p.status, PYR_ERR_INVALID);
    return;
  }
  for (int x = threadIdx.x; x < pages; x += kThreads) {
    const int id = pages_page(p, s, x);
    p.table[(size_t)d * p.max_pages + x] = id;
    atomicAdd(&p.refs[id], 1);
  }
  if (threadIdx.x == 0) p.lens[d] = len;
}

// Gives up the pages of list l from slot `first` on. A table entry is taken by exchange, so that a list named twice gives
// a page up once.
__device__ __forceinline__ void drop_pages(const PagesView& p, int l, int first) {
  int32_t* row = p.table + (size_t)l * p.max_pages;
  for (int x = first + threadIdx.x; x < p.max_pages; x += blockDim.x) {
    if (row[x] < 0) continue;
    const int id = atomicExch(&row[x], -1);
    if (id >= 0 && id < p.n_pages) atomicSub(&p.refs[id], 1);
  }
}

__global__ void __launch_bounds__(kThreads) trim_kernel(PagesView p, const int32_t* lists, int n, const int32_t* rows) {
  const int e = blockIdx.x;
  const int l = pages_list(p, lists, e);
  const int want = rows ? rows[e] : 0;
  if (l < 0 || want < 0) {
    if (threadIdx.x == 0) record(p.status, PYR_ERR_INVALID);
    return;
  }
  __shared__ int keep;
  if (threadIdx.x == 0) {
    const int len = atomicMin(&p.lens[l], want);
    keep = len < want ? (len < 0 ? 0 : len) : want;
  }
  __syncthreads();
  drop_pages(p, l, (keep + p.page_rows - 1) / p.page_rows);
}

// ------------------------------------------------------------------ compact
// Checks an entry as a whole: plan[e] = rows to move, -1 if it is refused.
__global__ void __launch_bounds__(kThreads) compact_plan_kernel(PagesMoveArgs a) {
  const int e = blockIdx.x, t = threadIdx.x;
  const PagesView& p = a.p;
  const int s = pages_list(p, a.src, e), d = pages_list(p, a.dst, e);
  const int cnt = a.counts ? a.counts[e] : a.n_rows;
  bool bad = s < 0 || d < 0 || cnt < 0 || cnt > a.n_rows;
  if (!bad) {
    const bool in_place = s == d;
    const int len = pages_len(p, s);
    for (int x = t; x < a.n; x += kThreads) bad = bad || (x != e && (a.dst[x] == d || a.src[x] == d));
    bad = bad || (int64_t)cnt > (int64_t)p.max_pages * p.page_rows || (!a.idx && cnt > len);
    const int pages = (cnt + p.page_rows - 1) / p.page_rows;
    const int from = (len + p.page_rows - 1) / p.page_rows;
    if (!bad)
      for (int x = t; x < pages; x += kThreads) {
        const int id = pages_page(p, d, x);
        bad = bad || id < 0 || (!in_place && p.refs[id] != 1);
      }
    for (int x = t; x < from; x += kThreads) bad = bad || pages_page(p, s, x) < 0;
    if (!bad && a.idx) {
      const int32_t* idx = a.idx + (int64_t)e * a.idx_stride;
      for (int g = 0; g < a.idx_groups; ++g)
        for (int x = t; x < cnt; x += kThreads) {
          const int32_t* row = idx + (int64_t)g * a.n_rows;
          const int v = row[x];
          bad = bad || v < 0 || v >= len;
          if (in_place) {
            bad = bad || (x > 0 && row[x - 1] >= v);
            if (v != x) {
              const int id = pages_page(p, d, x / p.page_rows);
              bad = bad || id < 0 || p.refs[id] != 1;
            }
          }
        }
    }
  }
  bad = __syncthreads_or(bad);
  if (t == 0) {
    a.plan[e] = bad ? -1 : cnt;
    if (bad) record(p.status, PYR_ERR_INVALID);
  }
}

// The bytes that one warp moves for a tile of destination rows, held in registers between the reads and the writes.
template <int D, int G>
struct TileRows {
  static constexpr int C = D / 32;                       // 16-byte pieces of a row of codes
  static constexpr int CP = kPageTile * C / 32;          // pieces a lane holds of K, and of V
  static constexpr int WP = (kPageTile * G + 31) / 32;   // words a lane holds of K, and of V
  uint4 k[CP], v[CP];
  uint32_t kw[WP], vw[WP];

  __device__ __forceinline__ void load(const PagesView& p, int l, int h, int src, int lane) {
    // lane r (< 16) knows source row r of the tile (-1: none)
    const uint8_t* base = nullptr;
    int r = 0;
    if (src >= 0) {
      const int page = pages_page(p, l, src / p.page_rows);
      if (page >= 0) { base = p.pool + pages_tile(p, page, h, src % p.page_rows / kPageTile); r = src % kPageTile; }
    }
    const unsigned long long addr = reinterpret_cast<unsigned long long>(base);
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int piece = i * 32 + lane, row = piece / C, c = piece % C;
      const uint8_t* b = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, addr, row));
      const int rr = __shfl_sync(0xffffffffu, r, row);
      if (b) {
        k[i] = *reinterpret_cast<const uint4*>(b + tile_k_row(D, rr) + 16 * c);
        v[i] = *reinterpret_cast<const uint4*>(b + tile_v_row(D, rr) + 16 * c);
      }
    }
#pragma unroll
    for (int i = 0; i < WP; ++i) {
      const int piece = i * 32 + lane, row = piece / G < kPageTile ? piece / G : 0, g = piece % G;
      const uint8_t* b = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, addr, row));
      const int rr = __shfl_sync(0xffffffffu, r, row);
      if (b && piece < kPageTile * G) {
        kw[i] = *reinterpret_cast<const uint32_t*>(b + tile_k_word(D, G, rr, g));
        vw[i] = *reinterpret_cast<const uint32_t*>(b + tile_v_word(D, G, rr, g));
      }
    }
  }
  __device__ __forceinline__ void store(uint8_t* tile, int rows, int lane) const {
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int piece = i * 32 + lane, row = piece / C, c = piece % C;
      if (row < rows) {
        *reinterpret_cast<uint4*>(tile + tile_k_row(D, row) + 16 * c) = k[i];
        *reinterpret_cast<uint4*>(tile + tile_v_row(D, row) + 16 * c) = v[i];
      }
    }
#pragma unroll
    for (int i = 0; i < WP; ++i) {
      const int piece = i * 32 + lane, row = piece / G, g = piece % G;
      if (row < rows) {
        *reinterpret_cast<uint32_t*>(tile + tile_k_word(D, G, row, g)) = kw[i];
        *reinterpret_cast<uint32_t*>(tile + tile_v_word(D, G, row, g)) = vw[i];
      }
    }
  }
};

// One warp per (entry, KV head, destination tile); where source and destination are one list, the first tile's warp takes
// all of the head's tiles in order. In place, idx ascends strictly, so row x comes from a row >= x: a tile's sources, and
// those of the tiles behind it, lie at or above its first row, and once a tile has been read nothing that is still to be
// read lies in it.
template <int D, int G>
__global__ void __launch_bounds__(kThreads) compact_move_kernel(PagesMoveArgs a, int tiles, int64_t items) {
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  int tile = (int)(item % tiles);
  const int h = (int)(item / tiles % a.p.Hkv);
  const int e = (int)(item / tiles / a.p.Hkv);
  const int cnt = a.plan[e];
  if (cnt <= 0) return;
  const int s = pages_list(a.p, a.src, e), d = pages_list(a.p, a.dst, e);
  const bool in_place = s == d;
  if (in_place && tile > 0) return;
  const int32_t* idx = a.idx ? a.idx + (int64_t)e * a.idx_stride + (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows : nullptr;
  if (in_place && !idx) return;
  const int end = in_place ? (cnt + kPageTile - 1) / kPageTile : min(tile + 1, (cnt + kPageTile - 1) / kPageTile);
  for (; tile < end; ++tile) {
    const int x = tile * kPageTile + lane;
    const int src = lane < kPageTile && x < cnt ? (idx ? idx[x] : x) : -1;
    const int rows = min(cnt - tile * kPageTile, kPageTile);
    if (in_place && __all_sync(0xffffffffu, src < 0 || src == x)) continue;      // nothing moves (and the page may be shared)
    TileRows<D, G> t;
    t.load(a.p, s, h, src, lane);
    __syncwarp();
    const int row0 = tile * kPageTile;
    const int page = pages_page(a.p, d, row0 / a.p.page_rows);
    if (page >= 0) t.store(a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile), rows, lane);
    __syncwarp();
  }
}

__global__ void __launch_bounds__(kThreads) compact_finish_kernel(PagesMoveArgs a) {
  const int e = blockIdx.x;
  const int cnt = a.plan[e];
  if (cnt < 0) return;
  const int s = pages_list(a.p, a.src, e), d = pages_list(a.p, a.dst, e);
  if (threadIdx.x == 0) a.p.lens[d] = cnt;
  if (s == d) drop_pages(a.p, d, (cnt + a.p.page_rows - 1) / a.p.page_rows);
}

template <int D, int G>
cudaError_t run_move(const PagesMoveArgs& a, int tiles, cudaStream_t s) {
  const int64_t items = (int64_t)a.n * a.p.Hkv * tiles;
  const int64_t grid = (items + kThreads / 32 - 1) / (kThreads / 32);
  if (grid > 0x7fffffffLL) return cudaErrorInvalidValue;
  compact_move_kernel<D, G><<<(unsigned)grid, kThreads, 0, s>>>(a, tiles, items);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_pages_reserve(const PagesReserveArgs& a, int* launches, cudaStream_t s) {
  const int words = (a.p.n_lists + 31) / 32;
  cudaError_t e = allow_shared<reserve_plan_kernel>(kMaxLists / 32 * 4);
  if (e != cudaSuccess) return e;
  reserve_plan_kernel<<<a.slices, kScanThreads, words * sizeof(uint32_t), s>>>(a, words);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  // enough CTAs to share out the heads when there are few lists to copy for
  int parts = 1;
  while (parts < 16 && parts < a.p.Hkv && (int64_t)a.n * parts < 256) parts *= 2;
  reserve_take_kernel<<<dim3(a.n, parts), kThreads, 0, s>>>(a);
  e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_fork(const PagesView& p, const int32_t* src, const int32_t* dst, int n, int* launches, cudaStream_t s) {
  fork_kernel<<<n, kThreads, 0, s>>>(p, src, dst, n);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_trim(const PagesView& p, const int32_t* lists, int n, const int32_t* rows, int* launches,
                              cudaStream_t s) {
  trim_kernel<<<n, kThreads, 0, s>>>(p, lists, n, rows);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_compact(const PagesMoveArgs& a, int* launches, cudaStream_t s) {
  compact_plan_kernel<<<a.n, kThreads, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  // a call whose two list arrays are one array compacts every entry in place: a warp per head is all it can use
  const int tiles = a.src == a.dst ? 1 : (a.n_rows + kPageTile - 1) / kPageTile;
  if (a.n_rows > 0) {
    const int G = a.p.D / a.p.group;
    if (a.p.D == 128) e = G == 4 ? run_move<128, 4>(a, tiles, s) : G == 2 ? run_move<128, 2>(a, tiles, s) : run_move<128, 1>(a, tiles, s);
    else e = G == 2 ? run_move<64, 2>(a, tiles, s) : run_move<64, 1>(a, tiles, s);
    if (e != cudaSuccess) return e;
    ++*launches;
  }
  compact_finish_kernel<<<a.n, kThreads, 0, s>>>(a);
  e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

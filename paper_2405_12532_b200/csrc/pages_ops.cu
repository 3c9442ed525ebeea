// Page management of the paged 4-bit cache: taking pages (with the copy that a shared, part-filled last page needs),
// forking, giving up and compacting lists. Tables, lengths and reference counts are device memory, so a call plans on
// the device, and every id that a table or a caller's list holds is range-checked before it is used.
#include "pyr_internal.h"

namespace pyr {
namespace {

constexpr int kThreads = 256;
constexpr int kListThreads = 128;        // of a CTA that serves one list's table (1280 lists: 6.0 us to fork, 7.4 with 256)
constexpr int kMoveThreads = 64;         // warps come and go on their own (64 lists of 32 heads, 1155 of 2176 rows: 160 us with 256, 152, 151)
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
struct Need { int err, old, slot, fresh; };        // fresh pages from slot `slot` on, and one more to copy page `old` to

__device__ __forceinline__ Need entry_need(const PagesReserveArgs& a, int i) {
  Need d{0, -1, 0, 0};
  const int l = pages_list(a.p, a.lists, i);
  const int add = a.rows ? a.rows[i] : a.rows_each;
  if (l < 0 || add < 0) {
    d.err = PYR_ERR_INVALID;
  } else if (add > 0) {
    const int len = pages_len(a.p, l);
    const int64_t rows = (int64_t)len + add;
    if (rows > (int64_t)a.p.max_pages * a.p.page_rows) {
      d.err = PYR_ERR_CAPACITY;
    } else {
      const int s1 = (int)((rows + a.p.page_rows - 1) / a.p.page_rows);
      if (len % a.p.page_rows) {               // the part-filled last page: a copy if others hold it too
        const int page = pages_page(a.p, l, len / a.p.page_rows);
        if (page < 0) d.err = PYR_ERR_INVALID;
        else if (a.p.refs[page] > 1) d.old = page;
      }
      d.slot = (len + a.p.page_rows - 1) / a.p.page_rows;
      while (d.slot < s1 && a.p.table[(size_t)l * a.p.max_pages + d.slot] >= 0) ++d.slot;   // reserved before
      d.fresh = s1 - d.slot;
    }
  }
  return d;
}

__global__ void __launch_bounds__(kScanThreads) reserve_plan_kernel(PagesReserveArgs a, int words) {
  extern __shared__ uint32_t seen[];     // a bit per list
  __shared__ long long sums[33];
  __shared__ int is_last, errors;
  const int t = threadIdx.x;
  long long total;
  let_next_start();
  // (looked up here, beside the pages, by every CTA: the one that plans then has it at hand)
  const Need first = t < a.n ? entry_need(a, t) : Need{0, -1, 0, 0};
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
  long long free_pages = total;
  if (a.slices > 1) {
    __threadfence();
    __syncthreads();
    if (t == 0) is_last = atomicAdd(&a.control[0], 1) == a.slices - 1;
    __syncthreads();
    if (!is_last) return;
    __threadfence();
    free_pages = 0;
    for (int s0 = 0; s0 < a.slices; s0 += kScanThreads) {
      const int s = s0 + t;
      const long long c = s < a.slices ? __ldcg(a.slice_first + s + 1) : 0;
      const long long before = free_pages + block_scan(c, sums, &total);
      if (s < a.slices) a.slice_first[s + 1] = (int32_t)(before + c);
      free_pages += total;
    }
  }
  for (int i = t; i < words; i += kScanThreads) seen[i] = 0;
  if (t == 0) { a.slice_first[0] = 0; a.control[0] = 0; errors = 0; }
  __syncthreads();

  long long taken = 0;
  for (int i0 = 0; i0 < a.n; i0 += kScanThreads) {
    const int i = i0 + t;
    Need d = i0 == 0 ? first : (i < a.n ? entry_need(a, i) : Need{0, -1, 0, 0});
    if (i < a.n) {
      const int l = pages_list(a.p, a.lists, i);
      if (l >= 0 && (atomicOr(&seen[l >> 5], 1u << (l & 31)) >> (l & 31) & 1u)) d.err = PYR_ERR_INVALID;
    }
    if (d.err) atomicCAS(&errors, 0, d.err);
    const long long need = d.err ? 0 : d.fresh + (d.old >= 0 ? 1 : 0);
    const long long base = taken + block_scan(need, sums, &total);
    taken += total;
    if (i < a.n)
      reinterpret_cast<int4*>(a.plan)[i] = make_int4((int)(base < 0x7fffffff ? base : 0x7fffffff), d.old, d.slot, d.fresh);
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

// Copies the first `rows` rows of the heads [h0, h1) of a page to another page, 16 bytes a thread at a time whatever the head:
// whole tiles as they lie, of a part-filled tile the rows' codes and (4 bytes at a time) words.
__device__ __forceinline__ void copy_rows_of_page(const PagesView& p, int from, int to, int h0, int h1, int rows) {
  const int G = p.D / p.group, half = kPageTile * p.D / 2, heads = h1 - h0;
  const size_t head_bytes = (size_t)p.tiles_per_page * p.tile_bytes;
  const uint8_t* s = p.pool + pages_tile(p, from, h0, 0);
  uint8_t* d = p.pool + pages_tile(p, to, h0, 0);
  const int whole = rows / kPageTile * p.tile_bytes, left = rows % kPageTile;
  const int codes = left * p.D / 2, words = left * G * 4;
  const int per16 = whole / 16 + 2 * codes / 16, per4 = 2 * words / 4;
  auto place = [&](int x) {                      // of the x-th 16-byte piece of a head
    const int o = x * 16;
    if (o < whole) return o;
    const int c = o - whole;
    return whole + (c < codes ? c : half + c - codes);
  };
#pragma unroll 4
  for (int x = threadIdx.x; x < heads * per16; x += kThreads) {
    const int h = x / per16;
    const size_t at = h * head_bytes + place(x - h * per16);
    *reinterpret_cast<uint4*>(d + at) = *reinterpret_cast<const uint4*>(s + at);
  }
#pragma unroll 2
  for (int x = threadIdx.x; x < heads * per4; x += kThreads) {
    const int h = x / per4, o = (x - h * per4) * 4;
    const size_t at = h * head_bytes + whole + 2 * half + (o < words ? o : kPageTile * G * 4 + o - words);
    *reinterpret_cast<uint32_t*>(d + at) = *reinterpret_cast<const uint32_t*>(s + at);
  }
}

// grid (entries, parts): part 0 writes the entry's table and counts, every part copies its share of the heads.
__global__ void __launch_bounds__(kThreads) reserve_take_kernel(PagesReserveArgs a) {
  wait_for_previous();
  const int i = blockIdx.x;
  const int4 pl = reinterpret_cast<const int4*>(a.plan)[i];
  if (a.control[1] == 0) return;
  const int base = pl.x, old = pl.y, slot = pl.z, fresh = pl.w;
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
    const int share = (a.p.Hkv + gridDim.y - 1) / gridDim.y, h0 = blockIdx.y * share, h1 = min(h0 + share, a.p.Hkv);
    if (h0 < h1) copy_rows_of_page(a.p, old, to, h0, h1, len % a.p.page_rows);
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
__global__ void __launch_bounds__(kListThreads) fork_kernel(PagesView p, const int32_t* src, const int32_t* dst, int n) {
  const int e = blockIdx.x;
  const int s = pages_list(p, src, e), d = pages_list(p, dst, e);
  bool bad = s < 0 || d < 0;
#pragma unroll 4
  for (int x = threadIdx.x; x < n; x += kListThreads) bad |= (x != e && dst[x] == d) | (src[x] == d);
  int pages = 0, len = 0;
  if (s >= 0 && d >= 0) {
    len = pages_len(p, s);
    pages = (len + p.page_rows - 1) / p.page_rows;
    bad = bad || p.lens[d] != 0 || p.table[(size_t)d * p.max_pages] >= 0;
    for (int x = threadIdx.x; x < pages; x += kListThreads) bad = bad || pages_page(p, s, x) < 0;
  }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) record(p.status, PYR_ERR_INVALID);
    return;
  }
  for (int x = threadIdx.x; x < pages; x += kListThreads) {
    const int id = pages_page(p, s, x);
    p.table[(size_t)d * p.max_pages + x] = id;
    atomicAdd(&p.refs[id], 1);
  }
  if (threadIdx.x == 0) p.lens[d] = len;
}

// Gives up the pages of list l from slot `first` on. A table entry is taken by exchange, so that a list named twice gives
// a page up once.
__device__ __forceinline__ void drop_pages(const PagesView& p, int l, int first, int index, int threads) {
  int32_t* row = p.table + (size_t)l * p.max_pages;
  for (int x = first + index; x < p.max_pages; x += threads) {
    if (row[x] < 0) continue;
    const int id = atomicExch(&row[x], -1);
    if (id >= 0 && id < p.n_pages) atomicSub(&p.refs[id], 1);
  }
}

__global__ void __launch_bounds__(kListThreads) trim_kernel(PagesView p, const int32_t* lists, int n, const int32_t* rows) {
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
  drop_pages(p, l, (keep + p.page_rows - 1) / p.page_rows, threadIdx.x, kListThreads);
}

// ------------------------------------------------------------------ compact
__device__ __forceinline__ int entry_count(const PagesMoveArgs& a, int e) { return a.counts ? a.counts[e] : a.n_rows; }

// Checks every entry before a row moves; grid (entries, index lists of an entry). Whatever is wrong sets refused[e].
__global__ void __launch_bounds__(kThreads) compact_check_kernel(PagesMoveArgs a) {
  const int e = blockIdx.x, t = threadIdx.x;
  const PagesView& p = a.p;
  let_next_start();
  const int s = pages_list(p, a.src, e), d = pages_list(p, a.dst, e);
  const int cnt = entry_count(a, e);
  bool bad = s < 0 || d < 0 || cnt < 0 || cnt > a.n_rows || (int64_t)cnt > (int64_t)p.max_pages * p.page_rows;
  if (!bad) {
    const bool in_place = s == d;
    const int len = pages_len(p, s);
    if (a.idx) {
      const int32_t* row = a.idx + (int64_t)e * a.idx_stride + (int64_t)blockIdx.y * a.n_rows;
#pragma unroll 4
      for (int x = t; x < cnt; x += kThreads) {
        const int v = row[x];
        bad |= v < 0 || v >= len;
        if (in_place) {
          bad |= x > 0 && row[x - 1] >= v;
          if (v != x) {
            const int id = pages_page(p, d, x / p.page_rows);
            bad |= id < 0 || p.refs[id] != 1;
          }
        }
      }
    } else {
      bad = cnt > len;
    }
    if (blockIdx.y == 0) {
#pragma unroll 4
      for (int x = t; x < a.n; x += kThreads) bad |= x != e && (a.dst[x] == d || a.src[x] == d);
      const int pages = (cnt + p.page_rows - 1) / p.page_rows, from = (len + p.page_rows - 1) / p.page_rows;
      for (int x = t; x < pages; x += kThreads) {
        const int id = pages_page(p, d, x);
        bad |= id < 0 || (!in_place && p.refs[id] != 1);
      }
      for (int x = t; x < from; x += kThreads) bad |= pages_page(p, s, x) < 0;
    }
  }
  if (__syncthreads_or(bad) && t == 0) {
    a.refused[e] = 1;
    record(p.status, PYR_ERR_INVALID);
  }
}

// Where a list's row lies: its tile (0: nowhere) and its row there.
struct RowPlace { unsigned long long tile; int row; };
__device__ __forceinline__ RowPlace row_place(const PagesView& p, int l, int h, int row) {
  RowPlace r{0, 0};
  if (row < 0) return r;
  const int slot = row / p.page_rows, in = row - slot * p.page_rows;
  const int page = pages_page(p, l, slot);
  if (page < 0) return r;
  r.tile = reinterpret_cast<unsigned long long>(p.pool + pages_tile(p, page, h, in / kPageTile));
  r.row = in % kPageTile;
  return r;
}

// A row's codes are 64 bytes (32 with 64 dimensions), and rows between kept ones are not wanted: without the hint the L2 cache
// fetches lines of 128 bytes (64 lists of 32 heads, 1155 of 2176 rows: 170 us and 1.56 times the kept rows' bytes read, 162 us and 1.13
// times with it).
__device__ __forceinline__ uint4 load_codes(const uint8_t* p) {
  uint4 r;
  asm volatile("ld.global.L2::64B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
  return r;
}

// The bytes that one warp moves for a tile of destination rows, held in registers between the reads and the writes.
template <int D, int G>
struct TileRows {
  static constexpr int C = D / 32;                       // 16-byte pieces of a row of codes
  static constexpr int CP = kPageTile * C / 32;          // pieces a lane holds of K, and of V
  static constexpr int WP = (kPageTile * G + 31) / 32;   // words a lane holds of K, and of V
  uint4 k[CP], v[CP];
  uint32_t kw[WP], vw[WP];

  // lanes first .. first + 15 know the source rows of the tile
  __device__ __forceinline__ void load(const RowPlace& from, int first, int lane) {
#pragma unroll
    for (int i = 0; i < CP; ++i) {
      const int piece = i * 32 + lane, row = piece / C, c = piece % C;
      const uint8_t* b = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, from.tile, first + row));
      const int rr = __shfl_sync(0xffffffffu, from.row, first + row);
      if (b) {
        k[i] = load_codes(b + tile_k_row(D, rr) + 16 * c);
        v[i] = load_codes(b + tile_v_row(D, rr) + 16 * c);
      }
    }
#pragma unroll
    for (int i = 0; i < WP; ++i) {
      const int piece = i * 32 + lane, row = piece / G < kPageTile ? piece / G : 0, g = piece % G;
      const uint8_t* b = reinterpret_cast<const uint8_t*>(__shfl_sync(0xffffffffu, from.tile, first + row));
      const int rr = __shfl_sync(0xffffffffu, from.row, first + row);
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

// What is left to do for an entry once its rows have moved, by `threads` threads: the length, and in place the pages behind it.
__device__ __forceinline__ void finish_entry(const PagesMoveArgs& a, int e, int index, int threads) {
  if (a.refused[e]) return;
  const int cnt = entry_count(a, e);
  const int s = pages_list(a.p, a.src, e), d = pages_list(a.p, a.dst, e);
  if (index == 0) a.p.lens[d] = cnt;
  if (s == d) drop_pages(a.p, d, (cnt + a.p.page_rows - 1) / a.p.page_rows, index, threads);
}

// Where no row moves.
__global__ void __launch_bounds__(kThreads) compact_finish_kernel(PagesMoveArgs a) {
  wait_for_previous();
  const int e = blockIdx.x;
  finish_entry(a, e, threadIdx.x, kThreads);
  __syncthreads();
  if (threadIdx.x == 0) a.refused[e] = 0;          // as the next call expects it
}

// Into another list: one warp per (entry, KV head, run of kRun destination tiles), the next tile's rows on their way while one
// is stored. (An entry whose list is its own destination is left to the first run's warp, tile by tile, see below.)
template <int D, int G, int kRun>
__device__ __forceinline__ void move_run(const PagesMoveArgs& a, int e, int h, int run, int lane) {
  const int cnt = entry_count(a, e), x0 = run * kRun * kPageTile;
  if (x0 >= cnt || a.refused[e]) return;
  const int s = pages_list(a.p, a.src, e), d = pages_list(a.p, a.dst, e);
  const int32_t* idx = a.idx ? a.idx + (int64_t)e * a.idx_stride + (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows : nullptr;
  if (s == d) {
    if (run != 0 || !idx) return;                // (a copy of a list to itself is done)
    for (int row0 = 0; row0 < cnt; row0 += kPageTile) {
      const int x = row0 + lane, src = lane < kPageTile && x < cnt ? idx[x] : -1;
      if (!__any_sync(0xffffffffu, src >= 0 && src != x)) continue;
      TileRows<D, G> rows;
      rows.load(row_place(a.p, s, h, src), 0, lane);
      __syncwarp();
      const int page = pages_page(a.p, d, row0 / a.p.page_rows);
      if (page >= 0) rows.store(a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile), min(cnt - row0, kPageTile), lane);
      __syncwarp();
    }
    return;
  }
  // source rows of the run (lane l: rows l, l + 32, .. of it) and the pages that its tiles go to (lane t: tile t), looked up
  // together: what follows needs no address that is still to be fetched
  constexpr int kRows = kRun * kPageTile, kPlaces = (kRows + 31) / 32;
  RowPlace from[kPlaces];
#pragma unroll
  for (int k = 0; k < kPlaces; ++k) {
    const int in = 32 * k + lane, x = x0 + in;
    from[k] = row_place(a.p, s, h, in < kRows && x < cnt ? (idx ? idx[x] : x) : -1);
  }
  const int to_row = x0 + (lane & (kRun - 1)) * kPageTile;
  const int to_page = to_row < cnt ? pages_page(a.p, d, to_row / a.p.page_rows) : -1;
  const unsigned long long to = to_page < 0 ? 0 : reinterpret_cast<unsigned long long>(
      a.p.pool + pages_tile(a.p, to_page, h, to_row % a.p.page_rows / kPageTile));
  TileRows<D, G> rows[2];
  rows[0].load(from[0], 0, lane);
#pragma unroll
  for (int t = 0; t < kRun; ++t) {
    if (t + 1 < kRun && x0 + (t + 1) * kPageTile < cnt) rows[(t + 1) & 1].load(from[(t + 1) >> 1], ((t + 1) & 1) * kPageTile, lane);
    uint8_t* tile = reinterpret_cast<uint8_t*>(__shfl_sync(0xffffffffu, to, t));
    const int n = cnt - x0 - t * kPageTile;
    if (n > 0 && tile) rows[t & 1].store(tile, min(n, kPageTile), lane);
  }
}

// The warp that is the last of its entry finishes it: no other looks at the entry's table any more.
template <int D, int G, int kRun>
__global__ void __launch_bounds__(kMoveThreads) compact_move_kernel(PagesMoveArgs a, int runs, int64_t items) {
  wait_for_previous();
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * (kMoveThreads / 32) + (threadIdx.x >> 5);
  if (item >= items) return;
  const int run = (int)(item % runs);
  const int h = (int)(item / runs % a.p.Hkv);
  const int e = (int)(item / runs / a.p.Hkv);
  move_run<D, G, kRun>(a, e, h, run, lane);
  __syncwarp();
  int order = 0;
  if (lane == 0) order = atomicAdd(&a.moved[e], 1);
  if (__shfl_sync(0xffffffffu, order, 0) != a.p.Hkv * runs - 1) return;
  finish_entry(a, e, lane, 32);
  __syncwarp();
  if (lane == 0) a.refused[e] = a.moved[e] = 0;    // as the next call expects them
}

// In place: one CTA per (entry, KV head), a tile a warp, front to back. idx ascends strictly, so row x comes from a row >= x:
// once the rows of a step's tiles have been read, nothing that later steps read lies in those tiles, and one barrier a step
// (between its reads and its writes) is enough.
template <int D, int G>
__global__ void __launch_bounds__(kThreads) compact_inplace_kernel(PagesMoveArgs a) {
  wait_for_previous();
  constexpr int kStep = kThreads / 32;
  __shared__ int is_last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int e = blockIdx.x / a.p.Hkv, h = blockIdx.x % a.p.Hkv;
  const int cnt = a.refused[e] ? 0 : entry_count(a, e);
  const int l = pages_list(a.p, a.dst, e);
  const int32_t* idx = a.idx + (int64_t)e * a.idx_stride + (int64_t)(a.idx_groups == 1 ? 0 : h) * a.n_rows;
  const int tiles = (cnt + kPageTile - 1) / kPageTile;
  TileRows<D, G> rows;
  for (int t0 = 0; t0 < tiles; t0 += kStep) {
    const int row0 = (t0 + warp) * kPageTile, x = row0 + lane;
    const int src = lane < kPageTile && x < cnt ? idx[x] : -1;
    // (a tile of which no row moves is not written: its page may be shared)
    const bool moves = __any_sync(0xffffffffu, src >= 0 && src != x);
    const int page = moves ? pages_page(a.p, l, row0 / a.p.page_rows) : -1;
    if (moves) rows.load(row_place(a.p, l, h, src), 0, lane);
    __syncthreads();
    if (page >= 0)
      rows.store(a.p.pool + pages_tile(a.p, page, h, row0 % a.p.page_rows / kPageTile), min(cnt - row0, kPageTile), lane);
  }
  // the CTA that is the last of its entry finishes it: no other looks at the entry's table any more
  __syncthreads();
  if (threadIdx.x == 0) is_last = atomicAdd(&a.moved[e], 1) == a.p.Hkv - 1;
  __syncthreads();
  if (!is_last) return;
  finish_entry(a, e, threadIdx.x, kThreads);
  __syncthreads();
  if (threadIdx.x == 0) a.refused[e] = a.moved[e] = 0;   // as the next call expects them
}

template <int D, int G, int kRun>
cudaError_t run_runs(const PagesMoveArgs& a, cudaStream_t s) {
  const int runs = (a.n_rows + kRun * kPageTile - 1) / (kRun * kPageTile);
  const int64_t items = (int64_t)a.n * a.p.Hkv * runs;
  const int64_t grid = (items + kMoveThreads / 32 - 1) / (kMoveThreads / 32);
  if (grid > 0x7fffffffLL || (int64_t)a.p.Hkv * runs > 0x7fffffffLL) return cudaErrorInvalidValue;
  return launch_behind(compact_move_kernel<D, G, kRun>, dim3((unsigned)grid), dim3(kMoveThreads), 0, s, a, runs, items);
}

template <int D, int G>
cudaError_t run_move(const PagesMoveArgs& a, cudaStream_t s) {
  if (a.src == a.dst) {                          // one array for both: every entry is compacted in place
    const int64_t heads = (int64_t)a.n * a.p.Hkv;
    if (heads > 0x7fffffffLL) return cudaErrorInvalidValue;
    return launch_behind(compact_inplace_kernel<D, G>, dim3((unsigned)heads), dim3(kThreads), 0, s, a);
  }
  // Runs of four tiles where there are enough of them to give every SM 32 warps (64 lists of 32 heads: 151 us), else a tile a
  // warp: then a warp's own latency is what counts (4 lists of 8 heads, 717 rows: 6.6 us, 11 with runs of four).
  const int sms = device_sm_count();
  if (sms <= 0) return cudaErrorUnknown;
  const int64_t runs = (int64_t)a.n * a.p.Hkv * ((a.n_rows + 4 * kPageTile - 1) / (4 * kPageTile));
  return runs >= 32LL * sms ? run_runs<D, G, 4>(a, s) : run_runs<D, G, 1>(a, s);
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
  e = launch_behind(reserve_take_kernel, dim3(a.n, parts), dim3(kThreads), 0, s, a);
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_fork(const PagesView& p, const int32_t* src, const int32_t* dst, int n, int* launches, cudaStream_t s) {
  fork_kernel<<<n, kListThreads, 0, s>>>(p, src, dst, n);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_trim(const PagesView& p, const int32_t* lists, int n, const int32_t* rows, int* launches,
                              cudaStream_t s) {
  trim_kernel<<<n, kListThreads, 0, s>>>(p, lists, n, rows);
  const cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess) ++*launches;
  return e;
}

cudaError_t launch_pages_compact(const PagesMoveArgs& a, int* launches, cudaStream_t s) {
  compact_check_kernel<<<dim3(a.n, a.idx ? a.idx_groups : 1), kThreads, 0, s>>>(a);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  ++*launches;
  const int G = a.p.D / a.p.group;
  if (a.n_rows == 0 || (a.src == a.dst && !a.idx)) e = launch_behind(compact_finish_kernel, dim3(a.n), dim3(kThreads), 0, s, a);
  else if (a.p.D == 128) e = G == 4 ? run_move<128, 4>(a, s) : G == 2 ? run_move<128, 2>(a, s) : run_move<128, 1>(a, s);
  else e = G == 2 ? run_move<64, 2>(a, s) : run_move<64, 1>(a, s);
  if (e == cudaSuccess) ++*launches;
  return e;
}

}  // namespace pyr

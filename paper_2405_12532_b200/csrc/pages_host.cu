// Host side of the paged 4-bit cache (pyr_pages_*): argument checks, carving of the caller's buffer, dispatch. Nothing here
// reads device memory: lengths and tables live on the device, and what depends on them is checked by the kernels.
#include <cmath>
#include <new>
#include <utility>

#include "pyr_internal.h"

namespace {

constexpr size_t kAlign = 256;
constexpr int32_t kMaxRows = 1 << 30;      // of a call's entry: row arithmetic stays within 32 bits
constexpr uint64_t kMaxPool = 1ull << 56;  // bytes of a pool
inline size_t align_up(size_t x) { return (x + kAlign - 1) / kAlign * kAlign; }

struct PagesLayout {
  size_t status, control, arrived, refused, moved, lens, refs, table, plan, free_ids, slice_first, partial, pool, total;
  int slices;
};

pyr_status_t validate(const pyr_pages_config_t* c) {
  if (!c) return PYR_ERR_NULL;
  if (c->n_kv_heads < 1 || c->n_pages < 1 || c->n_lists < 1 || c->max_pages < 1 || c->page_rows < 1 || c->flags != 0)
    return PYR_ERR_INVALID;
  if (c->head_dim != 64 && c->head_dim != 128) return PYR_ERR_UNSUPPORTED;
  if (c->group != 32 && c->group != 64 && c->group != 128) return PYR_ERR_UNSUPPORTED;
  if (c->group > c->head_dim) return PYR_ERR_INVALID;
  if (c->page_rows % pyr::kPageTile || c->page_rows > pyr::kMaxPageRows || c->n_lists > pyr::kMaxLists ||
      c->n_kv_heads > 65535)
    return PYR_ERR_UNSUPPORTED;
  // a list's length is an int32, and so is every page id that the reserve scan rounds up to whole slices
  if ((int64_t)c->max_pages * c->page_rows > 0x7fffffff - pyr::kMaxPageRows || c->n_pages > 0x7fffffff - pyr::kReserveSlice)
    return PYR_ERR_UNSUPPORTED;
  // the buffer's size in bytes must be a number of 64 bits with room to spare (the table's is: 2^19 lists of 2^27 pages)
  const uint64_t page_bytes = (uint64_t)c->n_kv_heads * (c->page_rows / pyr::kPageTile) * pyr::pages_tile_bytes(c->head_dim, c->group);
  if (page_bytes > kMaxPool / (uint64_t)c->n_pages) return PYR_ERR_UNSUPPORTED;
  return PYR_OK;
}

void plan(const pyr_pages_config_t* c, PagesLayout* l) {
  size_t off = 0;
  auto take = [&](size_t bytes) { const size_t at = off; off = align_up(off + bytes); return at; };
  l->slices = (c->n_pages + pyr::kReserveSlice - 1) / pyr::kReserveSlice;
  l->status = take(pyr::kStatusWords * 4);
  l->control = take(64 * 4);
  l->arrived = take((size_t)pyr::kAttnMaxCtas * 4);
  l->refused = take((size_t)c->n_lists * 4);
  l->moved = take((size_t)c->n_lists * 4);
  l->lens = take((size_t)c->n_lists * 4);
  l->refs = take((size_t)c->n_pages * 4);
  l->table = take((size_t)c->n_lists * c->max_pages * 4);
  l->plan = take((size_t)c->n_lists * 4 * 4);
  l->free_ids = take((size_t)l->slices * pyr::kReserveSlice * 4);
  l->slice_first = take((size_t)(l->slices + 1) * 4);
  l->partial = take((size_t)pyr::kAttnMaxCtas * 2 * pyr::kAttnCols * (c->head_dim + 2) * 4);
  l->pool = take((size_t)c->n_pages * c->n_kv_heads * (c->page_rows / pyr::kPageTile) *
                 pyr::pages_tile_bytes(c->head_dim, c->group));
  l->total = off;
}

}  // namespace

struct pyr_pages {
  pyr_pages_config_t cfg;
  PagesLayout lay;
  char* base;
  bool ready;        // pyr_pages_reset has been called
};

namespace {

template <class T>
T* at(const pyr_pages* h, size_t off) { return reinterpret_cast<T*>(h->base + off); }

pyr::PagesView view(const pyr_pages* h) {
  const pyr_pages_config_t& c = h->cfg;
  pyr::PagesView p;
  p.pool = at<uint8_t>(h, h->lay.pool);
  p.table = at<int32_t>(h, h->lay.table);
  p.lens = at<int32_t>(h, h->lay.lens);
  p.refs = at<int32_t>(h, h->lay.refs);
  p.status = at<int>(h, h->lay.status);
  p.Hkv = c.n_kv_heads; p.D = c.head_dim; p.group = c.group; p.page_rows = c.page_rows;
  p.tiles_per_page = c.page_rows / pyr::kPageTile;
  p.tile_bytes = pyr::pages_tile_bytes(c.head_dim, c.group);
  p.n_pages = c.n_pages; p.n_lists = c.n_lists; p.max_pages = c.max_pages;
  return p;
}

// handle and entry count of a launching call; an entry needs a list of its own only where lists are written, but no call
// has more entries than there are lists except attention, reading and forking from, which may repeat them
pyr_status_t check_call(const pyr_pages* h, int32_t n, bool distinct) {
  if (!h) return PYR_ERR_NULL;
  if (n < 0 || (distinct && n > h->cfg.n_lists)) return PYR_ERR_INVALID;
  return PYR_OK;
}

// With lists == NULL entry i is list i, so there cannot be more entries than lists.
bool default_lists_fit(const pyr_pages* h, const int32_t* lists, int32_t n) { return lists || n <= h->cfg.n_lists; }

// rows of [n, rows, heads, D] tensors: 16-byte aligned, innermost dimension contiguous (the stride of a dimension of size 1 is not
// looked at)
pyr_status_t check_rows(const pyr_pages* h, const void* a, const void* b, int32_t dtype, int64_t sb, int64_t sn, int64_t sh,
                        int64_t n, int64_t rows, int heads) {
  if ((!a || !b) && n > 0 && rows > 0) return PYR_ERR_NULL;      // (a tensor without elements needs no address)
  if (dtype != PYR_BF16 && dtype != PYR_F32) return PYR_ERR_UNSUPPORTED;
  const int D = h->cfg.head_dim, eb = dtype == PYR_BF16 ? 2 : 4;
  if (n <= 1) sb = 0;
  if (rows <= 1) sn = 0;
  if (heads <= 1) sh = 0;
  if (sb < 0 || sn < 0 || sh < 0 || (heads > 1 && sh < D)) return PYR_ERR_INVALID;
  if ((reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b)) % 16 || (sb * eb) % 16 || (sn * eb) % 16 ||
      (sh * eb) % 16)
    return PYR_ERR_INVALID;
  return PYR_OK;
}

// Whether a call's tiles, of all entries and heads, can be counted in 31 bits (a launch has a warp for each).
bool tiles_fit(const pyr_pages* h, int64_t n, int32_t n_rows) {
  const int64_t tiles = ((int64_t)n_rows + 2 * pyr::kPageTile - 2) / pyr::kPageTile;
  return tiles == 0 || n * h->cfg.n_kv_heads <= 0x7fffffff / tiles;
}

// Whether the rows of a tensor that is written lie apart: each stride passes everything that the smaller ones span.
bool rows_apart(const pyr_pages* h, int64_t sb, int64_t sn, int64_t sh, int64_t n, int64_t rows, int64_t heads) {
  struct { int64_t stride, size; } d[3] = {{sh, heads}, {sn, rows}, {sb, n}};
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2 - i; ++j)
      if (d[j].stride > d[j + 1].stride) std::swap(d[j], d[j + 1]);
  __int128 span = h->cfg.head_dim;
  for (const auto& x : d) {
    if (x.size <= 1) continue;
    if (x.stride < span) return false;
    span += (__int128)x.stride * (x.size - 1);
  }
  return true;
}

pyr_status_t check_idx(const pyr_pages* h, const int32_t* idx, int32_t groups, int64_t stride, int32_t n_rows) {
  if (!idx) return PYR_OK;
  if (groups != 1 && groups != h->cfg.n_kv_heads) return PYR_ERR_INVALID;
  return stride >= 0 ? (n_rows >= 0 ? PYR_OK : PYR_ERR_INVALID) : PYR_ERR_INVALID;
}

}  // namespace

// The last check of a launching call: everything that the arguments alone decide has been refused before it.
#define PYR_PAGES_READY(h) do { if (!(h)->ready) return PYR_ERR_ORDER; } while (0)
#define PYR_PAGES(call) do { int launches = 0; const cudaError_t e_ = (call); pyr::count_launches(launches); \
                             return e_ == cudaSuccess ? PYR_OK : PYR_ERR_CUDA; } while (0)

extern "C" {

pyr_status_t pyr_pages_bytes(const pyr_pages_config_t* cfg, size_t* bytes, size_t* align) {
  const pyr_status_t st = validate(cfg);
  if (st != PYR_OK) return st;
  if (!bytes) return PYR_ERR_NULL;
  PagesLayout lay;
  plan(cfg, &lay);
  *bytes = lay.total;
  if (align) *align = kAlign;
  return PYR_OK;
}

pyr_status_t pyr_pages_alloc(const pyr_pages_config_t* cfg, void* dev_buf, size_t bytes, pyr_pages_t** out) {
  const pyr_status_t st = validate(cfg);
  if (st != PYR_OK) return st;
  if (!dev_buf || !out) return PYR_ERR_NULL;
  if (reinterpret_cast<uintptr_t>(dev_buf) % kAlign) return PYR_ERR_INVALID;
  PagesLayout lay;
  plan(cfg, &lay);
  if (bytes < lay.total) return PYR_ERR_BUFFER_TOO_SMALL;
  pyr_pages* h = new (std::nothrow) pyr_pages();
  if (!h) return PYR_ERR_HOST_MEMORY;
  h->cfg = *cfg;
  h->lay = lay;
  h->base = static_cast<char*>(dev_buf);
  h->ready = false;
  *out = h;
  return PYR_OK;
}

pyr_status_t pyr_pages_free(pyr_pages_t* h) {
  if (!h) return PYR_ERR_NULL;
  delete h;
  return PYR_OK;
}

pyr_status_t pyr_pages_reset(pyr_pages_t* h, void* stream) {
  if (!h) return PYR_ERR_NULL;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess ||
      cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess)
    return PYR_ERR_CUDA;
  if (major != 10) return PYR_ERR_UNSUPPORTED;
  const PagesLayout& l = h->lay;
  // status, control words, arrival counters, refusals, move counters, lengths and reference counts lie one behind the other
  if (cudaMemsetAsync(h->base + l.status, 0, l.table - l.status, s) != cudaSuccess) return PYR_ERR_CUDA;
  if (cudaMemsetAsync(h->base + l.table, 0xff, l.plan - l.table, s) != cudaSuccess) return PYR_ERR_CUDA;
  h->ready = true;
  return PYR_OK;
}

pyr_status_t pyr_pages_view(const pyr_pages_t* h, void** pool, size_t* page_bytes, int32_t** table, int32_t** lens,
                            int32_t** refs) {
  if (!h) return PYR_ERR_NULL;
  const pyr::PagesView p = view(h);
  if (pool) *pool = p.pool;
  if (page_bytes) *page_bytes = pyr::pages_page_bytes(p);
  if (table) *table = p.table;
  if (lens) *lens = p.lens;
  if (refs) *refs = p.refs;
  return PYR_OK;
}

pyr_status_t pyr_pages_status(pyr_pages_t* h, void* stream, int32_t* host_status) {
  if (!h || !host_status) return PYR_ERR_NULL;
  if (!h->ready) return PYR_ERR_ORDER;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  int word = 0;
  if (cudaMemcpyAsync(&word, at<int>(h, h->lay.status), sizeof(int), cudaMemcpyDeviceToHost, s) != cudaSuccess ||
      cudaStreamSynchronize(s) != cudaSuccess)
    return PYR_ERR_CUDA;
  if (word != 0 && (cudaMemsetAsync(at<int>(h, h->lay.status), 0, sizeof(int), s) != cudaSuccess ||
                    cudaStreamSynchronize(s) != cudaSuccess))
    return PYR_ERR_CUDA;
  *host_status = word;
  return static_cast<pyr_status_t>(word);
}

pyr_status_t pyr_pages_reserve(pyr_pages_t* h, const int32_t* lists, int32_t n, const int32_t* rows, int32_t rows_each,
                               void* stream) {
  const pyr_status_t st = check_call(h, n, true);
  if (st != PYR_OK) return st;
  if (!rows && rows_each < 0) return PYR_ERR_INVALID;
  PYR_PAGES_READY(h);
  if (n == 0) return PYR_OK;
  pyr::PagesReserveArgs a;
  a.p = view(h);
  a.lists = lists; a.n = n; a.rows = rows; a.rows_each = rows_each;
  a.slices = h->lay.slices;
  a.free_ids = at<int32_t>(h, h->lay.free_ids);
  a.slice_first = at<int32_t>(h, h->lay.slice_first);
  a.plan = at<int32_t>(h, h->lay.plan);
  a.control = at<int32_t>(h, h->lay.control);
  PYR_PAGES(pyr::launch_pages_reserve(a, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_write(pyr_pages_t* h, const int32_t* lists, int32_t n, const int32_t* first, const void* k,
                             const void* v, int64_t sb, int64_t sn, int64_t sh, int32_t src_rows, int32_t dtype,
                             const int32_t* idx, int32_t idx_groups, int64_t idx_stride, const int32_t* counts,
                             int32_t n_rows, void* stream) {
  pyr_status_t st = check_call(h, n, true);
  if (st == PYR_OK) st = check_rows(h, k, v, dtype, sb, sn, sh, n, src_rows, h->cfg.n_kv_heads);
  if (st == PYR_OK) st = check_idx(h, idx, idx_groups, idx_stride, n_rows);
  if (st != PYR_OK) return st;
  if (n_rows < 0 || src_rows < 0 || (!idx && n_rows > src_rows)) return PYR_ERR_INVALID;
  if (n_rows > kMaxRows || !tiles_fit(h, n, n_rows)) return PYR_ERR_UNSUPPORTED;
  PYR_PAGES_READY(h);
  if (n == 0 || n_rows == 0) return PYR_OK;
  pyr::PagesWriteArgs a;
  a.p = view(h);
  a.lists = lists; a.n = n; a.first = first; a.k = k; a.v = v; a.sb = sb; a.sn = sn; a.sh = sh;
  a.src_rows = src_rows; a.dtype = dtype; a.idx = idx; a.idx_groups = idx ? idx_groups : 1; a.idx_stride = idx_stride;
  a.counts = counts; a.n_rows = n_rows;
  a.plan = at<int32_t>(h, h->lay.plan);
  PYR_PAGES(pyr::launch_pages_write(a, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_read(pyr_pages_t* h, const int32_t* lists, int32_t n, const int32_t* first, void* k, void* v,
                            int64_t sb, int64_t sn, int64_t sh, int32_t dtype, const int32_t* counts, int32_t n_rows,
                            void* stream) {
  pyr_status_t st = check_call(h, n, false);
  if (st == PYR_OK) st = check_rows(h, k, v, dtype, sb, sn, sh, n, n_rows, h->cfg.n_kv_heads);
  if (st != PYR_OK) return st;
  if (n_rows < 0 || !default_lists_fit(h, lists, n)) return PYR_ERR_INVALID;
  // rows that overlap would be written by several threads
  if (!rows_apart(h, sb, sn, sh, n, n_rows, h->cfg.n_kv_heads)) return PYR_ERR_INVALID;
  if (n_rows > kMaxRows || !tiles_fit(h, n, n_rows)) return PYR_ERR_UNSUPPORTED;
  PYR_PAGES_READY(h);
  if (n == 0 || n_rows == 0) return PYR_OK;
  pyr::PagesWriteArgs a;
  a.p = view(h);
  a.lists = lists; a.n = n; a.first = first; a.k = k; a.v = v; a.sb = sb; a.sn = sn; a.sh = sh;
  a.src_rows = n_rows; a.dtype = dtype; a.idx = nullptr; a.idx_groups = 1; a.idx_stride = 0;
  a.counts = counts; a.n_rows = n_rows;
  a.plan = nullptr;
  PYR_PAGES(pyr::launch_pages_read(a, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_attn(pyr_pages_t* h, const int32_t* lists, int32_t n, const void* q, int64_t qsb, int64_t qst,
                            int64_t qsh, void* out, int64_t osb, int64_t ost, int64_t osh, float* lse, int32_t q_len,
                            int32_t n_q_heads, int32_t dtype, float softmax_scale, void* stream) {
  pyr_status_t st = check_call(h, n, false);
  if (st != PYR_OK) return st;
  if (q_len < 1 || n_q_heads < 1 || n_q_heads % h->cfg.n_kv_heads || !default_lists_fit(h, lists, n)) return PYR_ERR_INVALID;
  if (!(softmax_scale >= 0.0f) || softmax_scale > 0x1p127f) return PYR_ERR_INVALID;     // (times log2 e it is a number)
  st = check_rows(h, q, q, dtype, qsb, qst, qsh, n, q_len, n_q_heads);
  if (st == PYR_OK) st = check_rows(h, out, out, dtype, osb, ost, osh, n, q_len, n_q_heads);
  if (st != PYR_OK) return st;
  const int64_t cols = (int64_t)q_len * (n_q_heads / h->cfg.n_kv_heads);
  if (cols > (1 << 20)) return PYR_ERR_UNSUPPORTED;
  if (!rows_apart(h, osb, ost, osh, n, q_len, n_q_heads)) return PYR_ERR_INVALID;
  PYR_PAGES_READY(h);
  if (n == 0) return PYR_OK;
  pyr::PagesAttnArgs a;
  a.p = view(h);
  a.lists = lists; a.n = n; a.q = q; a.out = out; a.lse = lse;
  a.qsb = qsb; a.qst = qst; a.qsh = qsh; a.osb = osb; a.ost = ost; a.osh = osh;
  a.T = q_len; a.Hq = n_q_heads; a.rep = n_q_heads / h->cfg.n_kv_heads; a.dtype = dtype;
  a.scale = softmax_scale > 0.0f ? softmax_scale : (float)(1.0 / std::sqrt((double)h->cfg.head_dim));
  a.partial = at<float>(h, h->lay.partial);
  a.arrived = at<int32_t>(h, h->lay.arrived);
  PYR_PAGES(pyr::launch_pages_attn(a, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_fork(pyr_pages_t* h, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  const pyr_status_t st = check_call(h, n, true);
  if (st != PYR_OK) return st;
  if (n > 0 && (!src || !dst)) return PYR_ERR_NULL;
  PYR_PAGES_READY(h);
  if (n == 0) return PYR_OK;
  PYR_PAGES(pyr::launch_pages_fork(view(h), src, dst, n, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_trim(pyr_pages_t* h, const int32_t* lists, int32_t n, const int32_t* rows, void* stream) {
  const pyr_status_t st = check_call(h, n, false);
  if (st != PYR_OK) return st;
  if (!default_lists_fit(h, lists, n)) return PYR_ERR_INVALID;
  PYR_PAGES_READY(h);
  if (n == 0) return PYR_OK;
  PYR_PAGES(pyr::launch_pages_trim(view(h), lists, n, rows, &launches, static_cast<cudaStream_t>(stream)));
}

pyr_status_t pyr_pages_compact(pyr_pages_t* h, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* idx,
                               int32_t idx_groups, int64_t idx_stride, const int32_t* counts, int32_t n_rows, void* stream) {
  pyr_status_t st = check_call(h, n, true);
  if (st == PYR_OK) st = check_idx(h, idx, idx_groups, idx_stride, n_rows);
  if (st != PYR_OK) return st;
  if (n_rows < 0) return PYR_ERR_INVALID;
  if (n_rows > kMaxRows || !tiles_fit(h, n, n_rows)) return PYR_ERR_UNSUPPORTED;
  if (n > 0 && (!src || !dst)) return PYR_ERR_NULL;
  PYR_PAGES_READY(h);
  if (n == 0) return PYR_OK;
  pyr::PagesMoveArgs a;
  a.p = view(h);
  a.src = src; a.dst = dst; a.n = n; a.idx = idx; a.idx_groups = idx ? idx_groups : 1; a.idx_stride = idx_stride;
  a.counts = counts; a.n_rows = n_rows;
  a.refused = at<int32_t>(h, h->lay.refused);
  a.moved = at<int32_t>(h, h->lay.moved);
  PYR_PAGES(pyr::launch_pages_compact(a, &launches, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"

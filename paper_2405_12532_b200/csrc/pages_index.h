// Addresses inside the paged cache, in 4 and in 8 bits: where a row, a code and a scale lie, and the checks that keep every access in
// bounds whatever the tables hold. Plain C++ (host and device), so that the arithmetic can be tested without a GPU.
#pragma once
#include <stddef.h>
#include <stdint.h>

#ifdef __CUDACC__
#define PYR_HD __host__ __device__ __forceinline__
#else
#define PYR_HD inline
#endif

namespace pyr {

constexpr int kPageTile = 16;            // rows of a tile
constexpr int kMaxPageRows = 1024;
constexpr int kMaxLists = 1 << 19;

struct PagesView {
  uint8_t* pool;       // [n_pages][Hkv][head_extra + tiles_per_page * tile_bytes]
  int32_t* table;      // [n_lists][max_pages]
  int32_t* lens;       // [n_lists]
  int32_t* refs;       // [n_pages]
  int* status;
  int Hkv, D, group, page_rows, tiles_per_page, tile_bytes;      // group 0: 8 bits
  int head_extra;      // bytes of a (page, head) before its tiles: 0 in 4 bits
  int n_pages, n_lists, max_pages;
};

PYR_HD int pages_tile_bytes(int D, int group) { return kPageTile * (D + 8 * (D / group)); }
PYR_HD int pages_head_bytes(const PagesView& p) { return p.tiles_per_page * p.tile_bytes + p.head_extra; }
PYR_HD size_t pages_page_bytes(const PagesView& p) { return (size_t)p.Hkv * pages_head_bytes(p); }

// The list of entry i, or -1 if its id is out of range.
PYR_HD int pages_list(const PagesView& p, const int32_t* lists, int i) {
  const int l = lists ? lists[i] : i;
  return l >= 0 && l < p.n_lists ? l : -1;
}
// The page in slot `slot` of list l (a valid id), or -1 if the slot or the page id is out of range.
PYR_HD int pages_page(const PagesView& p, int l, int64_t slot) {
  if (slot < 0 || slot >= p.max_pages) return -1;
  const int page = p.table[(size_t)l * p.max_pages + slot];
  return page >= 0 && page < p.n_pages ? page : -1;
}
// A list's length, 0 if the stored one is negative and the rows its table can hold if it is larger.
PYR_HD int pages_len(const PagesView& p, int l) {
  const int64_t most = (int64_t)p.max_pages * p.page_rows;
  const int len = p.lens[l];
  return len < 0 ? 0 : (len > most ? (int)most : len);
}
// Pages that hold `rows` rows of a list (at most those of a table: the sum stays within 32 bits, whose division takes a tenth of 64's).
PYR_HD int pages_for(const PagesView& p, int rows) { return (int)(((uint32_t)rows + (uint32_t)p.page_rows - 1u) / (uint32_t)p.page_rows); }
// Byte offset in the pool of tile `tile` (of the page) of head h.
PYR_HD size_t pages_tile(const PagesView& p, int page, int h, int tile) {
  return ((size_t)page * p.Hkv + h) * (size_t)pages_head_bytes(p) + p.head_extra + (size_t)tile * p.tile_bytes;
}

// Offsets inside a tile: codes of a row, (scale, zero) words.
PYR_HD int tile_k_row(int D, int r) { return r * (D / 2); }
PYR_HD int tile_v_row(int D, int r) { return kPageTile * (D / 2) + r * (D / 2); }
PYR_HD int tile_k_word(int D, int G, int r, int g) { return kPageTile * D + (r * G + g) * 4; }
PYR_HD int tile_v_word(int D, int G, int r, int g) { return kPageTile * D + kPageTile * G * 4 + (r * G + g) * 4; }

// Stored position of the 32-bit word of K codes that holds dimensions 8 w .. 8 w + 7, of the 16-bit half of V codes that
// holds dimensions 4 h .. 4 h + 3, and the inverse maps.
PYR_HD int k_word_slot(int D, int group, int w) {
  const int u = group / 32, g = w / (group / 8), in = w % (group / 8);
  return in / u * (D / 32) + g * u + in % u;
}
PYR_HD int v_half_slot(int D, int group, int h) {
  const int u = group / 32, g = h / (group / 4), in = h % (group / 4);
  return in / u * (D / 32) + g * u + in % u;
}
PYR_HD int k_slot_word(int D, int group, int slot) {
  const int u = group / 32, j = slot / (D / 32), r = slot % (D / 32);
  return r / u * (group / 8) + j * u + r % u;
}
PYR_HD int v_slot_half(int D, int group, int slot) {
  const int u = group / 32, i = slot / (D / 32), r = slot % (D / 32);
  return r / u * (group / 4) + i * u + r % u;
}

// The 8-bit format. A (page, head) begins with the least and the largest code of each dimension (D signed bytes each) and the
// two scales (K's, V's); its tiles hold the codes as bytes code + 128, K's and then V's, and the scales once more, so that a copy
// of a tile is all that attention needs of it.
constexpr int kPageRows8 = 128;          // rows of a page at most: a CTA stores them with two warps a tile
PYR_HD int pages8_tile_bytes(int D) { return 2 * kPageTile * D + 16; }
PYR_HD int pages8_head_extra(int D) { return 2 * D + 16; }
PYR_HD int tile8_scales(int D) { return 2 * kPageTile * D; }
// Byte of a K code. A lane reads 16 dimensions of a row; rows of 128 bytes have their halves swapped in odd rows, which
// spreads eight such reads over all banks.
PYR_HD int tile8_k(int D, int r, int d) { return r * D + 16 * ((d >> 4) ^ (D == 128 ? 4 * (r & 1) : 0)) + (d & 15); }
// Byte of a V code. A word is four rows of one dimension: those of a lane's two operand registers. Lane j's words lie
// together, an eighth of the dimensions in a row (16-byte chunks in an order that differs between the lanes, for the banks).
PYR_HD int tile8_v(int D, int r, int d) {
  const int j = (r & 7) >> 1, b = 2 * (r & 1) + (r >> 3), e = D / 8, w = d % e;
  return kPageTile * D + 4 * D * j + 4 * e * (d / e) + 16 * ((w >> 2) ^ (j & (e / 4 - 1))) + 4 * (w & 3) + b;
}

// Shared memory in which the selection keeps a list's scores and a KV head's queries, and what it may take.
constexpr int kSelect8Shared = 200 * 1024;
inline int64_t pages_select8_shared(int64_t max_pages, int D, int64_t rep) { return (max_pages + 3) / 4 * 16 + (rep + 7) / 8 * 8 * (2 * D + 4); }

// How the attention's work is dealt out. A unit is one tile of one (entry, KV head, column group); an entry without rows
// still has one tile per head, so that its zeros get written. Before its tiles each (entry, KV head, column group) has
// kAttnSegmentUnits units that stand for no tile, for what beginning and ending it costs. Units are numbered entry by entry,
// head by head, column group by column group, tile by tile. Where there are no more (entry, KV head, column group)s than CTAs
// and none is long, a CTA takes one of them and its warps share the tiles; else every warp takes the same number of consecutive units.
constexpr int kAttnSegmentUnits = 6;
PYR_HD int64_t attn_tiles(int len) { return len > 0 ? (len + kPageTile - 1) / kPageTile : 1; }
// The units of each of `workers` warps (at least `least`), -1 where they are more than a warp counts in 32 bits.
PYR_HD int64_t attn_share(int64_t total, int64_t workers, int64_t least) {
  // (64-bit divisions take a tenth of a microsecond each)
  const int64_t q = total >> 31 ? (total + workers - 1) / workers : (int64_t)(((uint32_t)total + (uint32_t)workers - 1u) / (uint32_t)workers);
  return q > (1 << 30) ? -1 : (q < least ? least : q);
}
// CTAs of a launch: as many as the machine holds at once, `most`, but no more than have `least` units each if every list were as
// long as its table.
inline int attn_ctas(const PagesView& p, int64_t n, int64_t column_groups, int64_t least, int64_t most) {
  const int64_t tiles = attn_tiles(p.max_pages * p.page_rows) + kAttnSegmentUnits;
  const unsigned __int128 units = (unsigned __int128)n * (uint64_t)p.Hkv * (uint64_t)column_groups * (uint64_t)tiles;
  const unsigned __int128 ctas = (units + (uint64_t)least - 1) / (uint64_t)least;
  return ctas < (uint64_t)most ? (int)ctas : (int)most;
}

}  // namespace pyr

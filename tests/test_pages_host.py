"""The paged 4-bit cache without a GPU: argument checks of the C ABI, byte accounting, and the address arithmetic that the
kernels share (csrc/pages_index.h, compiled for the host): stored order, offsets, and what bad tables turn into."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from oracle import pages as op
from paper_2405_12532_b200 import binding as pb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000          # never dereferenced on the host


def _cfg(**over):
    kw = dict(n_kv_heads=4, head_dim=128, n_pages=10, n_lists=5, max_pages=3, group=64, page_rows=32)
    kw.update(over)
    return pb.make_pages_config(**kw)


def _handle(ready=True, **over):
    cfg = _cfg(**over)
    nbytes, align = pb.pyr_pages_bytes(cfg)
    h = C.c_void_p()
    assert pb.lib().pyr_pages_alloc(C.byref(cfg), C.c_void_p(FAKE), nbytes, C.byref(h)) == pb.PYR_OK
    return h


@pytest.mark.parametrize("over,want", [
    (dict(head_dim=96), pb.PYR_ERR_UNSUPPORTED), (dict(group=16), pb.PYR_ERR_UNSUPPORTED),
    (dict(head_dim=64, group=128), pb.PYR_ERR_INVALID), (dict(page_rows=24), pb.PYR_ERR_UNSUPPORTED),
    (dict(page_rows=0), pb.PYR_ERR_INVALID), (dict(page_rows=2048), pb.PYR_ERR_UNSUPPORTED),
    (dict(n_pages=0), pb.PYR_ERR_INVALID), (dict(n_lists=0), pb.PYR_ERR_INVALID), (dict(max_pages=0), pb.PYR_ERR_INVALID),
    (dict(n_lists=(1 << 19) + 1), pb.PYR_ERR_UNSUPPORTED), (dict(flags=1), pb.PYR_ERR_INVALID),
    (dict(max_pages=1 << 26), pb.PYR_ERR_UNSUPPORTED), (dict(n_kv_heads=0), pb.PYR_ERR_INVALID),
    (dict(n_kv_heads=70000), pb.PYR_ERR_UNSUPPORTED),
])
def test_pages_config_is_checked(over, want):
    b = C.c_size_t(0)
    assert pb.lib().pyr_pages_bytes(C.byref(_cfg(**over)), C.byref(b), None) == want
    h = C.c_void_p()
    assert pb.lib().pyr_pages_alloc(C.byref(_cfg(**over)), C.c_void_p(FAKE), 1 << 40, C.byref(h)) == want


def test_pages_bytes_alloc_and_view():
    L = pb.lib()
    cfg = _cfg()
    nbytes, align = pb.pyr_pages_bytes(cfg)
    assert align == 256
    page = 4 * 2 * op.tile_bytes(128, 64)
    assert 10 * page <= nbytes <= 10 * page + (12 << 20)
    h = C.c_void_p()
    b = C.c_size_t(0)
    assert L.pyr_pages_bytes(None, C.byref(b), None) == pb.PYR_ERR_NULL
    assert L.pyr_pages_bytes(C.byref(cfg), None, None) == pb.PYR_ERR_NULL
    assert L.pyr_pages_alloc(C.byref(cfg), None, nbytes, C.byref(h)) == pb.PYR_ERR_NULL
    assert L.pyr_pages_alloc(C.byref(cfg), C.c_void_p(FAKE), nbytes - 1, C.byref(h)) == pb.PYR_ERR_BUFFER_TOO_SMALL
    assert L.pyr_pages_alloc(C.byref(cfg), C.c_void_p(FAKE + 16), nbytes, C.byref(h)) == pb.PYR_ERR_INVALID
    assert L.pyr_pages_alloc(C.byref(cfg), C.c_void_p(FAKE), nbytes, C.byref(h)) == pb.PYR_OK
    ptrs = [C.c_void_p() for _ in range(4)]
    size = C.c_size_t(0)
    assert L.pyr_pages_view(h, C.byref(ptrs[0]), C.byref(size), *[C.byref(p) for p in ptrs[1:]]) == pb.PYR_OK
    assert size.value == page
    spans = sorted([(ptrs[0].value, 10 * page), (ptrs[1].value, 5 * 3 * 4), (ptrs[2].value, 5 * 4), (ptrs[3].value, 10 * 4)])
    assert all(p % 256 == 0 for p, _ in spans)
    assert all(p + n <= q for (p, n), (q, _) in zip(spans, spans[1:]))
    assert spans[0][0] >= FAKE and spans[-1][0] + spans[-1][1] <= FAKE + nbytes
    assert L.pyr_pages_view(None, None, None, None, None, None) == pb.PYR_ERR_NULL
    assert L.pyr_pages_free(h) == pb.PYR_OK and L.pyr_pages_free(None) == pb.PYR_ERR_NULL


@pytest.mark.parametrize("over", [dict(n_pages=0x7fffffff - 4096, n_kv_heads=65535, page_rows=1024, group=32, max_pages=1),
                                  dict(n_pages=0x7fffffff - 4096, n_kv_heads=52429, page_rows=1024, group=32, max_pages=1),
                                  dict(n_pages=1 << 30, n_kv_heads=512, page_rows=1024, max_pages=1)])
def test_pools_whose_size_would_not_fit_are_refused(over):
    """(2^64 and more bytes would come out as a small number, and a small buffer would pass for such a pool.)"""
    b, h = C.c_size_t(0), C.c_void_p()
    assert pb.lib().pyr_pages_bytes(C.byref(_cfg(**over)), C.byref(b), None) == pb.PYR_ERR_UNSUPPORTED
    assert pb.lib().pyr_pages_alloc(C.byref(_cfg(**over)), C.c_void_p(FAKE), (1 << 64) - 1, C.byref(h)) == pb.PYR_ERR_UNSUPPORTED
    nbytes, _ = pb.pyr_pages_bytes(_cfg(n_pages=1 << 30, n_kv_heads=64, page_rows=32, max_pages=1))
    assert nbytes > (1 << 30) * 64 * 2 * op.tile_bytes(128, 64)


def test_pages_calls_need_a_reset_first():
    """Every launching call before pyr_pages_reset is out of order; nothing is launched."""
    L, h, P = pb.lib(), _handle(), C.c_void_p(FAKE)
    word = C.c_int32(0)
    before = pb.launch_count()
    assert L.pyr_pages_reserve(h, None, 1, None, 1, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_write(h, None, 1, None, P, P, 512, 512, 128, 1, pb.PYR_BF16, None, 1, 0, None, 1, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_read(h, None, 1, None, P, P, 512, 512, 128, pb.PYR_BF16, None, 1, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_attn(h, None, 1, P, 512, 512, 128, P, 512, 512, 128, None, 1, 4, pb.PYR_BF16, 0.0, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_fork(h, P, P, 1, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_trim(h, None, 1, None, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_compact(h, P, P, 1, None, 1, 0, None, 1, None) == pb.PYR_ERR_ORDER
    assert L.pyr_pages_status(h, None, C.byref(word)) == pb.PYR_ERR_ORDER
    for call in (lambda: L.pyr_pages_reserve(None, None, 1, None, 1, None), lambda: L.pyr_pages_reset(None, None),
                 lambda: L.pyr_pages_trim(None, None, 1, None, None)):
        assert call() == pb.PYR_ERR_NULL
    assert pb.launch_count() == before
    L.pyr_pages_free(h)


def test_pages_arguments_are_refused_before_any_launch():
    """What the arguments alone decide: null pointers, types, counts, strides that overlap or break the 16-byte rows, head counts,
    scales. (A valid call on the same handle is only out of order: it has not been reset.)"""
    L, h, P, N = pb.lib(), _handle(), C.c_void_p(FAKE), None
    before = pb.launch_count()
    INV, NUL, UNS, ORD = pb.PYR_ERR_INVALID, pb.PYR_ERR_NULL, pb.PYR_ERR_UNSUPPORTED, pb.PYR_ERR_ORDER

    def write(n=2, k=P, v=P, sb=5120, sn=512, sh=128, src=10, dtype=pb.PYR_BF16, idx=N, groups=1, istride=0, rows=10):
        return L.pyr_pages_write(h, N, n, N, k, v, sb, sn, sh, src, dtype, idx, groups, istride, N, rows, N)

    assert write() == ORD and write(idx=P, groups=4, istride=40, rows=99) == ORD and write(n=1, sb=7) == ORD
    assert write(k=N) == NUL and write(v=N) == NUL and write(dtype=5) == UNS
    assert write(n=-1) == INV and write(n=6) == INV and write(rows=-1) == INV and write(src=-1) == INV and write(rows=11) == INV
    assert write(idx=P, groups=2) == INV and write(idx=P, istride=-1) == INV and write(sh=64) == INV and write(sn=-512) == INV
    assert write(sn=516) == INV and write(k=C.c_void_p(FAKE + 8)) == INV and write(idx=P, rows=(1 << 30) + 1) == UNS

    def read(n=2, k=P, v=P, sb=5120, sn=512, sh=128, dtype=pb.PYR_F32, rows=10):
        return L.pyr_pages_read(h, N, n, N, k, v, sb, sn, sh, dtype, N, rows, N)

    assert read() == ORD and read(k=N) == NUL and read(dtype=9) == UNS and read(rows=-1) == INV and read(n=6) == INV
    assert read(sn=64) == INV and read(sb=64) == INV and read(n=1, sb=64) == ORD and read(rows=1, sn=64) == ORD

    def attn(n=2, q=P, out=P, qb=1024, qt=1024, qh=128, ob=1024, ot=1024, oh=128, lse=N, t=1, hq=8, dtype=pb.PYR_BF16, scale=0.0):
        return L.pyr_pages_attn(h, N, n, q, qb, qt, qh, out, ob, ot, oh, lse, t, hq, dtype, scale, N)

    assert attn() == ORD and attn(lse=P, scale=0.5) == ORD and attn(n=6) == INV and attn(n=-1) == INV
    assert attn(q=N) == NUL and attn(out=N) == NUL and attn(dtype=3) == UNS and attn(hq=6) == INV and attn(hq=0) == INV and attn(t=0) == INV
    assert attn(scale=-1.0) == INV and attn(scale=float("inf")) == INV and attn(scale=float("nan")) == INV
    assert attn(oh=64) == INV and attn(ob=64) == INV and attn(t=2, ot=64) == INV and attn(qh=132) == INV and attn(t=1 << 20) == UNS

    assert L.pyr_pages_reserve(h, N, 2, N, -1, N) == INV and L.pyr_pages_reserve(h, N, 6, N, 1, N) == INV
    assert L.pyr_pages_reserve(h, N, 2, P, -1, N) == ORD
    assert L.pyr_pages_fork(h, N, P, 1, N) == NUL and L.pyr_pages_fork(h, P, N, 1, N) == NUL and L.pyr_pages_fork(h, P, P, 6, N) == INV
    assert L.pyr_pages_trim(h, N, 6, N, N) == INV and L.pyr_pages_trim(h, P, -2, N, N) == INV
    assert L.pyr_pages_compact(h, N, P, 1, N, 1, 0, N, 1, N) == NUL and L.pyr_pages_compact(h, P, P, 1, P, 3, 0, N, 1, N) == INV
    assert L.pyr_pages_compact(h, P, P, 1, N, 1, 0, N, -1, N) == INV and L.pyr_pages_compact(h, P, P, 6, N, 1, 0, N, 1, N) == INV
    assert pb.launch_count() == before
    L.pyr_pages_free(h)


def test_tensors_to_be_written_must_not_overlap_themselves():
    """(Two threads would write one place, in any order.) Dimensions in any order of strides, and dimensions of size 1, are fine."""
    L, h, P, N = pb.lib(), _handle(), C.c_void_p(FAKE), None
    INV, ORD = pb.PYR_ERR_INVALID, pb.PYR_ERR_ORDER

    def read(sb, sn, sh, n=2, rows=10):
        return L.pyr_pages_read(h, N, n, N, P, P, sb, sn, sh, pb.PYR_BF16, N, rows, N)

    def attn(sb, st, sh, n=2, t=3, hq=8):
        return L.pyr_pages_attn(h, N, n, P, 0, 0, 128, P, sb, st, sh, N, t, hq, pb.PYR_BF16, 0.0, N)

    # 4 heads of 128: rows then heads, heads then rows, entries innermost, padded
    assert read(5120, 512, 128) == ORD and read(5120, 128, 1280) == ORD and read(128, 1024, 256) == ORD and read(9000, 640, 136) == ORD
    assert read(5120, 128, 128) == INV and read(512, 512, 128) == INV and read(5112, 512, 128) == INV and read(5120, 504, 128) == INV
    assert read(5120, 128, 1272) == INV and read(0, 512, 128) == INV and read(0, 512, 128, n=1) == ORD and read(512, 0, 128, rows=1) == ORD
    # 8 heads of 128, 3 tokens
    assert attn(3 * 1024, 1024, 128) == ORD and attn(3 * 1024, 128, 384) == ORD and attn(1024, 2048, 128) == ORD
    assert attn(1024, 1024, 128) == INV and attn(3 * 1024, 128, 128) == INV and attn(2 * 1024, 1024, 128) == INV
    assert attn(1024, 0, 128, t=1) == ORD and attn(0, 1024, 128, n=1) == ORD
    L.pyr_pages_free(h)


def test_calls_with_more_tiles_than_a_launch_has_warps_are_refused_whole():
    """(Refused by the second launch of a call, the first one's work would stay behind and spoil the next call.)"""
    L, h, P, N = pb.lib(), _handle(n_kv_heads=64), C.c_void_p(FAKE), None
    for rows, want in [(1 << 28, pb.PYR_ERR_ORDER), (1 << 30, pb.PYR_ERR_UNSUPPORTED)]:
        assert L.pyr_pages_write(h, N, 1, N, P, P, 0, 8192, 128, 10, pb.PYR_BF16, P, 1, 0, N, rows, N) == want
        assert L.pyr_pages_read(h, N, 1, N, P, P, 0, 8192, 128, pb.PYR_BF16, N, rows, N) == want
        assert L.pyr_pages_compact(h, P, C.c_void_p(FAKE + 64), 1, P, 1, 0, N, rows, N) == want
    L.pyr_pages_free(h)


def test_tensors_without_elements_need_no_address():
    """(An empty torch tensor's address is null.) The calls get past the checks of their arguments."""
    L, h, N, ORD = pb.lib(), _handle(), None, pb.PYR_ERR_ORDER
    bf = pb.PYR_BF16
    assert L.pyr_pages_write(h, N, 0, N, N, N, 0, 512, 128, 10, bf, N, 1, 0, N, 10, N) == ORD
    assert L.pyr_pages_write(h, N, 2, N, N, N, 0, 512, 128, 0, bf, N, 1, 0, N, 0, N) == ORD
    assert L.pyr_pages_read(h, N, 0, N, N, N, 0, 512, 128, bf, N, 10, N) == ORD
    assert L.pyr_pages_read(h, N, 2, N, N, N, 512, 512, 128, bf, N, 0, N) == ORD
    assert L.pyr_pages_attn(h, N, 0, N, 0, 0, 128, N, 0, 0, 128, N, 1, 8, bf, 0.0, N) == ORD
    assert L.pyr_pages_attn(h, N, 1, N, 0, 0, 128, N, 0, 0, 128, N, 1, 8, bf, 0.0, N) == pb.PYR_ERR_NULL
    L.pyr_pages_free(h)


HARNESS = r"""
#include "pages_index.h"
using namespace pyr;
extern "C" {
int k_slot(int D, int g, int w) { return k_word_slot(D, g, w); }
int k_back(int D, int g, int s) { return k_slot_word(D, g, s); }
int v_slot(int D, int g, int h) { return v_half_slot(D, g, h); }
int v_back(int D, int g, int s) { return v_slot_half(D, g, s); }
int k_word(int D, int G, int r, int g) { return tile_k_word(D, G, r, g); }
int v_word(int D, int G, int r, int g) { return tile_v_word(D, G, r, g); }
int k_row(int D, int r) { return tile_k_row(D, r); }
int v_row(int D, int r) { return tile_v_row(D, r); }
static PagesView make(int32_t* table, int32_t* lens, int n_pages, int n_lists, int max_pages, int page_rows) {
  PagesView p{};
  p.table = table; p.lens = lens; p.Hkv = 3; p.D = 128; p.group = 64; p.page_rows = page_rows;
  p.tiles_per_page = page_rows / kPageTile; p.tile_bytes = pages_tile_bytes(128, 64);
  p.n_pages = n_pages; p.n_lists = n_lists; p.max_pages = max_pages;
  return p;
}
int page(int32_t* table, int n_pages, int n_lists, int max_pages, int l, long long slot) {
  return pages_page(make(table, nullptr, n_pages, n_lists, max_pages, 32), l, slot);
}
int list(int32_t* lists, int n_lists, int i) { return pages_list(make(nullptr, nullptr, 1, n_lists, 1, 32), lists, i); }
int len(int32_t* lens, int max_pages, int page_rows, int l) { return pages_len(make(nullptr, lens, 1, 4, max_pages, page_rows), l); }
unsigned long long tile_at(int n_pages, int page_rows, int page, int h, int t) {
  return pages_tile(make(nullptr, nullptr, n_pages, 1, 1, page_rows), page, h, t);
}
}
"""


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("pages_index")
    src, so = d / "index.cpp", d / "index.so"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2405_12532_b200", "csrc"), str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.tile_at.restype = C.c_ulonglong
    lib.page.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_longlong]
    return lib


@pytest.mark.parametrize("D,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_stored_order_is_the_documented_one(index, D, group):
    """Every code, word and row has a place of its own, the maps invert each other, and they are those of the definition."""
    G = D // group
    ks = [index.k_slot(D, group, w) for w in range(D // 8)]
    vs = [index.v_slot(D, group, h) for h in range(D // 4)]
    assert sorted(ks) == list(range(D // 8)) and sorted(vs) == list(range(D // 4))
    assert [index.k_back(D, group, s) for s in ks] == list(range(D // 8))
    assert [index.v_back(D, group, s) for s in vs] == list(range(D // 4))
    assert all(8 * ks[d // 8] + d % 8 == op._word_of_k(D, group, d) for d in range(D))
    assert all(4 * vs[d // 4] + d % 4 == op._half_of_v(D, group, d) for d in range(D))
    used = []
    for r in range(16):
        used += [(index.k_row(D, r), D // 2), (index.v_row(D, r), D // 2)]
        for g in range(G):
            used += [(index.k_word(D, G, r, g), 4), (index.v_word(D, G, r, g), 4)]
    used.sort()
    assert all(a + n == b for (a, n), (b, _) in zip(used, used[1:]))
    assert used[0][0] == 0 and sum(used[-1]) == op.tile_bytes(D, group)


def test_bad_tables_lists_and_lengths_stay_in_bounds(index):
    """What device memory may hold - list ids, page ids, slots and lengths out of range - becomes "none" or is clamped."""
    table = np.array([[0, 9, -1], [10, 1 << 30, -(1 << 31)]], np.int32)
    at = lambda l, s: index.page(table.ctypes.data, 10, 2, 3, l, s)
    assert [at(0, s) for s in range(3)] == [0, 9, -1] and [at(1, s) for s in range(3)] == [-1, -1, -1]
    assert at(0, -1) == -1 and at(0, 3) == -1 and at(1, 1 << 40) == -1
    lists = np.array([0, 1, 2, -1, -(1 << 31), (1 << 31) - 1], np.int32)
    lp = lists.ctypes.data_as(C.c_void_p)
    assert [index.list(lp, 2, i) for i in range(6)] == [0, 1, -1, -1, -1, -1]
    assert index.list(None, 2, 1) == 1 and index.list(None, 2, 2) == -1
    lens = np.array([5, -7, 97, (1 << 31) - 1], np.int32)
    assert [index.len(lens.ctypes.data_as(C.c_void_p), 3, 32, i) for i in range(4)] == [5, 0, 96, 96]


def test_offsets_pass_32_bits(index):
    """The last tile of a pool of 600 000 pages lies beyond 2^32 bytes, where it should."""
    tb = op.tile_bytes(128, 64)
    assert index.tile_at(600000, 64, 599999, 2, 3) == ((599999 * 3 + 2) * 4 + 3) * tb > 1 << 32


@pytest.mark.parametrize("D,group", [(64, 32), (128, 64), (128, 128)])
def test_quantisation_bound_of_the_definition(D, group):
    """The oracle's quantisation: codes in 0 .. 15 without a clamp, values within half a step (and the roundings of
    (x - zero) * inv, at most 15 steps times 3 * 2^-24), zero below and scale times 15 above the group."""
    rng = np.random.default_rng(D + group)
    x = np.concatenate([rng.standard_normal((40, D)), 100 + 0.01 * rng.standard_normal((10, D)), rng.standard_normal((5, D)) * 1e30,
                        rng.standard_normal((5, D)) * 1e-25, np.full((2, D), -3.7), np.zeros((1, D))]).astype(np.float32)
    c, s, z = op.quantise(x, group)
    assert c.min() >= 0 and c.max() <= 15
    v = op.values(c, s, z)
    step = np.repeat(s, group, -1).astype(np.float64)
    assert np.all(np.abs(v - x) <= step * (0.5 + 15 * 3 * 2.0 ** -24))
    y = x.reshape(x.shape[0], -1, group).astype(np.float64)
    assert np.all(z <= y.min(-1)) and np.all(z + 15.0 * s.astype(np.float64) >= y.max(-1) * (1 - 2.0 ** -22) - 1e-30)
    bad = x.copy()
    bad[0, 3], bad[1, group - 1], bad[2, 0], bad[3, 0] = np.inf, np.nan, -np.inf, -3.4e38
    _, s, z = op.quantise(bad, group)
    assert np.isnan(s[:4, 0]).all() and np.isnan(z[:4, 0]).all() and np.isfinite(s[4:]).all()

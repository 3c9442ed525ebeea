"""The paged 8-bit cache without a GPU: argument checks of its calls, byte accounting, and the address arithmetic that the kernels
share (csrc/pages_index.h, compiled for the host)."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

from oracle import pages8 as o8
from paper_2405_12532_b200 import binding as pb

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x7F0000000000          # never dereferenced on the host
P, N = C.c_void_p(FAKE), None
INV, NUL, UNS, ORD = pb.PYR_ERR_INVALID, pb.PYR_ERR_NULL, pb.PYR_ERR_UNSUPPORTED, pb.PYR_ERR_ORDER


def _cfg(**over):
    kw = dict(n_kv_heads=4, head_dim=128, n_pages=10, n_lists=5, max_pages=3, page_rows=32, bits=8)
    kw.update(over)
    return pb.make_pages_config(**kw)


def _handle(**over):
    cfg = _cfg(**over)
    nbytes, _ = pb.pyr_pages_bytes(cfg)
    h = C.c_void_p()
    assert pb.lib().pyr_pages_alloc(C.byref(cfg), P, nbytes, C.byref(h)) == pb.PYR_OK
    return h


@pytest.mark.parametrize("over,want", [
    (dict(group=64), INV), (dict(page_rows=144), UNS), (dict(page_rows=24), UNS), (dict(head_dim=96), UNS), (dict(flags=1), INV),
    (dict(page_rows=0), INV), (dict(n_pages=0), INV), (dict(n_kv_heads=70000), UNS),
    (dict(n_pages=0x7fffffff - 4096, n_kv_heads=65535, page_rows=128, max_pages=1), UNS)])
def test_config_is_checked(over, want):
    b, h = C.c_size_t(0), C.c_void_p()
    assert pb.lib().pyr_pages_bytes(C.byref(_cfg(**over)), C.byref(b), None) == want
    assert pb.lib().pyr_pages_alloc(C.byref(_cfg(**over)), P, 1 << 62, C.byref(h)) == want


@pytest.mark.parametrize("D", [64, 128])
def test_bytes_and_view(D):
    L, h = pb.lib(), _handle(head_dim=D)
    size, pool = C.c_size_t(0), C.c_void_p()
    assert L.pyr_pages_view(h, C.byref(pool), C.byref(size), N, N, N) == pb.PYR_OK
    assert size.value == 4 * o8.head_bytes(D, 32)
    nbytes, _ = pb.pyr_pages_bytes(_cfg(head_dim=D))
    assert pool.value % 256 == 0 and pool.value + 10 * size.value <= FAKE + nbytes
    L.pyr_pages_free(h)
    with pytest.raises(ValueError):
        _cfg(bits=5)


class Append(C.Structure):
    _fields_ = ([(x, C.c_void_p) for x in ("lists", "first", "k", "v")] + [(x, C.c_int64) for x in ("stride_b", "stride_n", "stride_h")] +
                [("idx", C.c_void_p), ("idx_stride", C.c_int64), ("counts", C.c_void_p), ("pos", C.c_void_p), ("pos_stride", C.c_int64),
                 ("rope", C.c_void_p), ("q", C.c_void_p), ("q_out", C.c_void_p)] +
                [(x, C.c_int64) for x in ("q_stride_b", "q_stride_n", "q_stride_h", "o_stride_b", "o_stride_n", "o_stride_h")] +
                [(x, C.c_int32) for x in ("n", "src_rows", "dtype", "idx_groups", "n_rows", "n_pos", "n_q_heads")])


def _append(h, n=2, k=P, v=P, sb=5120, sn=512, sh=128, src=10, dtype=pb.PYR_BF16, pos=N, pstride=10, rope=P, n_pos=100, q=N, qo=N, qb=10240,
            qn=1024, qh=128, ob=10240, on=1024, oh=128, hq=8, idx=N, groups=1, istride=0, rows=10):
    x = Append(N, N, k, v, sb, sn, sh, idx, istride, N, pos, pstride, rope, q, qo, qb, qn, qh, ob, on, oh, n, src, dtype, groups, rows, n_pos, hq)
    return pb.lib().pyr_pages_append(h, C.byref(x), N)


def test_the_binding_packs_the_structure_of_the_header():
    """Field by field: what the binding's packed bytes say, read through the structure."""
    assert C.sizeof(Append) == (pb._APPEND.size + 7) // 8 * 8
    values = list(range(1, len(Append._fields_) + 1))
    x = Append.from_buffer_copy(pb._APPEND.pack(*values) + bytes(C.sizeof(Append) - pb._APPEND.size))
    assert [getattr(x, f) for f, _ in Append._fields_] == values
    with open(os.path.join(ROOT, "include", "pyr.h")) as f:
        text = f.read()
    body = text[text.index("const int32_t* lists;   /*"):text.index("} pyr_append_t;")]
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = re.findall(r"(\w+)\s*[;,]", body)
    assert names == [f for f, _ in Append._fields_]


def test_append_arguments():
    """(A valid call is only out of order: the handle has not been reset.)"""
    h, h4, before = _handle(), _handle(bits=4), pb.launch_count()
    Q = C.c_void_p(FAKE + (1 << 20))
    assert _append(h) == ORD and _append(h, pos=P) == ORD and _append(h, pos=P, q=P, qo=Q) == ORD and _append(h, pos=P, q=P, qo=P) == ORD
    assert _append(h, idx=P, groups=4, istride=40, rows=99) == ORD and _append(h, idx=P, pos=P) == ORD and _append(h, n=0, k=N, v=N) == ORD
    assert pb.lib().pyr_pages_append(h, N, N) == NUL
    assert _append(None) == NUL and _append(h, k=N) == NUL and _append(h, pos=P, rope=N) == NUL
    assert _append(h, pos=P, q=P) == NUL and _append(h, pos=P, qo=P) == NUL
    assert _append(h, dtype=4) == UNS and _append(h4) == UNS and _append(h, idx=P, rows=(1 << 30) + 1) == UNS
    assert _append(h, pos=P, q=P, qo=Q, hq=65536, qb=1 << 30, qn=1 << 24, ob=1 << 30, on=1 << 24) == UNS
    assert _append(h, n=6) == INV and _append(h, n=-1) == INV and _append(h, rows=11) == INV and _append(h, rows=-1) == INV
    assert _append(h, pos=P, n_pos=0) == INV and _append(h, pos=P, pstride=-1) == INV and _append(h, pos=P, rope=C.c_void_p(FAKE + 4)) == INV
    assert _append(h, q=P, qo=Q) == INV and _append(h, pos=P, q=P, qo=Q, idx=P) == INV and _append(h, pos=P, q=P, qo=Q, hq=0) == INV
    assert _append(h, pos=P, q=P, qo=P, on=2048, ob=20480) == INV              # in place needs the same strides
    assert _append(h, pos=P, q=P, qo=Q, on=512) == INV and _append(h, pos=P, q=P, qo=Q, qn=1028) == INV
    assert _append(h, idx=P, groups=2) == INV and _append(h, sh=64) == INV and _append(h, sn=516) == INV
    assert pb.launch_count() == before
    for x in (h, h4):
        pb.lib().pyr_pages_free(x)


def test_select_and_attn_blocks_arguments():
    L, h, h4, before = pb.lib(), _handle(), _handle(bits=4), pb.launch_count()

    def select(h=h, n=2, q=P, qb=1024, qt=1024, qh=128, t=1, hq=8, dtype=pb.PYR_BF16, slots=P, ns=2, first=1, last=1):
        return L.pyr_pages_select(h, N, n, q, qb, qt, qh, t, hq, dtype, slots, ns, first, last, N)

    assert select() == ORD and select(dtype=pb.PYR_F32) == ORD and select(n=0, q=N, slots=N) == ORD
    assert select(h=None) == NUL and select(q=N) == NUL and select(slots=N) == NUL and select(h=h4) == UNS and select(dtype=2) == UNS
    assert select(ns=0, first=0, last=0) == INV and select(first=-1) == INV and select(last=2) == INV and select(last=0x7fffffff) == INV
    assert select(t=0) == INV and select(hq=6) == INV and select(n=6) == INV and select(qh=132) == INV
    assert select(n=1, t=1 << 28) == UNS
    big = _handle(max_pages=50500)                                             # 4 * max_pages + 260 bytes a head, in eights, of 204 800
    assert select(h=big, hq=4) == ORD and select(h=big, hq=32, qb=4096) == ORD and select(h=big, hq=36, qb=8192) == UNS
    wide = _handle(max_pages=51200)
    assert select(h=wide, hq=4) == UNS

    def blocks(h=h, n=2, slots=P, ns=3, q=P, out=P, qb=1024, qt=1024, qh=128, ob=1024, ot=1024, oh=128, t=1, hq=8, dtype=pb.PYR_BF16, scale=0.0):
        return L.pyr_pages_attn_blocks(h, N, n, slots, ns, q, qb, qt, qh, out, ob, ot, oh, N, t, hq, dtype, scale, N)

    assert blocks() == ORD and blocks(n=0, slots=N, q=N, out=N) == ORD and blocks(h=None) == NUL and blocks(slots=N) == NUL and blocks(q=N) == NUL
    assert blocks(ns=0) == INV and blocks(scale=-1.0) == INV and blocks(t=0) == INV and blocks(hq=7) == INV and blocks(oh=64) == INV
    assert blocks(h=h4) == UNS and blocks(t=1 << 20) == UNS
    # calls that the formats do not share
    assert L.pyr_pages_compact(h, P, P, 1, N, 1, 0, N, 1, N) == UNS
    assert L.pyr_pages_attn(h, N, 2, P, 1024, 1024, 128, P, 1024, 1024, 128, N, 1, 8, pb.PYR_BF16, 0.0, N) == ORD
    assert L.pyr_pages_write(h, N, 2, N, P, P, 5120, 512, 128, 10, pb.PYR_BF16, N, 1, 0, N, 10, N) == ORD
    assert pb.launch_count() == before
    for x in (h, h4, big, wide):
        L.pyr_pages_free(x)


def test_rope_table_arguments():
    L, before = pb.lib(), pb.launch_count()
    t = lambda table=P, first=0, n=4, d=128, base=1e4: L.pyr_glue_rope_table(table, first, n, d, base, N)  # noqa: E731
    assert t(table=N) == NUL and t(first=-1) == INV and t(n=-1) == INV and t(d=7) == INV and t(d=0) == INV
    assert t(base=0.0) == INV and t(base=-1.0) == INV and t(base=float("nan")) == INV and t(base=float("inf")) == INV
    assert t(d=512) == UNS and t(first=1 << 31) == UNS and t(n=0, table=N) == pb.PYR_OK
    assert pb.launch_count() == before


HARNESS = r"""
#include "pages_index.h"
using namespace pyr;
extern "C" {
int k8(int D, int r, int d) { return tile8_k(D, r, d); }
int v8(int D, int r, int d) { return tile8_v(D, r, d); }
int scales8(int D) { return tile8_scales(D); }
int tile8(int D) { return pages8_tile_bytes(D); }
int extra8(int D) { return pages8_head_extra(D); }
unsigned long long tile_at(int D, int heads, int page_rows, int page, int h, int t) {
  PagesView p{};
  p.Hkv = heads; p.D = D; p.page_rows = page_rows; p.tiles_per_page = page_rows / kPageTile;
  p.tile_bytes = pages8_tile_bytes(D); p.head_extra = pages8_head_extra(D);
  return pages_tile(p, page, h, t);
}
long long shared8(long long pages, int D, long long rep) { return pages_select8_shared(pages, D, rep); }
}
"""


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("pages8_index")
    src, so = d / "index.cpp", d / "index.so"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2405_12532_b200", "csrc"), str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.tile_at.restype = C.c_ulonglong
    lib.shared8.restype = C.c_longlong
    lib.shared8.argtypes = [C.c_longlong, C.c_int, C.c_longlong]
    return lib


@pytest.mark.parametrize("D", [64, 128])
def test_codes_have_the_documented_places(index, D):
    k = [[index.k8(D, r, d) for d in range(D)] for r in range(16)]
    v = [[index.v8(D, r, d) for d in range(D)] for r in range(16)]
    assert k == [[o8.k_byte(D, r, d) for d in range(D)] for r in range(16)]
    assert v == [[o8.v_byte(D, r, d) for d in range(D)] for r in range(16)]
    assert sorted(np.ravel(k).tolist() + np.ravel(v).tolist()) == list(range(32 * D)) and index.scales8(D) == 32 * D
    assert index.tile8(D) == 32 * D + 16 and index.extra8(D) == 2 * D + 16
    # what the kernels store at once lies together: 4 (2) dimensions of a K row, words of 4 (2) dimensions of V
    w = D // 32
    for d in range(0, D, w):
        for r in range(16):
            assert [index.k8(D, r, d + i) - index.k8(D, r, d) for i in range(w)] == list(range(w)) and index.k8(D, r, d) % w == 0
        for j in range(4):
            at = index.v8(D, 2 * j, d)
            assert at % (4 * w) == 0
            assert [[index.v8(D, r, d + i) - at for r in (2 * j, 2 * j + 8, 2 * j + 1, 2 * j + 9)] for i in range(w)] == [
                [4 * i + b for b in range(4)] for i in range(w)]


def test_offsets_pass_32_bits(index):
    hb = o8.head_bytes(128, 128)
    assert index.tile_at(128, 40, 128, 600000, 39, 7) == (600000 * 40 + 39) * hb + 272 + 7 * 4112 > 1 << 32
    assert index.shared8(50500, 128, 1) == 204080 and index.shared8(5, 64, 9) == 32 + 16 * 132


def test_binding_refuses_tensors_it_cannot_pass_on():
    """(Tensors of the CPU: nothing gets as far as the library.)"""
    p = object.__new__(pb.PyrPages)
    p.cfg, p.device, p._index, p._heads, p._dim, p._args = _cfg(), torch.device("cpu"), -1, 4, 128, bytearray(pb._APPEND.size)
    p._call = None
    k = torch.zeros(2, 3, 4, 128, dtype=torch.bfloat16)
    pos, rope = torch.zeros(2, 1, 3, dtype=torch.int32), torch.zeros(5, 128)
    for bad in (dict(pos=pos[:, :, :2], rope=rope), dict(pos=pos, rope=rope.double()), dict(pos=pos, rope=rope[:, :64]), dict(pos=pos), dict(pos=pos.long(), rope=rope),
                dict(pos=pos, rope=rope.t().contiguous().t()), dict(pos=pos, rope=rope, q=k.float()), dict(pos=pos, rope=rope, q=k[:, :2]),
                dict(q_out=k), dict(pos=pos, rope=rope, q=k, q_out=k[:, :, :2])):
        with pytest.raises(ValueError):
            p.append(k, k, **bad)
    q = torch.zeros(2, 1, 8, 128, dtype=torch.bfloat16)
    slots = torch.zeros(2, 1, 4, 3, dtype=torch.int32)
    for bad in (slots.long(), slots[:, :, :2], slots[:1], slots.transpose(2, 3).contiguous().transpose(2, 3)):
        with pytest.raises(ValueError):
            p.attn_blocks(q, bad)
    with pytest.raises(ValueError):
        p.select(q, 4, out=slots)


def test_compiled_calls_leave_what_is_not_plainly_right_to_the_binding():
    """(Tensors of the CPU are none of theirs.) They load, and return None."""
    calls = pb._calls()
    if not calls:
        assert torch.version.cuda is None
        return
    before = pb.launch_count()
    c = calls.cache(FAKE, 0, 4, 128)
    k, q = torch.zeros(2, 3, 4, 128), torch.zeros(2, 1, 8, 128)
    ids, slots = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 1, 4, 3, dtype=torch.int32)
    assert calls.attn(c, q, ids, None, None, True, 0.0) is None and calls.attn(c, q, None, slots, None, False, 0.0) is None
    assert calls.attn(c, q, None, None, None, False, "x") is None and calls.attn(c, 5, None, None, None, False, 0.0) is None
    assert calls.select(c, q, 4, None, 0, 1, None) is None and calls.select(c, q, 0, None, 0, 0, None) is None and calls.select(c, q, 1 << 70, None, 0, 0, None) is None
    assert calls.append(c, k, k, ids, None, None, None, None, None, None, None) is None and calls.read(c, k, k, None, None, None) is None
    for bad in (lambda: calls.attn(c, q), lambda: calls.read(c), lambda: calls.setup(1), lambda: calls.cache(1)):
        with pytest.raises(TypeError):
            bad()
    with pytest.raises(ValueError):
        calls.read(5, k, k, None, None, None)
    assert pb.launch_count() == before

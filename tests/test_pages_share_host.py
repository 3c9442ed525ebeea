"""How the paged attention's work is counted out, on the CPU (csrc/pages_index.h, compiled for the host): shares that fit a warp's
32 bits, grids for tables of any size."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HARNESS = r"""
#include "pages_index.h"
using namespace pyr;
extern "C" {
long long share(long long total, long long workers, long long least) { return attn_share(total, workers, least); }
long long tiles(int len) { return attn_tiles(len); }
int ctas(int heads, int page_rows, int max_pages, long long n, long long groups, long long least, long long most) {
  PagesView p{};
  p.Hkv = heads; p.page_rows = page_rows; p.max_pages = max_pages;
  return attn_ctas(p, n, groups, least, most);
}
}
"""


@pytest.fixture(scope="module")
def index(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("pages_share")
    src, so = d / "share.cpp", d / "share.so"
    src.write_text(HARNESS)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover",
                    "-I", os.path.join(ROOT, "paper_2405_12532_b200", "csrc"), str(src), "-o", str(so)], check=True)
    lib = C.CDLL(str(so))
    lib.share.restype = lib.tiles.restype = C.c_longlong
    lib.share.argtypes = [C.c_longlong] * 3
    lib.ctas.argtypes = [C.c_int] * 3 + [C.c_longlong] * 4
    return lib


@pytest.mark.parametrize("workers", [1, 7, 1036, 1628, 7040])
def test_shares_cover_the_work_and_fit_32_bits(index, workers):
    for total in (1, 2, workers - 1, workers, workers + 1, (1 << 31) - 1, 1 << 31, (1 << 32) + 5, (1 << 30) * workers - 1,
                  (1 << 30) * workers):
        if total < 1:
            continue
        q = index.share(total, workers, 2)
        if total <= (1 << 30) * workers:
            assert q == max(2, -(-total // workers)) and q * workers >= total
        else:
            assert q == -1
    assert index.share(0, workers, 2) == 2
    for total in ((1 << 30) * workers + 1, 1 << 45, 1 << 57, (1 << 62) + 1):
        assert index.share(total, workers, 2) == (-1 if total > (1 << 30) * workers else -(-total // workers))


def test_grids_for_tables_of_any_size(index):
    """Large tables do not refuse a call, whatever its lists hold, and a product beyond 64 bits is still a large one."""
    assert index.tiles(0) == 1 and index.tiles(1) == 1 and index.tiles(17) == 2 and index.tiles((1 << 31) - 1025) == (1 << 27) - 64
    assert index.ctas(32, 64, 7, 1, 1, 22, 148) == -(-32 * (28 + 6) // 22)
    assert index.ctas(1, 16, 1, 1, 1, 22, 148) == 1
    assert index.ctas(8, 1024, 4096, 64, 2048, 22, 148) == 148                 # 2.8e11 units
    assert index.ctas(65535, 1024, 2097150, (1 << 31) - 1, 1 << 20, 22, 148) == 148        # 2^94

"""Softmax scales at the end of fp32's range, without a GPU: one that does not stay finite once the exponential's base is in it is
refused before any launch."""
import ctypes as C

import pytest

from paper_2405_12532_b200 import binding as pb

FAKE = 0x7F0000000000          # never dereferenced on the host


@pytest.mark.parametrize("scale,want", [(2.0 ** 127, pb.PYR_ERR_ORDER), (2.0 ** 127 * 1.0001, pb.PYR_ERR_INVALID),
                                        (3.4028234e38, pb.PYR_ERR_INVALID), (1e-45, pb.PYR_ERR_ORDER), (0.0, pb.PYR_ERR_ORDER)])
def test_softmax_scales_near_the_end_of_the_range(scale, want):
    """(A valid call is only out of order: the handle has not been reset.)"""
    cfg = pb.make_pages_config(n_kv_heads=4, head_dim=128, n_pages=10, n_lists=5, max_pages=3, group=64, page_rows=32)
    nbytes, _ = pb.pyr_pages_bytes(cfg)
    h, P, before = C.c_void_p(), C.c_void_p(FAKE), pb.launch_count()
    assert pb.lib().pyr_pages_alloc(C.byref(cfg), P, nbytes, C.byref(h)) == pb.PYR_OK
    got = pb.lib().pyr_pages_attn(h, None, 2, P, 1024, 1024, 128, P, 1024, 1024, 128, None, 1, 8, pb.PYR_BF16, scale, None)
    pb.lib().pyr_pages_free(h)
    assert got == want and pb.launch_count() == before

"""The compiled calls of the paged cache (csrc/pages_call.cpp) behave towards a program as the binding's own: the errors that they raise, and other threads beside them."""
import ctypes
import threading
import time

import pytest
import torch

from paper_2405_12532_b200 import binding as pb

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def _pages(**kw):
    p = pb.PyrPages(n_kv_heads=2, head_dim=64, page_rows=16, n_pages=4, n_lists=2, max_pages=2, **{"bits": 8, **kw})
    assert p._call is not None
    return p


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("compiled", [True, False])
def test_results_that_do_not_fit_raise_what_torch_raises(compiled, bits):
    """Results of 2^38 bytes and more, for queries that are one row seen many times: the device is not asked for such memory."""
    p = _pages(bits=bits)
    if not compiled:
        p._call = None
    row = torch.ones(1, 1, 2, 64, dtype=BF, device=DEV)
    zero = torch.zeros(1, 1, 1, dtype=torch.int32, device=DEV)
    wide, tall = row[:, :, :1].expand(1, 1, (1 << 31) - 2, 64), row.expand(1 << 20, 1 << 14, -1, -1)
    calls = [lambda: p.attn(wide), lambda: p.attn(tall, lse=True)]
    if bits == 8:
        calls += [lambda: p.select(tall, 8), lambda: p.attn_blocks(wide, zero.view(1, 1, 1, 1).repeat(1, 1, 2, 1)),
                  lambda: p.append(row, row, pos=zero, rope=torch.zeros(1, 64, device=DEV), q=wide)]
    torch.cuda.set_per_process_memory_fraction(0.5)
    try:
        for call in calls:
            with pytest.raises(torch.OutOfMemoryError):
                call()
    finally:
        torch.cuda.set_per_process_memory_fraction(1.0)
    assert p.attn(row, zero.view(1)).shape == row.shape and p.status() == 0


def test_other_threads_run_while_the_library_does():
    """A library call of 0.3 s (the C library's usleep in the place of all five, whose first argument is the handle): a thread that wakes up
    every 5 ms gets on meanwhile, as beside a call through ctypes."""
    libc = ctypes.CDLL(None)
    names = ("attn", "attn_blocks", "select", "append", "read")
    c = pb._calls().cache(300_000, torch.cuda.current_device(), 2, 64)
    k = torch.zeros(1, 1, 2, 64, device=DEV)
    slots, ticks, stop = torch.zeros(1, 1, 2, 1, dtype=torch.int32, device=DEV), [], threading.Event()

    def tick():
        while not stop.wait(0.005):
            ticks.append(time.monotonic())

    thread = threading.Thread(target=tick)
    pb._calls().setup(*[ctypes.cast(libc.usleep, ctypes.c_void_p).value] * len(names))
    try:
        thread.start()
        for call in (lambda: pb._calls().read(c, k, k, None, None, None), lambda: pb._calls().attn(c, k, None, None, k, False, 0.0),
                     lambda: pb._calls().attn(c, k, None, slots, k, False, 0.0), lambda: pb._calls().select(c, k, 1, None, 0, 0, slots),
                     lambda: pb._calls().append(c, k, k, None, None, None, None, None, None, None, None)):
            before = time.monotonic()
            call()
            after = time.monotonic()
            assert after - before >= 0.25 and sum(before < t < after for t in ticks) >= 10
    finally:
        pb._calls().setup(*[ctypes.cast(getattr(pb.lib(), "pyr_pages_" + x), ctypes.c_void_p).value for x in names])
        stop.set()
        thread.join()
    p = _pages()
    assert p.attn(k, torch.zeros(1, dtype=torch.int32, device=DEV)).shape == k.shape and p.status() == 0

"""The binding imports where torch has no CUDA parts, so that the host-only calls (byte accounting, argument checks) work there."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:      # as in a build of torch for the CPU
    delattr(torch._C, name)
from paper_2405_12532_b200 import binding as pb
cfg = pb.make_pages_config(n_kv_heads=2, head_dim=64, n_pages=4, n_lists=2, max_pages=2)
assert pb.pyr_pages_bytes(cfg)[0] > 0
assert pb.lib().pyr_recent_len_from_ratio is not None
"""


def test_the_binding_imports_without_the_cuda_parts_of_torch():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr

"""How the binding comes by its compiled calls (csrc/pages_call.cpp) and by the format of a cache, without a GPU."""
import warnings

import pytest

from paper_2405_12532_b200 import binding as pb


def test_a_compiled_module_that_does_not_load_is_done_without(tmp_path, monkeypatch):
    """What was built for another torch or Python: one warning, and the binding's own path from the first cache on."""
    bad = tmp_path / "_pages_call.so"
    bad.write_bytes(b"not a library")
    monkeypatch.setattr(pb, "_CALL_PATH", str(bad))
    monkeypatch.setattr(pb, "_call", None)
    with pytest.warns(RuntimeWarning, match="_pages_call.so"):
        assert pb._calls() is False
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert pb._calls() is False
    monkeypatch.setattr(pb, "_CALL_PATH", str(tmp_path / "none.so"))
    monkeypatch.setattr(pb, "_call", None)
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        assert pb._calls() is False                              # not built


def test_the_flag_of_the_header_names_the_format_too():
    """flags=PYR_PAGES_8BIT and bits=8 are the same configuration: no group of dimensions, since the scale is a page's."""
    shape = dict(n_kv_heads=2, head_dim=128, n_pages=4, n_lists=2, max_pages=2)
    by_flag, by_bits = (pb.make_pages_config(**shape, **kw) for kw in (dict(flags=pb.PYR_PAGES_8BIT), dict(bits=8)))
    assert bytes(by_flag) == bytes(by_bits) and pb.pyr_pages_bytes(by_flag) == pb.pyr_pages_bytes(by_bits)
    assert pb.make_pages_config(**shape).group == 64

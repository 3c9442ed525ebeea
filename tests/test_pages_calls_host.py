"""How the binding comes by its compiled calls (csrc/pages_call.cpp), without a GPU."""
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

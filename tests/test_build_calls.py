"""The build where Python's headers are not installed: the library is made all the same,
and only the client's attention, whose binding needs them, says what is missing."""
import importlib.machinery
import os
import sys
import sysconfig

import pytest


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """build.py over a source of its own, and what makes it see headers or none."""
    import __graft_entry__
    b = __graft_entry__._load_build_module()
    src = tmp_path / "one.cu"
    src.write_text('extern "C" int one() { return 1; }\n')
    monkeypatch.setattr(b, "_sources", lambda: [str(src)])
    monkeypatch.setattr(b, "BUILD", str(tmp_path / "obj"))
    monkeypatch.setattr(b, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(b, "CALLS", str(tmp_path / os.path.basename(b.CALLS)))
    real = sysconfig.get_paths

    def headers(there):
        none = lambda *a, **k: dict(real(*a, **k), include=str(tmp_path))  # noqa: E731
        monkeypatch.setattr(sysconfig, "get_paths", real if there else none)
    return b, headers


def test_library_without_python_headers(tree):
    b, headers = tree
    headers(False)
    assert b.needs_build()
    assert b.build() == b.LIB and os.path.exists(b.LIB) and not os.path.exists(b.CALLS)
    assert not b.needs_build()
    headers(True)
    assert b.needs_build()
    b.build()
    assert os.path.exists(b.CALLS) and not b.needs_build()


def test_module_is_named_for_its_interpreter(tree):
    b, _ = tree
    assert b.CALLS.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert sysconfig.get_config_var("EXT_SUFFIX") in importlib.machinery.EXTENSION_SUFFIXES


def test_calls_without_the_module_say_so(monkeypatch):
    import __graft_entry__
    __graft_entry__._load_build_module().build()
    import paper_2609_10264_gb300 as pv
    monkeypatch.setattr(pv, "_native", None)
    monkeypatch.setitem(sys.modules, "paper_2609_10264_gb300._calls", None)
    monkeypatch.delattr(pv, "_calls", raising=False)
    with pytest.raises(ImportError, match="Python's headers"):
        pv._open_calls()

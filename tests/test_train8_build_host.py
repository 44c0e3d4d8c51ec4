"""The optional marshalling module: built for the torch that is installed, and only then used."""
import types
import warnings

import pytest
import torch

from paper_1501_06633_b200 import build, train8


def test_the_built_module_names_its_torch():
    built = build.build_binding()
    if built is None:
        pytest.skip("no compiler, or no headers")
    from paper_1501_06633_b200 import _train8
    assert _train8.torch_version == torch.__version__
    assert not build.binding_stale(torch.__version__)


def test_another_torch_makes_it_stale_and_unused():
    if build.build_binding() is None:
        pytest.skip("no compiler, or no headers")
    assert build.binding_stale("0.0.1")          # whatever the files' times say
    train8._library()
    assert train8._usable(types.SimpleNamespace(torch_version=torch.__version__))
    for other in (types.SimpleNamespace(torch_version="0.0.1"), types.SimpleNamespace()):
        with pytest.warns(UserWarning, match="built for torch"):
            assert not train8._usable(other)


def test_building_without_a_compiler_leaves_the_module_out(monkeypatch):
    monkeypatch.setenv("CXX", "no-such-compiler")
    with pytest.warns(UserWarning, match="no-such-compiler"):
        assert build.build_binding(force=True) is None


def test_building_without_headers_leaves_the_module_out(monkeypatch, tmp_path):
    import sysconfig
    paths = dict(sysconfig.get_paths(), include=str(tmp_path))
    monkeypatch.setattr(sysconfig, "get_paths", lambda *a, **k: paths)
    with warnings.catch_warnings(record=True) as seen:
        warnings.simplefilter("always")
        assert build.build_binding(force=True) is None
    assert any("Python.h" in str(w.message) for w in seen)

"""The library and the module of the layer calls are built apart: the codec and the C ABI need no Python headers."""
import os
import subprocess
import sys

import pytest

import paper_1905_10830_b200 as tc
from paper_1905_10830_b200 import binding, build


@pytest.fixture
def scratch(tmp_path, monkeypatch):
    """The package's own built files, seen from a folder where the module is not built yet."""
    build.build_library()
    monkeypatch.setattr(build, "LAYERS", str(tmp_path / "_layers.so"))
    return tmp_path


def test_a_module_that_cannot_be_compiled_leaves_the_library(scratch, monkeypatch):
    bad = scratch / "bad.cpp"
    bad.write_text("#error no headers here\n")
    monkeypatch.setattr(build, "LAYERS_SRC", str(bad))
    with pytest.warns(RuntimeWarning, match="no headers here"):
        assert build.build_library() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.LAYERS)
    with pytest.raises(RuntimeError, match="no headers here"):
        build.build_layers()


def test_the_command_fails_where_the_module_cannot_be_compiled(scratch):
    bad = scratch / "bad.cpp"
    bad.write_text("#error no headers here\n")
    code = (f"from paper_1905_10830_b200 import build; build.LAYERS = {build.LAYERS!r}; build.LAYERS_SRC = {str(bad)!r}; "
            "import sys; sys.exit(build.main([]))")
    res = subprocess.run([sys.executable, "-c", code], cwd=build.ROOT, capture_output=True, text=True)
    assert res.returncode == 1 and "no headers here" in res.stderr and build.LIB in res.stdout


def test_a_module_of_another_torch_is_built_again(scratch, monkeypatch):
    import torch
    assert build.build_layers() == build.LAYERS
    first = os.stat(build.LAYERS)
    build.build_layers()
    assert os.stat(build.LAYERS).st_mtime_ns == first.st_mtime_ns               # the same torch, the same sources
    monkeypatch.setattr(torch, "__version__", "0.0.0+other")
    build.build_layers()
    assert os.stat(build.LAYERS).st_mtime_ns > first.st_mtime_ns


def test_a_module_of_another_torch_is_not_loaded(scratch, monkeypatch):
    monkeypatch.setattr(binding, "_layers", None)
    with open(build.LAYERS + ".built", "w") as f:
        f.write("torch 0.0.0+other, cpython-00")
    with pytest.raises(ImportError, match="0.0.0.other.*build"):
        binding._layer_calls()
    os.remove(build.LAYERS + ".built")                                           # not known: as it is
    assert binding._layer_calls() is not None


def test_the_layer_calls_say_what_is_missing(monkeypatch):
    build.build_library()
    monkeypatch.setattr(binding, "_layers", None)
    monkeypatch.setitem(sys.modules, "paper_1905_10830_b200._layers", None)
    monkeypatch.delattr(tc, "_layers", raising=False)
    with pytest.raises(ImportError, match="build"):
        binding._layer_calls()

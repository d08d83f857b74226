"""What `build` builds, and when: with the compilers' places taken by functions that write a file."""
import importlib.metadata
import os
import subprocess
import sys
import types
import warnings

import pytest
import torch

from paper_2306_08289_b200 import binding as B
from paper_2306_08289_b200 import build as build_mod
from paper_2306_08289_b200 import operators as ops


@pytest.fixture
def made(tmp_path, monkeypatch):
    """The names of what has been built, in order, into an empty place; set `broken` to let the second compiler fail."""
    out = types.SimpleNamespace(names=[], broken=False)
    monkeypatch.setattr(build_mod, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build_mod, "CALLS", str(tmp_path / "_calls.so"))

    def write(cmd):
        target = cmd[cmd.index("-o") + 1]
        with open(target, "w"):
            pass
        out.names.append(os.path.basename(target).split(".tmp")[0])

    def run(cmd, **kw):
        write(cmd)
        return subprocess.CompletedProcess(cmd, 0, "", "")

    def popen(cmd, **kw):
        if not out.broken:
            write(cmd)
        return types.SimpleNamespace(communicate=lambda: ("text", None), returncode=int(out.broken))

    monkeypatch.setattr(build_mod, "subprocess", types.SimpleNamespace(run=run, Popen=popen, PIPE=None, STDOUT=None))
    return out


def test_what_is_built_is_not_built_again(made):
    assert build_mod.build() == build_mod.LIB and made.names == ["lib.so", "_calls.so"]
    build_mod.build()
    assert made.names == ["lib.so", "_calls.so"] and build_mod.calls_version() == torch.__version__
    build_mod.build(force=True)
    assert made.names == ["lib.so", "_calls.so"] * 2
    assert sorted(os.listdir(os.path.dirname(build_mod.LIB))) == ["_calls.so", "_calls.so.torch", "lib.so"]


@pytest.mark.parametrize("how", ["no torch", "no CUDA in it"])
def test_the_library_needs_no_torch(made, monkeypatch, tmp_path, how):
    if how == "no torch":
        def absent(name):
            raise importlib.metadata.PackageNotFoundError(name)

        monkeypatch.setattr(build_mod.importlib.metadata, "version", absent)
    else:
        monkeypatch.setattr(build_mod.importlib.util, "find_spec", lambda name: types.SimpleNamespace(submodule_search_locations=[str(tmp_path)]))
    assert build_mod.torch_version() is None
    for _ in range(3):
        assert build_mod.build() == build_mod.LIB
    assert made.names == ["lib.so"]


def test_another_torch_has_its_side_built_again(made, monkeypatch):
    build_mod.build()
    monkeypatch.setattr(build_mod, "torch_version", lambda: "99.0")
    build_mod.build()
    build_mod.build()
    assert made.names == ["lib.so", "_calls.so", "_calls.so"] and build_mod.calls_version() == "99.0"


def test_a_failure_of_the_second_compiler_leaves_the_library_built(made):
    made.broken = True
    for _ in range(2):
        with pytest.raises(RuntimeError, match="g\\+\\+"):
            build_mod.build()
    assert made.names == ["lib.so"]
    made.broken = False
    build_mod.build()
    assert made.names == ["lib.so", "_calls.so"]


@pytest.mark.parametrize("how", ["missing", "of another torch"])
def test_calls_go_the_other_way_where_their_usual_side_cannot_be_loaded(monkeypatch, how):
    build_mod.build()
    monkeypatch.setattr(ops, "_calls", None)
    if how == "missing":
        monkeypatch.setitem(sys.modules, "paper_2306_08289_b200._calls", None)
    else:
        monkeypatch.setattr(build_mod, "calls_version", lambda: "1.0")
    t = torch.zeros(4, 8)
    with pytest.warns(RuntimeWarning, match="cannot be loaded"):
        assert ops._usual().rms_norm(t, None, None, 1e-6) is None
    with warnings.catch_warnings():
        warnings.simplefilter("error")  # it is said once
        for call in (lambda: ops.rms_norm(t), lambda: ops.route(t, 2), lambda: ops.clip_gradients([t], 1.0)):
            with pytest.raises(B.A2Error) as e:
                call()
            assert e.value.code == B.A2_EINVAL

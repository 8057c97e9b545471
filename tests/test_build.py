"""What is built when, and what is left when a part cannot be built (compilers replaced by a fake; no GPU)."""
import os
import types

import pytest

from paper_2510_08431_b200 import build


@pytest.fixture
def fake(tmp_path, monkeypatch):
    """build with its outputs in tmp_path; compilers write an empty file, or fail where `broken` names them."""
    f = types.SimpleNamespace(calls=[], broken=set(), dir=tmp_path)
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "HOST_LIB", str(tmp_path / "_host.so"))
    monkeypatch.setattr(build, "HOST_STAMP", str(tmp_path / "_host.so.stamp"))
    monkeypatch.setattr(build, "_nvcc", lambda: "nvcc")
    monkeypatch.setenv("CXX", "g++")

    def run(cmd, **kw):
        f.calls.append(cmd[0])
        if cmd[0] in f.broken:
            return types.SimpleNamespace(returncode=1, stdout="", stderr="no such header")
        open(cmd[cmd.index("-o") + 1], "w").close()
        return types.SimpleNamespace(returncode=0, stdout="", stderr="")

    monkeypatch.setattr(build.subprocess, "run", run)
    return f


def test_both_are_built_once(fake):
    assert build.build_library() == build.LIB
    assert fake.calls == ["nvcc", "g++"] and os.path.exists(build.LIB) and os.path.exists(build.HOST_LIB)
    build.build_library()
    assert fake.calls == ["nvcc", "g++"]
    build.build_library(force=True)
    assert fake.calls == ["nvcc", "g++"] * 2


def test_the_library_does_not_need_the_host_binding(fake):
    fake.broken.add("g++")
    with pytest.warns(RuntimeWarning, match="no such header"):
        assert build.build_library() == build.LIB
    assert os.path.exists(build.LIB) and not os.path.exists(build.HOST_LIB)
    with pytest.raises(RuntimeError):
        build.build_host()


def test_a_library_that_does_not_compile_is_an_error(fake):
    fake.broken.add("nvcc")
    with pytest.raises(RuntimeError, match="no such header"):
        build.build_library()


def test_another_torch_makes_the_host_binding_stale(fake, monkeypatch):
    import torch
    build.build_library()
    assert not build.host_is_stale()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build.host_is_stale()
    build.build_library()
    assert fake.calls == ["nvcc", "g++", "g++"] and not build.host_is_stale()
    os.remove(build.HOST_STAMP)
    assert build.host_is_stale()

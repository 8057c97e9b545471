"""Calls that can do without the host binding look for it once (no GPU)."""
import sys
import types

import pytest

from paper_2510_08431_b200 import attn_jvp as binding
from paper_2510_08431_b200 import build


@pytest.fixture
def unbound(monkeypatch):
    build.build_library()
    monkeypatch.setattr(binding, "_host_module", None)
    monkeypatch.setattr(binding, "_no_host", False, raising=False)
    return monkeypatch


def test_a_missing_binding_is_looked_for_once(unbound):
    tries = []

    def host():
        tries.append(1)
        raise RuntimeError("not there")

    unbound.setattr(binding, "host", host)
    assert not any(binding.has_host() for _ in range(5))
    assert len(tries) == 1


def test_a_binding_that_comes_later_is_used(unbound):
    with unbound.context() as m:
        m.setitem(sys.modules, "paper_2510_08431_b200._host", None)          # (an import of it raises ImportError)
        m.delattr(sys.modules["paper_2510_08431_b200"], "_host", raising=False)
        assert not binding.has_host()
        with pytest.raises(RuntimeError, match="build it with"):
            binding.host()
    binding.host()
    assert binding.has_host()


def test_a_binding_of_other_sources_is_a_missing_one(unbound):
    def bind(*addresses):
        raise TypeError("bind takes 9 arguments")

    old = types.SimpleNamespace(bind=bind)
    unbound.setitem(sys.modules, "paper_2510_08431_b200._host", old)
    unbound.setattr(sys.modules["paper_2510_08431_b200"], "_host", old, raising=False)
    assert not binding.has_host()
    with pytest.raises(RuntimeError, match="build it with"):
        binding.host()

"""The warning for a host binding that cannot be built names every call that needs it (compilers replaced by a fake; no GPU)."""
import ast
import fnmatch
import os
import re

import pytest

from paper_2510_08431_b200 import build
from tests.test_build import fake  # noqa: F401


def callers():
    """Public functions of the package whose body calls into the host binding."""
    found = set()
    for name in os.listdir(build.PKG):
        if name.endswith(".py"):
            with open(os.path.join(build.PKG, name)) as f:
                for node in ast.parse(f.read()).body:
                    if isinstance(node, ast.FunctionDef) and node.name not in ("host", "has_host") and any(
                            isinstance(n, ast.Call) and getattr(n.func, "attr", getattr(n.func, "id", "")) == "host" for n in ast.walk(node)):
                        found.add(node.name)
    return found


def test_the_warning_names_what_needs_the_binding(fake):  # noqa: F811
    fake.broken.add("g++")
    with pytest.warns(RuntimeWarning) as seen:
        build.build_library()
    (text,) = [str(w.message) for w in seen if "host binding" in str(w.message)]
    patterns = re.findall(r"[\w*]+", text.split("will not work")[0])
    names = callers()
    assert {"attention_jvp", "attention_backward", "rotary_table", "adaln_jvp", "block_select", "sparse_attention_jvp"} <= names
    for n in names:
        assert any(fnmatch.fnmatchcase(n, p) for p in patterns if len(p) > 3), n
    assert all(w in text for w in ("masks", "shared heads", "strided"))

"""Building: the library does without the compiled binding, which is kept apart for every Python and torch."""
import importlib.util
import os
import subprocess
import sys
import sysconfig

import pytest

from paper_2609_38169_gb300 import build_ext

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def child(code):
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


@pytest.mark.parametrize("lack", ["build_ext.BIND_SOURCE = 'missing.cpp'", "build_ext.sysconfig.get_paths = lambda: {'include': '/missing'}"],
                         ids=["source", "headers"])
def test_calls_that_need_no_binding_work_without_one(lack, tmp_path):
    pytest.importorskip("torch")
    child(f"""
from paper_2609_38169_gb300 import _lib, api as A, build_ext
import torch
build_ext.bind_so = lambda: {str(tmp_path / "bind.so")!r}
{lack}
assert A.stepq_kv_page_bytes(A.KvConfig(1, 1)) == 64 * 512
t = torch.zeros(1, 1, dtype=torch.int32)
try:
    A.stepq_kv_append(A.KvConfig(1, 1), 0, t, t, t, t, t)
except RuntimeError as e:
    assert "g++ failed" in str(e)
else:
    raise AssertionError
""")


def test_a_binding_for_every_python_and_torch(monkeypatch, tmp_path):
    pytest.importorskip("torch")
    places = {build_ext.bind_so()}
    abi = sysconfig.get_config_var
    monkeypatch.setattr(build_ext.sysconfig, "get_config_var", lambda n: "other-abi" if n == "SOABI" else abi(n))
    places.add(build_ext.bind_so())
    find = importlib.util.find_spec
    moved = importlib.util.spec_from_file_location("torch", str(tmp_path / "torch" / "__init__.py"))
    monkeypatch.setattr(build_ext.importlib.util, "find_spec", lambda n: moved if n == "torch" else find(n))
    places.add(build_ext.bind_so())
    assert len(places) == 3
    monkeypatch.setattr(build_ext.importlib.util, "find_spec", lambda n: None)
    assert build_ext.bind_so() is None

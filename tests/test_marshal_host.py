"""The library without the Python extension that the paged calls go through (csrc/marshal.cpp), and when that is built anew.  No GPU needed."""
import os
import shutil
import subprocess
import sys

import pytest

from paper_2602_08686_b200 import build as ckv_build

PROGRAM = r"""
import ctypes as C
import torch
from paper_2602_08686_b200 import binding as B
assert B.lib().ckv_version() > 0
s = B.ckv_shape(2, 32, 8, 128, 4096, 32, B.BF16, 0, 32 * 32 * 128, 32 * 128, 128, 8 * 4096 * 128, 4096 * 128, 128)
assert B.lib().ckv_workspace_bytes(C.byref(s), C.byref(B.ckv_params())) >= 0
z = lambda *n: torch.zeros(*n, dtype=torch.int32)
try:
    B.ckv_tree_masks(z(3), z(2), z(3, 1), torch.zeros(256, dtype=torch.uint8))
except ValueError as e:                          # arguments are checked all the same
    assert "CUDA tensors" in str(e)
else:
    raise AssertionError
try:
    B._paged_call("ckv_tree_masks", 0, None)
except RuntimeError as e:
    assert "_marshal.so" in str(e) and "paper_2602_08686_b200.build" in str(e) and isinstance(e.__cause__, ImportError)
else:
    raise AssertionError
"""


@pytest.mark.parametrize("what", ["missing", "broken"])
def test_only_the_paged_calls_need_it(tmp_path, what):
    ckv_build.build_lib()
    package = tmp_path / "paper_2602_08686_b200"
    shutil.copytree(ckv_build.HERE, package, ignore=shutil.ignore_patterns("csrc", "_build", "__pycache__", "_marshal.so"))
    if what == "broken":
        (package / "_marshal.so").write_bytes(b"of another system")
    subprocess.run([sys.executable, "-c", PROGRAM], check=True, cwd=tmp_path, env=dict(os.environ, PYTHONPATH=str(tmp_path)))


def test_it_is_built_for_the_python_and_torch_there_are(tmp_path, monkeypatch):
    ckv_build.build_lib()
    assert not ckv_build.marshal_stale()
    calls = []

    def compiler(cmd):
        calls.append(cmd)
        with open(cmd[cmd.index("-o") + 1], "w") as f:
            f.write("built")

    monkeypatch.setattr(ckv_build.subprocess, "check_call", compiler)
    monkeypatch.setattr(ckv_build, "MARSHAL", str(tmp_path / "_marshal.so"))
    monkeypatch.setattr(ckv_build, "MARSHAL_FOR", str(tmp_path / "_build" / "marshal_for"))
    ckv_build.build_marshal()                    # nobody knows what it was built for
    assert len(calls) == 1 and not ckv_build.marshal_stale()
    ckv_build.build_marshal()
    assert len(calls) == 1
    with open(ckv_build.MARSHAL_FOR, "w") as f:
        f.write(ckv_build.built_for().replace("torch ", "torch 1."))
    ckv_build.build_marshal()
    assert len(calls) == 2 and not ckv_build.marshal_stale()
    monkeypatch.setattr(ckv_build, "built_for", lambda: "another Python")
    ckv_build.build_marshal()
    assert len(calls) == 3

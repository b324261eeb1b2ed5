"""The compiled checks of tensors (csrc/marshal.cpp) with what they cannot answer: an error of the interpreter, and the process goes on.  Each runs in a process of its own."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_STORAGE = r"""
import types
import torch
from paper_2512_15550_amd import _marshal as M, binding as B
c = types.SimpleNamespace(torch_dtype=torch.float32, device=-1, _pointer=M.pointer, _pointers=M.pointers, _rows=M.rows)
whole = torch.zeros(3)
calls = {
    "_on": lambda t: B._on(c, "t", t, torch.float32, tuple(t.shape)),
    "_all_on": lambda t: B._all_on(c, "whole", whole, torch.float32, (3,), "t", t, torch.float32, tuple(t.shape)),
    "_rows_on": lambda t: B._rows_on(c, "t", t, t.shape[0], t.shape[1]),
}
refused = []
def asks(t):
    try:
        calls[%r](t)
    except RuntimeError as e:
        refused.append(str(e))
    return t.sum()
x = torch.zeros((3, 4, 128))
{
    "vmap": lambda: torch.vmap(asks)(torch.zeros((2, 3, 4, 128))),
    "grad": lambda: torch.func.grad(asks)(x),
    "jvp": lambda: torch.func.jvp(asks, (x,), (x,)),
}[%r]()
assert len(refused) == 1 and "storage" in refused[0] and "\n" not in refused[0], refused
assert calls[%r](x)
print("ok")
"""


@pytest.mark.parametrize("transform", ["vmap", "grad", "jvp"])
@pytest.mark.parametrize("call", ["_on", "_all_on", "_rows_on"])
def test_a_tensor_without_storage_is_refused(call, transform):
    r = subprocess.run([sys.executable, "-c", WITHOUT_STORAGE % (call, transform, call)], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "ok\n", f"status {r.returncode}\n" + r.stdout + r.stderr


def test_a_shape_of_no_whole_numbers_is_no_tensor_s_shape():
    """An answer, and no error left behind for the next call to trip over."""
    import torch

    from paper_2512_15550_amd import _marshal as M
    t, rows = torch.zeros((2, 3)), torch.zeros((2, 3, 128))
    for bad in ("3", 2 ** 70, None, 3.5):
        assert M.pointer(t, torch.float32, (2, bad), -1) == -1
        assert M.pointers(-1, "t", t, torch.float32, (2, 3), "t", t, torch.float32, (2, bad)) == 1
        assert M.rows(rows, torch.float32, 2, bad, -1) is None and M.rows(rows, torch.float32, bad, 3, -1) is None
        for device in ("cuda", 2 ** 70, None):
            assert M.pointer(t, torch.float32, (2, 3), device) == -1 and M.pointers(device, "t", t, torch.float32, (2, 3)) == 0
            assert M.rows(rows, torch.float32, 2, 3, device) is None
    assert M.pointer(t, torch.float32, (2, 3), -1) == t.data_ptr()

"""The binding's argument checks on tensors whose accessors throw or that have no memory: an error, never an abort.  Such
tensors are made without a GPU by fake tensors on a CUDA device and by function transforms of them; a child process, since
the failure that is guarded against would end the interpreter."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PRELUDE = """
import sys
sys.path.insert(0, %r)
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from paper_2601_02360_b200 import api, build
build.build_args()
c = api._checks()

def refused(call):
    try:
        got = call()
    except ValueError as e:
        print("refused:", str(e).splitlines()[0])
    else:
        raise SystemExit(f"not refused: {got}")
""" % ROOT


def _child(body):
    r = subprocess.run([sys.executable, "-c", PRELUDE + body], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout[-500:], r.stderr[-1500:])
    return r.stdout


BOTH = "(refused(lambda: c.ptr(t, 'x', 4, 1)), refused(lambda: c.rows(t, 'x', 2, 2, 1)), sys.exit(0))"


@pytest.mark.parametrize("how", ["torch.func.grad(lambda t: %s)(torch.empty(2, 2, device='cuda'))",
                                 "torch.vmap(lambda t: %s)(torch.empty(3, 2, 2, device='cuda'))"])
def test_accessors_that_throw_raise(how):
    out = _child("with FakeTensorMode(allow_non_fake_inputs=True):\n    " + how % BOTH)
    assert out.count("refused:") == 2


def test_a_tensor_without_memory_is_not_an_absent_one():
    out = _child("""
with FakeTensorMode(allow_non_fake_inputs=True):
    t = torch.empty(2, 2, device='cuda')
    refused(lambda: c.ptr(t, 'x', 4, 1))
    refused(lambda: c.rows(t, 'x', 2, 2, 1))
    assert c.ptr(t[:0], 'x', 0, 1) == 0 and c.ptr(None, 'x', 4, 1) == 0
""")
    assert out.count("refused:") == 2

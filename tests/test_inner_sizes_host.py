"""Sizes at and beyond the ends of what the inner-step calls take, without a GPU: nothing is launched."""
import os
import subprocess
import sys

import pytest

from paper_2601_02360_b200 import api, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000


@pytest.fixture(scope="module")
def lib():
    build.build()
    return api.load()


@pytest.mark.parametrize("n,d", [(5000, 0), (5000, 2 ** 32 - 1), (5000, 2 ** 32 - 3), (5000, 2 ** 31), (0, 0), (2 ** 63, 8)])
def test_the_workspace_of_a_size_that_is_refused(lib, n, d):
    # a child: the division that is guarded against would end the process
    code = f"import sys; sys.path.insert(0, {ROOT!r}); from paper_2601_02360_b200 import api; print(api.load().sl_embed_grad_workspace({n}, 10, {d}))"
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0 and int(r.stdout) == 0, (r.returncode, r.stderr[-300:])

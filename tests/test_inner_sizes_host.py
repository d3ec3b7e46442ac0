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


def test_widths_that_no_grid_holds_are_refused(lib):
    def call(d, dX=P):
        return lib.sl_embed_grad(P, dX, 0, 1.0, 5000, 1, 10, d, P, 0, 0, 1, P, 0, 0)
    UNS = api.SL_ERR_UNSUPPORTED
    assert call(65535 * 64 + 1) == UNS and call(65535 * 64 + 8, dX=P + 4) == UNS      # single elements: 64 columns to a CTA
    assert call(65535 * 128 + 8) == UNS and call(1 << 31) == UNS                      # vectors: 128


def test_empty_arrays_may_have_no_memory(lib):
    lay, OK = api.Layout([0, 0]).ref(), api.SL_OK
    hyper = (0, 1e-3, 0.9, 0.95, 1e-8, 1, 0, 0, 0)
    assert lib.sl_adamw(0, 0, 0, 0, 0, 0, 0, lay, *hyper) == OK and lib.sl_adamw8(0, 0, 0, 0, 0, 0, 0, 0, 0, lay, *hyper) == OK
    assert lib.sl_adamw8_pack(0, 0, lay, 0, 0, 0, 0, 0) == OK and lib.sl_adamw8_unpack(0, 0, 0, 0, lay, 0, 0, 0) == OK
    assert lib.sl_embed_lookup(0, P, P, P, 0, 1.0, 0, 2, 10, 8, 0, 0, 0, 0) == OK
    assert lib.sl_norm_block(0, 0, 0, 0, 0, P, P, 0, 0, 8, 8, 8, 1.0, 1e-6, 0, 0, 0, 0, 0, 0) == OK
    assert lib.sl_norm_block_grad(0, 0, 0, 0, 0, 0, 0, P, P, 0, 0, 0, 0, 8, 8, 8, 1.0, 0, 0, 0, 0, 0, 1, 0, 0, 0) == OK
    # what does not depend on their number is still checked
    INV = api.SL_ERR_INVALID_ARG
    assert lib.sl_embed_lookup(0, 0, P, P, 0, 1.0, 0, 2, 10, 8, 0, 0, 0, 0) == INV
    assert lib.sl_embed_lookup(0, P, P, P, 0, float("nan"), 0, 2, 10, 8, 0, 0, 0, 0) == INV
    assert lib.sl_norm_block(0, 0, 0, 0, 0, P, P, 0, 0, 0, 8, 8, 1.0, 1e-6, 0, 0, 0, 0, 0, 0) == INV
    assert lib.sl_adamw(0, 0, 0, 0, 0, 0, 0, lay, 0, -1.0, 0.9, 0.95, 1e-8, 1, 0, 0, 0) == INV

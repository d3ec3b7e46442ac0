"""sl_adamw8 over the whole range of eps that is accepted, against the numpy checker in float32.

theta starts at 0 and has no decay, so that it is the move itself: within 2^-20 of the checker's, plus the product's and theta's own
roundings (2 * 2^-24, and 2^-8 in bfloat16), or 2^-148 where it is subnormal.  Where eps < a 2^-41 or eps > 2^100 the root and the
quotient are the checker's operations: bit for bit."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api

pytestmark = pytest.mark.gpu
OFF = [0, 512, 1024, 1031, 2000, 2003, 5000]              # whole blocks on and off the grid of eight, short ones
BETA1, BETA2, LR = 0.9, 0.999, 1e-3


def _grad(n, seed):
    """zeros, gradients whose square is subnormal or zero, ordinary ones"""
    r = np.random.default_rng(seed)
    g = r.standard_normal(n).astype(np.float32)
    size = r.integers(0, 5, n)
    return np.where(size == 0, np.float32(0), g * np.asarray([0, 1e-3, 1e-19, 3e-22, 1e-25], np.float32)[size]).astype(np.float32)


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1.2e-38, 1e-30, 1e-20, 1e-15, 1e-12, 1e-11, 2e-11, 1e-8, 1e-3, 1e25, 1e31, 3e38])
@pytest.mark.parametrize("tt,gt", [("f", "f"), ("b", "b")])
def test_every_eps(eps, tt, gt):
    n = OFF[-1]
    dt = {"f": torch.float32, "b": torch.bfloat16}
    th = torch.zeros(n, dtype=dt[tt], device="cuda")
    s8 = api.alloc_states8(OFF)
    m, v, before = np.zeros(n, np.float32), np.zeros(n, np.float32), np.zeros(n, np.float32)
    for step in (1, 2):
        g = torch.from_numpy(_grad(n, step)).to(dt[gt])
        api.sl_adamw8(th, g.cuda(), *s8, OFF, LR, BETA1, BETA2, eps, step)
        want, m, v = oi.adamw(before, g.float().numpy(), m, v, OFF, None, LR, BETA1, BETA2, eps, step)
        got = th.float().cpu().numpy()
        assert np.isfinite(want).all() and np.isfinite(got).all()
        exact = eps < 2.0 ** -41 / np.sqrt(1 - BETA2 ** step) * (1 - 1e-6) or eps > 2.0 ** 100
        if exact:
            assert np.array_equal(got, torch.from_numpy(want).to(dt[tt]).float().numpy())
        else:
            move = np.abs(want.astype(np.float64) - before)
            tol = 2.0 ** -20 * move + 2.0 ** -23 * np.abs(want) + 2.0 ** -148 + (2.0 ** -8 * np.abs(want) if tt == "b" else 0)
            assert np.all(np.abs(got - want.astype(np.float64)) <= tol)
        q = oi.quantise(m, v, OFF)
        for a, b in zip(s8, q):
            assert np.array_equal(a.cpu().numpy(), b)
        m, v = oi.dequantise(*q, OFF)
        before = got

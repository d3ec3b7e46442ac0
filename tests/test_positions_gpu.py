"""Position tables that are longer than the batch."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("n,L", [(1, 2), (1, 5000), (7, 8), (9, 100), (100, 131072), (1500, 1501), (3000, 70000)])
@pytest.mark.parametrize("d", [24, 33])
def test_lookup_with_positions_that_no_token_has(n, L, d):
    r = np.random.default_rng(n + L)
    ids, T, P = r.integers(0, 50, n).astype(np.int32), r.standard_normal((50, d)).astype(np.float32), r.standard_normal((L, d)).astype(np.float32)
    X = torch.full((n, d), float("nan"), device="cuda")
    api.sl_embed_lookup(torch.from_numpy(ids).cuda(), torch.from_numpy(T).cuda(), None, torch.from_numpy(P).cuda(), 1.5, n, L, 50, d, X)
    assert np.array_equal(X.cpu().numpy(), np.float32(1.5) * T[ids] + P[:n])


@pytest.mark.parametrize("n,L", [(1, 2), (7, 5000), (1000, 1001), (2000, 2003), (3000, 9000)])
@pytest.mark.parametrize("d", [24, 33])
@pytest.mark.parametrize("acc", [False, True])
def test_gradient_of_positions_that_no_token_has(n, L, d, acc):
    r = np.random.default_rng(n + L)
    ids, dX = r.integers(0, 50, n).astype(np.int32), r.standard_normal((n, d)).astype(np.float32)
    old = r.standard_normal((L, d)).astype(np.float32)
    old[n:, ::2] = -0.0                                   # a sum of nothing would make it +0
    dT, dpos = torch.zeros(50, d, device="cuda"), torch.from_numpy(old).cuda()
    ws = torch.empty(api.sl_embed_grad_workspace(n, 50, d), dtype=torch.uint8, device="cuda")
    api.sl_embed_grad(torch.from_numpy(ids).cuda(), torch.from_numpy(dX).cuda(), 1.0, n, L, 50, d, dT, dpos, acc, ws)
    got = dpos.cpu().numpy()
    assert np.array_equal(got[:n], old[:n] + dX if acc else dX)
    assert np.array_equal(got[n:].view(np.int32), old[n:].view(np.int32)) if acc else not got[n:].any()
    want, _, mag, _ = oi.embed_grad(ids, dX, 1.0, L, 50, False)
    assert np.all(np.abs(dT.cpu().numpy() - want) <= (n + 4) * U * mag)

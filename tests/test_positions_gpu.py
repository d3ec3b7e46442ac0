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

"""What the inner-step calls take and refuse beside the ordinary: views that are negated when read, wrong shapes, empty
batches, other devices; and what their Python forms promise (orders of differentiation, flags, step counts)."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api, inner

pytestmark = pytest.mark.gpu


def _randn(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def test_views_that_are_negated_when_read():
    scale = torch.complex(torch.zeros(1, device="cuda"), torch.full((1,), 0.5, device="cuda")).conj().imag       # -0.5
    assert scale.is_neg() and scale.is_contiguous()
    a = [torch.zeros(8, device="cuda") for _ in range(4)]
    with pytest.raises(ValueError):
        api.sl_adamw(*a, [0, 8], 1e-3, 0.9, 0.95, 1e-8, 1, grad_scale=scale)
    n, d = 5, 24
    x, b, w, T = _randn(n, d), _randn(n, d, seed=1), _randn(d, seed=2), _randn(n, d, seed=3)
    with pytest.raises(ValueError):
        api.sl_norm_block(x, torch._neg_view(b), None, None, w, n, d, 1.0, 1e-6, x.clone(), x.clone())
    # the Python forms read what the tensor is
    for got, want in zip(inner.norm_block(torch._neg_view(x), torch._neg_view(b), torch._neg_view(T), torch._neg_view(w), w),
                         inner.norm_block(-x, -b, -T, -w, w)):
        assert torch.equal(got, want)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    assert torch.equal(inner.embed_lookup(ids, torch._neg_view(T)), -T)

"""sl_norm_block_grad on rows of very large and very small elements (eps = 0): the formula is homogeneous, and so are the bounds of
the ordinary range, which hold as long as squares of the elements and of their inverses stay in float32."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api
from test_norm_block_gpu import ALPHA, U, _bounds, _cuda, _f64, _inputs, _q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,d", [(5, 33), (9, 264), (4, 5001), (3, 8192)])
@pytest.mark.parametrize("exponent", [-55, -48, 0, 48, 55])
def test_gradient_of_scaled_rows(n, d, exponent):
    # below 0 it is b alone that is small: h keeps the normalised term
    x, b, g, wp, wn = _inputs(n, d, "all", "f", "f", "f")
    x, b = (np.ldexp(a, exponent).astype(np.float32) for a in (x, b))
    h64, _, rp, rn = oi.norm_block(*_f64(x, b, g, wp, wn), ALPHA, 0.0)
    h, rp, rn = (a.astype(np.float32) for a in (h64, rp, rn))
    dy = _q(np.random.default_rng(d).standard_normal((n, d)), "f")
    out = [torch.empty(n, d, device="cuda") for _ in range(3)] + [torch.empty(d, device="cuda") for _ in range(2)]
    ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
    api.sl_norm_block_grad(None, _cuda(dy), _cuda(h), _cuda(b), _cuda(g), _cuda(wp), _cuda(wn), _cuda(rp), _cuda(rn), n, d, ALPHA, *out, False, ws)
    f = _f64(None, dy, h, b, g, wp, wn, rp, rn)
    want, mags = oi.norm_block_grad(*f, float(np.float32(ALPHA))), _bounds(*f, ALPHA)
    gate = 2.4 * np.abs(f[4])
    for k, t in zip(("dx", "db", "dg", "dw_post", "dw_pre"), out):
        steps = n + 160 + gate.max() if k.startswith("dw") else 160 + np.maximum(gate, np.max(gate, 1, keepdims=True))
        assert np.all(np.abs(t.cpu().numpy() - want[k]) <= steps * U * mags[k] + 1e-37), k


@pytest.mark.parametrize("n,d", [(5, 33), (9, 264), (4, 5001), (3, 8192)])
@pytest.mark.parametrize("exponent", [-55, -48, 48, 55])
def test_gradient_of_a_scaled_stream(n, d, exponent):
    x, _, _, _, wn = _inputs(n, d, "first", "f", "f", "f")
    x = np.ldexp(x, exponent).astype(np.float32)
    rn = oi.norm_block(*_f64(x, None, None, None, wn), ALPHA, 0.0)[3].astype(np.float32)
    dy = _q(np.random.default_rng(d).standard_normal((n, d)), "f")
    dx, dw = torch.empty(n, d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
    api.sl_norm_block_grad(None, _cuda(dy), _cuda(x), None, None, None, _cuda(wn), None, _cuda(rn), n, d, ALPHA, dx, None, None, None, dw, False, ws)
    f = _f64(None, dy, x, None, None, None, wn, None, rn)
    want, mags = oi.norm_block_grad(*f, ALPHA), _bounds(*f, ALPHA)
    assert np.all(np.abs(dx.cpu().numpy() - want["dx"]) <= 160 * U * mags["dx"])
    assert np.all(np.abs(dw.cpu().numpy() - want["dw_pre"]) <= (n + 160) * U * mags["dw_pre"])

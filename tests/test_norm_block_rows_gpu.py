"""sl_norm_block / sl_norm_block_grad: what lies beside a row is not part of it.  Rows whose width is no multiple of 8 are read
by vectors that also hold elements of the rows beside them, of the gap between rows, or of what lies behind the array.  All
comparisons are bit for bit: the same row with other neighbours goes through the same operations."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api
from test_norm_block_gpu import ALPHA, DT, EPS, TYPES, U, _bounds, _check_forward, _cuda, _f64, _half_ulp, _inputs, _q

pytestmark = pytest.mark.gpu
NAN = float("nan")


def _beside(a, t, gap, fill):
    """the array as rows that lie `gap` elements apart, with `fill` between them"""
    n, d = a.shape
    w = torch.full((n, d + gap), fill, dtype=DT[t], device="cuda")
    w[:, :d] = torch.from_numpy(a).cuda()
    return w[:, :d]


def _both(x, b, g, wp, wn, res, act, gap=0, fill=0.0):
    """outputs of the forward call and of the gradient (of dh = h, dy = y), as numpy arrays"""
    n, d = x.shape
    db_, dg_ = _beside(b, act, gap, fill), _beside(g, act, gap, fill)
    h, y = torch.empty(n, d, dtype=DT[res], device="cuda"), torch.empty(n, d, dtype=DT[act], device="cuda")
    rp, rn = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    w = _cuda(wp), _cuda(wn)
    api.sl_norm_block(_cuda(x, res), db_, dg_, *w, n, d, ALPHA, EPS, h, y, rp, rn)
    dx, db, dg = torch.empty_like(h), _beside(b, act, gap, fill), _beside(b, act, gap, fill)
    dw = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
    api.sl_norm_block_grad(h, y, h, db_, dg_, *w, rp, rn, n, d, ALPHA, dx, db, dg, *dw, False, ws)
    rows = dict(h=h, y=y, rp=rp, rn=rn, dx=dx, db=db, dg=dg)
    return {k: t.float().cpu().numpy() for k, t in rows.items()}, [t.cpu().numpy() for t in dw]


@pytest.mark.parametrize("d", [33, 1001, 5001])           # lanes of a warp, a CTA, a cluster to a row
@pytest.mark.parametrize("res,act", TYPES)
@pytest.mark.parametrize("bad", [NAN, np.inf, -np.inf])
def test_a_gate_that_is_not_finite_stays_in_its_row(d, res, act, bad):
    n = 300
    x, b, g, wp, wn = _inputs(n, d, "all", res, act, "f")
    good, _ = _both(x, b, g, wp, wn, res, act)
    g = g.copy()
    g[7, 0], g[150, d - 1], g[151] = bad, bad, bad
    got, _ = _both(x, b, g, wp, wn, res, act)
    keep = np.setdiff1d(np.arange(n), [7, 150, 151])
    for k in good:
        assert np.array_equal(good[k][keep], got[k][keep]), k
    assert np.isnan(got["y"][7]).all() == np.isnan(bad)


@pytest.mark.parametrize("d,gap", [(33, 8), (1001, 8), (5001, 16), (12, 8)])
@pytest.mark.parametrize("res,act", TYPES)
def test_what_lies_between_rows_does_not_count(d, gap, res, act):
    a = _inputs(50, d, "all", res, act, "f")
    (one, w1), (two, w2) = _both(*a, res, act, gap, 0.0), _both(*a, res, act, gap, NAN)
    for k in one:
        assert np.isfinite(two[k]).all() and np.array_equal(one[k], two[k]), k
    assert all(np.array_equal(p, q) for p, q in zip(w1, w2))


@pytest.mark.parametrize("n,d", [(2, 1), (3, 1), (9, 1), (4, 2), (5, 3), (3, 4), (7, 5), (9, 6), (2, 7), (40, 3)])
@pytest.mark.parametrize("res,act", TYPES)
def test_narrow_rows(n, d, res, act):
    """rows narrower than a vector against the checker; the arrays end where their last row does, with NaN behind them"""
    x, b, g, wp, wn = _inputs(n, d, "all", res, act, "f")

    def tight(a, t):
        w = torch.full((n * d + 64,), NAN, dtype=DT[t], device="cuda")
        w[:n * d] = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().reshape(-1)
        return w[:n * d].view(n, d)
    h, y = tight(np.zeros((n, d)), res), tight(np.zeros((n, d)), act)
    rp, rn = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    ins = [tight(x, res), tight(b, act), tight(g, act), _cuda(wp), _cuda(wn)]
    api.sl_norm_block(*ins, n, d, ALPHA, EPS, h, y, rp, rn)
    _check_forward([t.float().cpu().numpy() for t in (h, y, rp, rn)], x, b, g, wp, wn, res, act)
    r = np.random.default_rng(n)
    dh, dy = _q(r.standard_normal((n, d)), res), _q(r.standard_normal((n, d)), act)
    outs = dict(dx=tight(dh, res), db=tight(dh, act), dg=tight(dh, act), dw_post=torch.empty(d, device="cuda"), dw_pre=torch.empty(d, device="cuda"))
    ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
    api.sl_norm_block_grad(tight(dh, res), tight(dy, act), h, *ins[1:], rp, rn, n, d, ALPHA, *outs.values(), False, ws)
    f = _f64(dh, dy, h.float().cpu().numpy(), b, g, wp, wn, rp.cpu().numpy(), rn.cpu().numpy())
    want, mags = oi.norm_block_grad(*f, float(np.float32(ALPHA))), _bounds(*f, ALPHA)
    gate = 2.4 * np.abs(f[4])
    for k, t in outs.items():                              # the bounds of the wider shapes
        steps = n + 160 + gate.max() if k.startswith("dw") else 160 + np.maximum(gate, np.max(gate, 1, keepdims=True))
        tol = steps * U * mags[k] + (0.0 if k.startswith("dw") else _half_ulp(want[k], res if k == "dx" else act))
        assert np.all(np.abs(t.float().cpu().numpy() - want[k]) <= tol + 1e-37), k

"""Arrays that start off the grid of vectors, each by itself and all together: sl_norm_block, its gradient and sl_embed_grad against the
64-bit checker, with the bounds of arrays on the grid."""
import numpy as np
import pytest
import torch

from oracle import inner as oi
from paper_2601_02360_b200 import api
from test_norm_block_gpu import ALPHA, DT, EPS, TYPES, U, _bounds, _check_forward, _cuda, _f64, _half_ulp, _inputs, _q

pytestmark = pytest.mark.gpu


def _place(a, t, shift, fill=float("nan")):
    """a copy that starts `shift` elements behind a boundary, with `fill` around it"""
    a = np.ascontiguousarray(a, dtype=np.float32)
    w = torch.full((a.size + 32,), fill, dtype=DT[t], device="cuda")
    w[shift:shift + a.size] = torch.from_numpy(a).cuda().reshape(-1)
    return w, w[shift:shift + a.size].view(a.shape)


def _untouched(w, shift, size):
    return bool(torch.isnan(w[:shift]).all()) and bool(torch.isnan(w[shift + size:]).all())


@pytest.mark.parametrize("n,d", [(7, 40), (5, 33), (20, 264), (6, 1001), (4, 5120)])
@pytest.mark.parametrize("res,act", TYPES)
def test_norm_block(n, d, res, act):
    x, b, g, wp, wn = _inputs(n, d, "all", res, act, "f")
    r = np.random.default_rng(n + d)
    h64, _, rp64, rn64 = oi.norm_block(*_f64(x, b, g, wp, wn), ALPHA, EPS)
    hq, rp32, rn32 = _q(h64, res), rp64.astype(np.float32), rn64.astype(np.float32)
    dh, dy = _q(r.standard_normal((n, d)), res), _q(r.standard_normal((n, d)), act)
    f = _f64(dh, dy, hq, b, g, wp, wn, rp32, rn32)
    want, mags = oi.norm_block_grad(*f, float(np.float32(ALPHA))), _bounds(*f, ALPHA)
    gate = 2.4 * np.abs(f[4])
    zero = np.zeros((n, d), np.float32)
    for which in (*range(5), "all"):                       # x, b, g, h, y of the forward call
        s = [(1 + i if which == "all" else 1) if which in (i, "all") else 0 for i in range(5)]
        (_, px), (_, pb), (_, pg) = _place(x, res, s[0]), _place(b, act, s[1]), _place(g, act, s[2])
        (wh, ph), (wy, py) = _place(zero, res, s[3]), _place(zero, act, s[4])
        rp, rn = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
        api.sl_norm_block(px, pb, pg, _place(wp, "f", 1)[1], _place(wn, "f", 3)[1], n, d, ALPHA, EPS, ph, py, rp, rn)
        _check_forward([t.float().cpu().numpy() for t in (ph, py, rp, rn)], x, b, g, wp, wn, res, act)
        assert _untouched(wh, s[3], n * d) and _untouched(wy, s[4], n * d)
    for which in (*range(8), "all"):                       # dh, dy, h, b, g, dx, db, dg of the gradient
        s = [(1 + i % 7 if which == "all" else 1) if which in (i, "all") else 0 for i in range(8)]
        ins = [_place(a, t, k)[1] for a, t, k in zip((dh, dy, hq, b, g), (res, act, res, act, act), s)]
        outs = [_place(zero, t, k) for t, k in zip((res, act, act), s[5:])]
        dw = [torch.empty(d, device="cuda") for _ in range(2)]
        ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device="cuda")
        api.sl_norm_block_grad(*ins, _cuda(wp), _cuda(wn), _cuda(rp32), _cuda(rn32), n, d, ALPHA, *(o[1] for o in outs), *dw, False, ws)
        for k, t in zip(("dx", "db", "dg", "dw_post", "dw_pre"), [o[1] for o in outs] + dw):
            steps = n + 160 + gate.max() if k.startswith("dw") else 160 + np.maximum(gate, np.max(gate, 1, keepdims=True))
            tol = steps * U * mags[k] + (0.0 if k.startswith("dw") else _half_ulp(want[k], res if k == "dx" else act))
            assert np.all(np.abs(t.float().cpu().numpy() - want[k]) <= tol + 1e-37), (which, k)
        assert all(_untouched(o[0], k, n * d) for o, k in zip(outs, s[5:]))


@pytest.mark.parametrize("n,L,V,d", [(300, 3, 40, 72), (5000, 333, 300, 64), (3000, 2, 5, 40)])
@pytest.mark.parametrize("dx,dt", [("f", "f"), ("b", "f"), ("b", "b")])
@pytest.mark.parametrize("acc", [False, True])
def test_embed_grad(n, L, V, d, dx, dt, acc):
    r = np.random.default_rng(n + V)
    ids = np.where(r.random(n) < 0.5, V // 2, r.integers(0, V, n)).astype(np.int32)        # one id with half of the tokens
    g, oldT, oldp = _q(r.standard_normal((n, d)), dx), _q(r.standard_normal((V, d)), dt), _q(r.standard_normal((L, d)), dt)
    want, wpos, mag, pmag = oi.embed_grad(ids, g, 0.3, L, V, True)
    if acc:
        want, mag, wpos, pmag = want + oldT, mag + np.abs(oldT), wpos + oldp, pmag + np.abs(oldp)
    count = np.bincount(ids, minlength=V)[:, None]
    d_ids = torch.cat([torch.zeros(1, dtype=torch.int32), torch.from_numpy(ids)]).cuda()[1:]
    ws = torch.empty(api.sl_embed_grad_workspace(n, V, d), dtype=torch.uint8, device="cuda")
    for s in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (3, 5, 7)):
        pX, (wT, dT), (wP, dpos) = _place(g, dx, s[0])[1], _place(oldT, dt, s[1]), _place(oldp, dt, s[2])
        api.sl_embed_grad(d_ids, pX, 0.3, n, L, V, d, dT, dpos, acc, ws)
        half = lambda a: 2.0 ** -8 * np.abs(a) if dt == "b" else 0  # noqa: E731
        assert np.all(np.abs(dT.float().cpu().numpy() - want) <= (count + 4) * U * mag + half(want))
        assert np.all(np.abs(dpos.float().cpu().numpy() - wpos) <= (n // L + 5) * U * pmag + half(wpos))
        assert _untouched(wT, s[1], V * d) and _untouched(wP, s[2], L * d)

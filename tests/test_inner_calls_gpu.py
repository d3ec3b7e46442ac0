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


def test_operands_of_another_shape_than_x():
    """the same rows in another shape give the same results, and every gradient has its tensor's shape"""
    B, L, d = 3, 5, 40
    g3 = [_randn(B, L, d, seed=i) for i in range(3)]
    w = [_randn(d, seed=7), _randn(d, seed=8)]
    wide = torch.cat([g3[1], g3[2]], -1)                  # b and g side by side

    def run(x, b, g, wp, wn):
        leaves = [t.detach().requires_grad_() for t in (x, b, g, wp, wn)]
        h, y = inner.norm_block(*leaves, 0.5)
        assert h.shape == x.shape and y.shape == x.shape
        grads = torch.autograd.grad((h * 2).sum() + (y * y).sum(), leaves)
        assert all(a.shape == t.shape for a, t in zip(grads, leaves))
        return [h, y, *grads]
    flat = lambda t: t.reshape(-1, d)  # noqa: E731
    want = run(*map(flat, g3), *w)
    for args in ((*g3, *w), (g3[0], flat(g3[1]), g3[2], *w), (flat(g3[0]), g3[1], flat(g3[2]), *w), (g3[0], wide[..., :d], wide[..., d:], *w),
                 (*g3, w[0].view(1, d), w[1].view(1, 1, d)), (g3[0].transpose(0, 1).contiguous().transpose(0, 1), *g3[1:], *w)):
        for a, b in zip(run(*args), want):
            assert torch.equal(a.reshape(b.shape), b)


def test_shapes_that_do_not_go_together_are_refused():
    n, d = 6, 24
    x, w = _randn(n, d), _randn(d, seed=1)
    for b in (_randn(n + 1, d), _randn(n - 1, d), _randn(1, d), _randn(d, n), _randn(n, 2 * d), _randn(n * d)):
        with pytest.raises(ValueError):
            inner.norm_block(x, b, None, w, w)
        with pytest.raises(ValueError):
            inner.norm_block(x, x.clone(), b, w, w)
    for bad in (_randn(2 * d), _randn(d - 1), _randn(d, 1), _randn(2, d)):
        with pytest.raises(ValueError):
            inner.norm_block(x, x.clone(), None, bad, w)
        with pytest.raises(ValueError):
            inner.norm_block(x, w_pre=bad)
    with pytest.raises(ValueError):
        inner.norm_block(torch.zeros((), device="cuda"), w_pre=w)
    ids = torch.arange(4, dtype=torch.int32, device="cuda")
    T = _randn(10, d)
    for tp in (_randn(11, d), _randn(20, d // 2), _randn(10, d + 1)):
        with pytest.raises(ValueError):
            inner.embed_lookup(ids, T, tp)
    for pos in (_randn(4, 2 * d), _randn(0, d), _randn(d), _randn(4, d - 1)):
        with pytest.raises(ValueError):
            inner.embed_lookup(ids, T, None, pos)
    assert torch.equal(inner.embed_lookup(ids[3], T), T[3])                   # one id without a dimension
    assert torch.equal(inner.embed_lookup(ids[3], T, None, T), T[3] + T[0])


@pytest.mark.parametrize("incoming", ["constant", "of the graph"])
@pytest.mark.parametrize("form", ["all", "first", "norm alone"])
def test_a_second_derivative_of_the_norm_block_is_an_error(form, incoming):
    n, d = 6, 40
    x, b, g, w = (_randn(*s, seed=i).requires_grad_() for i, s in enumerate([(n, d), (n, d), (n, d), (d,)]))
    up = torch.ones(n, d, device="cuda") if incoming == "constant" else x
    a = {"all": (x, b, g, w, w, 0.5), "first": (x, None, None, None, w), "norm alone": (x, b, None, w, None)}[form]

    def loss():
        return sum((t * up).sum() for t in inner.norm_block(*a) if t is not None)
    for leaf in (t for t in (x, b, w) if any(t is u for u in a)):
        if form == "norm alone" and leaf is x:
            continue                                      # h is linear in x
        first, = torch.autograd.grad(loss(), leaf, create_graph=True)
        with pytest.raises(RuntimeError, match="second derivative"):
            torch.autograd.grad((first ** 2).sum() + (leaf ** 2).sum(), leaf)
        with pytest.raises(RuntimeError, match="second derivative"):
            first.sum().backward()
    # a graph that is built and not used is no error, nor is one of other functions of the same tensors
    built, = torch.autograd.grad(loss() + (x ** 3).sum(), x, create_graph=True)
    plain, = torch.autograd.grad(loss() + (x ** 3).sum(), x)
    assert torch.equal(built, plain)
    two, = torch.autograd.grad((x ** 2).sum(), x, create_graph=True)
    assert torch.equal(torch.autograd.grad(two.sum(), x)[0], torch.full_like(x, 2.0))


def test_a_second_derivative_of_the_lookup():
    d = 40
    T, up = _randn(9, d, seed=5).requires_grad_(), _randn(6, d, seed=6).requires_grad_()
    ids = torch.arange(6, dtype=torch.int32, device="cuda")
    first, = torch.autograd.grad((inner.embed_lookup(ids, T) * up).sum(), T, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):              # the gradient is linear in what comes in
        torch.autograd.grad((first ** 2).sum(), up)
    first, = torch.autograd.grad(inner.embed_lookup(ids, T).sum(), T, create_graph=True)
    got, = torch.autograd.grad((first ** 2).sum() + (T ** 2).sum(), T)        # and does not depend on the table
    assert torch.equal(got, 2 * T)


def test_flags_of_the_norm_block_arrive_from_both_passes():
    # a row of several CTAs whose waits give up at once: nothing is left in flight, and the outputs are not to be used
    n, d = 64, 8192
    x, b, w = (_randn(*s, seed=i, dtype=torch.bfloat16).requires_grad_() for i, s in enumerate([(n, d), (n, d), (d,)]))
    forward, backward = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    try:
        api.sl_debug_set_wait_limit(-1)
        inner.norm_block(x, b, None, w, w, flags=forward)
        torch.cuda.synchronize()
        api.sl_debug_set_wait_limit(0)
        h, y = inner.norm_block(x, b, None, w, w, flags=backward)
        assert int(forward.item()) == api.SL_FLAG_TIMEOUT and int(backward.item()) == 0
        api.sl_debug_set_wait_limit(-1)
        (h.sum() + y.sum()).backward()
        torch.cuda.synchronize()
        assert int(backward.item()) == api.SL_FLAG_TIMEOUT
    finally:
        api.sl_debug_set_wait_limit(0)


class _OtherDevice:
    """The argument checks as they are when another device than that of the tensors is current."""

    def __init__(self, checks):
        self.checks = checks

    def __getattr__(self, name):
        return getattr(self.checks, name)

    def device(self):
        return torch.cuda.current_device() + 1


def test_tensors_of_another_device_are_refused(monkeypatch):
    n, d = 4, 8
    x, w, r = _randn(n, d), _randn(d), _randn(n)
    ids, ws = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    s8, lay = api.alloc_states8([0, 32]), api.Layout([0, 32])
    new = lambda: torch.empty(n, d, device="cuda")  # noqa: E731
    calls = [lambda: api.sl_adamw(new(), new(), new(), new(), lay, 1e-3, 0.9, 0.95, 1e-8, 1),
             lambda: api.sl_adamw8(new(), new(), *s8, lay, 1e-3, 0.9, 0.95, 1e-8, 1),
             lambda: api.sl_adamw8_pack(x, x.abs(), lay, *s8),
             lambda: api.sl_adamw8_unpack(*s8, lay, new(), new()),
             lambda: api.sl_embed_lookup(ids, x, None, None, 1.0, n, n, n, d, new()),
             lambda: api.sl_embed_grad(ids, x, 1.0, n, n, n, d, new(), None, False, ws),
             lambda: api.sl_norm_block(x, x, None, None, w, n, d, 1.0, 1e-6, new(), new()),
             lambda: api.sl_norm_block_grad(x, None, x, x, None, None, None, None, None, n, d, 1.0, new(), new(), None, None, None, False, ws)]
    for call in calls:
        call()
    checks = api._checks()
    assert checks.device() == torch.cuda.current_device()
    with pytest.raises(ValueError):
        checks.ptr(x, "x", 1, 1, checks.device() + 1)
    with pytest.raises(ValueError):
        checks.rows(x, "x", n, d, 1, checks.device() + 1)
    monkeypatch.setattr(api, "_args", _OtherDevice(checks))
    for call in calls:
        with pytest.raises(ValueError, match="current CUDA device"):
            call()


def test_no_tokens_and_no_elements():
    d, V, L = 24, 10, 4
    T, P, w = _randn(V, d).requires_grad_(), _randn(L, d, seed=1).requires_grad_(), _randn(d, seed=2).requires_grad_()
    ids = torch.zeros(0, 5, dtype=torch.int32, device="cuda")
    x = inner.embed_lookup(ids, T, T, P)
    assert x.shape == (0, 5, d)
    b = torch.zeros(0, 5, d, device="cuda", requires_grad=True)
    for form in ((x, b, b, w, w), (x, b, None, None, w), (x, b, None, w, None), (x, None, None, None, w)):
        h, y = inner.norm_block(*form)
        assert all(t is None or t.shape == x.shape for t in (h, y))
        loss = sum(t.sum() for t in (h, y) if t is not None)
        used = [T, P] + [t for t in (b, w) if any(t is u for u in form)]
        for t, g in zip(used, torch.autograd.grad(loss, used, retain_graph=True)):
            assert g.shape == t.shape and not g.any()
    for bits in (8, 32):
        opt = inner.AdamW(torch.zeros(0, device="cuda"), [0, 0], bits=bits)
        opt.step(torch.zeros(0, device="cuda"))
        assert opt.steps == 1 and all(t.numel() == 0 for t in opt.moments())
        opt.load_moments(*opt.moments(), 5)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_that_is_refused_does_not_count(bits):
    n = 600
    th, g = _randn(n), _randn(n, seed=1)
    one, two = (inner.AdamW(th.clone(), [0, n], bits=bits) for _ in range(2))
    for bad in (g[:-1], g.cpu(), g.double()):
        with pytest.raises(ValueError):
            one.step(bad)
    assert one.steps == 0
    for _ in range(2):
        one.step(g)
        two.step(g)
    assert one.steps == 2 and torch.equal(one.theta, two.theta)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_graph_of_the_old_parameters_is_refused_after_a_step(bits):
    d = 24
    theta, copy = torch.ones(d, device="cuda"), torch.ones(d, dtype=torch.bfloat16, device="cuda")
    opt = inner.AdamW(theta, [0, d], bits=bits, copy=copy)
    x = _randn(5, d)
    for w in (theta, copy):
        p = w.detach().requires_grad_()
        _, y = inner.norm_block(x, w_pre=p)
        y.sum().backward(retain_graph=True)
        opt.step(torch.ones(d, device="cuda"))
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


@pytest.mark.parametrize("bits", [8, 32])
def test_moments_of_another_size_are_refused(bits):
    n = 600
    opt = inner.AdamW(torch.zeros(n, device="cuda"), [0, n], bits=bits)
    opt.load_moments(_randn(n), _randn(n, seed=1).abs(), 7)
    before = [t.clone() for t in opt.states]
    for bad in (_randn(1), _randn(n + 1), _randn(n - 1)):
        for m, v in ((bad, _randn(n)), (_randn(n), bad.abs())):
            with pytest.raises(ValueError):
                opt.load_moments(m, v, 9)
    assert opt.steps == 7 and all(torch.equal(a, b) for a, b in zip(before, opt.states))

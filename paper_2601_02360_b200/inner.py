"""The inner step of a replica (Eq. 1) on torch tensors: autograd functions over the embedding lookup and the norm
block, and the AdamW step over an arena.  Marshalling only: every operation is one of the library's calls on the
current stream of its tensors' device; outputs and workspaces come from torch's allocator.

    x = embed_lookup(ids, T_S, T_perp, pos)                 # X^(0) of sections 2.3 / 2.4
    _, y = norm_block(x, None, None, None, w_in)            # norm before the first block
    x, y = norm_block(x, b, g, w_post, w_pre, alpha)        # after a block: norm, gate, residual, norm before the next
    opt = AdamW(theta, layout, bits=8)                      # theta: the arena the outer step works on
    opt.step(grad)                                          # grad: an arena of the same layout
"""
from __future__ import annotations

import functools
from typing import Optional, Sequence

import torch

from . import api


def _dense(t, *shape):
    """t without gaps (in another shape, if one is given); what is not needed is not done: on a tensor of a graph each operation
    costs a node, and 4 us a call."""
    if t is None:
        return None
    if shape and t.shape != shape:
        t = t.reshape(shape)
    if t.is_neg():
        t = t.resolve_neg()
    return t if t.is_contiguous() else t.contiguous()


class _Once(torch.autograd.Function):
    """Passes on gradients (behind the `k` tensors they depend on) into a graph that is being built: to differentiate them raises."""

    @staticmethod
    def forward(ctx, k, *tensors):
        return tensors[k:]

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("embed_lookup and norm_block have no second derivative: no graph records the kernels of their gradients")


def _once_differentiable(backward):
    """Gradients from kernels would be constants to a graph of the backward pass (create_graph=True), and whatever passes through
    them would be lost without an error.  They depend on the incoming gradients and on every saved tensor."""
    @functools.wraps(backward)
    def run(ctx, *grads):
        with torch.no_grad():
            out = backward(ctx, *grads)
        if not torch.is_grad_enabled():
            return out
        depend = [t for t in (*grads, *ctx.saved_tensors) if t is not None and t.requires_grad]
        given = iter(_Once.apply(len(depend), *depend, *(t for t in out if t is not None)))
        return tuple(None if t is None else next(given) for t in out)
    return run


class _EmbedLookup(torch.autograd.Function):
    """Dense arguments: ids in any shape, tables [V, d], positions [L, d]."""

    @staticmethod
    def forward(ctx, ids, T_S, T_perp, pos, L, scale, flags, out_dtype):
        V, d = T_S.shape
        n = ids.numel()
        X = torch.empty(n, d, dtype=out_dtype or T_S.dtype, device=T_S.device)
        with torch.cuda.device_of(T_S):
            api.sl_embed_lookup(ids, T_S, T_perp, pos, scale, n, L, V, d, X, flags)
        ctx.save_for_backward(ids)
        ctx.sizes = (n, L, V, d, scale, T_S.dtype, flags)
        return X.view(*ids.shape, d)

    @staticmethod
    @_once_differentiable
    def backward(ctx, dX):
        (ids,) = ctx.saved_tensors
        n, L, V, d, scale, dtype, flags = ctx.sizes
        need_s, need_p, need_pos = ctx.needs_input_grad[1:4]
        dT = torch.empty(V, d, dtype=dtype, device=dX.device)
        dpos = torch.empty(L, d, dtype=dtype, device=dX.device) if need_pos else None
        ws = torch.empty(api.sl_embed_grad_workspace(n, V, d), dtype=torch.uint8, device=dX.device)
        with torch.cuda.device_of(ids):
            api.sl_embed_grad(ids, _dense(dX), scale, n, L, V, d, dT, dpos, False, ws, flags)
        return None, (dT if need_s else None), (dT if need_p else None), dpos, None, None, None, None


def embed_lookup(ids, T_S, T_perp=None, pos=None, scale: float = 1.0, flags=None, out_dtype=None):
    """scale (T_S[ids] + T_perp[ids]) + pos[t mod L] for int32 ids of any shape, [..., d]; token t is the t-th of the
    flattened ids, L the rows of pos.  Differentiable in T_S, T_perp and pos; a second derivative raises RuntimeError."""
    if T_S.dim() != 2 or (T_perp is not None and T_perp.shape != T_S.shape):
        raise ValueError(f"T_S, T_perp: expected matrices of one shape, got {[list(t.shape) for t in (T_S, T_perp) if t is not None]}")
    if pos is not None and (pos.dim() != 2 or pos.shape[0] < 1 or pos.shape[1] != T_S.shape[1]):
        raise ValueError(f"pos: expected rows of {T_S.shape[1]}, got {list(pos.shape)}")
    L = pos.shape[0] if pos is not None else 1
    return _EmbedLookup.apply(_dense(ids), _dense(T_S), _dense(T_perp), _dense(pos), L, float(scale), flags, out_dtype)


class _NormBlock(torch.autograd.Function):
    """x dense [n, d]; b and g rows of d, evenly spaced; weights dense [d]."""

    @staticmethod
    def forward(ctx, x, b, g, w_post, w_pre, alpha, eps, flags):
        n, d = x.shape
        act = (b if b is not None else x).dtype
        h = torch.empty_like(x) if b is not None else None
        y = torch.empty(n, d, dtype=act, device=x.device) if w_pre is not None else None
        stat = lambda w: None if w is None else torch.empty(n, dtype=torch.float32, device=x.device)  # noqa: E731
        r_post, r_pre = stat(w_post), stat(w_pre)
        with torch.cuda.device_of(x):
            api.sl_norm_block(x, b, g, w_post, w_pre, n, d, alpha, eps, h, y, r_post, r_pre, flags)
        ctx.save_for_backward(h if h is not None else x, b, g, w_post, w_pre, r_post, r_pre)
        ctx.args = (n, d, alpha, flags)
        ctx.set_materialize_grads(False)
        return h, y

    @staticmethod
    @_once_differentiable
    def backward(ctx, dh, dy):
        h, b, g, w_post, w_pre, r_post, r_pre = ctx.saved_tensors
        n, d, alpha, flags = ctx.args
        if dh is None and dy is None:
            return (None,) * 8
        dh, dy = _dense(dh), _dense(dy)
        if dy is None:                    # nothing came back through the second norm
            zero_pre, w_pre, r_pre = (None if w_pre is None else torch.zeros_like(w_pre)), None, None
        dx = torch.empty_like(h)
        like = lambda t: None if t is None else torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)  # noqa: E731
        db, dg = like(b), like(g)
        dw_post, dw_pre = like(w_post), like(w_pre)
        ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device=h.device)
        with torch.cuda.device_of(h):
            api.sl_norm_block_grad(dh, dy, h, b, g, w_post, w_pre, r_post, r_pre, n, d, alpha, dx, db, dg, dw_post, dw_pre, False, ws, flags)
        if dy is None:
            dw_pre = zero_pre
        return dx, db, dg, dw_post, dw_pre, None, None, None


def _rows(name: str, t, n: int, d: int):
    """t as n dense rows of d; columns of a wider matrix stay where they are."""
    if t is None:
        return None
    if t.shape[-1:] != (d,) or t.numel() != n * d:
        raise ValueError(f"{name}: expected {n} rows of {d}, got {list(t.shape)}")
    v = t if t.dim() == 2 else t.reshape(n, d)
    return v if v.stride(1) == 1 and (n <= 1 or v.stride(0) >= d) and not v.is_neg() else _dense(v)


def _weight(name: str, w, d: int):
    if w is not None and (w.shape[-1:] != (d,) or w.numel() != d):
        raise ValueError(f"{name}: expected {d} elements, got {list(w.shape)}")
    return _dense(w, d)


def norm_block(x, b=None, g=None, w_post=None, w_pre=None, alpha: float = 1.0, eps: float = 1e-6, flags=None):
    """(h, y): h = x + alpha sigmoid(g) norm(b) w_post and y = norm(h) w_pre, each term left out where its tensor is
    None (no b: h is None and y = norm(x) w_pre; no w_pre: y is None).  x, b and g: rows of one width in any shape, as many of
    each; h and y have x's.  flags: int32 device word; SL_FLAG_TIMEOUT in it, from the forward or the backward pass, says that
    their results are not to be used.  Differentiable in every tensor; a second derivative raises RuntimeError."""
    d = x.shape[-1] if x.dim() else 0
    if d < 1:
        raise ValueError(f"x: expected rows, got {list(x.shape)}")
    n = x.numel() // d
    h, y = _NormBlock.apply(_dense(x, n, d), _rows("b", b, n, d), _rows("g", g, n, d), _weight("w_post", w_post, d),
                            _weight("w_pre", w_pre, d), float(alpha), float(eps), flags)
    if x.dim() == 2:
        return h, y
    return (None if h is None else h.view(x.shape)), (None if y is None else y.view(x.shape))


class AdamW:
    """InnerOpt of Eq. 1 over an arena: the tensors of `layout` back to back in `theta` (float32 or bfloat16), moments
    in 32 bits or in 8 (`bits`), weight decay per tensor.  `copy`: optional bfloat16 arena that always holds theta
    rounded.  The moments persist; the step count starts at 0."""

    def __init__(self, theta: torch.Tensor, layout, lr: float = 3e-4, betas: Sequence[float] = (0.9, 0.95), eps: float = 1e-8,
                 decay: Optional[Sequence[float]] = None, bits: int = 32, copy: Optional[torch.Tensor] = None):
        if bits not in (8, 32):
            raise ValueError(f"bits: expected 8 or 32, got {bits}")
        self.theta, self.layout, self.copy, self.bits = theta, api._layout(layout), copy, bits
        self.lr, self.betas, self.eps, self.decay, self.steps = lr, tuple(betas), eps, decay, 0
        n = self.layout.n_total
        self.states = api.alloc_states8(self.layout, theta.device) if bits == 8 else \
            tuple(torch.zeros(n, dtype=torch.float32, device=theta.device) for _ in range(2))
        self.flags = torch.zeros(1, dtype=torch.int32, device=theta.device)

    def step(self, grad: torch.Tensor, grad_scale: Optional[torch.Tensor] = None, stream=None) -> None:
        """One step from the gradient arena `grad`; `grad_scale` (a device scalar, float32) multiplies it first: a clipping
        coefficient costs no synchronisation.  If it is not finite the device skips the step and raises SL_FLAG_NONFINITE
        in `flags`; the step count goes on."""
        call = api.sl_adamw8 if self.bits == 8 else api.sl_adamw
        with torch.cuda.device_of(self.theta):
            call(self.theta, grad, *self.states, self.layout, self.lr, *self.betas, self.eps, self.steps + 1, decay=self.decay,
                 grad_scale=grad_scale, copy=self.copy, flags=self.flags, stream=stream)
        # as torch's in-place operations do: a graph that saved these parameters may not be used with the new ones
        torch.autograd.graph.increment_version(self.theta)
        if self.copy is not None:
            torch.autograd.graph.increment_version(self.copy)
        self.steps += 1                                   # a step that was refused does not count

    def moments(self):
        """(m, v) as float32: the moments themselves, or the values that their codes stand for."""
        if self.bits == 32:
            return self.states
        m, v = (torch.empty(self.layout.n_total, dtype=torch.float32, device=self.theta.device) for _ in range(2))
        with torch.cuda.device_of(self.theta):
            api.sl_adamw8_unpack(*self.states, self.layout, m, v)
        return m, v

    def load_moments(self, m: torch.Tensor, v: torch.Tensor, steps: int) -> None:
        """Takes over float32 moments (of either form: an optimiser can change its form between two steps)."""
        for name, t in (("m", m), ("v", v)):
            if t.numel() != self.layout.n_total:
                raise ValueError(f"{name}: expected {self.layout.n_total} elements, got {list(t.shape)}")
        if self.bits == 32:
            self.states[0].copy_(m)
            self.states[1].copy_(v)
        else:
            with torch.cuda.device_of(self.theta):
                api.sl_adamw8_pack(m, v, self.layout, *self.states)
        self.steps = steps

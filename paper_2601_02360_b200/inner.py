"""The inner step of a replica (Eq. 1) on torch tensors: autograd functions over the embedding lookup and the norm
block, and the AdamW step over an arena.  Marshalling only: every operation is one of the library's calls on the
current stream; outputs and workspaces come from torch's allocator.

    x = embed_lookup(ids, T_S, T_perp, pos)                 # X^(0) of sections 2.3 / 2.4
    _, y = norm_block(x, None, None, None, w_in)            # norm before the first block
    x, y = norm_block(x, b, g, w_post, w_pre, alpha)        # after a block: norm, gate, residual, norm before the next
    opt = AdamW(theta, layout, bits=8)                      # theta: the arena the outer step works on
    opt.step(grad)                                          # grad: an arena of the same layout
"""
from __future__ import annotations

from typing import Optional, Sequence

import torch

from . import api


def _dense(t):
    return None if t is None else t.resolve_neg().contiguous()


class _EmbedLookup(torch.autograd.Function):
    @staticmethod
    def forward(ctx, ids, T_S, T_perp, pos, scale, flags, out_dtype):
        V, d = T_S.shape
        n, L = ids.numel(), (pos.shape[0] if pos is not None else max(1, ids.shape[-1]))
        X = torch.empty(n, d, dtype=out_dtype or T_S.dtype, device=T_S.device)
        ids = _dense(ids)
        api.sl_embed_lookup(ids, _dense(T_S), _dense(T_perp), _dense(pos), scale, n, L, V, d, X, flags)
        ctx.save_for_backward(ids)
        ctx.sizes = (n, L, V, d, scale, T_S.dtype, flags)
        return X.view(*ids.shape, d)

    @staticmethod
    def backward(ctx, dX):
        (ids,) = ctx.saved_tensors
        n, L, V, d, scale, dtype, flags = ctx.sizes
        need_s, need_p, need_pos = ctx.needs_input_grad[1:4]
        dT = torch.empty(V, d, dtype=dtype, device=dX.device)
        dpos = torch.empty(L, d, dtype=dtype, device=dX.device) if need_pos else None
        ws = torch.empty(api.sl_embed_grad_workspace(n, V, d), dtype=torch.uint8, device=dX.device)
        api.sl_embed_grad(ids, _dense(dX), scale, n, L, V, d, dT, dpos, False, ws, flags)
        return None, (dT if need_s else None), (dT if need_p else None), dpos, None, None, None


def embed_lookup(ids, T_S, T_perp=None, pos=None, scale: float = 1.0, flags=None, out_dtype=None):
    """scale (T_S[ids] + T_perp[ids]) + pos[t mod L] for int32 ids of any shape, [..., d]; token t is the t-th of the
    flattened ids, L the rows of pos.  Differentiable in T_S, T_perp and pos."""
    return _EmbedLookup.apply(ids, T_S, T_perp, pos, float(scale), flags, out_dtype)


class _NormBlock(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, b, g, w_post, w_pre, alpha, eps):
        d = x.shape[-1]
        n = x.numel() // d
        x2 = _dense(x.reshape(n, d))
        rows = lambda t: None if t is None else _rows(t, n, d)  # noqa: E731
        b2, g2 = rows(b), rows(g)
        act = (b2 if b2 is not None else x2).dtype
        h = torch.empty_like(x2) if b2 is not None else None
        y = torch.empty(n, d, dtype=act, device=x.device) if w_pre is not None else None
        stat = lambda w: None if w is None else torch.empty(n, dtype=torch.float32, device=x.device)  # noqa: E731
        r_post, r_pre = stat(w_post), stat(w_pre)
        api.sl_norm_block(x2, b2, g2, _dense(w_post), _dense(w_pre), n, d, alpha, eps, h, y, r_post, r_pre)
        ctx.save_for_backward(h if h is not None else x2, b2, g2, w_post, w_pre, r_post, r_pre)
        ctx.args = (n, d, alpha, x.shape)
        ctx.set_materialize_grads(False)
        return (None if h is None else h.view(x.shape)), (None if y is None else y.view(x.shape))

    @staticmethod
    def backward(ctx, dh, dy):
        h, b, g, w_post, w_pre, r_post, r_pre = ctx.saved_tensors
        n, d, alpha, shape = ctx.args
        if dh is None and dy is None:
            return (None,) * 7
        dh, dy = (None if t is None else _dense(t.reshape(n, d)) for t in (dh, dy))
        if dy is None:                    # nothing came back through the second norm
            zero_pre, w_pre, r_pre = (None if w_pre is None else torch.zeros_like(w_pre)), None, None
        dx = torch.empty_like(h)
        like = lambda t: None if t is None else torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=t.device)  # noqa: E731
        db, dg = like(b), like(g)
        dw_post = None if w_post is None else torch.empty(d, dtype=w_post.dtype, device=h.device)
        dw_pre = None if w_pre is None else torch.empty(d, dtype=w_pre.dtype, device=h.device)
        ws = torch.empty(api.sl_norm_block_grad_workspace(n, d), dtype=torch.uint8, device=h.device)
        api.sl_norm_block_grad(dh, dy, h, b, g, _dense(w_post), _dense(w_pre), r_post, r_pre, n, d, alpha, dx, db, dg, dw_post, dw_pre, False,
                               ws)
        if dy is None:
            dw_pre = zero_pre
        back = lambda t: None if t is None else t.reshape(shape)  # noqa: E731
        return back(dx), back(db), back(dg), dw_post, dw_pre, None, None


def _rows(t, n: int, d: int):
    """t as n dense rows of d; columns of a wider matrix stay where they are."""
    t = t.resolve_neg()
    v = t.view(n, d) if t.dim() != 2 and t.is_contiguous() else t
    return v if v.dim() == 2 and v.stride(1) == 1 and (n <= 1 or v.stride(0) >= d) else t.reshape(n, d).contiguous()


def norm_block(x, b=None, g=None, w_post=None, w_pre=None, alpha: float = 1.0, eps: float = 1e-6):
    """(h, y): h = x + alpha sigmoid(g) norm(b) w_post and y = norm(h) w_pre, each term left out where its tensor is
    None (no b: h is None and y = norm(x) w_pre; no w_pre: y is None).  Differentiable in every tensor."""
    return _NormBlock.apply(x, b, g, w_post, w_pre, float(alpha), float(eps))


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
        self.steps += 1
        call = api.sl_adamw8 if self.bits == 8 else api.sl_adamw
        call(self.theta, grad, *self.states, self.layout, self.lr, *self.betas, self.eps, self.steps, decay=self.decay,
             grad_scale=grad_scale, copy=self.copy, flags=self.flags, stream=stream)

    def moments(self):
        """(m, v) as float32: the moments themselves, or the values that their codes stand for."""
        if self.bits == 32:
            return self.states
        m, v = (torch.empty(self.layout.n_total, dtype=torch.float32, device=self.theta.device) for _ in range(2))
        api.sl_adamw8_unpack(*self.states, self.layout, m, v)
        return m, v

    def load_moments(self, m: torch.Tensor, v: torch.Tensor, steps: int) -> None:
        """Takes over float32 moments (of either form: an optimiser can change its form between two steps)."""
        if self.bits == 32:
            self.states[0].copy_(m)
            self.states[1].copy_(v)
        else:
            api.sl_adamw8_pack(m, v, self.layout, *self.states)
        self.steps = steps

"""Heterogeneous pre-training in small: R replicas of a language model on one GPU, H inner AdamW steps each (Eq. 1),
then the outer SparseLoCo step (Eq. 2) and the embedding re-projection (Eqs. 3-4), round after round.

    python examples/train_replicas.py [--rounds 4] [--inner 20] [--bits 8] [--bf16]

The model: X^(0) = T_S[x] + T_perp[x] + pos, blocks of a gated MLP between norms, the scores against T_S + T_perp.
Embedding, norms, gates, residuals, their gradients and both optimisers run in the library's kernels; the dense
products and the loss are torch's.  The data is a fixed random Markov chain, so that there is something to learn.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2601_02360_b200 import api, build, inner  # noqa: E402


class Arena:
    """The tensors of a model back to back, as the outer step wants them; every tensor is a leaf whose gradient is a
    view of the gradient arena."""

    def __init__(self, shapes, device="cuda", dtype=torch.float32):
        self.shapes, offsets = shapes, [0]
        for _, shape in shapes:
            offsets.append(offsets[-1] + int(torch.Size(shape).numel()))
        self.layout = api.Layout(offsets)
        self.theta = torch.zeros(offsets[-1], dtype=dtype, device=device)
        self.grad = torch.zeros_like(self.theta)
        self.p = {}
        for (name, shape), o in zip(shapes, offsets):
            n = int(torch.Size(shape).numel())
            p = self.theta[o:o + n].view(shape).detach().requires_grad_()
            p.grad = self.grad[o:o + n].view(shape)
            self.p[name] = p


def shapes_of(V, d, ffn, layers):
    out = [("T_S", (V, d)), ("w_in", (d,))]
    for i in range(layers):
        out += [(f"up{i}", (d, 2 * ffn)), (f"down{i}", (ffn, 2 * d)), (f"post{i}", (d,)), (f"pre{i}", (d,))]
    return out


def init(arena, gen):
    for name, shape in arena.shapes:
        p = arena.p[name]
        with torch.no_grad():
            if len(shape) == 1:
                p.fill_(1.0)
            else:
                p.copy_(torch.randn(*shape, generator=gen, device=p.device) * (0.02 if name == "T_S" else shape[0] ** -0.5))


def loss_of(p, T_perp, pos, tokens, layers, ffn, alpha, flags):
    """Mean cross entropy of the next token; tokens: int32 [sequences, L + 1]."""
    ids, target = tokens[:, :-1].contiguous(), tokens[:, 1:].reshape(-1).long()
    d = T_perp.shape[1]
    x = inner.embed_lookup(ids, p["T_S"], T_perp, pos, scale=d ** 0.5, flags=flags).reshape(-1, d)
    _, y = inner.norm_block(x, w_pre=p["w_in"], flags=flags)
    for i in range(layers):
        a, u = (y @ p[f"up{i}"]).split(ffn, dim=1)
        wide = (F.silu(a) * u) @ p[f"down{i}"]               # the block's output and its gate, side by side
        x, y = inner.norm_block(x, wide[:, :d], wide[:, d:], p[f"post{i}"], p[f"pre{i}"], alpha, flags=flags)
    scores = (y @ (p["T_S"] + T_perp).t()).float()
    return F.cross_entropy(scores, target)


def clip(grad, most=1.0):
    """The factor that keeps the gradient's norm at `most`, on the device; NaN (which skips the step) if the norm is not finite."""
    norm = torch.linalg.vector_norm(grad.float())
    return torch.where(torch.isfinite(norm), (most / norm.clamp_min(most)), torch.nan).reshape(1)


def run(rounds=4, inner_steps=20, R=2, V=512, d=64, ffn=128, layers=2, L=32, batch=64, bits=8, bf16=False, lr=1e-2, k_sub=16, seed=0,
        report=print):
    """Trains and returns the mean loss of every inner step."""
    build.build()
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = torch.bfloat16 if bf16 else torch.float32
    chain = torch.randn(V, 8, generator=gen, device="cuda").argsort(1)     # what may follow a token: eight others
    follow = (torch.randint(0, V, (V, 8), generator=gen, device="cuda"))
    shared = Arena(shapes_of(V, d, ffn, layers), dtype=dtype)
    init(shared, gen)
    replicas = [Arena(shared.shapes, dtype=dtype) for _ in range(R)]
    U = torch.linalg.qr(torch.randn(d, k_sub, generator=gen, device="cuda"))[0].contiguous()
    api.sl_round_tf32(U, U.numel())
    T_perp = torch.zeros(V, d, dtype=dtype, device="cuda")
    pos = (torch.randn(L, d, generator=gen, device="cuda") * 0.02).to(dtype)
    decay = [0.1 if len(s) == 2 else 0.0 for _, s in shared.shapes]
    opts = [inner.AdamW(a.theta, a.layout, lr=lr, decay=decay, bits=bits) for a in replicas]
    err = [torch.zeros(shared.theta.numel(), dtype=torch.float32, device="cuda") for _ in range(R)]
    messages = api.alloc_messages(shared.layout, 4096, 64, 2, R)
    flags = torch.zeros(1, dtype=torch.int32, device="cuda")
    outer = api.sl_outer_step_bf16 if bf16 else api.sl_outer_step
    losses = []
    for t in range(rounds):
        for a in replicas:
            a.theta.copy_(shared.theta)                        # every replica starts from the shared parameters
        for s in range(inner_steps):
            mean = 0.0
            for a, opt in zip(replicas, opts):
                seq = [torch.randint(0, V, (batch,), generator=gen, device="cuda")]
                for _ in range(L):
                    pick = torch.randint(0, 8, (batch,), generator=gen, device="cuda")
                    seq.append(follow[seq[-1], chain[seq[-1], pick]])
                tokens = torch.stack(seq, 1).to(torch.int32)
                a.grad.zero_()
                loss = loss_of(a.p, T_perp, pos, tokens, layers, ffn, 0.5, flags)
                loss.backward()
                opt.step(a.grad, clip(a.grad))
                mean += loss.item() / R
            losses.append(mean)
        outer([a.theta for a in replicas], shared.theta, err, shared.layout, 0.95, 4096, 64, 2, 1.0, *messages, flags)
        if not bf16:                                           # T_S back into the subspace, the rest into T_perp
            api.sl_embed_reproject(shared.p["T_S"].detach(), T_perp, U, V, d, k_sub, flags)
        report(f"round {t}: loss {losses[-inner_steps]:.3f} -> {losses[-1]:.3f}")
    assert int(flags.item()) == 0 and all(int(o.flags.item()) == 0 for o in opts)
    return losses


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--rounds", type=int, default=4)
    ap.add_argument("--inner", type=int, default=20)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    ap.add_argument("--bf16", action="store_true")
    o = ap.parse_args()
    run(rounds=o.rounds, inner_steps=o.inner, bits=o.bits, bf16=o.bf16)

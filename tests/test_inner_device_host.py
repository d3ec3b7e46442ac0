"""Every library call of the Python forms runs on the device of its tensors.  Without a GPU: the calls and the device guard are
replaced by records of what was called under which guard."""
import torch

from paper_2601_02360_b200 import api, inner


class _Guard:
    active = []

    def __init__(self, t):
        assert isinstance(t, torch.Tensor)
        self.t = t

    def __enter__(self):
        _Guard.active.append(self.t)

    def __exit__(self, *_):
        _Guard.active.pop()


def test_every_call_is_made_under_the_guard(monkeypatch):
    seen = []

    def record(name, result=None):
        def call(*args, **kw):
            assert _Guard.active, name
            seen.append(name)
            return result
        monkeypatch.setattr(api, name, call)
    for name in ("sl_embed_lookup", "sl_embed_grad", "sl_norm_block", "sl_norm_block_grad", "sl_adamw", "sl_adamw8", "sl_adamw8_pack",
                 "sl_adamw8_unpack"):
        record(name)
    monkeypatch.setattr(api, "sl_embed_grad_workspace", lambda *a: 16)
    monkeypatch.setattr(api, "sl_norm_block_grad_workspace", lambda *a: 16)
    monkeypatch.setattr(torch.cuda, "device_of", _Guard)
    monkeypatch.setattr(api, "alloc_states8", lambda layout, device: tuple(torch.zeros(8) for _ in range(4)))
    T, w = torch.zeros(5, 8, requires_grad=True), torch.ones(8, requires_grad=True)
    x = inner.embed_lookup(torch.zeros(3, dtype=torch.int32), T)
    h, y = inner.norm_block(x, x, None, w, w)
    (h.sum() + y.sum()).backward()
    for bits in (32, 8):
        opt = inner.AdamW(torch.zeros(8), [0, 8], bits=bits)
        opt.step(torch.zeros(8))
        opt.load_moments(*opt.moments(), 3)
    assert not _Guard.active
    assert seen == ["sl_embed_lookup", "sl_norm_block", "sl_norm_block_grad", "sl_embed_grad", "sl_adamw", "sl_adamw8", "sl_adamw8_unpack",
                    "sl_adamw8_pack"]

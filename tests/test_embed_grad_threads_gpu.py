"""sl_embed_grad from several host threads at once: vocabularies whose sorts want different amounts of shared memory."""
import threading

import pytest
import torch

from paper_2601_02360_b200 import api

pytestmark = pytest.mark.gpu


def test_calls_of_two_threads_do_not_meet():
    n, d, calls = 3000, 16, 2000
    gen = torch.Generator(device="cuda").manual_seed(1)

    def prepare(V):
        ids = torch.randint(0, V, (n,), generator=gen, device="cuda", dtype=torch.int32)
        dX = torch.randn(n, d, generator=gen, device="cuda")
        ws = torch.empty(api.sl_embed_grad_workspace(n, V, d), dtype=torch.uint8, device="cuda")
        dT = torch.empty(V, d, device="cuda")
        api.sl_embed_grad(ids, dX, 1.0, n, n, V, d, dT, None, False, ws)
        return ids, dX, ws, dT, dT.clone()

    def work(V, a, stream):
        try:
            for _ in range(calls):
                api.sl_embed_grad(a[0], a[1], 1.0, n, n, V, d, a[3], None, False, a[2], stream=stream)
        except Exception as e:  # noqa: BLE001
            failures.append((V, e))
    failures, sizes = [], (200, 131072)                   # one digit of 8 bits, two of 9
    sets = [prepare(V) for V in sizes]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    threads = [threading.Thread(target=work, args=(V, a, st)) for V, a, st in zip(sizes, sets, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failures
    assert all(torch.equal(a[3], a[4]) for a in sets)

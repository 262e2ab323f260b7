"""Calls of several host threads, each on a stream of its own: as one after
another."""
import threading

import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def test_threads_with_their_own_streams():
    def problem(i):
        g = torch.Generator(device=DEV).manual_seed(i)
        n, v, d = (5, 40, 300, 700)[i], 3000 + i, 200
        h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
        w = torch.randn(v, d, device=DEV, generator=g).bfloat16()
        t = torch.randint(-1, v, (n,), device=DEV, generator=g)
        u = torch.randn(100 + 100 * i, 500, device=DEV, generator=g)
        r = torch.rand(n, device=DEV, generator=g)
        return {"in": (h, w, t, r, u), "out": (torch.empty(n, device=DEV), torch.empty(n, device=DEV),
                                               torch.empty_like(h), torch.empty_like(w),
                                               torch.empty_like(u, dtype=torch.bfloat16))}

    def run(p):
        h, w, t, r, u = p["in"]
        loss, lse, dh, dw, out = p["out"]
        efs.ef_vocab_loss(h, w, t, loss, lse)
        efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw)
        efs.ef_orthogonalize([u], [out])
    problems = [problem(i) for i in range(4)]
    torch.cuda.synchronize()
    states = [None] * 4

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                run(problems[i])
        states[i] = efs.ef_check_status(stream)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for x in threads:
        x.start()
    for x in threads:
        x.join()
    assert states == [efs.EF_OK] * 4
    got = [[x.clone() for x in p["out"]] for p in problems]
    for p, before in zip(problems, got):
        run(p)
        for x, y in zip(p["out"], before):
            assert torch.equal(x, y)

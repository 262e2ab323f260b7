"""Logits at the ends of bf16's range: a bias of the type's lowest value on
every word, as a mask that leaves nothing is often written, and the largest one.

There the log-sum-exp in fp32 is the logits' common value, whatever the words'
own logits are: z = bias (the product is below half an ulp of it), lse = z (so is
log v), loss = 0, and G = r (exp(0) - [v = t]), exact but for the rounding of G's
sums: the operator's formulas in fp32, where a 64-bit lse would keep log v."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"
LOWEST = torch.finfo(torch.bfloat16).min


def inputs(n, v, d, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    w = (torch.randn(v, d, device=DEV, generator=g) / d ** 0.5).bfloat16()
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    return h, w, t


# few rows (one pass, two passes), one tile row read as it lies and gathered, more
SHAPES = [(4, 300, 64), (4, 300, 1100), (12, 300, 64), (50, 300, 64), (50, 300, 65), (300, 300, 64)]


@pytest.mark.parametrize("n,v,d", SHAPES)
@pytest.mark.parametrize("value", [LOWEST, -LOWEST])
def test_every_word_at_an_end_of_the_range(n, v, d, value):
    h, w, t = inputs(n, v, d, n + d)
    b = torch.full((v,), value, device=DEV, dtype=torch.bfloat16)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse, bias=b)
    assert (lse == value).all() and (loss == 0).all()
    r = torch.ones(n, device=DEV)
    dh, dw, db = torch.empty_like(h), torch.empty_like(w), torch.empty_like(b)
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    p = torch.ones(n, v, device=DEV, dtype=torch.float64)
    p[torch.arange(n, device=DEV), t] = 0.0
    # sums of exact terms (G is 0 or 1) in fp32, rounded to bf16: 2^-8 of the result,
    # and (k / 16 + 4) 2^-23 of the terms' magnitudes
    for got, ref, mag, k in ((dh, p @ w.double(), p @ w.double().abs(), v),
                             (dw, p.T @ h.double(), p.T @ h.double().abs(), n),
                             (db, p.sum(0), p.sum(0), n)):
        assert bool(((got.double() - ref).abs()
                     <= 2.0 ** -8 * ref.abs() + (k / 16 + 4) * 2.0 ** -23 * mag).all())
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.parametrize("n,v,d", SHAPES)
def test_some_words_at_the_lowest_value(n, v, d):
    h, w, t = inputs(n, v, d, 7 + n + d)
    b = torch.zeros(v, device=DEV, dtype=torch.bfloat16)
    b[40:] = LOWEST
    t = t % 40
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse, bias=b)
    z = h.double() @ w[:40].double().T
    ref = torch.logsumexp(z, 1)
    # z: (d / 16 + 4) 2^-23 of the sum of magnitudes; exp and log: 2^-20
    off = (d / 16 + 4) * 2.0 ** -23 * float((h.double().abs() @ w.double().abs().T).max())
    bound = 2 * off + 2.0 ** -19 * (1 + float(z.abs().max()))
    assert float((lse.double() - ref).abs().max()) <= bound
    assert float((loss.double() - ref + z.gather(1, t[:, None])[:, 0]).abs().max()) <= bound
    r = torch.ones(n, device=DEV)
    dh, dw, db = torch.empty_like(h), torch.empty_like(w), torch.empty_like(b)
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    assert (dw[40:] == 0).all() and (db[40:] == 0).all()
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()

"""Rows of the vocabulary gradient that have no word with a probability (their
log-sum-exp is -inf, here by an infinity in the row's hidden state) take no part
in it: the gradient is, bit for bit, that of the same batch with those rows
skipped."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gradient(h, w, t, lse, r, b):
    dh, dw, db = torch.full_like(h, 7.0), torch.empty_like(w), torch.empty_like(b)
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    return dh, dw, db


# one pass and two passes of the few-row kernels, tiles, and the two ways of
# finding the rows
@pytest.mark.parametrize("n,d", [(4, 200), (12, 200), (4, 1100), (40, 200), (300, 72), (4500, 40)])
def test_rows_without_a_word_take_no_part(n, d):
    g = torch.Generator(device=DEV).manual_seed(n + d)
    w = (torch.rand(500, d, device=DEV, generator=g) + 0.125).bfloat16()  # all positive
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    b = torch.randn(500, device=DEV, generator=g).bfloat16()
    t = torch.randint(0, 500, (n,), device=DEV, generator=g)
    r = torch.rand(n, device=DEV, generator=g) + 0.5
    gone = torch.zeros(n, dtype=torch.bool, device=DEV)
    gone[1::3] = True
    h[gone, 5] = float("-inf")
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse, bias=b)
    assert (lse[gone] == float("-inf")).all() and (loss[gone] == float("inf")).all()
    assert torch.isfinite(lse[~gone]).all() and torch.isfinite(loss[~gone]).all()
    got = gradient(h, w, t, lse, r, b)
    t[gone] = -1
    want = gradient(h, w, t, lse, r, b)
    assert all(torch.isfinite(x).all() for x in want)
    assert (got[0][gone] == 0).all()
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.parametrize("n,d", [(4, 200), (4, 1100), (40, 200), (4500, 40)])
def test_rows_without_a_word_beside_infinite_weights(n, d):
    g = torch.Generator(device=DEV).manual_seed(n + d)
    w = torch.randn(300, d, device=DEV, generator=g).bfloat16()
    w[7, 3] = float("-inf")
    h = torch.rand(n, d, device=DEV, generator=g).bfloat16() + 0.125  # z of word 7: -inf
    b = torch.full((300,), float("-inf"), device=DEV, dtype=torch.bfloat16)
    t = torch.randint(0, 300, (n,), device=DEV, generator=g)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse, bias=b)
    assert (lse == float("-inf")).all()
    for x in gradient(h, w, t, lse, torch.ones(n, device=DEV), b):
        assert (x == 0).all()

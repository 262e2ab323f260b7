"""The language-model example: its layout on the CPU, its training on a GPU."""
import pytest
import torch

from paper_2108_00951_gb300 import lm_sgd


def test_parameter_views_cover_the_vector():
    m = lm_sgd.Model.create(11, 4, 3, device="cpu")
    emb, mats, bias = m.split(m.x)
    assert m.d == 11 * 4 + 3 * 16 + 11
    assert emb.shape == (11, 4) and len(mats) == 3 and mats[0].shape == (4, 4)
    for part in (emb, *mats, bias):
        part.add_(1.0)
    fresh = lm_sgd.Model.create(11, 4, 3, device="cpu")
    assert torch.equal(m.x, fresh.x + 1.0)


def test_text_is_seeded():
    a, b = (lm_sgd.make_text(50, 40, 3, seed=5, device="cpu") for _ in range(2))
    assert torch.equal(a, b) and int(a.max()) < 50 and a.shape == (3, 40)
    assert not torch.equal(a, lm_sgd.make_text(50, 40, 3, seed=6, device="cpu"))


@pytest.mark.gpu
def test_worker_gradient_matches_autograd():
    m = lm_sgd.Model.create(300, 32, 2, seed=1)
    text = lm_sgd.make_text(300, 100, 1, seed=2)[0]
    g = torch.empty(m.d, device="cuda")
    loss = lm_sgd.worker_gradient(m, text, g)
    # the same model in 64 bits, its word vectors rounded as the worker's are
    emb, mats, bias = (m.split(m.x))
    e = emb.bfloat16().double().requires_grad_()
    c = [x.double().requires_grad_() for x in mats]
    b = bias.bfloat16().double().requires_grad_()
    h = sum(e[torch.roll(text, j + 1)] @ c[j].T for j in range(2))
    ref = torch.nn.functional.cross_entropy((h @ e.T + b)[2:], text[2:])
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 2e-3
    got_e, got_c, got_b = m.split(g)
    # h, dh and the gradients are bf16: a few roundings of 2^-8
    for x, y in ((got_e, e.grad), (got_b, b.grad), *((p, q.grad) for p, q in zip(got_c, c))):
        assert float((x.double() - y).norm() / y.norm()) < 4 * 2.0 ** -8


@pytest.mark.gpu
def test_training_learns_the_chain():
    h = lm_sgd.run(words=500, width=64, workers=3, length=200, steps=60)
    first, last = h["loss"][0], sum(h["loss"][-5:]) / 5
    assert abs(first - 6.2146) < 0.5  # log 500
    assert last < first - 1.0
    assert 0 < sum(h["sent"]) < 60 * 3 * h["d"][0]

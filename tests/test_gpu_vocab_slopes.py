"""The vocabulary gradient against differences of the loss in 64 bits.

Central differences of step 2^-13 on copies in 64 bits: their own error is the
third derivative's, at most |x|^3 per row (x the other factor's entry) times
step^2 / 6 = 2.5e-9, and rounding, 2^-53 of the summed losses over the step,
below 1e-8 here. The operator's own error is bounded as in its formula's
test: G to 2^-8 (2^-16 in calls of at most 16 rows) plus the logits' and exp's,
2 off + 2^-18, of the terms' magnitudes, and 2^-8 of the result. Most of the
entries compared are at least four times their bound, so that a gradient of 0 or
of the wrong sign does not pass."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("n", [3, 16, 60, 300])
def test_gradient_is_the_slope_of_the_loss(n):
    v, d, step = 400, 96, 2.0 ** -13
    g = torch.Generator(device=DEV).manual_seed(n)
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    w = (torch.randn(v, d, device=DEV, generator=g) * (2.0 / d ** 0.5)).bfloat16()
    b = torch.randn(v, device=DEV, generator=g).bfloat16()
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    t[: n // 4] = 17  # a frequent word
    r = torch.rand(n, device=DEV, generator=g) + 0.5
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse, bias=b)
    dh, dw, db = torch.empty_like(h), torch.empty_like(w), torch.empty_like(b)
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    h64, w64, b64, r64 = h.double(), w.double(), b.double(), r.double()

    def total():
        z = h64 @ w64.T + b64
        return float((r64 * (torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0])).sum())
    z = h64 @ w64.T + b64
    grad = torch.softmax(z, 1)
    grad[torch.arange(n, device=DEV), t] -= 1.0
    grad = (grad * r64[:, None]).abs()
    off = (d / 16 + 4) * 2.0 ** -23 * float((h64.abs() @ w64.abs().T).max())
    part = 2 * off + 2.0 ** -18
    rounded = part + (2.0 ** -16 if n <= 16 else 2.0 ** -8) + (max(n, v) / 16 + 4) * 2.0 ** -23
    words = [17, int(t[n - 1]), 3, 399]
    spots = [(h64, dh, grad @ w64.abs(), rounded, (i, j)) for i in (0, n // 2, n - 1) for j in (0, 41, 95)]
    spots += [(w64, dw, grad.T @ h64.abs(), rounded, (i, j)) for i in words for j in (0, 41, 95)]
    spots += [(b64, db, grad.sum(0), part + 2.0 ** -18, (i,)) for i in words]
    clear = 0
    for x, got, mag, share, at in spots:
        keep = float(x[at])
        ends = []
        for s in (step, -step):
            x[at] = keep + s
            ends.append(total())
        x[at] = keep
        slope = (ends[0] - ends[1]) / (2 * step)
        bound = share * float(mag[at]) + 2.0 ** -8 * abs(slope) + 1e-6
        assert abs(float(got[at]) - slope) <= bound, (tuple(got.shape), at)
        clear += abs(slope) >= 4 * bound
    assert clear >= 0.8 * len(spots)

"""Softmax cross entropy against a vocabulary, and its gradient, against the
formulas in 64 bits.

Bounds. Products of bf16 are exact in fp32; a sum of d of them, 16 at a time,
is off by at most (d / 16 + 4) 2^-23 of the sum of their magnitudes (additions
may truncate). exp and log are good to 2^-20. G is rounded to bf16 (2^-8; not
in calls of at most 16 rows, which keep 16 bits), as is each output."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def matrix(rows, cols, pad=0, offset=0, scale=1.0, gen=None):
    """bf16 [rows, cols], rows `pad` further apart, `offset` elements past an
    allocation's start."""
    buf = torch.empty(rows * (cols + pad) + offset, device=DEV, dtype=torch.bfloat16)
    m = buf[offset:].view(rows, cols + pad)[:, :cols]
    m.copy_(torch.randn(rows, cols, device=DEV, generator=gen) * scale)
    return m


def inputs(n, v, d, bias=False, ignored=0.0, pad=0, offset=0, seed=0):
    g = torch.Generator(device=DEV).manual_seed(1000 * seed + n + v + d)
    h = matrix(n, d, pad, offset, gen=g)
    w = matrix(v, d, pad, offset, 2.0 / d ** 0.5, gen=g)
    b = torch.randn(v, device=DEV, generator=g).bfloat16() if bias else None
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    if ignored:
        t[torch.rand(n, device=DEV, generator=g) < ignored] = -100
    r = torch.rand(n, device=DEV, generator=g) / max(n, 1)
    return h, w, t, r, b


def loss(h, w, t, b=None):
    out = torch.full((h.shape[0],), float("nan"), device=DEV)
    lse = out.clone()
    efs.ef_vocab_loss(h, w, t, out, lse, bias=b)
    return out, lse


def grad(h, w, t, lse, r, b=None, pad=0, offset=0):
    dh = matrix(*h.shape, pad, offset)
    dw = matrix(*w.shape, pad, offset)
    db = torch.empty(w.shape[0], device=DEV, dtype=torch.bfloat16) if b is not None else None
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    return dh, dw, db


def formula(h, w, t, r, b=None):
    """z, lse, loss, G in 64 bits, and the bound of z's error."""
    z = h.double() @ w.double().T
    if b is not None:
        z = z + b.double()
    off = (h.shape[1] / 16 + 4) * 2.0 ** -23 * float((h.double().abs() @ w.double().abs().T).max())
    keep = t >= 0
    lse = torch.where(keep, torch.logsumexp(z, 1), torch.zeros_like(z[:, 0]))
    at = z.gather(1, t.clamp(min=0)[:, None])[:, 0]
    g = torch.softmax(z, 1).scatter_add_(1, t.clamp(min=0)[:, None], -torch.ones_like(at)[:, None])
    g = g * (r.double() * keep)[:, None]
    return z, lse, torch.where(keep, lse - at, torch.zeros_like(at)), g, off


def check_grad(got, g, h, w, b, off, few):
    dh, dw, db = got
    rounded = 2.0 ** -16 if few else 2.0 ** -8
    part = 2 * off + 2.0 ** -18
    for out, ref, mag, k in ((dh, g @ w.double(), g.abs() @ w.double().abs(), w.shape[0]),
                             (dw, g.T @ h.double(), g.abs().T @ h.double().abs(), h.shape[0])):
        bound = (rounded + part + (k / 16 + 4) * 2.0 ** -23) * mag + 2.0 ** -8 * ref.abs() + 1e-30
        assert bool(((out.double() - ref).abs() <= bound).all())
    if b is not None:
        ref = g.sum(0)
        bound = (part + 2.0 ** -18) * g.abs().sum(0) + 2.0 ** -8 * ref.abs() + 1e-30
        assert bool(((db.double() - ref).abs() <= bound).all())


SHAPES = [(1, 1, 1), (1, 5, 3), (2, 1000, 64), (3, 129, 650), (8, 2049, 72), (9, 300, 129),
          (16, 1000, 333), (17, 1000, 333), (64, 257, 65), (128, 1024, 128), (129, 513, 96),
          (200, 4001, 130), (257, 255, 512), (700, 1500, 650), (1000, 33, 7), (4097, 300, 40)]


@pytest.mark.parametrize("n,v,d", SHAPES)
@pytest.mark.parametrize("bias,ignored,pad,offset", [(False, 0.0, 0, 0), (True, 0.4, 0, 0),
                                                     (True, 0.0, 3, 1), (False, 0.3, 8, 2)])
def test_matches_the_formula(n, v, d, bias, ignored, pad, offset):
    h, w, t, r, b = inputs(n, v, d, bias, ignored, pad, offset)
    out, lse = loss(h, w, t, b)
    z, ref_lse, ref, g, off = formula(h, w, t, r, b)
    bound = 2 * off + 2.0 ** -19 * (1 + ref_lse.abs() + z.abs().max())
    assert bool(((lse.double() - ref_lse).abs() <= bound).all())
    assert bool(((out.double() - ref).abs() <= bound).all())
    got = grad(h, w, t, lse, r, b, pad, offset)
    check_grad(got, g, h, w, b, off, n <= 16)
    assert efs.ef_check_status() == efs.EF_OK


def test_wide_rows_leave_the_few_row_kernel():
    # 16 rows of 5001 do not fit beside the rings of the few-row kernel
    h, w, t, r, b = inputs(16, 300, 5001, True)
    out, lse = loss(h, w, t, b)
    _, ref_lse, ref, g, off = formula(h, w, t, r, b)
    assert bool(((out.double() - ref).abs() <= 2 * off + 1e-4).all())
    check_grad(grad(h, w, t, lse, r, b), g, h, w, b, off, False)


@pytest.mark.parametrize("n", [3, 300])
def test_gradient_by_differences(n):
    h, w, t, r, b = inputs(n, 400, 96, True)
    r.fill_(1.0)
    _, lse = loss(h, w, t, b)
    dh, dw, db = grad(h, w, t, lse, r, b)
    # steps of 2^-3 are exact in bf16 for values below 16; the third derivative
    # of the loss is below |w|^3 (or |h|^3) per row
    for x, dx, i, j in ((h, dh, 1, 5), (h, dh, n - 1, 95), (w, dw, 7, 0), (w, dw, int(t[0]), 3)):
        keep, ends = x[i, j].clone(), []
        for s in (1, -1):
            x[i, j] = keep.float().mul(16).round().div(16).add(s / 8.0).bfloat16()
            ends.append((float(x[i, j]), loss(h, w, t, b)[0].double().sum()))
        mid = ((ends[0][0] + ends[1][0]) / 2)
        x[i, j] = mid
        _, lse2 = loss(h, w, t, b)
        at = grad(h, w, t, lse2, r, b)[0 if dx is dh else 1][i, j]
        slope = (ends[0][1] - ends[1][1]) / (ends[0][0] - ends[1][0])
        x[i, j] = keep
        size = float((w if dx is dh else h).double().abs().max())
        bound = (n if dx is dw else 1) * size ** 3 / 384 + 2.0 ** -7 * abs(float(slope)) + 2e-3
        assert abs(float(at) - float(slope)) <= bound
    assert bool((db.double() - torch.autograd.functional.jacobian(
        lambda c: torch.nn.functional.cross_entropy(
            h.double() @ w.double().T + c, t, reduction="sum"), b.double())).abs().max() <= 0.05)


@pytest.mark.parametrize("n", [5, 40])
def test_words_ruled_out(n):
    h, w, t, r, b = inputs(n, 700, 64, True)
    b[100:650] = float("-inf")
    t[0], t[1] = 200, 10            # a target that is ruled out, and one that is not
    out, lse = loss(h, w, t, b)
    z = h.double() @ w.double().T + b.double()
    ref = torch.logsumexp(z, 1)
    assert bool(((lse.double() - ref).abs() < 1e-4).all())
    assert torch.isinf(out[0]) and out[0] > 0
    dh, dw, db = grad(h, w, t, lse, r, b)
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()
    gone = torch.ones(700, dtype=torch.bool, device=DEV)
    gone[:100] = gone[650:] = False
    gone[t] = False                 # (targets still get -r h)
    assert (dw[gone] == 0).all() and (db[gone] == 0).all()


@pytest.mark.parametrize("n", [4, 50])
def test_a_row_without_any_word(n):
    h, w, t, r, b = inputs(n, 300, 32, True)
    b.fill_(float("-inf"))
    out, lse = loss(h, w, t, b)
    assert (lse == float("-inf")).all() and (out == float("inf")).all()
    dh, dw, db = grad(h, w, t, lse, r, b)
    assert (dh == 0).all() and (dw == 0).all() and (db == 0).all()


@pytest.mark.parametrize("n", [6, 90])
def test_skipped_rows_may_hold_anything(n):
    h, w, t, r, b = inputs(n, 500, 64, True, pad=8)
    t[1::2] = -1
    out, lse = loss(h, w, t, b)
    got = [x.clone() for x in (out, lse, *grad(h, w, t, lse, r, b))]
    h[1::2] = float("nan")
    r[1::2] = float("inf")
    out, lse = loss(h, w, t, b)
    for x, y in zip((out, lse, *grad(h, w, t, lse, r, b)), got):
        assert torch.equal(x, y)
    assert (out[1::2] == 0).all() and (lse[1::2] == 0).all()


@pytest.mark.parametrize("n", [3, 70])
def test_nan_and_infinity_stay_in_their_row(n):
    h, w, t, r, b = inputs(n, 400, 64)
    clean, _ = loss(h, w, t)
    h[0, 3] = float("nan")
    h[2, 0] = float("inf")
    out, lse = loss(h, w, t)
    assert torch.isnan(out[0]) and torch.isnan(lse[0]) and torch.isnan(lse[2])
    keep = [i for i in range(n) if i not in (0, 2)]
    assert torch.equal(out[keep], clean[keep])
    dh, _, _ = grad(h, w, t, lse, r)
    assert torch.isnan(dh[0]).all() and torch.isfinite(dh[keep]).all()


@pytest.mark.parametrize("n", [4, 60, 5000])
def test_a_target_past_the_vocabulary_is_reported(n):
    h, w, t, r, _ = inputs(n, 50, 16)
    t[n - 1] = 50
    out, lse = loss(h, w, t)
    assert efs.ef_check_status() == efs.EF_ERR_BAD_INPUT
    assert out[n - 1] == 0 and lse[n - 1] == 0
    t[n - 1] = -1
    again, _ = loss(h, w, t)
    assert torch.equal(out, again)
    assert efs.ef_check_status() == efs.EF_OK


def test_no_rows():
    h, w, t, r, b = inputs(0, 300, 64, True)
    out, lse = loss(h, w, t, b)
    dh, dw, db = grad(h, w, t, lse, r, b)
    torch.cuda.synchronize()
    assert (dw == 0).all() and (db == 0).all()


def test_all_rows_skipped():
    for n in (5, 200):
        h, w, t, r, b = inputs(n, 300, 64, True)
        t.fill_(-1)
        out, lse = loss(h, w, t, b)
        dh, dw, db = grad(h, w, t, lse, r, b)
        assert all((x == 0).all() for x in (out, lse, dh, dw, db))


@pytest.mark.parametrize("n", [7, 333])
def test_equal_inputs_give_equal_bits(n):
    h, w, t, r, b = inputs(n, 5000, 200, True, 0.2)
    first = None
    for _ in range(3):
        out, lse = loss(h, w, t, b)
        got = [out, lse, *grad(h, w, t, lse, r, b)]
        assert first is None or all(torch.equal(x, y) for x, y in zip(got, first))
        first = got


def test_pieces_of_the_vocabulary_add_up():
    # 70,000 rows: G of 20,000 words is taken in three pieces
    h, w, t, r, b = inputs(70000, 20000, 32, True, 0.1)
    out, lse = loss(h, w, t, b)
    dh, dw, db = grad(h, w, t, lse, r, b)
    some = torch.arange(0, 70000, 997, device=DEV)
    _, ref_lse, ref, g, off = formula(h[some], w, t[some], r[some], b)
    assert bool(((out[some].double() - ref).abs() <= 2 * off + 1e-4).all())
    mag = g.abs() @ w.double().abs()
    bound = (2.0 ** -8 + 2 * off + 2.0 ** -10) * mag + 2.0 ** -8 * (g @ w.double()).abs() + 1e-30
    assert bool(((dh[some].double() - g @ w.double()).abs() <= bound).all())
    ref_w, ref_b = torch.zeros(20000, 32, device=DEV, dtype=torch.float64), 0
    mag_w, mag_b = torch.zeros_like(ref_w), 0
    for a in range(0, 70000, 5000):
        g = formula(h[a:a + 5000], w, t[a:a + 5000], r[a:a + 5000], b)[3]
        ref_w += g.T @ h[a:a + 5000].double()
        mag_w += g.abs().T @ h[a:a + 5000].double().abs()
        ref_b, mag_b = ref_b + g.sum(0), mag_b + g.abs().sum(0)
    assert bool(((dw.double() - ref_w).abs()
                 <= (2.0 ** -8 + 2 * off + 2.0 ** -10) * mag_w + 2.0 ** -8 * ref_w.abs()).all())
    assert bool(((db.double() - ref_b).abs()
                 <= (2 * off + 2.0 ** -16) * mag_b + 2.0 ** -8 * ref_b.abs()).all())


def test_other_stream_and_capture():
    h, w, t, r, b = inputs(150, 900, 128, True)
    out, lse = loss(h, w, t, b)
    ref = [out.clone(), lse.clone(), *grad(h, w, t, lse, r, b)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    dh, dw = torch.empty_like(h), torch.empty_like(w)
    db = torch.empty_like(b)
    with torch.cuda.stream(s):
        for _ in range(2):  # the stream's workspace grows outside the capture
            efs.ef_vocab_loss(h, w, t, out, lse, bias=b)
            efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    s.synchronize()
    for x, y in zip((out, lse, dh, dw, db), ref):
        assert torch.equal(x, y)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        efs.ef_vocab_loss(h, w, t, out, lse, bias=b)
        efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw, bias=b, dbias_out=db)
    for x in (out, lse, dh, dw, db):
        x.zero_()
    g.replay()
    torch.cuda.synchronize()
    for x, y in zip((out, lse, dh, dw, db), ref):
        assert torch.equal(x, y)


@pytest.mark.slow
@pytest.mark.parametrize("n", [2, 20])
def test_offsets_past_32_bits(n):
    # w of 2.3e9 elements: 4.6 GB
    v, d = 1_100_001, 2100
    g = torch.Generator(device=DEV).manual_seed(5)
    w = torch.empty(v, d, device=DEV, dtype=torch.bfloat16)
    for a in range(0, v, 50000):
        w[a:a + 50000] = torch.randn(min(50000, v - a), d, device=DEV, generator=g) * (2 / d ** 0.5)
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    t = torch.randint(v - 1000, v, (n,), device=DEV, generator=g)
    r = torch.ones(n, device=DEV)
    out, lse = loss(h, w, t)
    z = torch.cat([h.double() @ w[a:a + 50000].double().T for a in range(0, v, 50000)], 1)
    ref = torch.logsumexp(z, 1)
    assert bool(((lse.double() - ref).abs() < 2e-4).all())
    assert bool(((out.double() - ref + z.gather(1, t[:, None])[:, 0]).abs() < 4e-4).all())
    dh, dw, _ = grad(h, w, t, lse, r)
    p = torch.exp(z - ref[:, None])
    p.scatter_add_(1, t[:, None], -torch.ones(n, 1, device=DEV, dtype=torch.float64))
    last = slice(v - 1000, v)
    ref_w = p[:, last].T @ h.double()
    mag = p[:, last].abs().T @ h.double().abs()
    assert bool(((dw[last].double() - ref_w).abs() <= 2.0 ** -7 * mag).all())
    ref_h = torch.zeros(n, d, device=DEV, dtype=torch.float64)
    for a in range(0, v, 50000):
        ref_h += p[:, a:a + 50000] @ w[a:a + 50000].double()
    assert float((dh.double() - ref_h).norm() / ref_h.norm()) < 5e-3


@pytest.mark.parametrize("d", [1, 63, 64, 65, 129, 511, 640, 1023, 1024, 1025, 2048])
@pytest.mark.parametrize("n,v", [(1, 17), (8, 2439), (9, 16), (16, 5001)])
def test_few_rows_at_every_width(n, v, d):
    h, w, t, r, b = inputs(n, v, d, True, 0.2 if n > 1 else 0.0, pad=d % 3, seed=5)
    _, lse = loss(h, w, t, b)
    z, ref, _, g, off = formula(h, w, t, r, b)
    check_grad(grad(h, w, t, lse, r, b, pad=d % 3), g, h, w, b, off, True)
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.parametrize("n,d", [(4, 200), (4, 1100), (40, 200)])
def test_skipped_rows_have_no_gradient_beside_infinite_weights(n, d):
    h, w, t, r, _ = inputs(n, 500, d, seed=6)
    w[7, 3] = float("inf")
    t[1] = -1
    _, lse = loss(h, w, t)
    dh, _, _ = grad(h, w, t, lse, r)
    assert torch.all(dh[1] == 0)


@pytest.mark.parametrize("n", [17, 128, 129, 256, 257])
@pytest.mark.parametrize("d,pad", [(72, 0), (136, 8), (70, 2)])
def test_rows_that_lie_on_16_bytes(n, d, pad):
    h, w, t, r, b = inputs(n, 999, d, True, 0.3, pad, seed=8)
    t[0], t[n - 1] = -1, 5
    out, lse = loss(h, w, t, b)
    _, ref_lse, ref, g, off = formula(h, w, t, r, b)
    bound = 2 * off + 2.0 ** -18 * (1 + ref_lse.abs() + ref.abs())
    assert bool(((lse.double() - ref_lse).abs() <= bound).all())
    assert bool(((out.double() - ref).abs() <= bound).all())
    h[t < 0] = float("nan")
    again, lse_again = loss(h, w, t, b)
    assert torch.equal(again, out) and torch.equal(lse_again, lse)
    assert efs.ef_check_status() == efs.EF_OK
    t[3] = 999
    again, _ = loss(h, w, t, b)
    assert again[3] == 0 and torch.equal(again[4:], out[4:])
    assert efs.ef_check_status() == efs.EF_ERR_BAD_INPUT

"""Layer norm and its gradient against the formulas in 64 bits.

Bounds. A sum over a row runs through at most 31 additions in a thread (d / 1024 in rows of one
CTA), 5 in a warp, 7 over its CTA's warps and 7 over a cluster's CTAs: depth =
max(32, d / 1024) + 20 fp32 additions, so it is off by at most depth 2^-24 of the sum of magnitudes. From that,
with u = 2^-24:
  mean   dm = (depth + 2) u avg|x|
  rstd   relative dr = ((depth + 4) u (var + 0) + 2 (dm + u max|x|) avg|x - mean| + dm^2) / (2 (var + eps)) + 3 u
  y      |w| (|x'| (dr + 3 u) + rstd (dm + u |x - mean|)) + 2 u (|x' w| + |b|), then its rounding
and for the gradient, whose mean and rstd are inputs:
  x'     relative 2 u,   q relative u,   sums over a row (depth + 5) u of their magnitudes,
  dx     rstd times that, and 6 u of its terms; then its rounding
  dw, db n + 6 additions and roundings over the rows."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def matrix(rows, cols, dtype, pad=0, offset=0, values=None):
    buf = torch.full((rows * (cols + pad) + offset,), 7.0, device=DEV, dtype=dtype)
    m = buf[offset:].view(rows, cols + pad)[:, :cols]
    if values is not None:
        m.copy_(values)
    return m


def weights(d, dtype, gen, offset=0):
    w = torch.empty(d + offset, device=DEV, dtype=dtype)[offset:]
    return w.copy_(torch.randn(d, device=DEV, generator=gen))


def rounding(t):
    return torch.finfo(t).eps / 2 * (1 + 2.0 ** -8)


def check(n, d, xt, yt, wt, pad, offset, weight=True, bias=True, eps=1e-5, shift=2.0):
    g = torch.Generator(device=DEV).manual_seed(n + d)
    x = matrix(n, d, xt, pad, offset, torch.randn(n, d, device=DEV, generator=g) * 3 + shift)
    dy = matrix(n, d, yt, pad, offset, torch.randn(n, d, device=DEV, generator=g))
    w = weights(d, wt, g, offset) if weight else None
    b = weights(d, wt, g, offset) if bias else None
    y, dx = matrix(n, d, yt, pad, offset), matrix(n, d, xt, pad, offset)
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_layer_norm(x, y, w, b, eps, mean, rstd)
    depth = max(32, d // 1024) + 20
    eps = float(torch.tensor(eps))
    xx = x.double()
    mu = xx.mean(1, keepdim=True)
    var = (xx - mu).square().mean(1, keepdim=True)
    rs = (var + eps).rsqrt()
    ww = w.double() if weight else torch.ones(d, device=DEV, dtype=torch.float64)
    bb = b.double() if bias else torch.zeros(d, device=DEV, dtype=torch.float64)
    hat = (xx - mu) * rs
    dm = (depth + 2) * U * xx.abs().mean(1, keepdim=True)
    dr = ((depth + 4) * U * var + 2 * (dm + U * xx.abs().amax(1, keepdim=True))
          * (xx - mu).abs().mean(1, keepdim=True) + dm * dm) / (2 * (var + eps)) + 3 * U
    assert bool(((mean[:, None].double() - mu).abs() <= dm).all())
    assert bool(((rstd[:, None].double() - rs).abs() <= dr * rs).all())
    ref = hat * ww + bb
    bound = ww.abs() * (hat.abs() * (dr + 3 * U) + rs * (dm + U * (xx - mu).abs()))
    bound = bound + 2 * U * ((hat * ww).abs() + bb.abs()) + rounding(yt) * ref.abs() + 1e-37
    assert bool(((y.double() - ref).abs() <= bound).all())

    dw = torch.full((d,), 5.0, device=DEV, dtype=wt)
    db = torch.full((d,), 5.0, device=DEV, dtype=wt)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, dx, w, dw, db)
    m64, r64 = mean[:, None].double(), rstd[:, None].double()
    hat, gg = (xx - m64) * r64, dy.double()
    q = gg * ww
    s1, s2 = q.mean(1, keepdim=True), (q * hat).mean(1, keepdim=True)
    ref = r64 * (q - s1 - hat * s2)
    sums = q.abs().mean(1, keepdim=True) + hat.abs() * (q * hat).abs().mean(1, keepdim=True)
    bound = r64 * ((depth + 5) * U * sums + 6 * U * (q.abs() + s1.abs() + (hat * s2).abs()))
    assert bool(((dx.double() - ref).abs() <= bound + rounding(xt) * ref.abs() + 1e-37).all())
    for out, terms in ((dw, gg * hat), (db, gg)):
        ref = terms.sum(0)
        bound = (n + 6) * U * terms.abs().sum(0) + rounding(wt) * ref.abs() + 1e-37
        assert bool(((out.double() - ref).abs() <= bound).all())
    # each output by itself
    alone, one = matrix(n, d, xt, pad, offset), torch.empty_like(dw)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, alone, w)
    assert torch.equal(alone, dx)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, None, w, one)
    assert torch.equal(one, dw)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, None, w, None, one)
    assert torch.equal(one, db)
    assert efs.ef_check_status() == efs.EF_OK
    if pad:
        whole = y.as_strided((n, d + pad), (d + pad, 1), y.storage_offset())[:, d:]
        assert bool((whole[:-1] == 7.0).all())


SHAPES = [(1, 1), (1, 650), (3, 2), (5, 129), (8, 256), (9, 257), (17, 512), (700, 650), (40, 1000),
          (1300, 1024), (3, 1025), (77, 1500), (301, 2048), (640, 4096), (9, 4097), (330, 8192),
          (5, 8193), (160, 10000), (3, 28000), (4, 28001), (40, 40000)]
# rows in lanes of a warp, several a warp, the last warps and CTAs part full; clusters of each
# size; rows that one CTA goes through
MORE = [(5000, 3), (4999, 8), (3001, 17), (777, 33), (2500, 64), (1999, 128), (1001, 200), (9, 96), (700, 6001),
        (3, 16385), (70, 24576), (2, 33000), (5, 49153), (3, 65536), (2, 65537), (37, 70001)]


@pytest.mark.parametrize("n,d", SHAPES + MORE)
@pytest.mark.parametrize("xt,yt,wt,pad,offset", [(BF16, BF16, F32, 0, 0), (F32, F32, F32, 0, 0),
                                                 (F32, BF16, BF16, 3, 1), (BF16, F32, F32, 6, 2),
                                                 (BF16, BF16, BF16, 1, 1)])
def test_matches_the_formulas(n, d, xt, yt, wt, pad, offset):
    check(n, d, xt, yt, wt, pad, offset)


@pytest.mark.parametrize("n,d", [(6, 100), (300, 1111), (5, 9000), (2, 30000)])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(n, d, weight, bias):
    check(n, d, F32, F32, F32, 0, 0, weight, bias)


@pytest.mark.parametrize("d", [64, 650, 3000, 9000])
def test_large_means(d):
    check(20, d, F32, F32, F32, 0, 0, shift=1000.0)


@pytest.mark.parametrize("d", [24, 700, 3000, 9000])
def test_constant_and_unreadable_rows(d):
    x = torch.randn(6, d, device=DEV)
    x[1] = 3.0
    x[3, d // 2] = float("nan")
    x[4, 0] = float("inf")
    y, w = torch.empty_like(x), torch.rand(d, device=DEV) + 0.5
    b = torch.randn(d, device=DEV)
    mean, rstd = torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    efs.ef_layer_norm(x, y, w, b, 1e-5, mean, rstd)
    assert torch.equal(y[1], b)
    assert bool(y[3:5].isnan().all()) and bool(y[[0, 1, 2, 5]].isfinite().all())
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    efs.ef_layer_norm_grad(x, mean, rstd, torch.ones_like(x), dx, w, dw)
    assert bool(dx[3:5].isnan().all()) and bool(dx[[0, 1, 2, 5]].isfinite().all())


@pytest.mark.parametrize("d", [16, 900, 3000, 9000, 30000])
def test_no_rows(d):
    none = torch.empty(0, d, device=DEV)
    rows = torch.empty(0, device=DEV)
    dw, db = torch.ones(d, device=DEV), torch.ones(d, device=DEV)
    efs.ef_layer_norm(none, none.clone())
    efs.ef_layer_norm_grad(none, rows, rows, none.clone(), none.clone(), None, dw, db)
    assert bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("n,d", [(3, 50), (20, 650), (6, 2000), (4, 8500)])
def test_gradient_meets_differences(n, d):
    """Slopes of sum(dy y) of the 64-bit formula along random ways."""
    g = torch.Generator(device=DEV).manual_seed(d)
    x, dy = (torch.randn(n, d, device=DEV, generator=g) for _ in range(2))
    w, b = (torch.randn(d, device=DEV, generator=g) for _ in range(2))
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    efs.ef_layer_norm(x, y, w, b, 1e-5, mean, rstd)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, dx, w, dw, db)

    def value(x, w, b):
        z = x - x.mean(1, keepdim=True)
        z = z * (z.square().mean(1, keepdim=True) + 1e-5).rsqrt()
        return (dy.double() * (z * w + b)).sum()
    at = [t.double() for t in (x, w, b)]
    for i, grad in enumerate((dx, dw, db)):
        for _ in range(3):
            way = torch.randn(at[i].shape, device=DEV, dtype=torch.float64, generator=g)
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-4 * way, at[i] - 1e-4 * way
            slope = float((value(*up) - value(*down)) / 2e-4)
            got = float((grad.double() * way).sum())
            # central differences: 1e-8 of third derivatives; fp32 gradients: 2^-20 of their terms
            assert abs(got - slope) < 2.0 ** -18 * float((grad.double() * way).abs().sum()) + 1e-5


@pytest.mark.parametrize("n,d", [(9000, 24), (3000, 650), (500, 3000), (200, 9000), (100, 30000), (40, 70000)])
def test_equal_inputs_give_equal_bits(n, d):
    g = torch.Generator(device=DEV).manual_seed(n)
    x, dy = (torch.randn(n, d, device=DEV, generator=g).bfloat16() for _ in range(2))
    w = torch.rand(d, device=DEV, generator=g)
    mean, rstd = x.float().mean(1), x.float().std(1).reciprocal()
    outs = []
    for _ in range(3):
        dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
        efs.ef_layer_norm_grad(x, mean, rstd, dy, dx, w, dw, db)
        outs.append((dx, dw, db))
    for a in outs[1:]:
        assert all(torch.equal(p, q) for p, q in zip(a, outs[0]))


def rows_at(d):
    """Additions that a row's sum runs through, as above."""
    return max(32, d // 1024) + 20


@pytest.mark.parametrize("d", [1, 7, 13, 41, 55, 257, 1001, 2049, 4099, 9001, 33001, 70001])
@pytest.mark.parametrize("xt", [F32, BF16])
@pytest.mark.parametrize("eps", [1e-5, 1e-12])
def test_rows_of_one_value(d, xt, eps):
    """A row of one value is its mean exactly, and y the bias. bf16 (8 bits) adds up exactly to 65,536
    columns; else the sum's mean is off by k places of the value, k at most the additions, and the
    differences, k places each, are added exactly (d k < 2^24) and divided exactly. Their squares may be off by (additions + 3) u of k^2 places^2."""
    values = torch.tensor([1000.0, 1e4, 0.1, 1e5, -3.0, 100000.1, 1e-3], device=DEV)
    x = values[:, None].expand(-1, d).to(xt).contiguous()
    g = torch.Generator(device=DEV).manual_seed(d)
    w, b = weights(d, F32, g), weights(d, F32, g)
    y = torch.empty(len(x), d, device=DEV)
    mean, rstd = torch.empty(len(x), device=DEV), torch.empty(len(x), device=DEV)
    efs.ef_layer_norm(x, y, w, b, eps, mean, rstd)
    assert torch.equal(mean, x[:, 0].float())
    assert torch.equal(y, b.expand_as(y))
    k = (rows_at(d) + 2) * 2 * U * x[:, 0].double().abs()
    left = (rows_at(d) + 3) * U * k * k
    eps = float(torch.tensor(eps))
    want = eps ** -0.5
    assert bool((rstd.double() <= want * (1 + 3 * U)).all())
    assert bool((rstd.double() >= (eps + left).rsqrt() * (1 - 3 * U)).all())


@pytest.mark.parametrize("d", [7, 41, 55, 64, 200, 650, 1001, 3000, 4096, 9000, 9001, 33000, 70001])
@pytest.mark.parametrize("shift", [1e3, 1e5, -3e4])
def test_what_is_subtracted_is_the_mean_of_large_rows(d, shift):
    """With m the mean of the row's sum, off by at most e = (depth + 2) u avg|x|, t = x - m is off by u |t|,
    its mean c by dc = (depth + 3) u (avg|x - mean| + e), and x - m - c by dc + u (|x - mean| + |t|); the
    squares' mean less c^2 by (depth + 6) u (var + e^2) + 2 e dc + dc^2."""
    g = torch.Generator(device=DEV).manual_seed(d)
    n, depth, eps = 23, rows_at(d), 1e-5
    x = torch.randn(n, d, device=DEV, generator=g) + shift
    w, b = weights(d, F32, g), weights(d, F32, g)
    y, mean, rstd = torch.empty_like(x), torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_layer_norm(x, y, w, b, eps, mean, rstd)
    xx, ww, bb, eps = x.double(), w.double(), b.double(), float(torch.tensor(eps))
    mu = xx.mean(1, keepdim=True)
    t = xx - mu
    var = t.square().mean(1, keepdim=True)
    rs = (var + eps).rsqrt()
    e = (depth + 2) * U * xx.abs().mean(1, keepdim=True)
    dc = (depth + 3) * U * (t.abs().mean(1, keepdim=True) + e)
    dr = ((depth + 6) * U * (var + e * e) + 2 * e * dc + dc * dc) / (2 * (var + eps)) * 1.01 + 3 * U
    assert bool(((mean[:, None].double() - mu).abs() <= dc + U * (mu.abs() + dc)).all())
    assert bool(((rstd[:, None].double() - rs).abs() <= dr * rs).all())
    hat = t * rs
    bound = ww.abs() * (hat.abs() * (dr + 3 * U) + rs * (dc + U * (2 * t.abs() + e)))
    bound = bound + 2 * U * ((hat * ww).abs() + bb.abs())
    assert bool(((y.double() - (hat * ww + bb)).abs() <= bound).all())


# groups that take more rows than their ring has places, and the ends of the last round part full:
# lanes (8 places forward, 6 back), warps (4, 3), a CTA of 16 and of 32 values a thread, clusters
TALL = [(1100003, 3), (270001, 64), (90001, 200), (12001, 650), (5001, 2048), (3001, 4096), (1501, 8192),
        (1201, 10000), (521, 24576), (303, 24209), (300, 32768)]


@pytest.mark.parametrize("n,d", TALL)
@pytest.mark.parametrize("xt,yt,wt,pad,offset", [(BF16, BF16, F32, 0, 0), (F32, BF16, BF16, 3, 1)])
def test_rows_go_round_the_ring(n, d, xt, yt, wt, pad, offset):
    check(n, d, xt, yt, wt, pad, offset)


@pytest.mark.parametrize("n,d", [(40000, 24), (90001, 200), (12001, 650), (3001, 4095), (700, 8192), (520, 10000), (9, 70001)])
@pytest.mark.parametrize("xt", [F32, BF16])
def test_large_means_in_some_rows_of_many(n, d, xt):
    """Rows that are corrected among rows that are not: each as it is by itself."""
    g = torch.Generator(device=DEV).manual_seed(n)
    x = torch.randn(n, d, device=DEV, generator=g)
    x += torch.where(torch.rand(n, 1, device=DEV, generator=g) < 0.3, 500.0, 0.0)
    x[1], x = 77.7, x.to(xt)
    x[1] = x[1, 0]
    w, b = weights(d, F32, g), weights(d, F32, g)
    y, mean, rstd = (torch.empty(s, device=DEV) for s in ((n, d), (n,), (n,)))
    efs.ef_layer_norm(x, y, w, b, 1e-5, mean, rstd)
    assert torch.equal(y[1], b) and float(mean[1]) == float(x[1, 0])
    for i in (0, 1, 2, n // 2, n - 2, n - 1):
        y1, m1, r1 = torch.empty(1, d, device=DEV), torch.empty(1, device=DEV), torch.empty(1, device=DEV)
        # (as many rows, so that the same kernel takes it)
        efs.ef_layer_norm(x[i:i + 1].expand(n, d).contiguous(), full := torch.empty(n, d, device=DEV), w, b, 1e-5,
                          ms := torch.empty(n, device=DEV), rs := torch.empty(n, device=DEV))
        for rows, one in ((full, y[i]), (ms, mean[i]), (rs, rstd[i])):
            assert torch.equal(rows, one.expand_as(rows))


@pytest.mark.parametrize("n,d", [(5, 3), (300, 24), (40, 650), (9, 2048), (6, 4097), (4, 9000), (3, 70001)])
@pytest.mark.parametrize("xt,yt", [(F32, F32), (BF16, BF16), (F32, BF16)])
@pytest.mark.parametrize("pad,offset", [(3, 1), (8, 8), (1, 2)])
def test_nothing_beside_the_rows_is_written(n, d, xt, yt, pad, offset):
    g = torch.Generator(device=DEV).manual_seed(d)

    def guarded(dtype):
        buf = torch.full((offset + n * (d + pad) + 5,), 7.0, device=DEV, dtype=dtype)
        rows = buf[offset:offset + n * (d + pad)].view(n, d + pad)
        return buf, rows[:, :d]

    def rest(buf, m):
        keep = torch.ones_like(buf, dtype=torch.bool)
        keep[offset:offset + n * (d + pad)].view(n, d + pad)[:, :d] = False
        return buf[keep]
    x = torch.randn(n, d, device=DEV, generator=g).to(xt)
    x[0] += 300.0
    dy = torch.randn(n, d, device=DEV, generator=g).to(yt)
    (by, y), (bx, dx) = guarded(yt), guarded(xt)
    vectors = torch.full((6, d + 16), 7.0, device=DEV)
    mean, rstd = torch.full((n + 4,), 7.0, device=DEV), torch.full((n + 4,), 7.0, device=DEV)
    efs.ef_layer_norm(x, y, None, None, 1e-5, mean, rstd)
    efs.ef_layer_norm_grad(x, mean, rstd, dy, dx, None, vectors[1, :d], vectors[4, :d])
    assert bool((rest(by, y) == 7.0).all()) and bool((rest(bx, dx) == 7.0).all())
    assert bool((mean[n:] == 7.0).all()) and bool((rstd[n:] == 7.0).all())
    assert bool((vectors[[0, 2, 3, 5]] == 7.0).all()) and bool((vectors[[1, 4], d:] == 7.0).all())
    assert not bool((vectors[[1, 4], :d] == 7.0).all()) and bool(dx.isfinite().all())
    assert efs.ef_check_status() == efs.EF_OK

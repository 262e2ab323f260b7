"""Orthogonalised updates against five Newton-Schulz steps in 64 bits.

Bounds, relative in the 2-norm: 2e-3 before the rounding of the bf16 output (fp16
operands, whose roundings the steps amplify), 1e-4 where the shorter side is at
most 128 (operands of 22 bits); the output's rounding is at most 2^-8."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"
A, B, C = 3.4445, -4.7750, 2.0315


def exact(u):
    x = u.double()
    x = x / x.norm()
    left = x.shape[0] <= x.shape[1]
    for _ in range(5):
        g = x @ x.T if left else x.T @ x
        p = B * g + C * (g @ g)
        x = A * x + (p @ x if left else x @ p)
    return x


def matrix(r, c, dtype=torch.float32, kind="noise", pad=0, offset=0, seed=0, scale=1e-3):
    g = torch.Generator(device=DEV).manual_seed(31 * r + c + seed)
    x = torch.randn(r, c, device=DEV, generator=g)
    if kind == "decades":  # singular values over four decades
        k = min(r, c)
        q = torch.linalg.qr(torch.randn(k, k, device=DEV, generator=g))[0]
        s = torch.logspace(0, -4, k, device=DEV)
        x = (q * s) @ x if r <= c else x @ (s[:, None] * q.T)
    elif kind == "low":
        x = torch.randn(r, 2, device=DEV, generator=g) @ torch.randn(2, c, device=DEV, generator=g)
    buf = torch.empty(r * (c + pad) + offset, device=DEV, dtype=dtype)
    m = buf[offset:].view(r, c + pad)[:, :c]
    m.copy_(x * scale)
    return m


def run(us, moms=None, mu=0.0, pad=0, offset=0):
    outs = []
    for u in us:
        buf = torch.full((u.shape[0] * (u.shape[1] + pad) + offset,), float("nan"), device=DEV,
                         dtype=torch.bfloat16)
        outs.append(buf[offset:].view(u.shape[0], u.shape[1] + pad)[:, :u.shape[1]])
    efs.ef_orthogonalize(us, outs, momenta=moms, momentum=mu)
    assert efs.ef_check_status() == efs.EF_OK
    return outs


def check(u, out):
    ref = exact(u)
    tol = (1e-4 if min(u.shape) <= 128 else 2e-3) + 2.0 ** -8
    assert float((out.double() - ref).norm()) <= tol * float(ref.norm())


SHAPES = [(1, 1), (1, 300), (300, 1), (2, 3), (5, 64), (64, 5), (17, 33), (64, 576), (576, 64),
          (128, 128), (127, 2000), (2000, 127), (64, 4096), (3, 9000), (9000, 3), (128, 5000),
          (129, 129), (129, 1000), (1000, 129), (256, 256), (300, 333), (650, 2600), (2600, 650),
          (1023, 511)]


@pytest.mark.parametrize("r,c", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_matches_the_steps(r, c, dtype):
    u = matrix(r, c, dtype)
    check(u, run([u])[0])


@pytest.mark.parametrize("r,c", [(60, 500), (128, 200), (200, 128), (300, 900), (900, 300)])
@pytest.mark.parametrize("pad,offset", [(1, 1), (2, 2), (4, 0), (8, 8), (3, 5)])
def test_strides_and_alignment(r, c, pad, offset):
    for dtype in (torch.float32, torch.bfloat16):
        u = matrix(r, c, dtype, pad=pad, offset=offset)
        check(u, run([u], pad=pad, offset=offset)[0])


@pytest.mark.parametrize("r,c", [(64, 300), (300, 64), (200, 500), (700, 260)])
@pytest.mark.parametrize("kind", ["decades", "low"])
def test_small_singular_values(r, c, kind):
    u = matrix(r, c, kind=kind)
    if kind == "low":  # directions of U's own rounding are amplified alike by both
        u = u.double().float()
    check(u, run([u])[0])


@pytest.mark.parametrize("shapes", [[(64, 27), (64, 576), (64, 576), (10, 512)],
                                    [(300, 200), (64, 64), (200, 300), (650, 300)],
                                    [(130 + i, 140) for i in range(15)],
                                    [(3 + i, 20) for i in range(80)]])
def test_lists_and_momentum(shapes):
    us = [matrix(r, c, seed=i) for i, (r, c) in enumerate(shapes)]
    ms = [matrix(r, c, seed=100 + i) for i, (r, c) in enumerate(shapes)]
    before = [m.clone() for m in ms]
    outs = run(us, ms, 0.875)
    for u, m, old, out in zip(us, ms, before, outs):
        # one fused multiply-add: exact in 64 bits (0.875 is), then one rounding
        assert torch.equal(m, (0.875 * old.double() + u.double()).float())
        check((u + m), out)


def test_values_pull_to_one():
    out = run([matrix(200, 700)])[0].double()
    s = torch.linalg.svdvals(out)
    assert float(s.min()) > 0.6 and float(s.max()) < 1.3


def test_scale_does_not_matter():
    u = matrix(150, 400)
    ref = run([u])[0]
    for k in (2.0 ** -30, 2.0 ** 40):  # powers of two: the same bits
        assert torch.equal(run([u * k])[0], ref)


def test_zero_and_what_is_not_a_number():
    for shape in ((20, 50), (200, 300)):
        z = torch.zeros(shape, device=DEV)
        assert (run([z])[0] == 0).all()
        for bad in (float("nan"), float("inf")):
            u = matrix(*shape)
            u[3, 4] = bad
            other = matrix(*shape, seed=9)
            out = run([u, other])
            assert torch.isnan(out[0]).all()
            check(other, out[1])


def test_empty_matrices_are_passed_over():
    u = matrix(30, 40)
    empty = [torch.empty(0, 5, device=DEV), torch.empty(5, 0, device=DEV)]
    outs = [torch.empty(x.shape, device=DEV, dtype=torch.bfloat16) for x in (empty[0], u, empty[1])]
    efs.ef_orthogonalize([empty[0], u, empty[1]], outs)
    check(u, outs[1])
    efs.ef_orthogonalize(empty, [outs[0], outs[2]])
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.parametrize("shapes", [[(64, 576)], [(300, 500), (64, 64)], [(513, 1025)]])
def test_equal_inputs_give_equal_bits(shapes):
    us = [matrix(r, c) for r, c in shapes]
    first = run(us)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(run(us), first))


@pytest.mark.parametrize("shapes", [[(64, 576)], [(300, 500), (64, 64)]])
def test_other_stream_and_capture(shapes):
    us = [matrix(r, c) for r, c in shapes]
    ref = run(us)
    outs = [torch.empty_like(x) for x in ref]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(2):  # the stream's workspace grows outside the capture
            efs.ef_orthogonalize(us, outs)
    s.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, ref))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        efs.ef_orthogonalize(us, outs)
    for x in outs:
        x.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, ref))


def test_refuses_overlap_and_shapes():
    u = matrix(20, 30)
    out = torch.empty(20, 30, device=DEV, dtype=torch.bfloat16)
    with pytest.raises(efs.EfError):
        efs.ef_orthogonalize([u], [out], momenta=[u], momentum=0.5)
    with pytest.raises(efs.EfError):
        efs.ef_orthogonalize([u, u], [out, out])
    with pytest.raises(ValueError):
        efs.ef_orthogonalize([u], [out[:, :29]])
    with pytest.raises(ValueError):
        efs.ef_orthogonalize([u.T], [torch.empty(30, 20, device=DEV, dtype=torch.bfloat16)])
    with pytest.raises(TypeError):
        efs.ef_orthogonalize([u, u.bfloat16()], [out, out.clone()])


@pytest.mark.parametrize("cols", [(27, 576), (100, 700, 1152), (64, 300, 500, 900, 1152)])
def test_small_matrices_of_few_and_of_many_shapes(cols):
    us = [matrix(64 + 16 * (i % 3), c, seed=i) for i, c in enumerate(cols)]
    moms = [torch.randn_like(u) * 1e-3 for u in us]
    want = [0.9 * m.double() + u.double() for m, u in zip(moms, us)]
    outs = run(us, moms, 0.9)
    for u, m, w, out in zip(us, moms, want, outs):
        assert float((m.double() - w).abs().max()) <= 2.0 ** -23 * float(w.abs().max())
        check(u.double() + m.double(), out)

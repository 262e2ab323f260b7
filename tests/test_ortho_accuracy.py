"""How far orthogonalised updates are from the steps in 64 bits, beside the
rounding of their bf16 output.

With e = |bf16(ref) - ref| (about 1.65e-3 |ref|) and an error before the rounding
of at most p |ref|, independent of it, the outputs are within sqrt(e^2 +
(p |ref|)^2) of ref; the roundings' own spread over a few hundred entries and more
is below 2 %. p = 1e-4 where the shorter side is at most 128 (operands hi + lo of
fp16, 22 bits): at most 1.002 e. Operands of one fp16 plane would leave 1e-3 there,
1.17 e. p = 2e-3 for larger sides."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

DEV = "cuda"


def steps(x, operand=lambda y: y):
    """Five steps on the shorter side; `operand` is applied to what a product reads."""
    x = x / x.norm()
    if x.shape[0] > x.shape[1]:
        return steps(x.T, operand).T
    for _ in range(5):
        o = operand(x)
        a = o @ o.T
        o = operand(a)
        b = -4.7750 * o + 2.0315 * (o @ o)
        x = 3.4445 * x + operand(b) @ operand(x)
    return x


def matrix(r, c, kind, device):
    g = torch.Generator(device=device).manual_seed(31 * r + c)
    x = torch.randn(r, c, device=device, generator=g)
    if kind == "decades":  # singular values over four decades
        k = min(r, c)
        q = torch.linalg.qr(torch.randn(k, k, device=device, generator=g))[0]
        s = torch.logspace(0, -4, k, device=device)
        x = (q * s) @ x if r <= c else x @ (s[:, None] * q.T)
    elif kind == "strong":
        k = min(4, r, c)
        x += 0.5 * (torch.randn(r, k, device=device, generator=g)
                    @ torch.randn(k, c, device=device, generator=g))
    return (x * 1e-3).float()


def within(out, ref, p):
    e = float((ref.bfloat16().double() - ref).norm())
    return float((out.double() - ref).norm()) <= 1.02 * (e ** 2 + (p * float(ref.norm())) ** 2) ** 0.5


SMALL = [(1, 300), (300, 1), (5, 640), (17, 33), (64, 576), (576, 64), (128, 128), (127, 2000),
         (2000, 127), (64, 4096), (128, 5000), (9000, 3)]
LARGE = [(129, 129), (129, 1000), (1000, 129), (256, 256), (300, 333), (650, 2600), (2600, 650)]


@pytest.mark.gpu
@pytest.mark.parametrize("r,c", SMALL + LARGE)
@pytest.mark.parametrize("kind", ["noise", "strong", "decades"])
def test_error_beside_the_rounding(r, c, kind):
    u = matrix(r, c, kind, DEV)
    out = torch.empty(r, c, device=DEV, dtype=torch.bfloat16)
    efs.ef_orthogonalize([u], [out])
    assert efs.ef_check_status() == efs.EF_OK
    assert within(out, steps(u.double()), 1e-4 if min(r, c) <= 128 else 2e-3)


@pytest.mark.gpu
def test_small_sides_in_the_phases():
    # more than three layouts: the list goes through the phases
    shapes = [(64, 200), (64, 576), (100, 900), (128, 1152), (33, 2000), (900, 100), (120, 3000)]
    us = [matrix(r, c, "strong", DEV) for r, c in shapes]
    outs = [torch.empty(u.shape, device=DEV, dtype=torch.bfloat16) for u in us]
    efs.ef_orthogonalize(us, outs)
    assert efs.ef_check_status() == efs.EF_OK
    for u, out in zip(us, outs):
        assert within(out, steps(u.double()), 1e-4), tuple(u.shape)


@pytest.mark.parametrize("r,c", [(64, 576), (128, 128), (64, 300)])
@pytest.mark.parametrize("kind", ["noise", "strong"])
def test_the_bound_shows_a_lost_plane(r, c, kind):
    u = matrix(r, c, kind, "cpu").double()
    ref = steps(u)

    def plane(y):  # fp16's 11 bits, scaled as the kernels' operands are
        return (y * 8192).half().double() / 8192

    def planes(y):
        return plane(y) + plane((y - plane(y)) * 2048) / 2048
    assert not within(steps(u, plane).bfloat16(), ref, 1e-4)
    assert within(steps(u, planes).bfloat16(), ref, 1e-4)

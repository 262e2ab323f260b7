"""Orthogonalised updates large enough for pairs of CTAs (the symmetric products'
256 x 256 tiles on and below the diagonal fill half of the SMs: 76 of them on 152),
and lists of more than 48 matrices through the phases, against the steps in 64 bits.

Bounds as for smaller ones, relative in the 2-norm: 2e-3 before the rounding of
the bf16 output (1e-4 where the shorter side is at most 128), that rounding at
most 2^-8."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def exact(u):
    x = u.double()
    x = x / x.norm()
    left = x.shape[0] <= x.shape[1]
    for _ in range(5):
        g = x @ x.T if left else x.T @ x
        p = -4.7750 * g + 2.0315 * (g @ g)
        x = 3.4445 * x + (p @ x if left else x @ p)
    return x


def matrix(r, c, seed, dtype=torch.float32, pad=0):
    """Rows `pad` entries further apart; a few strong directions over noise."""
    g = torch.Generator(device=DEV).manual_seed(1000003 * r + 1009 * c + seed)
    x = torch.randn(r, c, device=DEV, generator=g)
    k = min(4, r, c)
    x += 0.5 * (torch.randn(r, k, device=DEV, generator=g) @ torch.randn(k, c, device=DEV, generator=g))
    m = torch.empty(r, c + pad, device=DEV, dtype=dtype)[:, :c]
    m.copy_(x * 1e-3)
    return m


def outputs(us, pad=0):
    return [torch.full((u.shape[0], u.shape[1] + pad), float("nan"), device=DEV,
                       dtype=torch.bfloat16)[:, :u.shape[1]] for u in us]


def check(u, out):
    ref = exact(u)
    tol = (1e-4 if min(u.shape) <= 128 else 2e-3) + 2.0 ** -8
    assert float((out.double() - ref).norm()) <= tol * float(ref.norm()), tuple(u.shape)


@pytest.mark.parametrize("r,c", [(3100, 3333), (3333, 3100), (3200, 3200), (2999, 3500)])
@pytest.mark.parametrize("dtype,pad", [(torch.float32, 0), (torch.bfloat16, 3)])
def test_one_large_matrix(r, c, dtype, pad):
    u = matrix(r, c, 1, dtype, pad)
    out, again = outputs([u], pad), outputs([u], pad)
    efs.ef_orthogonalize([u], out)
    efs.ef_orthogonalize([u], again)
    assert efs.ef_check_status() == efs.EF_OK
    check(u, out[0])
    assert torch.equal(out[0], again[0])


LISTS = {
    "one shape": [(300, 400)] * 26,
    "tall and wide": [(300, 400), (400, 300), (257, 700), (700, 257)] * 7,
    # sides up to 128 (operands hi + lo) beside larger ones, more shapes than a launch takes
    "sides of 64 to 300": [(64 + 13 * (i % 19), 150 + 41 * (i % 7)) for i in range(100)],
    # joined K parts in pairs: few tiles each, deep
    "deep": [(200, 3000), (3000, 200), (512, 2304)] * 9 + [(100, 5000)] * 20 + [(5000, 100)] * 20,
    # two preparing launches, without pairs
    "many": [(150, 200), (200, 150), (129, 260)] * 20,
}


@pytest.mark.parametrize("name", sorted(LISTS))
@pytest.mark.parametrize("momentum", [None, 0.875])
def test_lists(name, momentum):
    us = [matrix(r, c, i) for i, (r, c) in enumerate(LISTS[name])]
    before = None if momentum is None else [matrix(r, c, 500 + i) for i, (r, c) in enumerate(LISTS[name])]
    runs = []
    for _ in range(2):
        ms = None if before is None else [m.clone() for m in before]
        outs = outputs(us)
        efs.ef_orthogonalize(us, outs, momenta=ms, momentum=momentum or 0.0)
        assert efs.ef_check_status() == efs.EF_OK
        runs.append((outs, ms or []))
    for x, y in zip(runs[0][0] + runs[0][1], runs[1][0] + runs[1][1]):
        assert torch.equal(x, y)
    outs, ms = runs[0]
    for i, u in enumerate(us):
        if ms:  # one fused multiply-add, exact in 64 bits (0.875 is), then one rounding
            assert torch.equal(ms[i], (momentum * before[i].double() + u.double()).float())
            check(u + ms[i], outs[i])
        else:
            check(u, outs[i])

"""AdamW over lists of tensors against the formulas in 64 bits, and its 8-bit
states against their definition.

Bounds, u = 2^-24: m is two products and a sum, each rounded, of constants rounded
to fp32: 4 u of its terms; v, a product more: 5 u. The update's root and quotient
are good to 2^-21 together, so p is off by 2^-20 lr |update| and 3 u |p|."""
import math

import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24
B1, B2, LR, EPS, WD = 0.9, 0.999, 1e-2, 1e-8, 0.1


def views(sizes, dtype, offset, gen, scale=1.0, positive=False):
    """Tensors of the sizes one behind another in a buffer, from `offset` on."""
    flat = torch.empty(sum(sizes) + offset, device=DEV, dtype=dtype)[offset:]
    x = torch.randn(sum(sizes), device=DEV, generator=gen) * scale
    flat.copy_(x.abs() if positive else x)
    return flat, list(flat.split(sizes))


SIZES = [[1], [5000], [4096, 4097, 3], [64, 128, 10, 512, 0, 1, 9000], [7] * 30, [130000, 1, 2, 3]]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("gt,offset,copy", [(F32, 0, False), (BF16, 0, True), (F32, 1, True), (BF16, 3, False)])
def test_matches_the_formulas(sizes, gt, offset, copy):
    g = torch.Generator(device=DEV).manual_seed(sum(sizes))
    p, ps = views(sizes, F32, offset, g)
    gr, gs = views(sizes, gt, offset, g, 0.1)
    m, ms = views(sizes, F32, offset, g, 0.1)
    v, vs = views(sizes, F32, offset, g, 0.01, True)
    c, cs = views(sizes, BF16, offset, g)
    for step in (1, 7, 3000):
        p0, g0, m0, v0 = (t.double() for t in (p, gr, m, v))
        efs.ef_adamw(ps, gs, ms, vs, step, LR, B1, B2, EPS, WD, copies=cs if copy else None)
        m1, v1 = B1 * m0 + (1 - B1) * g0, B2 * v0 + (1 - B2) * g0 * g0
        up = (m1 / (1 - B1 ** step)) / ((v1 / (1 - B2 ** step)).sqrt() + EPS)
        p1 = p0 * (1 - LR * WD) - LR * up
        assert bool(((m.double() - m1).abs() <= 4 * U * (m0.abs() + 0.1 * g0.abs())).all())
        assert bool(((v.double() - v1).abs() <= 5 * U * v1).all())
        # (an m whose terms cancel has a larger relative error, which p takes over)
        dm = 4 * U * (m0.abs() + 0.1 * g0.abs()) / m1.abs().clamp(min=1e-30)
        assert bool(((p.double() - p1).abs() <= (2.0 ** -20 + dm) * LR * up.abs() + 3 * U * p0.abs()).all())
        if copy:
            assert torch.equal(c, p.bfloat16())


def test_many_tensors():
    """More than one launch takes."""
    sizes = [(37 * i) % 301 for i in range(1000)]
    g = torch.Generator(device=DEV).manual_seed(1)
    p, ps = views(sizes, F32, 0, g)
    gr, gs = views(sizes, F32, 0, g)
    (m, ms), (v, vs) = views(sizes, F32, 0, g), views(sizes, F32, 0, g, 1.0, True)
    q, n, w = p.clone(), m.clone(), v.clone()
    efs.ef_adamw(ps, gs, ms, vs, 3, LR)
    efs.ef_adamw([q], [gr], [n], [w], 3, LR)
    assert torch.equal(p, q) and torch.equal(m, n) and torch.equal(v, w)


def test_values_at_the_ends():
    """Zeros, infinities, NaN, subnormal and huge gradients stay in their entries."""
    vals = [0.0, math.inf, -math.inf, math.nan, 1e-42, 1e19, 3e38, -1e-30, 1.0]
    gr = torch.tensor(vals * 30, device=DEV)
    p, m, v = torch.ones_like(gr), torch.zeros_like(gr), torch.zeros_like(gr)
    efs.ef_adamw([p], [gr], [m], [v], 1, LR, B1, B2, EPS, 0.0)
    p, m, v = p.view(30, -1), m.view(30, -1), v.view(30, -1)
    assert torch.equal(p[0, [0, 4, 8]], p[29, [0, 4, 8]])
    assert bool((p[:, 0] == 1.0).all()) and bool((m[:, 0] == 0.0).all())
    assert bool(p[:, 3].isnan().all()) and bool(v[:, 3].isnan().all())
    assert bool(p[:, [0, 4, 5, 7, 8]].isfinite().all())
    assert bool((p[:, 8] == p[0, 8]).all()) and abs(float(p[0, 8]) - (1 - LR)) < 1e-6


def test_device_scalars_and_gradient_scale():
    g = torch.Generator(device=DEV).manual_seed(2)
    x = [torch.randn(5000, device=DEV, generator=g) for _ in range(4)]
    x[3].abs_()
    a, b = [t.clone() for t in x], [t.clone() for t in x]
    efs.ef_adamw([a[0]], [a[1] * 0.25], [a[2]], [a[3]], 12, 3e-3, weight_decay=0.02)
    efs.ef_adamw([b[0]], [b[1]], [b[2]], [b[3]], torch.tensor([12], device=DEV),
                 torch.tensor([3e-3], device=DEV), weight_decay=0.02, grad_scale=torch.tensor([0.25], device=DEV))
    assert torch.equal(a[2], b[2]) and torch.equal(a[3], b[3])
    assert float((a[0] - b[0]).abs().max()) < 2.0 ** -20 * 3e-3 * 10 + 2.0 ** -23 * 5
    c = [t.clone() for t in x]
    efs.ef_adamw([c[0]], [c[1] * 0.25], [c[2]], [c[3]], 12, torch.tensor(3e-3, device=DEV), weight_decay=0.02)
    assert float((a[0] - c[0]).abs().max()) < 2.0 ** -23 * 5


# ------------------------------------------------------------ states in 8 bits
def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(seed, step, k, n):
    key = mix(mix(seed & 0xFFFFFFFF) ^ (seed >> 32))
    key = mix((mix((key + step) & 0xFFFFFFFF) + 0x9E3779B9 * k) & 0xFFFFFFFF)
    return mix((torch.arange(n) + key) & 0xFFFFFFFF)


def values(codes, exponents, signed):
    """In 64 bits, from the definition."""
    n, top = codes.numel(), 14 if signed else 30
    c = codes.cpu().long()
    a = c & 127 if signed else c
    e = exponents.cpu().long().clamp(min=35).repeat_interleave(128)[:n] - 127
    f, k = a >> 3, a & 7
    x = torch.where(f > 0, (8.0 + k) * 2.0 ** (e - top + f - 3).double(), k * 2.0 ** (e - top - 2).double())
    x = torch.where(a == (127 if signed else 255), math.nan, x)
    return torch.where(c != a, -x, x)


def held(x, signed, r):
    """Codes and exponents of fp32 values x with the 16 random bits r, in 64 bits."""
    n, top = x.numel(), 14 if signed else 30
    x = x.cpu().double()
    fine = x.abs() < 2.0 ** 127
    mag = torch.where(fine, x.abs(), 0.0)
    blocks = torch.zeros((n + 127) // 128 * 128, dtype=torch.float64)
    blocks[:n] = mag
    e = torch.frexp(blocks.view(-1, 128).amax(1))[1] - 1
    e = torch.where(blocks.view(-1, 128).amax(1) > 0, e, -92).clamp(min=-92)
    low = (e - top + 1).repeat_interleave(128)[:n]
    at = torch.where(mag > 0, torch.maximum(torch.frexp(mag)[1] - 1, low), low)
    code = (at - low) * 8 + torch.floor(torch.ldexp(mag, 3 - at) + (r + 0.5) / 65536).long()
    if not signed:
        code = torch.where((code == 0) & (mag > 0), 1, code)
    code = torch.where(fine, code, 127 if signed else 255)
    code = code + 128 * torch.signbit(x) if signed else code
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def eight(sizes, offset=0):
    codes = [torch.zeros(n + offset, device=DEV, dtype=torch.uint8)[offset:] for n in sizes]
    return codes, [torch.zeros(efs.exponents_for(n), device=DEV, dtype=torch.uint8) for n in sizes]


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("gt,offset,copy", [(F32, 0, False), (BF16, 0, True), (F32, 1, True)])
def test_states_in_8_bits(sizes, gt, offset, copy):
    g = torch.Generator(device=DEV).manual_seed(sum(sizes))
    p, ps = views(sizes, F32, offset, g)
    c, cs = views(sizes, BF16, offset, g)
    (m, me), (v, ve) = eight(sizes, offset), eight(sizes, offset)
    seed = 0x123456789ABC
    for step in (1, 2, 3, 40):
        scale = torch.exp(4 * torch.randn(sum(sizes), device=DEV, generator=g))
        gr, gs = views(sizes, gt, offset, g, scale)
        m0 = [values(a, b, True) for a, b in zip(m, me)]
        v0 = [values(a, b, False) for a, b in zip(v, ve)]
        p0 = [t.double().cpu() for t in ps]
        efs.ef_adamw(ps, gs, m, v, step, LR, B1, B2, EPS, WD, me, ve, cs if copy else None, seed=seed)
        mo, vo = [[torch.empty(n, device=DEV, dtype=dt) for n in sizes] for dt in (F32, F32)]
        efs.ef_adamw_states(m, v, me, ve, mo, vo)
        for k, n in enumerate(sizes):
            if n == 0:
                continue
            # fp32, each operation rounded
            g32 = gs[k].float().cpu()
            m1 = m0[k].float() * B1 + g32 * (1 - B1)
            v1 = v0[k].float() * B2 + g32 * g32 * (1 - B2)
            r = random_bits(seed, step, k, n)
            for got, ex, want in ((m[k], me[k], held(m1, True, r & 0xFFFF)),
                                  (v[k], ve[k], held(v1, False, r >> 16))):
                assert torch.equal(got.cpu(), want[0]) and torch.equal(ex.cpu(), want[1])
            assert torch.equal(mo[k].cpu().double(), values(m[k], me[k], True))
            assert torch.equal(vo[k].cpu().double(), values(v[k], ve[k], False))
            up = (m1.double() / (1 - B1 ** step)) / ((v1.double() / (1 - B2 ** step)).sqrt() + EPS)
            p1 = p0[k] * (1 - LR * WD) - LR * up
            off = (ps[k].double().cpu() - p1).abs()
            assert bool((off <= 2.0 ** -20 * LR * up.abs() + 3 * U * p0[k].abs()).all())
        if copy:
            assert torch.equal(c, p.bfloat16())


def test_8_bit_values_at_the_ends():
    n = 128 * 6 + 5
    vals = [math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, 2e-38, 1.5, 3e38, -3e38, 1e19, 1e-19]
    gr = torch.tensor((vals * 100)[:n], device=DEV)
    gr[128:256] = 0.0
    gr[256:384] = 1e-30
    p = torch.ones(n, device=DEV)
    (m, me), (v, ve) = eight([n]), eight([n])
    for step in (1, 2):
        m0, v0 = values(m[0], me[0], True), values(v[0], ve[0], False)
        efs.ef_adamw([p], [gr], m, v, step, LR, B1, B2, EPS, 0.0, me, ve, seed=9)
        m1 = m0.float() * B1 + gr.cpu() * (1 - B1)
        v1 = v0.float() * B2 + gr.cpu() * gr.cpu() * (1 - B2)
        r = random_bits(9, step, 0, n)
        for got, ex, x, signed, bits in ((m[0], me[0], m1, True, r & 0xFFFF), (v[0], ve[0], v1, False, r >> 16)):
            codes, exps = held(x, signed, bits)
            nan = 127 if signed else 255
            # (the sign of a NaN is not part of the result)
            a, b = got.cpu() & nan, codes & nan
            assert torch.equal(a, b) and torch.equal(ex.cpu(), exps)
    assert bool((p[128:256] == 1.0).all())
    out = [torch.empty(n, device=DEV, dtype=BF16) for _ in range(2)]
    efs.ef_adamw_states(m, v, me, ve, [out[0]], [out[1]])
    want = values(v[0], ve[0], False)
    assert torch.equal(out[1].double().cpu().nan_to_num(-1.0), want.nan_to_num(-1.0))
    assert bool((values(v[0], ve[0], False)[v1 > 0] > 0).all())


def test_rounding_is_unbiased():
    """v of constant gradients, which rounding to nearest would stop below a tenth of
    its value, follows the average in fp32. The rounding of one step moves an entry by a
    step of at most v / 8 with a probability that makes its mean right: after t steps of
    b2 = 0.99 the deviations of an entry add up to a variance of at most
    (0.01 v)(v / 8) / (1 - 0.99^2), 0.063 v^2; the mean over 2^16 entries is within 6 deviations
    of 0.25 / 256 of the right one."""
    n = 1 << 16
    p, gr = torch.zeros(n, device=DEV), torch.full((n,), 0.5, device=DEV)
    (m, me), (v, ve) = eight([n]), eight([n])
    for step in range(1, 301):
        efs.ef_adamw([p], [gr], m, v, step, 0.0, 0.9, 0.99, EPS, 0.0, me, ve, seed=4)
    mean = float(values(v[0], ve[0], False).mean())
    want = 0.25 * (1 - 0.99 ** 300)
    assert abs(mean - want) < 6 * 0.25 / 256 * want
    mean = float(values(m[0], me[0], True).mean())
    # m: steps of at most m / 8 ten times as often: (0.1 m)(m / 8) / (1 - 0.81) = 0.066 m^2
    assert abs(mean - 0.5 * (1 - 0.9 ** 300)) < 6 * 0.26 / 256 * 0.5


def test_seeds_steps_and_tensors_round_differently():
    def codes(seed, step, k):
        sizes = [300] * (k + 1)
        g = torch.Generator(device=DEV).manual_seed(5)
        x = torch.randn(300, device=DEV, generator=g)
        (m, me), (v, ve) = eight(sizes), eight(sizes)
        efs.ef_adamw([torch.zeros(300, device=DEV) for _ in sizes], [x.clone() for _ in sizes], m, v, step, 0.0,
                     m_exponents=me, v_exponents=ve, seed=seed)
        return torch.cat([m[k], v[k]])
    first = codes(1, 1, 0)
    assert torch.equal(first, codes(1, 1, 0))
    for other in (codes(2, 1, 0), codes(1, 2, 0), codes(1, 1, 1), codes(1 + (1 << 32), 1, 0)):
        assert 60 < int((other != first).sum()) < 540  # of 600, a third or so


def test_a_tensor_list_is_the_list():
    g = torch.Generator(device=DEV).manual_seed(6)
    x = [[torch.rand(n, device=DEV, generator=g) for n in (300, 5)] for _ in range(4)]
    y = [[t.clone() for t in row] for row in x]
    efs.ef_adamw(*x, 2, LR)
    efs.ef_adamw(*[efs.TensorList(row) for row in y], 2, LR)
    assert all(torch.equal(a, b) for r, s in zip(x, y) for a, b in zip(r, s))

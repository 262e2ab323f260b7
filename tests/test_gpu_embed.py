"""Embedding rows by token and the table's gradient, against the formulas in 64 bits.

Bounds. A row of the lookup is one fp32 product, rounded to the output's type. A
sum of k rows in fp32 is off by at most k 2^-24 of the sum of their magnitudes,
its product with the scale (and its addition to what was there) by 2^-24 of the
result, then the result is rounded to the table's type."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16


def matrix(rows, cols, dtype, pad=0, offset=0, gen=None, scale=1.0):
    buf = torch.full((rows * (cols + pad) + offset,), 7.0, device=DEV, dtype=dtype)
    m = buf[offset:].view(rows, cols + pad)[:, :cols]
    if gen is not None:
        m.copy_(torch.randn(rows, cols, device=DEV, generator=gen) * scale)
    return m, buf


def around(m, buf, offset):
    """The entries of buf outside its matrix."""
    keep = torch.ones_like(buf, dtype=torch.bool)
    cols = m.shape[1]
    keep[offset:].view(m.shape[0], -1)[:, :cols] = False
    return buf[keep]


def tokens(n, v, gen, padding=0.2):
    t = torch.exp(torch.rand(n, device=DEV, generator=gen) * torch.log(torch.tensor(float(v)))).long() - 1
    t = t.clamp(0, v - 1)
    t[torch.rand(n, device=DEV, generator=gen) < padding] = -1 - torch.randint(0, 1 << 40, (1,)).item()
    return t


LAYOUTS = [(BF16, BF16, 0, 0), (F32, F32, 0, 0), (F32, BF16, 2, 2), (BF16, F32, 3, 1), (BF16, BF16, 6, 2)]


@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (1, 50, 650), (16, 28869, 650), (3, 7, 1023), (700, 31, 8),
                                   (513, 1000, 96), (5000, 300, 257), (2, 3, 9000)])
@pytest.mark.parametrize("tt,ot,pad,offset", LAYOUTS)
def test_lookup(n, v, d, tt, ot, pad, offset):
    g = torch.Generator(device=DEV).manual_seed(n + v + d)
    table, _ = matrix(v, d, tt, pad, offset, g)
    out, buf = matrix(n, d, ot, pad, offset)
    t = tokens(n, v, g)
    efs.ef_embed(table, t, out, scale=1.7)
    ref = table.double()[t.clamp(min=0)] * float(torch.tensor(1.7)) * (t >= 0)[:, None]
    off = (out.double() - ref).abs()
    assert bool((off <= (torch.finfo(ot).eps / 2 + 2.0 ** -24) * (1 + 2.0 ** -8) * ref.abs()).all())
    assert bool((around(out, buf, offset) == 7.0).all())
    assert efs.ef_check_status() == efs.EF_OK


def check_gradient(n, v, d, dt, tt, pad, offset, add, seed=0, t=None, scale=0.37):
    g = torch.Generator(device=DEV).manual_seed(n + v + d + seed)
    dout, _ = matrix(n, d, dt, pad, offset, g)
    dtable, buf = matrix(v, d, tt, pad, offset, g if add else None)
    t = tokens(n, v, g) if t is None else t
    before = dtable.double().clone()
    dout[t < 0] = float("nan")  # (padding is not used)
    efs.ef_embed_grad(dout, t, dtable, scale=scale, accumulate=add)
    keep = t >= 0
    s = float(torch.tensor(scale))
    rows = dout[keep].double()
    zero = torch.zeros(v, d, device=DEV, dtype=torch.float64)
    ref = zero.index_add(0, t[keep], rows) * s
    mag = zero.index_add(0, t[keep], rows.abs()) * s
    count = torch.zeros(v, device=DEV, dtype=torch.float64).index_add(0, t[keep], torch.ones_like(rows[:, 0]))
    if add:
        untouched = count == 0
        assert torch.equal(dtable[untouched].double(), before[untouched])
        ref = ref + before
    bound = (count[:, None] + 2) * 2.0 ** -24 * mag + (torch.finfo(tt).eps / 2) * ref.abs() * (1 + 2.0 ** -8)
    # (the addition to what was there may round a sum that then cancels)
    bound = bound + 2.0 ** -24 * ref.abs() + 2.0 ** -140
    assert bool(((dtable.double() - ref).abs() <= bound).all())
    assert bool((around(dtable, buf, offset) == 7.0).all())
    assert efs.ef_check_status() == efs.EF_OK
    return dout, t, dtable


@pytest.mark.parametrize("n,v,d", [(1, 1, 1), (2, 5, 3), (700, 900, 650), (33, 4000, 1001), (2048, 40, 72),
                                   (2049, 300, 257), (2500, 1, 8), (4096, 511, 96), (4097, 512, 130),
                                   (10000, 100000, 33), (70001, 3000, 64), (20000, 300000, 16)])
@pytest.mark.parametrize("dt,tt,pad,offset", LAYOUTS)
@pytest.mark.parametrize("add", [False, True])
def test_gradient(n, v, d, dt, tt, pad, offset, add):
    check_gradient(n, v, d, dt, tt, pad, offset, add)


@pytest.mark.parametrize("n", [600, 2048, 2049, 40000, 65536, 131075])
@pytest.mark.parametrize("kind", ["one", "none", "two", "runs", "last"])
def test_gradient_of_uneven_tokens(n, kind):
    v, d = 777, 300
    t = {"one": torch.full((n,), 5, device=DEV), "none": torch.full((n,), -1, device=DEV),
         "two": torch.arange(n, device=DEV) % 2 * (v - 1),
         "runs": (torch.arange(n, device=DEV) // 97) % v,
         "last": torch.where(torch.arange(n, device=DEV) == n - 1, v - 1, 3)}[kind]
    check_gradient(n, v, d, BF16, F32, 0, 0, False, t=t)
    check_gradient(n, v, d, F32, BF16, 0, 0, True, t=t)


def test_long_lists():
    """Sorting CTAs of several tiles, and tokens with thousands of shares."""
    for n, v, d in ((700003, 5000, 8), (620000, 3, 40)):
        g = torch.Generator(device=DEV).manual_seed(n)
        t = tokens(n, v, g, padding=0.01)
        check_gradient(n, v, d, BF16, F32, 0, 0, False, t=t)
        check_gradient(n, v, d, F32, BF16, 0, 0, True, t=t)
    t = torch.full((400000,), 1, device=DEV)
    t[-1] = 2
    check_gradient(400000, 4, 24, BF16, F32, 0, 0, False, t=t)
    check_gradient(400000, 4, 600, BF16, BF16, 0, 0, False, t=t)


@pytest.mark.parametrize("seed", range(4))
def test_runs_of_many_pieces(seed):
    """Words that go on over some, 16, 17 and many pieces of the sorted list, and begin where
    the last piece of another one lies."""
    g = torch.Generator().manual_seed(seed)
    runs = [16 * 16, 16 * 17, 16 * 16 - 1, 16 * 16 + 1, 16 * 17 + 1, 1, 16 * 32, 16 * 33 + 5, 3, 16 * 48 + 2, 17, 16]
    runs += torch.randint(1, 1200, (16,), generator=g).tolist()
    for factor in (1, 4):  # pieces of 16 positions and of more
        t = torch.repeat_interleave(torch.arange(len(runs)) + 1, torch.tensor(runs) * factor)
        t = torch.cat([torch.full((seed * 5,), 0), t])
        t = t[torch.randperm(t.numel(), generator=g)].to(DEV)
        check_gradient(t.numel(), len(runs) + 2, 40, BF16, F32, 0, 0, False, t=t)
        check_gradient(t.numel(), len(runs) + 2, 33, F32, BF16, 0, 0, True, t=t)
        check_gradient(t.numel(), len(runs) + 2, 520, BF16, BF16, 0, 0, True, t=t)
        check_gradient(t.numel(), len(runs) + 2, 520, BF16, BF16, 0, 0, False, t=t)


@pytest.mark.parametrize("n,v,d", [(500, 60, 5000), (1000, 300, 2500), (1200, 30, 700), (90, 20, 9999), (257, 40, 9217),
                                   (256, 40, 9300)])
def test_gradient_of_wide_rows(n, v, d):
    check_gradient(n, v, d, BF16, F32, 0, 0, False)
    check_gradient(n, v, d, F32, BF16, 0, 0, True)
    check_gradient(n, v, d, F32, BF16, 3, 1, False)


def test_many_digits():
    """Words beyond two digits of nine bits, and beyond three."""
    for v in ((1 << 18) - 1, 1 << 18, (1 << 27) + 5):
        g = torch.Generator(device=DEV).manual_seed(v)
        n, d = 5000, 4
        t = torch.randint(0, v, (n,), device=DEV, generator=g)
        t[:1000] = t[1000:2000]
        t[17] = v - 1
        dout = torch.randn(n, d, device=DEV, generator=g)
        dtable = torch.full((v, d), 3.0, device=DEV)
        efs.ef_embed_grad(dout, t, dtable, accumulate=True)
        words, at = torch.unique(t, return_inverse=True)
        ref = torch.zeros(len(words), d, device=DEV, dtype=torch.float64).index_add(0, at, dout.double()) + 3.0
        assert bool(((dtable[words].double() - ref).abs() < 8 * 2.0 ** -22).all())
        dtable[words] = 3.0
        assert bool((dtable == 3.0).all())
        del dtable


@pytest.mark.parametrize("n", [300, 9000])
def test_equal_inputs_give_equal_bits(n):
    g = torch.Generator(device=DEV).manual_seed(n)
    dout = torch.randn(n, 320, device=DEV, generator=g)
    t = tokens(n, 200, g)
    out = [torch.empty(200, 320, device=DEV) for _ in range(3)]
    for o in out:
        efs.ef_embed_grad(dout, t, o)
    assert torch.equal(out[0], out[1]) and torch.equal(out[0], out[2])


@pytest.mark.parametrize("n", [5, 300, 5000])
def test_bad_tokens_are_latched(n):
    v, d = 100, 24
    g = torch.Generator(device=DEV).manual_seed(n)
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    good = t.clone()
    t[n // 2], good[n // 2] = v, -1
    t[0], good[0] = 1 << 62, -1
    table = torch.randn(v, d, device=DEV, generator=g)
    out, want = torch.empty(n, d, device=DEV), torch.empty(n, d, device=DEV)
    efs.ef_embed(table, t, out)
    assert efs.ef_check_status() == efs.EF_ERR_BAD_INPUT
    efs.ef_embed(table, good, want)
    assert efs.ef_check_status() == efs.EF_OK
    assert torch.equal(out, want)
    dt, want = torch.empty(v, d, device=DEV), torch.empty(v, d, device=DEV)
    efs.ef_embed_grad(out, t, dt)
    assert efs.ef_check_status() == efs.EF_ERR_BAD_INPUT
    efs.ef_embed_grad(out, good, want)
    assert efs.ef_check_status() == efs.EF_OK
    assert torch.equal(dt, want)


def test_no_tokens():
    table = torch.randn(30, 8, device=DEV)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    efs.ef_embed(table, none, torch.empty(0, 8, device=DEV))
    out = torch.full((30, 8), 2.0, device=DEV)
    efs.ef_embed_grad(torch.empty(0, 8, device=DEV), none, out, accumulate=True)
    assert bool((out == 2.0).all())
    efs.ef_embed_grad(torch.empty(0, 8, device=DEV), none, out)
    assert bool((out == 0.0).all())


def test_gradient_is_the_lookups():
    """<dout, lookup(table)> is linear in the table; its slope is the gradient."""
    g = torch.Generator(device=DEV).manual_seed(3)
    n, v, d = 3000, 400, 40
    t, dout = tokens(n, v, g), torch.randn(n, d, device=DEV, generator=g)
    dt, out = torch.empty(v, d, device=DEV), torch.empty(n, d, device=DEV)
    efs.ef_embed_grad(dout, t, dt, scale=1.5)
    for _ in range(5):
        way = torch.randn(v, d, device=DEV, generator=g)
        efs.ef_embed(way, t, out, scale=1.5)
        left, right = (dout.double() * out).sum(), (dt.double() * way).sum()
        size = (dout.double() * out).abs().sum()
        assert abs(float(left - right)) < 3000 * 2.0 ** -24 * float(size)


@pytest.mark.parametrize("n,v,d", [(2100, 300, 40), (9000, 5000, 136), (70000, 3000, 64)])
@pytest.mark.parametrize("add", [False, True])
def test_lists_one_after_another(n, v, d, add):
    """Sorted lists of one scratch, each launch begun as the one before ends: none sees another's."""
    g = torch.Generator(device=DEV).manual_seed(n)
    lists = [tokens(n, v, g) for _ in range(8)]
    dout = torch.randn(n, d, device=DEV, generator=g)
    out = [torch.ones(v, d, device=DEV) for _ in lists]
    torch.cuda.synchronize()
    for t, o in zip(lists, out):
        efs.ef_embed_grad(dout, t, o, accumulate=add)
    zero = torch.zeros(v, d, device=DEV, dtype=torch.float64)
    for t, o in zip(lists, out):
        keep = t >= 0
        ref = zero.index_add(0, t[keep], dout[keep].double()) + float(add)
        mag = zero.index_add(0, t[keep], dout[keep].double().abs()) + float(add)
        count = zero.index_add(0, t[keep], torch.ones(int(keep.sum()), d, device=DEV, dtype=torch.float64))
        assert bool(((o.double() - ref).abs() <= (count + 2) * 2.0 ** -24 * mag).all())
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.parametrize("n,v,d", [(65536, 3000, 520), (70001, 40, 1024), (65536, 50001, 1000)])
@pytest.mark.parametrize("dt,tt", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("add", [False, True])
def test_long_lists_of_wide_rows(n, v, d, dt, tt, add):
    """Lists from 65,536 tokens on, whose lanes take 16 columns where nothing is added."""
    check_gradient(n, v, d, dt, tt, 0, 0, add)


@pytest.mark.parametrize("dt,tt", [(BF16, BF16), (BF16, F32), (F32, BF16), (F32, F32)])
def test_runs_of_many_pieces_of_wide_rows(dt, tt):
    """Words that end, go on and begin in pieces of 128 positions, some of them whole."""
    g = torch.Generator().manual_seed(9)
    runs = [128 * 16, 128 * 17, 128 * 16 - 1, 128 * 16 + 1, 128 * 17 + 1, 1, 128 * 33 + 5, 3, 128, 127, 129, 17, 128 * 40 + 2]
    runs += torch.randint(1, 400, (230,), generator=g).tolist()
    t = torch.repeat_interleave(torch.arange(len(runs)) + 1, torch.tensor(runs))
    t = torch.cat([t, torch.full((70001 - t.numel(),), len(runs) + 1)]) if t.numel() < 70001 else t
    t = t[torch.randperm(t.numel(), generator=g)].to(DEV)
    assert t.numel() >= 65536
    check_gradient(t.numel(), len(runs) + 3, 520, dt, tt, 0, 0, False, t=t)
    t[::7] = -1
    check_gradient(t.numel(), len(runs) + 3, 1024, dt, tt, 0, 0, False, t=t)

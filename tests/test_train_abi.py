"""Host-side checks of the embedding, layer norm and AdamW entry points: bad calls
are refused before any CUDA work (no GPU; the pointers are never dereferenced)."""
import ctypes

import pytest
import torch

import paper_2108_00951_gb300 as efs

A, B, C, D, E, F, G, H = (0x10000000 * i for i in range(1, 9))
BAD = efs.EF_ERR_INVALID_ARG
NAN, INF = float("nan"), float("inf")


def embed(table=A, ldt=64, tt=0, token=B, n=10, v=100, d=64, scale=1.0, out=C, ldo=64, ot=0):
    return efs.load_library().ef_embed(table, ldt, tt, token, n, v, d, scale, out, ldo, ot, None)


@pytest.mark.parametrize("kw", [
    dict(table=0), dict(token=0), dict(out=0), dict(table=A + 2), dict(table=A + 1, tt=1), dict(out=C + 2),
    dict(token=B + 4), dict(ldt=63), dict(ldo=63), dict(tt=2), dict(ot=-1), dict(v=0), dict(d=0),
    dict(n=(1 << 30) + 1), dict(v=(1 << 30) + 1), dict(d=(1 << 20) + 1, ldt=1 << 21, ldo=1 << 21), dict(ldt=(1 << 36) + 1),
    dict(scale=NAN), dict(scale=INF), dict(out=A), dict(out=A + 4 * 64 * 99), dict(out=B - 4 * 64 * 10 + 4),
])
def test_embed_rejects(kw):
    assert embed(**kw) == BAD


def embed_grad(dout=A, ldd=64, dt=0, token=B, n=10, v=100, d=64, scale=1.0, add=0, dtable=C, ldt=64, tt=0):
    return efs.load_library().ef_embed_grad(dout, ldd, dt, token, n, v, d, scale, add, dtable, ldt, tt, None)


@pytest.mark.parametrize("kw", [
    dict(dout=0), dict(token=0), dict(dtable=0), dict(dout=A + 2), dict(dtable=C + 1, tt=1), dict(token=B + 4),
    dict(ldd=63), dict(ldt=63), dict(dt=3), dict(tt=2), dict(v=0), dict(d=0), dict(n=(1 << 30) + 1),
    dict(scale=NAN), dict(dtable=A), dict(dtable=B - 4 * 64 * 100 + 4), dict(n=0, dtable=0),
])
def test_embed_grad_rejects(kw):
    assert embed_grad(**kw) == BAD


def norm(x=A, ldx=64, xt=0, w=B, b=C, wt=0, eps=1e-5, n=10, d=64, y=D, ldy=64, yt=0, mean=E, rstd=F):
    return efs.load_library().ef_layer_norm(x, ldx, xt, w, b, wt, eps, n, d, y, ldy, yt, mean, rstd, None)


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(y=0), dict(x=A + 2), dict(y=D + 1, yt=1), dict(w=B + 2), dict(b=C + 1, wt=1), dict(mean=E + 2),
    dict(rstd=F + 1), dict(ldx=63), dict(ldy=63), dict(xt=2), dict(wt=2), dict(yt=2), dict(eps=-1e-9),
    dict(eps=NAN), dict(eps=INF), dict(d=0), dict(n=(1 << 30) + 1), dict(y=A), dict(mean=A), dict(rstd=E + 36),
    dict(mean=B + 4), dict(y=C - 4),
])
def test_layer_norm_rejects(kw):
    assert norm(**kw) == BAD


def norm_grad(x=A, ldx=64, xt=0, w=B, wt=0, mean=C, rstd=D, dy=E, lddy=64, dyt=0, n=10, d=64, dx=F, lddx=64,
              dw=G, db=H):
    return efs.load_library().ef_layer_norm_grad(x, ldx, xt, w, wt, mean, rstd, dy, lddy, dyt, n, d, dx, lddx,
                                                 dw, db, None)


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(dy=0), dict(mean=0), dict(rstd=0), dict(x=A + 1), dict(dy=E + 2), dict(dx=F + 2), dict(dw=G + 2),
    dict(db=H + 1, wt=1), dict(mean=C + 2), dict(ldx=63), dict(lddy=63), dict(lddx=63), dict(xt=2), dict(dyt=2),
    dict(d=0), dict(dx=A), dict(dx=E), dict(dw=B), dict(db=G + 4 * 63), dict(dw=F + 8), dict(n=(1 << 30) + 1),
])
def test_layer_norm_grad_rejects(kw):
    assert norm_grad(**kw) == BAD


def words(x):
    return None if x is None else (ctypes.c_uint64 * max(len(x), 1))(*x)


def adamw(n=2, numel=(100, 300), p=(A, A + 400), g=(B, B + 400), gt=0, m=(C, C + 400), v=(D, D + 400), me=None,
          ve=None, copy=(E, E + 200), lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, wd=0.0, step=1, lr_dev=None, step_dev=None,
          scale=None):
    return efs.load_library().ef_adamw(n, words(numel), words(p), words(g), gt, words(m), words(v), words(me),
                                       words(ve), words(copy), lr, b1, b2, eps, wd, step, 0, lr_dev, step_dev,
                                       scale, None)


@pytest.mark.parametrize("kw", [
    dict(n=(1 << 20) + 1), dict(gt=2), dict(lr=NAN), dict(lr=INF), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0),
    dict(b2=NAN), dict(eps=-1e-9), dict(eps=1e-39), dict(eps=INF), dict(wd=NAN), dict(step=0), dict(lr_dev=F + 2),
    dict(step_dev=F + 4), dict(scale=F + 1), dict(numel=None), dict(p=None), dict(g=None), dict(m=None), dict(v=None),
    dict(p=(0, A)), dict(g=(B, 0)), dict(m=(C + 2, C + 400)), dict(copy=(E, 0)), dict(copy=(E + 1, E + 200)),
    dict(g=(B + 1, B + 400), gt=1), dict(me=(F, F + 1)), dict(ve=(F, F + 1)), dict(me=(F, 0), ve=(G, G + 1)),
    dict(p=(A, A + 396)), dict(p=(A + 400, A + 400)), dict(g=(A, B)), dict(v=(C, D)), dict(copy=(B, E)),
    dict(me=(F, F), ve=(G, G + 3)), dict(lr_dev=A + 8), dict(step_dev=D + 8), dict(numel=(100, (1 << 32) - 4095)),
    # out of order, one inside another
    dict(p=(A + 1000, A), m=(A + 1100, C)),
])
def test_adamw_rejects(kw):
    assert adamw(**kw) == BAD


def states(n=1, numel=(300,), m=(A,), v=(B,), me=(C,), ve=(D,), mo=(E,), vo=(F,), ot=0):
    return efs.load_library().ef_adamw_states(n, words(numel), words(m), words(v), words(me), words(ve), words(mo),
                                              words(vo), ot, None)


@pytest.mark.parametrize("kw", [
    dict(ot=2), dict(m=None), dict(v=None), dict(me=None), dict(ve=None), dict(mo=None), dict(vo=None), dict(m=(0,)),
    dict(ve=(0,)), dict(mo=(E + 2,)), dict(vo=(F + 1,), ot=1), dict(mo=(A + 299,), ot=0), dict(mo=(F + 596,), ot=1),
    dict(mo=(C,)), dict(n=(1 << 20) + 1), dict(numel=((1 << 32),)),
])
def test_adamw_states_rejects(kw):
    assert states(**kw) == BAD


def test_nothing_to_do():
    assert embed(n=0, token=0, out=0) == efs.EF_OK
    assert embed_grad(n=0, token=0, dout=0, add=1) == efs.EF_OK
    assert norm(n=0, x=0, y=0) == efs.EF_OK
    assert norm_grad(dx=0, dw=0, db=0) == efs.EF_OK
    assert norm_grad(n=0, x=0, dy=0, mean=0, rstd=0, dx=0, dw=0, db=0) == efs.EF_OK
    assert adamw(n=0) == efs.EF_OK
    assert adamw(numel=(0, 0), p=(0, 0), g=(0, 0), m=(0, 0), v=(0, 0), copy=(0, 0)) == efs.EF_OK
    assert states(n=0) == efs.EF_OK and states(numel=(0,), m=(0,), mo=(0,)) == efs.EF_OK


@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
def test_lists_that_lie_anyhow_pass_the_checks():
    for kw in (dict(), dict(p=(A + 5000, A)), dict(m=(A + 2000, C), v=(A + 2400, D)), dict(g=(A + 0x1000, A + 0x1000)),
               dict(copy=None), dict(me=(F, F + 1), ve=(G, G + 1)), dict(lr_dev=B, scale=B)):
        assert adamw(**kw) not in (efs.EF_OK, BAD)  # no GPU: a CUDA status


def test_binding_refuses():
    x, y, t = torch.zeros(3, 8), torch.zeros(3, 8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: efs.ef_embed(x, t, y), lambda: efs.ef_embed(None, t, y), lambda: efs.ef_embed_grad(x, t, y),
                 lambda: efs.ef_layer_norm(x, y), lambda: efs.ef_layer_norm(x[0], y),
                 lambda: efs.ef_layer_norm_grad(x, x[:, 0], x[:, 0], y, x.clone()),
                 lambda: efs.TensorList([x]), lambda: efs.TensorList([None]),
                 lambda: efs.ef_adamw([x], [x], [x], [x], 1, 1e-3), lambda: efs.ef_adamw([], [x], [], [], 1, 1e-3)):
        if not torch.cuda.is_available():
            with pytest.raises((TypeError, RuntimeError, AssertionError)):
                call()
    assert efs.exponents_for(0) == 0 and efs.exponents_for(128) == 1 and efs.exponents_for(129) == 2


@pytest.mark.gpu
def test_binding_refuses_on_a_gpu():
    x, t = torch.zeros(3, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    table, f = torch.zeros(5, 8, device="cuda"), torch.zeros(3, device="cuda")
    w = torch.zeros(8, device="cuda")
    refused = [
        lambda: efs.ef_embed(table, t[:2], x), lambda: efs.ef_embed(table, t.int(), x),
        lambda: efs.ef_embed(table, t, x[:, :7]), lambda: efs.ef_embed(table.half(), t, x),
        lambda: efs.ef_embed(table, t, x.t().contiguous().t()), lambda: efs.ef_embed(table, t.cpu(), x),
        lambda: efs.ef_embed_grad(x, t, table[:, :7]), lambda: efs.ef_embed_grad(x.double(), t, table),
        lambda: efs.ef_embed(table, t, x, scale="a"),
        lambda: efs.ef_layer_norm(x, x[:2].clone()), lambda: efs.ef_layer_norm(x, x.clone(), w[:7]),
        lambda: efs.ef_layer_norm(x, x.clone(), w, w.bfloat16()), lambda: efs.ef_layer_norm(x, x.clone(), w.double()),
        lambda: efs.ef_layer_norm(x, x.clone(), mean_out=f[:2]),
        lambda: efs.ef_layer_norm(x, x),  # overlap
        lambda: efs.ef_layer_norm_grad(x, None, f, x.clone(), x.clone()),
        lambda: efs.ef_layer_norm_grad(x, f, f, x.clone(), x.bfloat16()),
        lambda: efs.ef_layer_norm_grad(x, f, f, x.clone(), None, w, w.bfloat16()),
        lambda: efs.TensorList([x, x.bfloat16()]), lambda: efs.TensorList([x.t()]), lambda: efs.TensorList([x, f.cpu()]),
        lambda: efs.ef_adamw([f], [w], [f.clone()], [f.clone()], 1, 1e-3),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [], 1, 1e-3),
        lambda: efs.ef_adamw([f.bfloat16()], [f.clone()], [f.clone()], [f.clone()], 1, 1e-3),
        lambda: efs.ef_adamw([f], [f], [f.clone()], [f], 1, 1e-3),  # overlap
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], 0, 1e-3),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], -1, 1e-3),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], 1, 1e-3, m_exponents=[f]),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], 1, 1e-3, copies=[f.clone()]),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], t[:0], 1e-3),
        lambda: efs.ef_adamw([f], [f.clone()], [f.clone()], [f.clone()], 1, f.double()),
    ]
    for i, call in enumerate(refused):
        with pytest.raises((TypeError, ValueError, efs.EfError)):
            call()
            pytest.fail("not refused: %d" % i)
    efs.ef_adamw([], [], [], [], 1, 1e-3)
    assert efs.ef_check_status() == efs.EF_OK

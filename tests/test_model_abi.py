"""Host-side checks of the language-model operators' entry points: bad calls
are refused before any CUDA work (no GPU; the pointers are never
dereferenced)."""
import ctypes

import pytest
import torch

import paper_2108_00951_gb300 as efs

vp = ctypes.c_void_p
H, W, B, T, LOSS, LSE = (0x10000000 * i for i in range(1, 7))
DH, DW, DB, R = (0x70000000 + 0x10000000 * i for i in range(4))


def _loss(h=H, ldh=64, w=W, ldw=64, bias=B, target=T, n=10, v=100, d=64, loss=LOSS, lse=LSE):
    return efs.load_library().ef_vocab_loss(h, ldh, w, ldw, bias, target, n, v, d, loss, lse, None)


@pytest.mark.parametrize("kwargs", [
    dict(h=0), dict(w=0), dict(target=0), dict(loss=0), dict(lse=0), dict(h=H + 1), dict(w=W + 1),
    dict(bias=B + 1), dict(target=T + 4), dict(loss=LOSS + 2), dict(lse=LSE + 1),
    dict(ldh=63), dict(ldw=63), dict(v=0), dict(d=0), dict(d=(1 << 20) + 1), dict(n=(1 << 30) + 1),
    dict(v=(1 << 30) + 1), dict(ldw=(1 << 36) + 1),
    dict(loss=LSE + 36), dict(loss=H), dict(lse=W + 2 * 64 * 99), dict(lse=T + 72),
    dict(loss=B + 196),
])
def test_vocab_loss_rejects(kwargs):
    assert _loss(**kwargs) == efs.EF_ERR_INVALID_ARG


def _grad(h=H, ldh=64, w=W, ldw=64, bias=B, target=T, lse=LSE, r=R, n=10, v=100, d=64, dh=DH,
          lddh=64, dw=DW, lddw=64, db=DB):
    return efs.load_library().ef_vocab_loss_grad(h, ldh, w, ldw, bias, target, lse, r, n, v, d, dh,
                                                 lddh, dw, lddw, db, None)


@pytest.mark.parametrize("kwargs", [
    dict(h=0), dict(w=0), dict(lse=0), dict(r=0), dict(dh=0), dict(dw=0), dict(dh=DH + 1),
    dict(dw=DW + 1), dict(db=DB + 1), dict(r=R + 2), dict(lddh=63), dict(lddw=63),
    dict(bias=0),                       # db without a bias
    dict(dh=H), dict(dw=W + 128), dict(dw=DH + 1270), dict(db=DW), dict(dh=LSE), dict(db=R),
    dict(n=(1 << 30) + 1), dict(v=0), dict(d=0),
])
def test_vocab_loss_grad_rejects(kwargs):
    assert _grad(**kwargs) == efs.EF_ERR_INVALID_ARG


def _ortho(n=2, rows=(4, 6), cols=(8, 5), u=(H, W), ld_u=(8, 5), kind=0, m=(B, T), ld_m=(8, 5),
           mu=0.9, out=(LOSS, LSE), ld_out=(8, 5)):
    def words(x):
        return None if x is None else (ctypes.c_uint64 * max(len(x), 1))(*x)
    return efs.load_library().ef_orthogonalize(n, words(rows), words(cols), words(u), words(ld_u),
                                               kind, words(m), words(ld_m), mu, words(out),
                                               words(ld_out), None)


@pytest.mark.parametrize("kwargs", [
    dict(n=4097), dict(kind=2), dict(mu=float("nan")), dict(mu=float("inf")), dict(rows=None),
    dict(u=None), dict(out=None), dict(ld_m=None), dict(u=(0, W)), dict(out=(LOSS, 0)),
    dict(m=(B, 0)), dict(u=(H + 2, W)), dict(u=(H + 1, W), kind=1), dict(m=(B + 2, T)),
    dict(out=(LOSS + 1, LSE)), dict(ld_u=(7, 5)), dict(ld_m=(8, 4)), dict(ld_out=(7, 5)),
    dict(rows=((1 << 20) + 1, 6)), dict(out=(LOSS, LOSS + 62)), dict(out=(H + 32, LSE)),
    dict(m=(B, B)), dict(m=(H, T)), dict(ld_u=((1 << 36) + 1, 5)),
])
def test_orthogonalize_rejects(kwargs):
    assert _ortho(**kwargs) == efs.EF_ERR_INVALID_ARG


def test_nothing_to_do():
    assert _loss(n=0) == efs.EF_OK
    assert _ortho(n=0) == efs.EF_OK
    assert _ortho(rows=(0, 6), cols=(8, 0), u=(0, 0), m=(0, 0), out=(0, 0)) == efs.EF_OK


def test_binding_refuses():
    h, w = torch.zeros(3, 8, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16)
    t, f = torch.zeros(3, dtype=torch.int64), torch.zeros(3)
    with pytest.raises(TypeError):
        efs.ef_vocab_loss(h, w, t, f, f.clone())
    with pytest.raises(TypeError):
        efs.ef_vocab_loss(None, w, t, f, f.clone())
    with pytest.raises(TypeError):
        efs.ef_vocab_loss_grad(h, w, t, f, f.clone(), h.clone(), w.clone())
    with pytest.raises(TypeError):
        efs.ef_orthogonalize([w], [w.clone()])
    with pytest.raises(TypeError):
        efs.ef_orthogonalize([f], [f.clone()])
    with pytest.raises(ValueError):
        efs.ef_orthogonalize([w], [])
    with pytest.raises(ValueError):
        efs.ef_orthogonalize([w], [w.clone()], momenta=[])
    with pytest.raises(TypeError):
        efs.ef_orthogonalize([], [], momentum="x")
    efs.ef_orthogonalize([], [])

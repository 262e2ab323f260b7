"""Waits of the products that run out: the call reports a timeout (or, where no
wait took that long, is right), whatever it had under way has ended before its
kernel, and the next calls on the stream are right."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


def without_patience(call):
    """The call with waits that end at once; its status."""
    torch.cuda.synchronize()
    assert efs.ef_check_status() == efs.EF_OK
    efs.ef_test_set_lookback_fault(0, 0)
    try:
        call()
        status = efs.ef_check_status()
    finally:
        efs.ef_test_set_lookback_fault(-1)
    assert efs.ef_check_status() == efs.EF_OK
    return status


# a tile row (single CTAs) and pairs, several deep tiles a CTA
@pytest.mark.parametrize("n,v,d", [(100, 130000, 4096), (600, 80000, 4096)])
def test_loss_and_gradient(n, v, d):
    g = torch.Generator(device=DEV).manual_seed(n)
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    w = torch.empty(v, d, device=DEV, dtype=torch.bfloat16).normal_(0, 2.0 / d ** 0.5, generator=g)
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    r = torch.rand(n, device=DEV, generator=g)
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dh, dw = torch.empty_like(h), torch.empty_like(w)

    def forward():
        efs.ef_vocab_loss(h, w, t, loss, lse)

    def backward():
        efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw)
    forward()
    backward()
    want = [x.clone() for x in (loss, lse, dh, dw)]
    for call in (forward, backward):
        for _ in range(3):
            status = without_patience(call)
            assert status in (efs.EF_OK, efs.EF_ERR_TIMEOUT)
            if status == efs.EF_OK:
                assert all(torch.equal(x, y) for x, y in zip((loss, lse, dh, dw), want))
            forward()
            backward()
            assert efs.ef_check_status() == efs.EF_OK
            assert all(torch.equal(x, y) for x, y in zip((loss, lse, dh, dw), want))


# on chip; phases with joined K parts; phases in pairs
@pytest.mark.parametrize("shapes", [[(64, 576)] * 4, [(256, 2304), (700, 300)], [(3200, 3200)],
                                    [(512, 2304)] * 40])
def test_orthogonalised_updates(shapes):
    g = torch.Generator(device=DEV).manual_seed(7)
    us = [torch.randn(r, c, device=DEV, generator=g) for r, c in shapes]
    outs = [torch.empty(r, c, device=DEV, dtype=torch.bfloat16) for r, c in shapes]

    def call():
        efs.ef_orthogonalize(us, outs)
    call()
    want = [x.clone() for x in outs]
    for _ in range(3):
        status = without_patience(call)
        assert status in (efs.EF_OK, efs.EF_ERR_TIMEOUT)
        if status == efs.EF_OK:
            assert all(torch.equal(x, y) for x, y in zip(outs, want))
        call()
        assert efs.ef_check_status() == efs.EF_OK
        assert all(torch.equal(x, y) for x, y in zip(outs, want))

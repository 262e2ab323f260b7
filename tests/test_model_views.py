"""Views that interleave in memory, as column blocks of one buffer do: the
language-model operators take them wherever no element is shared. (The refusals
need no GPU: the pointers are never dereferenced.)"""
import ctypes

import pytest
import torch

import paper_2108_00951_gb300 as efs

DEV = "cuda"
BASE, ELSE = 0x10000000, 0x50000000


def ortho_status(mats):
    """(rows, cols, u, ld_u, m, ld_m, out, ld_out) of each, addresses in bytes, fp32."""
    def words(i):
        return (ctypes.c_uint64 * len(mats))(*[x[i] for x in mats])
    r, c, u, ld_u, m, ld_m, out, ld_out = (words(i) for i in range(8))
    return efs.load_library().ef_orthogonalize(len(mats), r, c, u, ld_u, 0, m, ld_m, 0.5, out, ld_out, None)


def blocks(out_at, m_at=(ELSE, ELSE + 0x100000), ld_out=(20, 20)):
    return [(6, 10, 0x90000000 + 0x100000 * i, 10, m_at[i], 10, out_at[i], ld_out[i]) for i in range(2)]


@pytest.mark.parametrize("mats", [
    blocks((BASE, BASE + 18)),                      # one column shared
    blocks((BASE, BASE + 2 * 20 * 3)),              # the same columns, other rows
    blocks((BASE, BASE - 18 + 40)),                 # from the row's last columns into the next
    blocks((BASE + 20, BASE + 2)),
    blocks((BASE, BASE + 22), ld_out=(20, 22)),     # other strides, ranges that meet
    blocks((BASE, BASE + 20), m_at=(ELSE, ELSE + 40 * 5)),
])
def test_shared_elements_are_refused(mats):
    assert ortho_status(mats) == efs.EF_ERR_INVALID_ARG


@pytest.mark.parametrize("mats", [
    blocks((BASE, BASE + 20)), blocks((BASE + 20, BASE)), blocks((BASE, BASE + 40 * 6)),
    blocks((BASE, BASE + 20 + 40 * 3)),             # the other columns, from another row on
    # a single row in the gap between two rows of the other
    [(6, 10, 0x90000000, 10, ELSE, 10, BASE, 20), (1, 10, 0x91000000, 10, ELSE + 0x100000, 10, BASE + 60, 999)],
])
@pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
def test_column_blocks_pass_the_checks(mats):
    assert ortho_status(mats) not in (efs.EF_OK, efs.EF_ERR_INVALID_ARG)  # no GPU: a CUDA status


def vocab_status(h, dh, ld, lddh=None, w=ELSE):
    return efs.load_library().ef_vocab_loss_grad(
        h, ld, w, 8, None, 0x60000000, 0x70000000, 0x80000000, 5, 9, 8, dh, lddh or ld, 0x90000000, 8,
        None, None)


def test_gradient_beside_its_input():
    assert vocab_status(BASE, BASE + 14, 16) == efs.EF_ERR_INVALID_ARG
    assert vocab_status(BASE, BASE + 16, 16, 24) == efs.EF_ERR_INVALID_ARG
    assert vocab_status(BASE, BASE + 16, 15) == efs.EF_ERR_INVALID_ARG
    # strides so large that products of sizes would not fit 64 bits
    lib = efs.load_library()
    assert lib.ef_vocab_loss(BASE, 1 << 36, BASE + 0x1000, 8, None, 0x60000000, 1 << 30, 9, 8, 0x70000000,
                             0x80000000, None) == efs.EF_ERR_INVALID_ARG
    if not torch.cuda.is_available():
        assert vocab_status(BASE, BASE + 16, 16) != efs.EF_ERR_INVALID_ARG


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [(60, 100, 41), (300, 200, 130)])
@pytest.mark.parametrize("r", [64, 250])
def test_updates_of_column_blocks(cols, r):
    g = torch.Generator(device=DEV).manual_seed(r + cols[0])
    all_u = torch.randn(r, sum(cols), device=DEV, generator=g)
    all_m = torch.randn(r, sum(cols), device=DEV, generator=g)
    all_out = torch.full((r, sum(cols) + 1), 7.0, device=DEV, dtype=torch.bfloat16)
    apart_u = [x.clone() for x in all_u.split(cols, 1)]
    apart_m = [x.clone() for x in all_m.split(cols, 1)]
    apart = [torch.empty_like(x, dtype=torch.bfloat16) for x in apart_u]
    efs.ef_orthogonalize(apart_u, apart, momenta=apart_m, momentum=0.9)
    efs.ef_orthogonalize(list(all_u.split(cols, 1)), list(all_out[:, :-1].split(cols, 1)),
                         momenta=list(all_m.split(cols, 1)), momentum=0.9)
    assert torch.equal(all_m, torch.cat(apart_m, 1))
    for x, y in zip(all_out[:, :-1].split(cols, 1), apart):
        # (sums of squares run in the same order, whatever the alignment)
        assert torch.equal(x, y)
    assert (all_out[:, -1] == 7.0).all()
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.gpu
@pytest.mark.parametrize("n,d", [(5, 200), (5, 1100), (100, 136), (300, 65)])
def test_gradients_beside_their_inputs(n, d):
    g = torch.Generator(device=DEV).manual_seed(n + d)
    v = 700
    rows = torch.randn(n, 2 * d, device=DEV, generator=g).bfloat16()
    words = torch.randn(v, 2 * d, device=DEV, generator=g).bfloat16()
    t = torch.randint(-1, v, (n,), device=DEV, generator=g)
    r = torch.rand(n, device=DEV, generator=g)
    h, dh, w, dw = rows[:, :d], rows[:, d:], words[:, :d], words[:, d:]
    keep = h.clone(), w.clone()
    loss, lse = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    efs.ef_vocab_loss(h, w, t, loss, lse)
    want = torch.empty_like(keep[0]), torch.empty_like(keep[1])
    efs.ef_vocab_loss_grad(*keep, t, lse, r, *want)
    efs.ef_vocab_loss_grad(h, w, t, lse, r, dh, dw)
    assert torch.equal(h, keep[0]) and torch.equal(w, keep[1])
    assert torch.equal(dh, want[0]) and torch.equal(dw, want[1])
    assert efs.ef_check_status() == efs.EF_OK

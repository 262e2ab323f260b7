"""Captured calls and the growth of the workspace: a graph's replays stay right
after larger calls on its stream, and report their errors; growth while a call is
captured is refused."""
import pytest
import torch

import paper_2108_00951_gb300 as efs

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.fixture(autouse=True)
def fresh_workspaces():
    efs.ef_workspace_release()
    yield


def problem(n, v, d, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + n + v + d)
    h = torch.randn(n, d, device=DEV, generator=g).bfloat16()
    w = torch.randn(v, d, device=DEV, generator=g).bfloat16()
    t = torch.randint(0, v, (n,), device=DEV, generator=g)
    f = {"device": DEV, "dtype": torch.float32}
    return {"h": h, "w": w, "t": t, "r": torch.rand(n, device=DEV, generator=g), "loss": torch.empty(n, **f),
            "lse": torch.empty(n, **f), "dh": torch.empty_like(h), "dw": torch.empty_like(w)}


def step(p):
    efs.ef_vocab_loss(p["h"], p["w"], p["t"], p["loss"], p["lse"])
    efs.ef_vocab_loss_grad(p["h"], p["w"], p["t"], p["lse"], p["r"], p["dh"], p["dw"])


def update(u, out):
    efs.ef_orthogonalize([u], [out])


def captured(stream, call):
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream, capture_error_mode="thread_local"):
        call()
    return graph


@pytest.mark.parametrize("n", [5, 200])
def test_replays_after_a_larger_call(n):
    side = torch.cuda.Stream()
    small, large = problem(n, 1000, 96), problem(3000, 9000, 300)
    u = torch.randn(200, 333, device=DEV)
    out = torch.empty_like(u, dtype=torch.bfloat16)
    big = torch.randn(1500, 900, device=DEV)
    big_out = torch.empty_like(big, dtype=torch.bfloat16)

    def both():
        step(small)
        update(u, out)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    keys = ("loss", "lse", "dh", "dw")
    want = [small[k].clone() for k in keys] + [out.clone()]
    graph = captured(side, both)
    for later in (lambda: step(large), lambda: update(big, big_out)):
        with torch.cuda.stream(side):
            later()  # grows the scratch
            # (takes what growth may have freed: a replay into it would be seen)
            taken = [torch.full((1 << 20,), 7, device=DEV, dtype=torch.int32) for _ in range(64)]
            for x in [small[k] for k in keys] + [out]:
                x.fill_(float("nan"))
            graph.replay()
        side.synchronize()
        for x, y in zip([small[k] for k in keys] + [out], want):
            assert torch.equal(x, y)
        assert all((x == 7).all() for x in taken)
        with torch.cuda.stream(side):  # a call of the stream's own beside the graph
            both()
        side.synchronize()
        for x, y in zip([small[k] for k in keys] + [out], want):
            assert torch.equal(x, y)
        assert efs.ef_check_status(side) == efs.EF_OK


def test_replays_report_after_the_other_workspace_grew():
    side = torch.cuda.Stream()
    p = problem(40, 500, 64)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(p)
    side.synchronize()
    graph = captured(side, lambda: step(p))
    d = 3_000_000
    g, e = torch.randn(d, device=DEV), torch.zeros(d, device=DEV)
    idx, val = torch.empty(d, device=DEV, dtype=torch.int32), torch.empty(d, device=DEV)
    count = torch.empty(1, device=DEV, dtype=torch.int32)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        efs.ef_hard_threshold(g, e, 1.0, 2.0, idx, val, count)  # grows the workspace
        p["t"][3] = 500  # past the vocabulary
        graph.replay()
    assert efs.ef_check_status(side) == efs.EF_ERR_BAD_INPUT
    with torch.cuda.stream(side):
        p["t"][3] = 499
        graph.replay()
    assert efs.ef_check_status(side) == efs.EF_OK


@pytest.mark.parametrize("warm", [False, True])
def test_growth_while_captured_is_refused(warm):
    side = torch.cuda.Stream()
    small, large = problem(30, 300, 64), problem(400, 3000, 128)
    u = torch.randn(400, 700, device=DEV)
    out = torch.empty_like(u, dtype=torch.bfloat16)
    torch.cuda.synchronize()
    if warm:
        with torch.cuda.stream(side):
            step(small)
        side.synchronize()
    mark = torch.zeros(1, device=DEV)

    def calls():
        for call in (lambda: step(large), lambda: update(u, out)):
            with pytest.raises(efs.EfError) as err:
                call()
            assert err.value.status == efs.EF_ERR_NO_MEMORY
        mark.add_(1.0)
    graph = captured(side, calls)  # (an invalid capture raises here)
    graph.replay()
    torch.cuda.synchronize()
    assert float(mark) == 1.0

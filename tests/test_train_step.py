"""Embedding, layer norm, loss, their gradients and AdamW run together, as a training
step calls them; and the example that does."""
import pytest
import torch

import paper_2108_00951_gb300 as efs
from paper_2108_00951_gb300 import lm_sgd

DEV = "cuda"


def test_the_norms_vectors_are_at_the_end():
    m = lm_sgd.Model.create(11, 4, 3, device="cpu", norm=True)
    assert m.d == 11 * 4 + 3 * 16 + 11 + 8
    emb, mats, bias = m.split(m.x)
    scale, shift = m.norm_vectors(m.x)
    assert bias.numel() == 11 and scale.shape == shift.shape == (4,)
    for part in (emb, *mats, bias, scale, shift):
        part.add_(1.0)
    assert torch.equal(m.x, lm_sgd.Model.create(11, 4, 3, device="cpu", norm=True).x + 1.0)
    assert lm_sgd.Model.create(11, 4, 3, device="cpu").norm_vectors(m.x) == ()


def test_unknown_rules_are_refused():
    m = lm_sgd.Model.create(11, 4, 3, device="cpu")
    with pytest.raises(ValueError):
        lm_sgd.Vectors(m, torch.zeros_like(m.x), "adam", 0.1, 0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("length", [100, 3000])
def test_worker_gradient_with_a_norm_matches_autograd(length):
    m = lm_sgd.Model.create(300, 32, 2, seed=1, norm=True)
    m.norm_vectors(m.x)[0].uniform_(0.5, 1.5)
    m.norm_vectors(m.x)[1].uniform_(-0.5, 0.5)
    text = lm_sgd.make_text(300, length, 1, seed=2)[0]
    g = torch.empty(m.d, device=DEV)
    loss = lm_sgd.worker_gradient(m, text, g)
    emb, mats, bias = m.split(m.x)
    e = emb.bfloat16().double().requires_grad_()
    c = [x.double().requires_grad_() for x in mats]
    b = bias.bfloat16().double().requires_grad_()
    w, s = (x.double().requires_grad_() for x in m.norm_vectors(m.x))
    h = sum(e[torch.roll(text, j + 1)] @ c[j].T for j in range(2))
    y = torch.nn.functional.layer_norm(h, (32,), w, s, 1e-5)
    ref = torch.nn.functional.cross_entropy((y @ e.T + b)[2:], text[2:])
    ref.backward()
    assert abs(float(loss) - float(ref.detach())) < 2e-3
    got_e, got_c, got_b = m.split(g)
    # y, dy and the decoder's gradients are bf16: a few roundings of 2^-8, of which the
    # norm's Jacobian takes a part out of dy and leaves its rounding
    for x, z in ((got_e, e.grad), (got_b, b.grad), *((p, q.grad) for p, q in zip(got_c, c)),
                 *zip(m.norm_vectors(g), (w.grad, s.grad))):
        assert float((x.double() - z).norm() / z.norm()) < 6 * 2.0 ** -8
    assert efs.ef_check_status() == efs.EF_OK


@pytest.mark.gpu
@pytest.mark.parametrize("rule", ["sgd", "adamw", "adamw8"])
@pytest.mark.parametrize("norm", [False, True])
def test_the_example_runs(rule, norm):
    h = lm_sgd.run(words=300, width=32, workers=2, length=80, steps=4, norm=norm, rule=rule)
    assert len(h["loss"]) == 4 and all(x == x and x < 20 for x in h["loss"])
    assert all(0 < x <= 2 * h["d"][0] for x in h["sent"])


@pytest.mark.gpu
@pytest.mark.parametrize("rule", ["sgd", "adamw", "adamw8"])
def test_vectors_follow_their_rule(rule):
    g = torch.Generator(device=DEV).manual_seed(3)
    m = lm_sgd.Model.create(101, 12, 1, seed=3, norm=True)
    delta = torch.randn(m.d, device=DEV, generator=g)
    start = m.x.clone()
    v = lm_sgd.Vectors(m, delta, rule, 0.01, 0.03)
    v.update()
    n = 101 * 12
    table, mats, rest = slice(0, n), slice(n, n + 144), slice(n + 144, m.d)
    assert torch.equal(m.x[mats], start[mats])
    if rule == "sgd":
        want = start - 0.01 * delta
        want[-24:] = start[-24:] - 0.03 * delta[-24:]
    else:  # the first step of AdamW: lr times the sign, with eps beside |g|
        want = start - 0.01 * delta / (delta.abs() + 1e-8)
    for part in (table, rest):
        assert float((m.x[part] - want[part]).abs().max()) < 2.0 ** -20


def step(tensors, text, words):
    """Lookup, norm, loss, gradients and update; returns the loss."""
    t = tensors
    efs.ef_embed(t["table16"], text, t["x"], scale=2.0)
    efs.ef_layer_norm(t["x"], t["h"], t["w"], t["b"], 1e-5, t["mean"], t["rstd"])
    efs.ef_vocab_loss(t["h"], t["out16"], t["target"], t["loss"], t["lse"])
    efs.ef_vocab_loss_grad(t["h"], t["out16"], t["target"], t["lse"], t["r"], t["dh"], t["dout"])
    efs.ef_layer_norm_grad(t["x"], t["mean"], t["rstd"], t["dh"], t["dx"], t["w"], t["dw"], t["db"])
    efs.ef_embed_grad(t["dx"], text, t["dtable"], scale=2.0)


def tensors(n, v, d, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + n)
    f, h = {"device": DEV}, {"device": DEV, "dtype": torch.bfloat16}
    t = {"table": torch.randn(v, d, device=DEV, generator=g), "out": torch.randn(v, d, device=DEV, generator=g) / d ** 0.5,
         "w": torch.rand(d, device=DEV, generator=g) + 0.5, "b": torch.randn(d, device=DEV, generator=g),
         "target": torch.randint(-1, v, (n,), device=DEV, generator=g), "r": torch.full((n,), 1.0 / n, **f),
         "x": torch.empty(n, d, **f), "dx": torch.empty(n, d, **f), "h": torch.empty(n, d, **h), "dh": torch.empty(n, d, **h),
         "dout": torch.empty(v, d, **h), "dtable": torch.empty(v, d, **f), "dw": torch.empty(d, **f),
         "db": torch.empty(d, **f), "table16": torch.empty(v, d, **h), "out16": torch.empty(v, d, **h)}
    for k in ("mean", "rstd", "loss", "lse"):
        t[k] = torch.empty(n, **f)
    t["table16"].copy_(t["table"])
    t["out16"].copy_(t["out"])
    return t, torch.randint(-1, v, (n,), device=DEV, generator=g)


@pytest.mark.gpu
@pytest.mark.parametrize("n,v,d", [(1, 50, 40), (12, 500, 650), (700, 900, 129), (3000, 400, 256)])
def test_a_step_matches_autograd(n, v, d):
    t, text = tensors(n, v, d)
    step(t, text, v)
    table = t["table16"].double().requires_grad_()
    out = t["out16"].double().requires_grad_()
    w, b = t["w"].double().requires_grad_(), t["b"].double().requires_grad_()
    x = 2.0 * table[text.clamp(min=0)] * (text >= 0)[:, None]
    y = torch.nn.functional.layer_norm(x, (d,), w, b, 1e-5)
    z = y @ out.T
    at = z.gather(1, t["target"].clamp(min=0)[:, None])[:, 0]
    keep = t["target"] >= 0
    loss = (torch.logsumexp(z, 1) - at) * keep
    (loss.sum() / n).backward()
    # h is rounded to bf16: its logits are off by 2^-9 of |h| |w| times a random sign each
    size = (y.detach().abs() @ out.detach().abs().T).max()
    assert bool(((t["loss"].double() - loss.detach()).abs() < 2.0 ** -7 * size).all())
    if bool(keep.any()):
        for got, ref in ((t["dout"], out.grad), (t["dw"], w.grad), (t["db"], b.grad), (t["dtable"], table.grad)):
            # bf16 hidden states, G and dh, each 2^-9 of its size on the average, before sums of
            # random signs; a padded position's row (x = 0) has no gradient but for rounding
            assert float((got.double() - ref).norm()) < 2.0 ** -5 * float(ref.norm()) + 1e-9
    # one step of AdamW over all of it, and the copies that the next step reads
    params, grads = [t["table"], t["out"], t["w"], t["b"]], [t["dtable"], t["dout"].float(), t["dw"], t["db"]]
    m, s = ([torch.zeros_like(p) for p in params] for _ in range(2))
    copies = [t["table16"], t["out16"], torch.empty_like(t["w"], dtype=torch.bfloat16),
              torch.empty_like(t["b"], dtype=torch.bfloat16)]
    want = [p.double() - 1e-2 * g.double() / (g.double().abs() + 1e-8) for p, g in zip(params, grads)]
    efs.ef_adamw(params, grads, m, s, 1, 1e-2, weight_decay=0.0, copies=copies)
    for p, c, x in zip(params, copies, want):
        assert float((p.double() - x).abs().max()) < 2.0 ** -20
        assert torch.equal(c, p.bfloat16())
    assert efs.ef_check_status() == efs.EF_OK


# ---------------------------------------------------------------- graphs, streams
@pytest.mark.gpu
@pytest.mark.parametrize("n", [40, 2500])
def test_a_step_captured_and_replayed(n):
    """Replays with other tokens, step numbers and rates give what calls give, also
    after a larger call has grown the stream's scratch."""
    efs.ef_workspace_release()
    v, d = 300, 136
    side = torch.cuda.Stream()
    t, text = tensors(n, v, d)
    big, big_text = tensors(9000, 700, 200)
    params, grads = [t["table"], t["w"], t["b"]], [t["dtable"], t["dw"], t["db"]]
    state = lambda: [torch.zeros(p.shape, device=DEV, dtype=torch.uint8) for p in params]  # noqa: E731
    exps = lambda: [torch.zeros(efs.exponents_for(p.numel()), device=DEV, dtype=torch.uint8) for p in params]  # noqa: E731
    m, s, me, se = state(), state(), exps(), exps()
    number, rate = torch.zeros(1, device=DEV, dtype=torch.int64), torch.full((1,), 1e-2, device=DEV)
    copies = [t["table16"], *(torch.empty_like(p, dtype=torch.bfloat16) for p in params[1:])]

    def whole():
        step(t, text, v)
        efs.ef_adamw(params, grads, m, s, number, rate, m_exponents=me, v_exponents=se, copies=copies, seed=5)
    kept = [*params, *m, *s, *me, *se, *copies]
    torch.cuda.synchronize()
    first = [x.clone() for x in kept]

    def restart():
        for x, y in zip(kept, first):
            x.copy_(y)

    def inputs(k):
        g = torch.Generator(device=DEV).manual_seed(k)
        text.copy_(torch.randint(-1, v, (n,), device=DEV, generator=g))
        number.fill_(k + 1)
        rate.fill_(1e-2 / (k + 1))
    with torch.cuda.stream(side):
        inputs(0)
        whole()  # grows the scratch
        restart()
        want = []
        for k in range(3):
            inputs(k)
            whole()
            want.append([x.clone() for x in kept])
        restart()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
        whole()
    with torch.cuda.stream(side):
        restart()
        for k in range(3):
            inputs(k)
            if k == 1:
                step(big, big_text, 700)  # grows it again
            graph.replay()
            for x, y in zip(kept, want[k]):
                assert torch.equal(x, y)
    assert efs.ef_check_status(side) == efs.EF_OK


@pytest.mark.gpu
def test_growth_while_captured_is_refused():
    efs.ef_workspace_release()
    side = torch.cuda.Stream()
    t, text = tensors(3000, 200, 64)
    x, dy = t["x"], t["dh"]
    t["mean"].fill_(0.0)
    t["rstd"].fill_(1.0)
    x.normal_()
    dy.normal_()
    torch.cuda.synchronize()
    mark = torch.zeros(1, device=DEV)

    def calls():
        for call in (lambda: efs.ef_embed(t["table"], text, x), lambda: efs.ef_embed_grad(t["dx"], text, t["dtable"]),
                     lambda: efs.ef_layer_norm_grad(x, t["mean"], t["rstd"], dy, t["dx"], None, t["dw"])):
            with pytest.raises(efs.EfError) as err:
                call()
            assert err.value.status == efs.EF_ERR_NO_MEMORY
        # these need none
        efs.ef_layer_norm(x, t["h"])
        efs.ef_adamw([t["w"]], [t["b"]], [torch.zeros_like(t["w"])], [torch.zeros_like(t["w"])], 1, 0.1)
        mark.add_(1.0)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side, capture_error_mode="thread_local"):
        calls()
    before = t["w"].clone()
    graph.replay()
    torch.cuda.synchronize()
    assert float(mark) == 1.0 and not torch.equal(before, t["w"])


@pytest.mark.gpu
def test_steps_on_several_streams_at_once():
    n, v, d = 2600, 300, 96
    pairs = [tensors(n, v, d, seed=k) for k in range(4)]
    want = []
    for t, text in pairs:
        step(t, text, v)
        want.append([t[k].clone() for k in ("loss", "dtable", "dout", "dw", "db")])
        for k in ("loss", "dtable", "dout", "dw", "db"):
            t[k].fill_(float("nan"))
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, (t, text) in zip(streams, pairs):
            with torch.cuda.stream(stream):
                step(t, text, v)
    torch.cuda.synchronize()
    for (t, _), ref in zip(pairs, want):
        for k, x in zip(("loss", "dtable", "dout", "dw", "db"), ref):
            assert torch.equal(t[k], x), k


@pytest.mark.gpu
def test_calls_from_several_threads():
    import threading
    n, v, d = 2300, 200, 80
    pairs = [tensors(n, v, d, seed=k) for k in range(4)]
    want = []
    for t, text in pairs:
        step(t, text, v)
        want.append([t[k].clone() for k in ("dtable", "dw")])
    streams = [torch.cuda.Stream() for _ in pairs]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(streams[i]):
            for _ in range(10):
                step(*pairs[i], v)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    for (t, _), ref in zip(pairs, want):
        for k, x in zip(("dtable", "dw"), ref):
            assert torch.equal(t[k], x)

"""Operators of a language-model training step around the compression and the
exchange, and what they are measured on.

  loss   ef_vocab_loss: softmax cross entropy of hidden states against a large
         vocabulary, without the logits in memory (evaluation, scoring)
  grad   ef_vocab_loss_grad: its gradient, from the log-sum-exp of the loss call
  step   both, as a training step calls them
  orth   ef_orthogonalize: momentum and the orthogonalised update (five
         Newton-Schulz steps) of a list of weight matrices

Formulas. z = h w^T + b; lse_n = log sum_v exp z_nv; loss_n = lse_n - z_n,t(n);
G_nv = r_n (exp(z_nv - lse_n) - [v = t(n)]); dh = G w, dw = G^T h, db = sum_n G_n.
A row with a negative target is skipped: loss and log-sum-exp 0, no gradient.
m <- mu m + u, U = u + m (or U = u); X = U / |U|_F; five times, on the shorter
side, A = X X^T, X <- 3.4445 X + (-4.775 A + 2.0315 A A) X.
"""
import math

import torch

own = False
DEV = "cuda"
MU = 0.9
NS = (3.4445, -4.7750, 2.0315)


# ------------------------------------------------------------------- cases
def _vocab(name, op, n, v, d, **more):
    c = {"name": name, "op": op, "n": n, "v": v, "d": d, "bias": False, "ignored": 0.0, "pad": 0}
    c.update(more)
    return c


def _orth(name, shapes, dtype="f32", momentum=False):
    return {"name": name, "op": "orth", "shapes": shapes, "dtype": dtype, "momentum": momentum}


RESNET18 = ("64x27*1,64x576*4,128x576*1,128x1152*3,128x64*1,256x1152*1,256x2304*3,256x128*1,"
            "512x2304*1,512x4608*3,512x256*1,10x512*1")


def listed():
    return [
        # one token scored by the LSTM workload's decoder (28,869 words, width
        # 650): latency, the weight matrix read once, rows that start at any
        # multiple of 4 bytes
        _vocab("score_token", "loss", 1, 28869, 650, bias=True),
        # a short text scored by a model of 65,537 words, rows padded to 16 bytes
        _vocab("score_text", "loss", 96, 65537, 1021, pad=3),
        # evaluation of a batch of ordinary size
        _vocab("loss_eval", "loss", 4096, 50001, 1024),
        # the largest evaluation: 8192 tokens, 128,000 words, width 4096
        _vocab("loss_large", "loss", 8192, 128000, 4096),
        # the LSTM workload's training step: 20 sequences of 35 tokens
        _vocab("lstm_step", "step", 700, 28869, 650, bias=True),
        # the gradient of a handful of tokens
        _vocab("grad_few", "grad", 5, 28869, 650, bias=True),
        # an instruction batch: 40 % of its tokens carry no loss, odd sizes
        _vocab("step_masked", "step", 2051, 50001, 1000, ignored=0.4),
        # the largest gradient
        _vocab("grad_large", "grad", 8192, 128000, 2048),
        # one convolution's weights: latency
        _orth("orth_conv", "64x576*1"),
        # every weight matrix of the ResNet-18 workload after an exchange
        _orth("orth_resnet18", RESNET18, momentum=True),
        # the LSTM workload's six recurrent matrices and a ragged one, bf16 updates
        _orth("orth_lstm", "2600x650*6,333x1111*1", dtype="bf16"),
        # the VGG-16 workload's fully connected layers
        _orth("orth_vgg16_fc", "25088x4096*1,4096x4096*1,4096x1000*1", momentum=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.65:
        op = rng.choice(["loss", "grad", "step"])
        while True:
            n, v, d = _log(rng, 1, 8192), _log(rng, 1000, 128000), _log(rng, 64, 4096)
            if n * v * d <= 8192 * 128000 * 1024:
                break
        return {"op": op, "n": n, "v": v, "d": d, "bias": rng.random() < 0.5,
                "ignored": rng.choice([0.0, 0.0, 0.3]), "pad": rng.choice([0, 0, (-d) % 8])}
    kinds, cost = [], 0.0
    for _ in range(rng.choice([1, 1, 2, 3, 5])):
        r, c, k = _log(rng, 1, 4096), _log(rng, 16, 8192), rng.choice([1, 1, 2, 4])
        cost += k * r * c * min(r, c)
        if cost > 2e11:
            break
        kinds.append("%dx%d*%d" % (r, c, k))
    return {"op": "orth", "shapes": ",".join(kinds) or "%dx512*1" % rng.randrange(3, 512),
            "dtype": rng.choice(["f32", "bf16"]), "momentum": rng.random() < 0.4}


def _shapes(case):
    out = []
    for part in case["shapes"].split(","):
        size, k = part.split("*")
        r, c = size.split("x")
        out += [(int(r), int(c))] * int(k)
    return out


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _inputs(case, seed):
    g = _gen(seed)
    if case["op"] == "orth":
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        u, m = [], []
        for r, c in _shapes(case):
            # gradients of a layer: a few strong directions over noise
            k = min(4, r, c)
            x = torch.randn(r, c, device=DEV, generator=g)
            x += 0.5 * (torch.randn(r, k, device=DEV, generator=g)
                        @ torch.randn(k, c, device=DEV, generator=g))
            u.append((x * 1e-3).to(dtype))
            if case["momentum"]:
                m.append(torch.randn(r, c, device=DEV, generator=g) * 2e-3)
        return {"u": u, "m": m}
    n, v, d = case["n"], case["v"], case["d"]
    h = torch.randn(n, d, device=DEV, generator=g)
    w = torch.empty(v, d + case["pad"], device=DEV, dtype=torch.bfloat16)[:, :d]
    step = max(1, (1 << 27) // d)
    for a in range(0, v, step):
        w[a:a + step] = torch.randn(min(step, v - a), d, device=DEV, generator=g) * (2.0 / d ** 0.5)
    # words by a Zipf law, their log frequency in the bias
    rank = torch.arange(v, device=DEV, dtype=torch.float32)
    t = torch.exp(torch.rand(n, device=DEV, generator=g) * math.log(v)).to(torch.int64) - 1
    t = t.clamp_(0, v - 1)
    if case["ignored"]:
        t[torch.rand(n, device=DEV, generator=g) < case["ignored"]] = -100
    valid = max(1, int((t >= 0).sum()))
    h2 = torch.empty(n, d + case["pad"], device=DEV, dtype=torch.bfloat16)[:, :d]
    h2.copy_(h)
    s = {"h": h2, "w": w, "t": t, "r": torch.full((n,), 1.0 / valid, device=DEV), "b": None}
    if case["bias"]:
        s["b"] = (4.0 - torch.log(rank + 3.0)).to(torch.bfloat16)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["op"] = case["op"]
    if case["op"] == "orth":
        s["out"] = [torch.empty_like(u, dtype=torch.bfloat16) for u in s["u"]]
        return s
    n, v, d = case["n"], case["v"], case["d"]
    f = {"device": DEV, "dtype": torch.float32}
    if case["op"] != "grad":
        s["loss"], s["lse"] = torch.empty(n, **f), torch.empty(n, **f)
    else:
        # the loss call of the same step left its log-sum-exp
        s["lse"] = torch.cat([_logsumexp(_logits(s, a, a + 1024)) for a in range(0, n, 1024)])
        s["lse"][s["t"] < 0] = 0.0
    if case["op"] != "loss":
        b = {"device": DEV, "dtype": torch.bfloat16}
        s["dh"], s["dw"] = torch.empty(n, d, **b), torch.empty(v, d, **b)
        s["db"] = torch.empty(v, **b) if case["bias"] else None
    return s


# -------------------------------------------------------------- plain form
def _logits(s, lo=0, hi=None):
    z = s["h"][lo:hi].float() @ s["w"].float().T
    return z if s["b"] is None else z.add_(s["b"].float())


def _logsumexp(z):
    top = z.max(dim=1).values
    return top + (z - top[:, None]).exp_().sum(dim=1).log()


def _plain_loss(s):
    z = _logits(s)
    lse = _logsumexp(z)
    at = z.gather(1, s["t"].clamp(min=0)[:, None])[:, 0]
    none = torch.zeros_like(lse)
    return torch.where(s["t"] >= 0, lse - at, none), torch.where(s["t"] >= 0, lse, none)


def _plain_grad(s, lse):
    p = _logits(s).sub_(lse[:, None]).exp_()
    r = torch.where(s["t"] >= 0, s["r"], torch.zeros_like(s["r"]))
    p.scatter_add_(1, s["t"].clamp(min=0)[:, None], torch.full_like(r, -1.0)[:, None])
    p *= r[:, None]
    out = {"dh": (p @ s["w"].float()).bfloat16(), "dw": (p.T @ s["h"].float()).bfloat16()}
    if s["b"] is not None:
        out["db"] = p.sum(dim=0).bfloat16()
    return out


def _plain_orth(u, m):
    x = u.float()
    if m is not None:
        m.mul_(MU).add_(x)
        x = x + m
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / x.square().sum().sqrt()
    a, b, c = NS
    for _ in range(5):
        g = x @ x.T
        x = a * x + (b * g + c * (g @ g)) @ x
    return (x.T if tall else x).bfloat16().contiguous()


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "orth":
        m = s["m"] or [None] * len(s["u"])
        return {"out": [_plain_orth(u, x) for u, x in zip(s["u"], m)], "m": s["m"]}
    out, lse = {}, s["lse"]
    if s["op"] != "grad":
        out["loss"], lse = _plain_loss(s)
        out["lse"] = lse
    if s["op"] != "loss":
        out.update(_plain_grad(s, lse))
    return out


# ---------------------------------------------------------- the operators
def _run_own(s):
    import paper_2108_00951_gb300 as efs
    if s["op"] == "orth":
        efs.ef_orthogonalize(s["u"], s["out"], momenta=s["m"] or None, momentum=MU)
        return {"out": s["out"], "m": s["m"]}
    out = {}
    if s["op"] != "grad":
        efs.ef_vocab_loss(s["h"], s["w"], s["t"], s["loss"], s["lse"], bias=s["b"])
        out["loss"], out["lse"] = s["loss"], s["lse"]
    if s["op"] != "loss":
        efs.ef_vocab_loss_grad(s["h"], s["w"], s["t"], s["lse"], s["r"], s["dh"], s["dw"],
                               bias=s["b"], dbias_out=s["db"])
        out["dh"], out["dw"] = s["dh"], s["dw"]
        if s["db"] is not None:
            out["db"] = s["db"]
    return out


# -------------------------------------------------------------------- work
def work(case):
    if case["op"] == "orth":
        size = 4 if case["dtype"] == "f32" else 2
        nbytes = flops = 0
        for r, c in _shapes(case):
            s = min(r, c)
            nbytes += r * c * (size + 2 + (8 if case["momentum"] else 0))
            # the two symmetric products need half of their entries
            flops += 5 * (r * c * s + s ** 3 + 2 * r * c * s)
        return {"bytes": nbytes, "flops": flops}
    n, v, d = case["n"], case["v"], case["d"]
    bias = 2 * v if case["bias"] else 0
    nbytes, flops = 0, 0
    rows = n * (1.0 - case["ignored"])
    if case["op"] != "grad":  # logits
        nbytes += 2 * (n + v) * d + bias + 16 * n
        flops += 2 * rows * v * d
    if case["op"] != "loss":  # logits again, and the two products with them
        nbytes += 4 * (n + v) * d + 2 * bias + 16 * n
        flops += 6 * rows * v * d
    return {"bytes": nbytes, "flops": flops}


# ------------------------------------------------------------ in 64 bits
def _double_products(case):
    if case["op"] == "orth":
        return sum(20 * r * c * min(r, c) + 10 * min(r, c) ** 3 for r, c in _shapes(case))
    return case["n"] * case["v"] * case["d"] * {"loss": 2, "grad": 8, "step": 6}[case["op"]]


def exact(case, seed):
    if _double_products(case) > 6e12:  # too long in 64 bits
        return None
    s = _inputs(case, seed)
    if case["op"] == "orth":
        outs, ms = [], []
        for i, u in enumerate(s["u"]):
            x = u.double()
            if s["m"]:
                ms.append(MU * s["m"][i].double() + x)
                x = x + ms[-1]
            x = x / torch.linalg.matrix_norm(x)
            left = x.shape[0] <= x.shape[1]
            for _ in range(5):
                if left:
                    y = x @ x.mT
                    x = torch.addmm(x, torch.addmm(y, y, y, beta=NS[1], alpha=NS[2]), x, beta=NS[0])
                else:
                    y = x.mT @ x
                    x = torch.addmm(x, x, torch.addmm(y, y, y, beta=NS[1], alpha=NS[2]),
                                    beta=NS[0])
            outs.append(x)
        return {"out": outs, "m": ms}
    n, v, d = case["n"], case["v"], case["d"]
    w = s["w"].double()
    b = s["b"].double() if s["b"] is not None else torch.zeros(v, device=DEV, dtype=torch.float64)
    loss, lse, dh = [], [], []
    dw, db = torch.zeros(v, d, device=DEV, dtype=torch.float64), torch.zeros_like(b)
    step = max(1, (1 << 29) // v)
    for a in range(0, n, step):
        h, t, r = s["h"][a:a + step].double(), s["t"][a:a + step], s["r"][a:a + step].double()
        z = torch.addmm(b, h, w.mT)
        z32 = torch.logsumexp(z, 1)
        keep = t >= 0
        rows = torch.arange(len(t), device=DEV)[keep]
        one = torch.zeros_like(z32)
        one[rows] = z32[rows] - z[rows, t[keep]]
        loss.append(one)
        lse.append(z32 * keep)
        if case["op"] != "loss":
            q = torch.softmax(z, 1)
            q[rows, t[keep]] -= 1.0
            q *= (r * keep)[:, None]
            dh.append(q @ w)
            dw += q.mT @ h
            db += q.sum(0)
    out = {}
    if case["op"] != "grad":
        out["loss"], out["lse"] = torch.cat(loss), torch.cat(lse)
    if case["op"] != "loss":
        out["dh"], out["dw"] = torch.cat(dh), dw
        if case["bias"]:
            out["db"] = db
    return out

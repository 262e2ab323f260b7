"""More operators of a language-model training step around the compression and
the exchange, and what they are measured on.

  lookup   ef_embed: rows of an embedding table by token, scaled
  lookgrad ef_embed_grad: the table's gradient, rows of equal tokens summed; over
           the whole table, or added to a gradient that is there (tied weights)
  norm     ef_layer_norm: layer norm's forward pass
  normstep ef_layer_norm and ef_layer_norm_grad, as a training step calls them
  adamw    ef_adamw: an AdamW step over many tensors at once, states in 32 bits
  adamw8   the same with states in 8 bits, and ef_adamw_states, which gives the
           values that they stand for (what a checkpoint holds)

Formulas. out_i = s table[t_i]; dtable_w = s sum_{i: t_i = w} dout_i; a negative
token is padding: a row of zeros, no gradient.
x' = (x - mean) rstd, mean = avg x, rstd = (avg (x - mean)^2 + eps)^(-1/2),
y = x' w + b; q = dy w, dx = rstd (q - avg q - x' avg(q x')),
dw = sum_rows dy x', db = sum_rows dy.
m <- b1 m + (1 - b1) g, v <- b2 v + (1 - b2) g^2,
p <- p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps).

States in 8 bits: blocks of 128 entries of a tensor share E, the exponent of the
largest magnitude (at least -92). An entry is a sign (m only), an exponent field f
(4 bits in m, 5 in v) and 3 bits k: (8 + k) 2^(E - top + f - 3), or k 2^(E - top - 2)
where f = 0, with top = 14 in m and 30 in v. Rounding is stochastic: up where the
part below the last place, plus a random number of 16 bits, carries; but a positive
v is held as its lowest positive value at least. (From 2^127 on an entry is held as
NaN, its highest code.)
"""
import math

import torch

own = False
DEV = "cuda"
EPS_NORM = 1e-5
STEP, LR, B1, B2, EPS, WD = 1000, 1e-3, 0.9, 0.999, 1e-8, 0.01
BLOCK = 128
TOP, LEAST = {"m": 14, "v": 30}, -92


# ------------------------------------------------------------------- cases
def _embed(name, op, n, v, d, **more):
    c = {"name": name, "op": op, "n": n, "v": v, "d": d, "dtype": "bf16", "table": "bf16",
         "padding": 0.0, "add": False, "pad": 0}
    c.update(more)
    return c


def _norm(name, op, n, d, **more):
    c = {"name": name, "op": op, "n": n, "d": d, "x": "bf16", "y": "bf16", "w": "f32", "pad": 0}
    c.update(more)
    return c


def _adamw(name, op, sizes, grad="f32", copy=False):
    return {"name": name, "op": op, "sizes": sizes, "grad": grad, "copy": copy}


# the parameter tensors of this repository's workloads, times each size
RESNET18_VECTORS = "64*10,128*10,256*10,512*10,10*1"
LSTM = "18764850*1,1690000*6,2600*6,28869*1"
RESNET50 = ("9408*1,64*14,4096*1,36864*3,16384*4,256*8,16384*2,128*16,32768*1,147456*4,65536*4,"
            "512*10,131072*1,65536*3,256*24,131072*1,589824*6,262144*6,1024*14,524288*1,262144*5,"
            "512*12,524288*1,2359296*3,1048576*3,2048*8,2097152*1,1048576*2,2048000*1,1000*1")


def listed():
    return [
        # the next token of 16 sequences that are being scored: latency
        _embed("lookup_tokens", "lookup", 16, 28869, 650),
        # a large batch through a table of 50,001 words, scaled by its width's root
        _embed("lookup_batch", "lookup", 65536, 50001, 1024, padding=0.1),
        # the LSTM workload's step, 20 sequences of 35 tokens: the decoder's gradient
        # of the tied table is there, the lookup's is added to it
        _embed("lookgrad_lstm", "lookgrad", 700, 28869, 650, dtype="f32", table="f32", add=True),
        # a batch of ordinary size whose sequences are padded, rows on odd strides
        _embed("lookgrad_padded", "lookgrad", 8191, 50001, 1001, padding=0.3),
        # the largest gradient of a table, in fp32 for the compression
        _embed("lookgrad_large", "lookgrad", 131075, 128000, 1024, table="f32"),
        # one token's hidden state in front of the decoder: latency
        _norm("norm_token", "norm", 1, 650),
        # the LSTM workload's step
        _norm("norm_lstm", "normstep", 700, 650, w="bf16"),
        # an odd width, a residual stream in 32 bits
        _norm("norm_odd", "normstep", 4099, 1001, x="f32"),
        # the largest batch
        _norm("norm_large", "normstep", 32768, 4096),
        # the norm and bias vectors of the ResNet-18 workload: latency
        _adamw("adamw_vectors", "adamw", RESNET18_VECTORS),
        # the LSTM workload's 14 tensors, bf16 gradients, a bf16 copy for the next step
        _adamw("adamw_lstm", "adamw", LSTM, grad="bf16", copy=True),
        # the ResNet-50 workload's 161 tensors with states in 8 bits
        _adamw("adamw8_resnet50", "adamw8", RESNET50),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["lookup", "lookgrad", "lookgrad", "norm", "normstep", "normstep", "adamw",
                       "adamw8"])
    if kind in ("lookup", "lookgrad"):
        while True:
            n, v, d = _log(rng, 1, 131072), _log(rng, 50, 128000), _log(rng, 8, 4096)
            if (n + v) * d <= (131072 + 128000) * 1024:
                break
        return {"op": kind, "n": n, "v": v, "d": d, "dtype": rng.choice(["bf16", "f32"]),
                "table": rng.choice(["bf16", "f32"]), "padding": rng.choice([0.0, 0.0, 0.3]),
                "add": kind == "lookgrad" and rng.random() < 0.4, "pad": rng.choice([0, 0, (-d) % 8])}
    if kind in ("norm", "normstep"):
        while True:
            n, d = _log(rng, 1, 32768), _log(rng, 16, 24576)
            if n * d <= 32768 * 2048:
                break
        return {"op": kind, "n": n, "d": d, "x": rng.choice(["bf16", "f32"]),
                "y": rng.choice(["bf16", "f32"]), "w": rng.choice(["bf16", "f32"]),
                "pad": rng.choice([0, 0, (-d) % 8])}
    parts, total = [], 0
    for _ in range(rng.choice([1, 2, 4, 8, 16])):
        size, k = _log(rng, 1, 1 << 23), rng.choice([1, 1, 2, 5])
        if total + size * k > 28_000_000:
            continue
        total += size * k
        parts.append("%d*%d" % (size, k))
    return {"op": kind, "sizes": ",".join(parts) or "%d*1" % rng.randrange(3, 5000),
            "grad": rng.choice(["f32", "bf16"]), "copy": rng.random() < 0.3}


def _sizes(case):
    out = []
    for part in case["sizes"].split(","):
        size, k = part.split("*")
        out += [int(size)] * int(k)
    return out


# ------------------------------------------------------------------ inputs
def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _rows(rows, cols, pad, dtype):
    """A matrix whose rows lie `pad` entries apart."""
    return torch.empty(rows, cols + pad, device=DEV, dtype=dtype)[:, :cols]


def _randn(g, rows, cols, scale, pad, dtype):
    m = _rows(rows, cols, pad, dtype)
    step = max(1, (1 << 26) // cols)
    for a in range(0, rows, step):
        m[a:a + step] = torch.randn(min(step, rows - a), cols, device=DEV, generator=g) * scale
    return m


def _tokens(g, n, v, padding):
    """Words by a Zipf law; padded positions are negative."""
    t = torch.exp(torch.rand(n, device=DEV, generator=g, dtype=torch.float64) * math.log(v))
    t = (t.to(torch.int64) - 1).clamp_(0, v - 1)
    if padding:
        t[torch.rand(n, device=DEV, generator=g) < padding] = -1
    return t


M32 = 0xFFFFFFFF


def _mix(x):
    """A permutation of 32 bits (of an int64 tensor, or of a number)."""
    x = x ^ (x >> 16)
    x = (x * 0x6A09E667) & M32
    x = x ^ (x >> 15)
    x = (x * 0xBB67AE85) & M32
    return x ^ (x >> 16)


def _random(seed, step, sizes):
    """The 32 random bits of each entry of each tensor: the low half is m's, the high v's."""
    key = _mix(_mix(seed & M32) ^ (seed >> 32))
    key = _mix((key + step) & M32)
    return [_mix((torch.arange(n, device=DEV) + _mix((key + 0x9E3779B9 * k) & M32)) & M32)
            for k, n in enumerate(sizes)]


def _adamw_inputs(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    sizes = _sizes(case)
    d = sum(sizes)
    # gradients whose size differs from tensor to tensor, and from row to row of a
    # tensor: bursts of 64 of one scale
    each = torch.exp(2.0 * torch.randn(len(sizes), device=DEV, generator=g)) * 1e-3
    per = torch.repeat_interleave(each, torch.tensor(sizes, device=DEV))
    burst = torch.exp(torch.randn((d + 63) // 64, device=DEV, generator=g))
    per *= torch.repeat_interleave(burst, 64)[:d]
    s = {"p": torch.randn(d, device=DEV, generator=g) * 0.05,
         "g": (per * torch.randn(d, device=DEV, generator=g)).to(_type(case["grad"])),
         "seed": seed * 0x10001 + 7}
    m = per * 0.2 * torch.randn(d, device=DEV, generator=g)
    v = per * per * (0.5 + torch.rand(d, device=DEV, generator=g))
    if case["copy"]:
        s["copy"] = torch.empty(d, device=DEV, dtype=torch.bfloat16)
    if case["op"] == "adamw":
        s["m"], s["v"] = m, v
        return s
    # where each entry lies among the blocks, and its random number
    blocks = [(n + BLOCK - 1) // BLOCK for n in sizes]
    first = [0]
    for b in blocks:
        first.append(first[-1] + b)
    begin = [0]
    for n in sizes:
        begin.append(begin[-1] + n)
    shift = torch.tensor([BLOCK * f - b for f, b in zip(first, begin)][:len(sizes)], device=DEV)
    s["at"] = torch.arange(d, device=DEV) + torch.repeat_interleave(
        shift, torch.tensor(sizes, device=DEV))
    s["first"], s["begin"], s["blocks"] = first, begin, first[-1]
    random = torch.zeros(first[-1] * BLOCK, device=DEV, dtype=torch.int64)
    random[s["at"]] = torch.cat(_random(s["seed"], STEP, sizes))
    s["random"] = random.to(torch.int32).view(-1, BLOCK)  # (the low 32 bits)
    for key, x in (("m", m), ("v", v)):  # states of an earlier step, rounded to nearest
        full = torch.zeros(first[-1] * BLOCK, device=DEV)
        full[s["at"]] = x
        s[key], s[key + "_e"] = _encode(full.view(-1, BLOCK), key, None)
    return s


def _inputs(case, seed):
    if case["op"] in ("adamw", "adamw8"):
        return _adamw_inputs(case, seed)
    g = torch.Generator(device=DEV).manual_seed(seed)
    if case["op"] in ("norm", "normstep"):
        n, d, pad = case["n"], case["d"], case["pad"]
        s = {"x": _randn(g, n, d, 1.0, pad, _type(case["x"]))}
        # a few channels are large, all have a mean of their own
        size = torch.where(torch.rand(d, device=DEV, generator=g) < 0.01, 20.0, 1.0)
        size = size * torch.exp(0.3 * torch.randn(d, device=DEV, generator=g))
        mean = 0.3 * torch.randn(d, device=DEV, generator=g)
        step = max(1, (1 << 26) // d)
        for a in range(0, n, step):
            s["x"][a:a + step] = s["x"][a:a + step].float() * size + mean
        s["w"] = (1.0 + 0.1 * torch.randn(d, device=DEV, generator=g)).to(_type(case["w"]))
        s["b"] = (0.1 * torch.randn(d, device=DEV, generator=g)).to(_type(case["w"]))
        if case["op"] == "normstep":
            s["dy"] = _randn(g, n, d, 1e-3, pad, _type(case["y"]))
        return s
    n, v, d, pad = case["n"], case["v"], case["d"], case["pad"]
    s = {"t": _tokens(g, n, v, case["padding"]), "scale": d ** 0.5}
    if case["op"] == "lookup":
        s["table"] = _randn(g, v, d, 0.02, pad, _type(case["table"]))
        return s
    s["dout"] = _randn(g, n, d, 1e-3, pad, _type(case["dtype"]))
    s["dtable"] = _rows(v, d, pad, _type(case["table"]))
    if case["add"]:
        s["dtable"].copy_(_randn(g, v, d, 1e-3, 0, torch.float32))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["op"], s["case"] = case["op"], case
    if case["op"] == "lookup":
        s["out"] = _rows(case["n"], case["d"], case["pad"], _type(case["dtype"]))
    elif case["op"] in ("norm", "normstep"):
        n, d = case["n"], case["d"]
        s["y"] = _rows(n, d, case["pad"], _type(case["y"]))
        if case["op"] == "normstep":
            s["mean"], s["rstd"] = (torch.empty(n, device=DEV) for _ in range(2))
            s["dx"] = _rows(n, d, case["pad"], _type(case["x"]))
            s["dw"], s["db"] = (torch.empty(d, device=DEV, dtype=_type(case["w"])) for _ in range(2))
    elif case["op"] in ("adamw", "adamw8"):
        _lists(s, case)
    return s


def _lists(s, case):
    """The tensors of the model as views of its flat vectors, and the lists of them
    that a program's calls pass."""
    sizes = _sizes(case)
    flat = ["p", "g"] + (["m", "v"] if case["op"] == "adamw" else []) + (["copy"] if "copy" in s else [])
    s["list"] = {k: s[k].split(sizes) for k in flat}
    if case["op"] == "adamw8":
        d = sum(sizes)
        for key in ("m", "v"):
            codes = s[key].view(-1)
            s["list"][key] = [codes[BLOCK * f:BLOCK * f + n] for f, n in zip(s["first"], sizes)]
            s["list"][key + "_e"] = [s[key + "_e"][a:b] for a, b in zip(s["first"], s["first"][1:])]
            s[key + "_value"] = torch.empty(d, device=DEV, dtype=torch.bfloat16)
            s["list"][key + "_value"] = s[key + "_value"].split(sizes)
    if own:  # checked once and kept, as the tensors of a model are
        import paper_2108_00951_gb300 as efs
        s["list"] = {k: efs.TensorList(x) for k, x in s["list"].items()}


# -------------------------------------------------------------- plain form
def _plain_lookup(s):
    keep = (s["t"] >= 0)[:, None]
    rows = s["table"][s["t"].clamp(min=0)].float() * s["scale"]
    s["out"].copy_(torch.where(keep, rows, torch.zeros_like(rows)))
    return s["out"]


def _plain_lookgrad(s):
    v, d = s["dtable"].shape
    keep = s["t"] >= 0
    rows = torch.where(keep[:, None], s["dout"].float(), 0.0)
    total = torch.zeros(v, d, device=rows.device).index_add_(0, s["t"].clamp(min=0), rows)
    total *= s["scale"]
    if s["case"]["add"]:
        total += s["dtable"].float()
    s["dtable"].copy_(total)
    return s["dtable"]


def _plain_norm(s):
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    x = x - mean
    rstd = 1.0 / (x.square().mean(dim=1, keepdim=True) + EPS_NORM).sqrt()
    x *= rstd
    s["y"].copy_(x * s["w"].float() + s["b"].float())
    if s["op"] == "norm":
        return {"y": s["y"]}
    dy = s["dy"].float()
    s["mean"].copy_(mean[:, 0])
    s["rstd"].copy_(rstd[:, 0])
    s["dw"].copy_((dy * x).sum(dim=0))
    s["db"].copy_(dy.sum(dim=0))
    q = dy * s["w"].float()
    both = (q * x).mean(dim=1, keepdim=True)
    s["dx"].copy_((q - q.mean(dim=1, keepdim=True) - x * both) * rstd)
    return _norm_out(s)


def _norm_out(s):
    return {k: s[k] for k in ("y", "mean", "rstd", "dx", "dw", "db")}


def _power(e):
    """2^e as fp32, for e (int32) from -126 to 127."""
    return ((e + 127) << 23).view(torch.float32)


def _encode(x, key, random):
    """Blocks [blocks, 128] as codes and exponents: uint8 tensors. Rounded as the
    random numbers say, or to nearest without any."""
    top, nan = TOP[key], 127 if key == "m" else 255
    mag = x.abs()
    fine = mag < 2.0 ** 127
    mag = torch.where(fine, mag, 0.0)
    e = torch.frexp(mag.amax(dim=1)).exponent.sub_(1).clamp_(min=LEAST)
    e = torch.where(mag.amax(dim=1) > 0, e, LEAST)
    low = (e - top + 1)[:, None]  # the exponent of f = 1
    at = torch.where(mag > 0, torch.maximum(torch.frexp(mag).exponent - 1, low), low)
    up = 0.5 if random is None else (random.float() + 0.5) / 65536.0
    code = (at - low) * 8 + torch.floor(mag * _power(3 - at) + up).to(torch.int32)
    if key == "v":
        code = torch.where((code == 0) & (mag > 0), 1, code)
    code = torch.where(fine, code, nan)
    if key == "m":
        code = code + 128 * torch.signbit(x)
    return code.to(torch.uint8), (e + 127).to(torch.uint8)


def _decode(codes, exponents, key):
    c = codes.to(torch.int32)
    e = exponents.to(torch.int32).clamp(min=LEAST + 127)[:, None] - 127
    a = c & 127 if key == "m" else c
    f, k = a >> 3, a & 7
    x = torch.where(f > 0, 8 + k, k).float() * _power((f - 1).clamp(min=0)) * _power(e - TOP[key] - 2)
    x = torch.where(a == (127 if key == "m" else 255), math.nan, x)
    return torch.where(c > 127, -x, x) if key == "m" else x


def _constants():
    return 1.0 - B1 ** STEP, 1.0 - B2 ** STEP


def _plain_adamw(s):
    g = s["g"].float()
    if s["op"] == "adamw8":
        full = torch.zeros(s["blocks"] * BLOCK, device=g.device)
        full[s["at"]] = g
        g = full.view(-1, BLOCK)
        m, v = _decode(s["m"], s["m_e"], "m"), _decode(s["v"], s["v_e"], "v")
    else:
        m, v = s["m"], s["v"]
    m = m * B1 + g * (1.0 - B1)
    v = v * B2 + g * g * (1.0 - B2)
    one, two = _constants()
    u = (m / one) / ((v / two).sqrt() + EPS)
    if s["op"] == "adamw8":
        u = u.view(-1)[s["at"]]
    s["p"].copy_(s["p"] * (1.0 - LR * WD) - LR * u)
    if "copy" in s:
        s["copy"].copy_(s["p"])
    if s["op"] == "adamw":
        s["m"].copy_(m)
        s["v"].copy_(v)
        return _adamw_out(s)
    r = s["random"]
    for key, x, bits in (("m", m, r & 0xFFFF), ("v", v, (r >> 16) & 0xFFFF)):
        codes, exponents = _encode(x, key, bits)
        s[key].copy_(codes)
        s[key + "_e"].copy_(exponents)
        s[key + "_value"].copy_(_decode(codes, exponents, key).view(-1)[s["at"]])
    return _adamw_out(s)


def _adamw_out(s):
    """(The values of 8-bit entries, 4 bits times a power of two, are numbers of bf16.)"""
    keys = ("p", "copy", "m", "v") if s["op"] == "adamw" else ("p", "copy", "m_value", "v_value")
    return {k: s[k] for k in keys if k in s}


def run(s):
    if own:
        return _run_own(s)
    if s["op"] == "lookup":
        return _plain_lookup(s)
    if s["op"] == "lookgrad":
        return _plain_lookgrad(s)
    if s["op"] in ("norm", "normstep"):
        return _plain_norm(s)
    return _plain_adamw(s)


# ---------------------------------------------------------- the operators
def _run_own(s):
    import paper_2108_00951_gb300 as efs
    op = s["op"]
    if op == "lookup":
        efs.ef_embed(s["table"], s["t"], s["out"], scale=s["scale"])
        return s["out"]
    if op == "lookgrad":
        efs.ef_embed_grad(s["dout"], s["t"], s["dtable"], scale=s["scale"],
                          accumulate=s["case"]["add"])
        return s["dtable"]
    if op == "norm":
        efs.ef_layer_norm(s["x"], s["y"], s["w"], s["b"], EPS_NORM)
        return {"y": s["y"]}
    if op == "normstep":
        efs.ef_layer_norm(s["x"], s["y"], s["w"], s["b"], EPS_NORM, s["mean"], s["rstd"])
        efs.ef_layer_norm_grad(s["x"], s["mean"], s["rstd"], s["dy"], s["dx"], s["w"], s["dw"],
                               s["db"])
        return _norm_out(s)
    x = s["list"]
    efs.ef_adamw(x["p"], x["g"], x["m"], x["v"], STEP, LR, B1, B2, EPS, WD,
                 m_exponents=x.get("m_e"), v_exponents=x.get("v_e"), copies=x.get("copy"),
                 seed=s["seed"])
    if op == "adamw8":
        efs.ef_adamw_states(x["m"], x["v"], x["m_e"], x["v_e"], x["m_value"], x["v_value"])
    return _adamw_out(s)


# -------------------------------------------------------------------- work
def _distinct(case):
    """Expected number of different words among the tokens."""
    v, n = case["v"], case["n"] * (1.0 - case["padding"])
    k = torch.arange(1, v + 1, dtype=torch.float64)
    p = torch.log1p(1.0 / k) / math.log(max(v, 2))
    return float((1.0 - torch.exp(n * torch.log1p(-p.clamp(max=0.999)))).sum())


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "lookup":
        return {"bytes": _distinct(case) * case["d"] * size[case["table"]] + 8 * case["n"]
                + case["n"] * case["d"] * size[case["dtype"]], "flops": case["n"] * case["d"]}
    if case["op"] == "lookgrad":
        rows = case["n"] * (1.0 - case["padding"])
        out = 2 * _distinct(case) if case["add"] else case["v"]
        return {"bytes": rows * case["d"] * size[case["dtype"]] + 8 * case["n"]
                + out * case["d"] * size[case["table"]], "flops": rows * case["d"]}
    if case["op"] in ("norm", "normstep"):
        n, d, x, y, w = case["n"], case["d"], size[case["x"]], size[case["y"]], size[case["w"]]
        nbytes, flops = n * d * (x + y) + 2 * d * w, 8 * n * d
        if case["op"] == "normstep":  # x again, dy, dx; mean and rstd both ways
            nbytes += n * d * (2 * x + y) + 3 * d * w + 16 * n
            flops += 14 * n * d
        return {"bytes": nbytes, "flops": flops}
    d, blocks = sum(_sizes(case)), sum((n + BLOCK - 1) // BLOCK for n in _sizes(case))
    nbytes = d * (8 + size[case["grad"]] + (2 if case["copy"] else 0))
    # 8 bits: both states read and written, then read again and written as values
    nbytes += 16 * d if case["op"] == "adamw" else d * (4 + 2 + 4) + 6 * blocks
    return {"bytes": nbytes, "flops": 14 * d}


# ------------------------------------------------------------ in 64 bits
def _exact_norm(s):
    y, dx, mean, rstd = [], [], [], []
    n, d = s["x"].shape
    w, b = s["w"].double(), s["b"].double()
    dw, db = torch.zeros_like(w), torch.zeros_like(w)
    step = max(1, (1 << 25) // d)
    for a in range(0, n, step):
        x = s["x"][a:a + step].double()
        var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
        r = torch.rsqrt(var + EPS_NORM)
        hat = (x - mu) * r
        y.append(torch.addcmul(b, hat, w))
        if "dy" not in s:
            continue
        dy = s["dy"][a:a + step].double()
        dw += torch.einsum("nd,nd->d", dy, hat)
        db += torch.einsum("nd->d", dy)
        # dx is dy w times the Jacobian: what is left without its mean and its
        # projection on the normalised row
        q = dy * w
        q = q - q.sum(1, keepdim=True) / d
        dx.append(r * (q - hat * (torch.einsum("nd,nd->n", q, hat) / d)[:, None]))
        mean.append(mu[:, 0])
        rstd.append(r[:, 0])
    if "dy" not in s:
        return {"y": torch.cat(y)}
    return {"y": torch.cat(y), "mean": torch.cat(mean), "rstd": torch.cat(rstd),
            "dx": torch.cat(dx), "dw": dw, "db": db}


def _exact_held(x, s, key, shift):
    """The values that 8-bit states hold x [d] (fp64) as: to the next multiple of an
    entry's place below or above."""
    sign_bits, top = (x < 0), TOP[key]
    full = torch.zeros(s["blocks"] * BLOCK, device=DEV, dtype=torch.float64)
    full[s["at"]] = x.abs()
    full = full.view(-1, BLOCK)
    largest = full.amax(1, keepdim=True)
    e = torch.floor(torch.log2(largest.clamp(min=2.0 ** LEAST)))
    place = torch.floor(torch.log2(full.clamp(min=1e-300)))
    place = 2.0 ** (torch.maximum(place, e - top + 1) - 3)
    u = (((s["random"] >> shift) & 0xFFFF).double() + 0.5) / 65536.0
    held = torch.floor(full / place + u) * place
    if key == "v":
        held = torch.where((full > 0) & (held == 0), place, held)
    held = held.view(-1)[s["at"]]
    return torch.where(sign_bits, -held, held)


def _exact_start(codes, exponents, key):
    """A state's values at the start, from a table of the 256 codes."""
    c = torch.arange(256, device=DEV)
    a = c & 127 if key == "m" else c
    table = torch.where(a < 8, a * 0.125, (1.0 + (a & 7) * 0.125) * 2.0 ** ((a >> 3) - 1).double())
    table = torch.where(c != a, -table, table)
    scale = 2.0 ** (exponents.double() - 127 - TOP[key] + 1)
    return table[codes.long()] * scale[:, None]


def _exact_adamw(s):
    g = s["g"].double()
    if s["op"] == "adamw8":
        m, v = (_exact_start(s[k], s[k + "_e"], k).view(-1)[s["at"]] for k in ("m", "v"))
    else:
        m, v = s["m"].double(), s["v"].double()
    m = torch.lerp(g, m, B1)
    v = torch.lerp(g.square(), v, B2)
    one, two = _constants()
    den = torch.add(v.div(two).sqrt_(), EPS)
    p = torch.addcdiv(s["p"].double() * (1.0 - LR * WD), m, den, value=-LR / one)
    out = {"p": p}
    if "copy" in s:
        out["copy"] = p
    if s["op"] == "adamw":
        return {**out, "m": m, "v": v}
    return {**out, "m_value": _exact_held(m, s, "m", 0), "v_value": _exact_held(v, s, "v", 16)}


def exact(case, seed):
    s = _inputs(case, seed)
    s["op"] = case["op"]
    if case["op"] == "lookup":
        wide = torch.cat([s["table"].double() * s["scale"],
                          torch.zeros(1, case["d"], device=DEV, dtype=torch.float64)])
        return wide[s["t"]]  # (-1: the row of zeros)
    if case["op"] == "lookgrad":
        v, d = s["dtable"].shape
        # sorted, so that equal tokens lie together; their sums are differences of
        # nothing but their own rows
        t, order = torch.sort(s["t"], stable=True)
        order = order[t >= 0]
        words, counts = torch.unique_consecutive(t[t >= 0], return_counts=True)
        out = s["dtable"].double() if case["add"] else torch.zeros(v, d, device=DEV,
                                                                   dtype=torch.float64)
        if len(words):
            rows = torch.segment_reduce(s["dout"][order].double(), "sum", lengths=counts, axis=0)
            out[words] += rows * s["scale"]
        return out
    if case["op"] in ("norm", "normstep"):
        return _exact_norm(s)
    return _exact_adamw(s)

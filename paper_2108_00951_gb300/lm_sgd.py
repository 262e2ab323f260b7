"""Distributed EF-SGD on a small language model, every step of a worker after
its context in the library's kernels.

The model is log-bilinear: the hidden state of a position is the sum over the
`context` words before it of a matrix times the word's vector, the vectors are
the decoder's (tied, as in the LSTM / WikiText-2 workload of the paper's Table 1),
and the next word has the softmax of the hidden state against them plus a bias:

    h_t = sum_j C_j E[w_{t-j}],     p(w | t) = softmax(E h_t + b)_w,

with `norm` the softmax is of E LN(h_t) + b, LN a layer norm with its own scale and
shift. One iteration of Algorithm 1 with n workers:

    E[w_{t-j}], and their gradient added to dL/dE     ef_embed, ef_embed_grad
    LN(h), dL/dh and its vectors' gradients           ef_layer_norm, ef_layer_norm_grad
    loss, dL/dh, dL/dE, dL/db of a worker's text     ef_vocab_loss, ef_vocab_loss_grad
    a = e + g, Delta_i = C(a), e <- a - C(a)          ef_hard_threshold
    Delta = (1/n) sum_i Delta_i                       sparse_aggregate
    C_j <- C_j - lr_c orthogonalised(Delta, momentum)  ef_orthogonalize
    E, b and the norm's vectors: x <- x - lr Delta, or AdamW with states in 32 or 8
    bits (`rule`)                                     ef_adamw

The first words of each text have no full context: their targets are negative,
so they take no part. The products of the context's chain rule are computed with
torch, as the logistic regression's local gradients are in ef_sgd. The text is
synthetic: a seeded first-order chain over the vocabulary with a few likely
successors per word.
"""
from __future__ import annotations

import dataclasses
from typing import Dict, List

import torch

from . import _binding as efs


@dataclasses.dataclass
class Model:
    """One flat fp32 parameter vector (as the compression sees it) and its views."""
    words: int
    width: int
    context: int
    x: torch.Tensor
    norm: bool = False

    @staticmethod
    def create(words: int, width: int, context: int, seed: int = 0, device="cuda",
               norm: bool = False) -> "Model":
        g = torch.Generator(device="cpu").manual_seed(seed)
        e = torch.randn(words * width, generator=g) * 0.1
        c = torch.randn(context * width * width, generator=g) * (0.5 / width ** 0.5)
        parts = [e, c, torch.zeros(words)]
        if norm:
            parts += [torch.ones(width), torch.zeros(width)]
        return Model(words, width, context, torch.cat(parts).to(device), norm)

    @property
    def d(self) -> int:
        return self.x.numel()

    def split(self, flat: torch.Tensor):
        """(E, [C_j], b) as views of a flat vector."""
        v, w, k = self.words, self.width, self.context
        e, c = v * w, k * w * w
        return (flat[:e].view(v, w), list(flat[e:e + c].view(k, w, w).unbind(0)),
                flat[e + c:e + c + v])

    def norm_vectors(self, flat: torch.Tensor):
        """(scale, shift) of the layer norm as views of a flat vector; () without one."""
        return tuple(flat[self.d - 2 * self.width:].split(self.width)) if self.norm else ()


def make_text(words: int, length: int, workers: int, seed: int = 0, device="cuda") -> torch.Tensor:
    """int64 [workers, length]: a chain in which each word has four likely
    successors (90 %), anything else otherwise."""
    g = torch.Generator(device="cpu").manual_seed(seed)
    successors = torch.randint(0, words, (words, 4), generator=g)
    text = torch.empty(workers, length, dtype=torch.int64)
    text[:, 0] = torch.randint(0, words, (workers,), generator=g)
    for t in range(1, length):
        pick = successors[text[:, t - 1], torch.randint(0, 4, (workers,), generator=g)]
        other = torch.randint(0, words, (workers,), generator=g)
        text[:, t] = torch.where(torch.rand(workers, generator=g) < 0.9, pick, other)
    return text.to(device)


def worker_gradient(model: Model, text: torch.Tensor, out: torch.Tensor) -> torch.Tensor:
    """Mean loss of one worker's text (fp32, on the device); its gradient goes to
    `out` (fp32 [d])."""
    n, k, width = text.numel(), model.context, model.width
    emb, mats, bias = model.split(model.x)
    emb16, bias16 = emb.bfloat16(), bias.bfloat16()
    target = text.clone()
    target[:k] = -1  # no full context
    before = [torch.roll(text, j + 1) for j in range(k)]
    places = [torch.empty(n, width, device=emb.device, dtype=torch.bfloat16) for _ in before]
    for w, p in zip(before, places):
        efs.ef_embed(emb16, w, p)
    h32 = sum(p.float() @ m.T for p, m in zip(places, mats))
    f = {"device": h32.device, "dtype": torch.float32}
    if model.norm:
        h = torch.empty_like(h32, dtype=torch.bfloat16)
        mean, rstd = torch.empty(n, **f), torch.empty(n, **f)
        weight, shift = model.norm_vectors(model.x)
        efs.ef_layer_norm(h32, h, weight, shift, mean_out=mean, rstd_out=rstd)
    else:
        h = h32.bfloat16()
    loss, lse = torch.empty(n, **f), torch.empty(n, **f)
    scale = torch.full((n,), 1.0 / (n - k), **f)
    dh, de, db = torch.empty_like(h), torch.empty_like(emb16), torch.empty_like(bias16)
    efs.ef_vocab_loss(h, emb16, target, loss, lse, bias=bias16)
    efs.ef_vocab_loss_grad(h, emb16, target, lse, scale, dh, de, bias=bias16, dbias_out=db)
    g_emb, g_mats, g_bias = model.split(out)
    g_emb.copy_(de)
    g_bias.copy_(db)
    if model.norm:
        dh32 = torch.empty_like(h32)
        efs.ef_layer_norm_grad(h32, mean, rstd, dh, dh32, weight, *model.norm_vectors(out))
    else:
        dh32 = dh.float()
    for w, p, m, g in zip(before, places, mats, g_mats):
        torch.matmul(dh32.T, p.float(), out=g)
        efs.ef_embed_grad(dh32 @ m, w, g_emb, accumulate=True)
    return loss.sum() / (n - k)


class Vectors:
    """The parameters that are no matrices of the context, and the rule that updates
    them from the exchanged gradient."""

    def __init__(self, model: Model, delta: torch.Tensor, rule: str, lr: float, lr_norm: float,
                 seed: int = 0):
        if rule not in ("sgd", "adamw", "adamw8"):
            raise ValueError("rule must be sgd, adamw or adamw8")
        emb, _, bias = model.split(model.x)
        d_emb, _, d_bias = model.split(delta)
        params = [emb, bias, *model.norm_vectors(model.x)]
        grads = [d_emb, d_bias, *model.norm_vectors(delta)]
        self.rule, self.lr, self.seed, self.step = rule, lr, seed, 0
        self.pairs = [(p, g, lr if i < 2 else lr_norm) for i, (p, g) in enumerate(zip(params, grads))]
        if rule == "sgd":
            return
        eight = rule == "adamw8"
        kind = torch.uint8 if eight else torch.float32
        states = [[torch.zeros(p.shape, device=p.device, dtype=kind) for p in params] for _ in "mv"]
        self.lists = [efs.TensorList(x) for x in (params, grads, *states)]
        self.exponents = [None, None]
        if eight:
            self.exponents = [efs.TensorList([torch.zeros(efs.exponents_for(p.numel()), device=p.device,
                                                          dtype=torch.uint8) for p in params])
                              for _ in "mv"]

    def update(self) -> None:
        self.step += 1
        if self.rule == "sgd":
            for p, g, lr in self.pairs:
                p.add_(g, alpha=-lr)
            return
        efs.ef_adamw(*self.lists, self.step, self.lr, weight_decay=0.0,
                     m_exponents=self.exponents[0], v_exponents=self.exponents[1], seed=self.seed)


def run(words: int = 2000, width: int = 96, context: int = 2, workers: int = 4, length: int = 256,
        steps: int = 100, lam: float = 2e-4, lr_matrix: float = 0.02, lr_table: float = 20.0,
        momentum: float = 0.9, seed: int = 0, device="cuda", norm: bool = False,
        rule: str = "sgd", lr_norm: float = 0.1, lr_adamw: float = 0.01) -> Dict[str, List[float]]:
    """Trains for `steps` iterations; records the workers' mean loss and the
    coordinates sent at each."""
    model = Model.create(words, width, context, seed, device, norm)
    text = make_text(words, length * steps, workers, seed, device)
    d = model.d
    f = {"device": device, "dtype": torch.float32}
    g, delta = torch.empty(d, **f), torch.empty(d, **f)
    e = torch.zeros(workers, d, **f)
    idx = [torch.empty(d, device=device, dtype=torch.int32) for _ in range(workers)]
    val = [torch.empty(d, **f) for _ in range(workers)]
    counts = torch.empty(workers, device=device, dtype=torch.int32)
    _, d_mats, _ = model.split(delta)
    _, mats, _ = model.split(model.x)
    vectors = Vectors(model, delta, rule, lr_table if rule == "sgd" else lr_adamw, lr_norm, seed)
    moments = [torch.zeros_like(m) for m in mats]
    ortho = [torch.empty_like(m, dtype=torch.bfloat16) for m in mats]
    losses, sent = [], []
    for t in range(steps):
        total = torch.zeros((), device=device)
        for w in range(workers):
            total += worker_gradient(model, text[w, t * length:(t + 1) * length], g)
            efs.ef_hard_threshold(g, e[w], 1.0, lam, idx[w], val[w], counts[w:w + 1])
        efs.sparse_aggregate(idx, val, counts, d, delta)
        delta /= workers
        efs.ef_orthogonalize(d_mats, ortho, momenta=moments, momentum=momentum)
        for m, o in zip(mats, ortho):
            m.add_(o, alpha=-lr_matrix)
        vectors.update()
        losses.append(total / workers)
        sent.append(counts.sum())
    if efs.ef_check_status() != efs.EF_OK:
        raise RuntimeError("device error during the run")
    return {"loss": torch.stack(losses).tolist(), "sent": torch.stack(sent).tolist(),
            "d": [float(d)]}


if __name__ == "__main__":
    import argparse
    import json
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--words", type=int, default=2000)
    ap.add_argument("--width", type=int, default=96)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--lam", type=float, default=2e-4)
    ap.add_argument("--norm", action="store_true", help="a layer norm before the decoder")
    ap.add_argument("--rule", choices=("sgd", "adamw", "adamw8"), default="sgd",
                    help="how the table, the bias and the norm's vectors are updated")
    args = ap.parse_args()
    h = run(words=args.words, width=args.width, workers=args.workers, steps=args.steps,
            lam=args.lam, norm=args.norm, rule=args.rule)
    print(json.dumps({"loss_first": h["loss"][0], "loss_last": sum(h["loss"][-10:]) / 10,
                      "density": sum(h["sent"]) / (len(h["sent"]) * args.workers * h["d"][0])}))

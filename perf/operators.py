"""Workloads of the operators on token sequences: the embedding lookup and its gradient, the gated linear recurrence, and the loss
that distils a teacher's top logits.

A case is one operator at one size and type; a pass is one call (for the recurrence in training: the forward and the backward
call).  `own` chooses between the library's entry points and plain torch operations in 32 bits, which need nothing of this library.

    embedding   y[n] = scale * W[tok[n]];  dW[v] = scale * sum over n with tok[n] = v of dy[n]     (ids outside the table: zeros, no gradient)
    recurrence  a = sigmoid(z), h_t = a_t h_{t-1} + (1 - a_t) v_t, y_t = h_t
    distill     w tau^2 KL(softmax(teacher / tau) | softmax(s / tau)) + (1 - w) CE(s, label), with the gradient for s times `scale`
"""
from __future__ import annotations

import math
import random

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}


def _embed(name, op, **kw):
    return dict(dict(name=name, op=op, dtype="bf16", tokens=16384, vocab=32000, channels=1024, padded=0.0), **kw)


def _recur(name, op, **kw):
    return dict(dict(name=name, op=op, dtype="bf16", batch=8, steps=2048, channels=1024, ragged=False), **kw)


def _distill(name, **kw):
    return dict(dict(name=name, op="distill", dtype="bf16", rows=4096, vocab=32000, top=64, tau=2.0, weight=0.7, padded=0.0), **kw)


def listed():
    return [
        # The first layer of a training step: 16 k tokens of a batch, rows of 2 KB.
        _embed("embed-bf16", "embed"),
        # A toy vocabulary on a handful of tokens, rows of no round number of bytes, some of them padding: nothing but latency.
        _embed("embed-grad-small-fp32", "embed-grad", dtype="fp32", tokens=97, vocab=1000, channels=100, padded=0.1),
        # The same batch as the first case on its way back: most of the time goes into the rows of the table no token names.
        _embed("embed-grad-bf16", "embed-grad"),
        # A large vocabulary and a large batch: the sort has work to do, and the commonest tokens have thousands of rows each.
        _embed("embed-grad-large-bf16", "embed-grad", tokens=131072, vocab=131072, channels=1024),
        # Serving: one new token for each of 64 sequences, from the state carried so far.
        _recur("recur-step-bf16", "recur-forward", batch=64, steps=1),
        # Serving: the prompt of one long sequence.
        _recur("recur-prompt-bf16", "recur-forward", batch=1, steps=16384, channels=2048),
        # Training: a batch of medium-length sequences, forward and backward.
        _recur("recur-train-bf16", "recur-train"),
        # Training on one very long sequence of odd length: few channels, everything along the sequence.
        _recur("recur-train-long-bf16", "recur-train", batch=1, steps=60001, channels=512),
        # Training in fp32 on a padded batch of short sequences of different lengths.
        _recur("recur-train-ragged-fp32", "recur-train", dtype="fp32", batch=12, steps=777, channels=200, ragged=True),
        # The classes and samples of this library's own image workloads.
        _distill("distill-classes-fp32", dtype="fp32", rows=1024, vocab=10, top=4),
        # Token-level distillation with both terms.
        _distill("distill-bf16"),
        # A vocabulary of odd size in fp32, the teacher's distribution only; some rows are padding.
        _distill("distill-large-fp32", dtype="fp32", rows=1500, vocab=100003, top=200, tau=1.0, weight=1.0, padded=0.1),
    ]


def _log_int(rng, lo, hi):
    """An integer in lo..hi, uniform over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng: random.Random):
    op = rng.choice(["embed", "embed-grad", "embed-grad", "recur-forward", "recur-train", "recur-train", "distill", "distill"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if op.startswith("embed"):
        c = _embed(None, op, dtype=dtype, tokens=_log_int(rng, 1, 131072), vocab=_log_int(rng, 10, 131072), padded=rng.choice([0.0, 0.0, 0.2]))
        c["channels"] = _log_int(rng, 1, max(1, min(2048, 131072 * 1024 // max(c["tokens"], c["vocab"]))))
        if rng.random() < 0.6:
            c["channels"] = min(1024, -(-c["channels"] // 64) * 64)
    elif op.startswith("recur"):
        c = _recur(None, op, dtype=dtype, batch=_log_int(rng, 1, 64), channels=_log_int(rng, 3, 2048), ragged=rng.random() < 0.3)
        if rng.random() < 0.6:
            c["channels"] = -(-c["channels"] // 64) * 64
        c["steps"] = _log_int(rng, 1, max(1, min(60001, (1 << 24) // (c["batch"] * c["channels"]))))
    else:
        c = _distill(None, dtype=dtype, vocab=_log_int(rng, 2, 200000), tau=rng.choice([1.0, 1.5, 2.0, 4.0]), weight=rng.choice([0.5, 0.9, 1.0]),
                     padded=rng.choice([0.0, 0.0, 0.3]))
        c["top"] = min(c["vocab"], _log_int(rng, 1, 256))
        c["rows"] = _log_int(rng, 1, max(1, min(16384, (1 << 27) // c["vocab"])))
    del c["name"]
    return c


def _tokens(case, g):
    """Ids of which the v-th commonest occurs about 1 / v as often as the commonest, as words do; padding as -1."""
    u = torch.rand(case["tokens"], generator=g, device="cuda", dtype=torch.float64)
    tok = (torch.exp(u * math.log(case["vocab"] + 1)) - 1).long().clamp_(0, case["vocab"] - 1)
    shuffled = torch.randperm(case["vocab"], generator=g, device="cuda")
    tok = shuffled[tok].int()
    if case["padded"]:
        tok[torch.rand(case["tokens"], generator=g, device="cuda") < case["padded"]] = -1
    return tok


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = DTYPES[case["dtype"]]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = dict(op=case["op"])
    if case["op"].startswith("embed"):
        s.update(tokens=_tokens(case, g), vocab=case["vocab"], scale=math.sqrt(case["channels"]))
        if case["op"] == "embed":
            s["table"] = (normal(case["vocab"], case["channels"]) / math.sqrt(case["channels"])).to(t)
        else:
            s["dy"] = (normal(case["tokens"], case["channels"]) * 1e-3).to(t)
    elif case["op"].startswith("recur"):
        b, n, c = case["batch"], case["steps"], case["channels"]
        # one tensor of 2 c channels, as a projection in front of the layer leaves it: gates, which mostly keep the state, then values
        x = normal(b, n, 2 * c)
        x[..., :c].mul_(1.5).add_(2.0)
        s.update(x=x.to(t), state=normal(b, c), lengths=None)
        if case["ragged"]:
            s["lengths"] = torch.randint(0, n + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        if case["op"] == "recur-train":
            s.update(dy=normal(b, n, c).to(t), dstate=normal(b, c))
    else:
        m, v, k = case["rows"], case["vocab"], case["top"]
        s.update(logits=(normal(m, v) * 2).to(t), tau=case["tau"], weight=case["weight"], scale=1.0 / m)
        s["labels"] = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
        if case["padded"]:
            s["labels"][torch.rand(m, generator=g, device="cuda") < case["padded"]] = -1
        # distinct ids of a row: a random start and a step without a common factor with the vocabulary
        step = next(p for p in (7919, 104729, 1) if v % p)
        start = torch.randint(0, v, (m, 1), generator=g, device="cuda")
        s["ids"] = ((start + step * torch.arange(k, device="cuda")) % v).int()
        s["teacher"] = (normal(m, k) * 2).sort(1, descending=True).values.contiguous()
    torch.cuda.synchronize()
    return s


def run(state):
    return _own(state) if own else _plain(state)


def _own(s):
    from paper_2509_05679_b200 import operators as ops
    if s["op"] == "embed":
        return ops.embedding(s["tokens"], s["table"], scale=s["scale"])
    if s["op"] == "embed-grad":
        return ops.embedding_grad(s["tokens"], s["dy"], s["vocab"], scale=s["scale"])
    if s["op"] == "distill":
        return ops.distill_loss(s["logits"], s["labels"], s["ids"], s["teacher"], temperature=s["tau"], weight=s["weight"], scale=s["scale"])
    x = s["x"]
    c = x.shape[2] // 2
    z, v = x[..., :c], x[..., c:]
    if s["op"] == "recur-forward":
        return ops.recurrence(z, v, state=s["state"], lengths=s["lengths"])
    y, last, saved = ops.recurrence(z, v, state=s["state"], lengths=s["lengths"], for_grad=True)
    dx = torch.empty_like(x)
    dstate = ops.recurrence_grad(z, v, s["dy"], saved, dstate=s["dstate"], lengths=s["lengths"], dgate=dx[..., :c], dvalue=dx[..., c:])
    return y, last, dx, dstate


# ---- plain forms: elementary operations in 32 bits, rounded once at the end

def _plain(s):
    if s["op"] == "embed":
        tok = s["tokens"].long()
        ok = ((tok >= 0) & (tok < s["vocab"]))[:, None]
        return (s["table"][tok.clamp(0, s["vocab"] - 1)].float() * s["scale"] * ok).to(s["table"].dtype)
    if s["op"] == "embed-grad":
        tok = s["tokens"].long()
        ok = ((tok >= 0) & (tok < s["vocab"]))[:, None]
        dw = torch.zeros(s["vocab"], s["dy"].shape[1], device="cuda")
        return dw.index_add_(0, tok.clamp(0, s["vocab"] - 1), s["dy"].float() * s["scale"] * ok)
    if s["op"] == "distill":
        return _plain_distill(s)
    return _plain_recurrence(s)


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along dimension 1 from 0, and the products of a: distances 1, 2, 4, ... combined one after the other."""
    a, h, d = a.clone(), u.clone(), 1
    while d < h.shape[1]:
        h2 = torch.cat([h[:, :d], h[:, d:] + a[:, d:] * h[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        h, d = h2, 2 * d
    return h, a


def _plain_recurrence(s):
    x = s["x"]
    n, c = x.shape[1], x.shape[2] // 2
    z, v = x[..., :c].float(), x[..., c:].float()
    a, b = 1 / (1 + torch.exp(-z)), 1 / (1 + torch.exp(z))
    u = b * v
    live = None
    if s["lengths"] is not None:
        live = (torch.arange(n, device="cuda")[None, :] < s["lengths"][:, None])[..., None]
        a, u = torch.where(live, a, 1.0), torch.where(live, u, 0.0)
    h, p = _scan(a, u)
    h = h + p * s["state"][:, None]
    last = h[:, -1].clone()
    y = (h if live is None else h * live).to(x.dtype)
    if s["op"] == "recur-forward":
        return y, last
    dy = s["dy"].float() if live is None else s["dy"].float() * live
    # e_t = d_t - dy_t, the gradient that later steps send back: e_t = a_{t+1} (e_{t+1} + dy_{t+1}); the last one is dstate
    ar, r = a.flip(1), (a * dy).flip(1)
    g, p = _scan(ar, r)
    g = (g + p * s["dstate"][:, None]).flip(1)                      # g_t = a_t d_t
    d = dy + torch.cat([g[:, 1:], s["dstate"][:, None]], 1)
    before = torch.cat([s["state"][:, None], h[:, :-1]], 1)
    dz, dv = a * b * d * (before - v), b * d
    if live is not None:
        dz, dv = dz * live, dv * live
    return y, last, torch.cat([dz, dv], 2).to(x.dtype), g[:, 0].clone()


def _plain_distill(s):
    x = s["logits"].float()
    m = x.max(1, keepdim=True).values
    live = s["labels"] >= 0
    y = s["labels"].clamp(min=0).long()[:, None]
    e = torch.exp((x - m) / s["tau"])
    total = e.sum(1, keepdim=True)
    t = (s["teacher"] - s["teacher"].max(1, keepdim=True).values) / s["tau"]
    p = torch.exp(t)
    psum = p.sum(1, keepdim=True)
    logp, p = t - torch.log(psum), p / psum
    ids = s["ids"].long()
    logq = (x.gather(1, ids) - m) / s["tau"] - torch.log(total)
    loss = s["weight"] * s["tau"] ** 2 * (p * (logp - logq)).sum(1)
    grad = (e / total).scatter_add_(1, ids, -p) * (s["weight"] * s["tau"])
    if s["weight"] < 1:
        e = torch.exp(x - m)
        total = e.sum(1, keepdim=True)
        loss = loss + (1 - s["weight"]) * (torch.log(total) - (x.gather(1, y) - m))[:, 0]
        grad = grad + (1 - s["weight"]) * (e / total).scatter_add_(1, y, -torch.ones_like(total))
    return loss * live, (grad * live[:, None] * s["scale"]).to(s["logits"].dtype)


def work(case):
    z = SIZE[case["dtype"]]
    if case["op"].startswith("embed"):
        n, v, c = case["tokens"], case["vocab"], case["channels"]
        if case["op"] == "embed-grad":
            return {"bytes": 4 * n + z * n * c + 4 * v * c, "flops": 2 * n * c}
        return {"bytes": 4 * n + z * c * (n + _distinct(n, v)), "flops": n * c}
    if case["op"].startswith("recur"):
        b, n, c = case["batch"], case["steps"], case["channels"]
        if case["op"] == "recur-forward":
            return {"bytes": 3 * z * b * n * c + 8 * b * c, "flops": 8 * b * n * c}
        return {"bytes": 6 * z * b * n * c + 16 * b * c, "flops": 24 * b * n * c}
    m, v, k = case["rows"], case["vocab"], case["top"]
    return {"bytes": 2 * z * m * v + 8 * m * k + 8 * m, "flops": (8 if case["weight"] == 1 else 14) * m * v}


def _distinct(n, v):
    """About how many different ids n of _tokens' are."""
    total, lo = 0.0, 1
    while lo <= v:                                                  # ranks in octaves: P(rank r) = 1 / (r ln(v + 1))
        hi = min(v + 1, 2 * lo)
        total += (hi - lo) * (1 - math.exp(-n / (math.sqrt(lo * hi) * math.log(v + 1))))
        lo = hi
    return int(total)


# ---- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "embed":
        w = torch.cat([s["table"].double(), torch.zeros(1, case["channels"], device="cuda", dtype=torch.float64)])
        tok = torch.where((s["tokens"] < 0) | (s["tokens"] >= case["vocab"]), case["vocab"], s["tokens"]).long()
        return w[tok] * s["scale"]
    if case["op"] == "embed-grad":
        keep = (s["tokens"] >= 0) & (s["tokens"] < case["vocab"])
        tok, rows = s["tokens"][keep].long(), s["dy"][keep].double()
        order = torch.argsort(tok)
        ids, count = torch.unique_consecutive(tok[order], return_counts=True)
        dw = torch.zeros(case["vocab"], case["channels"], device="cuda", dtype=torch.float64)
        if len(ids):
            ends = torch.cumsum(count, 0)
            for lo in range(0, case["channels"], 128):              # running sums of a slice of the channels at a time
                run_ = torch.cumsum(rows[order, lo:lo + 128], 0)[ends - 1]
                dw[ids, lo:lo + 128] = torch.diff(run_, dim=0, prepend=torch.zeros_like(run_[:1])) * s["scale"]
        return dw
    if case["op"] == "distill":
        return _exact_distill(case, s)
    b, n, c = case["batch"], case["steps"], case["channels"]
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((b,), n, device="cuda", dtype=torch.int32)
    h, ys, hs = s["state"].double(), [], []
    for t in range(n):                                              # step by step, as it is defined
        live = (t < lengths)[:, None]
        a = torch.sigmoid(s["x"][:, t, :c].double())
        new = a * h + (1 - a) * s["x"][:, t, c:].double()
        hs.append(h)
        h = torch.where(live, new, h)
        ys.append(torch.where(live, new, 0.0))
    y = torch.stack(ys, 1)
    if case["op"] == "recur-forward":
        return y, h
    del ys
    d, dxs = s["dstate"].double(), []
    for t in reversed(range(n)):
        live = (t < lengths)[:, None]
        a, v = torch.sigmoid(s["x"][:, t, :c].double()), s["x"][:, t, c:].double()
        full = d + s["dy"][:, t].double()
        dxs.append(torch.where(live.expand(b, 2 * c), torch.cat([a * (1 - a) * full * (hs[t] - v), (1 - a) * full], 1), 0.0))
        d = torch.where(live, a * full, d)
        hs[t] = None
    return y, h, torch.stack(dxs[::-1], 1), d


def _exact_distill(case, s):
    loss, grad = [], []
    rows = max(1, (1 << 25) // case["vocab"])
    for lo in range(0, case["rows"], rows):
        x = s["logits"][lo:lo + rows].double()
        lab, ids = s["labels"][lo:lo + rows].long(), s["ids"][lo:lo + rows].long()
        p = torch.log_softmax(s["teacher"][lo:lo + rows].double() / s["tau"], 1)
        q = torch.log_softmax(x / s["tau"], 1)
        live = (lab >= 0).double()
        one = torch.zeros_like(x).scatter_(1, lab.clamp(min=0)[:, None], 1.0)
        soft = torch.zeros_like(x).scatter_add_(1, ids, p.exp())
        hard = torch.log_softmax(x, 1)
        w, tau = s["weight"], s["tau"]
        loss.append(live * (w * tau * tau * (p.exp() * (p - q.gather(1, ids))).sum(1) - (1 - w) * (hard * one).sum(1)))
        grad.append((live * s["scale"])[:, None] * (w * tau * (q.exp() - soft) + (1 - w) * (hard.exp() - one)))
    return torch.cat(loss), torch.cat(grad)

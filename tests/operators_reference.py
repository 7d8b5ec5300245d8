"""Plain 64-bit forms of the operators on token sequences, with bounds on what 32-bit evaluations of them can be off by.

Every function returns exact values and, beside each, how far a result may be from it.  U = 2^-24 is the largest relative rounding error of one fp32
operation; a stored result adds half a step of its type (`store`).  A sum of terms evaluated in any order is off by at most (operations on the longest path)
x U x (sum of the terms' magnitudes); how the bounds count those operations stands beside them."""
import torch

U = 2.0 ** -24
F64 = torch.float64


def store(exact, err, dtype):
    """Bound of a result that is `err` off before it is rounded to dtype (the step of what is rounded, and the least normal number where values fall below it)."""
    info = torch.finfo(dtype)
    return err + info.eps / 2 * (exact.abs() + err) + info.tiny * info.eps


def embedding(tokens, table, scale):
    """One product: one rounding in 32 bits, one of the store."""
    v = table.shape[0]
    t = tokens.long()
    ok = ((t >= 0) & (t < v))[..., None]
    y = torch.where(ok, table.to(F64)[t.clamp(0, v - 1)] * scale, 0.0)
    return y, store(y, U * y.abs(), table.dtype)


def embedding_grad(tokens, dy, vocab, scale, start=None):
    """A row is a sum of `count` terms, times the scale, plus what was there: count + 1 operations at the most, in any order."""
    t = tokens.long().reshape(-1)
    keep = (t >= 0) & (t < vocab)
    rows = dy.reshape(-1, dy.shape[-1])[keep].to(F64) * scale
    t = t[keep]
    zero = torch.zeros(vocab, dy.shape[-1], dtype=F64, device=dy.device)
    # by products with a 0/1 matrix, not by scattered adds: a definition of its own
    dw, mag = zero.clone(), zero.clone()
    for lo in range(0, vocab, 4096):
        hot = (torch.arange(lo, min(vocab, lo + 4096), device=dy.device)[:, None] == t[None, :]).to(F64)
        dw[lo:lo + 4096] = hot @ rows
        mag[lo:lo + 4096] = hot @ rows.abs()
    count = torch.bincount(t, minlength=vocab).to(F64)[:, None]
    if start is not None:
        dw, mag = dw + start.to(F64), mag + start.to(F64).abs()
    return dw, (count + 1) * U * mag * 1.001


# Recurrence.  h_t is the sum of u_s a_{s+1} ... a_t over s <= t (u_0 = h_0), in whatever order the steps are combined: by each of the a's the term takes at
# most K roundings (the gate's own error, a product, a sum) and, where parts of the sequence are joined as a tree, two per level more, LEVELS in all.
# The gate: exp to 2 units of 2 U and z log2(e) to |z| U, a sum, a reciprocal to 2 U, a product: (8 + |z|) U, product and sum of the step 2 U.
LEVELS = 40


def _k(z):
    z = z.to(F64)
    return 12 + z[z.isfinite()].abs().amax() if z.isfinite().any() else torch.tensor(12.0, dtype=F64, device=z.device)


def recurrence(gate, value, state, lengths):
    """(y, its bound, last state, its bound, (h before every step, its bound))"""
    b, n, c = gate.shape
    z, v = gate.to(F64), value.to(F64)
    k = _k(gate)
    h = torch.zeros(b, c, dtype=F64, device=gate.device) if state is None else state.to(F64)
    m, w = h.abs(), torch.zeros_like(h)                     # sum of |terms|; sum of |terms| x their steps
    ys, es, hs, he = [], [], [], []
    for t in range(n):
        live = torch.ones(b, 1, dtype=torch.bool, device=gate.device) if lengths is None else (t < lengths)[:, None]
        hs.append(h)
        he.append(U * (k * w + LEVELS * m))
        a, g = torch.sigmoid(z[:, t]), torch.sigmoid(-z[:, t])
        u = g * v[:, t]
        h = torch.where(live, a * h + u, h)
        w = torch.where(live, a * (w + m) + u.abs(), w)
        m = torch.where(live, a * m + u.abs(), m)
        ys.append(torch.where(live, h, 0.0))
        es.append(torch.where(live, U * (k * w + LEVELS * m), 0.0))
    stack = lambda x: torch.stack(x, 1) if x else torch.zeros(b, 0, c, dtype=F64, device=gate.device)
    y = stack(ys)
    return y, store(y, stack(es), gate.dtype), h, U * (k * w + LEVELS * m) + U * h.abs(), (stack(hs), stack(he))


def recurrence_grad(gate, value, state, lengths, dy, dstate):
    """((dgate, bound), (dvalue, bound), (dstate of h_0, bound)).  d_t is a sum like h's, backwards; dvalue and dgate are products of it, with the errors of
    their factors added up: those of a and 1 - a, k U each, of d, and of h_{t-1} - value_t."""
    b, n, c = gate.shape
    z, v = gate.to(F64), value.to(F64)
    k = _k(gate)
    _, _, _, _, (hs, he) = recurrence(gate, value, state, lengths)
    g = torch.zeros(b, c, dtype=F64, device=gate.device) if dstate is None else dstate.to(F64)
    m, w = g.abs(), torch.zeros_like(g)
    dz, ez, dv, ev = ([None] * n for _ in range(4))
    for t in reversed(range(n)):
        live = torch.ones(b, 1, dtype=torch.bool, device=gate.device) if lengths is None else (t < lengths)[:, None]
        a, q = torch.sigmoid(z[:, t]), torch.sigmoid(-z[:, t])
        d, dm, dw = g + dy[:, t].to(F64), m + dy[:, t].to(F64).abs(), w
        de = U * (k * dw + (LEVELS + 1) * dm)
        diff = hs[:, t] - v[:, t]
        fe = he[:, t] + 2 * U * (hs[:, t].abs() + v[:, t].abs())
        dv[t] = torch.where(live, q * d, 0.0)
        ev[t] = torch.where(live, q * (de + (k + 2) * U * dm), 0.0)
        dz[t] = torch.where(live, a * q * d * diff, 0.0)
        ez[t] = torch.where(live, a * q * (diff.abs() * (de + (2 * k + 4) * U * dm) + dm * fe), 0.0)
        g = torch.where(live, a * d, g)
        w = torch.where(live, a * (dw + dm), w)
        m = torch.where(live, a * dm, m)
    stack = lambda x: torch.stack(x, 1) if x else torch.zeros(b, 0, c, dtype=F64, device=gate.device)
    dz, ez, dv, ev = map(stack, (dz, ez, dv, ev))
    return (dz, store(dz, ez, gate.dtype)), (dv, store(dv, ev, gate.dtype)), (g, U * (k * w + (LEVELS + 1) * m) + U * g.abs())


def distill(logits, labels, ids, teacher, tau, weight, scale, grad_dtype):
    """((loss, bound), (gradient, bound)).  An exponential of x = (s - max) / tau is off by (3 |x| + 4) U relative (difference, product, the function), a sum over the
    vocabulary in at least 256 parts by `depth` U more, a logarithm of it by as much absolutely.  An exponential below TINY, the least normal number, may count as
    zero (it is one of a sum that is at least 1, the maximum's own): that takes at most TINY from q, V TINY from the sum, which is nothing beside U."""
    TINY = 2.0 ** -126
    m, v = logits.shape
    x = logits.to(F64)
    live = torch.ones(m, dtype=torch.bool, device=logits.device) if labels is None else (labels >= 0) & (labels < v)
    y = None if labels is None else torch.where(live, labels, 0).long()
    depth = -(-v // 256) + 12
    xm = x.amax(1, keepdim=True)
    loss, lerr = torch.zeros(m, dtype=F64, device=logits.device), torch.zeros(m, dtype=F64, device=logits.device)
    grad, gerr = torch.zeros_like(x), torch.zeros_like(x)

    def softmax(t):
        """softmax(x / t), the logarithm, relative error of the first, absolute error of the second"""
        lq = torch.log_softmax(x / t, 1)
        far = ((x - xm) / t).abs()
        far = torch.where(far.isfinite(), far, 0.0)
        q = lq.exp()
        mean = (q * far).sum(1, keepdim=True)               # errors of the sum: each term's, weighed by it
        sums = (3 * mean + 4 + depth) * U
        return q, lq, (3 * far + 6) * U + sums, (3 * far + 4) * U + sums + U * lq.abs() + 2 * U * (lq + far).abs()

    if weight > 0 and ids.shape[1]:
        inside = (ids >= 0) & (ids < v)
        at = torch.where(inside, ids, 0).long()
        t = torch.where(inside, teacher.to(F64), -torch.inf)
        taught = t.amax(1, keepdim=True) != -torch.inf
        lp = torch.log_softmax(torch.where(taught, t, 0.0) / tau, 1)
        p = torch.where(taught, lp.exp(), 0.0)
        far = (t - t.amax(1, keepdim=True)).abs() / tau
        far = torch.where(far.isfinite(), far, 0.0)
        perr = (3 * far + 10 + 3 * (p * far).sum(1, keepdim=True) + 20) * U          # relative
        q, lq, qrel, lqabs = softmax(tau)
        some = p > 0
        diff = torch.where(some, lp - lq.gather(1, at), 0.0)
        loss = weight * tau ** 2 * (p * diff).sum(1)
        lerr = weight * tau ** 2 * (p * torch.where(some, lqabs.gather(1, at) + perr * (1 + diff.abs()) + U * lp.abs(), 0.0) + (12 + 4) * U * (p * diff.abs())).sum(1)
        soft = torch.zeros_like(x).scatter_add_(1, at, torch.where(inside, p, 0.0))
        serr = torch.zeros_like(x).scatter_add_(1, at, torch.where(inside, p * (perr + ids.shape[1] * U), 0.0))
        on = taught.to(F64) * weight * tau
        grad = on * (q - soft)
        gerr = on * (q * qrel + serr + 4 * U * (q + soft) + TINY)
    if weight < 1:
        q, lq, qrel, lqabs = softmax(1.0)
        one = torch.zeros_like(x).scatter_(1, y[:, None], 1.0)
        hard = -lq.gather(1, y[:, None])[:, 0]
        loss = loss + (1 - weight) * hard
        lerr = lerr + (1 - weight) * (lqabs.gather(1, y[:, None])[:, 0] + 2 * U * hard.abs())
        grad = grad + (1 - weight) * (q - one)
        gerr = gerr + (1 - weight) * (q * qrel + 4 * U * (q + one) + TINY)
    lerr = lerr + 4 * U * loss.abs()
    gerr = gerr + 2 * U * grad.abs()
    live2 = live[:, None]
    loss, lerr = torch.where(live, loss, 0.0), torch.where(live, lerr, 0.0)
    grad, gerr = torch.where(live2, grad * scale, 0.0), torch.where(live2, gerr * abs(scale), 0.0)
    return (loss, lerr), (grad, store(grad, gerr, grad_dtype))


def check(got, exact, bound, what):
    """Within the bound everywhere; infinities and NaN where the exact values have them."""
    got = got.to(F64)
    assert got.shape == exact.shape, (what, got.shape, exact.shape)
    if not got.numel():
        return
    fine = exact.isfinite()
    assert torch.equal(got.isnan(), exact.isnan()), f"{what}: NaN in the wrong places"
    odd = ~fine & ~exact.isnan()
    assert torch.equal(got[odd], exact[odd]), f"{what}: infinities"
    off = torch.where(fine, (got - exact).abs() - bound, -1.0)
    worst = off.argmax()
    assert off.max() <= 0, f"{what}: {got.flatten()[worst].item()} for {exact.flatten()[worst].item()}, bound {bound.flatten()[worst].item()} at {worst.item()}"

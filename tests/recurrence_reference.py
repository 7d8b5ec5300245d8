"""The recurrence of operators_reference.py on long sequences: the same values and bounds, found in pieces of a sequence side by side instead of step by step, and how the
library cuts a launch, by which the long tests choose their sizes."""
import math

import torch

from operators_reference import F64, LEVELS, U, _k, store

# (sequences, steps, channels): between them every cut, rows on 16 bytes and not, slices that are not full, and rounds enough to use every stage of the rings three times
SHAPES = [(64, 4000, 24), (64, 4000, 17), (9, 8000, 136), (9, 16000, 72), (1, 33000, 24), (2, 33000, 17), (64, 2000, 72), (40, 8000, 24), (40, 8000, 17), (20, 16000, 24),
          (150, 700, 128), (150, 200, 256), (40, 200, 1030)]
CUTS = {(64, 1), (32, 1), (8, 1), (8, 4), (8, 8), (4, 1), (4, 2), (4, 4), (4, 8)}
STAGES = 3                                       # of the longest ring


def cut(b, n, c):
    """(threads along the channels, CTAs of a cluster): the least of the model's times, as csrc/recur.cu has it."""
    best, least = (64, 1), math.inf
    for cx in (64, 32, 8, 4):
        tile = 256 // cx * 4
        tiles, groups = -(-n // tile), b * -(-c // (4 * cx))
        r = 1
        while r <= (1 if cx > 8 else 8) and (r == 1 or r <= tiles):
            rounds, w = -(-tiles // r), groups * r / 148
            each = 1.5 + 0.9 * min(1.0, max(0.0, w - 1.0))
            if cx > 8:
                each *= 1.2
            if r > 1:
                each += 0.6
            us = (5 if r > 1 else 3) + (rounds * each if w <= 2 else math.ceil(w / 2) * (rounds * each + 1))
            if us < least - 1e-9:
                best, least = (cx, r), us
            r *= 2
    return best


def rounds(b, n, c, bf16, back):
    """How often a CTA goes through its ring's tiles: 4 steps a thread, forward in bf16 8."""
    cx, r = cut(b, n, c)
    tile = 256 // cx * (8 if bf16 and not back else 4)
    return -(-(-(-n // tile)) // r)


def scan(a, u, start, live):
    """x_t = a_t x_{t-1} + u_t (a = 1, u = 0 where not live).  Before every step and at the end: x, and for its bound m, the same of the terms' magnitudes, and w, those times the steps
    they went through: w_t = a_t (w_{t-1} + m_{t-1}) + |u_t|."""
    b, n, c = a.shape
    size = max(1, math.isqrt(n))
    pieces = -(-n // size)
    pad = pieces * size - n

    def cutup(x, fill):
        x = torch.cat([x, torch.full((b, pad, x.shape[2]), fill, dtype=x.dtype, device=x.device)], 1)
        return x.view(b, pieces, size, x.shape[2])
    a, u, live = cutup(a, 1.0), cutup(u, 0.0), cutup(live.expand(b, n, 1), False)

    def through(t, x, m, w):
        at, ut = a[:, :, t], u[:, :, t]
        return at * x + ut, at * m + ut.abs(), torch.where(live[:, :, t], at * (w + m) + ut.abs(), w)
    zero = torch.zeros(b, pieces, c, dtype=F64, device=a.device)
    x, m, w, prod = zero, zero, zero, torch.ones_like(zero)
    for t in range(size):
        x, m, w = through(t, x, m, w)
        prod = prod * a[:, :, t]
    count = live.sum(2).to(F64)                             # steps of a piece that count
    at, starts = (start, start.abs(), torch.zeros_like(start)), []
    for p in range(pieces):
        starts.append(at)
        at = (prod[:, p] * at[0] + x[:, p], prod[:, p] * at[1] + m[:, p], prod[:, p] * (at[2] + count[:, p] * at[1]) + w[:, p])
    state = tuple(torch.stack(s, 1) for s in zip(*starts))
    before = []
    for t in range(size):
        before.append(state)
        state = through(t, *state)
    join = lambda i: torch.stack([s[i] for s in before], 2).reshape(b, pieces * size, c)[:, :n]
    return (join(0), join(1), join(2)), at


def recurrence(gate, value, state, lengths, dy=None, dstate=None):
    """{name: (exact, bound)} of y, last and, given dy, dgate, dvalue and first: operators_reference.recurrence and recurrence_grad."""
    b, n, c = gate.shape
    k = _k(gate)
    live = torch.ones(b, n, 1, dtype=torch.bool, device=gate.device) if lengths is None else (torch.arange(n, device=gate.device)[None, :] < lengths[:, None])[..., None]
    z, v = torch.where(live, gate, 0.0).to(F64), torch.where(live, value, 0.0).to(F64)
    zero = torch.zeros(b, c, dtype=F64, device=gate.device)
    a, q = torch.where(live, torch.sigmoid(z), 1.0), torch.sigmoid(-z)
    u = torch.where(live, q * v, 0.0)
    (h, m, w), (last, lm, lw) = scan(a, u, zero if state is None else state.to(F64), live)
    err = lambda m, w, levels=LEVELS: U * (k * w + levels * m)
    y = torch.where(live, a * h + u, 0.0)
    ye = torch.where(live, err(a * m + u.abs(), a * (w + m) + u.abs()), 0.0)
    out = dict(y=(y, store(y, ye, gate.dtype)), last=(last, err(lm, lw) + U * last.abs()))
    if dy is None:
        return out
    e = torch.where(live, dy, 0.0).to(F64)
    back = lambda x: x.flip(1)
    (g, gm, gw), (first, fm, fw) = scan(back(a), back(torch.where(live, a * e, 0.0)), zero if dstate is None else dstate.to(F64), back(live))
    d, dm, dw = back(g) + e, back(gm) + e.abs(), back(gw)
    de, diff = err(dm, dw, LEVELS + 1), h - v
    fe = err(m, w) + 2 * U * (h.abs() + v.abs())
    dv, dz = torch.where(live, q * d, 0.0), torch.where(live, a * q * d * diff, 0.0)
    ev = torch.where(live, q * (de + (k + 2) * U * dm), 0.0)
    ez = torch.where(live, a * q * (diff.abs() * (de + (2 * k + 4) * U * dm) + dm * fe), 0.0)
    out.update(dgate=(dz, store(dz, ez, gate.dtype)), dvalue=(dv, store(dv, ev, gate.dtype)), first=(first, err(fm, fw, LEVELS + 1) + U * first.abs()))
    return out

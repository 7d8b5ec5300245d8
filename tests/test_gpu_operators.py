"""The operators on token sequences against their definitions in 64 bits, with bounds on what 32-bit arithmetic and one rounding of the result can be off
by (operators_reference.py), at the sizes, strides and masks where they can go wrong; repeated, captured and concurrent calls."""
import zlib

import pytest
import torch

import operators_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16]
NAN = float("nan")


@pytest.fixture(scope="module")
def ops():
    from paper_2509_05679_b200 import operators
    return operators


def _gen(*key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def _normal(g, *shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _f32(v):
    """A Python number as the library gets it."""
    return float(torch.tensor(v, dtype=torch.float32))


def _tokens(g, n, vocab, kind):
    if kind == "one":
        return torch.full((n,), vocab // 2, device="cuda", dtype=torch.int32)
    if kind == "none":
        t = torch.full((n,), -1, device="cuda", dtype=torch.int32)
        t[1::2] = vocab
        t[2::4] = -2 ** 31
        t[3::4] = 2 ** 31 - 1
        return t
    if kind == "skewed":        # the commonest id a quarter of all, the next an eighth, ...
        u = torch.rand(n, generator=g, device="cuda")
        return (-torch.log2(u.clamp(min=1e-9)) * 0.5).floor().int() % vocab
    t = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "padded":
        t[torch.rand(n, generator=g, device="cuda") < 0.4] = -1
    return t


# ---- embedding

EMBED = [(1, 1, 1), (1, 10, 8), (5, 3, 7), (33, 1000, 100), (64, 2, 64), (257, 70001, 24), (512, 9000, 36), (513, 1, 5), (1000, 50, 129), (2100, 300, 40), (700, 128, 1024),
         (300, 37, 2050), (1025, 148, 12), (1537, 149, 3), (9001, 40, 4)]


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("n,vocab,c", EMBED)
@pytest.mark.parametrize("kind", ["uniform", "padded", "none"])
def test_embedding(ops, n, vocab, c, dtype, kind):
    g = _gen("embed", n, vocab, c, kind)
    table = _normal(g, vocab, c, dtype=dtype)
    tok = _tokens(g, n, vocab, kind)
    y = ops.embedding(tok, table, scale=1.7)
    ref.check(y, *ref.embedding(tok, table, _f32(1.7)), "y")
    # rows apart, on an odd address: what is between them stays
    wide = torch.full((n * (c + 3) + 1,), 7.0, dtype=dtype, device="cuda")
    out = wide[1:].view(n, c + 3)[:, :c]
    ops.embedding(tok, table, scale=1.7, out=out)
    assert torch.equal(out, y)
    assert (wide[1:].view(n, c + 3)[:, c:] == 7).all() and wide[0] == 7


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_embedding_of_a_table_on_an_odd_address(ops, dtype):
    g = _gen("odd")
    flat = _normal(g, 1 + 50 * 64, dtype=dtype)
    tok = _tokens(g, 100, 50, "uniform")
    table = flat[1:].view(50, 64)
    ref.check(ops.embedding(tok, table), *ref.embedding(tok, table, 1.0), "y")


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("kind", ["uniform", "padded", "one", "none", "skewed"])
@pytest.mark.parametrize("n,vocab,c", EMBED)
def test_embedding_gradient(ops, n, vocab, c, kind, dtype):
    g = _gen("grad", n, vocab, c, kind)
    tok = _tokens(g, n, vocab, kind)
    dy = _normal(g, n, c, dtype=dtype)
    dy[(tok < 0) | (tok >= vocab)] = NAN                    # rows that take no part
    dw = ops.embedding_grad(tok, dy, vocab, scale=0.3)
    ref.check(dw, *ref.embedding_grad(tok, dy, vocab, _f32(0.3)), "dtable")
    assert torch.equal(dw, ops.embedding_grad(tok, dy, vocab, scale=0.3, out=torch.full_like(dw, NAN)))        # all written, same bits
    # added to what is there; rows of dy apart, on an odd address
    start = _normal(g, vocab, c)
    unused = torch.ones(vocab, dtype=torch.bool, device="cuda")
    unused[tok[(tok >= 0) & (tok < vocab)].long()] = False
    start[unused] = NAN
    wide = torch.full((n * (c + 5) + 1,), NAN, dtype=dtype, device="cuda")
    apart = wide[1:].view(n, c + 5)[:, :c]
    apart.copy_(dy)
    dw = ops.embedding_grad(tok, apart, vocab, scale=0.3, out=start.clone(), accumulate=True)
    exact, bound = ref.embedding_grad(tok, dy, vocab, _f32(0.3), torch.where(unused[:, None], 0.0, start))
    ref.check(torch.where(unused[:, None], 0.0, dw), exact, bound, "dtable, added")
    assert dw[unused].isnan().all()


@pytest.mark.parametrize("kind", ["uniform", "padded", "one", "skewed"])
@pytest.mark.parametrize("n,vocab,c", [(9000, 1000, 64), (40000, 33000, 16), (70000, 300000, 8), (150001, 17, 40), (3000, 4000003, 2)])
def test_embedding_gradient_of_many_tokens(ops, n, vocab, c, kind):
    g = _gen("many", n, vocab, c, kind)
    tok = _tokens(g, n, vocab, kind)
    dy = _normal(g, n, c, dtype=torch.bfloat16)
    dw = ops.embedding_grad(tok, dy, vocab)
    keep = tok >= 0
    exact = torch.zeros(vocab, c, dtype=ref.F64, device="cuda").index_add_(0, tok[keep].long(), dy[keep].to(ref.F64))
    mag = torch.zeros(vocab, c, dtype=ref.F64, device="cuda").index_add_(0, tok[keep].long(), dy[keep].to(ref.F64).abs())
    count = torch.bincount(tok[keep].long(), minlength=vocab).to(ref.F64)[:, None]
    ref.check(dw, exact, (count + 1) * ref.U * mag * 1.001, "dtable")
    assert torch.equal(dw, ops.embedding_grad(tok, dy, vocab))


def test_embedding_of_nothing(ops):
    table = torch.ones(4, 6, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert ops.embedding(none, table).shape == (0, 6)
    assert (ops.embedding_grad(none, torch.empty(0, 6, device="cuda"), 4, out=torch.full((4, 6), NAN, device="cuda")) == 0).all()
    kept = torch.full((4, 6), 3.0, device="cuda")
    assert (ops.embedding_grad(none, torch.empty(0, 6, device="cuda"), 4, out=kept, accumulate=True) == 3).all()


def test_embedding_of_a_tensor_of_tokens(ops):
    g = _gen("shape")
    tok = _tokens(g, 24, 9, "uniform").view(2, 3, 4)
    table = _normal(g, 9, 5)
    y = ops.embedding(tok, table)
    assert y.shape == (2, 3, 4, 5) and torch.equal(y, table[tok.long()])
    assert torch.equal(ops.embedding_grad(tok, y, 9), ops.embedding_grad(tok.view(-1), y.view(-1, 5), 9))


# ---- recurrence

RECUR = [(1, 1, 1), (3, 1, 64), (70, 1, 1030), (2, 5, 3), (1, 33, 8), (5, 16, 136), (2, 129, 100), (3, 1000, 64), (1, 5000, 72), (9, 64, 512), (1, 2049, 17), (33, 20, 256)]


def _layout(g, b, n, c, dtype, layout):
    """gate and value with the layout's strides."""
    if layout == "halves":
        x = _normal(g, b, n, 2 * c, dtype=dtype)
        return x[..., :c], x[..., c:]
    if layout == "time-major":
        return _normal(g, n, b, c, dtype=dtype).transpose(0, 1), _normal(g, n, b, c, dtype=dtype).transpose(0, 1)
    if layout == "odd":
        x = _normal(g, b * n * (2 * c + 1) + 1, dtype=dtype)[1:].view(b, n, 2 * c + 1)
        return x[..., :c], x[..., c + 1:]
    return _normal(g, b, n, c, dtype=dtype), _normal(g, b, n, c, dtype=dtype)


def _lengths(g, b, n, kind):
    if kind == "full":
        return None
    t = torch.randint(0, n + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
    t[0] = 0
    if b > 1:
        t[1] = n + 5               # clamped
    if b > 2:
        t[2] = -3
    return t


def _run_recurrence(ops, gate, value, state, lengths, dy, dstate, dx):
    y, last, saved = ops.recurrence(gate, value, state=state, lengths=lengths, for_grad=True)
    first = ops.recurrence_grad(gate, value, dy, saved, dgate=dx[0], dvalue=dx[1], dstate=dstate, lengths=lengths)
    return y, last, first


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("kind,layout", [("full", "halves"), ("ragged", "plain"), ("full", "time-major"), ("ragged", "odd")])
@pytest.mark.parametrize("b,n,c", RECUR)
def test_recurrence_and_gradient(ops, b, n, c, kind, layout, dtype):
    g = _gen("recur", b, n, c, kind, layout)
    gate, value = _layout(g, b, n, c, dtype, layout)
    gate.mul_(2).add_(1)
    lengths = _lengths(g, b, n, kind)
    state, dstate = (_normal(g, b, c), _normal(g, b, c)) if layout != "plain" else (None, None)
    dy = _normal(g, b, n, c, dtype=dtype)
    clean = [t.clone() for t in (gate, value, dy)]
    if lengths is not None:                                 # what does not count may hold anything
        dead = torch.arange(n, device="cuda")[None, :] >= lengths[:, None]
        for t in (gate, value, dy):
            t[dead] = NAN
        for t in clean:
            t[dead] = 0
    dx = _layout(g, b, n, c, dtype, layout)
    for t in dx:
        t.fill_(NAN)
    y, last, first = _run_recurrence(ops, gate, value, state, lengths, dy, dstate, dx)
    ey, by, el, bl, _ = ref.recurrence(clean[0], clean[1], state, lengths)
    ref.check(y, ey, by, "y")
    ref.check(last, el, bl, "state")
    (ez, bz), (ev, bv), (ef, bf) = ref.recurrence_grad(clean[0], clean[1], state, lengths, clean[2], dstate)
    ref.check(dx[0], ez, bz, "dgate")
    ref.check(dx[1], ev, bv, "dvalue")
    ref.check(first, ef, bf, "dstate")
    # the forward call alone, and once more: the same bits
    again, last2 = ops.recurrence(gate, value, state=state, lengths=lengths)
    assert torch.equal(again, y) and torch.equal(last, last2)
    keep = [t.clone() for t in dx]
    _, _, first2 = _run_recurrence(ops, gate, value, state, lengths, dy, dstate, dx)
    assert torch.equal(first, first2) and all(torch.equal(p, q) for p, q in zip(keep, dx))


def test_recurrence_gradient_against_differences(ops):
    """fp32, loss = sum of y * dy + sum of state * dstate: central differences of step s are off by s^2 times a third derivative (here below 10 for every input) and by
    the loss's own rounding over s."""
    g = _gen("diff")
    b, n, c = 2, 40, 3
    gate, value, state = _normal(g, b, n, c), _normal(g, b, n, c), _normal(g, b, c)
    dy, dstate = _normal(g, b, n, c), _normal(g, b, c)
    dx = torch.empty_like(gate), torch.empty_like(value)
    first = _run_recurrence(ops, gate, value, state, None, dy, dstate, dx)[2]

    def loss():
        y, _, last, _, _ = ref.recurrence(gate.double(), value.double(), state, None)
        return float((y * dy.double()).sum() + (last * dstate.double()).sum())

    s = 2.0 ** -10
    for t, grad in ((gate, dx[0]), (value, dx[1]), (state, first)):
        flat, want = t.view(-1), grad.reshape(-1)
        for i in range(0, flat.numel(), 17):
            old = float(flat[i])
            flat[i] = old + s
            hi, up = loss(), float(flat[i])
            flat[i] = old - s
            lo, down = loss(), float(flat[i])
            flat[i] = old
            assert abs((hi - lo) / (up - down) - float(want[i])) <= 10 * s * s + 1e-5, (i, hi, lo, want[i])


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
def test_recurrence_of_closed_and_open_gates(ops, dtype):
    """Gates of +infinity and far out keep the state to the last bit; -infinity and far below take the value."""
    g = _gen("gates")
    b, n, c = 2, 300, 24
    gate = torch.full((b, n, c), float("inf"), device="cuda", dtype=dtype)
    gate[:, :, 1::4] = 1e4
    gate[:, :, 2::4] = float("-inf")
    gate[:, :, 3::4] = -1e4
    value, state = _normal(g, b, n, c, dtype=dtype), _normal(g, b, c)
    y, last = ops.recurrence(gate, value, state=state)
    assert torch.equal(last[:, 0::4], state[:, 0::4]) and torch.equal(last[:, 1::4], state[:, 1::4])
    assert torch.equal(y[:, :, 2::4], value[:, :, 2::4]) and torch.equal(y[:, :, 3::4], value[:, :, 3::4])


@pytest.mark.parametrize("bad", [NAN, float("inf")], ids=str)
@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("b,n,c", [(2, 700, 40), (1, 5000, 16), (3, 1100, 300)])
def test_recurrence_keeps_what_is_not_finite_in_its_channel_and_direction(ops, b, n, c, dtype, bad):
    """A value that is not finite reaches the steps behind it, a dy the steps in front of it; all others keep their bits."""
    g = _gen("bad", b, n, c)
    gate, value, dy = (_normal(g, b, n, c, dtype=dtype) for _ in range(3))

    def passes(value, dy):
        y, last, saved = ops.recurrence(gate, value, for_grad=True)
        dgate, dvalue = torch.empty_like(gate), torch.empty_like(gate)
        first = ops.recurrence_grad(gate, value, dy, saved, dgate=dgate, dvalue=dvalue)
        return y, last, dgate, dvalue, first
    clean = passes(value, dy)
    s, t, k = b - 1, n // 3, c // 2
    spoilt = value.clone()
    spoilt[s, t, k] = bad
    y, last, dgate, dvalue, first = passes(spoilt, dy)
    assert not y[s, t:, k].isfinite().any() and not last[s, k].isfinite() and not dgate[s, t:, k].isfinite().any()
    for got, want in zip((y, last, dgate, dvalue, first), clean):
        if got.dim() == 3 and got is not dvalue:
            got[s, t:, k] = want[s, t:, k]
        elif got is last:
            got[s, k] = want[s, k]
        assert torch.equal(got, want)
    spoilt = dy.clone()
    spoilt[s, t, k] = bad
    y, last, dgate, dvalue, first = passes(value, spoilt)
    assert not dvalue[s, :t + 1, k].isfinite().any() and not first[s, k].isfinite()
    for got, want in zip((y, last, dgate, dvalue, first), clean):
        if got is dgate or got is dvalue:
            got[s, :t + 1, k] = want[s, :t + 1, k]
        elif got is first:
            got[s, k] = want[s, k]
        assert torch.equal(got, want)


def test_recurrence_step_by_step_continues_a_sequence(ops):
    """Single steps from the carried state, the state updated in place."""
    g = _gen("steps")
    b, n, c = 5, 50, 96
    gate, value = _normal(g, b, n, c, dtype=torch.bfloat16), _normal(g, b, n, c, dtype=torch.bfloat16)
    exact, bound, last, lbound, _ = ref.recurrence(gate, value, None, None)
    state = torch.zeros(b, c, device="cuda")
    for t in range(n):
        y, state = ops.recurrence(gate[:, t:t + 1], value[:, t:t + 1], state=state)
        ref.check(y[:, 0], exact[:, t], bound[:, t], f"step {t}")
    ref.check(state, last, lbound, "state")


def test_recurrence_of_no_steps(ops):
    state = torch.randn(3, 5, device="cuda")
    none = torch.empty(3, 0, 5, device="cuda")
    y, last, saved = ops.recurrence(none, none, state=state, for_grad=True)
    assert y.shape == (3, 0, 5) and torch.equal(last, state)
    assert torch.equal(ops.recurrence_grad(none, none, none, saved, dgate=none, dvalue=none, dstate=state), state)
    assert (ops.recurrence(none, none)[1] == 0).all()
    empty = torch.empty(0, 4, 5, device="cuda")
    assert ops.recurrence(empty, empty)[0].shape == (0, 4, 5)


def test_recurrence_beyond_32_bit_offsets(ops):
    """The last sequence starts behind 2^32 bytes and behind 2^31 elements of the batch."""
    b, n, c = 3, 40, 64
    stride = (1 << 30) + 8
    flat = torch.zeros(2 * stride + n * c, dtype=torch.bfloat16, device="cuda")
    g = _gen("far")
    value = flat.as_strided((b, n, c), (stride, c, 1))
    value.copy_(_normal(g, b, n, c))
    gate = _normal(g, b, n, c, dtype=torch.bfloat16)
    y, last = ops.recurrence(gate, value)
    ey, by, el, bl, _ = ref.recurrence(gate, value, None, None)
    ref.check(y, ey, by, "y")
    out = flat.as_strided((b, n, c), (stride, c, 1))
    kept = value.clone()
    saved = ops.recurrence(gate, kept, for_grad=True, out=out)[2]
    assert torch.equal(out, y) and saved.numel() > 0


# ---- distillation

DISTILL = [(900, 800, 17), (1800, 2000, 9), (1, 1, 1), (3, 2, 2), (4, 10, 4), (130, 10, 4), (7, 33, 1), (6, 1000, 20), (5, 1025, 300), (3, 4099, 64), (9, 32000, 64), (2, 50257, 8), (3, 100003, 1000), (2, 262144, 5)]


def _teacher(g, m, v, k, kind):
    ids = torch.stack([torch.randperm(max(v, k), generator=g, device="cuda")[:k] % v for _ in range(m)]).int()
    t = _normal(g, m, k) * 2
    if kind == "twice":
        ids[:, k // 2:] = ids[:, :k - k // 2].clone()
        ids[0] = int(ids[0, 0])
    if kind == "short":                # lists of different lengths, some empty; entries of no weight
        cut = torch.randint(0, k + 1, (m,), generator=g, device="cuda")
        ids[torch.arange(k, device="cuda")[None, :] >= cut[:, None]] = -1
        ids[0] = v
        t[:, k // 3] = float("-inf")
        t[ids < 0] = NAN
    return ids, t


@pytest.mark.parametrize("types", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.bfloat16)], ids=str)
@pytest.mark.parametrize("kind,tau,weight", [("plain", 1.0, 1.0), ("plain", 2.0, 0.6), ("twice", 1.5, 0.5), ("short", 4.0, 0.9), ("plain", 1.0, 0.3), ("plain", 3.0, 0.0)])
@pytest.mark.parametrize("m,v,k", DISTILL)
def test_distillation(ops, m, v, k, kind, tau, weight, types):
    g = _gen("distill", m, v, k, kind, tau)
    logits = _normal(g, m, v, dtype=types[0]) * 3
    ids, teacher = _teacher(g, m, v, k, kind)
    labels = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
    labels[m // 2] = -100
    labels[m // 3] = v
    scale = 1.0 / m
    out = torch.full((m, v), NAN, dtype=types[1], device="cuda")
    loss, grad = ops.distill_loss(logits, labels, ids, teacher, temperature=tau, weight=weight, scale=scale, out=out)
    (el, bl), (eg, bg) = ref.distill(logits, labels, ids, teacher, _f32(tau), _f32(weight), _f32(scale), types[1])
    ref.check(loss, el, bl, "loss")
    ref.check(grad, eg, bg, "gradient")
    # the loss alone; rows apart on an odd address; in place
    only, none = ops.distill_loss(logits, labels, ids, teacher, temperature=tau, weight=weight, grad=False)
    assert none is None and torch.equal(only, loss)
    wide = torch.full((m * (v + 3) + 1,), NAN, dtype=types[0], device="cuda")
    apart = wide[1:].view(m, v + 3)[:, :v]
    apart.copy_(logits)
    loss2, _ = ops.distill_loss(apart, labels, ids, teacher, temperature=tau, weight=weight, scale=scale, out=out.fill_(NAN))
    ref.check(loss2, el, bl, "loss, rows apart")
    ref.check(out, eg, bg, "gradient, rows apart")
    if types[0] == types[1]:
        ops.distill_loss(apart, labels, ids, teacher, temperature=tau, weight=weight, scale=scale, out=apart)
        assert torch.equal(apart, out)
        assert wide[1:].view(m, v + 3)[:, v:].isnan().all()


def test_distillation_without_labels(ops):
    g = _gen("nolabels")
    logits = _normal(g, 5, 77)
    ids, teacher = _teacher(g, 5, 77, 9, "plain")
    loss, grad = ops.distill_loss(logits, None, ids, teacher, temperature=2.0)
    (el, bl), (eg, bg) = ref.distill(logits, None, ids, teacher, 2.0, 1.0, 1.0, torch.float32)
    ref.check(loss, el, bl, "loss")
    ref.check(grad, eg, bg, "gradient")


@pytest.mark.parametrize("dtype", DTYPES, ids=str)
@pytest.mark.parametrize("v", [40, 5000, 70000])
def test_distillation_of_masked_logits(ops, v, dtype):
    """Logits of -infinity (no gradient there), of the type's lowest and largest values, a row of nothing but the lowest, a NaN that stays in its row."""
    g = _gen("masked", v)
    logits = _normal(g, 6, v, dtype=dtype)
    ids, teacher = _teacher(g, 6, v, 7, "plain")
    labels = torch.zeros(6, dtype=torch.int32, device="cuda")
    allowed = torch.zeros(6, v, dtype=torch.bool, device="cuda").scatter_(1, ids.long(), True)
    allowed[:, 0] = True
    logits[0] = torch.where(allowed[0], logits[0], float("-inf"))
    logits[1] = torch.where(allowed[1], logits[1], torch.finfo(dtype).min)
    logits[2] = torch.finfo(dtype).min
    logits[3, v // 2] = NAN
    logits[4] *= 30
    loss, grad = ops.distill_loss(logits, labels, ids, teacher, temperature=0.5, weight=0.5)
    (el, bl), (eg, bg) = ref.distill(logits, labels, ids, teacher, 0.5, 0.5, 1.0, dtype)
    assert loss[3].isnan() and grad[3].isnan().all()
    keep = torch.tensor([0, 1, 2, 4, 5], device="cuda")
    ref.check(loss[keep], el[keep], bl[keep], "loss")
    ref.check(grad[keep], eg[keep], bg[keep], "gradient")
    assert (grad[0][~allowed[0]] == 0).all()


def test_distillation_of_nothing(ops):
    none = torch.empty(0, 8, device="cuda")
    loss, grad = ops.distill_loss(none, None, none.int()[:, :3].contiguous(), none[:, :3].contiguous())
    assert loss.shape == (0,) and grad.shape == (0, 8)
    x = torch.randn(3, 8, device="cuda")
    empty = torch.empty(3, 0, device="cuda")
    loss, grad = ops.distill_loss(x, None, empty.int(), empty)          # a teacher without entries has nothing to say
    assert (loss == 0).all() and (grad == 0).all()


def test_distillation_gradient_against_differences(ops):
    """fp32 gradient against central differences of the 64-bit loss: step s, third derivatives below 10."""
    g = _gen("ddiff")
    m, v, k = 3, 21, 5
    logits = _normal(g, m, v)
    ids, teacher = _teacher(g, m, v, k, "twice")
    labels = torch.tensor([3, -1, 20], dtype=torch.int32, device="cuda")
    _, grad = ops.distill_loss(logits, labels, ids, teacher, temperature=1.5, weight=0.5)
    s = 2.0 ** -10
    x = logits.double()

    def loss(x):
        return float(ref.distill(x, labels, ids, teacher, 1.5, 0.5, 1.0, torch.float32)[0][0].sum())

    for i in range(0, m * v, 2):
        d = torch.zeros(m * v, dtype=ref.F64, device="cuda")
        d[i] = s
        diff = (loss(x + d.view(m, v)) - loss(x - d.view(m, v))) / (2 * s)
        assert abs(diff - float(grad.view(-1)[i])) <= 10 * s * s + 1e-6


# ---- how they are called

def _all_calls(ops, seed, n=3000, vocab=500, c=64):
    """A run of the operators as a training step uses them: tokens -> embedding -> projection -> recurrence -> logits -> loss and back.  Returns a function that
    runs it into its own outputs, and the outputs."""
    g = _gen("run", seed)
    b, t = 6, n // 6
    tok = _tokens(g, n, vocab, "skewed").view(b, t)
    table = _normal(g, vocab, c, dtype=torch.bfloat16)
    w = _normal(g, c, 2 * c, dtype=torch.bfloat16) / 8
    head = _normal(g, c, vocab, dtype=torch.bfloat16) / 8
    ids, teacher = _teacher(g, n, vocab, 12, "plain")
    labels = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    out = {}

    def run():
        e = ops.embedding(tok, table, scale=2.0)
        x = e @ w
        y, last, saved = ops.recurrence(x[..., :c], x[..., c:], for_grad=True)
        logits = (y.view(n, c) @ head).contiguous()
        loss, dl = ops.distill_loss(logits, labels, ids, teacher, temperature=2.0, weight=0.5, scale=1.0 / n)
        dy = (dl @ head.t()).view(b, t, c)
        dx = torch.empty_like(x)
        ops.recurrence_grad(x[..., :c], x[..., c:], dy, saved, dgate=dx[..., :c], dvalue=dx[..., c:])
        dt = ops.embedding_grad(tok, dx @ w.t(), vocab, scale=2.0)
        for k, v in dict(y=y, last=last, loss=loss, dl=dl, dx=dx, dt=dt).items():
            out[k] = v
    return run, out


def test_calls_on_another_stream_and_two_at_once(ops):
    pairs = [_all_calls(ops, i) for i in range(2)]
    want = []
    for run, out in pairs:
        run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in out.items()})
    streams = [torch.cuda.Stream() for _ in pairs]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for s, (run, _) in zip(streams, pairs):
            with torch.cuda.stream(s):
                run()
    torch.cuda.synchronize()
    for (_, out), w in zip(pairs, want):
        assert all(torch.equal(out[k], w[k]) for k in w)


def test_calls_in_graphs_that_share_a_pool(ops):
    """Two captured runs, replayed in turn on new inputs' places: what each leaves is what the calls leave."""
    pairs = [_all_calls(ops, i) for i in range(2)]
    want = []
    for run, out in pairs:
        run()
        torch.cuda.synchronize()
        want.append({k: v.clone() for k, v in out.items()})
    graphs, outs = [], []
    pool = torch.cuda.graph_pool_handle()
    for run, out in pairs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, pool=pool):
            run()
        graphs.append(graph)
        outs.append(dict(out))
    for _ in range(3):
        for graph, out, w in zip(graphs, outs, want):
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(out[k], w[k]) for k in w)


def test_first_calls_inside_a_capture(ops):
    """What a kernel is set up with is set up inside the capture too: rows over a cluster, a sequence over a cluster, many tokens; none of these sizes is used elsewhere."""
    g = _gen("capture")
    logits = _normal(g, 5, 70001)
    ids, teacher = _teacher(g, 5, 70001, 33, "plain")
    gate, value = _normal(g, 1, 7000, 40, dtype=torch.bfloat16), _normal(g, 1, 7000, 40, dtype=torch.bfloat16)
    tok, dy = _tokens(g, 5000, 900, "skewed"), _normal(g, 5000, 20, dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = [*ops.distill_loss(logits, None, ids, teacher, temperature=1.5), *ops.recurrence(gate, value), ops.embedding_grad(tok, dy, 900)]
    for t in got:
        t.fill_(NAN)
    for _ in range(2):
        graph.replay()
    want = [*ops.distill_loss(logits, None, ids, teacher, temperature=1.5), *ops.recurrence(gate, value), ops.embedding_grad(tok, dy, 900)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    (el, bl), (eg, bg) = ref.distill(logits, None, ids, teacher, 1.5, 1.0, 1.0, torch.float32)
    ref.check(want[0], el, bl, "loss")
    ref.check(want[1], eg, bg, "gradient")


def test_recurrence_of_broadcast_inputs(ops):
    """One gate for all sequences, for all steps, and one value for both: strides of zero."""
    g = _gen("broadcast")
    b, n, c = 4, 300, 64
    for dtype in DTYPES:
        value, dy = _normal(g, b, n, c, dtype=dtype), _normal(g, b, n, c, dtype=dtype)
        for gate in (_normal(g, 1, n, c, dtype=dtype).expand(b, n, c), _normal(g, b, 1, c, dtype=dtype).expand(b, n, c), _normal(g, 1, 1, c, dtype=dtype).expand(b, n, c)):
            dx = torch.empty_like(value), torch.empty_like(value)
            got = _run_recurrence(ops, gate, value, None, None, dy, None, dx)
            dense = gate.contiguous()
            dw = torch.empty_like(value), torch.empty_like(value)
            want = _run_recurrence(ops, dense, value, None, None, dy, None, dw)
            assert all(torch.equal(p, q) for p, q in zip((*got, *dx), (*want, *dw)))
            ref.check(got[0], *ref.recurrence(dense, value, None, None)[:2], "y")


@pytest.mark.parametrize("b,n,c", [(3, 70, 64), (1, 6000, 72), (2, 1, 40)])
def test_recurrence_bits_do_not_depend_on_alignment(ops, b, n, c):
    """Tensor copies, 4-byte copies and single loads see the same tiles."""
    g = _gen("aligned", b, n, c)
    for dtype in DTYPES:
        data = [_normal(g, b, n, c, dtype=dtype) for _ in range(3)]
        runs = []
        for off in (0, 2, 1):
            gate, value, dy = (torch.empty(b * n * c + 8, dtype=dtype, device="cuda")[off:off + b * n * c].view(b, n, c).copy_(t) for t in data)
            dx = torch.empty_like(gate), torch.empty_like(gate)
            runs.append((*_run_recurrence(ops, gate, value, None, None, dy, None, dx), *dx))
        for other in runs[1:]:
            assert all(torch.equal(p, q) for p, q in zip(runs[0], other))


@pytest.mark.parametrize("n", [1, 50, 9000])
def test_recurrence_updates_a_state_in_place(ops, n):
    import ctypes
    from paper_2509_05679_b200 import binding
    g = _gen("place", n)
    b, c = 2, 48
    gate, value, state = _normal(g, b, n, c), _normal(g, b, n, c), _normal(g, b, c)
    y, last = ops.recurrence(gate, value, state=state)
    s = binding.fdg_recurrence(0, b, n, c, n * c, c, n * c, c, n * c, c)
    out = torch.empty_like(y)
    assert binding.lib().fdg_recurrence_forward(ctypes.byref(s), gate.data_ptr(), value.data_ptr(), None, state.data_ptr(), out.data_ptr(), state.data_ptr(), None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(out, y) and torch.equal(state, last)


@pytest.mark.parametrize("v", [40, 3000])
def test_distillation_of_a_teacher_of_nan(ops, v):
    """A NaN among a row's entries is the row's; where it is all there is too."""
    g = _gen("nan", v)
    logits = _normal(g, 4, v)
    ids, teacher = _teacher(g, 4, v, 6, "plain")
    teacher[1, 2] = NAN
    teacher[2] = NAN
    loss, grad = ops.distill_loss(logits, None, ids, teacher, temperature=2.0)
    assert torch.equal(loss.isnan(), torch.tensor([False, True, True, False], device="cuda"))
    (el, bl), (eg, bg) = ref.distill(logits, None, ids, teacher, 2.0, 1.0, 1.0, torch.float32)
    ref.check(loss, el, bl, "loss")
    ref.check(grad[[0, 3]], eg[[0, 3]], bg[[0, 3]], "gradient")


def test_embedding_beyond_32_bit_offsets(ops):
    """A table of more than 2^31 elements and a gradient of more than 2^32 bytes: the last rows."""
    v, c = (1 << 21) + 5, 1032
    g = _gen("large")
    table = torch.zeros(v, c, dtype=torch.bfloat16, device="cuda")
    table[-8:] = _normal(g, 8, c)
    for n in (100, 3000):
        tok = torch.randint(v - 8, v, (n,), generator=g, device="cuda", dtype=torch.int32)
        y = ops.embedding(tok, table, scale=2.0)
        assert torch.equal(y, table[tok.long()] * 2)
        dw = ops.embedding_grad(tok, y, v)
        exact, bound = ref.embedding_grad(tok - (v - 8), y, 8, 1.0)
        ref.check(dw[-8:], exact, bound, "dtable")
        assert not dw[:-8].any()
        del dw


def test_distillation_beyond_32_bit_offsets(ops):
    m, v = 17000, 131073
    g = _gen("long")
    logits = torch.zeros(m, v, dtype=torch.bfloat16, device="cuda")
    logits[-3:] = _normal(g, 3, v)
    ids = torch.arange(4, device="cuda", dtype=torch.int32).expand(m, 4).contiguous()
    teacher = _normal(g, m, 4)
    loss, grad = ops.distill_loss(logits, None, ids, teacher, out=logits)
    check = torch.zeros(3, v, dtype=torch.bfloat16, device="cuda")
    g = _gen("long")
    check[:] = _normal(g, 3, v)
    (el, bl), (eg, bg) = ref.distill(check, None, ids[-3:], teacher[-3:], 1.0, 1.0, 1.0, torch.bfloat16)
    ref.check(loss[-3:], el, bl, "loss")
    ref.check(grad[-3:], eg, bg, "gradient")


def test_refusals_of_tensors(ops):
    """What the host can see to be wrong is refused, and nothing is written."""
    from paper_2509_05679_b200.binding import FdgError
    f = lambda *s, dtype=torch.float32, device="cuda": torch.zeros(*s, dtype=dtype, device=device)
    i = lambda *s: f(*s, dtype=torch.int32)
    bad = [
        lambda: ops.embedding(i(4), f(4, 4, device="cpu")),
        lambda: ops.embedding(f(4), f(4, 4)),
        lambda: ops.embedding(i(4).long(), f(4, 4)),
        lambda: ops.embedding(i(8)[::2], f(4, 4)),
        lambda: ops.embedding(i(4), f(4, 4, dtype=torch.float16)),
        lambda: ops.embedding(i(4), f(4, 8)[:, ::2]),
        lambda: ops.embedding(i(4), f(4, 4), out=f(4, 5)),
        lambda: ops.embedding(i(4), f(4, 4), out=f(4, 4, dtype=torch.bfloat16)),
        lambda: ops.embedding(i(4), f(4, 4), out=f(1, 4).expand(4, 4)),
        lambda: ops.embedding_grad(i(4), f(5, 4), 4),
        lambda: ops.embedding_grad(i(4), f(4, 4), 4, accumulate=True),
        lambda: ops.embedding_grad(i(4), f(4, 4), 4, out=f(4, 4, dtype=torch.bfloat16)),
        lambda: ops.embedding_grad(i(4), f(4, 4), 0),
        lambda: ops.embedding_grad(i(4), f(4, 4, device="cpu"), 4),
        lambda: ops.recurrence(f(2, 3, 4), f(2, 3, 5)),
        lambda: ops.recurrence(f(2, 3, 4), f(2, 3, 4, dtype=torch.bfloat16)),
        lambda: ops.recurrence(f(2, 3, 4), f(2, 3, 4), state=f(2, 5)),
        lambda: ops.recurrence(f(2, 3, 4), f(2, 3, 4), lengths=i(3)),
        lambda: ops.recurrence(f(2, 3, 4), f(2, 3, 4), out=f(1, 3, 4).expand(2, 3, 4)),
        lambda: ops.recurrence(f(2, 3, 8)[..., ::2], f(2, 3, 4)),
        lambda: ops.recurrence_grad(f(2, 3, 4), f(2, 3, 4), f(2, 3, 4), f(7, dtype=torch.uint8), dgate=f(2, 3, 4), dvalue=f(2, 3, 4)),
        lambda: ops.distill_loss(f(3, 8), None, i(3, 2), f(3, 2), weight=0.5),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 2), f(3, 3)),
        lambda: ops.distill_loss(f(3, 8), i(4), i(3, 2), f(3, 2)),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 2), f(3, 2), temperature=0.0),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 2), f(3, 2), temperature=NAN),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 2), f(3, 2), weight=1.5),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 1025), f(3, 1025)),
        lambda: ops.distill_loss(f(1, 262145), i(1), i(1, 2), f(1, 2)),
        lambda: ops.distill_loss(f(3, 8, dtype=torch.bfloat16), i(3), i(3, 2), f(3, 2), out=f(3, 8)),
        lambda: ops.distill_loss(f(3, 8), i(3), i(3, 2), f(3, 2), out=f(1, 8).expand(3, 8)),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(FdgError):
            call()
            pytest.fail(f"call {n} went through")
    torch.cuda.synchronize()


def test_refusals_of_addresses(ops):
    """Host memory, addresses off their elements' boundary and short workspaces, straight through the C interface."""
    import ctypes
    from paper_2509_05679_b200 import binding
    L = binding.lib()
    host, dev, tok = torch.zeros(64), torch.zeros(64, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    a = lambda t, off=0: t.data_ptr() + off
    assert L.fdg_embedding_forward(a(tok), 8, a(host), 0, 4, 4, 1.0, a(dev), 4, None) == 1
    assert b"current device" in L.fdg_op_last_error()
    assert L.fdg_embedding_forward(a(tok), 8, a(dev, 2), 0, 4, 4, 1.0, a(dev), 4, None) == 1
    assert b"aligned" in L.fdg_op_last_error()
    assert L.fdg_embedding_forward(a(tok), 8, a(dev), 2, 4, 4, 1.0, a(dev), 4, None) == 1
    assert L.fdg_embedding_forward(a(tok), 8, a(dev), 0, 4, 4, 1.0, a(dev), 3, None) == 1
    assert L.fdg_embedding_forward(a(tok), -1, a(dev), 0, 4, 4, 1.0, a(dev), 4, None) == 1
    need = ctypes.c_size_t()
    assert L.fdg_embedding_workspace(100000, 50000, 64, ctypes.byref(need)) == 0
    if need.value:
        big = torch.zeros(need.value, dtype=torch.uint8, device="cuda")
        assert L.fdg_embedding_backward(a(tok), 100000, a(dev), 0, 64, 50000, 64, 1.0, 0, a(dev), a(big), need.value - 1, None) == 1
        assert b"workspace" in L.fdg_op_last_error()
        assert L.fdg_embedding_backward(a(tok), 100000, a(dev), 0, 64, 50000, 64, 1.0, 0, a(dev), a(big, 16), need.value, None) == 1
    s = binding.fdg_recurrence(0, 1, 2, 4, 8, 4, 8, 4, 8, 3)           # rows of y overlap
    assert L.fdg_recurrence_forward(ctypes.byref(s), a(dev), a(dev, 64), None, None, a(dev, 128), None, None, None) == 1
    assert b"overlap" in L.fdg_op_last_error()
    s.y_step = 4
    assert L.fdg_recurrence_forward(ctypes.byref(s), a(dev), a(host), None, None, a(dev, 128), None, None, None) == 1
    torch.cuda.synchronize()

"""Operators on token sequences where a call goes to an edge: rows without a term, many rounds of a recurrence's tiles, gates far below zero, sums that have to be exact,
inputs that autograd follows."""
import pytest
import torch

import operators_reference as ref

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def ops():
    from paper_2509_05679_b200 import operators
    return operators


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


# ---- distillation

@pytest.mark.parametrize("types", [(F32, F32), (BF16, BF16), (F32, BF16)], ids=str)
@pytest.mark.parametrize("v", [40, 5000, 70000])
@pytest.mark.parametrize("how", ["ids", "weights", "top"])
def test_a_row_without_an_entry_has_no_gradient_whatever_its_logits(ops, how, v, types):
    """Weight 1: a padding row that the teacher says nothing about adds no loss and no gradient, NaN and infinities in its logits or not; the rows beside it keep theirs."""
    g = _gen(v)
    m, k = 7, 5
    logits = _normal(g, m, v, dtype=types[0])
    ids = torch.stack([torch.randperm(v, generator=g, device="cuda")[:k] for _ in range(m)]).int()
    teacher = _normal(g, m, k)
    silent = torch.tensor([1, 2, 4, 5], device="cuda")
    logits[1], logits[2, v // 2], logits[4], logits[5, 0] = NAN, INF, -INF, NAN
    if how == "ids":
        ids[silent] = -1
    elif how == "weights":
        teacher[silent] = -INF
    else:
        ids, teacher = ids[:, :0].contiguous(), teacher[:, :0].contiguous()
        silent = torch.arange(m, device="cuda")
    heard = torch.tensor([i for i in range(m) if i not in silent.tolist()], device="cuda", dtype=torch.long)
    out = torch.full((m, v), NAN, dtype=types[1], device="cuda")
    loss, _ = ops.distill_loss(logits, None, ids, teacher, temperature=2.0, scale=0.5, out=out)
    assert (loss[silent] == 0).all() and (out[silent] == 0).all()
    if len(heard):
        (el, bl), (eg, bg) = ref.distill(logits[heard], None, ids[heard], teacher[heard], 2.0, 1.0, 0.5, types[1])
        ref.check(loss[heard], el, bl, "loss")
        ref.check(out[heard], eg, bg, "gradient")
    if types[0] == types[1]:
        ops.distill_loss(logits, None, ids, teacher, temperature=2.0, scale=0.5, out=logits)
        assert torch.equal(logits, out)


# ---- recurrence: gates far below zero

@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("steps", [1, 9])
def test_gates_far_below_zero(ops, steps, dtype):
    """sigmoid is held to its own size down to the least normal number, 2^-126 at gate -87.3, and stays there below: what a state and a gradient keep of it is a product with it.
    One sequence a gate, values of zero, so that a state is the product of its gates' sigmoids and nothing else (only the first step's gate is far below zero: a second one would
    underflow); dgate of that step is a (1 - a) dy (h_0 - 0)."""
    gates = torch.cat([-torch.arange(60.0, 90.0, 0.25, device="cuda"), torch.tensor([-87.33, -87.34, -88.0, -100.0, -1000.0, -1e30, -INF], device="cuda")]).to(dtype)
    b, c = len(gates), 24
    gate = torch.zeros(b, steps, c, device="cuda", dtype=dtype)
    gate[:, 0] = gates[:, None]
    value = torch.zeros_like(gate)
    g = _gen(5)
    state, dstate = 1 + torch.rand(b, c, generator=g, device="cuda"), 1 + torch.rand(b, c, generator=g, device="cuda")
    y, last, saved = ops.recurrence(gate, value, state=state, for_grad=True)
    dgate, dvalue = torch.empty_like(gate), torch.empty_like(gate)
    first = ops.recurrence_grad(gate, value, torch.zeros_like(gate), saved, dgate=dgate, dvalue=dvalue, dstate=dstate)
    z = gates.double()
    a = torch.sigmoid(z).clamp(min=2.0 ** -126)[:, None]
    q = torch.sigmoid(-z)[:, None]
    behind = 0.5 ** (steps - 1)                                # sigmoid(0) of the steps behind: exact, but for results below the least normal number
    # the gate: (8 + |z|) U (operators_reference); products: 2 U a step; 2^-149 for what falls below the least normal number
    rel = (8 + z.abs().clamp(max=87.4) + 2 * (steps + 3))[:, None] * ref.U
    def near(got, want, what):
        ref.check(got, want, ref.store(want, rel * want.abs() + 2.0 ** -149 * (steps + 3), got.dtype), what)
    near(last, a * behind * state.double(), "state")
    near(y[:, 0], a * state.double(), "y")
    near(first, a * behind * dstate.double(), "gradient of the first state")
    near(dgate[:, 0], a * q * behind * dstate.double() * state.double(), "dgate")
    near(dvalue[:, 0], q * behind * dstate.double(), "dvalue")


# ---- inputs that autograd follows

def test_tensors_that_autograd_follows_are_refused(ops):
    """A result without a history would lose the gradient without a word; where nothing is recorded (no_grad, a detached tensor) the call goes through."""
    from paper_2509_05679_b200.binding import FdgError
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    x = lambda *s: torch.zeros(*s, device="cuda")
    p = lambda *s: torch.zeros(*s, device="cuda", requires_grad=True)
    saved = ops.recurrence(x(2, 3, 4), x(2, 3, 4), for_grad=True)[2]
    ids = torch.zeros(2, 1, dtype=torch.int32, device="cuda")
    calls = [
        lambda f: ops.embedding(tok, f(5, 4)),
        lambda f: ops.embedding(tok, x(5, 4), out=f(4, 4)),
        lambda f: ops.embedding_grad(tok, f(4, 4), 5),
        lambda f: ops.embedding_grad(tok, x(4, 4), 5, out=f(5, 4)),
        lambda f: ops.recurrence(f(2, 3, 4), x(2, 3, 4)),
        lambda f: ops.recurrence(x(2, 3, 4), f(2, 3, 8)[..., 4:]),
        lambda f: ops.recurrence(x(2, 3, 4), x(2, 3, 4), state=f(2, 4)),
        lambda f: ops.recurrence_grad(x(2, 3, 4), x(2, 3, 4), f(2, 3, 4), saved, dgate=x(2, 3, 4), dvalue=x(2, 3, 4)),
        lambda f: ops.recurrence_grad(x(2, 3, 4), x(2, 3, 4), x(2, 3, 4), saved, dgate=x(2, 3, 4), dvalue=x(2, 3, 4), dstate=f(2, 4)),
        lambda f: ops.distill_loss(f(2, 9), None, ids, x(2, 1)),
        lambda f: ops.distill_loss(x(2, 9), None, ids, f(2, 1)),
    ]
    for n, call in enumerate(calls):
        with pytest.raises(FdgError, match="no_grad"):
            call(p)
            pytest.fail(f"call {n} went through")
        with torch.no_grad():
            call(p)
        call(lambda *s: p(*s).detach())


# ---- embedding gradient: sums that have to be exact

@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("kind", ["uniform", "padded", "one", "skewed", "two"])
@pytest.mark.parametrize("n,vocab,c", [(512, 40, 24), (513, 1, 5), (9000, 1000, 64), (20000, 3, 1032), (40000, 33000, 16), (70000, 300000, 8), (131072, 5, 256), (150001, 17, 40),
                                       (300007, 32000, 3), (1000003, 700, 2)])
def test_embedding_gradient_of_whole_numbers(ops, n, vocab, c, kind, dtype):
    """Whole numbers up to 8: a sum of a million of them is exact in 32 bits in any order, so a row left out, taken twice or added to a wrong token shows, however many there are."""
    g = _gen(n + c)
    tok = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    if kind == "padded":
        tok[torch.rand(n, generator=g, device="cuda") < 0.4] = -1
        tok[n // 2] = vocab
    elif kind == "one":
        tok[:] = vocab // 2
    elif kind == "two":                                     # runs of one token that end inside a tile, over many tiles
        tok[:] = 0
        tok[n // 3:] = vocab - 1
    elif kind == "skewed":
        tok = ((torch.rand(n, generator=g, device="cuda").clamp(min=1e-6).log2() * -0.5).floor().int()) % vocab
    dy = torch.randint(-8, 9, (n, c), generator=g, device="cuda", dtype=torch.int32)
    keep = (tok >= 0) & (tok < vocab)
    want = torch.zeros(vocab, c, dtype=torch.int64, device="cuda").index_add_(0, tok[keep].long(), dy[keep].long())
    rows = dy.to(dtype)
    rows[~keep] = NAN
    dw = ops.embedding_grad(tok, rows, vocab)
    assert torch.equal(dw, want.float())
    start = torch.randint(-1000, 1000, (vocab, c), generator=g, device="cuda", dtype=torch.int32)
    dw = ops.embedding_grad(tok, rows, vocab, scale=0.5, out=start.float(), accumulate=True)
    assert torch.equal(dw, (start + want.double() * 0.5).float())


# ---- calls that differ from one another in layout, and replays on other data

@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_broadcast_rows_and_odd_addresses(ops, dtype):
    """One gradient row and one row of logits for all (strides of zero), ids and results on the address after the first: as the dense calls."""
    g = _gen(11)
    for n, vocab, c in [(300, 50, 40), (3001, 700, 64), (3001, 700, 33)]:
        tok = torch.randint(-1, vocab, (n + 1,), generator=g, device="cuda", dtype=torch.int32)[1:]
        row = torch.randint(-8, 9, (1, c), generator=g, device="cuda").to(dtype)
        want = torch.zeros(vocab, c, device="cuda", dtype=torch.int64).index_add_(0, tok[tok >= 0].long(), row.long().expand(int((tok >= 0).sum()), c))
        out = torch.full((vocab * c + 1,), NAN, device="cuda")[1:].view(vocab, c)
        assert torch.equal(ops.embedding_grad(tok, row.expand(n, c), vocab, out=out), want.float())
        table = _normal(g, vocab, c, dtype=dtype)
        assert torch.equal(ops.embedding(tok, table), torch.where((tok >= 0)[:, None], table[tok.clamp(min=0).long()], 0.0))
    for v in (70, 6001, 70001):
        m, k = 5, 6
        row, teacher = _normal(g, 1, v, dtype=dtype), _normal(g, m, k)
        ids = torch.randint(0, v, (m, k), generator=g, device="cuda", dtype=torch.int32)
        labels = torch.randint(0, v, (m,), generator=g, device="cuda", dtype=torch.int32)
        a = ops.distill_loss(row.expand(m, v), labels, ids, teacher, temperature=1.5, weight=0.5)
        b = ops.distill_loss(row.expand(m, v).contiguous(), labels, ids, teacher, temperature=1.5, weight=0.5)
        (el, bl), (eg, bg) = ref.distill(row.expand(m, v), labels, ids, teacher, 1.5, 0.5, 1.0, dtype)
        for loss, grad in (a, b):
            ref.check(loss, el, bl, "loss")
            ref.check(grad, eg, bg, "gradient")


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("b,n,c", [(1, 1, 8), (3, 1, 20), (1, 900, 24), (6, 130, 40), (2, 2500, 17)])
def test_a_recurrence_whose_tensors_lie_differently(ops, b, n, c, dtype):
    """Gates time-major, values inside a wider tensor, dy one row for all steps, results in layouts of their own: as with dense tensors, bit by bit."""
    g = _gen(b + n + c)
    gate, value, row = _normal(g, b, n, c, dtype=dtype), _normal(g, b, n, c, dtype=dtype), _normal(g, b, 1, c, dtype=dtype)
    state, dstate = _normal(g, b, c), _normal(g, b, c)
    tm = lambda t: torch.empty(n, b, c, dtype=dtype, device="cuda").transpose(0, 1).copy_(t)
    wide = lambda t: torch.full((b, n, 3 * c + 2), NAN, dtype=dtype, device="cuda")[..., c + 1:2 * c + 1].copy_(t)
    runs = []
    for ga, va, dy, y, dz, dv in [(gate, value, row.expand(b, n, c).contiguous(), None, torch.empty_like(gate), torch.empty_like(gate)),
                                  (tm(gate), wide(value), row.expand(b, n, c), wide(gate), wide(gate), tm(gate))]:
        y, last, saved = ops.recurrence(ga, va, state=state, for_grad=True, out=y)
        first = ops.recurrence_grad(ga, va, dy, saved, dgate=dz, dvalue=dv, dstate=dstate)
        runs.append((y, last, first, dz, dv))
    assert all(torch.equal(p, q) for p, q in zip(*runs))


def test_a_captured_run_answers_for_the_data_it_is_replayed_on(ops):
    """Captured once; the data of every replay are others: ids with other repetitions, lengths, lists of the teacher, labels."""
    g = _gen(21)
    b, n, c, vocab, k = 3, 700, 40, 300, 5
    tok = torch.zeros(b * n, dtype=torch.int32, device="cuda")
    x, dy, state = torch.zeros(b, n, 2 * c, device="cuda", dtype=BF16), torch.zeros(b, n, c, device="cuda", dtype=BF16), torch.zeros(b, c, device="cuda")
    lengths = torch.full((b,), n, dtype=torch.int32, device="cuda")
    logits, labels = torch.zeros(b * n, vocab, device="cuda"), torch.zeros(b * n, dtype=torch.int32, device="cuda")
    ids, teacher = torch.zeros(b * n, k, dtype=torch.int32, device="cuda"), torch.zeros(b * n, k, device="cuda")
    wide, wids, wteacher = torch.zeros(4, 70000, device="cuda"), torch.zeros(4, k, dtype=torch.int32, device="cuda"), torch.zeros(4, k, device="cuda")

    def run():
        y, last, saved = ops.recurrence(x[..., :c], x[..., c:], state=state, lengths=lengths, for_grad=True)
        dx = torch.empty_like(x)
        first = ops.recurrence_grad(x[..., :c], x[..., c:], dy, saved, dgate=dx[..., :c], dvalue=dx[..., c:], dstate=state, lengths=lengths)
        return [y, last, dx, first, ops.embedding_grad(tok, dy.view(b * n, c), vocab), *ops.distill_loss(logits, labels, ids, teacher, temperature=2.0, weight=0.5),
                *ops.distill_loss(wide, None, wids, wteacher, temperature=2.0)]
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for i in range(4):
        tok.copy_(torch.randint(-1, vocab >> (3 * i) or 1, (b * n,), generator=g, device="cuda"))
        for t in (x, dy, state, logits, teacher, wide, wteacher):
            t.copy_(_normal(g, *t.shape))
        lengths.copy_(torch.randint(0, n + 1, (b,), generator=g, device="cuda"))
        labels.copy_(torch.randint(-1, vocab, (b * n,), generator=g, device="cuda"))
        for t, v in ((ids, vocab), (wids, 70000)):
            t.copy_(torch.randint(-1, v if i % 2 else 3, t.shape, generator=g, device="cuda"))       # (every other time: entries with the same id)
        for t in got:
            t.fill_(NAN)
        graph.replay()
        assert all(torch.equal(p, q) for p, q in zip(got, run()))

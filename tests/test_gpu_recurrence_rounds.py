"""The recurrence far along a sequence: every cut of a launch, both types and directions, with rounds enough that every stage of a ring is filled again and again, against the
definition in 64 bits."""
import pytest
import torch

import operators_reference as ref
import recurrence_reference as long_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    from paper_2509_05679_b200 import operators
    return operators


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("ragged", [False, True], ids=["full", "ragged"])
@pytest.mark.parametrize("b,n,c", long_ref.SHAPES)
def test_many_rounds(ops, b, n, c, ragged, dtype):
    """Gates that keep most of a state, so that what a round hands on is seen through the next one; rows on 16, 4 and single elements' bytes."""
    g = torch.Generator(device="cuda").manual_seed(b * n + c)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")
    gate, value, dy = (normal(b, n, c) * 1.5 + 3).to(dtype), normal(b, n, c).to(dtype), normal(b, n, c).to(dtype)
    state, dstate = normal(b, c), normal(b, c)
    lengths = None
    if ragged:
        lengths = torch.randint(0, n + 1, (b,), generator=g, device="cuda", dtype=torch.int32)
        lengths[0] = n - 1
        if b > 2:
            lengths[1], lengths[2] = 0, n
    want = long_ref.recurrence(gate, value, state, lengths, dy, dstate)
    runs = []
    for off in (0, 2, 1):
        at = [torch.empty(b * n * c + 8, dtype=dtype, device="cuda")[off:off + b * n * c].view(b, n, c).copy_(t) for t in (gate, value, dy)]
        y, last, saved = ops.recurrence(at[0], at[1], state=state, lengths=lengths, for_grad=True)
        dx = torch.full_like(at[0], float("nan")), torch.full_like(at[0], float("nan"))
        first = ops.recurrence_grad(*at, saved, dgate=dx[0], dvalue=dx[1], dstate=dstate, lengths=lengths)
        runs.append(dict(y=y, last=last, dgate=dx[0], dvalue=dx[1], first=first))
        for name, got in runs[-1].items():
            ref.check(got, *want[name], f"{name} at offset {off}")
    for other in runs[1:]:
        assert all(torch.equal(other[name], got) for name, got in runs[0].items())

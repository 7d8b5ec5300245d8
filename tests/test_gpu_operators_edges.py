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

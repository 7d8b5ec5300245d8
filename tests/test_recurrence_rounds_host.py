"""What the long tests of the recurrence rest on: their sizes reach every cut of a launch with many rounds, and their reference is the step by step one."""
import ctypes as C
import math
import random

import pytest
import torch

import operators_reference as ref
import recurrence_reference as long_ref


def test_every_cut_goes_round_its_rings():
    """In either type and direction: a ring has at most 3 stages, so 7 rounds use each a third time, and both parities of its barrier."""
    seen = {}
    for s in long_ref.SHAPES:
        for bf16 in (False, True):
            for back in (False, True):
                seen.setdefault(long_ref.cut(*s), []).append(long_ref.rounds(*s, bf16, back))
    assert set(seen) == long_ref.CUTS
    assert all(min(r) >= 2 * long_ref.STAGES + 1 for r in seen.values()), seen
    # and there are no other cuts
    rng = random.Random(0)
    draw = lambda most: int(math.exp(rng.uniform(0, math.log(most))))
    assert {long_ref.cut(draw(2000), draw(1e6), draw(20000)) for _ in range(20000)} <= long_ref.CUTS


def test_the_cut_is_the_librarys():
    """As far as the library tells: the saved states are one for 256 / cx x 4 steps."""
    from paper_2509_05679_b200 import binding, build
    build.build_lib()
    size = C.c_size_t()
    rng = random.Random(1)
    draw = lambda most: int(math.exp(rng.uniform(0, math.log(most))))
    for b, n, c in long_ref.SHAPES + [(draw(500), draw(1e5), draw(4096)) for _ in range(2000)]:
        s = binding.fdg_recurrence(1, b, n, c, *[0] * 10)
        if binding.lib().fdg_recurrence_saved(C.byref(s), C.byref(size)) == 0:
            tile = 256 // long_ref.cut(b, n, c)[0] * 4
            assert size.value == 4 * b * c * -(-n // tile), (b, n, c)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=str)
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("n", [1, 2, 37, 150])
def test_the_long_reference_is_the_short_one(n, ragged, dtype):
    g = torch.Generator().manual_seed(n)
    b, c = 4, 5
    gate, value, dy = (torch.randn(b, n, c, generator=g).to(dtype) for _ in range(3))
    state, dstate = torch.randn(b, c, generator=g), torch.randn(b, c, generator=g)
    lengths = torch.tensor([0, n, n // 2, n + 3], dtype=torch.int32) if ragged else None
    got = long_ref.recurrence(gate, value, state, lengths, dy, dstate)
    y, ey, last, el, _ = ref.recurrence(gate, value, state, lengths)
    dz, dv, first = ref.recurrence_grad(gate, value, state, lengths, dy, dstate)
    for name, want in dict(y=(y, ey), last=(last, el), dgate=dz, dvalue=dv, first=first).items():
        for a, b_ in zip(got[name], want):
            torch.testing.assert_close(a, b_, rtol=1e-11, atol=1e-15, msg=lambda m: f"{name}: {m}")


@pytest.mark.parametrize("at", [512, 1024])
def test_a_lost_state_is_outside_the_long_tests_bounds(at):
    """A round that starts from nothing instead of from the state in front of it, with the gates of those tests."""
    g = torch.Generator().manual_seed(at)
    b, n, c = 2, 1500, 6
    gate, value, dy = torch.randn(b, n, c, generator=g) * 1.5 + 3, torch.randn(b, n, c, generator=g), torch.randn(b, n, c, generator=g)
    want = long_ref.recurrence(gate, value, None, None, dy)
    lost = torch.cat([long_ref.recurrence(gate[:, :at], value[:, :at], None, None)["y"][0], long_ref.recurrence(gate[:, at:], value[:, at:], None, None)["y"][0]], 1)
    for dtype in (torch.float32, torch.bfloat16):
        y, bound = long_ref.recurrence(gate.to(dtype), value.to(dtype), None, None)["y"]
        ref.check(y.to(dtype), y, bound, "y")
    with pytest.raises(AssertionError):
        ref.check(lost, *want["y"], "y")
    cut = [long_ref.recurrence(t[0], t[1], None, None, t[2])["dvalue"][0] for t in [[x[:, :at] for x in (gate, value, dy)], [x[:, at:] for x in (gate, value, dy)]]]
    with pytest.raises(AssertionError):
        ref.check(torch.cat(cut, 1), *want["dvalue"], "dvalue")

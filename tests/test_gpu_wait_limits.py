"""Waits of the recurrence's kernels that run out: everything that hangs on what was waited for is NaN, in the same round too, a training step reports it, and the device goes on.
The limit is the environment's and is read once, so every case is a process of its own.  A limit of 0 gives up without a look: the copies and messages themselves arrive."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)

OPERATORS = """
import torch
from paper_2509_05679_b200 import operators as ops
LOST = {lost}
# (sequences, steps, channels, several CTAs a sequence): one round and many, with and without clusters
for b, n, c, cluster in [(1, 1000, 64, True), (1, 5000, 72, True), (1, 20000, 16, True), (9, 640, 512, False), (200, 300, 256, False), (40, 33, 2048, False)]:
    for dtype in (torch.float32, torch.bfloat16):
        g = torch.Generator(device="cuda").manual_seed(n)
        gate, value, dy = (torch.randn(b, n, c, generator=g, device="cuda").to(dtype) for _ in range(3))
        state = torch.randn(b, c, generator=g, device="cuda")
        lengths = torch.full((b,), n - 3, dtype=torch.int32, device="cuda")
        y, last, saved = ops.recurrence(gate, value, state=state, lengths=lengths, for_grad=True)
        dgate, dvalue = torch.empty_like(gate), torch.empty_like(gate)
        first = ops.recurrence_grad(gate, value, dy, torch.zeros_like(saved), dgate=dgate, dvalue=dvalue, dstate=state, lengths=lengths)
        torch.cuda.synchronize()
        lost = LOST == "copies" or (LOST == "peers" and cluster)
        for name, t in dict(y=y, dgate=dgate, dvalue=dvalue).items():
            assert (t[:, n - 3:] == 0).all(), (b, n, c, dtype, name, "steps that do not count")
            assert t[:, :n - 3].isnan().all() if lost else t.isfinite().all(), (b, n, c, dtype, name, t[:, :n - 3].isnan().float().mean().item())
        for name, t in dict(last=last, first=first).items():
            assert t.isnan().all() if lost else t.isfinite().all(), (b, n, c, dtype, name)
        if lost:
            assert saved.view(torch.float32).isnan().any()
assert float(torch.ones(1000, device="cuda").sum()) == 1000
print("fine")
"""

STEP = """
import sys
sys.path.insert(0, "tests")
import numpy as np, torch
from paper_2509_05679_b200 import binding, synth as sy
from harness import make_ctx
for dtype in ("fp32", "bf16"):
    layers = [(sy.EMBEDDING, 50, 32, 1, 0), (sy.CONV1X1, 32, 64, 1, 1), (sy.RECURRENCE, 64, 32, 1, 0), (sy.GLOBAL_AVGPOOL, 32, 32, 1, 0), (sy.LINEAR, 32, 10, 1, 1)]
    net = sy.Net("tokens", layers, [], 1, 24, 1, 10, 2, 4, 0.1, dtype)
    ctx = make_ctx(net, sy.init_params(net.layers, 0))
    x, y = binding.to_device(dtype, sy.batch_inputs(net, 0)), torch.from_numpy(sy.batch_labels(net, 0)).cuda()
    for call in (lambda: ctx.step(x, y, want_loss=True), ctx.params):
        try:
            call()
            raise SystemExit("went through")
        except binding.FdgError as e:
            assert e.status == 7, e
    ctx.close()
print("fine")
"""


def _run(script, limit):
    env = {k: v for k, v in os.environ.items() if k != "FDG_WAIT_CYCLES"}
    if limit is not None:
        env["FDG_WAIT_CYCLES"] = limit
    r = subprocess.run([sys.executable, "-c", script], cwd=ROOT, env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip().endswith("fine"), r.stdout[-2000:] + r.stderr[-2000:]


@pytest.mark.parametrize("limit,lost", [(None, ""), ("plenty", ""), ("4000000000,4000000000", ""), ("0,4000000000", "copies"), ("4000000000,0", "peers"), ("0", "copies")])
def test_outputs_behind_a_wait_that_ran_out_are_nan(limit, lost):
    _run(OPERATORS.format(lost=repr(lost)), limit)


def test_a_step_reports_a_wait_that_ran_out():
    _run(STEP, "0")

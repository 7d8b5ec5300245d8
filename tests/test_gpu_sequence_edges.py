"""Networks of token sequences through fdg_step where their layers meet others: ReLU layers behind an embedding and a recurrence, modules that run in worker groups between modules that
do not, replicas whose embedding gradients take the sorted form."""
import numpy as np
import pytest

from paper_2509_05679_b200 import synth as sy
from harness import make_ctx, make_oracle, max_rel_err, run_parity

pytestmark = pytest.mark.gpu

TAIL = [(sy.GLOBAL_AVGPOOL, 16, 16, 1, 0), (sy.LINEAR, 16, 10, 1, 1)]


@pytest.mark.parametrize("splits,stream", [([], 16), ([2], 32), ([4], 6)], ids=str)
def test_relu_behind_an_embedding_and_a_recurrence(orc, splits, stream):
    """As layers of their own, and as a module's last and first; on data that keep fp32 and the oracle on the same side of every kink (so without padding, whose zeros lie on it)."""
    import torch
    from paper_2509_05679_b200 import binding
    layers = [(sy.EMBEDDING, 20, 16, 1, 1), (sy.RELU, 16, 16, 1, 0), (sy.CONV1X1, 16, 32, 1, 1), (sy.RECURRENCE, 32, 16, 1, 0), (sy.RELU, 16, 16, 1, 0)] + TAIL
    net = sy.Net("tokens", layers, splits, 1, 9, 1, 10, 2, 4, 0.1, "fp32")
    p0 = sy.perturb_params(sy.init_params(net.layers, 0), net.layers, 7, 0.1)
    o, ctx = make_oracle(orc, net, p0), make_ctx(net, p0)
    orc.kink_margin(True)
    for t in range(2 * len(splits) + 4):
        x, y = sy.batch_inputs(net, t, stream), sy.batch_labels(net, t, stream)
        x = np.where(x < 0, np.int32(7), x)
        lo, _ = o.step(x, y, net.lr)
        lg = ctx.step(binding.to_device("fp32", x), torch.from_numpy(y).cuda(), want_loss=True)
        assert np.isnan(lg) == np.isnan(lo) and (np.isnan(lo) or abs(lg - lo) <= 1e-5 * lo), t
        assert max_rel_err(ctx.params(), o.params(0), net.layers)[0] <= 1e-5, t
    ctx.close()
    assert orc.kink_margin(True) >= 2e-6


def _middle(dtype, flags=1):
    """recurrences in the first and the last module, convolutions alone in the middle one"""
    layers = [(sy.EMBEDDING, 40, 16, 1, 0), (sy.CONV1X1, 16, 32, 1, flags), (sy.RECURRENCE, 32, 16, 1, 0),
              (sy.CONV1X1, 16, 24, 1, flags), (sy.CONV3X3, 24, 16, 1, 0),
              (sy.CONV1X1, 16, 32, 1, flags), (sy.RECURRENCE, 32, 16, 1, 0)] + TAIL
    return sy.Net("tokens", layers, [3, 5], 2, 12, 1, 10, 4, 3, 0.05, dtype)


@pytest.mark.parametrize("groups", [2, 4])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_a_module_in_worker_groups_between_two_that_run_whole(orc, dtype, groups):
    tol = dict(param_tol=1e-5, loss_tol=1e-5) if dtype == "fp32" else dict(grad_tol=2e-2, loss_tol=1e-2)
    run_parity(orc, _middle(dtype), 10, worker_groups=groups, **tol)


def test_layouts_of_streams_leave_the_same_weights():
    """Modules with a recurrence run over all workers whatever worker_groups says, so every weight of such a network is the same, and with one stream."""
    import torch
    from paper_2509_05679_b200 import binding
    layers = [(sy.EMBEDDING, 50, 64, 1, 1), (sy.CONV1X1, 64, 128, 1, 1), (sy.RECURRENCE, 128, 64, 1, 0), (sy.CONV1X1, 64, 128, 1, 1), (sy.RECURRENCE, 128, 64, 1, 0),
              (sy.GLOBAL_AVGPOOL, 64, 64, 1, 0), (sy.LINEAR, 64, 10, 1, 1)]
    net = sy.Net("tokens", layers, [3], 1, 32, 1, 10, 4, 4, 0.1, "bf16")
    p0 = sy.round_to_bf16(sy.init_params(net.layers, 0))
    out = []
    for kw in (dict(), dict(serial=True), dict(worker_groups=2), dict(worker_groups=4)):
        ctx = make_ctx(net, p0, grid_sms=148, **kw)
        for t in range(12):
            x, y = binding.to_device("bf16", sy.batch_inputs(net, t)), torch.from_numpy(sy.batch_labels(net, t)).cuda()
            ctx.step(x, y)
            ctx.wait_ingest()
        out.append(ctx.params())
        ctx.close()
    assert np.isfinite(out[0]).all() and not np.array_equal(out[0], p0)
    assert all(np.array_equal(out[0], o) for o in out[1:])


def test_replicas_with_many_padded_ids(orc):
    """640 ids a worker and step, some of them padding: the sorted form of the gradient, once per replica in one workspace."""
    import torch
    from paper_2509_05679_b200 import binding
    layers = [(sy.EMBEDDING, 70, 24, 1, 1), (sy.CONV1X1, 24, 32, 1, 1), (sy.RECURRENCE, 32, 16, 1, 0)] + TAIL
    net = sy.Net("tokens", layers, [2], 1, 80, 1, 10, 3, 8, 0.1, "fp32")
    P = np.array([[0.6, 0.3, 0.1], [0.2, 0.7, 0.1], [0.3, 0.1, 0.6]])
    p0 = sy.init_params(net.layers, 0)
    o = orc.Oracle(net.layers, net.splits, 3, 8, (1, 80, 1), 10, P=P)
    ctx = make_ctx(net, p0, mixing=P)
    o.set_params(p0)
    for r in range(1, 3):
        q = (p0 * (1 + 0.1 * r)).astype(np.float32)
        o.set_params(q, r)
        ctx.set_params_worker(r, q)
    for t in range(6):
        x, y = sy.batch_inputs(net, t), sy.batch_labels(net, t)
        assert (x.reshape(3, -1) == -1).any(1).all()
        o.step(x, y, net.lr)
        ctx.step(binding.to_device("fp32", x), torch.from_numpy(y).cuda())
        for r in range(3):
            assert max_rel_err(ctx.params_worker(r), o.params(r), net.layers)[0] <= 1e-5, (t, r)
    ctx.close()


def test_a_callers_streams_profiles_and_a_second_run():
    """A distilling network on the caller's streams, under the profiler and after a second fdg_set_params: the same weights, and the operators' kernels in the profile."""
    import torch
    from paper_2509_05679_b200 import binding
    layers = [(sy.EMBEDDING, 60, 32, 1, 1), (sy.CONV1X1, 32, 64, 1, 1), (sy.RECURRENCE, 64, 32, 1, 0), (sy.CONV1X1, 32, 32, 1, 1), (sy.RECURRENCE, 32, 16, 1, 0)] + TAIL
    net = sy.Net("tokens", layers, [3], 1, 40, 1, 10, 2, 8, 0.1, "bf16")
    p0 = sy.round_to_bf16(sy.init_params(net.layers, 0))
    streams = [torch.cuda.Stream() for _ in range(2)]
    out = []
    for kw, profile in ((dict(), False), (dict(streams=[s.cuda_stream for s in streams]), False), (dict(), True)):
        ctx = make_ctx(net, p0, grid_sms=148, **kw)
        ctx.set_distill(4, 2.0, 0.5)
        for _ in range(2):
            ctx.set_params(p0)
            ctx.profile(profile)
            for t in range(9):
                held = [binding.to_device("bf16", sy.batch_inputs(net, t))] + [torch.from_numpy(a).cuda() for a in (sy.batch_labels(net, t), *sy.batch_teacher(net, t, 4))]
                torch.cuda.synchronize()
                ctx.step_distill(*held)
                ctx.wait_ingest()
            out.append(ctx.params())
        if profile:
            seen = {name for name, r in ctx.profile_read().items() if r["launches"] > 0}
            ctx.profile(False)
            assert {"embed_fwd", "embed_grad", "recur_fwd", "recur_bwd", "distill"} <= seen
        ctx.close()
    assert np.isfinite(out[0]).all() and not np.array_equal(out[0], p0)
    assert all(np.array_equal(out[0], o) for o in out[1:])


def test_operators_captured_under_the_profiler(orc):
    """A caller's graph of operators recorded while a context's profiler is on: its launches are counted, have no time, and no step is blamed for them; calls outside of it are timed."""
    import torch
    from paper_2509_05679_b200 import binding, operators as ops
    net = sy.Net("mlp", [(sy.LINEAR, 8, 16, 1, 1), (sy.LINEAR, 16, 10, 1, 1)], [], 1, 1, 8, 10, 2, 8, 0.1, "fp32")
    ctx = make_ctx(net, sy.init_params(net.layers, 0))
    x, y = binding.to_device("fp32", sy.batch_inputs(net, 0)), torch.from_numpy(sy.batch_labels(net, 0)).cuda()
    tok = torch.zeros(700, dtype=torch.int32, device="cuda")
    dy = torch.ones(700, 32, device="cuda")
    run = lambda: (ops.embedding_grad(tok, dy, 50), ops.recurrence(dy.view(7, 100, 32), dy.view(7, 100, 32)))
    run()
    ctx.profile(True)
    run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    graph.replay()
    want = run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1][0], want[1][0])
    seen = ctx.profile_read()
    ctx.profile(False)
    ctx.step(x, y)
    assert ctx.step(x, y, want_loss=True) > 0
    for name in ("embed_grad", "recur_fwd"):
        assert seen[name]["launches"] == 3 and seen[name]["ms"] > 0
    ctx.close()

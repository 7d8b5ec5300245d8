"""Networks of token sequences through fdg_step: embedding, per-token convolutions, gated recurrences, pooling and a linear layer, with the labels' loss and
with a teacher's, split into modules, over workers and weight replicas, against the oracle (tolerances of the framework's other parity tests)."""
import numpy as np
import pytest

from paper_2509_05679_b200 import synth as sy
from harness import grad_max_err, grad_rel_l2, make_ctx, make_oracle, max_rel_err, run_parity

pytestmark = pytest.mark.gpu


def _net(dtype, widths, shape, workers, batch, splits=(), vocab=50, classes=10, residual=False, flags=sy.FLAG_SCALED):
    """embedding -> (1x1 convolution -> recurrence) per width -> average -> linear"""
    layers = [(sy.EMBEDDING, vocab, widths[0], 1, flags)]
    c = widths[0]
    for w in widths[1:]:
        if residual:
            layers.append((sy.RES_BEGIN, c, c, 1, 0))
        layers += [(sy.CONV1X1, c, 2 * w, 1, sy.FLAG_BIAS), (sy.RECURRENCE, 2 * w, w, 1, 0)]
        if residual:
            layers.append((sy.RES_ADD, c, w, 1, 0))
        c = w
    layers += [(sy.GLOBAL_AVGPOOL, c, c, 1, 0), (sy.LINEAR, c, classes, 1, sy.FLAG_BIAS)]
    return sy.Net("tokens", layers, list(splits), shape[0], shape[1], 1, classes, workers, batch, 0.1, dtype)


CASES = [((5, 7, 6), (1, 1), 1, 1, ()), ((24, 24, 16), (1, 13), 2, 3, (3,)), ((32, 32, 48), (6, 10), 3, 4, (1, 3)), ((64, 64, 128), (4, 16), 2, 8, (3,)),
         ((16, 33), (1, 700), 2, 2, (2,)), ((20, 8), (3, 50), 9, 7, ())]


def _id(c):
    return f"{'-'.join(map(str, c[0]))}_{c[1][0]}x{c[1][1]}_{c[2]}x{c[3]}_K{len(c[4]) + 1}"


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_fp32(orc, case):
    widths, shape, workers, batch, splits = case
    run_parity(orc, _net("fp32", widths, shape, workers, batch, splits), 2 * len(splits) + 6, param_tol=1e-5, loss_tol=1e-5)


@pytest.mark.parametrize("case", CASES, ids=_id)
def test_bf16(orc, case):
    widths, shape, workers, batch, splits = case
    run_parity(orc, _net("bf16", widths, shape, workers, batch, splits), 2 * len(splits) + 6, grad_tol=2e-2, loss_tol=1e-2)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_residual_blocks_add_to_a_recurrences_input_gradient(orc, dtype):
    """The block's input has two readers, and a recurrence directly behind a block's beginning adds its gradient to the shortcut's."""
    tol = dict(param_tol=1e-5, loss_tol=1e-5) if dtype == "fp32" else dict(grad_tol=2e-2, loss_tol=1e-2)
    run_parity(orc, _net(dtype, (24, 24, 24), (2, 9), 2, 4, (5,), residual=True), 6, **tol)
    layers = [(sy.EMBEDDING, 30, 32, 1, 0), (sy.RES_BEGIN, 32, 32, 1, 0), (sy.RECURRENCE, 32, 16, 1, 0), (sy.CONV1X1, 16, 32, 1, 1), (sy.RES_ADD, 32, 32, 1, 0),
              (sy.GLOBAL_AVGPOOL, 32, 32, 1, 0), (sy.LINEAR, 32, 10, 1, 1)]
    run_parity(orc, sy.Net("tokens", layers, [], 1, 20, 1, 10, 2, 4, 0.1, dtype), 4, **tol)


def test_recurrence_as_the_networks_first_layer(orc):
    """On real inputs: nobody wants the input's gradient."""
    layers = [(sy.RECURRENCE, 12, 6, 1, 0), (sy.GLOBAL_AVGPOOL, 6, 6, 1, 0), (sy.LINEAR, 6, 10, 1, 1)]
    run_parity(orc, sy.Net("series", layers, [1], 3, 17, 12, 10, 2, 5, 0.1, "fp32"), 6, param_tol=1e-5, loss_tol=1e-5)


def test_many_classes_and_relu_behind_an_embedding(orc):
    layers = [(sy.EMBEDDING, 40, 16, 1, 0), (sy.CONV1X1, 16, 32, 1, 1), (sy.RECURRENCE, 32, 16, 1, 0), (sy.GLOBAL_AVGPOOL, 16, 16, 1, 0), (sy.LINEAR, 16, 300, 1, 1)]
    run_parity(orc, sy.Net("tokens", layers, [2], 1, 9, 1, 300, 2, 4, 0.1, "fp32"), 6, param_tol=1e-5, loss_tol=1e-5)


def test_one_stream_worker_groups_and_many_streams_agree():
    """serial, worker_groups (ignored where a layer runs over all workers) and the streams of the default leave the same weights."""
    import torch
    from paper_2509_05679_b200 import binding
    net = _net("bf16", (64, 64, 64), (1, 32), 4, 4, (3,))
    p0 = sy.round_to_bf16(sy.init_params(net.layers, 0))
    out = []
    for kw in (dict(grid_sms=148), dict(serial=True, grid_sms=148), dict(worker_groups=4, grid_sms=148)):
        ctx = make_ctx(net, p0, **kw)
        for t in range(12):
            x, y = binding.to_device("bf16", sy.batch_inputs(net, t)), torch.from_numpy(sy.batch_labels(net, t)).cuda()
            ctx.step(x, y)
            ctx.wait_ingest()       # from here on their memory may become the next batch's
        out.append(ctx.params())
        ctx.close()
    assert np.array_equal(out[0], out[1])
    assert np.array_equal(out[0][:net.layers[0][1] * 64], out[2][:net.layers[0][1] * 64])
    assert np.isfinite(out[0]).all() and not np.array_equal(out[0], p0)


def test_host_inputs_and_two_runs_of_a_context(orc):
    net = _net("fp32", (24, 16), (1, 11), 2, 3, (2,))
    p0 = sy.init_params(net.layers, 0)
    ctx = make_ctx(net, p0)
    runs = []
    for _ in range(2):
        ctx.set_params(p0)
        for t in range(7):
            ctx.step_host(sy.batch_inputs(net, t), sy.batch_labels(net, t))
        runs.append(ctx.params())
    ctx.close()
    o = make_oracle(orc, net, p0)
    for t in range(7):
        o.step(sy.batch_inputs(net, t), sy.batch_labels(net, t), net.lr)
    assert np.array_equal(runs[0], runs[1])
    assert max_rel_err(runs[0], o.params(0), net.layers)[0] <= 1e-5


def test_one_replica_per_worker(orc):
    """A mixing matrix: every worker has a table of its own."""
    import torch
    from paper_2509_05679_b200 import binding
    net = _net("fp32", (16, 24), (1, 12), 3, 4, (2,))
    P = np.array([[0.6, 0.3, 0.1], [0.2, 0.7, 0.1], [0.3, 0.1, 0.6]])
    p0 = sy.init_params(net.layers, 0)
    o = orc.Oracle(net.layers, net.splits, 3, 4, (1, 12, 1), 10, P=P)
    ctx = make_ctx(net, p0, mixing=P)
    o.set_params(p0)
    for r in range(1, 3):
        q = (p0 * (1 + 0.1 * r)).astype(np.float32)
        o.set_params(q, r)
        ctx.set_params_worker(r, q)
    for t in range(7):
        x, y = sy.batch_inputs(net, t), sy.batch_labels(net, t)
        o.step(x, y, net.lr)
        ctx.step(binding.to_device("fp32", x), torch.from_numpy(y).cuda())
        for r in range(3):
            assert max_rel_err(ctx.params_worker(r), o.params(r), net.layers)[0] <= 1e-5, (t, r)
    ctx.close()


def _distil(orc, net, steps, top, tau, weight, *, odd=False, pinned=False, P=None, pair_bn=False, **kw):
    """Both sides step with a teacher; schedule, loss and parameters (fp32) or gradients (bf16) agree.  odd: labels and ids outside, entries of no weight."""
    import torch
    from paper_2509_05679_b200 import binding
    p0 = sy.init_params(net.layers, 0)
    if net.dtype == "bf16":
        p0 = sy.round_to_bf16(p0)
    o = orc.Oracle(net.layers, net.splits, net.n_workers, net.batch, (net.in_h, net.in_w, net.in_c), net.classes, P=P)
    o.storage_bf16(net.dtype == "bf16")
    o.set_distill(top, tau, weight)
    o.set_params(p0)
    ctx = make_ctx(net, p0, mixing=P, **kw)
    ctx.set_distill(top, tau, weight)
    for t in range(steps):
        x, y = sy.batch_inputs(net, t), sy.batch_labels(net, t)
        ids, teacher = sy.batch_teacher(net, t, top)
        if odd:
            y[t % net.M], ids[(t + 1) % net.M, 0], ids[(t + 2) % net.M] = -1, net.classes, -5
            teacher[(t + 3) % net.M, -1] = -np.inf
        lo, _ = o.step(x, y, net.lr, ids, teacher)
        put = (lambda a: torch.from_numpy(a).pin_memory()) if pinned else (lambda a: torch.from_numpy(a).cuda())
        held = [put(a) for a in (y, ids, teacher)]
        torch.cuda.synchronize()
        lg = ctx.step_distill(binding.to_device(net.dtype, x), *held, want_loss=True)
        ctx.wait_ingest()
        assert all((a == b).all() for a, b in zip(ctx.trace(), o.trace()))
        assert np.isnan(lg) == np.isnan(lo)
        if not np.isnan(lo):
            assert abs(lg - lo) <= (1e-5 if net.dtype == "fp32" else 1e-2) * abs(lo), (t, lg, lo)
        if net.dtype == "fp32":
            for r in range(net.n_workers if P is not None else 1):
                assert max_rel_err(ctx.params_worker(r), o.params(r), net.layers)[0] <= 1e-5, t
        else:
            g = np.mean([o.grads(s) for s in range(net.n_workers)], axis=0)
            assert grad_rel_l2(ctx.grads(), g, net.layers, pair_bn=pair_bn)[0] <= 2e-2, t
            assert grad_max_err(ctx.grads(), g, net.layers, pair_bn=pair_bn)[0] <= 3e-2, t
    ctx.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("classes,top,tau,weight,odd", [(10, 4, 2.0, 0.7, False), (10, 10, 1.0, 1.0, True), (300, 7, 1.5, 0.5, True), (2000, 64, 4.0, 0.9, False)])
def test_distillation(orc, classes, top, tau, weight, odd, dtype):
    _distil(orc, _net(dtype, (32, 32), (1, 15), 2, 4, (2,), classes=classes), 8, top, tau, weight, odd=odd)


def test_distillation_of_networks_of_images_and_vectors(orc):
    layers, _ = sy.resnet_layers(widths=(64,), blocks=1, in_c=3, classes=10)
    _distil(orc, sy.without_relu(sy.Net("image", layers, [], 8, 8, 3, 10, 2, 4, 0.05, "bf16")), 3, 4, 2.0, 0.5, pair_bn=True)          # (see harness.gradient_groups)
    orc.kink_margin(True)
    _distil(orc, sy.Net("mlp", sy.mlp_layers([12, 32, 24, 10]), [2], 1, 1, 12, 10, 2, 8, 0.05, "fp32"), 8, 4, 2.0, 0.5)
    assert orc.kink_margin(True) >= 2e-6            # nearer to a kink, fp32 and fp64 may take different branches


@pytest.mark.parametrize("net", ["mlp", "resnet"])
def test_without_the_teachers_term_it_is_cross_entropy(net):
    """weight 0 against the labels' loss on the same forward pass (ReLU layers included): the fused head, off here, applies the mask of the layer below, which has to be
    applied all the same.  The error gradients of the logits are rounded once on either side, from values off by a few fp32 roundings."""
    import torch
    from paper_2509_05679_b200 import binding
    if net == "mlp":
        net = sy.Net("mlp", sy.mlp_layers([64, 64, 128, 10]), [], 1, 1, 64, 10, 2, 32, 0.01, "bf16")
    else:
        net = sy.Net("image", sy.resnet_layers(widths=(64, 128), blocks=1, in_c=3, classes=10)[0], [], 16, 16, 3, 10, 2, 4, 0.01, "bf16")
    p0 = sy.round_to_bf16(sy.init_params(net.layers, 0))
    x, y = binding.to_device("bf16", sy.batch_inputs(net, 0)), torch.from_numpy(sy.batch_labels(net, 0)).cuda()
    ids, teacher = (torch.from_numpy(a).cuda() for a in sy.batch_teacher(net, 0, 3))
    a, b = make_ctx(net, p0), make_ctx(net, p0)
    b.set_distill(3, 2.0, 0.0)
    la, lb = a.step(x, y, want_loss=True), b.step_distill(x, y, ids, teacher, want_loss=True)
    assert abs(la - lb) <= 1e-5 * la
    assert grad_rel_l2(b.grads(), a.grads(), net.layers)[0] <= 2e-2
    assert grad_max_err(b.grads(), a.grads(), net.layers)[0] <= 3e-2
    a.close()
    b.close()


def test_distillation_from_pinned_memory_and_over_replicas(orc):
    net = _net("fp32", (16, 16), (1, 9), 3, 2, (2,))
    _distil(orc, net, 7, 3, 2.0, 0.5, pinned=True)
    _distil(orc, net, 7, 3, 2.0, 0.5, P=np.array([[0.5, 0.5, 0], [0.5, 0.25, 0.25], [0, 0.25, 0.75]]))
    _distil(orc, net, 7, 3, 2.0, 0.5, serial=True)


def test_parameters_are_laid_out_with_the_table_first():
    net = _net("bf16", (24, 16), (1, 8), 1, 2)
    ctx = make_ctx(net, sy.init_params(net.layers, 0))
    lay = ctx.param_layout()
    ctx.close()
    assert lay[0] == (0, 0, "W", (50, 24), 0, 1200)
    assert [(r[0], r[2], tuple(r[3])) for r in lay] == [(i, n, tuple(s)) for i, n, s, _ in sy.param_shapes(net.layers)]


def test_refused_networks_and_calls():
    import torch
    from paper_2509_05679_b200 import binding
    tail = [(sy.GLOBAL_AVGPOOL, 8, 8, 1, 0), (sy.LINEAR, 8, 10, 1, 1)]

    def make(layers, shape=(1, 6, 1)):
        binding.Context(layers, [], 1, 2, 0.1, dtype="fp32", in_shape=shape, num_classes=10).close()

    for layers, shape in [([(sy.EMBEDDING, 9, 8, 1, 0)] + tail, (1, 6, 2)), ([(sy.EMBEDDING, 0, 8, 1, 0)] + tail, (1, 6, 1)),
                          ([(sy.CONV1X1, 1, 1, 1, 0), (sy.EMBEDDING, 9, 8, 1, 0)] + tail, (1, 6, 1)), ([(sy.EMBEDDING, 9, 16, 1, 0), (sy.RECURRENCE, 16, 16, 1, 0)] + tail, (1, 6, 1)),
                          ([(sy.EMBEDDING, 9, 12, 1, 0), (sy.RECURRENCE, 16, 8, 1, 0)] + tail, (1, 6, 1))]:
        with pytest.raises(binding.FdgError) as e:
            make(layers, shape)
        assert e.value.status == 3
    make([(sy.EMBEDDING, 9, 16, 1, 0), (sy.RECURRENCE, 16, 8, 1, 0)] + tail)

    net = _net("fp32", (8, 8), (1, 6), 1, 2)
    p0 = sy.init_params(net.layers, 0)
    x, y = binding.to_device("fp32", sy.batch_inputs(net, 0)), torch.zeros(2, dtype=torch.int32, device="cuda")
    ids, teacher = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, 3, device="cuda")
    ctx = make_ctx(net, p0)

    def status(f):
        with pytest.raises(binding.FdgError) as e:
            f()
        return e.value.status

    assert status(lambda: ctx.step_distill(x, y, ids, teacher)) == 8                  # not set
    for bad in ((0, 1.0, 0.5), (1025, 1.0, 0.5), (3, 0.0, 0.5), (3, float("nan"), 0.5), (3, 1.0, 1.5), (3, 1.0, float("nan"))):
        assert status(lambda: ctx.set_distill(*bad)) == 1
    ctx.set_distill(3, 2.0, 0.5)
    assert status(lambda: ctx.set_distill(3, 2.0, 0.5)) == 8                          # twice
    assert status(lambda: ctx.step(x, y)) == 8
    assert status(lambda: ctx.step_distill(x, y, None, teacher)) == 1
    assert status(lambda: ctx.step_distill(x, y, ids, np.zeros((2, 3), np.float32))) == 1       # pageable host memory
    assert status(lambda: ctx.step_distill(np.zeros(12, np.int32), y, ids, teacher)) == 1
    assert ctx.step_distill(x, y, ids, teacher, want_loss=True) > 0
    ctx.close()
    ctx = make_ctx(net, p0)
    ctx.step(x, y)
    assert status(lambda: ctx.set_distill(3, 2.0, 0.5)) == 8                          # after a step
    ctx.close()

"""Pins of the oracle's layers for token sequences (embedding, gated recurrence) and of its distillation loss: gradients against central differences,
values against straight-line forms."""
import numpy as np
import pytest

from oracle import oracle as orc
from paper_2509_05679_b200 import synth as sy


def _net(workers=2, batch=3, splits=()):
    layers = [(sy.EMBEDDING, 11, 6, 1, sy.FLAG_SCALED), (sy.CONV1X1, 6, 8, 1, sy.FLAG_BIAS), (sy.RECURRENCE, 8, 4, 1, 0), (sy.GLOBAL_AVGPOOL, 4, 4, 1, 0),
              (sy.LINEAR, 4, 5, 1, sy.FLAG_BIAS)]
    return sy.Net("tokens", layers, list(splits), 2, 7, 1, 5, workers, batch, 0.1, "fp32")


def test_gradient_of_embedding_and_recurrence_against_differences():
    net = _net()
    p = sy.perturb_params(sy.init_params(net.layers, 3), net.layers, 4, 0.3).astype(np.float64)
    x, y = sy.batch_inputs(net, 0), sy.batch_labels(net, 0)
    assert (x == -1).any() and x.dtype == np.int32
    shape = (net.in_h, net.in_w, net.in_c)
    _, g = orc.plain_loss_grad(net.layers, net.n_workers, net.batch, shape, p, x, y)
    g = g / net.n_workers                            # mean over all samples
    h = 1e-5
    for i in range(p.size):
        q = p.copy()
        q[i] += h
        hi, _ = orc.plain_loss_grad(net.layers, net.n_workers, net.batch, shape, q, x, y, want_grad=False)
        q[i] -= 2 * h
        lo, _ = orc.plain_loss_grad(net.layers, net.n_workers, net.batch, shape, q, x, y, want_grad=False)
        assert abs((hi - lo) / (2 * h) - g[i]) <= 1e-8, i       # h^2 times a third derivative, rounding of 1e-16 / h


def test_logits_of_embedding_and_recurrence_in_numpy():
    net = _net(1, 2)
    p = sy.perturb_params(sy.init_params(net.layers, 1), net.layers, 2, 0.3).astype(np.float64)
    x = sy.batch_inputs(net, 5)
    x[0, 0, 0, 0], x[1, 1, 3, 0] = 11, 400000         # outside the table
    table, w, b, wl, bl = np.split(p, np.cumsum([66, 48, 8, 20]))
    table, w, wl = table.reshape(11, 6), w.reshape(8, 6), wl.reshape(5, 4)
    ids = x.reshape(2, 14)
    e = np.where(((ids >= 0) & (ids < 11))[..., None], np.sqrt(np.float32(6)).astype(np.float64) * table[np.clip(ids, 0, 10)], 0.0)
    u = e @ w.T + b
    h = np.zeros((2, 4))
    total = 0
    for t in range(14):
        a = 1 / (1 + np.exp(-u[:, t, :4]))
        h = a * h + (1 - a) * u[:, t, 4:]
        total = total + h
    np.testing.assert_allclose(orc.plain_logits(net.layers, 1, 2, (2, 7, 1), p, x, 5), total / 14 @ wl.T + bl, rtol=1e-12, atol=1e-12)


@pytest.mark.parametrize("tau,weight", [(1.0, 1.0), (2.0, 0.4), (0.7, 0.0)])
def test_distillation_step_in_torch(tau, weight):
    """One module, one worker: the update is lr times torch's gradient of the loss."""
    import torch
    net = _net(1, 4)
    top = 3
    p = sy.perturb_params(sy.init_params(net.layers, 1), net.layers, 2, 0.3).astype(np.float64)
    x, y = sy.batch_inputs(net, 0), sy.batch_labels(net, 0)
    ids, teacher = sy.batch_teacher(net, 0, top)
    y[1], ids[2, 1], teacher[3, 0] = -1, -1, -np.inf
    o = orc.Oracle(net.layers, [], 1, 4, (2, 7, 1), 5)
    o.set_distill(top, tau, weight)
    o.set_params(p)
    loss, _ = o.step(x, y, 0.5, ids, teacher)
    z = torch.tensor(orc.plain_logits(net.layers, 1, 4, (2, 7, 1), p, x, 5), requires_grad=True)
    t = torch.where(torch.tensor(ids) >= 0, torch.tensor(teacher, dtype=torch.float64), -torch.inf)
    q = torch.softmax(t / tau, 1)
    lq = torch.log_softmax(z / tau, 1).gather(1, torch.tensor(ids).clamp(min=0).long())
    kl = torch.where(q > 0, q * (torch.log(q.clamp(min=1e-300)) - lq), 0.0).sum(1)
    ce = -torch.log_softmax(z, 1).gather(1, torch.tensor(y).clamp(min=0).long()[:, None])[:, 0]
    rows = (weight * tau ** 2 * kl + (1 - weight) * ce) * (torch.tensor(y) >= 0)
    assert abs(loss - float(rows.mean().detach())) <= 1e-12
    rows.mean().backward()
    bias = (p - o.params())[-5:] / 0.5                # gradient of the last bias: the logits' summed over the samples
    np.testing.assert_allclose(bias, z.grad.sum(0).numpy(), rtol=1e-9, atol=1e-12)


def test_split_network_distils_with_its_batch():
    """The teacher travels with its batch: with zero step size every batch's loss is the one-module loss of the same batch."""
    a, b = _net(2, 3), _net(2, 3, (2, 3))
    p = sy.init_params(a.layers, 1).astype(np.float64)
    run = []
    for net in (a, b):
        o = orc.Oracle(net.layers, net.splits, 2, 3, (2, 7, 1), 5)
        o.set_distill(2, 1.5, 0.5)
        o.set_params(p)
        losses = {}
        for t in range(6):
            loss, batch = o.step(sy.batch_inputs(net, t), sy.batch_labels(net, t), 0.0, *sy.batch_teacher(net, t, 2))
            losses[batch] = loss
        run.append(losses)
    for batch in range(4):
        assert abs(run[0][batch] - run[1][batch]) <= 1e-14

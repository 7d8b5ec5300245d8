"""The operators' entry points without a GPU: arguments that no device is needed for are refused with a message, sizes are answered, and a
good call reports that there is no device instead of falling back."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def L():
    from paper_2509_05679_b200 import binding, build
    build.build_lib()
    return binding.lib()


def _rec(**kw):
    from paper_2509_05679_b200 import binding
    d = dict(dtype=1, batch=2, steps=5, channels=8, gate_batch=80, gate_step=16, value_batch=80, value_step=16, y_batch=40, y_step=8, dy_batch=40, dy_step=8,
             dgate_batch=80, dgate_step=16, dvalue_batch=80, dvalue_step=16)
    d.update(kw)
    return binding.fdg_recurrence(**d)


def _dis(**kw):
    from paper_2509_05679_b200 import binding
    d = dict(logits_dtype=1, dlogits_dtype=1, top=4, rows=3, vocab=100, logits_stride=100, dlogits_stride=100, temperature=2.0, weight=0.5, scale=1.0)
    d.update(kw)
    return binding.fdg_distill(**d)


def test_workspace_and_saved_sizes(L):
    n = C.c_size_t(77)
    assert L.fdg_embedding_workspace(0, 1, 1, C.byref(n)) == 0
    assert L.fdg_embedding_workspace(1 << 20, 1 << 17, 1024, C.byref(n)) == 0
    assert L.fdg_recurrence_saved(C.byref(_rec()), C.byref(n)) == 0 and n.value >= 2 * 8 * 4
    assert L.fdg_recurrence_saved(C.byref(_rec(steps=0)), C.byref(n)) == 0 and n.value == 0
    assert L.fdg_recurrence_saved(C.byref(_rec(batch=0)), C.byref(n)) == 0 and n.value == 0


@pytest.mark.parametrize("args", [(-1, 10, 4), (10, 0, 4), (10, 10, 0), (1 << 31, 10, 4), (10, (1 << 31) - 1, 4), (10, 10, (1 << 20) + 1)])
def test_embedding_sizes_are_refused(L, args):
    n = C.c_size_t(77)
    assert L.fdg_embedding_workspace(*args, C.byref(n)) == 1 and n.value == 77
    assert b"fdg_embedding_workspace" in L.fdg_op_last_error()
    assert L.fdg_embedding_forward(None, args[0], None, 1, args[1], args[2], 1.0, None, 1 << 20, None) == 1
    assert L.fdg_embedding_backward(None, args[0], None, 1, 1 << 20, args[1], args[2], 1.0, 0, None, None, 1 << 40, None) == 1


def test_embedding_arguments_are_refused(L):
    assert L.fdg_embedding_workspace(1, 1, 1, None) == 1
    assert L.fdg_embedding_forward(None, 4, None, 2, 10, 4, 1.0, None, 4, None) == 1
    assert L.fdg_embedding_forward(None, 4, None, 1, 10, 4, 1.0, None, 3, None) == 1
    assert L.fdg_embedding_backward(None, 4, None, 1, -1, 10, 4, 1.0, 0, None, None, 1 << 40, None) == 1


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(batch=-1), dict(steps=-1), dict(steps=1 << 31), dict(channels=0), dict(channels=(1 << 20) + 1),
                                 dict(batch=1 << 20, steps=1 << 20, channels=1 << 10), dict(gate_step=-16), dict(value_batch=1 << 46), dict(y_step=7), dict(y_batch=39),
                                 dict(y_batch=0)])
def test_recurrence_shapes_are_refused(L, bad):
    assert L.fdg_recurrence_forward(C.byref(_rec(**bad)), None, None, None, None, None, None, None, None) == 1
    assert b"fdg_recurrence_forward" in L.fdg_op_last_error()


@pytest.mark.parametrize("bad", [dict(dgate_step=7), dict(dvalue_batch=9), dict(dy_batch=-1), dict(dgate_batch=0)])
def test_recurrence_gradients_shapes_are_refused(L, bad):
    assert L.fdg_recurrence_backward(C.byref(_rec(**bad)), *[None] * 10) == 1
    assert b"fdg_recurrence_backward" in L.fdg_op_last_error()


def test_recurrence_without_a_shape_is_refused(L):
    assert L.fdg_recurrence_saved(None, None) == 1
    assert L.fdg_recurrence_saved(C.byref(_rec()), None) == 1
    assert L.fdg_recurrence_forward(None, *[None] * 8) == 1
    assert L.fdg_recurrence_backward(None, *[None] * 10) == 1


@pytest.mark.parametrize("bad,status", [(dict(logits_dtype=3), 1), (dict(rows=-1), 1), (dict(vocab=0), 3), (dict(vocab=262145), 3), (dict(top=-1), 3), (dict(top=1025), 3),
                                        (dict(temperature=0.0), 1), (dict(temperature=-1.0), 1), (dict(temperature=float("nan")), 1), (dict(temperature=float("inf")), 1),
                                        (dict(weight=-0.1), 1), (dict(weight=1.1), 1), (dict(weight=float("nan")), 1), (dict(logits_stride=-1), 1)])
def test_distillation_arguments_are_refused(L, bad, status):
    assert L.fdg_distill_loss(C.byref(_dis(**bad)), None, 16, None, None, None, None, None) == status
    assert b"fdg_distill_loss" in L.fdg_op_last_error()


def test_distillation_outputs_are_refused(L):
    assert L.fdg_distill_loss(None, *[None] * 7) == 1
    assert L.fdg_distill_loss(C.byref(_dis()), None, None, None, None, None, None, None) == 1                       # no labels, weight 0.5
    assert L.fdg_distill_loss(C.byref(_dis(dlogits_dtype=0)), None, 16, None, None, None, 16, None) == 3            # bf16 logits, fp32 gradient
    assert L.fdg_distill_loss(C.byref(_dis(dlogits_stride=99)), None, 16, None, None, None, 16, None) == 1
    assert L.fdg_distill_loss(C.byref(_dis(logits_dtype=0)), 16, 16, None, None, None, 16, None) == 1               # in place with another type


def test_a_good_call_without_a_device_says_so(L):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    assert L.fdg_embedding_forward(16, 4, 16, 1, 10, 4, 1.0, 16, 4, None) == 4
    assert L.fdg_embedding_backward(16, 4, 16, 1, 4, 10, 4, 1.0, 0, 16, 256, 1 << 40, None) == 4
    assert L.fdg_recurrence_forward(C.byref(_rec()), *[16] * 7, None) == 4
    assert L.fdg_recurrence_backward(C.byref(_rec()), *[16] * 9, None) == 4
    assert L.fdg_distill_loss(C.byref(_dis()), 16, 16, 16, 16, 16, 32, None) == 4
    assert b"device" in L.fdg_op_last_error()


def test_tensors_on_the_host_are_refused():
    import torch
    from paper_2509_05679_b200 import operators as ops
    from paper_2509_05679_b200.binding import FdgError
    with pytest.raises(FdgError):
        ops.embedding(torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4))
    with pytest.raises(FdgError):
        ops.embedding_grad(torch.zeros(4, dtype=torch.int32), torch.zeros(4, 4), 4)
    with pytest.raises(FdgError):
        ops.recurrence(torch.zeros(1, 2, 4), torch.zeros(1, 2, 4))
    with pytest.raises(FdgError):
        ops.distill_loss(torch.zeros(2, 4), None, torch.zeros(2, 1, dtype=torch.int32), torch.zeros(2, 1))

"""The operators on token sequences, on torch tensors (see ``include/fdg.h`` for what they compute): embedding lookup and its gradient,
gated linear recurrence and its gradient, distillation loss with its gradient.

Arguments are marshalled and checked here; the work is done by the library's kernels, on torch's current stream of the tensors' device.
Outputs (unless given) and workspaces come from torch's caching allocator on that stream, so calls can be captured into a CUDA graph
like torch's own.  There is no CPU path.  Nothing is recorded for autograd: the gradients are calls of their own.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import binding
from .binding import FdgError

_DTYPE = {torch.float32: 0, torch.bfloat16: 1}


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise FdgError(1, what)


def _tensor(name: str, t, dtypes, ndim: int, like: Optional[torch.Tensor] = None, contiguous: bool = False) -> None:
    """t is a CUDA tensor of one of these types and this many dimensions, on `like`'s device, its last dimension dense."""
    _need(isinstance(t, torch.Tensor) and t.is_cuda, f"{name} must be a CUDA tensor")
    _need(t.dtype in dtypes, f"{name} must be of type {' or '.join(str(d) for d in dtypes)}, not {t.dtype}")
    _need(t.dim() == ndim, f"{name} must have {ndim} dimensions, not {t.dim()}")
    _need(like is None or t.device == like.device, f"{name} must be on the same device as the other tensors")
    if contiguous:
        _need(t.is_contiguous(), f"{name} must be contiguous")
    else:
        _need(t.shape[-1] <= 1 or t.stride(-1) == 1, f"the last dimension of {name} must be dense")


def _shape(name: str, t: torch.Tensor, shape) -> None:
    _need(tuple(t.shape) == tuple(shape), f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")


def _call(t: torch.Tensor, fn: str, *args) -> None:
    """fn(*args, stream) with t's device current, on torch's current stream of it."""
    L = binding.lib()
    if torch.cuda.current_device() == t.device.index:
        st = getattr(L, fn)(*args, torch.cuda.current_stream().cuda_stream or None)
    else:
        with torch.cuda.device(t.device):
            st = getattr(L, fn)(*args, torch.cuda.current_stream().cuda_stream or None)
    if st != 0:
        raise FdgError(st, (L.fdg_op_last_error() or b"").decode())


def _addr(t: Optional[torch.Tensor]):
    return t.data_ptr() or None if t is not None else None


def _row_stride(t: torch.Tensor) -> int:
    """Of a 2-D tensor's rows; of a single row, where torch's number says nothing, its length."""
    return t.stride(0) if t.shape[0] > 1 else max(1, t.shape[1])


def embedding(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``scale * table[tokens]``; rows of zeros for ids outside the table.  tokens: int32, any shape, contiguous; table [vocab, channels]
    fp32 or bf16, contiguous; out: [tokens.numel(), channels] of its type (rows may be apart), by default a new tensor of tokens' shape + [channels]."""
    _tensor("table", table, _DTYPE, 2, contiguous=True)
    _tensor("tokens", tokens, (torch.int32,), tokens.dim() if isinstance(tokens, torch.Tensor) else 1, table, contiguous=True)
    vocab, c = table.shape
    n = tokens.numel()
    res = out
    if out is None:
        res = torch.empty(*tokens.shape, c, dtype=table.dtype, device=table.device)
        out = res.view(n, c)
    _tensor("out", out, (table.dtype,), 2, table)
    _shape("out", out, (n, c))
    _call(table, "fdg_embedding_forward", _addr(tokens), n, _addr(table), _DTYPE[table.dtype], vocab, c, scale, _addr(out), _row_stride(out))
    return res


def embedding_grad(tokens: torch.Tensor, dy: torch.Tensor, vocab: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   accumulate: bool = False) -> torch.Tensor:
    """Gradient of `embedding`'s table, fp32 [vocab, channels]: row v is ``scale *`` the sum of dy's rows whose token is v.  accumulate: added to
    ``out``, whose other rows stay as they are.  tokens: int32, contiguous; dy: tokens' shape + [channels], or [tokens.numel(), channels] with rows apart."""
    _need(isinstance(dy, torch.Tensor) and isinstance(tokens, torch.Tensor), "tokens and dy must be CUDA tensors")
    if dy.dim() != 2:
        _need(dy.dim() > 0 and tuple(dy.shape[:-1]) == tuple(tokens.shape) and dy.is_contiguous(), "dy must be contiguous, of tokens' shape and the channels")
        dy = dy.view(-1 if dy.shape[-1] else 0, dy.shape[-1])
    _tensor("dy", dy, _DTYPE, 2)
    _tensor("tokens", tokens, (torch.int32,), tokens.dim(), dy, contiguous=True)
    n, c = dy.shape
    _need(tokens.numel() == n, f"dy must have a row for each of the {tokens.numel()} tokens, not {n}")
    _need(out is not None or not accumulate, "accumulate needs the gradient to add to")
    if out is None:
        out = torch.empty(vocab, c, dtype=torch.float32, device=dy.device)
    _tensor("out", out, (torch.float32,), 2, dy, contiguous=True)
    _shape("out", out, (vocab, c))
    need = C.c_size_t()
    st = binding.lib().fdg_embedding_workspace(n, vocab, c, C.byref(need))
    if st != 0:
        raise FdgError(st, (binding.lib().fdg_op_last_error() or b"").decode())
    ws = torch.empty(need.value, dtype=torch.uint8, device=dy.device) if need.value else None
    _call(dy, "fdg_embedding_backward", _addr(tokens), n, _addr(dy), _DTYPE[dy.dtype], _row_stride(dy), vocab, c, scale, int(accumulate), _addr(out), _addr(ws), need.value)
    return out


def _recurrence_shape(gate, value, **strided) -> binding.fdg_recurrence:
    _tensor("gate", gate, _DTYPE, 3)
    _tensor("value", value, (gate.dtype,), 3, gate)
    _shape("value", value, gate.shape)
    s = binding.fdg_recurrence(_DTYPE[gate.dtype], *gate.shape)
    for name, t in dict(gate=gate, value=value, **strided).items():
        _tensor(name, t, (gate.dtype,), 3, gate)
        _shape(name, t, gate.shape)
        b, n, c = t.shape                      # of an extent of 1 torch's stride says nothing
        step = t.stride(1) if n > 1 else max(c, 1)
        setattr(s, name + "_step", step)
        setattr(s, name + "_batch", t.stride(0) if b > 1 else step * max(n, 1))
    return s


def _state(name, t, gate):
    if t is not None:
        _tensor(name, t, (torch.float32,), 2, gate, contiguous=True)
        _shape(name, t, (gate.shape[0], gate.shape[2]))


def _lengths(t, gate):
    if t is not None:
        _tensor("lengths", t, (torch.int32,), 1, gate, contiguous=True)
        _shape("lengths", t, (gate.shape[0],))


def recurrence(gate: torch.Tensor, value: torch.Tensor, *, state: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
               for_grad: bool = False, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, ...]:
    """``h_t = a_t h_{t-1} + (1 - a_t) value_t`` with ``a = sigmoid(gate)``: (y, state after the last step) and, for_grad, what `recurrence_grad` needs.
    gate, value: [batch, steps, channels] fp32 or bf16, last dimension dense, other strides free; state: fp32 [batch, channels], zeros by default;
    lengths: int32 [batch], steps behind which do not count."""
    s = _recurrence_shape(gate, value)
    _state("state", state, gate)
    _lengths(lengths, gate)
    y = torch.empty(gate.shape, dtype=gate.dtype, device=gate.device) if out is None else out
    t = _recurrence_shape(gate, value, y=y)
    s.y_batch, s.y_step = t.y_batch, t.y_step
    last = torch.empty(gate.shape[0], gate.shape[2], dtype=torch.float32, device=gate.device)
    saved = None
    if for_grad:
        need = C.c_size_t()
        st = binding.lib().fdg_recurrence_saved(C.byref(s), C.byref(need))
        if st != 0:
            raise FdgError(st, (binding.lib().fdg_op_last_error() or b"").decode())
        saved = torch.empty(need.value, dtype=torch.uint8, device=gate.device)
    _call(gate, "fdg_recurrence_forward", C.byref(s), _addr(gate), _addr(value), _addr(lengths), _addr(state), _addr(y), _addr(last), _addr(saved))
    return (y, last, saved) if for_grad else (y, last)


def recurrence_grad(gate: torch.Tensor, value: torch.Tensor, dy: torch.Tensor, saved: torch.Tensor, *, dgate: torch.Tensor, dvalue: torch.Tensor,
                    dstate: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradients of `recurrence` for dy and, optionally, dstate (of the state after the last step): written to dgate and dvalue (tensors like
    gate and value, strides of their own; halves of one tensor, say); the gradient of the initial state is returned.  gate, value, lengths: those of the forward call."""
    s = _recurrence_shape(gate, value, dy=dy, dgate=dgate, dvalue=dvalue)
    _state("dstate", dstate, gate)
    _lengths(lengths, gate)
    _tensor("saved", saved, (torch.uint8,), 1, gate, contiguous=True)
    need = C.c_size_t()
    st = binding.lib().fdg_recurrence_saved(C.byref(s), C.byref(need))
    if st != 0:
        raise FdgError(st, (binding.lib().fdg_op_last_error() or b"").decode())
    _need(saved.numel() == need.value, f"saved must have {need.value} bytes (those of the forward call of this shape), not {saved.numel()}")
    first = torch.empty(gate.shape[0], gate.shape[2], dtype=torch.float32, device=gate.device)
    _call(gate, "fdg_recurrence_backward", C.byref(s), _addr(gate), _addr(value), _addr(lengths), _addr(saved), _addr(dy), _addr(dstate), _addr(dgate), _addr(dvalue),
          _addr(first))
    return first


def distill_loss(logits: torch.Tensor, labels: Optional[torch.Tensor], ids: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0, weight: float = 1.0,
                 scale: float = 1.0, grad: bool = True, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(loss of every row, gradient for the logits times `scale`): ``weight * temperature^2 * KL(teacher | student)`` over the teacher's top entries
    plus ``(1 - weight) *`` cross-entropy with the label.  logits: [rows, vocab] fp32 or bf16, rows may be apart; labels: int32 [rows] (a label
    outside the vocabulary takes its row out) or None with weight 1; ids int32, teacher fp32: [rows, top].  out: where the gradient goes (logits itself,
    or a bf16 tensor for fp32 logits); grad = False: the loss alone."""
    _tensor("logits", logits, _DTYPE, 2)
    m, v = logits.shape
    _tensor("ids", ids, (torch.int32,), 2, logits, contiguous=True)
    _tensor("teacher", teacher, (torch.float32,), 2, logits, contiguous=True)
    _need(ids.shape[0] == m, f"ids must have {m} rows, not {ids.shape[0]}")
    _shape("teacher", teacher, ids.shape)
    if labels is not None:
        _tensor("labels", labels, (torch.int32,), 1, logits, contiguous=True)
        _shape("labels", labels, (m,))
    _need(grad or out is None, "out is for the gradient")
    if grad and out is None:
        out = torch.empty(m, v, dtype=logits.dtype, device=logits.device)
    if grad:
        _tensor("out", out, _DTYPE, 2, logits)
        _shape("out", out, (m, v))
    loss = torch.empty(m, dtype=torch.float32, device=logits.device)
    d = binding.fdg_distill(_DTYPE[logits.dtype], _DTYPE[out.dtype] if grad else 0, ids.shape[1], m, v, _row_stride(logits), _row_stride(out) if grad else 0,
                            temperature, weight, scale)
    _call(logits, "fdg_distill_loss", C.byref(d), _addr(logits), _addr(labels), _addr(ids), _addr(teacher), _addr(loss), _addr(out) if grad else None)
    return loss, out

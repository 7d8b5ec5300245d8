"""The operators on token sequences, on torch tensors (see ``include/fdg.h`` for what they compute): embedding lookup and its gradient,
gated linear recurrence and its gradient, distillation loss with its gradient.

Arguments are marshalled and checked here; the work is done by the library's kernels, on torch's current stream of the tensors' device.
Outputs (unless given) and workspaces come from torch's caching allocator on that stream, so calls can be captured into a CUDA graph
like torch's own.  There is no CPU path.  Nothing is recorded for autograd: the gradients are calls of their own, and a tensor that autograd follows
(requires_grad, under grad mode) is refused; call under ``torch.no_grad()`` or pass ``t.detach()``.

The host's share of a small call is most of its time, so a check that holds costs a comparison and no text is made for it.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Tuple

import torch

from . import binding
from .binding import FdgError

_F32, _I32, _U8 = torch.float32, torch.int32, torch.uint8
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}
_fn = {}
_grad_mode = torch.is_grad_enabled


def _refuse(what: str):
    raise FdgError(1, what)


def _call(device: torch.device, name: str, *args) -> None:
    """The library's function name(*args, stream) with `device` current, on torch's current stream of it."""
    f = _fn.get(name)
    if f is None:
        f = _fn[name] = getattr(binding.lib(), name)
    i = device.index
    if torch.cuda.current_device() == i:
        st = f(*args, torch._C._cuda_getCurrentRawStream(i) or None)
    else:
        with torch.cuda.device(i):
            st = f(*args, torch._C._cuda_getCurrentRawStream(i) or None)
    if st != 0:
        raise FdgError(st, (binding.lib().fdg_op_last_error() or b"").decode())


def _bytes(name: str, *args) -> int:
    """A size that the library's function name(*args, &size) answers."""
    n = C.c_size_t()
    st = getattr(binding.lib(), name)(*args, C.byref(n))
    if st != 0:
        raise FdgError(st, (binding.lib().fdg_op_last_error() or b"").decode())
    return n.value


def _addr(t: Optional[torch.Tensor]):
    return (t.data_ptr() or None) if t is not None else None


def _dense(name: str, t, dtype, shape, device) -> None:
    """t is a contiguous CUDA tensor of this type, shape (as far as given) and device."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a CUDA tensor")
    if t.requires_grad and _grad_mode():
        _refuse(f"{name} requires a gradient, which nothing here records: call under torch.no_grad(), or pass {name}.detach()")
    if t.dtype is not dtype:
        _refuse(f"{name} must be of type {dtype}, not {t.dtype}")
    if device is not None and t.device != device:
        _refuse(f"{name} must be on the same device as the other tensors")
    if shape is not None and t.shape != shape:
        _refuse(f"{name} must have shape {tuple(shape)}, not {tuple(t.shape)}")
    if not t.is_contiguous():
        _refuse(f"{name} must be contiguous")


def _rows(name: str, t, dtype, ndim: int, shape, device):
    """The strides of a CUDA tensor of this type (None: fp32 or bf16), shape (as far as given) and device whose last dimension is dense.  An extent of 1 has any
    stride in torch: it gets the one of a contiguous tensor."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        _refuse(f"{name} must be a CUDA tensor")
    if t.requires_grad and _grad_mode():
        _refuse(f"{name} requires a gradient, which nothing here records: call under torch.no_grad(), or pass {name}.detach()")
    if t.dtype is not dtype and (dtype is not None or t.dtype not in _DTYPE):
        _refuse(f"{name} must be of type {dtype or 'float32 or bfloat16'}, not {t.dtype}")
    if device is not None and t.device != device:
        _refuse(f"{name} must be on the same device as the other tensors")
    s = t.shape
    if len(s) != ndim:
        _refuse(f"{name} must have {ndim} dimensions, not {len(s)}")
    if shape is not None and s != shape:
        _refuse(f"{name} must have shape {tuple(shape)}, not {tuple(s)}")
    st = t.stride()
    if st[-1] != 1 and s[-1] > 1:
        _refuse(f"the last dimension of {name} must be dense")
    c = s[-1] or 1
    if ndim == 2:
        return st[0] if s[0] > 1 else c
    step = st[1] if s[1] > 1 else c
    return (st[0] if s[0] > 1 else step * (s[1] or 1)), step


def embedding(tokens: torch.Tensor, table: torch.Tensor, *, scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """``scale * table[tokens]``; rows of zeros for ids outside the table.  tokens: int32, any shape, contiguous; table [vocab, channels]
    fp32 or bf16, contiguous; out: [tokens.numel(), channels] of its type (rows may be apart), by default a new tensor of tokens' shape + [channels]."""
    _rows("table", table, None, 2, None, None)
    dev, dtype = table.device, table.dtype
    _dense("table", table, dtype, None, dev)
    _dense("tokens", tokens, _I32, None, dev)
    vocab, c = table.shape
    n = tokens.numel()
    if out is None:
        out = table.new_empty((*tokens.shape, c))
        stride = c
    else:
        stride = _rows("out", out, dtype, 2, (n, c), dev)
    _call(dev, "fdg_embedding_forward", _addr(tokens), n, _addr(table), _DTYPE[dtype], vocab, c, scale, _addr(out), stride)
    return out


def embedding_grad(tokens: torch.Tensor, dy: torch.Tensor, vocab: int, *, scale: float = 1.0, out: Optional[torch.Tensor] = None,
                   accumulate: bool = False) -> torch.Tensor:
    """Gradient of `embedding`'s table, fp32 [vocab, channels]: row v is ``scale *`` the sum of dy's rows whose token is v.  accumulate: added to
    ``out``, whose other rows stay as they are.  tokens: int32, contiguous; dy: tokens' shape + [channels], or [tokens.numel(), channels] with rows apart."""
    _dense("tokens", tokens, _I32, None, None)
    dev = tokens.device
    if isinstance(dy, torch.Tensor) and dy.dim() != 2:
        if dy.dim() == 0 or dy.shape[:-1] != tokens.shape or not dy.is_contiguous():
            _refuse("dy must be contiguous, of tokens' shape and the channels")
        dy = dy.view(tokens.numel(), dy.shape[-1])
    stride = _rows("dy", dy, None, 2, None, dev)
    n, c = dy.shape
    if tokens.numel() != n:
        _refuse(f"dy must have a row for each of the {tokens.numel()} tokens, not {n}")
    need = _bytes("fdg_embedding_workspace", n, vocab, c)
    if out is None:
        if accumulate:
            _refuse("accumulate needs the gradient to add to")
        out = dy.new_empty((vocab, c), dtype=_F32)
    else:
        _dense("out", out, _F32, (vocab, c), dev)
    ws = dy.new_empty(need, dtype=_U8) if need else None
    _call(dev, "fdg_embedding_backward", _addr(tokens), n, _addr(dy), _DTYPE[dy.dtype], stride, vocab, c, scale, int(accumulate), _addr(out), _addr(ws), need)
    return out


def recurrence(gate: torch.Tensor, value: torch.Tensor, *, state: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None,
               for_grad: bool = False, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, ...]:
    """``h_t = a_t h_{t-1} + (1 - a_t) value_t`` with ``a = sigmoid(gate)``: (y, state after the last step) and, for_grad, what `recurrence_grad` needs.
    gate, value: [batch, steps, channels] fp32 or bf16, last dimension dense, other strides free; state: fp32 [batch, channels], zeros by default;
    lengths: int32 [batch], steps behind which do not count."""
    gs = _rows("gate", gate, None, 3, None, None)
    shape, dtype, dev = gate.shape, gate.dtype, gate.device
    vs = _rows("value", value, dtype, 3, shape, dev)
    b, n, c = shape
    if state is not None:
        _dense("state", state, _F32, (b, c), dev)
    if lengths is not None:
        _dense("lengths", lengths, _I32, (b,), dev)
    if out is None:
        out = gate.new_empty(shape)
        ys = max(n, 1) * c, c
    else:
        ys = _rows("out", out, dtype, 3, shape, dev)
    s = binding.fdg_recurrence(_DTYPE[dtype], b, n, c, *gs, *vs, *ys)
    last = gate.new_empty((b, c), dtype=_F32) if state is None else torch.empty_like(state)
    saved = gate.new_empty(_bytes("fdg_recurrence_saved", C.byref(s)), dtype=_U8) if for_grad else None
    _call(dev, "fdg_recurrence_forward", C.byref(s), _addr(gate), _addr(value), _addr(lengths), _addr(state), _addr(out), _addr(last), _addr(saved))
    return (out, last, saved) if for_grad else (out, last)


def recurrence_grad(gate: torch.Tensor, value: torch.Tensor, dy: torch.Tensor, saved: torch.Tensor, *, dgate: torch.Tensor, dvalue: torch.Tensor,
                    dstate: Optional[torch.Tensor] = None, lengths: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Gradients of `recurrence` for dy and, optionally, dstate (of the state after the last step): written to dgate and dvalue (tensors like
    gate and value, strides of their own; halves of one tensor, say); the gradient of the initial state is returned.  gate, value, lengths: those of the forward call."""
    gs = _rows("gate", gate, None, 3, None, None)
    shape, dtype, dev = gate.shape, gate.dtype, gate.device
    b, n, c = shape
    s = binding.fdg_recurrence(_DTYPE[dtype], b, n, c, *gs, *_rows("value", value, dtype, 3, shape, dev), 0, 0, *_rows("dy", dy, dtype, 3, shape, dev),
                               *_rows("dgate", dgate, dtype, 3, shape, dev), *_rows("dvalue", dvalue, dtype, 3, shape, dev))
    if dstate is not None:
        _dense("dstate", dstate, _F32, (b, c), dev)
    if lengths is not None:
        _dense("lengths", lengths, _I32, (b,), dev)
    _dense("saved", saved, _U8, None, dev)
    need = _bytes("fdg_recurrence_saved", C.byref(s))
    if saved.numel() != need:
        _refuse(f"saved must have {need} bytes (those of the forward call of this shape), not {saved.numel()}")
    first = gate.new_empty((b, c), dtype=_F32)
    _call(dev, "fdg_recurrence_backward", C.byref(s), _addr(gate), _addr(value), _addr(lengths), _addr(saved), _addr(dy), _addr(dstate), _addr(dgate), _addr(dvalue),
          _addr(first))
    return first


def distill_loss(logits: torch.Tensor, labels: Optional[torch.Tensor], ids: torch.Tensor, teacher: torch.Tensor, *, temperature: float = 1.0, weight: float = 1.0,
                 scale: float = 1.0, grad: bool = True, out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(loss of every row, gradient for the logits times `scale`): ``weight * temperature^2 * KL(teacher | student)`` over the teacher's top entries
    plus ``(1 - weight) *`` cross-entropy with the label.  logits: [rows, vocab] fp32 or bf16, rows may be apart; labels: int32 [rows] (a label
    outside the vocabulary takes its row out) or None with weight 1; ids int32, teacher fp32: [rows, top].  out: where the gradient goes (logits itself,
    or a bf16 tensor for fp32 logits); grad = False: the loss alone."""
    stride = _rows("logits", logits, None, 2, None, None)
    dev, dtype = logits.device, logits.dtype
    m, v = logits.shape
    _dense("ids", ids, _I32, None, dev)
    if ids.dim() != 2 or ids.shape[0] != m:
        _refuse(f"ids must have {m} rows of the teacher's entries, not {tuple(ids.shape)}")
    _dense("teacher", teacher, _F32, ids.shape, dev)
    if labels is not None:
        _dense("labels", labels, _I32, (m,), dev)
    to, ostride = _F32, 0
    if not grad:
        if out is not None:
            _refuse("out is for the gradient")
    elif out is None:
        out, to, ostride = logits.new_empty((m, v)), dtype, v
    else:
        ostride = _rows("out", out, None, 2, (m, v), dev)
        to = out.dtype
    loss = logits.new_empty(m, dtype=_F32)
    d = binding.fdg_distill(_DTYPE[dtype], _DTYPE[to], ids.shape[1], m, v, stride, ostride, temperature, weight, scale)
    _call(dev, "fdg_distill_loss", C.byref(d), _addr(logits), _addr(labels), _addr(ids), _addr(teacher), _addr(loss), _addr(out))
    return loss, out

"""Python binding of libones' operators for a scheduled job's training step (include/ones_train.h): argument checks and
marshalling only.  The arithmetic runs in the library's HIP kernels; PyTorch supplies the tensors and the stream (the current one
of the tensors' device).  There is no CPU fallback: without the built library or without a GPU this raises.

The ``*_forward`` and ``*_backward`` functions are the library's calls; ``layer_norm``, ``gated_recurrence`` and
``linear_cross_entropy`` are the same under autograd.  ``gated_recurrence_step`` is the single-token form,
``orthogonal_update`` the optimizer's step.

All of them may be captured into a graph.  Autograd's own rule stays: a backward pass under capture must not meet leaves that an eager
graph still holds; the ``*_backward`` calls know no such state."""
from __future__ import annotations

import ctypes as C

import torch

from . import ones
from .ones import OnesError  # noqa: F401

EXPORTS = ["ones_layer_norm_forward", "ones_layer_norm_workspace_bytes", "ones_layer_norm_backward",
           "ones_recurrence_carry_bytes", "ones_recurrence_workspace_bytes", "ones_recurrence_forward",
           "ones_recurrence_backward", "ones_recurrence_step", "ones_cross_entropy_forward_workspace_bytes",
           "ones_cross_entropy_backward_workspace_bytes", "ones_cross_entropy_forward", "ones_cross_entropy_backward",
           "ones_orthogonal_update_workspace_bytes", "ones_orthogonal_update"]

_P, _I64, _I32, _F32, _SIZE = C.c_void_p, C.c_int64, C.c_int32, C.c_float, C.c_size_t
_ARGUMENTS = {
    "ones_layer_norm_forward": [_P, _I64, _I64, _I64, _I32, _P, _P, _I32, _F32, _P, _P, _P, _P],
    "ones_layer_norm_workspace_bytes": [_I64, _I64],
    "ones_layer_norm_backward": [_P, _I64, _P, _I64, _I64, _I64, _I32, _P, _I32, _P, _P, _P, _P, _P, _P, _SIZE, _P],
    "ones_recurrence_carry_bytes": [_I64, _I64, _I64],
    "ones_recurrence_workspace_bytes": [_I64, _I64, _I64],
    "ones_recurrence_forward": [_P, _I64, _I64, _P, _I64, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _P, _P, _SIZE, _P],
    "ones_recurrence_backward": [_P, _I64, _I64, _P, _P, _I64, _I64, _P, _I64, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _P,
                                 _P, _SIZE, _P],
    "ones_recurrence_step": [_P, _I64, _P, _I64, _I64, _I64, _I32, _P, _P, _P],
    "ones_cross_entropy_forward_workspace_bytes": [_I64, _I64, _I64, _I32],
    "ones_cross_entropy_backward_workspace_bytes": [_I64, _I64, _I64, _I32],
    "ones_cross_entropy_forward": [_P, _I64, _P, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _SIZE, _P],
    "ones_cross_entropy_backward": [_P, _P, _I64, _P, _I64, _I64, _I64, _I64, _I32, _P, _P, _P, _P, _P, _SIZE, _P],
    "ones_orthogonal_update_workspace_bytes": [_I64, _I64, _I64],
    "ones_orthogonal_update": [_P, _P, _I64, _I64, _I64, _I32, _F32, _I32, _I32, _P, _F32, _P, _I32, _P, _SIZE, _P],
}
_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_FLOAT = (torch.float32,)
_lib = None
# current_device() and current_stream(device).cuda_stream, without what these do around it: 3 us of a call's 15
_device, _stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def load():
    """The library with the argument types of these functions; raises if it has not been built."""
    global _lib
    if _lib is None:
        L = ones.load()
        for name, arguments in _ARGUMENTS.items():
            f = getattr(L, name)
            f.argtypes = arguments
            f.restype = _SIZE if name.endswith("_bytes") else C.c_int
        _lib = L
    return _lib


def _call(device, function, *args):
    """A call of the library with the tensors' device current (it mostly is already), on its current stream."""
    stream = _stream(device.index)
    if _device() == device.index:
        rc = function(*args, stream)
    else:
        with torch.cuda.device(device):
            rc = function(*args, stream)
    if rc:
        raise OnesError(rc, _lib.ones_strerror(rc).decode())


def _check(t, name, shape, types, device=None):
    if isinstance(t, torch.Tensor) and t.dtype in types and t.is_cuda and (shape is None or t.shape == shape) and (device is None or t.device == device):
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name}: a tensor is wanted")
    if t.dtype not in types:
        raise TypeError(f"{name}: {t.dtype} is not one of {', '.join(str(d) for d in types)}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: shape {tuple(t.shape)}, wanted {tuple(shape)}")
    if device is not None and t.device != device:
        raise ValueError(f"{name}: on {t.device}, the others on {device}")
    if not t.is_cuda:
        raise OnesError(-101, f"{name}: on {t.device}; libones has no CPU path")


def _dense(t, name, shape, types, device):
    """Checked, without gaps (copied if it has any), None stays None."""
    if t is None:
        return None
    _check(t, name, shape, types, device)
    return t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _like(t):
    """A new tensor like t without gaps."""
    return torch.empty_like(t, memory_format=torch.contiguous_format)


# what autograd has to know of a tensor that a call has written in place: a backward pass that saved it raises then
_changed = torch.autograd.graph.increment_version


def _scratch(nbytes, device):
    """Workspace of one call from torch's allocator, whose blocks are 512-byte aligned and reused in stream order."""
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _rows(t):
    """(t as rows of one dimension, elements between two of them); copied where it cannot be seen as such."""
    d = t.shape[-1]
    if t.dim() == 2 and (t.stride(1) == 1 or d == 1) and t.stride(0) >= d:
        return t, t.stride(0)
    t = t.contiguous()
    return t.view(-1, d) if d else t.reshape(-1, d), d


# ------------------------------------------------------------------ layer norm --------
def _norm_weights(weight, bias, x):
    kinds = (torch.float32, x.dtype)
    shape = x.shape[-1:]
    weight, bias = _dense(weight, "weight", shape, kinds, x.device), _dense(bias, "bias", shape, kinds, x.device)
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise TypeError("weight and bias: one type for both")
    return weight, bias, weight.dtype if weight is not None else bias.dtype if bias is not None else torch.float32


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5):
    """ones_layer_norm_forward over the last dimension: (y, mean, rstd), the latter float32 without that dimension."""
    _check(x, "x", None, _TYPES)
    if x.dim() < 1:
        raise ValueError("x: at least one dimension is wanted")
    weight, bias, kind = _norm_weights(weight, bias, x)
    device, (rows, stride) = x.device, _rows(x)
    y = _like(x)
    mean, rstd = torch.empty((2, *x.shape[:-1]), dtype=torch.float32, device=device).unbind(0)
    n, d = rows.shape
    _call(device, load().ones_layer_norm_forward, rows.data_ptr(), stride, n, d, _TYPES[x.dtype], _ptr(weight), _ptr(bias),
          _TYPES[kind], eps, y.data_ptr(), mean.data_ptr(), rstd.data_ptr())
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, want_bias=True):
    """ones_layer_norm_backward: (dx, dweight, dbias).  dweight has the weight's type (float32 without one); dbias is None if
    not wanted."""
    _check(x, "x", None, _TYPES)
    device = x.device
    _check(dy, "dy", x.shape, (x.dtype,), device)
    weight, _, kind = _norm_weights(weight, None, x)
    lead = x.shape[:-1]
    mean, rstd = _dense(mean, "mean", lead, _FLOAT, device), _dense(rstd, "rstd", lead, _FLOAT, device)
    (rows, stride), (grad, grad_stride) = _rows(x), _rows(dy)
    n, d = rows.shape
    dx = _like(x)
    dweight = torch.empty(d, dtype=kind, device=device) if weight is None else torch.empty_like(weight)
    dbias = torch.empty_like(dweight) if want_bias else None
    L = load()
    nbytes = L.ones_layer_norm_workspace_bytes(n, d)
    scratch = _scratch(nbytes, device)
    _call(device, L.ones_layer_norm_backward, grad.data_ptr(), grad_stride, rows.data_ptr(), stride, n, d, _TYPES[x.dtype],
          _ptr(weight), _TYPES[kind], mean.data_ptr(), rstd.data_ptr(), dx.data_ptr(), dweight.data_ptr(), _ptr(dbias),
          _ptr(scratch), nbytes)
    return dx, dweight, dbias


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.kinds = (weight is not None, bias.dtype if bias is not None else None)
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dweight, dbias = layer_norm_backward(dy, x, weight, mean, rstd, ctx.kinds[1] is not None)
        return dx, dweight if ctx.kinds[0] else None, dbias if dbias is None else dbias.to(ctx.kinds[1]), None


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension, differentiable in x, weight and bias."""
    return _LayerNorm.apply(x, weight, bias, eps)


# ------------------------------------------------------- gated recurrence --------
def _steps(t):
    """(t, elements between sequences, elements between steps); copied if its channels do not lie one after another."""
    if (t.stride(2) != 1 and t.shape[2] > 1) or min(t.stride()) < 0:
        t = t.contiguous()
    return t, t.stride(0), t.stride(1)


def _recurrence_inputs(gate, x, lengths):
    _check(x, "x", None, _TYPES)
    if x.dim() != 3:
        raise ValueError(f"x: [batch, steps, channels] is wanted, got {tuple(x.shape)}")
    _check(gate, "gate", x.shape, (x.dtype,), x.device)
    return _dense(lengths, "lengths", x.shape[:1], (torch.int32,), x.device)


def gated_recurrence_forward(gate, x, state=None, lengths=None):
    """ones_recurrence_forward over x [batch, steps, channels]: (h, last, carry).  state, last: float32 [batch, channels];
    lengths: int32 [batch]; carry is what the backward call takes."""
    lengths = _recurrence_inputs(gate, x, lengths)
    b, t, c = x.shape
    state = _dense(state, "state", (b, c), (torch.float32,), x.device)
    (g, gb, gs), (u, ub, us) = _steps(gate), _steps(x)
    L = load()
    h = torch.empty((b, t, c), dtype=x.dtype, device=x.device)
    last = torch.empty((b, c), dtype=torch.float32, device=x.device)
    carry = torch.empty(L.ones_recurrence_carry_bytes(b, t, c) // 4, dtype=torch.float32, device=x.device)
    nbytes = L.ones_recurrence_workspace_bytes(b, t, c)
    scratch = _scratch(nbytes, x.device)
    _call(x.device, L.ones_recurrence_forward, g.data_ptr(), gb, gs, u.data_ptr(), ub, us, b, t, c, _TYPES[x.dtype], _ptr(state),
          _ptr(lengths), h.data_ptr(), last.data_ptr(), carry.data_ptr(), _ptr(scratch), nbytes)
    return h, last, carry


def gated_recurrence_backward(dh, dlast, gate, x, carry, lengths=None):
    """ones_recurrence_backward: (dgate, dx, dstate).  dlast (of the last state, float32) may be None."""
    lengths = _recurrence_inputs(gate, x, lengths)
    b, t, c = x.shape
    _check(dh, "dh", x.shape, (x.dtype,), x.device)
    dlast = _dense(dlast, "dlast", (b, c), (torch.float32,), x.device)
    L = load()
    carry = _dense(carry, "carry", (L.ones_recurrence_carry_bytes(b, t, c) // 4,), (torch.float32,), x.device)
    (g, gb, gs), (u, ub, us), (d, db, ds) = _steps(gate), _steps(x), _steps(dh)
    dgate, dx = (torch.empty((b, t, c), dtype=x.dtype, device=x.device) for _ in range(2))
    dstate = torch.empty((b, c), dtype=torch.float32, device=x.device)
    nbytes = L.ones_recurrence_workspace_bytes(b, t, c)
    scratch = _scratch(nbytes, x.device)
    _call(x.device, L.ones_recurrence_backward, d.data_ptr(), db, ds, _ptr(dlast), g.data_ptr(), gb, gs, u.data_ptr(), ub, us, b, t, c,
          _TYPES[x.dtype], carry.data_ptr(), _ptr(lengths), dgate.data_ptr(), dx.data_ptr(), dstate.data_ptr(), _ptr(scratch), nbytes)
    return dgate, dx, dstate


def gated_recurrence_step(gate, x, state):
    """ones_recurrence_step: one step of every sequence.  gate, x [batch, channels] or [batch, 1, channels]; state (float32
    [batch, channels], without gaps) is updated in place; returns h shaped like x."""
    _check(x, "x", None, _TYPES)
    if x.dim() not in (2, 3) or (x.dim() == 3 and x.shape[1] != 1):
        raise ValueError(f"x: [batch, channels] or [batch, 1, channels] is wanted, got {tuple(x.shape)}")
    _check(gate, "gate", x.shape, (x.dtype,), x.device)
    b, c = x.shape[0], x.shape[-1]
    _check(state, "state", (b, c), (torch.float32,), x.device)
    if not state.is_contiguous():
        raise ValueError("state: updated in place, it may have no gaps")
    if c > 1 and (gate.stride(-1) != 1 or gate.stride(0) < 0):
        gate = gate.contiguous()
    if c > 1 and (x.stride(-1) != 1 or x.stride(0) < 0):
        x = x.contiguous()
    h = _like(x)
    _call(x.device, load().ones_recurrence_step, gate.data_ptr(), gate.stride(0), x.data_ptr(), x.stride(0), b, c, _TYPES[x.dtype],
          state.data_ptr(), h.data_ptr())
    _changed(state)
    return h


class _GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, state, lengths):
        h, last, carry = gated_recurrence_forward(gate, x, state, lengths)
        ctx.save_for_backward(gate, x, carry, lengths)
        ctx.set_materialize_grads(False)
        return h, last

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dlast):
        gate, x, carry, lengths = ctx.saved_tensors
        if dh is None:
            dh = torch.zeros((), dtype=x.dtype, device=x.device).expand(x.shape)
        dgate, dx, dstate = gated_recurrence_backward(dh, dlast, gate, x, carry, lengths)
        return dgate, dx, dstate if ctx.needs_input_grad[2] else None, None


def gated_recurrence(gate, x, state=None, lengths=None):
    """h_t = a_t h_{t-1} + (1 - a_t) x_t with a = sigmoid(gate) over the steps of x [batch, steps, channels], differentiable in
    gate, x and state: (h, last)."""
    return _GatedRecurrence.apply(gate, x, state, lengths)


# ------------------------------------------- cross entropy over a vocabulary --------
_HALVES = (torch.bfloat16, torch.float16)
_WHOLE = (torch.int64, torch.int32)


def _loss_inputs(x, weight, target):
    _check(x, "x", None, _HALVES)
    device = x.device
    _check(weight, "weight", None, (x.dtype,), device)
    if x.dim() != 2 or weight.dim() != 2 or x.shape[1] != weight.shape[1]:
        raise ValueError(f"x [rows, cols] and weight [vocabulary, cols] are wanted, got {tuple(x.shape)} and {tuple(weight.shape)}")
    _check(target, "target", x.shape[:1], _WHOLE, device)
    if target.dtype != torch.int64:
        target = target.long()
    (x, x_stride), (weight, w_stride) = _rows(x), _rows(weight)
    n, d = x.shape
    x_at, w_at = x.data_ptr(), weight.data_ptr()
    wide = not ((d | x_stride | w_stride) % 8 or (x_at | w_at) % 16 or max(x_stride, w_stride) > 1 << 20)
    return device, (x_at, x_stride, w_at, w_stride, n, d, weight.shape[0]), wide, (x, weight, target.contiguous())


def linear_cross_entropy_forward(x, weight, target):
    """ones_cross_entropy_forward: (loss, lse), float32 per row of x [rows, cols], for logits x weight^T over weight
    [vocabulary, cols].  Rows with a target below 0 have no loss."""
    device, operands, wide, (x, weight, target) = _loss_inputs(x, weight, target)
    n, d, v = operands[4:]
    L = load()
    # two tensors, not views of one: the caller may change the loss in place while lse is kept for the backward call
    loss, lse = (torch.empty(n, dtype=torch.float32, device=device) for _ in range(2))
    nbytes = L.ones_cross_entropy_forward_workspace_bytes(n, d, v, wide)
    scratch = _scratch(nbytes, device)
    _call(device, L.ones_cross_entropy_forward, *operands, _TYPES[x.dtype], target.data_ptr(), loss.data_ptr(), lse.data_ptr(),
          _ptr(scratch), nbytes)
    return loss, lse


def linear_cross_entropy_backward(dloss, x, weight, target, lse):
    """ones_cross_entropy_backward: (dx, dweight) for the gradient dloss (float32) of every row's loss."""
    device, operands, wide, (x, weight, target) = _loss_inputs(x, weight, target)
    n, d, v = operands[4:]
    dloss, lse = _dense(dloss, "dloss", x.shape[:1], _FLOAT, device), _dense(lse, "lse", x.shape[:1], _FLOAT, device)
    L = load()
    dx, dweight = _like(x), _like(weight)
    nbytes = L.ones_cross_entropy_backward_workspace_bytes(n, d, v, wide)
    scratch = _scratch(nbytes, device)
    _call(device, L.ones_cross_entropy_backward, dloss.data_ptr(), *operands, _TYPES[x.dtype], target.data_ptr(), lse.data_ptr(),
          dx.data_ptr(), dweight.data_ptr(), _ptr(scratch), nbytes)
    return dx, dweight


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, target):
        loss, lse = linear_cross_entropy_forward(x, weight, target)
        ctx.save_for_backward(x, weight, target, lse)
        return loss

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss):
        return *linear_cross_entropy_backward(dloss, *ctx.saved_tensors), None


def linear_cross_entropy(x, weight, target):
    """The loss of every row under autograd: the mean over the rows that count is ``loss.sum() / (target >= 0).sum()``."""
    return _LinearCrossEntropy.apply(x, weight, target)


# --------------------------------------------------- orthogonalised update --------
COEFFICIENTS = (3.4445, -4.7750, 2.0315)      # singular values from 0.01 to 1 end between 0.7 and 1.2 after five steps


def orthogonal_update(grad, momentum=None, beta=0.95, nesterov=True, steps=5, coefficients=COEFFICIENTS, eps=1e-7, dtype=None):
    """ones_orthogonal_update: the update for weights whose gradient is grad [rows, cols] or [count, rows, cols], all matrices of
    one call together.  momentum (float32, shaped like grad, without gaps) is updated in place; without one grad itself is
    orthogonalised.  dtype: of the result, bfloat16 or float16 (default: grad's, bfloat16 for float32); a float16 result is right to its own
    rounding and takes up to 2.6 times as long, a bfloat16 one is off by 1.4 times its own rounding."""
    _check(grad, "grad", None, _TYPES)
    if grad.dim() not in (2, 3):
        raise ValueError(f"grad: [rows, cols] or [count, rows, cols] is wanted, got {tuple(grad.shape)}")
    if momentum is not None:
        _check(momentum, "momentum", grad.shape, (torch.float32,), grad.device)
        if not momentum.is_contiguous():
            raise ValueError("momentum: updated in place, it may have no gaps")
    dtype = dtype or (grad.dtype if grad.dtype in _HALVES else torch.bfloat16)
    if dtype not in _HALVES:
        raise TypeError(f"dtype: {dtype} is not bfloat16 or float16")
    if len(coefficients) != 3:
        raise ValueError("coefficients: three numbers are wanted")
    grad = grad.contiguous()
    count, (m, n) = (1 if grad.dim() == 2 else grad.shape[0]), grad.shape[-2:]
    update = torch.empty(grad.shape, dtype=dtype, device=grad.device)
    L = load()
    nbytes = L.ones_orthogonal_update_workspace_bytes(count, m, n)
    scratch = _scratch(nbytes, grad.device)
    _call(grad.device, L.ones_orthogonal_update, grad.data_ptr(), _ptr(momentum), count, m, n, _TYPES[grad.dtype], beta, int(nesterov),
          steps, (C.c_float * 3)(*coefficients), eps, update.data_ptr(), _TYPES[dtype], _ptr(scratch), nbytes)
    if momentum is not None:
        _changed(momentum)
    return update

"""ctypes binding of libflowpool's training operators (include/flowpool_train.h). Argument marshalling only.

Every function has the name of the C entry point it calls, takes torch tensors
(inputs, outputs and workspaces are the caller's; the library allocates
nothing) and checks what a kernel could not: shapes, types, devices and
strides. Streams are given as in ``paper_2606_23087_amd.flowpool``: a torch
stream, a raw hipStream_t, or None for torch's current stream. As there, a
tensor that another stream still uses has to be kept alive and ordered by the
caller. The tensors have to be on the current device. A non-OK status raises
``FlowPoolError``.

    workspace = torch.empty(vocab_loss_workspace(rows, hidden, vocab), dtype=torch.uint8, device="cuda")
    vocab_loss_forward(x, weight, labels, loss, lse, None, workspace)
    vocab_loss_backward(x, weight, labels, lse, None, dx, dweight, workspace)
"""

from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence

import torch

from .flowpool import FP_EINVAL, FlowPoolError, _check, _lib, _stream  # noqa: F401  (FlowPoolError: for callers)

FP_F32, FP_BF16, FP_F16 = 0, 1, 2
FP_LOSS_MEAN, FP_LOSS_SUM = 0, 1
FP_ADAMW_BLOCK = 256
TYPES = {torch.float32: FP_F32, torch.bfloat16: FP_BF16, torch.float16: FP_F16}
REDUCTIONS = {"mean": FP_LOSS_MEAN, "sum": FP_LOSS_SUM}


class fp_adamw_tensor(C.Structure):
    _fields_ = [("param", C.c_void_p), ("grad", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("copy", C.c_void_p),
                ("n", C.c_int64), ("weight_decay", C.c_float), ("reserved", C.c_int32)]


class fp_adamw_config(C.Structure):
    _fields_ = [("lr", C.c_double), ("beta1", C.c_double), ("beta2", C.c_double), ("eps", C.c_double),
                ("step", C.c_int64), ("param_type", C.c_int32), ("grad_type", C.c_int32),
                ("state_bits", C.c_int32), ("copy_type", C.c_int32)]


_P, _I32, _I64, _F32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
_SIGS = {
    "norm_forward": (_I32, [_P, _I64, _P, _P, _P, _I64, _P, _P, _I64, _I32, _F32, _I32, _I32, _P]),
    "norm_workspace": (_I64, [_I64, _I32]),
    "norm_backward": (_I32, [_P, _I64, _P, _I64, _P, _P, _P, _P, _I64, _P, _P, _I64, _I32, _I32, _I32, _I32, _P, _I64, _P]),
    "vocab_loss_workspace": (_I64, [_I64, _I32, _I32, _I32]),
    "vocab_loss_forward": (_I32, [_P, _I64, _P, _I64, _P, _I64, _I32, _I32, _I32, _I32, _P, _P, _P, _P, _I64, _P]),
    "vocab_loss_backward": (_I32, [_P, _I64, _P, _I64, _P, _P, _P, _I64, _I32, _I32, _I32, _I32, _P, _I64, _P, _I64, _I32, _I32,
                                   _P, _I64, _P]),
    "adamw_step": (_I32, [C.POINTER(fp_adamw_tensor), _I32, C.POINTER(fp_adamw_config), _P, _P]),
    "adamw_table_bytes": (_I64, [_I32]),
    "adamw_table_write": (_I32, [C.POINTER(fp_adamw_tensor), _I32, C.POINTER(fp_adamw_config), _P, _I64, C.POINTER(_I64), _P]),
    "adamw_table_step": (_I32, [_P, _I64, C.POINTER(fp_adamw_config), _P, _P]),
    "adamw_state_values": (_I32, [_P, _P, _P, _I64, _I32, _P]),
}
for _name, (_res, _args) in _SIGS.items():
    _f = getattr(_lib, _name)
    _f.restype = _res
    _f.argtypes = _args

EXPORTED = tuple(_SIGS)


# ------------------------------------------------------------------ checks

def _device(x: torch.Tensor, name: str):
    if not x.is_cuda:
        raise ValueError(f"{name} must be on the GPU")
    return x.device


def _on(x: torch.Tensor, name: str, device) -> None:
    if x.device != device:
        raise ValueError(f"{name} is on {x.device}, the call's other tensors on {device}")


def _queue(stream, device):
    """The stream of a call on tensors of `device`, which has to be the current one: the library launches there."""
    here = torch._C._cuda_getDevice()
    if device.index != here:
        raise ValueError(f"the tensors are on {device}, the current device is {here}")
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(here)
    if isinstance(stream, torch.cuda.Stream) and stream.device != device:
        raise ValueError(f"stream is of {stream.device}, the tensors are on {device}")
    return _stream(stream)


def _matrix(x: torch.Tensor, name: str, device, dtype=None, shape=None) -> int:
    """Row stride of a [rows, columns] tensor whose rows are contiguous."""
    _on(x, name, device)
    if x.dim() != 2:
        raise ValueError(f"{name} must have 2 dimensions, has {x.dim()}")
    if dtype is not None and x.dtype != dtype:
        raise ValueError(f"{name} is {x.dtype}, must be {dtype}")
    if x.dtype not in TYPES:
        raise ValueError(f"{name} is {x.dtype}, must be one of {', '.join(map(str, TYPES))}")
    if shape is not None and tuple(x.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(x.shape)}, must have {tuple(shape)}")
    if x.shape[1] > 1 and x.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if x.shape[0] < 2:              # the stride of a dimension of one element says nothing
        return _round_up(x.shape[1], 16 // x.element_size())
    if x.stride(0) < x.shape[1]:
        raise ValueError(f"{name} has overlapping rows")
    return x.stride(0)


def _round_up(n: int, to: int) -> int:
    return -(-n // to) * to


def _vector(x: Optional[torch.Tensor], name: str, device, dtypes, n: int) -> Optional[int]:
    if x is None:
        return None
    _on(x, name, device)
    if x.dtype not in dtypes:
        raise ValueError(f"{name} is {x.dtype}, must be {' or '.join(map(str, dtypes))}")
    if x.numel() != n or not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {n} elements")
    return x.data_ptr()


def _room(x: Optional[torch.Tensor], device):
    """Address and bytes of a workspace."""
    if x is None:
        return None, 0
    _on(x, "workspace", device)
    if not x.is_contiguous():
        raise ValueError("workspace must be contiguous")
    return x.data_ptr(), x.nbytes


def _bytes(n: int, where: str) -> int:
    if n < 0:
        _check(int(n), where)
    return int(n)


def _weights(weight, bias, device, dtype, hidden):
    """Addresses of weight and bias, and their type."""
    given = [w for w in (weight, bias) if w is not None]
    wtype = given[0].dtype if given else dtype
    ok = (torch.float32,) if wtype == torch.float32 else (dtype,)
    return _vector(weight, "weight", device, ok, hidden), _vector(bias, "bias", device, ok, hidden), TYPES[ok[0]]


# ------------------------------------------------------------------ layer norm

def norm_forward(x, weight, bias, y, mean, rstd, eps: float = 1e-5, stream=None) -> None:
    """Layer norm of the rows of x into y; mean and rstd (f32, a value a row) are what norm_backward needs."""
    dev = _device(x, "x")
    xs = _matrix(x, "x", dev)
    rows, hidden = x.shape
    ys = _matrix(y, "y", dev, x.dtype, x.shape)
    w, b, wtype = _weights(weight, bias, dev, x.dtype, hidden)
    f32 = (torch.float32,)
    _check(_lib.norm_forward(x.data_ptr(), xs, w, b, y.data_ptr(), ys, _vector(mean, "mean", dev, f32, rows),
                             _vector(rstd, "rstd", dev, f32, rows), rows, hidden, eps, TYPES[x.dtype], wtype, _queue(stream, dev)),
           "norm_forward")


def norm_workspace(rows: int, hidden: int) -> int:
    """Bytes of workspace norm_backward needs."""
    return _bytes(_lib.norm_workspace(rows, hidden), "norm_workspace")


def norm_backward(dy, x, weight, mean, rstd, dx, dweight, dbias, workspace, accumulate: bool = False, stream=None) -> None:
    """Gradients of norm_forward: dx, and the f32 sums dweight and dbias (None: not computed), added to what they hold
    with ``accumulate``."""
    dev = _device(x, "x")
    xs = _matrix(x, "x", dev)
    rows, hidden = x.shape
    gs = _matrix(dy, "dy", dev, x.dtype, x.shape)
    ds = _matrix(dx, "dx", dev, x.dtype, x.shape)
    w, _, wtype = _weights(weight, None, dev, x.dtype, hidden)
    f32 = (torch.float32,)
    room, size = _room(workspace, dev)
    _check(_lib.norm_backward(dy.data_ptr(), gs, x.data_ptr(), xs, w, _vector(mean, "mean", dev, f32, rows),
                              _vector(rstd, "rstd", dev, f32, rows), dx.data_ptr(), ds, _vector(dweight, "dweight", dev, f32, hidden),
                              _vector(dbias, "dbias", dev, f32, hidden), rows, hidden, TYPES[x.dtype], wtype, int(accumulate),
                              room, size, _queue(stream, dev)), "norm_backward")


# ------------------------------------------------------------------ vocabulary loss

def vocab_loss_workspace(rows: int, hidden: int, vocab: int, backward: bool = True) -> int:
    """Bytes of workspace of vocab_loss_forward alone, or of either call."""
    return _bytes(_lib.vocab_loss_workspace(rows, hidden, vocab, int(backward)), "vocab_loss_workspace")


def _loss_operands(x, weight, labels, lse):
    dev = _device(x, "x")
    xs = _matrix(x, "x", dev)
    ws = _matrix(weight, "weight", dev, x.dtype)
    if weight.shape[1] != x.shape[1]:
        raise ValueError(f"weight has rows of {weight.shape[1]}, x of {x.shape[1]}")
    return (dev, x.data_ptr(), xs, weight.data_ptr(), ws, _vector(labels, "labels", dev, (torch.int32,), x.shape[0]),
            _vector(lse, "lse", dev, (torch.float32,), x.shape[0]))


def vocab_loss_forward(x, weight, labels, loss, lse, n_labelled, workspace, reduction: str = "mean", stream=None) -> None:
    """Softmax cross entropy of the labelled rows of x over the classes of weight. loss: f32 [1]; lse: f32, a value a
    row, for vocab_loss_backward; n_labelled: int32 [1] or None."""
    dev, xp, xs, wp, ws, lab, lsep = _loss_operands(x, weight, labels, lse)
    room, size = _room(workspace, dev)
    _check(_lib.vocab_loss_forward(xp, xs, wp, ws, lab, x.shape[0], x.shape[1], weight.shape[0], TYPES[x.dtype],
                                   REDUCTIONS[reduction], _vector(loss, "loss", dev, (torch.float32,), 1), lsep,
                                   _vector(n_labelled, "n_labelled", dev, (torch.int32,), 1), room, size, _queue(stream, dev)),
           "vocab_loss_forward")


def vocab_loss_backward(x, weight, labels, lse, dloss, dx, dweight, workspace, reduction: str = "mean",
                        accumulate: bool = False, stream=None) -> None:
    """Gradients of vocab_loss_forward (dx or dweight None: not computed). dloss: f32 [1], None = 1. With ``accumulate``
    dweight (f32) is added to."""
    dev, xp, xs, wp, ws, lab, lsep = _loss_operands(x, weight, labels, lse)
    dxs = _matrix(dx, "dx", dev, x.dtype, x.shape) if dx is not None else 0
    dws = 0
    if dweight is not None:
        dws = _matrix(dweight, "dweight", dev, None, weight.shape)
    room, size = _room(workspace, dev)
    _check(_lib.vocab_loss_backward(xp, xs, wp, ws, lab, lsep, _vector(dloss, "dloss", dev, (torch.float32,), 1), x.shape[0],
                                    x.shape[1], weight.shape[0], TYPES[x.dtype], REDUCTIONS[reduction],
                                    dx.data_ptr() if dx is not None else None, dxs,
                                    dweight.data_ptr() if dweight is not None else None, dws,
                                    TYPES[dweight.dtype] if dweight is not None else TYPES[x.dtype], int(accumulate), room, size,
                                    _queue(stream, dev)), "vocab_loss_backward")


# ------------------------------------------------------------------ AdamW

class AdamwTensors:
    """The tensors of an optimizer, checked and listed once (``adamw_tensors``): it keeps them alive, and their table on
    the GPU. It may be dropped while a step is queued, on any stream; a captured step needs it for as long as its graph is
    replayed."""

    def __init__(self, array, n, types, held, device):
        self.array, self.n, self.types, self._held = array, n, types, held
        self.table, self.groups, self._streams = None, 0, set()
        if device is not None:
            self.table = torch.empty(_bytes(_lib.adamw_table_bytes(n), "adamw_table_bytes"), dtype=torch.uint8, device=device)
            groups = C.c_int64()
            with torch.cuda.device(device):
                _check(_lib.adamw_table_write(array, n, C.byref(fp_adamw_config(0.0, 0.0, 0.0, 0.0, 1, *types)), self.table.data_ptr(),
                                              self.table.nbytes, C.byref(groups), _stream(None)), "adamw_table_write")
                torch.cuda.current_stream().synchronize()       # steps may run on any stream
            self.groups = groups.value
            self._streams.add(torch.cuda.current_stream(device).cuda_stream)

    def used_on(self, stream: int) -> None:
        """Tells the allocator that the step's stream uses what the step reads by address alone: a tensor that is freed goes
        to its own stream's next allocation, whatever another one still has queued."""
        if stream not in self._streams:
            device = self.table.device
            torch_stream = torch.cuda.ExternalStream(stream, device) if stream else torch.cuda.default_stream(device)
            for t in (self.table, *(t for group in self._held if group is not None for t in group)):
                t.record_stream(torch_stream)
            self._streams.add(stream)


def _one_type(tensors, name, allowed):
    kinds = {t.dtype for t in tensors}
    if len(kinds) > 1 or not kinds <= set(allowed):
        raise ValueError(f"{name} must all be one of {', '.join(map(str, allowed))}, are {', '.join(map(str, kinds))}")
    return next(iter(kinds)) if kinds else allowed[0]


def adamw_tensors(params: Sequence, grads: Sequence, m: Sequence, v: Sequence, scales: Optional[Sequence] = None,
                  copies: Optional[Sequence] = None, weight_decay=0.0) -> AdamwTensors:
    """The tensors of adamw_step, in place: parameters (f32 or bf16), gradients, states m and v (f32, or uint8 with
    ``scales``: for each tensor f32 [2, ceil(n / 256)], m's and v's), 16-bit copies of f32 parameters, and weight decay (one
    number, or one a tensor). All are contiguous. The list holds their addresses, and making it waits for the current stream
    (0.73 ms in all for 290 tensors): gradients are best zeroed in place, for ones that are allocated anew need a new list."""
    params, grads, m, v = list(params), list(grads), list(m), list(v)
    n = len(params)
    scales = None if scales is None else list(scales)
    copies = None if copies is None else list(copies)
    decay = [float(weight_decay)] * n if isinstance(weight_decay, (int, float)) else [float(d) for d in weight_decay]
    for name, l in (("grads", grads), ("m", m), ("v", v), ("scales", scales), ("copies", copies), ("weight_decay", decay)):
        if l is not None and len(l) != n:
            raise ValueError(f"{name} has {len(l)} entries, params {n}")
    f32, half = torch.float32, (torch.bfloat16, torch.float16)
    ptype = _one_type(params, "params", (f32, torch.bfloat16))
    gtype = _one_type(grads, "grads", (f32, *half))
    state = f32 if scales is None else torch.uint8
    ctype = None if copies is None else _one_type(copies, "copies", half)
    array = (fp_adamw_tensor * max(n, 1))()
    for i in range(n):
        dev, k = _device(params[i], "params"), params[i].numel()
        _on(params[i], f"params[{i}]", params[0].device)
        t = array[i]
        t.param = _vector(params[i], f"params[{i}]", dev, (ptype,), k)
        t.grad = _vector(grads[i], f"grads[{i}]", dev, (gtype,), k)
        t.m, t.v = _vector(m[i], f"m[{i}]", dev, (state,), k), _vector(v[i], f"v[{i}]", dev, (state,), k)
        if scales is not None:
            runs = -(-k // FP_ADAMW_BLOCK)
            if tuple(scales[i].shape) != (2, runs):
                raise ValueError(f"scales[{i}] has shape {tuple(scales[i].shape)}, must have (2, {runs})")
            t.m_scale, t.v_scale = (_vector(scales[i][j], f"scales[{i}]", dev, (f32,), runs) for j in (0, 1))
        if copies is not None:
            t.copy = _vector(copies[i], f"copies[{i}]", dev, (ctype,), k)
        t.n, t.weight_decay = k, decay[i]
    types = (TYPES[ptype], TYPES[gtype], 32 if scales is None else 8, -1 if ctype is None else TYPES[ctype])
    return AdamwTensors(array, n, types, (params, grads, m, v, scales, copies), params[0].device if n else None)


def adamw_step(tensors: AdamwTensors, step: int, lr: float, beta1: float = 0.9, beta2: float = 0.999, eps: float = 1e-8,
               grad_scale=None, stream=None) -> None:
    """One AdamW step, the ``step``-th (from 1). grad_scale: f32 [1] on the GPU, a factor of the gradients; a step whose
    grad_scale is not finite changes nothing."""
    scale = None
    if grad_scale is not None:
        scale = _vector(grad_scale, "grad_scale", _device(grad_scale, "grad_scale"), (torch.float32,), 1)
    config = fp_adamw_config(lr, beta1, beta2, eps, step, *tensors.types)
    if tensors.table is None:
        _check(_lib.adamw_step(tensors.array, tensors.n, C.byref(config), scale, _stream(stream)), "adamw_step")
    else:
        if grad_scale is not None:
            _on(grad_scale, "grad_scale", tensors.table.device)
        queue = _queue(stream, tensors.table.device)
        tensors.used_on(queue)
        _check(_lib.adamw_table_step(tensors.table.data_ptr(), tensors.groups, C.byref(config), scale, queue),
               "adamw_table_step")


def adamw_state_values(codes, scales, out, moment: int, stream=None) -> None:
    """The f32 values that an 8-bit state and its scales stand for (moment 1: m, 2: v), to save or inspect them."""
    dev = _device(codes, "codes")
    n = codes.numel()
    _check(_lib.adamw_state_values(_vector(codes, "codes", dev, (torch.uint8,), n),
                                   _vector(scales, "scales", dev, (torch.float32,), -(-n // FP_ADAMW_BLOCK)),
                                   _vector(out, "out", dev, (torch.float32,), n), n, moment, _queue(stream, dev)),
           "adamw_state_values")

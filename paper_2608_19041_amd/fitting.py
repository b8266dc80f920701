"""Operators that fit the energy MLP with weights of each element type.

Rows of atoms go through layers whose weights belong to the row's group (its
element type), the gradients of such a layer, and the Newton-Schulz update of
the weights (the Muon optimiser).  Argument marshalling only, as in the rest
of the binding: every step runs in the HIP kernels of the library, on the
caller's stream, and scratch comes from torch's allocator on that stream.
Nothing here is recorded by autograd: a layer's gradients come from
``grouped_linear_backward``, and tensors that autograd would have to follow are
refused (where it records, i.e. not under ``torch.no_grad()`` or within the
methods of a ``torch.autograd.Function``).

    ptr, order = group_rows(species, 118)
    y, z = grouped_linear(x, w, ptr, order, bias=b, activation="silu", preact=True)
    dx, dw, db = grouped_linear_backward(dy, x, w, ptr, order, preact=z)
    muon_step([w], [dw], [momentum], lr=0.02)
"""
from __future__ import annotations

import ctypes
import functools
import math

from . import _check, _ptr, _require, library

F32, F16, BF16 = 0, 1, 2
ACTIVATIONS = {None: 0, "silu": 1}
#: the quintic iteration of the Muon optimiser
MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)
MAX_STACKS = 32


class _Grouped(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int), ("n_groups", ctypes.c_int), ("k", ctypes.c_int),
                ("n_out", ctypes.c_int), ("n", ctypes.c_int64), ("group_ptr", ctypes.c_void_p),
                ("order", ctypes.c_void_p), ("x", ctypes.c_void_p), ("ldx", ctypes.c_int64),
                ("weight", ctypes.c_void_p)]


class _Stack(ctypes.Structure):
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("batch", ctypes.c_int64),
                ("rows", ctypes.c_int), ("cols", ctypes.c_int)]


class _Update(ctypes.Structure):
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("momentum_buf", ctypes.c_void_p), ("batch", ctypes.c_int64),
                ("rows", ctypes.c_int), ("cols", ctypes.c_int)]


class _Newton(ctypes.Structure):
    _fields_ = [("steps", ctypes.c_int), ("a", ctypes.c_float), ("b", ctypes.c_float),
                ("c", ctypes.c_float), ("eps", ctypes.c_float)]


@functools.lru_cache(maxsize=None)
def _codes():
    import torch
    return {torch.float32: F32, torch.float16: F16, torch.bfloat16: BF16}


def _int(v):
    """``v`` as the library takes it: beyond 32 bits the nearest, which it refuses."""
    v = int(v)
    return v if -2 ** 31 <= v < 2 ** 31 else (2 ** 31 - 1 if v > 0 else -2 ** 31)


def _dtype_code(t, name):
    import torch
    code = _codes().get(t.dtype) if isinstance(t, torch.Tensor) and t.is_cuda else None
    if code is None:
        raise ValueError(f"{name} must be a CUDA tensor of float32, float16 or bfloat16")
    return code


def _rows(t, dtype, shape, device, name):
    """A matrix of rows any distance apart; returns the distance in entries."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{name} must be a tensor of {dtype} on {device}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if shape[1] > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have unit stride within a row")
    ld = t.stride(0) if shape[0] > 1 else shape[1]
    if ld != 0 and ld < shape[1]:
        raise ValueError(f"the rows of {name} overlap")
    return ld


def _same(t, dtype, shape, device, name):
    _require(t, dtype, None, name)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}")


def _unrecorded(**tensors):
    """Refuses tensors whose gradients autograd would silently lose here."""
    import torch
    if torch.is_grad_enabled():
        for name, t in tensors.items():
            if t is not None and t.requires_grad:
                raise ValueError(f"{name} requires a gradient, which nothing here records: "
                                 "call under torch.no_grad() or detach it")


class _launch:
    """The stream's handle, with ``device`` current and torch's allocator on that stream.

    The common call, on the current device's current stream, only looks the handle up.
    """

    def __init__(self, device, stream):
        import torch
        self._guards = ()
        if stream is None and device.index == torch.cuda.current_device():
            self._handle = torch._C._cuda_getCurrentRawStream(device.index)
            return
        if stream is None:
            stream = torch.cuda.current_stream(device)
        elif stream.device != device:
            raise ValueError(f"the stream is of {stream.device}, the tensors are on {device}")
        self._guards = (torch.cuda.device(device), torch.cuda.stream(stream))
        self._handle = stream.cuda_stream

    def __enter__(self):
        for guard in self._guards:
            guard.__enter__()
        return self._handle

    def __exit__(self, *error):
        for guard in reversed(self._guards):
            guard.__exit__(*error)


def _scratch(device, *sizes_of):
    """(tensor or None, bytes) for calls that follow each other.

    Each of ``sizes_of`` writes a call's scratch to its argument, and refuses
    what the call would refuse by its sizes.
    """
    import torch
    most, need = 0, ctypes.c_int64(0)
    for size_of in sizes_of:
        _check(size_of(ctypes.byref(need)))
        most = max(most, need.value)
    return torch.empty(most, dtype=torch.uint8, device=device) if most else None, most


def group_rows(group, n_groups: int, stream=None):
    """(group_ptr int64 [n_groups + 1], order int32 [n]): the rows in group order.

    ``group``: int32 [n].  Rows keep their order within a group; rows whose id
    is outside [0, n_groups) belong to no group and come last.
    """
    import torch
    _require(group, torch.int32, None, "group")
    if group.dim() != 1:
        raise ValueError("group must have one dimension")
    n, n_groups, lib = group.shape[0], _int(n_groups), library()
    with _launch(group.device, stream) as st:
        work, size = _scratch(group.device,
                              lambda need: lib.dpa4c_group_rows_work(n, n_groups, need))
        ptr = torch.empty(n_groups + 1, dtype=torch.int64, device=group.device)
        order = torch.empty(n, dtype=torch.int32, device=group.device)
        _check(lib.dpa4c_group_rows(_ptr(group), n, n_groups, _ptr(ptr), _ptr(order), _ptr(work), size,
                                    st))
    return ptr, order


def _layer(x, weight, group_ptr, order):
    import torch
    code = _dtype_code(weight, "weight")
    if weight.dim() != 3 or not weight.is_contiguous():
        raise ValueError("weight must be contiguous with shape [groups, k, n]")
    groups, k, n_out = weight.shape
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be a matrix of rows")
    n = x.shape[0]
    ldx = _rows(x, weight.dtype, (n, k), weight.device, "x")
    _same(group_ptr, torch.int64, (groups + 1,), weight.device, "group_ptr")
    if order is not None:
        _same(order, torch.int32, (n,), weight.device, "order")
    return _Grouped(code, _int(groups), _int(k), _int(n_out), n, group_ptr.data_ptr(),
                    None if order is None else order.data_ptr(), x.data_ptr(), ldx,
                    weight.data_ptr())


def grouped_linear(x, weight, group_ptr, order=None, bias=None, activation=None, residual=False,
                   preact=False, stream=None):
    """y = act(x W_g + b_g) (+ x), with the weights of each row's group.

    x [n, k] (rows may be any distance apart), weight [groups, k, m], bias
    [groups, m] or None, all of one type (float32, float16, bfloat16);
    group_ptr and order as ``group_rows`` gives them (order None: the rows are
    in group order already).  ``activation``: None or "silu"; ``residual``
    adds x (k = m).  With ``preact`` returns (y, z), z the value before the
    activation.  Rows of no group give zeros.
    """
    import torch
    layer = _layer(x, weight, group_ptr, order)
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation must be one of {list(ACTIVATIONS)}")
    if residual and layer.k != layer.n_out:
        raise ValueError("a residual needs as many outputs as inputs")
    if bias is not None:
        _same(bias, weight.dtype, (layer.n_groups, layer.n_out), weight.device, "bias")
    _unrecorded(x=x, weight=weight, bias=bias)
    lib = library()
    with _launch(weight.device, stream) as st:
        work, size = _scratch(weight.device,
                              lambda need: lib.dpa4c_grouped_linear_work(ctypes.byref(layer), need))
        y = torch.empty(layer.n, layer.n_out, dtype=weight.dtype, device=weight.device)
        z = torch.empty_like(y) if preact else None
        _check(lib.dpa4c_grouped_linear(ctypes.byref(layer), _ptr(bias), ACTIVATIONS[activation],
                                        int(bool(residual)), _ptr(y), _ptr(z), _ptr(work), size,
                                        st))
    return (y, z) if preact else y


def grouped_linear_backward(dy, x, weight, group_ptr, order=None, preact=None, residual=False,
                            need=(True, True, True), stream=None):
    """(dx, dw, db) of ``grouped_linear`` from dy = dL/dy.

    ``preact``: z of the forward pass of a layer with SiLU; None: the layer had
    no activation.  ``need`` says which gradients to form; the others are None.
    """
    import torch
    layer = _layer(x, weight, group_ptr, order)
    n, m, dev = layer.n, layer.n_out, weight.device
    if residual and layer.k != m:
        raise ValueError("a residual needs as many outputs as inputs")
    ldy = _rows(dy, weight.dtype, (n, m), dev, "dy")
    ldz = 0 if preact is None else _rows(preact, weight.dtype, (n, m), dev, "preact")
    _unrecorded(dy=dy, x=x, weight=weight, preact=preact)
    lib = library()
    with _launch(dev, stream) as st:
        work, size = _scratch(dev, lambda size: lib.dpa4c_grouped_linear_backward_work_of(
            ctypes.byref(layer), preact is not None, *(bool(w) for w in need), size))
        dx = torch.empty(n, layer.k, dtype=weight.dtype, device=dev) if need[0] else None
        dw = torch.empty_like(weight) if need[1] else None
        db = torch.empty(layer.n_groups, m, dtype=weight.dtype, device=dev) if need[2] else None
        _check(lib.dpa4c_grouped_linear_backward(
            ctypes.byref(layer), _ptr(dy), ldy, _ptr(preact), ldz, int(bool(residual)), _ptr(dx),
            _ptr(dw), _ptr(db), _ptr(work), size, st))
    return dx, dw, db


def _stack_list(name, tensors):
    import torch
    if isinstance(tensors, torch.Tensor):
        raise ValueError(f"{name} must be a list of tensors")
    tensors = list(tensors)
    for t in tensors:
        _dtype_code(t, name)
        if t.dim() < 2 or not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous matrices or stacks of matrices")
        if t.dtype != tensors[0].dtype or t.device != tensors[0].device:
            raise ValueError(f"{name} must share one type and one device")
        shape = t.shape
        if shape[-1] < 1 or shape[-2] < 1:
            raise ValueError(f"{name} must not have empty matrices")
    return tensors


def _shape(t):
    """batch, rows, cols of a matrix or a stack of them"""
    *batch, rows, cols = t.shape
    return math.prod(batch), rows if rows < 2 ** 31 else _int(rows), cols if cols < 2 ** 31 else _int(cols)


def _pointers(tensors):
    """Where the tensors are; 0 for those without entries."""
    return [t.data_ptr() for t in tensors]


def _calls(struct, tensors, *pointers):
    """Tensors of these shapes at the matching pointers as arrays of ``struct``, MAX_STACKS at a time."""
    every = [struct(*at, *_shape(t)) for t, *at in zip(tensors, *pointers)]
    return [(struct * len(part))(*part)
            for part in (every[at:at + MAX_STACKS] for at in range(0, len(every), MAX_STACKS))]


def _newton(steps, coefficients, eps):
    a, b, c = (float(v) for v in coefficients)
    return _Newton(_int(steps), a, b, c, float(eps))


def orthogonalize(matrices, steps: int = 5, coefficients=MUON_COEFFICIENTS, eps: float = 1e-7,
                  stream=None):
    """Newton-Schulz orthogonalisation of every matrix; a list of results.

    ``matrices``: a list of contiguous matrices or stacks [..., rows, cols] of
    one type.  X = G / (|G| + eps), then ``steps`` times A = X X^T,
    X <- a X + (b A + c A A) X, on the shorter side.
    """
    import torch
    matrices = _stack_list("matrices", matrices)
    if not matrices:
        return []
    for t in matrices:
        _unrecorded(matrices=t)
    how, lib, dev = _newton(steps, coefficients, eps), library(), matrices[0].device
    code = _dtype_code(matrices[0], "matrices")
    with _launch(dev, stream) as st:
        out = [torch.empty_like(t) for t in matrices]
        calls = _calls(_Stack, matrices, _pointers(matrices), _pointers(out))
        work, size = _scratch(dev, *(
            functools.partial(lib.dpa4c_orthogonalize_work, len(c), c) for c in calls))
        for c in calls:
            _check(lib.dpa4c_orthogonalize(code, len(c), c, ctypes.byref(how), _ptr(work), size, st))
    return out


def muon_step(params, grads, momenta, lr: float, momentum: float = 0.95, nesterov: bool = True,
              weight_decay: float = 0.0, steps: int = 5, coefficients=MUON_COEFFICIENTS,
              eps: float = 1e-7, stream=None):
    """One Muon update of every weight matrix, in place.

    M <- momentum M + G; U = G + momentum M (``nesterov``) or M;
    W <- (1 - lr weight_decay) W - lr sqrt(max(1, cols / rows)) NS(U).
    ``params``, ``grads``: lists of contiguous matrices or stacks of one type;
    ``momenta``: float32 tensors of the same shapes; each tensor once.  As an optimiser's step does,
    this writes parameters that require a gradient; autograd notices the write.
    """
    import torch
    params, grads, momenta = _stack_list("params", params), list(grads), list(momenta)
    if not len(params) == len(grads) == len(momenta):
        raise ValueError("params, grads and momenta must have the same length")
    if not params:
        return
    dev = params[0].device
    for w, g, m in zip(params, grads, momenta):
        _same(g, w.dtype, w.shape, dev, "grads")
        _same(m, torch.float32, w.shape, dev, "momenta")
    # all matrices are updated together: one listed twice would be written by both
    at_w, at_g, at_m = (_pointers(ts) for ts in (params, grads, momenta))
    written = [p for p in at_w + at_m if p]
    if len(set(written)) < len(written) or not set(at_m).isdisjoint(filter(None, at_g)):
        raise ValueError("params and momenta must not share memory with each other, nor momenta with grads")
    how, lib, code = _newton(steps, coefficients, eps), library(), _dtype_code(params[0], "params")
    with _launch(dev, stream) as st:
        # the sizes of all calls are checked before the first changes a weight
        calls = _calls(_Update, params, at_w, at_g, at_m)
        work, size = _scratch(dev, *(
            functools.partial(lib.dpa4c_muon_step_work, len(c), c) for c in calls))
        torch.autograd.graph.increment_version(params + momenta)
        for c in calls:
            _check(lib.dpa4c_muon_step(code, len(c), c, ctypes.byref(how), float(lr),
                                       float(momentum), int(bool(nesterov)), float(weight_decay),
                                       _ptr(work), size, st))

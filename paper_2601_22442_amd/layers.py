"""The layers that own a stage's parameters, and the gradient norm over many tensors (include/asyncmesh.h).

Argument checks and marshalling only, as in the binding of the stage.  Every call takes the R replicas in one go, as lists
of R tensors: weights are usually views into `Stage.fwd[i]`, gradients views into the flat arrays that `Stage.step` reads.
Work is enqueued on the current stream; outputs and workspaces come from PyTorch's allocator on that stream.
"""
from __future__ import annotations

import ctypes as C

import torch

from .binding import BF16, F32, MAX_REPLICAS, _check, _on, lib

ACT_NONE, ACT_RELU, ACT_GELU, ACT_GELU_TANH, ACT_SILU = range(5)
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}


class LinearConfig(C.Structure):
    """Mirror of am_linear_config."""
    _fields_ = [("replicas", C.c_uint32), ("dtype", C.c_uint32), ("grad_dtype", C.c_uint32), ("act", C.c_uint32),
                ("rows", C.c_uint64), ("in_", C.c_uint64), ("out", C.c_uint64),
                ("x_stride", C.c_uint64), ("y_stride", C.c_uint64), ("pre_stride", C.c_uint64), ("residual_stride", C.c_uint64),
                ("dx_stride", C.c_uint64)]


class LinearBuffers(C.Structure):
    """Mirror of am_linear_buffers."""
    _fields_ = [(name, C.c_void_p) for name in ("x", "w", "bias", "residual", "y", "pre", "dy", "dx", "dw", "db", "workspace")] + \
               [("workspace_bytes", C.c_uint64)]


lib.am_linear_workspace.argtypes = [C.POINTER(LinearConfig), C.POINTER(LinearBuffers), C.c_int, C.POINTER(C.c_uint64)]
lib.am_linear.argtypes = [C.POINTER(LinearConfig), C.POINTER(LinearBuffers), C.c_void_p]
lib.am_linear_backward.argtypes = [C.POINTER(LinearConfig), C.POINTER(LinearBuffers), C.c_int, C.c_void_p]


def _replicas(name, tensors, count=None):
    tensors = list(tensors)
    if not 1 <= len(tensors) <= MAX_REPLICAS:
        raise ValueError(f"{name}: {len(tensors)} tensors, 1 to {MAX_REPLICAS} replicas expected")
    if count is not None and len(tensors) != count:
        raise ValueError(f"{name}: {len(tensors)} tensors for {count} replicas")
    return tensors


def _matching(name, tensors, shape, dtype, device, dense=False):
    """The raw pointers are all the C side sees: what could make a kernel read past an allocation is refused here.  Returns
    the row stride that all replicas share (0: rows are dense)."""
    stride = None
    for i, t in enumerate(tensors):
        if not (isinstance(t, torch.Tensor) and t.device == device and t.dtype == dtype and tuple(t.shape) == shape):
            raise ValueError(f"{name}[{i}] must be a {dtype} tensor of shape {shape} on {device}, got "
                             f"{(tuple(t.shape), t.dtype, t.device) if isinstance(t, torch.Tensor) else type(t).__name__}")
        if t.is_contiguous():
            row = 0
        elif dense or len(shape) != 2 or (shape[1] > 1 and t.stride(1) != 1) or (shape[0] > 1 and t.stride(0) < shape[1]):
            raise ValueError(f"{name}[{i}] has strides {t.stride()}: " + ("it must be contiguous" if dense else "rows must be dense and not overlap"))
        else:
            row = t.stride(0) if shape[0] > 1 else 0
        if stride is not None and row != stride:
            raise ValueError(f"{name}: all replicas must have the same row stride")
        stride = row
    return stride


def _device_of(name, t):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be tensors on a GPU")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, not {t.dtype}")
    return t.device


def _table(tensors):
    return (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])


def _workspace(nbytes, device):
    return torch.empty(nbytes, dtype=torch.uint8, device=device) if nbytes else None


def _linear_call(cfg, tables, backward, accumulate, device):
    buf = LinearBuffers()
    for name, table in tables.items():
        setattr(buf, name, C.addressof(table))
    need = C.c_uint64(0)
    with _on(device):
        _check(lib.am_linear_workspace(C.byref(cfg), C.byref(buf), int(backward), C.byref(need)))
        space = _workspace(need.value, device)
        if space is not None:
            buf.workspace, buf.workspace_bytes = space.data_ptr(), need.value
        stream = torch.cuda.current_stream(device).cuda_stream
        if backward:
            _check(lib.am_linear_backward(C.byref(cfg), C.byref(buf), int(accumulate), stream))
        else:
            _check(lib.am_linear(C.byref(cfg), C.byref(buf), stream))


def _check_product(x, w):
    x = _replicas("x", x)
    w = _replicas("w", w, len(x))
    device = _device_of("x", x[0])
    if x[0].dim() != 2 or w[0].dim() != 2:
        raise ValueError("x and w must be lists of two-dimensional tensors")
    rows, width = x[0].shape
    out = w[0].shape[0]
    if width == 0 or out == 0:
        raise ValueError(f"a product of {width} by {out} columns")
    dtype = x[0].dtype
    x_stride = _matching("x", x, (rows, width), dtype, device)
    _matching("w", w, (out, width), dtype, device, dense=True)
    return x, w, device, dtype, rows, width, out, x_stride


def linear(x, w, bias=None, act=ACT_NONE, residual=None, with_pre=False):
    """y = act(x w^T + bias) + residual for every replica (am_linear): lists of R tensors, x [rows, in], w [out, in], bias [out],
    residual [rows, out], all bfloat16 or all float32; rows of x and residual may be a stride apart.  Returns the list of
    y, with with_pre the pair (y, pre), pre = x w^T + bias as linear_backward takes it."""
    x, w, device, dtype, rows, width, out, x_stride = _check_product(x, w)
    R = len(x)
    tables = {"x": _table(x), "w": _table(w)}
    cfg = LinearConfig(replicas=R, dtype=_DTYPES[dtype], grad_dtype=_DTYPES[dtype], act=act, rows=rows, in_=width, out=out, x_stride=x_stride)
    if bias is not None:
        bias = _replicas("bias", bias, R)
        _matching("bias", bias, (out,), dtype, device, dense=True)
        tables["bias"] = _table(bias)
    if residual is not None:
        residual = _replicas("residual", residual, R)
        cfg.residual_stride = _matching("residual", residual, (rows, out), dtype, device)
        tables["residual"] = _table(residual)
    y = [torch.empty((rows, out), dtype=dtype, device=device) for _ in range(R)]
    tables["y"] = _table(y)
    pre = None
    if with_pre:
        pre = [torch.empty((rows, out), dtype=dtype, device=device) for _ in range(R)]
        tables["pre"] = _table(pre)
    _linear_call(cfg, tables, False, False, device)
    return (y, pre) if with_pre else y


def linear_backward(dy, x, w, act=ACT_NONE, pre=None, dw=None, db=None, accumulate=False, need_dx=True):
    """The gradients of linear (am_linear_backward).  dy [rows, out]; pre as linear gave it (needed with an activation).  dw [out, in]
    and db [out] are where the gradients go (None: not wanted), float32 or x's type, usually views into the arrays that the step
    reads; accumulate adds to what is there.  Returns the list of dx (None without need_dx).  A residual's gradient is dy."""
    x, w, device, dtype, rows, width, out, x_stride = _check_product(x, w)
    R = len(x)
    if not (need_dx or dw is not None or db is not None):
        raise ValueError("no gradient is wanted: need_dx is off, dw and db are None")
    dy = _replicas("dy", dy, R)
    cfg = LinearConfig(replicas=R, dtype=_DTYPES[dtype], grad_dtype=_DTYPES[dtype], act=act, rows=rows, in_=width, out=out, x_stride=x_stride)
    cfg.y_stride = _matching("dy", dy, (rows, out), dtype, device)
    tables = {"dy": _table(dy), "x": _table(x), "w": _table(w)}
    if act != ACT_NONE:
        if pre is None:
            raise ValueError("the gradient of an activation needs pre")
        pre = _replicas("pre", pre, R)
        cfg.pre_stride = _matching("pre", pre, (rows, out), dtype, device)
        tables["pre"] = _table(pre)
    grad_dtype = None
    for name, grads, shape in (("dw", dw, (out, width)), ("db", db, (out,))):
        if grads is None:
            continue
        grads = _replicas(name, grads, R)
        if grad_dtype is None:
            grad_dtype = grads[0].dtype
            if grad_dtype not in (torch.float32, dtype):
                raise ValueError(f"{name} must be float32 or {dtype}, not {grad_dtype}")
        _matching(name, grads, shape, grad_dtype, device, dense=True)
        tables[name] = _table(grads)
    if grad_dtype is not None:
        cfg.grad_dtype = _DTYPES[grad_dtype]
    dx = None
    if need_dx:
        dx = [torch.empty((rows, width), dtype=dtype, device=device) for _ in range(R)]
        tables["dx"] = _table(dx)
    _linear_call(cfg, tables, True, accumulate, device)
    return dx

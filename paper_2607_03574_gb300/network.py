"""Network operators: what a network that proposes the lanes' parameters is built of.

    y = layer_norm(x, weight, bias)                  # over the last dimension
    h = gated(x, w_gate, w_up, "silu")               # act(x Wg^T) * (x Wu^T)
    z = dropout(h, p, seed, offset, residual=x)      # residual + dropout, the mask never stored

These three are differentiable torch ops on the current stream, like ``loss_op(tape)``; each is
made of raw calls (``*_forward``, ``*_backward``) that take outputs, a workspace and a stream and
map one to one onto the C ABI (``ndvm_layer_norm_*``, ``ndvm_dropout``, ``ndvm_gated_*``).

Layouts: the last dimension is contiguous and the leading ones are rows with one stride (a raw
call refuses anything else, a differentiable op copies it).  Types: float32, float16 and bfloat16;
the gated projection takes the 16-bit ones.  There is no CPU path.
"""
from __future__ import annotations

import ctypes

from . import NdvmError, _check, _on_stream, _stream_ptr, _torch, load

ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}

_types = {}


def _type(t, name):
    if not _types:
        torch = _torch()
        _types.update({torch.float32: 1, torch.float16: 2, torch.bfloat16: 3})
    code = _types.get(t.dtype)
    if code is None:
        raise NdvmError(3, f"{name}: unsupported dtype {t.dtype}")
    return code


def _rows(t, name):
    """(rows, cols, row stride) of a tensor whose last dimension is contiguous."""
    shape, dim = t.shape, t.dim()
    if dim == 0:
        raise NdvmError(1, f"{name} must have at least one dimension")
    cols = shape[-1]
    if t.is_contiguous():
        rows = 1
        for n in shape[:-1]:
            rows *= n
        return rows, cols, cols
    strides = t.stride()
    rows, step = 1, None
    ok = strides[-1] == 1 or cols == 1
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if step is None:
            step = s
        elif s != step * rows:
            ok = False
        rows *= n
    step = cols if step is None else step
    if not ok:
        raise NdvmError(1, f"{name} must be rows of contiguous elements with one row stride")
    return rows, cols, step


def _on_device(x, named):
    """Every tensor on x's device, which is the current one (the kernels launch there)."""
    if not x.is_cuda:
        raise NdvmError(1, "x must be a CUDA tensor (the network operators have no CPU path)")
    device = x.device
    if device.index != _torch().cuda.current_device():
        raise NdvmError(1, f"x is on {device}, which is not the current device")
    for name, t in named:
        if t is not None and t.device != device:
            raise NdvmError(1, f"{name} is on {t.device}, x on {device}")


def _like(t, name, shape, dtype):
    if t.shape != shape or t.dtype != dtype:
        raise NdvmError(1, f"{name} must have shape {tuple(shape)} and dtype {dtype}")


def _vector(t, name, cols):
    if t is None:
        return None
    if t.dim() != 1 or t.shape[0] != cols or not t.is_contiguous():
        raise NdvmError(1, f"{name} must be a contiguous vector of {cols} elements")
    return t.data_ptr()


def _weight_type(x_type, weight, bias):
    ref = weight if weight is not None else bias
    if ref is None:
        return x_type
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise NdvmError(1, "weight and bias must have the same dtype")
    return _type(ref, "weight")


def _workspace(given, nbytes, device, stream):
    """(tensor, its address, its bytes): the caller's workspace or one that belongs to `stream`."""
    if given is not None:
        if not given.is_cuda or given.device != device or not given.is_contiguous():
            raise NdvmError(1, f"workspace must be a contiguous tensor on {device}")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if not nbytes:
        return None, None, 0
    torch = _torch()
    with _on_stream(stream):
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
    return ws, ws.data_ptr(), nbytes


# ------------------------------------------------------------------------------- layer norm
def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, y=None, stats=None, want_stats=True, stream=None):
    """(y, stats): layer norm over the last dimension.  weight and bias: vectors of x's type or float32.
    stats: float32 [2, rows], means and reciprocal deviations for the backward pass (None with
    want_stats=False).  Outputs this call allocates belong to `stream`."""
    torch = _torch()
    lib = load()
    _on_device(x, (("weight", weight), ("bias", bias), ("y", y), ("stats", stats)))
    code = _type(x, "x")
    wcode = _weight_type(code, weight, bias)
    rows, cols, xs = _rows(x, "x")
    if y is None or (stats is None and want_stats):
        with _on_stream(stream):
            if y is None:
                y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            if stats is None and want_stats:
                stats = torch.empty((2, rows), dtype=torch.float32, device=x.device)
    _like(y, "y", x.shape, x.dtype)
    if stats is not None:
        _like(stats, "stats", (2, rows), torch.float32)
        if not stats.is_contiguous():
            raise NdvmError(1, "stats must be contiguous")
    _check(lib.ndvm_layer_norm_forward(code, wcode, rows, cols, x.data_ptr(), xs, _vector(weight, "weight", cols),
                                       _vector(bias, "bias", cols), eps, y.data_ptr(), _rows(y, "y")[2],
                                       None if stats is None else stats.data_ptr(), _stream_ptr(stream)))
    return y, stats


def layer_norm_backward(dy, x, weight, stats, wants=(True, True, True), dx=None, dweight=None, dbias=None,
                        wtype=None, workspace=None, stream=None):
    """(dx, dweight, dbias) of layer_norm_forward; `wants` says which (the others are None).  dweight and
    dbias have weight's type (`wtype` where there is no weight; x's by default)."""
    torch = _torch()
    lib = load()
    _on_device(x, (("dy", dy), ("weight", weight), ("stats", stats), ("dx", dx), ("dweight", dweight), ("dbias", dbias)))
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    _like(dy, "dy", x.shape, x.dtype)
    _like(stats, "stats", (2, rows), torch.float32)
    if not stats.is_contiguous():
        raise NdvmError(1, "stats must be contiguous")
    wdtype = weight.dtype if weight is not None else (wtype or x.dtype)
    with _on_stream(stream):
        if dx is None and wants[0]:
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if dweight is None and wants[1]:
            dweight = torch.empty(cols, dtype=wdtype, device=x.device)
        if dbias is None and wants[2]:
            dbias = torch.empty(cols, dtype=wdtype, device=x.device)
    if dx is not None:
        _like(dx, "dx", x.shape, x.dtype)
    for name, t in (("dweight", dweight), ("dbias", dbias)):
        if t is not None:
            _like(t, name, (cols,), wdtype)
    need = lib.ndvm_layer_norm_workspace_bytes(rows, cols) if dweight is not None or dbias is not None else 0
    ws, wp, nbytes = _workspace(workspace, need, x.device, stream)
    wcode = _weight_type(code, dweight if weight is None else weight, dbias)
    _check(lib.ndvm_layer_norm_backward(code, wcode, rows, cols, dy.data_ptr(), _rows(dy, "dy")[2], x.data_ptr(), xs,
                                        _vector(weight, "weight", cols), stats.data_ptr(),
                                        None if dx is None else dx.data_ptr(), 0 if dx is None else _rows(dx, "dx")[2],
                                        _vector(dweight, "dweight", cols), _vector(dbias, "dbias", cols), wp, nbytes,
                                        _stream_ptr(stream)))
    return dx, dweight, dbias


# ---------------------------------------------------------------------------------- dropout
def dropout_forward(x, p, seed, offset=0, residual=None, y=None, stream=None):
    """residual + (kept ? x / (1 - p) : 0): element i (row-major) takes word offset + i of the sequence that
    `seed` names (0 <= seed, offset < 2^64; offset a multiple of 4).  y may be x or residual."""
    torch = _torch()
    lib = load()
    _on_device(x, (("residual", residual), ("y", y)))
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise NdvmError(1, "seed and offset must be in [0, 2^64)")
    if residual is not None:
        _like(residual, "residual", x.shape, x.dtype)
    if y is None:
        with _on_stream(stream):
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    _like(y, "y", x.shape, x.dtype)
    if x.numel():
        _check(lib.ndvm_dropout(code, rows, cols, x.data_ptr(), xs, None if residual is None else residual.data_ptr(),
                                0 if residual is None else _rows(residual, "residual")[2], p, seed, offset, y.data_ptr(),
                                _rows(y, "y")[2], _stream_ptr(stream)))
    return y


def dropout_backward(dy, p, seed, offset=0, dx=None, stream=None):
    """The gradient of dropout_forward's x: the same words drawn again (residual's gradient is dy itself)."""
    return dropout_forward(dy, p, seed, offset, None, dx, stream)


# ------------------------------------------------------------------------- gated projection
def _activation(name):
    code = ACTIVATIONS.get(name)
    if code is None:
        raise NdvmError(1, f"unknown activation {name!r}: one of {', '.join(ACTIVATIONS)}")
    return code


def _gated_shapes(x, w_gate, w_up):
    rows, k, xs = _rows(x, "x")
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape or w_gate.shape[1] != k:
        raise NdvmError(1, f"w_gate and w_up must both be (n, {k}) matrices")
    if w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise NdvmError(1, "x, w_gate and w_up must have the same dtype")
    return rows, k, w_gate.shape[0], xs, _rows(w_gate, "w_gate")[2], _rows(w_up, "w_up")[2]


def _aligned(px, xs, pg, gs, pu, us):
    """Whether the products can read every operand where it lies (addresses, row strides in elements)."""
    return int((px | pg | pu) % 16 == 0 and (xs | gs | us) % 8 == 0 and xs != 0 and gs != 0 and us != 0)


def gated_forward(x, w_gate, w_up, activation="silu", h=None, workspace=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T): x (..., k), both weights (n, k), h (..., n); 16-bit types.  Outputs
    and the workspace that this call allocates belong to `stream`."""
    torch = _torch()
    lib = load()
    act = _activation(activation)
    _on_device(x, (("w_gate", w_gate), ("w_up", w_up), ("h", h)))
    code = _type(x, "x")
    rows, k, n, xs, gs, us = _gated_shapes(x, w_gate, w_up)
    shape = x.shape[:-1] + (n,)
    if h is None:
        with _on_stream(stream):
            h = torch.empty(shape, dtype=x.dtype, device=x.device)
    _like(h, "h", shape, x.dtype)
    px, pg, pu = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    need = lib.ndvm_gated_workspace_bytes(rows, k, n, 0, _aligned(px, xs, pg, gs, pu, us))
    ws, wp, nbytes = _workspace(workspace, need, x.device, stream)
    _check(lib.ndvm_gated_forward(code, act, rows, k, n, px, xs, pg, gs, pu, us, h.data_ptr(), _rows(h, "h")[2], wp, nbytes,
                                  _stream_ptr(stream)))
    return h


def gated_backward(dh, x, w_gate, w_up, activation="silu", wants=(True, True, True), dx=None, dw_gate=None, dw_up=None,
                   workspace=None, stream=None):
    """(dx, dw_gate, dw_up) of gated_forward; `wants` says which (the others are None)."""
    torch = _torch()
    lib = load()
    act = _activation(activation)
    _on_device(x, (("dh", dh), ("w_gate", w_gate), ("w_up", w_up), ("dx", dx), ("dw_gate", dw_gate), ("dw_up", dw_up)))
    code = _type(x, "x")
    rows, k, n, xs, gs, us = _gated_shapes(x, w_gate, w_up)
    _like(dh, "dh", x.shape[:-1] + (n,), x.dtype)
    with _on_stream(stream):
        if dx is None and wants[0]:
            dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        if dw_gate is None and wants[1]:
            dw_gate = torch.empty((n, k), dtype=x.dtype, device=x.device)
        if dw_up is None and wants[2]:
            dw_up = torch.empty((n, k), dtype=x.dtype, device=x.device)
    if dx is not None:
        _like(dx, "dx", x.shape, x.dtype)
    for name, t in (("dw_gate", dw_gate), ("dw_up", dw_up)):
        if t is not None:
            _like(t, name, (n, k), x.dtype)
            if not t.is_contiguous():
                raise NdvmError(1, f"{name} must be contiguous")
    px, pg, pu, ph, hs = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr(), dh.data_ptr(), _rows(dh, "dh")[2]
    need = lib.ndvm_gated_workspace_bytes(rows, k, n, 1, _aligned(px, xs, pg, gs, pu, us))
    ws, wp, nbytes = _workspace(workspace, need, x.device, stream)
    _check(lib.ndvm_gated_backward(code, act, rows, k, n, ph, hs, px, xs, pg, gs, pu, us,
                                   None if dx is None else dx.data_ptr(), 0 if dx is None else _rows(dx, "dx")[2],
                                   None if dw_gate is None else dw_gate.data_ptr(),
                                   None if dw_up is None else dw_up.data_ptr(), wp, nbytes, _stream_ptr(stream)))
    return dx, dw_gate, dw_up


# ----------------------------------------------------------------------- differentiable ops
def _rowed(t):
    """t, or a contiguous copy where its layout is not rows of contiguous elements."""
    if t is None or t.is_contiguous():
        return t
    try:
        _rows(t, "")
        return t
    except NdvmError:
        return t.contiguous()


_ops = None


def _make_ops():
    global _ops
    torch = _torch()
    once = torch.autograd.function.once_differentiable

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, eps):
            y, stats = layer_norm_forward(x, weight, bias, eps)
            ctx.save_for_backward(x, weight, stats)
            ctx.wtype = None if bias is None else bias.dtype
            return y

        @staticmethod
        @once
        def backward(ctx, dy):
            x, weight, stats = ctx.saved_tensors
            return layer_norm_backward(_rowed(dy), x, weight, stats, ctx.needs_input_grad[:3], wtype=ctx.wtype) + (None,)

    class Drop(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, seed, offset, residual):
            ctx.draw = (p, seed, offset)
            return dropout_forward(x, p, seed, offset, residual)

        @staticmethod
        @once
        def backward(ctx, dy):
            dx = dropout_backward(_rowed(dy), *ctx.draw) if ctx.needs_input_grad[0] else None
            return dx, None, None, None, dy if ctx.needs_input_grad[4] else None

    class Gated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w_gate, w_up, activation):
            ctx.save_for_backward(x, w_gate, w_up)
            ctx.activation = activation
            return gated_forward(x, w_gate, w_up, activation)

        @staticmethod
        @once
        def backward(ctx, dh):
            return gated_backward(_rowed(dh), *ctx.saved_tensors, ctx.activation, ctx.needs_input_grad[:3]) + (None,)

    _ops = Norm, Drop, Gated
    return _ops


def _recorded(*tensors):
    return _torch().is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension as a differentiable op (gradients of x, weight and bias)."""
    x = _rowed(x)
    if not _recorded(x, weight, bias):
        return layer_norm_forward(x, weight, bias, eps, want_stats=False)[0]
    return (_ops or _make_ops())[0].apply(x, weight, bias, eps)


def dropout(x, p, seed, offset=0, residual=None):
    """residual + dropout(x) as a differentiable op; see dropout_forward for what is drawn.  Give each call of
    a step its own offset range, and each step another seed or range."""
    x, residual = _rowed(x), _rowed(residual)
    if not _recorded(x, residual):
        return dropout_forward(x, p, seed, offset, residual)
    return (_ops or _make_ops())[1].apply(x, p, seed, offset, residual)


def gated(x, w_gate, w_up, activation="silu"):
    """act(x w_gate^T) * (x w_up^T) as a differentiable op (gradients of x and both weights)."""
    x, w_gate, w_up = _rowed(x), _rowed(w_gate), _rowed(w_up)
    if not _recorded(x, w_gate, w_up):
        return gated_forward(x, w_gate, w_up, activation)
    return (_ops or _make_ops())[2].apply(x, w_gate, w_up, activation)


def check_operators():
    """Synchronize and raise if a kernel of the operators gave up waiting since the last check."""
    _check(load().ndvm_check_operators())

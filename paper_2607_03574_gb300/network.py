"""Network operators: what a network that proposes the lanes' parameters is built of.

    y = layer_norm(x, weight, bias)                  # over the last dimension
    h = gated(x, w_gate, w_up, "silu")               # act(x Wg^T) * (x Wu^T)
    z = dropout(h, p, seed, offset, residual=x)      # residual + dropout, the mask never stored

These three are differentiable torch ops on the current stream, like ``loss_op(tape)`` (their autograd
nodes are in ``csrc/net/torch_ops.cpp``).  Under them are raw calls (``*_forward``, ``*_backward``) that take
outputs, a workspace and a stream and map one to one onto the C ABI (``ndvm_layer_norm_*``,
``ndvm_dropout``, ``ndvm_gated_*``).

Layouts: the last dimension is contiguous and the leading ones are rows with one stride, 0 or at least a
row's length (a raw call refuses anything else, a differentiable op copies it).  Types: float32, float16 and bfloat16;
the gated projection takes the 16-bit ones.  There is no CPU path.

No second derivatives and no forward mode, and neither torch.jit.trace nor torch.fx can record a call: each of these
raises.  ``check_operators()`` says whether a kernel has given up a wait, after which its outputs are not valid.
"""
from __future__ import annotations

import ctypes

import paper_2607_03574_gb300 as _nd

from . import NdvmError, _check, _on_stream, _torch, load

ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2, "sigmoid": 3}

_torch_module = None
_types = {}
_modes = None  # torch's questions that _recorded asks


def _start():
    """torch and the library, looked up once (the calls below are short beside an import's lookups)."""
    global _torch_module, _modes
    torch = _torch()
    c = torch._C
    _modes = (c._get_tracing_state, c._len_torch_dispatch_stack, c._dispatch_tls_is_dispatch_key_included, c.DispatchKey.PreDispatch,
              c._get_dispatch_mode, c._TorchDispatchModeKey.PROXY)
    _types.update({torch.float32: 1, torch.float16: 2, torch.bfloat16: 3})
    _torch_module = torch
    return torch


def _type(t, name):
    code = _types.get(t.dtype)
    if code is None:
        raise NdvmError(3, f"{name}: unsupported dtype {t.dtype}")
    return code


def _rows(t, name):
    """(rows, cols, row stride) of a tensor whose last dimension is contiguous."""
    shape = t.shape
    if not shape:
        raise NdvmError(1, f"{name} must have at least one dimension")
    cols = shape[-1]
    if cols == 1 and t.is_neg():  # (with more columns such a view is not contiguous)
        raise NdvmError(1, f"{name}'s memory holds the opposite sign (a view of a conjugate): use resolve_neg()")
    if t.is_contiguous():
        if len(shape) == 2:
            return shape[0], cols, cols
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
    if not ok or (rows > 1 and 0 < step < cols):
        raise NdvmError(1, f"{name} must be rows of contiguous elements with one row stride (0, or at least a row's length)")
    return rows, cols, step


def _recorded():
    """Whether torch records a program here (torch.jit.trace, or torch.fx's proxies): it would record an output's
    allocation and not the launch that fills it."""
    tracing, depth, included, pre_dispatch, mode, proxy = _modes
    return tracing() is not None or included(pre_dispatch) or (depth() > 0 and mode(proxy) is not None)


def _device(torch, x):
    """The index of x's device, which has to be the current one (the kernels launch there)."""
    if _recorded():
        raise NdvmError(3, "the network operators cannot be traced: the trace would not hold their launches")
    device = x.get_device()
    if device < 0:
        raise NdvmError(1, "x must be a CUDA tensor (the network operators have no CPU path)")
    if device != torch._C._cuda_getDevice():
        raise NdvmError(1, f"x is on cuda:{device}, which is not the current device")
    return device


def _same_device(device, t, name):
    if t.get_device() != device:
        raise NdvmError(1, f"{name} is on {t.device}, x on cuda:{device}")


def _stream(torch, stream, device):
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _given(t, name, shape, dtype, device):
    """Checks an output (or a tensor of a known shape) that the caller gave."""
    if t.shape != shape or t.dtype != dtype:
        raise NdvmError(1, f"{name} must have shape {tuple(shape)} and dtype {dtype}")
    _same_device(device, t, name)


def _vector(t, name, cols, device):
    """The address of a vector of `cols` elements, or None."""
    if t is None:
        return None
    if t.shape != (cols,) or not t.is_contiguous() or (cols == 1 and t.is_neg()):
        raise NdvmError(1, f"{name} must be a contiguous vector of {cols} elements")
    _same_device(device, t, name)
    return t.data_ptr()


def _stats(stats, rows, device):
    _given(stats, "stats", (2, rows), _torch_module.float32, device)
    if not stats.is_contiguous():
        raise NdvmError(1, "stats must be contiguous")
    return stats.data_ptr()


def _new(torch, shape, dtype, device, stream):
    """An uninitialised tensor that belongs to `stream` (torch's allocator; None: the current one)."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _on_stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _workspace(torch, given, nbytes, device, stream):
    """(tensor, its address, its bytes): the caller's workspace or one that belongs to `stream`."""
    if given is not None:
        _same_device(device, given, "workspace")
        if not given.is_contiguous():
            raise NdvmError(1, "workspace must be contiguous")
        return given, given.data_ptr(), given.numel() * given.element_size()
    if not nbytes:
        return None, None, 0
    ws = _new(torch, nbytes, torch.uint8, device, stream)
    return ws, ws.data_ptr(), nbytes


# ------------------------------------------------------------------------------- layer norm
def _weight_type(x_code, weight, bias):
    if weight is None:
        return x_code if bias is None else _type(bias, "bias")
    if bias is not None and weight.dtype != bias.dtype:
        raise NdvmError(1, "weight and bias must have the same dtype")
    return _type(weight, "weight")


def layer_norm_forward(x, weight=None, bias=None, eps=1e-5, y=None, stats=None, want_stats=True, stream=None):
    """(y, stats): layer norm over the last dimension.  weight and bias: vectors of x's type or float32.
    stats: float32 [2, rows], means and reciprocal deviations for the backward pass (None with
    want_stats=False).  Outputs this call allocates belong to `stream`."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    if y is None:
        y, ys = _new(torch, x.shape, x.dtype, device, stream), cols
    else:
        _given(y, "y", x.shape, x.dtype, device)
        ys = _rows(y, "y")[2]
    if stats is not None:
        sp = _stats(stats, rows, device)
    elif want_stats:
        stats = _new(torch, (2, rows), torch.float32, device, stream)
        sp = stats.data_ptr()
    else:
        sp = None
    status = lib.ndvm_layer_norm_forward(code, _weight_type(code, weight, bias), rows, cols, x.data_ptr(), xs,
                                         _vector(weight, "weight", cols, device), _vector(bias, "bias", cols, device), eps,
                                         y.data_ptr(), ys, sp, _stream(torch, stream, device))
    if status:
        _check(status)
    return y, stats


def layer_norm_backward(dy, x, weight, stats, wants=(True, True, True), dx=None, dweight=None, dbias=None,
                        wtype=None, workspace=None, stream=None):
    """(dx, dweight, dbias) of layer_norm_forward; `wants` says which (the others are None).  dweight and
    dbias have weight's type (`wtype` where there is no weight; x's by default)."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    _given(dy, "dy", x.shape, x.dtype, device)
    sp = _stats(stats, rows, device)
    wdtype = weight.dtype if weight is not None else (wtype or x.dtype)
    xp = dxs = dwp = dbp = None
    if dx is not None:
        _given(dx, "dx", x.shape, x.dtype, device)
        xp, dxs = dx.data_ptr(), _rows(dx, "dx")[2]
    elif wants[0]:
        dx = _new(torch, x.shape, x.dtype, device, stream)
        xp, dxs = dx.data_ptr(), cols
    if dweight is not None:
        _given(dweight, "dweight", (cols,), wdtype, device)
        dwp = _vector(dweight, "dweight", cols, device)
    elif wants[1]:
        dweight = _new(torch, cols, wdtype, device, stream)
        dwp = dweight.data_ptr()
    if dbias is not None:
        _given(dbias, "dbias", (cols,), wdtype, device)
        dbp = _vector(dbias, "dbias", cols, device)
    elif wants[2]:
        dbias = _new(torch, cols, wdtype, device, stream)
        dbp = dbias.data_ptr()
    need = lib.ndvm_layer_norm_workspace_bytes(rows, cols) if dwp is not None or dbp is not None else 0
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_layer_norm_backward(code, _weight_type(code, dweight if weight is None else weight, dbias), rows, cols,
                                          dy.data_ptr(), _rows(dy, "dy")[2], x.data_ptr(), xs,
                                          _vector(weight, "weight", cols, device), sp, xp, dxs or 0, dwp, dbp, wp, nbytes,
                                          _stream(torch, stream, device))
    if status:
        _check(status)
    return dx, dweight, dbias


# ---------------------------------------------------------------------------------- dropout
def dropout_forward(x, p, seed, offset=0, residual=None, y=None, stream=None):
    """residual + (kept ? x / (1 - p) : 0): element i (row-major) takes word offset + i of the sequence that
    `seed` names (0 <= seed, offset < 2^64; offset a multiple of 4).  y may be x or residual."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    if not (0 <= seed < 1 << 64 and 0 <= offset < 1 << 64):
        raise NdvmError(1, "seed and offset must be in [0, 2^64)")
    rp, rs = None, 0
    if residual is not None:
        _given(residual, "residual", x.shape, x.dtype, device)
        rp, rs = residual.data_ptr(), _rows(residual, "residual")[2]
    if y is None:
        y, ys = _new(torch, x.shape, x.dtype, device, stream), cols
    else:
        _given(y, "y", x.shape, x.dtype, device)
        ys = _rows(y, "y")[2]
    status = lib.ndvm_dropout(code, rows, cols, x.data_ptr(), xs, rp, rs, p, seed, offset, y.data_ptr(), ys,
                              _stream(torch, stream, device))
    if status:
        _check(status)
    return y


def dropout_backward(dy, p, seed, offset=0, dx=None, stream=None):
    """The gradient of dropout_forward's x: the same words drawn again (residual's gradient is dy itself)."""
    return dropout_forward(dy, p, seed, offset, None, dx, stream)


# ------------------------------------------------------------------------- gated projection
def _gated_operands(x, w_gate, w_up, activation, device):
    """(activation, rows, k, n, addresses and row strides of x, w_gate and w_up, whether the products can read
    every one of them where it lies)."""
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise NdvmError(1, f"unknown activation {activation!r}: one of {', '.join(ACTIVATIONS)}")
    rows, k, xs = _rows(x, "x")
    if w_gate.dim() != 2 or w_gate.shape != w_up.shape or w_gate.shape[1] != k:
        raise NdvmError(1, f"w_gate and w_up must both be (n, {k}) matrices")
    if w_gate.dtype != x.dtype or w_up.dtype != x.dtype:
        raise NdvmError(1, "x, w_gate and w_up must have the same dtype")
    _same_device(device, w_gate, "w_gate")
    _same_device(device, w_up, "w_up")
    gs, us = _rows(w_gate, "w_gate")[2], _rows(w_up, "w_up")[2]
    px, pg, pu = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    ready = int((px | pg | pu) % 16 == 0 and (xs | gs | us) % 8 == 0 and xs != 0 and gs != 0 and us != 0)
    return act, rows, k, w_gate.shape[0], (px, xs, pg, gs, pu, us), ready


def gated_kept(x, w_gate, stream=None):
    """A tensor for gated_forward's `kept`: float32 [2, rows, stride], a row's first n elements in use."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    return _new(torch, (2, _rows(x, "x")[0], lib.ndvm_gated_kept_stride(w_gate.shape[0])), torch.float32, _device(torch, x), stream)


def _kept(torch, lib, kept, rows, n, device):
    if kept is None:
        return None
    _given(kept, "kept", (2, rows, lib.ndvm_gated_kept_stride(n)), torch.float32, device)
    if not kept.is_contiguous():
        raise NdvmError(1, "kept must be contiguous")
    return kept.data_ptr()


def gated_forward(x, w_gate, w_up, activation="silu", h=None, kept=None, workspace=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T): x (..., k), both weights (n, k), h (..., n); 16-bit types.  kept: a tensor of
    gated_kept that receives the two products for gated_backward.  Outputs and the workspace that this call
    allocates belong to `stream`."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    act, rows, k, n, operands, ready = _gated_operands(x, w_gate, w_up, activation, device)
    shape = x.shape[:-1] + (n,)
    if h is None:
        h, hs = _new(torch, shape, x.dtype, device, stream), n
    else:
        _given(h, "h", shape, x.dtype, device)
        hs = _rows(h, "h")[2]
    need = 0 if ready else lib.ndvm_gated_workspace_bytes(rows, k, n, 0, 0)
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_gated_forward_keep(code, act, rows, k, n, *operands, h.data_ptr(), hs,
                                         _kept(torch, lib, kept, rows, n, device), wp, nbytes, _stream(torch, stream, device))
    if status:
        _check(status)
    return h


def gated_backward(dh, x, w_gate, w_up, activation="silu", wants=(True, True, True), dx=None, dw_gate=None, dw_up=None,
                   kept=None, workspace=None, stream=None):
    """(dx, dw_gate, dw_up) of gated_forward; `wants` says which (the others are None).  kept: what the forward
    call kept (None: the two products are computed again)."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    act, rows, k, n, operands, ready = _gated_operands(x, w_gate, w_up, activation, device)
    _given(dh, "dh", x.shape[:-1] + (n,), x.dtype, device)
    xp = gp = up = None
    dxs = 0
    if dx is not None:
        _given(dx, "dx", x.shape, x.dtype, device)
        xp, dxs = dx.data_ptr(), _rows(dx, "dx")[2]
    elif wants[0]:
        dx = _new(torch, x.shape, x.dtype, device, stream)
        xp, dxs = dx.data_ptr(), k
    for name, t in (("dw_gate", dw_gate), ("dw_up", dw_up)):
        if t is not None:
            _given(t, name, (n, k), x.dtype, device)
            if not t.is_contiguous():
                raise NdvmError(1, f"{name} must be contiguous")
    if dw_gate is None and wants[1]:
        dw_gate = _new(torch, (n, k), x.dtype, device, stream)
    if dw_up is None and wants[2]:
        dw_up = _new(torch, (n, k), x.dtype, device, stream)
    if dw_gate is not None:
        gp = dw_gate.data_ptr()
    if dw_up is not None:
        up = dw_up.data_ptr()
    ph, hs = dh.data_ptr(), _rows(dh, "dh")[2]
    need = lib.ndvm_gated_workspace_bytes(rows, k, n, 1, int(ready and (ph | 2 * hs) % 16 == 0 and hs != 0))
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_gated_backward_kept(code, act, rows, k, n, ph, hs, *operands,
                                          _kept(torch, lib, kept, rows, n, device), xp, dxs, gp, up, wp, nbytes,
                                          _stream(torch, stream, device))
    if status:
        _check(status)
    return dx, dw_gate, dw_up


# ----------------------------------------------------------------------- differentiable ops
_ops = None


def _load_ops():
    """The module of autograd nodes (built first if it is missing or out of date)."""
    global _ops
    import importlib.machinery
    import importlib.util

    from . import build
    _start()
    load()
    build.build(torch_ops=True)
    loader = importlib.machinery.ExtensionFileLoader("ndvm_torch", build.TORCH_OPS)
    ops = importlib.util.module_from_spec(importlib.util.spec_from_loader("ndvm_torch", loader))
    loader.exec_module(ops)
    _ops = ops
    return ops


def _refuse(raw, *args):
    """Raises what is wrong with an op's arguments: the raw call on them says it."""
    raw(*args)
    raise NdvmError(3, "the differentiable op does not take these arguments")


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """Layer norm over the last dimension as a differentiable op (gradients of x, weight and bias)."""
    try:
        y = (_ops or _load_ops()).layer_norm(x, weight, bias, eps)
    except TypeError:
        y = None
    return _refuse(layer_norm_forward, x, weight, bias, eps) if y is None else y


def dropout(x, p, seed, offset=0, residual=None):
    """residual + dropout(x) as a differentiable op; see dropout_forward for what is drawn.  Give each call of
    a step its own offset range, and each step another seed or range."""
    try:
        y = (_ops or _load_ops()).dropout(x, p, seed, offset, residual)
    except TypeError:
        y = None
    return _refuse(dropout_forward, x, p, seed, offset, residual) if y is None else y


def gated(x, w_gate, w_up, activation="silu", keep=None):
    """act(x w_gate^T) * (x w_up^T) as a differentiable op (gradients of x and both weights).  keep: whether the two
    products are held for the backward pass, as float32 (8 bytes an element of the result), instead of computed
    again; None: where that is the faster (k >= 1536, or results of up to 2^21 elements)."""
    try:
        y = (_ops or _load_ops()).gated(x, w_gate, w_up, ACTIVATIONS.get(activation, -1), -1 if keep is None else int(bool(keep)))
    except TypeError:
        y = None
    return _refuse(gated_forward, x, w_gate, w_up, activation) if y is None else y


def check_operators():
    """Synchronize and raise if a kernel of the operators gave up waiting since the last check."""
    _check(load().ndvm_check_operators())

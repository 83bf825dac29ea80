"""Network operators: what a network that proposes the lanes' parameters is built of.

    y = layer_norm(x, weight, bias)                  # over the last dimension
    h = gated(x, w_gate, w_up, "silu")               # act(x Wg^T) * (x Wu^T)
    z = dropout(h, p, seed, offset, residual=x)      # residual + dropout, the mask never stored
    y, x = rms_norm(x, weight, residual=h)           # of x + h, which is returned beside it
    y = linear(x, w, bias, "silu", residual)         # act(x w^T + bias) + residual; keep="8bit": less is held for its gradient

These are differentiable torch ops on the current stream, like ``loss_op(tape)`` (their autograd
nodes are in ``csrc/net/torch_ops.cpp``).  Under them are raw calls (``*_forward``, ``*_backward``) that take
outputs, a workspace and a stream and map one to one onto the C ABI (``ndvm_layer_norm_*``,
``ndvm_dropout``, ``ndvm_gated_*``, ``ndvm_rms_norm_*``, ``ndvm_linear_*``).

A trained network is scored on 8-bit operands, without gradients:

    q = quantize(w)                                  # once: 8-bit blocks (Quantized)
    h, x = rms_norm_quantized(x, weight, residual=y)
    y = linear_quantized(h, q, bias, "silu")

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
_NONE = 4  # no activation (dense layers alone)

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


# ----------------------------------------------------------------------------------- rms norm
def _rms_stats(rstd, rows, device):
    _given(rstd, "rstd", (rows,), _torch_module.float32, device)
    if not rstd.is_contiguous():
        raise NdvmError(1, "rstd must be contiguous")
    return rstd.data_ptr()


def _like(t, name, x, device):
    """(address, row stride) of a tensor of x's shape and type, or (None, 0)."""
    if t is None:
        return None, 0
    _given(t, name, x.shape, x.dtype, device)
    return t.data_ptr(), _rows(t, name)[2]


def rms_norm_forward(x, weight=None, eps=1e-6, residual=None, y=None, sum=None, rstd=None, want_rstd=True, stream=None):
    """(y, sum, rstd): s / sqrt(mean(s^2) + eps) * weight over the last dimension, s = x + residual rounded to x's type
    (sum; None without a residual).  weight: a vector of x's type or float32.  rstd: float32 [rows] for the backward pass
    (None with want_rstd=False).  sum may be x or residual.  Outputs this call allocates belong to `stream`."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    rp, rs = _like(residual, "residual", x, device)
    if sum is not None and residual is None:
        raise NdvmError(1, "a sum is written where there is a residual")
    if y is None:
        y = _new(torch, x.shape, x.dtype, device, stream)
    if sum is None and residual is not None:
        sum = _new(torch, x.shape, x.dtype, device, stream)
    if rstd is None and want_rstd:
        rstd = _new(torch, (rows,), torch.float32, device, stream)
    yp, ys = _like(y, "y", x, device)
    sp, ss = _like(sum, "sum", x, device)
    status = lib.ndvm_rms_norm_forward(code, _weight_type(code, weight, None), rows, cols, x.data_ptr(), xs, rp, rs,
                                       _vector(weight, "weight", cols, device), eps, yp, ys, sp, ss,
                                       None if rstd is None else _rms_stats(rstd, rows, device), _stream(torch, stream, device))
    if status:
        _check(status)
    return y, sum, rstd


def rms_norm_backward(dy, s, weight, rstd, dsum=None, wants=(True, True), dx=None, dweight=None, wtype=None, workspace=None,
                      stream=None):
    """(dx, dweight) of rms_norm_forward, s being its sum (its x without a residual); dx is the residual's gradient too.
    `wants` says which (the others are None).  dweight has weight's type (`wtype` where there is none; x's by default)."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, s)
    code = _type(s, "s")
    rows, cols, xs = _rows(s, "s")
    dyp, dys = _like(dy, "dy", s, device)
    dsp, dss = _like(dsum, "dsum", s, device)
    wdtype = weight.dtype if weight is not None else (wtype or s.dtype)
    if dx is None and wants[0]:
        dx = _new(torch, s.shape, s.dtype, device, stream)
    if dweight is None and wants[1]:
        dweight = _new(torch, (cols,), wdtype, device, stream)
    xp, dxs = _like(dx, "dx", s, device)
    dwp = None
    if dweight is not None:
        _given(dweight, "dweight", (cols,), wdtype, device)
        dwp = _vector(dweight, "dweight", cols, device)
    need = lib.ndvm_rms_norm_workspace_bytes(rows, cols) if dwp is not None else 0
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_rms_norm_backward(code, _weight_type(code, dweight if weight is None else weight, None), rows, cols, dyp, dys,
                                        dsp, dss, s.data_ptr(), xs, _vector(weight, "weight", cols, device),
                                        _rms_stats(rstd, rows, device), xp, dxs, dwp, wp, nbytes, _stream(torch, stream, device))
    if status:
        _check(status)
    return dx, dweight


# -------------------------------------------------------------------------------- 8-bit blocks
class Quantized:
    """A tensor in 8-bit blocks: 32 consecutive elements of the last dimension share a scale 2^e, the least from e = -127 on
    with which none is over 448 in size; an element is the nearest e4m3 value to v / 2^e.  A block with an infinity or a
    NaN is NaN.

    values: float8_e4m3fn of the tensor's shape, rows with one stride that is a multiple of 16 and starts on 16 bytes.  A row's
    bytes go up to a multiple of 16: those behind its last element are written as 0 where the blocks are.
    scales: uint8 [rows / 128, columns / 128, 32, 4, 4] (both rounded up), e + 127 at [row / 128, column / 128, row % 32,
    row / 32 % 4, column / 32 % 4].  quantize() and rms_norm_quantized() make them."""

    __slots__ = ("values", "scales", "rows", "cols", "stride")

    def __init__(self, values, scales):
        try:
            sizes = (_ops or _load_ops()).blocks_of(values, scales)
        except TypeError:
            sizes = None
        self.values, self.scales = values, scales
        self.rows, self.cols, self.stride = sizes or self._sizes(values, scales)

    @staticmethod
    def _sizes(values, scales):
        """(rows, cols, row stride), or what is wrong."""
        torch = _torch_module or _start()
        if values.dtype != torch.float8_e4m3fn or scales.dtype != torch.uint8:
            raise NdvmError(3, "8-bit blocks are float8_e4m3fn values with uint8 scales")
        if not values.is_cuda or scales.device != values.device:
            raise NdvmError(1, "values and scales must be CUDA tensors of one device")
        rows, cols, stride = _rows(values, "values")
        if (rows > 1 and (stride % 16 or stride < cols)) or values.data_ptr() % 16:
            raise NdvmError(1, "values must be rows that start on 16 bytes")
        if scales.shape != (-(-rows // 128), -(-cols // 128), 32, 4, 4) or not scales.is_contiguous() or scales.data_ptr() % 16:
            raise NdvmError(1, f"scales must be contiguous, of shape {(-(-rows // 128), -(-cols // 128), 32, 4, 4)}, and start on 16 bytes")
        return rows, cols, stride

    @classmethod
    def _of(cls, values, scales, rows, cols, stride):
        """(what this package has made needs no checks)"""
        q = cls.__new__(cls)
        q.values, q.scales, q.rows, q.cols, q.stride = values, scales, rows, cols, stride
        return q

    @property
    def shape(self):
        return self.values.shape

    @property
    def device(self):
        return self.values.device

    def __repr__(self):
        return f"Quantized(shape={tuple(self.shape)}, device={self.device})"

    def dequantize(self, dtype=None, out=None, stream=None):
        """What the blocks stand for, rounded to dtype (float32 by default); what rounding lifts beyond its largest finite
        value becomes that value."""
        torch = _torch_module or _start()
        lib = _nd._lib or load()
        device = _device(torch, self.values)
        if out is None:
            out = _new(torch, self.shape, dtype or torch.float32, device, stream)
        else:
            _given(out, "out", self.shape, dtype or out.dtype, device)
        status = lib.ndvm_dequantize(_type(out, "out"), self.rows, self.cols, self.values.data_ptr(), self.stride, self.scales.data_ptr(),
                                     out.data_ptr(), _rows(out, "out")[2], _stream(torch, stream, device))
        if status:
            _check(status)
        return out


def _new_quantized(torch, shape, rows, cols, device, stream):
    """Room for blocks of `shape`."""
    pitch = -(-cols // 16) * 16
    values = _new(torch, shape[:-1] + (pitch,), torch.float8_e4m3fn, device, stream)[..., :cols]
    scales = _new(torch, (-(-rows // 128), -(-cols // 128), 32, 4, 4), torch.uint8, device, stream)
    return Quantized._of(values, scales, rows, cols, pitch)


def _given_quantized(q, name, shape, device):
    if not isinstance(q, Quantized) or q.shape != shape:
        raise NdvmError(1, f"{name} must be Quantized of shape {tuple(shape)}")
    _same_device(device, q.values, name)


def quantize_forward(x, out=None, stream=None):
    """Quantized: 8-bit blocks of x (..., cols); float32, float16, bfloat16.  out: a Quantized of x's shape to write to."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    if out is None:
        out = _new_quantized(torch, x.shape, rows, cols, device, stream)
    else:
        _given_quantized(out, "out", x.shape, device)
    status = lib.ndvm_quantize(code, rows, cols, x.data_ptr(), xs, out.values.data_ptr(), out.stride, out.scales.data_ptr(),
                               _stream(torch, stream, device))
    if status:
        _check(status)
    return out


def rms_norm_quantized_forward(x, weight=None, eps=1e-6, residual=None, out=None, sum=None, stream=None):
    """(y, sum): rms_norm_forward with y as 8-bit blocks (Quantized) of what is not rounded in between."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    rows, cols, xs = _rows(x, "x")
    rp, rs = _like(residual, "residual", x, device)
    if sum is not None and residual is None:
        raise NdvmError(1, "a sum is written where there is a residual")
    if sum is None and residual is not None:
        sum = _new(torch, x.shape, x.dtype, device, stream)
    sp, ss = _like(sum, "sum", x, device)
    if out is None:
        out = _new_quantized(torch, x.shape, rows, cols, device, stream)
    else:
        _given_quantized(out, "out", x.shape, device)
    status = lib.ndvm_rms_norm_quantized(code, _weight_type(code, weight, None), rows, cols, x.data_ptr(), xs, rp, rs,
                                         _vector(weight, "weight", cols, device), eps, out.values.data_ptr(), out.stride,
                                         out.scales.data_ptr(), sp, ss, _stream(torch, stream, device))
    if status:
        _check(status)
    return out, sum


# -------------------------------------------------------------------------------- dense layers
def _activation(activation):
    if activation is None:
        return _NONE
    act = ACTIVATIONS.get(activation)
    if act is None:
        raise NdvmError(1, f"unknown activation {activation!r}: None or one of {', '.join(ACTIVATIONS)}")
    return act


def _matrix(w, name, x, k, device):
    """(n, row stride) of a weight matrix (n, k) of x's type."""
    if w.dim() != 2 or w.shape[1] != k:
        raise NdvmError(1, f"{name} must be an (n, {k}) matrix")
    if w.dtype != x.dtype:
        raise NdvmError(1, f"x and {name} must have the same dtype")
    _same_device(device, w, name)
    return w.shape[0], _rows(w, name)[2]


def _ready(pointer, stride, rows, cols):
    """Whether the products can read a matrix of 16-bit elements where it lies."""
    return pointer % 16 == 0 and (rows <= 1 or (stride % 8 == 0 and stride >= cols))


def linear_kept(x, w, keep=None, stream=None):
    """What linear_forward's `kept` takes: float32 [rows, stride], a row's first n elements in use, or with keep="8bit" a
    Quantized [rows, n]."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    rows, n, device = _rows(x, "x")[0], w.shape[0], _device(torch, x)
    if keep == "8bit":
        return _new_quantized(torch, (rows, n), rows, n, device, stream)
    if keep is not None:
        raise NdvmError(1, f"unknown keep {keep!r}: None or '8bit'")
    return _new(torch, (rows, lib.ndvm_linear_kept_stride(n)), torch.float32, device, stream)


def _linear_kept(torch, lib, kept, rows, n, device):
    """(z, z_values, z_scales) of linear_kept's tensor."""
    if kept is None:
        return None, None, None
    if isinstance(kept, Quantized):
        _given_quantized(kept, "kept", (rows, n), device)
        if rows > 1 and kept.stride != -(-n // 16) * 16:
            raise NdvmError(1, "kept must be one of linear_kept")
        return None, kept.values.data_ptr(), kept.scales.data_ptr()
    _given(kept, "kept", (rows, lib.ndvm_linear_kept_stride(n)), torch.float32, device)
    if not kept.is_contiguous():
        raise NdvmError(1, "kept must be contiguous")
    return kept.data_ptr(), None, None


def linear_forward(x, w, bias=None, activation=None, residual=None, y=None, kept=None, workspace=None, stream=None):
    """y = act(x w^T + bias) + residual: x (..., k), w (n, k), bias (n) of x's type or float32, y and residual (..., n);
    16-bit types.  kept: a tensor of linear_kept that receives x w^T + bias for linear_backward.  y may be residual.
    Outputs and the workspace that this call allocates belong to `stream`."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, x)
    code = _type(x, "x")
    act = _activation(activation)
    rows, k, xs = _rows(x, "x")
    n, ws_ = _matrix(w, "w", x, k, device)
    shape = x.shape[:-1] + (n,)
    if y is None:
        y, ys = _new(torch, shape, x.dtype, device, stream), n
    else:
        _given(y, "y", shape, x.dtype, device)
        ys = _rows(y, "y")[2]
    rp, rs = _like(residual, "residual", y, device)
    if rows == 1 and not isinstance(kept, Quantized):  # (vectors: no workspace, whatever the operands start on)
        need = 0
    else:
        need = lib.ndvm_linear_workspace_bytes(act, rows, k, n, 0, int(_ready(x.data_ptr(), xs, rows, k) and _ready(w.data_ptr(), ws_, n, k)), 0)
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_linear_forward(code, _weight_type(code, None, bias), act, rows, k, n, x.data_ptr(), xs, w.data_ptr(), ws_,
                                     _vector(bias, "bias", n, device), rp, rs, y.data_ptr(), ys,
                                     *_linear_kept(torch, lib, kept, rows, n, device), wp, nbytes, _stream(torch, stream, device))
    if status:
        _check(status)
    return y


def linear_backward(dy, x, w, activation=None, wants=(True, True, True), dx=None, dw=None, dbias=None, btype=None, kept=None,
                    workspace=None, stream=None):
    """(dx, dw, dbias) of linear_forward; `wants` says which (the others are None; the residual's gradient is dy itself).
    x: as the forward call had it, or a Quantized of it.  kept: what the forward call kept (needed with an activation).
    dbias has dtype `btype` (x's by default)."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    device = _device(torch, w)
    code = _type(w, "w")
    act = _activation(activation)
    held = isinstance(x, Quantized)
    if held:
        _same_device(device, x.values, "x")
        rows, k, xs, xp = x.rows, x.cols, 0, None
        n, ws_ = _matrix(w, "w", w, k, device)
    else:
        _same_device(device, x, "x")
        rows, k, xs = _rows(x, "x")
        n, ws_ = _matrix(w, "w", x, k, device)
        xp = x.data_ptr()
    _given(dy, "dy", x.shape[:-1] + (n,), w.dtype, device)
    dys = _rows(dy, "dy")[2]
    bdtype = btype or w.dtype
    if dx is None and wants[0]:
        dx = _new(torch, x.shape, w.dtype, device, stream)
    if dw is None and wants[1]:
        dw = _new(torch, (n, k), w.dtype, device, stream)
    if dbias is None and wants[2]:
        dbias = _new(torch, (n,), bdtype, device, stream)
    dxp = dxs = dwp = dbp = None
    if dx is not None:
        _given(dx, "dx", x.shape, w.dtype, device)
        dxp, dxs = dx.data_ptr(), _rows(dx, "dx")[2]
    if dw is not None:
        _given(dw, "dw", (n, k), w.dtype, device)
        if not dw.is_contiguous():
            raise NdvmError(1, "dw must be contiguous")
        dwp = dw.data_ptr()
    if dbias is not None:
        _given(dbias, "dbias", (n,), bdtype, device)
        dbp = _vector(dbias, "dbias", n, device)
    ready = (held or _ready(xp, xs, rows, k)) and _ready(w.data_ptr(), ws_, n, k) and _ready(dy.data_ptr(), dys, rows, n)
    need = lib.ndvm_linear_workspace_bytes(act, rows, k, n, 1, int(ready), int(held))
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_linear_backward(code, _weight_type(code, None, dbias), act, rows, k, n, dy.data_ptr(), dys, xp, xs,
                                      x.values.data_ptr() if held else None, x.stride if held else 0,
                                      x.scales.data_ptr() if held else None, w.data_ptr(), ws_,
                                      *_linear_kept(torch, lib, kept, rows, n, device), dxp, dxs or 0, dwp, dbp, wp, nbytes,
                                      _stream(torch, stream, device))
    if status:
        _check(status)
    return dx, dw, dbias


def linear_quantized_forward(x, w, bias=None, activation=None, residual=None, dtype=None, y=None, workspace=None, stream=None):
    """linear_forward of x (..., k) and w (n, k) in 8-bit blocks (Quantized).  dtype: of y and residual, bfloat16 (the
    default where neither is given) or float16; bias of that type or float32."""
    torch = _torch_module or _start()
    lib = _nd._lib or load()
    if not isinstance(x, Quantized) or not isinstance(w, Quantized):
        raise NdvmError(1, "x and w must be Quantized")
    device = _device(torch, x.values)
    act = _activation(activation)
    if len(w.shape) != 2 or w.cols != x.cols:
        raise NdvmError(1, f"w must be an (n, {x.cols}) matrix")
    _same_device(device, w.values, "w")
    shape = x.shape[:-1] + (w.rows,)
    if y is None:
        y, ys = _new(torch, shape, dtype or (torch.bfloat16 if residual is None else residual.dtype), device, stream), w.rows
    else:
        _given(y, "y", shape, dtype or y.dtype, device)
        ys = _rows(y, "y")[2]
    code = _type(y, "y")
    rp, rs = _like(residual, "residual", y, device)
    need = lib.ndvm_linear_quantized_workspace_bytes(x.rows, x.cols, w.rows)
    ws, wp, nbytes = _workspace(torch, workspace, need, device, stream)
    status = lib.ndvm_linear_quantized(code, _weight_type(code, None, bias), act, x.rows, x.cols, w.rows, x.values.data_ptr(), x.stride,
                                       x.scales.data_ptr(), w.values.data_ptr(), w.stride, w.scales.data_ptr(),
                                       _vector(bias, "bias", w.rows, device), rp, rs, y.data_ptr(), ys, wp, nbytes,
                                       _stream(torch, stream, device))
    if status:
        _check(status)
    return y


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


def rms_norm(x, weight=None, eps=1e-6, residual=None):
    """s / sqrt(mean(s^2) + eps) * weight over the last dimension as a differentiable op, s = x.  With a residual, s = x +
    residual rounded to their type, and the result is (y, s)."""
    try:
        y = (_ops or _load_ops()).rms_norm(x, weight, eps, residual)
    except TypeError:
        y = None
    if y is None:
        _refuse(rms_norm_forward, x, weight, eps, residual)
    return y[0] if residual is None else tuple(y)


def linear(x, w, bias=None, activation=None, residual=None, keep=None):
    """act(x w^T + bias) + residual as a differentiable op (gradients of all four; 16-bit types, bias also float32).
    With an activation, x w^T + bias is held for the backward pass as float32.  keep="8bit": it and x are held as
    8-bit blocks instead (a bit over a byte an element each), and the gradients are those at what the blocks stand for."""
    if keep is not None and keep != "8bit":
        raise NdvmError(1, f"unknown keep {keep!r}: None or '8bit'")
    act = _activation(activation)
    try:
        y = (_ops or _load_ops()).linear(x, w, bias, act, residual, keep is not None)
    except TypeError:
        y = None
    return _refuse(linear_forward, x, w, bias, activation, residual) if y is None else y


def quantize(x):
    """8-bit blocks of x (..., cols), a Quantized: float32, float16, bfloat16, rows of any layout.  Has no gradient: raises
    where one would be recorded."""
    try:
        q = (_ops or _load_ops()).quantize(x)
    except TypeError:
        q = None
    return _refuse(quantize_forward, x) if q is None else Quantized._of(*q)


def rms_norm_quantized(x, weight=None, eps=1e-6, residual=None):
    """rms_norm whose y is a Quantized, made of what is not rounded in between; with a residual (y, s).  Has no gradient:
    raises where one would be recorded."""
    try:
        q = (_ops or _load_ops()).rms_norm_quantized(x, weight, eps, residual)
    except TypeError:
        q = None
    if q is None:
        _refuse(rms_norm_quantized_forward, x, weight, eps, residual)
    y = Quantized._of(*q[:5])
    return y if residual is None else (y, q[5])


def linear_quantized(x, w, bias=None, activation=None, residual=None, dtype=None):
    """act(x w^T + bias) + residual of x (..., k) and w (n, k) in 8-bit blocks (Quantized), in dtype: bfloat16 or float16
    (the residual's, or bfloat16, by default).  Has no gradient: raises where one would be recorded."""
    act = _activation(activation)
    y = None
    if isinstance(x, Quantized) and isinstance(w, Quantized):
        if dtype is None:
            dtype = (_torch_module or _start()).bfloat16 if residual is None else residual.dtype
        try:
            y = (_ops or _load_ops()).linear_quantized(x.values, x.scales, x.rows, x.cols, x.stride, w.values, w.scales, w.rows, w.cols, w.stride,
                                                       bias, act, residual, _types.get(dtype, 0))
        except TypeError:
            y = None
    return _refuse(linear_quantized_forward, x, w, bias, activation, residual, dtype) if y is None else y


def check_operators():
    """Synchronize and raise if a kernel of the operators gave up waiting since the last check."""
    _check(load().ndvm_check_operators())

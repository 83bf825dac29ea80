"""The root-mean-square norm, 8-bit blocks and dense layers without a GPU: arguments are checked before any launch."""
import pytest

F64, F32, F16, BF16 = 0, 1, 2, 3
OK, INVALID, UNSUPPORTED = 0, 1, 3
BIG = 1 << 62
A, B, C, D = 0x1000, 0x2000, 0x3000, 0x10000  # addresses that are never read: every call here is refused (or has nothing to do)


@pytest.fixture()
def lib(ndvm):
    return ndvm.load()


def rms(lib, dtype=BF16, wtype=BF16, rows=4, cols=8, x=A, xs=8, r=None, rs=0, w=B, eps=1e-5, y=C, ys=8, sum=None, ss=8, rstd=None):
    return lib.ndvm_rms_norm_forward(dtype, wtype, rows, cols, x, xs, r, rs, w, eps, y, ys, sum, ss, rstd, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F64}, UNSUPPORTED), ({"wtype": F16}, UNSUPPORTED), ({"dtype": F32}, UNSUPPORTED), ({"rows": -1}, INVALID), ({"cols": 0}, INVALID),
    ({"rows": BIG}, INVALID), ({"cols": BIG}, INVALID), ({"rows": (1 << 31) - 127}, INVALID), ({"x": None}, INVALID), ({"y": None}, INVALID),
    ({"x": A + 1}, INVALID), ({"y": C + 1}, INVALID), ({"w": B + 1}, INVALID), ({"rstd": C + 2}, INVALID), ({"xs": 7}, INVALID), ({"ys": 0}, INVALID),
    ({"r": A + 1, "rs": 8}, INVALID), ({"r": A, "rs": 7}, INVALID), ({"sum": C}, INVALID), ({"r": A, "rs": 8, "sum": C, "ss": 0}, INVALID),
    ({"r": A, "rs": 8, "sum": C + 1}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": float("nan")}, INVALID), ({"rows": 0, "x": None, "y": None}, OK)])
def test_rms_norm_forward_arguments(lib, change, status):
    assert rms(lib, **change) == status
    assert status == OK or lib.ndvm_last_error()


def rms_back(lib, dtype=BF16, wtype=F32, rows=4, cols=8, dy=A, ds=8, dsum=None, dss=8, s=A, xs=8, w=B, rstd=C, dx=C, dxs=8, dw=C, ws=A, nbytes=1 << 30):
    return lib.ndvm_rms_norm_backward(dtype, wtype, rows, cols, dy, ds, dsum, dss, s, xs, w, rstd, dx, dxs, dw, ws, nbytes, None)


@pytest.mark.parametrize("change", [
    {"dy": None}, {"s": None}, {"rstd": None}, {"rstd": C + 2}, {"ds": 3}, {"dsum": A + 1}, {"dsum": A, "dss": 7}, {"dxs": 0}, {"dx": C + 1},
    {"dw": C + 2}, {"ws": None}, {"ws": A + 8}, {"nbytes": 8}, {"cols": 0}, {"rows": -1}])
def test_rms_norm_backward_arguments(lib, change):
    assert rms_back(lib, **change) == INVALID


def test_rms_norm_workspace(lib):
    f = lib.ndvm_rms_norm_workspace_bytes
    assert f(-1, 8) == f(4, 0) == 0 and f(5, 8192) == 5 * 8192 * 4 and f(1 << 20, 8192) == 912 * 8192 * 4 and f(1000, 8193) == 64 * 8193 * 4


BLOCKS = [{"v": None}, {"s": None}, {"v": A + 8}, {"s": B + 4}, {"vs": 8}, {"vs": 24}, {"vs": -16}, {"rows": -1}, {"cols": 0}, {"rows": (1 << 31) - 127}]


def quant(lib, dtype=BF16, rows=4, cols=20, x=C, xs=20, v=A, vs=32, s=B):
    return lib.ndvm_quantize(dtype, rows, cols, x, xs, v, vs, s, None)


def dequant(lib, dtype=BF16, rows=4, cols=20, x=C, xs=20, v=A, vs=32, s=B):
    return lib.ndvm_dequantize(dtype, rows, cols, v, vs, s, x, xs, None)


def rms_quant(lib, dtype=BF16, rows=4, cols=20, x=C, xs=20, r=None, rs=20, v=A, vs=32, s=B, sum=None):
    return lib.ndvm_rms_norm_quantized(dtype, dtype, rows, cols, x, xs, r, rs, None, 1e-6, v, vs, s, sum, 20, None)


@pytest.mark.parametrize("call", [quant, dequant, rms_quant])
def test_blocks_arguments(lib, call):
    for change in BLOCKS + [{"x": None}, {"x": C + 1}, {"xs": 19}]:
        assert call(lib, **change) == INVALID, change
    assert call(lib, dtype=F64) == UNSUPPORTED and call(lib, rows=0, x=None, v=None, s=None) == OK
    if call is dequant:
        assert call(lib, xs=0) == INVALID  # (an output's rows are apart)
    if call is rms_quant:
        assert call(lib, sum=C) == INVALID  # (a sum goes with a residual)


def test_scale_bytes(lib):
    f = lib.ndvm_quantized_scale_bytes
    assert f(0, 8) == 0 and f(1, 1) == 512 and f(128, 128) == 512 and f(129, 128) == 1024 and f(129, 129) == 2048 and f(-1, 8) == 0


def lin(lib, dtype=BF16, btype=F32, act=0, rows=4, k=8, n=16, x=A, xs=8, w=B, ws=8, b=C, r=None, rs=16, y=C, ys=16, z=None, zv=None, zs=None, room=None, nbytes=0):
    return lib.ndvm_linear_forward(dtype, btype, act, rows, k, n, x, xs, w, ws, b, r, rs, y, ys, z, zv, zs, room, nbytes, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F32}, UNSUPPORTED), ({"dtype": F64}, UNSUPPORTED), ({"btype": F16}, UNSUPPORTED), ({"act": 5}, INVALID), ({"act": -1}, INVALID),
    ({"rows": -1}, INVALID), ({"k": 0}, INVALID), ({"n": 0}, INVALID), ({"rows": 1 << 31}, INVALID), ({"k": 1 << 31}, INVALID), ({"n": 1 << 31}, INVALID),
    ({"x": None}, INVALID), ({"w": None}, INVALID), ({"y": None}, INVALID), ({"b": C + 2}, INVALID), ({"xs": 7}, INVALID), ({"ws": 5}, INVALID),
    ({"ys": 15}, INVALID), ({"x": A + 1}, INVALID), ({"r": A, "rs": 7}, INVALID), ({"r": A + 1}, INVALID), ({"z": C + 4}, INVALID),
    ({"z": C, "zv": A, "zs": B}, INVALID), ({"zv": A}, INVALID), ({"zs": B}, INVALID), ({"zv": A + 8, "zs": B}, INVALID), ({"xs": 9}, INVALID),
    ({"w": B + 2}, INVALID), ({"rows": 0}, OK)])
def test_linear_forward_arguments(lib, change, status):
    assert lin(lib, **change) == status  # (operands that are not aligned need a workspace)


def lin_back(lib, dtype=BF16, btype=F32, act=0, rows=4, k=8, n=16, dy=A, ds=16, x=A, xs=8, xv=None, xvs=16, xsc=None, w=B, ws=8, z=C, zv=None, zs=None, dx=C,
             dxs=8, dw=C, db=C, room=D, nbytes=1 << 30):
    return lib.ndvm_linear_backward(dtype, btype, act, rows, k, n, dy, ds, x, xs, xv, xvs, xsc, w, ws, z, zv, zs, dx, dxs, dw, db, room, nbytes, None)


@pytest.mark.parametrize("change", [
    {"dy": None}, {"ds": 15}, {"dx": C + 1}, {"dxs": 0}, {"dw": C + 1}, {"db": C + 2}, {"room": None}, {"room": D + 16}, {"nbytes": 16}, {"act": 7}, {"k": 0},
    {"x": None}, {"w": None}, {"z": None}, {"z": C + 8}, {"zv": A, "zs": B}, {"z": None, "zv": A}, {"xv": A, "xsc": B}, {"x": None, "xv": A, "xsc": B + 4},
    {"x": None, "xv": A, "xsc": B, "xvs": 8}])
def test_linear_backward_arguments(lib, change):
    assert lin_back(lib, **change) == INVALID


def lin_quant(lib, dtype=BF16, btype=BF16, act=4, rows=4, k=8, n=16, xv=A, xs=16, xsc=B, wv=A, ws=16, wsc=B, b=None, r=None, rs=16, y=C, ys=16, room=None, nbytes=0):
    return lib.ndvm_linear_quantized(dtype, btype, act, rows, k, n, xv, xs, xsc, wv, ws, wsc, b, r, rs, y, ys, room, nbytes, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F32}, UNSUPPORTED), ({"btype": F16}, UNSUPPORTED), ({"act": 5}, INVALID), ({"k": 0}, INVALID), ({"xv": None}, INVALID), ({"xsc": None}, INVALID),
    ({"xs": 8}, INVALID), ({"xv": A + 8}, INVALID), ({"wv": None}, INVALID), ({"ws": 24}, INVALID), ({"wsc": B + 8}, INVALID), ({"y": None}, INVALID),
    ({"ys": 0}, INVALID), ({"r": A + 1}, INVALID), ({"k": 1 << 16, "xs": 1 << 16, "ws": 1 << 16}, INVALID), ({"rows": 0}, OK)])
def test_linear_quantized_arguments(lib, change, status):
    assert lin_quant(lib, **change) == status  # (a long contraction of few tiles is split, which needs a workspace)


def test_linear_workspace_sizes(lib):
    f = lib.ndvm_linear_workspace_bytes
    assert f(0, -1, 8, 8, 1, 1, 0) == f(0, 4, 0, 8, 1, 1, 0) == f(5, 4, 8, 8, 1, 1, 0) == f(0, 4, 8, 1 << 31, 1, 1, 0) == 0
    assert f(0, 1000, 256, 512, 1, 1, 0) >= 1000 * 512 * 2  # dz
    assert f(0, 1000, 256, 512, 1, 0, 0) > f(0, 1000, 256, 512, 1, 1, 1) > f(0, 1000, 256, 512, 1, 1, 0) > f(4, 1000, 256, 512, 1, 1, 0)
    assert lib.ndvm_linear_kept_stride(5) == 8 and lib.ndvm_linear_kept_stride(0) == 0
    assert lib.ndvm_linear_quantized_workspace_bytes(4, 8, 0) == 0


def test_ops_without_a_gpu_raise(ndvm):
    import torch
    x = torch.ones(4, 8)
    for call in (lambda: ndvm.rms_norm(x), lambda: ndvm.rms_norm(x, residual=x), lambda: ndvm.linear(x.half(), x.half()), lambda: ndvm.quantize(x),
                 lambda: ndvm.rms_norm_quantized(x), lambda: ndvm.linear_quantized(x, x), lambda: ndvm.Quantized(x, x)):
        with pytest.raises(ndvm.NdvmError):
            call()
    for call in (lambda: ndvm.linear(x, x, keep="4bit"), lambda: ndvm.linear(x, x, activation="tanh")):
        with pytest.raises(ndvm.NdvmError, match="unknown"):
            call()

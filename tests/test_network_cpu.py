"""The network operators' C ABI without a GPU: arguments are checked before any launch."""
import ctypes

import pytest

F64, F32, F16, BF16 = 0, 1, 2, 3
OK, INVALID, UNSUPPORTED = 0, 1, 3
BIG = 1 << 62


@pytest.fixture()
def lib(ndvm):
    return ndvm.load()


# addresses that are never read: every call here is refused (or has nothing to do)
A, B, C = 0x1000, 0x2000, 0x3000


def norm(lib, dtype=BF16, wtype=BF16, rows=4, cols=8, x=A, xs=8, w=B, b=B, eps=1e-5, y=C, ys=8, stats=None):
    return lib.ndvm_layer_norm_forward(dtype, wtype, rows, cols, x, xs, w, b, eps, y, ys, stats, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F64}, UNSUPPORTED), ({"dtype": 9}, UNSUPPORTED), ({"wtype": F16}, UNSUPPORTED), ({"dtype": F32}, UNSUPPORTED),
    ({"rows": -1}, INVALID), ({"cols": 0}, INVALID), ({"rows": BIG}, INVALID), ({"cols": BIG}, INVALID),
    ({"rows": 1 << 40, "cols": 1 << 40}, INVALID), ({"rows": 1 << 31}, INVALID), ({"x": None}, INVALID), ({"y": None}, INVALID), ({"x": A + 1}, INVALID),
    ({"y": C + 1}, INVALID), ({"w": B + 1}, INVALID), ({"stats": C + 2}, INVALID), ({"xs": 7}, INVALID), ({"xs": -8}, INVALID),
    ({"ys": 0}, INVALID), ({"ys": 7}, INVALID), ({"xs": BIG}, INVALID), ({"eps": -1.0}, INVALID), ({"eps": float("nan")}, INVALID),
    ({"eps": float("inf")}, INVALID), ({"rows": 0, "x": None, "y": None}, OK)])
def test_layer_norm_forward_arguments(lib, change, status):
    assert norm(lib, **change) == status
    assert status == OK or lib.ndvm_last_error()


def norm_back(lib, dtype=BF16, wtype=F32, rows=4, cols=8, dy=A, ds=8, x=A, xs=8, w=B, stats=C, dx=C, dxs=8, dw=C, db=C, ws=A,
              nbytes=1 << 30):
    return lib.ndvm_layer_norm_backward(dtype, wtype, rows, cols, dy, ds, x, xs, w, stats, dx, dxs, dw, db, ws, nbytes, None)


@pytest.mark.parametrize("change", [
    {"dy": None}, {"x": None}, {"stats": None}, {"stats": C + 2}, {"ds": 3}, {"dxs": 0}, {"dx": C + 1}, {"dw": C + 2},
    {"db": C + 1}, {"ws": None}, {"ws": A + 8}, {"nbytes": 8}, {"cols": 0}, {"rows": -1}])
def test_layer_norm_backward_arguments(lib, change):
    assert norm_back(lib, **change) == INVALID


def test_layer_norm_workspace_grows_with_the_columns(lib):
    assert lib.ndvm_layer_norm_workspace_bytes(-1, 8) == 0 and lib.ndvm_layer_norm_workspace_bytes(4, 0) == 0
    assert lib.ndvm_layer_norm_workspace_bytes(1000, 4096) >= 2 * 4096 * 4


def drop(lib, dtype=F32, rows=4, cols=8, x=A, xs=8, r=B, rs=8, p=0.5, seed=1, offset=0, y=C, ys=8):
    return lib.ndvm_dropout(dtype, rows, cols, x, xs, r, rs, p, seed, offset, y, ys, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F64}, UNSUPPORTED), ({"rows": -1}, INVALID), ({"cols": -1}, INVALID), ({"rows": BIG}, INVALID), ({"x": None}, INVALID),
    ({"y": None}, INVALID), ({"x": A + 2}, INVALID), ({"r": B + 2}, INVALID), ({"xs": 7}, INVALID), ({"rs": 1}, INVALID),
    ({"ys": 0}, INVALID), ({"p": 1.0}, INVALID), ({"p": -1e-9}, INVALID), ({"p": float("nan")}, INVALID), ({"offset": 2}, INVALID),
    ({"rows": 0}, OK), ({"cols": 0}, OK)])
def test_dropout_arguments(lib, change, status):
    assert drop(lib, **change) == status


def gate(lib, dtype=BF16, act=0, rows=4, k=8, n=16, x=A, xs=8, g=B, gs=8, u=B, us=8, h=C, hs=16, ws=None, nbytes=0):
    return lib.ndvm_gated_forward(dtype, act, rows, k, n, x, xs, g, gs, u, us, h, hs, ws, nbytes, None)


@pytest.mark.parametrize("change,status", [
    ({"dtype": F32}, UNSUPPORTED), ({"dtype": F64}, UNSUPPORTED), ({"act": 4}, INVALID), ({"act": -1}, INVALID), ({"rows": -1}, INVALID),
    ({"k": 0}, INVALID), ({"n": 0}, INVALID), ({"rows": 1 << 31}, INVALID), ({"k": 1 << 31}, INVALID), ({"n": 1 << 31}, INVALID),
    ({"x": None}, INVALID), ({"g": None}, INVALID), ({"u": None}, INVALID), ({"h": None}, INVALID), ({"xs": 7}, INVALID),
    ({"gs": 5}, INVALID), ({"us": -8}, INVALID), ({"hs": 15}, INVALID), ({"x": A + 1}, INVALID), ({"h": C + 1}, INVALID),
    ({"rows": 0}, OK)])
def test_gated_forward_arguments(lib, change, status):
    assert gate(lib, **change) == status


def gate_back(lib, dtype=BF16, act=0, rows=4, k=8, n=16, dh=A, ds=16, x=A, xs=8, g=B, gs=8, u=B, us=8, dx=C, dxs=8, dg=C, du=C,
              ws=0x10000, nbytes=1 << 30):
    return lib.ndvm_gated_backward(dtype, act, rows, k, n, dh, ds, x, xs, g, gs, u, us, dx, dxs, dg, du, ws, nbytes, None)


@pytest.mark.parametrize("change", [
    {"dh": None}, {"ds": 15}, {"dx": C + 1}, {"dxs": 0}, {"dg": C + 1}, {"du": C + 1}, {"ws": None}, {"ws": 0x10010},
    {"nbytes": 16}, {"act": 7}, {"k": 0}, {"x": None}])
def test_gated_backward_arguments(lib, change):
    assert gate_back(lib, **change) == INVALID


def test_gated_workspace_sizes(lib):
    f = lib.ndvm_gated_workspace_bytes
    assert f(-1, 8, 8, 1, 1) == f(4, 0, 8, 1, 1) == f(4, 8, 1 << 31, 1, 1) == 0
    assert f(1000, 256, 512, 1, 1) >= 2 * 1000 * 512 * 2  # dG and dU
    assert f(1000, 256, 512, 1, 0) >= f(1000, 256, 512, 1, 1)


def test_row_layouts(ndvm):
    import torch
    from paper_2607_03574_gb300.network import _rows
    t = torch.empty(3, 4, 10)
    assert _rows(t, "t") == (12, 10, 10) and _rows(t[..., :7], "t") == (12, 7, 10) and _rows(t[0, 0], "t") == (1, 10, 10)
    assert _rows(t[:, :1, :7], "t") == (3, 7, 40) and _rows(t[0, :1].expand(6, 10), "t") == (6, 10, 0)
    assert _rows(t[..., :1], "t") == (12, 1, 10)
    for bad in (t[:, :2, :7], t.transpose(1, 2), t[..., ::2], t.permute(1, 0, 2)):
        with pytest.raises(ndvm.NdvmError):
            _rows(bad, "t")


def test_ops_without_a_gpu_raise(ndvm):
    import torch
    x = torch.ones(4, 8)
    for call in (lambda: ndvm.layer_norm(x), lambda: ndvm.dropout(x, 0.1, 0), lambda: ndvm.gated(x, x, x)):
        with pytest.raises(ndvm.NdvmError):
            call()

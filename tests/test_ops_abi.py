"""The C ABI of include/lce_ops.h on the CPU: exported, named alike in the binding, and invalid calls
refused before anything is enqueued. No pointer below is dereferenced on the device: every call fails
validation, or has nothing to do."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WS_SMALL = 0, 1, 2, 3
FP32, BF16, FP16 = 0, 1, 2
X, R, G, Y, S, RS, SC, DY, DS, DX, DG, WS = (0x100000000 + k * 0x10000000 for k in range(12))  # far apart


@pytest.fixture(scope="module")
def lib():
    from paper_2603_16428_amd import ops
    return ops._library()


def test_header_and_binding_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lce_ops.h")).read(), flags=re.S)
    from paper_2603_16428_amd import ops
    names = sorted(set(re.findall(r"\b(lce_[a-z_]+)\s*\(", text)))
    assert names == sorted(ops.EXPORTED)
    for n in names:
        assert hasattr(lib, n), n


def _forward(lib, **kw):
    a = dict(x=X, x_ld=64, r=R, r_ld=64, g=G, N=4, H=64, dtype=BF16, eps=1e-5, y=Y, y_ld=64, s=S, s_ld=64, rstd=RS)
    a.update(kw)
    return lib.lce_add_rmsnorm_forward(a["x"], a["x_ld"], a["r"], a["r_ld"], a["g"], a["N"], a["H"], a["dtype"], a["eps"],
                                       a["y"], a["y_ld"], a["s"], a["s_ld"], a["rstd"], None)


def _quant(lib, **kw):
    a = dict(x=X, x_ld=64, r=R, r_ld=64, g=G, N=4, H=64, dtype=BF16, eps=1e-5, group=0, y=Y, y_ld=64, sc=SC, s=S, s_ld=64,
             rstd=RS)
    a.update(kw)
    return lib.lce_add_rmsnorm_quant(a["x"], a["x_ld"], a["r"], a["r_ld"], a["g"], a["N"], a["H"], a["dtype"], a["eps"],
                                     a["group"], a["y"], a["y_ld"], a["sc"], a["s"], a["s_ld"], a["rstd"], None)


ROWS = [
    (dict(x=None), INVALID), (dict(g=None), INVALID), (dict(y=None), INVALID), (dict(N=-1), INVALID), (dict(H=0), INVALID),
    (dict(dtype=3), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(x_ld=-1), INVALID), (dict(y_ld=63), INVALID), (dict(s_ld=63), INVALID), (dict(H=32769), UNSUPPORTED),
    (dict(N=1 << 31), UNSUPPORTED), (dict(x_ld=(1 << 30) + 1), UNSUPPORTED), (dict(N=0), OK), (dict(N=0, x=None), OK),
    (dict(x=X + 1), INVALID), (dict(g=G + 1), INVALID), (dict(s=S + 1), INVALID), (dict(rstd=RS + 2), INVALID),
    # Outputs over inputs or over each other, partly or with another pitch.
    (dict(y=X + 16), INVALID), (dict(y=X, y_ld=72), INVALID), (dict(s=R + 2), INVALID), (dict(y=S), INVALID), (dict(y=G), INVALID), (dict(y=G, N=1), INVALID),
    (dict(rstd=X + 8), INVALID), (dict(rstd=Y + 4 * 128 - 4), INVALID), (dict(s=Y + 64), INVALID),
    # Columns of one wider buffer that do overlap.
    (dict(x_ld=256, y=X + 2 * 63, y_ld=256), INVALID), (dict(x_ld=256, y=X - 2 * 63, y_ld=256), INVALID),
    (dict(x_ld=96, y=X + 2 * 64, y_ld=96), INVALID),
]


@pytest.mark.parametrize("kw,status", ROWS)
def test_forward_validation(lib, kw, status):
    assert _forward(lib, **kw) == status


@pytest.mark.parametrize("kw,status", [r for r in ROWS if r[0] not in (dict(y=S),)] + [
    (dict(group=16), INVALID), (dict(group=-1), INVALID), (dict(group=256), INVALID), (dict(sc=None), INVALID),
    (dict(sc=X), INVALID), (dict(sc=Y + 128), INVALID), (dict(y=X), INVALID), (dict(y=X, y_ld=128), INVALID),
    (dict(sc=RS + 12), INVALID)])
def test_quant_validation(lib, kw, status):
    if kw.get("rstd") == Y + 4 * 128 - 4:
        kw = dict(rstd=Y + 4 * 64 - 4)
    assert _quant(lib, **kw) == status


def _backward(lib, **kw):
    a = dict(dy=DY, dy_ld=64, ds=DS, ds_ld=64, x=X, x_ld=64, r=R, r_ld=64, g=G, rstd=RS, N=4, H=64, dtype=BF16, dx=DX, dx_ld=64, dg=DG,
             ws=WS, wsb=1 << 20)
    a.update(kw)
    return lib.lce_add_rmsnorm_backward(a["dy"], a["dy_ld"], a["ds"], a["ds_ld"], a["x"], a["x_ld"], a["r"], a["r_ld"], a["g"],
                                        a["rstd"], a["N"], a["H"], a["dtype"], a["dx"], a["dx_ld"], a["dg"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INVALID), (dict(x=None), INVALID), (dict(g=None), INVALID), (dict(rstd=None), INVALID),
    (dict(dx=None), INVALID), (dict(N=-1), INVALID), (dict(H=0), INVALID), (dict(dtype=9), INVALID),
    (dict(dy_ld=-4), INVALID), (dict(dx_ld=60), INVALID), (dict(H=40000), UNSUPPORTED), (dict(ws=None), WS_SMALL),
    (dict(wsb=8), WS_SMALL), (dict(ws=WS + 64), INVALID), (dict(ws=X), INVALID), (dict(ws=DX), INVALID), (dict(dy=DY + 1), INVALID),
    (dict(rstd=RS + 1), INVALID), (dict(dg=DG + 1), INVALID), (dict(dx=DY + 2), INVALID), (dict(dx=X, dx_ld=72), INVALID), (dict(dx=R - 2), INVALID), (dict(dx=G, N=1), INVALID), (dict(dg=G), INVALID),
    (dict(dg=DX), INVALID), (dict(dx=RS), INVALID), (dict(N=0, dg=None), OK), (dict(N=0, dg=None, ws=None), OK),
])
def test_backward_validation(lib, kw, status):
    assert _backward(lib, **kw) == status


def test_backward_workspace(lib):
    f = lib.lce_add_rmsnorm_workspace_size
    assert f(-1, 64, BF16) == 0 and f(4, 0, BF16) == 0 and f(4, 64, 5) == 0 and f(4, 32769, BF16) == 0
    assert f(0, 64, BF16) > 0 and f(1, 4096, BF16) >= 4096 * 4
    # At most 1024 rows of partial sums, whatever N is.
    assert f(1 << 30, 4096, BF16) <= 1024 * 4096 * 4
    assert f(1 << 30, 32768, FP32) <= 1024 * 32768 * 4


@pytest.mark.parametrize("H", [5, 64, 128, 200, 256, 500, 512, 768, 1000, 1024, 2048, 4096, 6000, 8192, 12288, 16384, 20000, 32768])
def test_backward_workspace_of_a_batch_serves_smaller_ones(lib, H):
    size = lib.lce_add_rmsnorm_workspace_size
    sizes = [size(N, H, BF16) for N in [*range(5000), *range(5000, 300000, 997), 1 << 30]]
    assert sizes == sorted(sizes)
    # And the call takes it (up to the check behind the size's: an unaligned workspace).
    for N in (1, 15, 100, 127, 128, 255):
        assert _backward(lib, N=N, H=H, dtype=BF16, wsb=size(256, H, BF16), ws=WS + 64, **{k: H for k in ("dy_ld", "ds_ld", "x_ld", "r_ld", "dx_ld")}) == INVALID


class Tensor(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32), ("reserved", ctypes.c_int32)]


def _list(*entries):
    return (Tensor * len(entries))(*[Tensor(p, n, t, 0) for p, n, t in entries])


def _clip(lib, grads, out=None, count=None, kind=0, max_norm=1.0, norm=SC, ws=WS, wsb=1 << 20):
    outs = None if out is None else (ctypes.c_void_p * len(out))(*out)
    return lib.lce_clip_grad_norm(grads, len(grads) if count is None else count, kind, max_norm, outs, norm, ws, wsb, None)


def test_clip_validation(lib):
    a, b = (X, 100, BF16), (R, 100, FP32)
    assert _clip(lib, _list(a), count=0) == INVALID and _clip(lib, _list(a), count=-1) == INVALID
    assert lib.lce_clip_grad_norm(None, 1, 0, 1.0, None, SC, WS, 1 << 20, None) == INVALID
    assert _clip(lib, _list(a), kind=2) == INVALID and _clip(lib, _list(a), norm=None) == INVALID
    assert _clip(lib, _list(a), max_norm=-1.0) == INVALID and _clip(lib, _list(a), max_norm=float("nan")) == INVALID
    assert _clip(lib, _list((None, 1, BF16))) == INVALID and _clip(lib, _list((X, -1, BF16))) == INVALID
    assert _clip(lib, _list((X, 1, 3))) == INVALID
    assert _clip(lib, _list((X + 1, 8, BF16))) == INVALID and _clip(lib, _list((X + 2, 8, FP32))) == INVALID
    assert _clip(lib, _list(a), out=[Y + 1]) == INVALID and _clip(lib, _list(a), norm=SC + 2) == INVALID
    assert _clip(lib, _list(a), norm=X + 196) == INVALID and _clip(lib, _list(a), ws=X - 256) == INVALID
    assert _clip(lib, _list(a), ws=WS + 8) == INVALID
    assert _clip(lib, _list(a), ws=None) == WS_SMALL and _clip(lib, _list(a), wsb=64) == WS_SMALL
    assert _clip(lib, _list(*[(X + 512 * k, 100, BF16) for k in range(300)]),
                 wsb=lib.lce_grad_norm_workspace_size(112)) == WS_SMALL
    assert _clip(lib, _list((X, 1 << 45, BF16))) == UNSUPPORTED
    assert _clip(lib, _list((X, 1 << 60, BF16))) == UNSUPPORTED
    # Written memory that overlaps: the same tensor twice, a part of another, outputs over other inputs or outputs.
    assert _clip(lib, _list(a, b, a)) == INVALID
    assert _clip(lib, _list(a, (X + 198, 1, BF16))) == INVALID
    assert _clip(lib, _list((X + 100, 100, BF16), a)) == INVALID
    assert _clip(lib, _list(a, b), out=[Y, Y + 100]) == INVALID
    assert _clip(lib, _list(a, b), out=[R, Y]) == INVALID
    assert _clip(lib, _list(a, b), out=[X + 2, Y]) == INVALID
    assert _clip(lib, _list(a, b), out=[Y, None]) == INVALID
    # A read of the one by the other: the first's output is the second's input.
    assert _clip(lib, _list(a, a), out=[X, Y]) == INVALID


def test_grad_norm_validation(lib):
    a = (X, 100, BF16)
    f = lib.lce_grad_norm
    assert f(_list(a), 0, 0, SC, WS, 1 << 20, None) == INVALID and f(None, 1, 0, SC, WS, 1 << 20, None) == INVALID
    assert f(_list(a), 1, 7, SC, WS, 1 << 20, None) == INVALID and f(_list(a), 1, 0, None, WS, 1 << 20, None) == INVALID
    assert f(_list(a), 1, 0, SC, None, 1 << 20, None) == WS_SMALL and f(_list(a), 1, 0, SC, WS, 0, None) == WS_SMALL
    assert lib.lce_grad_norm_workspace_size(0) == 0 and lib.lce_grad_norm_workspace_size(-3) == 0
    sizes = [lib.lce_grad_norm_workspace_size(n) for n in (1, 112, 113, 1000)]
    assert 0 < sizes[0] == sizes[1] < sizes[2] < sizes[3]


@pytest.mark.parametrize("count", [1, 200])
def test_grad_norm_writes_no_gradient(lib, count):
    """The norm and the workspace (its table of more than 112 gradients too) overlap neither a gradient nor each other.
    (Gradients that are only read may overlap: the GPU tests read one twice.)"""
    need = lib.lce_grad_norm_workspace_size(count)
    grads = [(X + 4096 * k, 100, BF16) for k in range(count - 1)] + [(R, 1 << 20, FP32)]
    for entries in (grads, grads[::-1]):
        for norm, ws in ((R, WS), (R + (4 << 20) - 4, WS), (SC, R), (SC, R + (4 << 20) - 256), (SC, R - need + 256), (WS, WS), (WS + need - 4, WS)):
            assert lib.lce_grad_norm(_list(*entries), count, 0, norm, ws, 1 << 20, None) == INVALID


def test_binding_refuses():
    import torch
    import paper_2603_16428_amd as lce
    x, g = torch.zeros(2, 8), torch.zeros(8)
    for call in (lambda: lce.add_rmsnorm_forward(x, x, g), lambda: lce.add_rmsnorm_quant(x, x, g),
                 lambda: lce.add_rmsnorm(x, None, g), lambda: lce.rmsnorm(x, g), lambda: lce.add_rmsnorm_quant(x, x, g, group_size=7),
                 lambda: lce.add_rmsnorm_backward(x, x, x, x, g, g), lambda: lce.grad_norm([]), lambda: lce.grad_norm([None]),
                 lambda: lce.grad_norm([x]), lambda: lce.clip_grad_norm_([x], 1.0), lambda: lce.clip_grad_norm(x, 1.0),
                 lambda: lce.grad_norm([x], 1.0), lambda: lce.clip_grad_norm_([x], 1.0, 3.0)):
        with pytest.raises(ValueError):
            call()


def test_row_pitch():
    """The rows that a tensor's leading dimensions make up (the pitch the kernels get)."""
    import torch
    from paper_2603_16428_amd.ops import _dense, _pitch
    t = torch.zeros(3, 4, 16)
    assert _pitch(t, "t") == 16 and _pitch(t[:, :, 2:7], "t") == 16 and _pitch(t[:, 1], "t") == 64
    assert _pitch(t[0, 0], "t") == 16 and _pitch(t[1:2, :, :5], "t") == 16 and _pitch(t[:, 1:2, :5], "t") == 64
    assert _pitch(torch.zeros(1, 8).expand(5, 8), "t") == 0 and _pitch(torch.zeros(4, 1), "t") == 1
    for bad in (t[:, :, ::2], t.transpose(1, 2), t[:, :3, :5], t.transpose(0, 1), torch.zeros(3, 1, 8).expand(3, 4, 8)):
        with pytest.raises(ValueError):
            _pitch(bad, "t")
    assert _dense(t.transpose(0, 2)) and _dense(t[1:]) and not _dense(t[:, 1:]) and not _dense(torch.zeros(1).expand(3))
    assert _dense(t.permute(2, 0, 1)[3:4, :1, :1]) and not _dense(torch.zeros(6).as_strided((2, 2), (1, 1)))

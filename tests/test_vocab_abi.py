"""The C ABI of include/lce_vocab.h on the CPU: exported, named alike in the binding, and invalid calls refused before
anything is enqueued. No pointer below is dereferenced: every call fails validation, or has nothing to do."""
import ctypes
import math
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED, WS_SMALL = 0, 1, 2, 3
FP32, BF16, FP16 = 0, 1, 2
TOK, W, OUT, G, DW, WS, C, S, C2, S2, U, LP, ROW = (0x100000000 + k * 0x10000000 for k in range(13))  # far apart
BIG = 1 << 27


@pytest.fixture(scope="module")
def lib():
    from paper_2603_16428_amd import vocab
    return vocab._library()


def test_header_and_binding_agree(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "lce_vocab.h")).read(), flags=re.S)
    from paper_2603_16428_amd import vocab
    names = sorted(set(re.findall(r"\b(lce_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(vocab.EXPORTED)
    for n in names:
        assert hasattr(lib, n), n


def _forward(lib, **kw):
    a = dict(tok=TOK, size=8, N=4, w=W, ld=64, V=100, H=64, dtype=BF16, scale=1.0, out=OUT, out_ld=64) | kw
    return lib.lce_embedding_forward(a["tok"], a["size"], a["N"], a["w"], a["ld"], a["V"], a["H"], a["dtype"], a["scale"], a["out"], a["out_ld"], None)


COMMON = [(dict(size=2), INVALID), (dict(N=-1), INVALID), (dict(V=0), INVALID), (dict(H=0), INVALID), (dict(dtype=3), INVALID),
          (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(V=1 << 31), UNSUPPORTED), (dict(H=(1 << 20) + 1), UNSUPPORTED),
          (dict(N=1 << 31), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(tok=None), INVALID), (dict(w=None), INVALID), (dict(out=None), INVALID), (dict(ld=-1), INVALID), (dict(out_ld=63), INVALID), (dict(N=0), OK),
    (dict(tok=TOK + 4), INVALID), (dict(w=W + 1), INVALID), (dict(out=OUT + 1), INVALID), (dict(out=W + 128), INVALID), (dict(out=TOK + 16), INVALID),
    (dict(out_ld=(1 << 30) + 1), UNSUPPORTED)])
def test_embedding_forward(lib, kw, status):
    assert _forward(lib, **kw) == status


def _backward(lib, **kw):
    a = dict(g=G, ld=64, tok=TOK, size=8, N=4, V=100, H=64, dtype=BF16, scale=1.0, pad=-1, dw=DW, dw_ld=64, acc=0, ws=WS, wsb=1 << 20) | kw
    return lib.lce_embedding_backward(a["g"], a["ld"], a["tok"], a["size"], a["N"], a["V"], a["H"], a["dtype"], a["scale"], a["pad"], a["dw"], a["dw_ld"],
                                      a["acc"], a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(g=None), INVALID), (dict(tok=None), INVALID), (dict(dw=None), INVALID), (dict(pad=-2), INVALID), (dict(pad=100), INVALID), (dict(ld=-1), INVALID),
    (dict(dw_ld=63), INVALID), (dict(ws=None), WS_SMALL), (dict(wsb=100), WS_SMALL), (dict(ws=WS + 64), INVALID), (dict(dw=G), INVALID), (dict(dw=TOK), INVALID),
    (dict(ws=DW), INVALID), (dict(ws=G), INVALID), (dict(ws=TOK), INVALID), (dict(N=0, acc=1), OK), (dict(N=0, acc=1, g=None, tok=None, ws=None), OK),
    (dict(tok=TOK + 2), INVALID), (dict(g=G + 1), INVALID), (dict(dw=DW + 1), INVALID), (dict(N=(1 << 28) + 1), UNSUPPORTED)])
def test_embedding_backward(lib, kw, status):
    assert _backward(lib, **kw) == status


def test_embedding_workspace(lib):
    f = lib.lce_embedding_workspace_size
    assert f(-1, 64) == 0 and f(4, 0) == 0 and f((1 << 28) + 1, 64) == 0 and f(4, (1 << 20) + 1) == 0 and f(0, 64) > 0
    for H in (1, 7, 64, 768, 4096):
        sizes = [f(N, H) for N in [*range(0, 3000, 7), *range(30000, 70000, 13), 1 << 20, 1 << 28]]
        assert sizes == sorted(sizes)
    for N in (1, 100, 40000):
        sizes = [f(N, H) for H in range(1, 300)]
        assert sizes == sorted(sizes)


MX = [(dict(N=-1), INVALID), (dict(H=0), INVALID), (dict(H=16), INVALID), (dict(H=48), INVALID), (dict(dtype=4), INVALID), (dict(H=(1 << 20) + 32), UNSUPPORTED),
      (dict(N=1 << 31), UNSUPPORTED), (dict(c=None), INVALID), (dict(s=None), INVALID), (dict(c=C + 8), INVALID), (dict(x=None), INVALID), (dict(x=W + 1), INVALID),
      (dict(c=W), INVALID), (dict(s=W + 4), INVALID), (dict(N=0), OK)]


@pytest.mark.parametrize("kw,status", MX + [(dict(ld=-1), INVALID), (dict(s=C), INVALID), (dict(x=C), INVALID)])
def test_mxfp4_quantize(lib, kw, status):
    a = dict(x=W, ld=64, N=4, H=64, dtype=BF16, c=C, s=S) | kw
    assert lib.lce_mxfp4_quantize(a["x"], a["ld"], a["N"], a["H"], a["dtype"], a["c"], a["s"], None) == status


@pytest.mark.parametrize("kw,status", MX + [(dict(ld=63), INVALID)])
def test_mxfp4_dequantize(lib, kw, status):
    a = dict(x=W, ld=64, N=4, H=64, dtype=BF16, c=C, s=S) | kw
    assert lib.lce_mxfp4_dequantize(a["c"], a["s"], a["N"], a["H"], a["dtype"], a["x"], a["ld"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), INVALID), (dict(V=-1), INVALID), (dict(H=40), INVALID), (dict(dtype=-1), INVALID), (dict(M=1 << 31), UNSUPPORTED), (dict(V=1 << 31), UNSUPPORTED),
    (dict(H=(1 << 20) + 32), UNSUPPORTED), (dict(M=0), OK), (dict(V=0), OK), (dict(c=None), INVALID), (dict(s=None), INVALID), (dict(wc=None), INVALID),
    (dict(ws=None), INVALID), (dict(out=None), INVALID), (dict(c=C + 1), INVALID), (dict(wc=C2 + 8), INVALID), (dict(out_ld=99), INVALID), (dict(out=OUT + 1), INVALID),
    (dict(out=C), INVALID), (dict(out=S2), INVALID), (dict(out=C2 + 64), INVALID), (dict(M=1 << 30, V=1 << 30, out_ld=1 << 30), UNSUPPORTED)])
def test_mxfp4_matmul(lib, kw, status):
    a = dict(c=C, s=S, M=4, wc=C2, ws=S2, V=100, H=64, dtype=BF16, out=OUT, out_ld=100) | kw
    if a["M"] == 1 << 30:  # too many tiles; nothing near anything else
        a |= dict(c=1 << 50, s=1 << 51, wc=1 << 52, ws=1 << 53, out=1 << 60)
    assert lib.lce_mxfp4_matmul(a["c"], a["s"], a["M"], a["wc"], a["ws"], a["V"], a["H"], a["dtype"], a["out"], a["out_ld"], None) == status


def _sample(lib, t=1.0, p=1.0, m=0.0, k=0, ts=None, ps=None, ms=None, ks=None, settings=True, **kw):
    from paper_2603_16428_amd.vocab import SampleSettings
    a = dict(z=W, ld=1000, N=4, V=1000, dtype=BF16, u=U, tok=TOK, lp=LP, ws=WS, wsb=1 << 20) | kw
    return lib.lce_sample(a["z"], a["ld"], a["N"], a["V"], a["dtype"], a["u"], SampleSettings(t, p, m, k, ts, ps, ms, ks) if settings else None, a["tok"], a["lp"],
                          a["ws"], a["wsb"], None)


@pytest.mark.parametrize("kw,status", [
    (dict(N=-1), INVALID), (dict(V=0), INVALID), (dict(V=(1 << 20) + 1), UNSUPPORTED), (dict(N=(1 << 16) + 1), UNSUPPORTED), (dict(dtype=5), INVALID),
    (dict(settings=False), INVALID), (dict(t=-1.0), INVALID), (dict(t=math.nan), INVALID), (dict(p=-0.1), INVALID), (dict(p=math.nan), INVALID), (dict(m=-0.1), INVALID),
    (dict(m=1.5), INVALID), (dict(m=math.nan), INVALID), (dict(k=-1), INVALID), (dict(N=0), OK), (dict(N=0, z=None), OK), (dict(N=0, t=-1.0), INVALID),
    (dict(z=None), INVALID), (dict(u=None), INVALID), (dict(tok=None), INVALID), (dict(z=W + 1), INVALID), (dict(u=U + 2), INVALID), (dict(tok=TOK + 4), INVALID),
    (dict(lp=LP + 2), INVALID), (dict(ts=ROW + 2), INVALID), (dict(ks=ROW + 1), INVALID), (dict(ld=-1), INVALID), (dict(ws=None), WS_SMALL), (dict(wsb=8), WS_SMALL),
    (dict(ws=WS + 8), INVALID), (dict(tok=W + 8), INVALID), (dict(lp=U), INVALID), (dict(lp=TOK + 4), INVALID), (dict(ws=W), INVALID), (dict(ws=TOK), INVALID),
    (dict(lp=ROW, ps=ROW), INVALID), (dict(tok=ROW, ks=ROW), INVALID)])
def test_sample(lib, kw, status):
    assert _sample(lib, **kw) == status


def test_sample_workspace(lib):
    f = lib.lce_sample_workspace_size
    assert f(-1, 5) == 0 and f(1, 0) == 0 and f(1, (1 << 20) + 1) == 0 and f((1 << 16) + 1, 5) == 0 and f(0, 5) > 0
    sizes = [f(N, 50257) for N in range(100)]
    assert sizes == sorted(sizes)


def test_binding_refuses():
    import paper_2603_16428_amd as lce
    x, t = torch.zeros(2, 32), torch.zeros(2, dtype=torch.int64)
    c, s = torch.zeros(2, 16, dtype=torch.uint8), torch.zeros(2, 1, dtype=torch.uint8)
    for call in (lambda: lce.embedding_forward(t, x), lambda: lce.embedding(t, x), lambda: lce.embedding_backward(x, t, 5), lambda: lce.mxfp4_quantize(x),
                 lambda: lce.mxfp4_dequantize(c, s), lambda: lce.mxfp4_matmul(c, s, c, s), lambda: lce.mxfp4_linear(x, c, s), lambda: lce.sample(x, torch.zeros(2))):
        with pytest.raises(ValueError):
            call()


def test_mxfp4_matmul_of_too_many_tiles(lib):
    """The header's limit, on both sides of 128 rows (at the limit itself a launch is tried, which needs a GPU)."""
    text = open(os.path.join(ROOT, "include", "lce_vocab.h")).read()
    most = eval(re.search(r"LCE_MXFP4_MAX_TILES \((.*)\)", text).group(1))
    far = [(1 << 50) + k * (1 << 45) for k in range(5)]

    def call(M, V):
        return lib.lce_mxfp4_matmul(far[0], far[1], M, far[2], far[3], V, 32, BF16, far[4], V, None)

    for M, V in ((49, 256 * most + 1), (128, 256 * most + 1), (129, 256 * most + 1), (256 * most + 1, 1), (256 * 2048 + 1, 256 * (most // 2048)),
                 (256 * 2048, 256 * (most // 2048) + 1)):
        assert call(M, V) == UNSUPPORTED, (M, V)

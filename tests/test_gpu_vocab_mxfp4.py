"""Rows in 4 bits, their values and their product on the GPU against float64.

Quantising is exact but for the rounding to a code, so codes and scales are equal to the definition's. A product's bound: an fp32 sum of
K terms, in whatever order, is at most K w off, relative to the sum of the terms' magnitudes (w = 2^-24), and rounded once.
"""
import math

import pytest
import torch

from oracle import vocab as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
W = 2.0 ** -24


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


BORDERS = [0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.5, 0.2, 0.3, 0.7, 0.8, 1.2, 1.3, 1.7, 1.8, 2.4, 2.6, 3.4, 3.6, 4.9, 5.1, 6.5]


@pytest.mark.parametrize("dtype", list(DT))
def test_every_border(lce, dtype):
    """Every border between two codes and both sides of it, at scales from the smallest to the largest of the type."""
    b = torch.tensor(BORDERS, dtype=torch.float64)
    powers = {"fp16": (-24, -14, -3, 0, 5, 13), "bf16": (-133, -126, -125, -60, 0, 60, 125), "fp32": (-149, -140, -127, -126, -125, 0, 60, 125)}[dtype]
    rows = [s * b * 2.0 ** p for p in powers for s in (1, -1)] + [torch.zeros(32), -torch.zeros(32)]
    x = torch.stack([r.double() for r in rows]).to(DT[dtype])
    codes, scales = lce.mxfp4_quantize(x.cuda())
    want_codes, want_scales = O.mxfp4_quantize(x)
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), O.mxfp4_pack(want_codes))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("H", [32, 64, 96, 128, 160, 1024, 1056, 2048, 4096, 4128, 8192])
def test_quantize(lce, H, dtype):
    g = torch.Generator().manual_seed(H)
    x = (torch.randn((9, H), generator=g) * torch.exp(3 * torch.randn((9, H // 32, 1), generator=g)).expand(9, H // 32, 32).reshape(9, H)).to(DT[dtype])
    codes, scales = lce.mxfp4_quantize(x.cuda())
    want_codes, want_scales = O.mxfp4_quantize(x)
    assert torch.equal(scales.cpu(), want_scales) and torch.equal(codes.cpu(), O.mxfp4_pack(want_codes))


def test_quantize_values_that_are_not_finite(lce):
    x = torch.ones((4, 96), device="cuda")
    x[0, 33], x[1, 0], x[2, 95] = math.nan, math.inf, -math.inf
    codes, scales = lce.mxfp4_quantize(x)
    assert scales.tolist() == [[125, 255, 125], [255, 125, 125], [125, 125, 255], [125, 125, 125]]
    assert not bool(codes[0, 16:32].any() or codes[1, :16].any() or codes[2, 32:].any())
    y = lce.mxfp4_dequantize(codes, scales, torch.float32)
    assert torch.equal(y.isnan(), (scales == 255).repeat_interleave(32, 1))
    # A product's values that the group enters are NaN, and no others.
    out = lce.mxfp4_matmul(codes, scales, *lce.mxfp4_quantize(torch.ones((70, 96), device="cuda")), torch.float32)
    assert torch.equal(out.isnan().all(1), torch.tensor([True, True, True, False], device="cuda")) and bool((out[3] == 96).all())
    out = lce.mxfp4_matmul(*lce.mxfp4_quantize(torch.ones((70, 96), device="cuda")), codes, scales, torch.float32)
    assert torch.equal(out.isnan().all(0), torch.tensor([True, True, True, False], device="cuda")) and bool((out[:, 3] == 96).all())


def test_shapes_strides_and_alignment(lce):
    wide = torch.randn((24, 500), device="cuda").to(torch.bfloat16)
    for at, H in ((1, 64), (8, 96), (3, 160)):
        x = wide[:, at:at + H]
        codes, scales = lce.mxfp4_quantize(x.view(2, 3, 4, H))
        assert codes.shape == (2, 3, 4, H // 2) and scales.shape == (2, 3, 4, H // 32)
        same = lce.mxfp4_quantize(x.contiguous())
        assert torch.equal(codes.view(24, -1), same[0]) and torch.equal(scales.view(24, -1), same[1])
        buf = torch.full((24, 400), 7.0, dtype=torch.float16, device="cuda")
        out = buf[:, 3:3 + H]
        lce.mxfp4_dequantize(codes.view(24, -1), scales.view(24, -1), torch.float16, out=out)
        assert torch.equal(out.double().cpu(), O.mxfp4_values(*same))
        assert bool((buf[:, :3] == 7).all() and (buf[:, 3 + H:] == 7).all())
        given = torch.empty_like(same[0]), torch.empty_like(same[1])
        assert lce.mxfp4_quantize(x, *given)[0] is given[0] and torch.equal(given[1], same[1])
    row = wide[3, :64]
    codes, scales = lce.mxfp4_quantize(row)
    assert codes.shape == (32,) and scales.shape == (2,) and lce.mxfp4_dequantize(codes, scales).shape == (64,)
    none = lce.mxfp4_quantize(wide[:0, :64])
    assert none[0].shape == (0, 32) and lce.mxfp4_dequantize(*none).shape == (0, 64) and lce.mxfp4_matmul(*none, *lce.mxfp4_quantize(wide[:, :64])).shape == (0, 24)
    assert lce.mxfp4_matmul(*lce.mxfp4_quantize(wide[:, :64]), *none).shape == (24, 0)


@pytest.mark.parametrize("dtype", list(DT))
def test_every_code_and_scale(lce, dtype):
    codes = torch.arange(256, dtype=torch.uint8).view(1, 16, 16).expand(256, 16, 16).reshape(256, 256).contiguous()
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1).expand(256, 16).contiguous()
    got = lce.mxfp4_dequantize(codes.cuda(), scales.cuda(), DT[dtype]).cpu()
    want = O.mxfp4_values(codes, scales).to(DT[dtype])
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0).double(), want.nan_to_num(0.0).double())


def _packed(N, H, seed, least=118):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, 256, (N, H // 2), generator=g, dtype=torch.uint8), torch.randint(least, least + 16, (N, H // 32), generator=g, dtype=torch.uint8)


def _check_product(got, x, w):
    a, b = O.mxfp4_values(*x), O.mxfp4_values(*w)
    want, size = a @ b.T, a.abs() @ b.abs().T
    got = got.cpu()
    u = torch.finfo(got.dtype).eps / 2
    bound = a.shape[1] * W * size
    step = 2.0 ** -25 if got.dtype is torch.float16 else 0.0  # half a step of its smallest values
    off = (got.double() - want).abs() - (bound + u * (want.abs() + bound) + step)
    assert got.shape == want.shape and not bool((off > 0).any()), float(off.max())


# Rows of x around the borders of the tiles (16, 32, 48; 128; 256), rows of W around 32, 64 and 256 (and 16384, from where a workgroup
# takes 64), more and fewer than 128 tiles of 256 x 256, K with whole and part steps of 256, one and several runs of 8192, scales' rows at any alignment.
@pytest.mark.parametrize("M,H,V", [
    (1, 32, 1), (1, 32, 5), (1, 256, 32), (2, 64, 33), (16, 96, 31), (17, 288, 100), (16, 1024, 1000), (32, 4096, 65), (33, 800, 63), (48, 2080, 130), (5, 8192, 66),
    (5, 8224, 66), (3, 16672, 40), (48, 20480, 33), (1, 1024, 16385), (5, 96, 16384), (20, 288, 16400), (40, 544, 16390), (48, 768, 16448), (49, 32, 7), (64, 4096, 257),
    (65, 256, 256), (100, 288, 255), (128, 512, 300), (129, 32, 515), (129, 2048, 64), (256, 96, 257), (257, 1056, 300), (300, 4096, 513), (600, 160, 900), (1, 1 << 20, 3), (60, 1 << 20, 2),
    (129, 288, 33000), (300, 96, 16500), (700, 1056, 11100), (1300, 32, 6000)])
@pytest.mark.parametrize("dtype", list(DT))
def test_product(lce, M, H, V, dtype):
    least = 112 if dtype == "fp16" else 118  # so that no sum leaves its range
    x, w = _packed(M, H, 1, least), _packed(V, H, 2, least)
    _check_product(lce.mxfp4_matmul(*(t.cuda() for t in x), *(t.cuda() for t in w), DT[dtype]), x, w)


@pytest.mark.parametrize("M", [3, 60, 200])
def test_scales_at_their_ends(lce, M):
    """Scale bytes 0 and 254: products far below and far above fp32's range are 0 and infinite, others are right."""
    x = torch.full((M, 16), 0x22, dtype=torch.uint8, device="cuda")  # ones
    lo, mid, hi = (torch.full((M, 1), b, dtype=torch.uint8, device="cuda") for b in (0, 127, 254))
    w = x[:1].expand(40, 16).contiguous()
    for a, b, want in ((lo, lo, 0.0), (mid, mid, 32.0), (hi, lo, 32.0), (hi, hi, math.inf), (lo, mid, 2.0 ** -122)):
        got = lce.mxfp4_matmul(x, a, w, b[:1].expand(40, 1).contiguous(), torch.float32)
        assert bool((got == want).all()), (want, got[0, 0])


@pytest.mark.parametrize("M", [7, 70, 300])
def test_product_into_a_wider_buffer(lce, M):
    x, w = _packed(M, 320, 3), _packed(301, 320, 4)
    buf = torch.full((M, 500), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, 5:306]
    assert lce.mxfp4_matmul(*(t.cuda() for t in x), *(t.cuda() for t in w), out=out) is out
    _check_product(out, x, w)
    assert bool((buf[:, :5] == 7).all() and (buf[:, 306:] == 7).all())


def test_linear(lce):
    g = torch.Generator().manual_seed(5)
    hidden, weight = torch.randn((2, 3, 320), generator=g).to(torch.bfloat16).cuda(), torch.randn((100, 320), generator=g).cuda()
    codes, scales = lce.mxfp4_quantize(weight)
    got = lce.mxfp4_linear(hidden, codes, scales)
    assert got.shape == (2, 3, 100) and got.dtype == torch.bfloat16
    x = lce.mxfp4_quantize(hidden.view(6, 320))
    _check_product(got.view(6, 100), tuple(t.cpu() for t in x), (codes.cpu(), scales.cpu()))
    out = torch.empty_like(got)
    assert lce.mxfp4_linear(hidden, codes, scales, out=out) is out and torch.equal(out, got)


def test_offsets_past_32_bits(lce):
    """A weight of 4.4 GB (both ways of reading it) and a result of 2.6 billion values: the last rows are right."""
    V, H = 1_050_000, 8448
    codes = torch.zeros((V, H // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((V, H // 32), 127, dtype=torch.uint8, device="cuda")
    w = _packed(3, H, 6)
    codes[-3:], scales[-3:] = w[0].cuda(), w[1].cuda()
    for M in (2, 130):
        x = _packed(M, H, 7)
        out = lce.mxfp4_matmul(*(t.cuda() for t in x), codes, scales)
        _check_product(out[:, -3:], x, w)
        assert not bool(out[:, :-3].any())
    del codes, scales, out
    x, w = _packed(20000, 32, 8), _packed(131080, 32, 9)
    out = lce.mxfp4_matmul(*(t.cuda() for t in x), *(t.cuda() for t in w))
    for at in (slice(0, 300), slice(19700, 20000)):
        _check_product(out[at, -300:], (x[0][at], x[1][at]), (w[0][-300:], w[1][-300:]))


def test_refusals(lce):
    x = torch.randn((4, 64), device="cuda")
    c, s = lce.mxfp4_quantize(x)
    for call in (lambda: lce.mxfp4_quantize(x[:, :48]), lambda: lce.mxfp4_quantize(x.double()), lambda: lce.mxfp4_quantize(x.t()), lambda: lce.mxfp4_quantize(x, codes=c[:2]),
                 lambda: lce.mxfp4_quantize(x, scales=s.float()), lambda: lce.mxfp4_quantize(x, codes=torch.empty((4, 64), dtype=torch.uint8, device="cuda")[:, ::2]),
                 lambda: lce.mxfp4_dequantize(c, s[:, :1]), lambda: lce.mxfp4_dequantize(c.int(), s), lambda: lce.mxfp4_dequantize(c, s, torch.float64),
                 lambda: lce.mxfp4_dequantize(c, s, out=x), lambda: lce.mxfp4_matmul(c, s, c[:, :16].contiguous(), s[:, :1].contiguous()),
                 lambda: lce.mxfp4_matmul(c, s, c.view(2, 2, 32), s.view(2, 2, 2)), lambda: lce.mxfp4_matmul(c, s, c.cpu(), s.cpu()),
                 lambda: lce.mxfp4_matmul(c, s, c, s, torch.int8), lambda: lce.mxfp4_matmul(c, s, c, s, out=x), lambda: lce.mxfp4_dequantize(c.t().contiguous().t(), s)):
        with pytest.raises(ValueError):
            call()
    raw = torch.empty(4 * 32 + 8, dtype=torch.uint8, device="cuda")
    with pytest.raises(lce.LCEError):  # not 16-byte aligned
        lce.mxfp4_matmul(raw[8:].view(4, 32), s, c, s)
    followed = torch.randn((4, 4), device="cuda", requires_grad=True) * 1.0
    with pytest.raises(ValueError):
        lce.mxfp4_matmul(c, s, c, s, torch.float32, out=followed)


def test_streams_and_graphs(lce):
    hidden = torch.randn((5, 1056), device="cuda").to(torch.bfloat16)
    many = torch.randn((140, 1056), device="cuda").to(torch.float16)
    w = lce.mxfp4_quantize(torch.randn((700, 1056), device="cuda"))

    def everything():
        return lce.mxfp4_linear(hidden, *w), lce.mxfp4_linear(many, *w), lce.mxfp4_dequantize(*lce.mxfp4_quantize(many), torch.float32)

    want = everything()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = everything()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = everything()
    for k in range(4):
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
        hidden.mul_(-0.7)
        many.add_(0.125)
        want = everything()
        torch.cuda.synchronize()


def test_a_weight_of_more_rows_than_a_launch_has_threads(lce):
    """2^29 rows and some, for few rows of x: the rows around the pieces' borders and the last ones are right, all others zero."""
    V = (1 << 29) + 77
    codes = torch.zeros((V, 16), dtype=torch.uint8, device="cuda")
    scales = torch.full((V, 1), 127, dtype=torch.uint8, device="cuda")
    at = torch.cat([torch.arange(k - 40, k + 40) for k in (40, 1 << 28, 1 << 29)] + [torch.arange(V - 3, V)])
    w = _packed(len(at), 32, 10)
    codes[at.cuda()], scales[at.cuda()] = w[0].cuda(), w[1].cuda()
    for M in (1, 9):
        x = _packed(M, 32, 11)
        out = lce.mxfp4_matmul(*(t.cuda() for t in x), codes, scales)
        _check_product(out[:, at.cuda()], x, w)
        out[:, at.cuda()] = 0
        assert not bool(out.any())

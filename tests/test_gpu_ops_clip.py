"""The global gradient norm and clipping on the GPU, against float64.

Bounds, with u = eps / 2 of the type and w = 2^-24: squares are summed in fp64, so the norm is its fp32 rounding
off (w, and 1e-12 for the sums); a clipped value is its type's rounding off, and 2 w for the factor's rounding
and the fp32 product.
"""
import math

import pytest
import torch

from oracle import ops as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
W = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def _tensors(sizes, dtypes, seed=0, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return [(scale * 10.0 ** float(torch.empty(()).uniform_(-2, 1, generator=gen)) * torch.randn(s, generator=gen)).to(DT[dtypes[k % len(dtypes)]]).cuda()
            for k, s in enumerate(sizes)]


def _check(norm, outs, grads, max_norm, norm_type=2.0):
    want, clipped = O.clip(grads, max_norm, norm_type)
    assert norm.shape == () and norm.dtype == torch.float32
    assert abs(float(norm) - float(want)) <= (W * 1.001 + 1e-12) * float(want)
    for o, c, g in zip(outs, clipped, grads):
        u = torch.finfo(g.dtype).eps / 2
        small = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[g.dtype]
        off = (o.cpu().double() - c).abs() - ((u * (1 + 2 * W) + 2 * W) * c.abs() + small)
        assert o.shape == g.shape and (off.numel() == 0 or float(off.max()) <= 0)


# Sizes around a thread's 16 bytes, a workgroup's 16 KB piece and more pieces than workgroups; empty ones; scalars.
SIZES = {
    "one": [(1,)], "scalar": [()], "few": [(3,), (0,), (4097,), (5, 7)], "pieces": [(4095,), (4096,), (4097,), (8191,), (8192,), (8193,)],
    "ends": [(8192 * 3 + 1,), (16384,), (16385,), (1,), (8192 * 2 - 1,)], "empty": [(0,), (0, 5)], "large": [(1000, 4099), (40000, 1111), (7,)],
    "hundred": [(k % 7 + 1, 100 + k) for k in range(112)], "more": [(k % 7, 100 + k) for k in range(113)],
    "many": [(37 * (k % 11) + k,) for k in range(1000)],
}


@pytest.mark.parametrize("norm_type", [2.0, INF])
@pytest.mark.parametrize("dtypes", [("bf16",), ("fp16",), ("fp32",), ("bf16", "fp32", "fp16")], ids="-".join)
@pytest.mark.parametrize("name", list(SIZES))
def test_norm_and_clip(lce, name, dtypes, norm_type):
    grads = _tensors(SIZES[name], dtypes, seed=len(name))
    total = float(O.grad_norm(grads, norm_type))
    assert abs(float(lce.grad_norm(grads, norm_type)) - total) <= (W * 1.001 + 1e-12) * total
    for limit in (0.3 * total, 2.0 * total + 1.0):
        before = [g.clone() for g in grads]
        norm, outs = lce.clip_grad_norm(grads, limit, norm_type)
        assert all(torch.equal(a, b) for a, b in zip(grads, before))
        _check(norm, outs, grads, limit, norm_type)
        here = [g.clone() for g in grads]
        again = lce.clip_grad_norm_(here, limit, norm_type)
        assert torch.equal(again, norm) and all(torch.equal(a, b) for a, b in zip(here, outs))
        if limit > total:
            assert all(torch.equal(a, b) for a, b in zip(here, grads))


def test_views_strides_and_alignment(lce):
    """Views back to back in one buffer (any element's alignment), transposed ones, channels last; what lies
    between the views stays."""
    gen = torch.Generator().manual_seed(8)
    for dtype in DT.values():
        flat = torch.randn(200000, generator=gen).to(dtype).cuda()
        cuts = [(1, 3), (5, 8200), (8206, 1), (8207, 30001), (38211, 99999)]
        grads = [flat[a:a + n] for a, n in cuts]
        before = flat.clone()
        norm, outs = lce.clip_grad_norm(grads, 10.0)
        assert torch.equal(flat, before)
        _check(norm, outs, grads, 10.0)
        lce.clip_grad_norm_(grads, 10.0)
        keep = torch.ones(200000, dtype=torch.bool, device="cuda")
        for (a, n), o in zip(cuts, outs):
            assert torch.equal(flat[a:a + n], o)
            keep[a:a + n] = False
        assert torch.equal(flat[keep], before[keep])
    t = torch.randn(300, 70, generator=gen).cuda().t()
    c = torch.randn(2, 3, 5, 7, generator=gen).cuda().to(memory_format=torch.channels_last)
    norm, outs = lce.clip_grad_norm([t, None, c], 1.0)
    assert outs[0].stride() == t.stride() and outs[1].stride() == c.stride()
    _check(norm, outs, [t, c], 1.0)
    # Outputs given, one of them the gradient itself, another at another alignment.
    buf = torch.zeros(c.numel() + 1, device="cuda")
    out = [t, buf[1:].as_strided(c.shape, c.stride())]
    keep, want = t.clone(), O.clip([t, c], 2.0)
    norm, got = lce.clip_grad_norm([t, c], 2.0, out=out)
    assert got[0] is t and buf[0] == 0
    _check(norm, got, [keep, c], 2.0)
    assert torch.allclose(got[1].cpu().double(), want[1][1], rtol=1e-6)


def test_extreme_values(lce):
    """Squares that fp32 would lose: the sums are in fp64."""
    for dtype, scale in (("fp32", 1e-30), ("fp32", 1e30), ("bf16", 1e-30), ("bf16", 1e30), ("fp16", 1e-6)):
        grads = _tensors([(5000,), (9, 11)], (dtype,), seed=4, scale=scale)
        total = float(O.grad_norm(grads))
        norm, outs = lce.clip_grad_norm(grads, 0.5 * total)
        _check(norm, outs, grads, 0.5 * total)


def test_limits(lce):
    grads = _tensors([(5000,), (9, 11)], ("bf16", "fp32"))
    _, outs = lce.clip_grad_norm(grads, 0.0)
    assert not any(o.any() for o in outs)
    _, outs = lce.clip_grad_norm(grads, INF)
    assert all(torch.equal(o, g) for o, g in zip(outs, grads))
    zero = [torch.zeros(100, device="cuda")]
    norm, outs = lce.clip_grad_norm(zero, 1.0)
    assert float(norm) == 0.0 and not outs[0].any()


@pytest.mark.parametrize("norm_type", [2.0, INF])
def test_not_finite(lce, norm_type):
    for where in (0, 8191, 40000):
        grads = _tensors([(40001,), (300,)], ("bf16", "fp32"))
        grads[0][where] = float("nan")
        assert lce.grad_norm(grads, norm_type).isnan()
        norm, outs = lce.clip_grad_norm(grads, 1.0, norm_type)
        assert norm.isnan() and all(o.isnan().all() for o in outs)
        lce.clip_grad_norm_(grads, 1.0, norm_type)
        assert all(g.isnan().all() for g in grads)
        grads = _tensors([(40001,), (300,)], ("bf16", "fp32"))
        grads[0][where] = -INF
        assert float(lce.grad_norm(grads, norm_type)) == INF
        norm, outs = lce.clip_grad_norm(grads, 1.0, norm_type)
        assert float(norm) == INF and int(outs[0].isnan().sum()) == 1 and int((outs[0] == 0).sum()) == 40000 and not outs[1].any()
        norm, outs = lce.clip_grad_norm(grads, INF, norm_type)
        assert all(torch.equal(o, g) for o, g in zip(outs, grads))


def test_more_than_32_bits_of_values(lce):
    n = (1 << 31) + 12345
    big = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    norm = lce.clip_grad_norm_([big, torch.ones(7, device="cuda")], 1e9)
    assert abs(float(norm) - math.sqrt(n + 7)) <= W * 1.001 * math.sqrt(n + 7)
    lce.clip_grad_norm_(big, 0.25 * math.sqrt(n))
    assert float(big[-1]) == 0.25 and float(big[0]) == 0.25 and bool((big[::1 << 20] == 0.25).all())


def test_deterministic(lce):
    grads = _tensors([(1 << 20,), (777, 333)], ("bf16", "fp32"), seed=2)
    want = lce.grad_norm(grads)
    for _ in range(3):
        assert torch.equal(lce.grad_norm(grads), want)


def test_versions_and_refusals(lce):
    x = torch.ones(5, device="cuda", requires_grad=True)
    y = x * 2
    z = (y * y).sum()
    lce.clip_grad_norm_(y.detach(), 1.0)  # y, which the product saved, has changed
    with pytest.raises(RuntimeError):
        z.backward()
    g = torch.ones(64, device="cuda")
    two = torch.ones(4, 64, device="cuda")
    bad = [lambda: lce.grad_norm([g.double()]), lambda: lce.grad_norm([g.expand(3, 64)]), lambda: lce.grad_norm([two[:, :32]]),
           lambda: lce.grad_norm([two[::2]]), lambda: lce.clip_grad_norm_([g, g.cpu()], 1.0), lambda: lce.grad_norm([g], 1.0),
           lambda: lce.clip_grad_norm([g], 1.0, out=[g[:32]]), lambda: lce.clip_grad_norm([g], 1.0, out=[]),
           lambda: lce.clip_grad_norm([two], 1.0, out=[two.clone().t().contiguous().t()]),
           lambda: lce.clip_grad_norm_([torch.nn.Parameter(g)], 1.0), lambda: lce.clip_grad_norm([torch.nn.Parameter(g)], 1.0),
           lambda: lce.clip_grad_norm([torch._neg_view(g)], 1.0), lambda: lce.clip_grad_norm([g], 1.0, out=[torch._neg_view(g.clone())]),
           lambda: lce.clip_grad_norm([g], 1.0, out=[g.half()]), lambda: lce.grad_norm([g.to_sparse()])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    ws = torch.empty(64, dtype=torch.uint8, device="cuda")
    for call, status in [(lambda: lce.clip_grad_norm_([g, g], 1.0), 1), (lambda: lce.clip_grad_norm_([g[:40], g[30:]], 1.0), 1),
                         (lambda: lce.clip_grad_norm([g[:32], g[32:]], 1.0, out=[g[32:], g[:32]]), 1),
                         (lambda: lce.clip_grad_norm_([g], -1.0), 1), (lambda: lce.clip_grad_norm_([g], float("nan")), 1),
                         (lambda: lce.grad_norm([g], workspace=ws), 3)]:
        with pytest.raises(lce.LCEError) as e:
            call()
        assert e.value.status == status
    assert bool((g == 1).all())
    assert float(lce.grad_norm([g, g])) == pytest.approx(math.sqrt(128), rel=W)  # reading twice is fine


def test_gradients_with_a_graph(lce):
    """Gradients made under create_graph: the values are as ever, and differentiating them raises."""
    x = torch.linspace(-1.0, 2.0, 500, device="cuda").requires_grad_()
    y = torch.linspace(1.0, 3.0, 300, device="cuda")
    g, = torch.autograd.grad((x ** 3).sum(), x, create_graph=True)
    want, clipped = O.clip([g, y], 2.0)
    for norm, outs in [(lce.grad_norm([g, y]), None), lce.clip_grad_norm([g, y], 2.0),
                       lce.clip_grad_norm([y, g], 2.0, out=[y.new_empty(300), y.new_empty(500)])]:
        assert abs(float(norm.detach()) - float(want)) <= (W * 1.001 + 1e-12) * float(want)
        for t in (norm, *(outs or ())):
            if t.requires_grad:
                with pytest.raises(RuntimeError):
                    torch.autograd.grad((t * t).sum() + (g * g).sum(), x, retain_graph=True)
        assert norm.requires_grad
    norm, outs = lce.clip_grad_norm([g, y], 2.0)
    _check(norm.detach(), [t.detach() for t in outs], [g.detach(), y], 2.0)
    assert outs[0].requires_grad and outs[1].requires_grad
    with torch.no_grad():
        assert not lce.grad_norm([g, y]).requires_grad
    norm = lce.clip_grad_norm_([g, y], 2.0)
    assert not norm.requires_grad and torch.equal(g.detach(), outs[0].detach()) and g.requires_grad
    # Nothing to follow: constants.
    norm, outs = lce.clip_grad_norm([y], 2.0)
    assert not norm.requires_grad and not outs[0].requires_grad and isinstance(outs, list)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(y, torch.ones_like(y))
        with pytest.raises(RuntimeError):
            lce.grad_norm([dual])


def test_weights_are_not_scaled(lce):
    """Leaves that require a gradient, and parameters of any class, frozen ones too: refused, and left as they were."""
    class Weight(torch.nn.Parameter):
        pass

    w = torch.ones(64, device="cuda")
    leaf = w.clone().requires_grad_()
    for bad in (leaf, Weight(w.clone()), Weight(w.clone(), requires_grad=False), torch.nn.Parameter(w.clone(), requires_grad=False)):
        for call in (lambda: lce.clip_grad_norm_([w.clone(), bad], 1.0), lambda: lce.clip_grad_norm_(bad, 1.0)):
            with pytest.raises(ValueError):
                call()
        with torch.no_grad(), pytest.raises(ValueError):
            lce.clip_grad_norm_([bad], 1.0)
        assert torch.equal(bad.detach(), w)
    with pytest.raises(ValueError):
        lce.clip_grad_norm([Weight(w)], 1.0)
    # What a leaf's backward leaves in .grad is clipped, also where it has a graph.
    (leaf ** 2).sum().backward()
    assert float(lce.clip_grad_norm_([leaf.grad], 1.0)) == 16.0 and float(lce.grad_norm(leaf.grad)) == pytest.approx(1.0, abs=1e-6)
    leaf.grad = torch.autograd.grad((leaf ** 2).sum(), leaf, create_graph=True)[0]
    # 2 / (16 + 1e-6), one w below 0.125: the factor's rounding, the product's and the 1e-6 are 3 w together.
    assert float(lce.clip_grad_norm_([leaf.grad], 1.0)) == 16.0 and abs(float(leaf.grad[0].detach()) - 2 / (16 + 1e-6)) <= 3 * W * 0.125


@pytest.mark.parametrize("count", [20, 130])
def test_streams_and_graphs(lce, count):
    """Clipping captured with few tensors (in the launch's arguments) and with many (their table in the workspace),
    two graphs with a workspace each, replayed in turn on values changed in place."""
    grads = _tensors([(100 + 31 * k,) for k in range(count)], ("bf16", "fp32"), seed=11)
    outs = [[torch.empty_like(g) for g in grads] for _ in range(2)]
    spaces = [torch.empty(lce.grad_norm_workspace_size(count), dtype=torch.uint8, device="cuda") for _ in range(2)]
    limits = (3.0, 40.0)

    def eager():
        return [(n.clone(), o) for n, o in (lce.clip_grad_norm(grads, lim) for lim in limits)]

    want = eager()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        norm, got = lce.clip_grad_norm(grads, limits[0])
    side.synchronize()
    assert torch.equal(norm, want[0][0]) and all(torch.equal(a, b) for a, b in zip(got, want[0][1]))
    graphs = []
    for lim, out, ws in zip(limits, outs, spaces):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            norm, _ = lce.clip_grad_norm(grads, lim, out=out, workspace=ws)
        graphs.append((g, norm))
    for k in range(4):
        for (g, norm), out in zip(graphs, outs):
            for t in (norm, *out):
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for (_, norm), out, (wn, wo) in zip(graphs, outs, want):
            assert torch.equal(norm, wn) and all(torch.equal(a, b) for a, b in zip(out, wo)), k
        for t in grads:
            t.mul_(0.5)
        want = eager()
        torch.cuda.synchronize()

"""The embedding lookup and its gradient on the GPU against float64.

Bounds, with u = eps / 2 of the type (half a step), w = 2^-24 (fp32's) and S the sum of the terms' magnitudes: a chunk adds at most
64 rows in fp32, chunks are joined with the rounding errors kept (two more), so a sum is at most 68 w S off before its
rounding u, and an earlier value adds its own w.
"""
import math

import pytest
import torch

from oracle import vocab as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
W = 2.0 ** -24


def _u(dtype):
    return torch.finfo(dtype).eps / 2


def _step(dtype):  # half a step of the smallest values
    return {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -150}[dtype]


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def _inputs(N, H, V, dtype, seed=0, invalid=True):
    g = torch.Generator().manual_seed(100000 * seed + N + 7 * H + 13 * V)
    weight, grad = torch.randn((V, H), generator=g), torch.randn((N, H), generator=g)
    # Frequent ones and rare ones, some outside the matrix.
    tokens = (torch.exp(torch.rand(N, generator=g) * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    if invalid:
        tokens[torch.rand(N, generator=g) < 0.05] = -1
        tokens[torch.rand(N, generator=g) < 0.05] = V
    return tokens.cuda(), weight.to(DT[dtype]).cuda(), grad.to(DT[dtype]).cuda()


def _check_rows(out, tokens, weight, scale=1.0):
    want = O.embedding(tokens, weight, scale)
    got = out.detach().cpu().double()
    assert got.shape == want.shape and torch.equal(got.isnan(), want.isnan())
    off = (got - want).abs() - ((_u(out.dtype) * (1 + 4 * W) + 2 * W) * want.abs() + _step(out.dtype))
    assert not bool((off > 0).any())


def _check_gradient(got, grad, tokens, V, scale=1.0, padding_idx=None, old=None):
    want, size = O.embedding_backward(grad, tokens, V, scale, padding_idx)
    bound = 70 * W * size
    if old is not None:
        want = want + old.detach().cpu().double()
        bound = bound + 2 * W * old.detach().cpu().double().abs()
    off = (got.detach().cpu().double() - want).abs() - (bound + _u(got.dtype) * (1 + W) * (want.abs() + bound) + _step(got.dtype))
    assert got.shape == want.shape and not bool((off > 0).any()), float(off.max())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("H", [1, 5, 8, 9, 64, 127, 128, 129, 136, 1000, 1024, 1025, 1032, 2056, 4096, 4099, 8200])
def test_forward(lce, H, dtype):
    for N, V in ((1, 1), (3, 500), (70, 33)):
        tokens, weight, _ = _inputs(N, H, V, dtype)
        _check_rows(lce.embedding_forward(tokens, weight), tokens, weight)
        _check_rows(lce.embedding_forward(tokens.int(), weight, 0.37), tokens, weight, float(torch.tensor(0.37)))


def test_forward_shapes_strides_and_alignment(lce):
    tokens, weight, _ = _inputs(24, 300, 50, "bf16")
    tokens = tokens.view(2, 3, 4)
    for at, H in ((1, 200), (3, 129), (8, 64)):
        buf = torch.full((24, 700), 7.0, dtype=torch.bfloat16, device="cuda")
        out = buf[:, 5:5 + H].view(2, 3, 4, H)
        assert lce.embedding_forward(tokens, weight[:, at:at + H], 2.0, out=out) is out
        _check_rows(out, tokens, weight[:, at:at + H], 2.0)
        assert bool((buf[:, :5] == 7).all() and (buf[:, 5 + H:] == 7).all())
    one = weight[:1].expand(50, 300)
    _check_rows(lce.embedding_forward(tokens, one), tokens, one)
    assert lce.embedding_forward(tokens[:0], weight).shape == (0, 3, 4, 300)
    _check_rows(lce.embedding_forward(tokens[0, 0, 0], weight), tokens[0, 0, 0], weight)


# Numbers of positions around the borders of a tile (2048), of tiles merged in LDS (2, 4, 8, 16), and of longer runs.
@pytest.mark.parametrize("N,H,V,dtype", [
    (1, 8, 1, "bf16"), (2, 3, 5, "fp32"), (31, 64, 7, "fp16"), (32, 72, 1, "bf16"), (33, 72, 1, "fp32"), (65, 1, 300, "fp32"), (700, 4096, 90, "bf16"),
    (2047, 24, 50, "bf16"), (2048, 24, 5000, "fp32"), (2049, 24, 64, "fp16"), (4097, 136, 63, "bf16"), (5000, 2056, 300, "bf16"), (8193, 16, 65, "fp32"),
    (9001, 7, 50257, "bf16"), (16385, 8, 4096, "fp16"), (32768, 9, 4095, "fp32"), (32769, 8, 100, "fp32"), (70001, 40, 1000, "bf16"), (600000, 2, 128256, "fp32")])
def test_gradient(lce, N, H, V, dtype):
    tokens, weight, grad = _inputs(N, H, V, dtype)
    got = lce.embedding_backward(grad, tokens, V)
    _check_gradient(got, grad, tokens, V)
    assert torch.equal(got, lce.embedding_backward(grad, tokens.int(), V))
    got = lce.embedding_backward(grad, tokens, V, 0.5, V // 2)
    _check_gradient(got, grad, tokens, V, 0.5, V // 2)
    assert not bool(got[V // 2].any())
    old = weight.clone()
    assert lce.embedding_backward(grad, tokens, V, 0.5, V // 2, grad_weight=weight, accumulate=True) is weight
    _check_gradient(weight, grad, tokens, V, 0.5, V // 2, old)
    named = torch.zeros(V + 1, dtype=torch.bool, device="cuda")
    named[tokens.clamp(0, V)] = True
    named[V // 2] = False
    assert torch.equal(weight[~named[:V]], old[~named[:V]])


@pytest.mark.parametrize("kind", ["one", "all", "none", "padding"])
def test_gradient_of_few_or_all_tokens(lce, kind):
    """One token at every position; every token once; none that counts; the padding token alone."""
    N, H, V = 5000, 40, 5000
    tokens = {"one": torch.full((N,), 3), "all": torch.randperm(N), "none": torch.full((N,), V + 5), "padding": torch.full((N,), 7)}[kind].cuda()
    grad = torch.randn((N, H), device="cuda")
    pad = 7 if kind == "padding" else None
    got = lce.embedding_backward(grad, tokens, V, 1.0, pad)
    _check_gradient(got, grad, tokens, V, 1.0, pad)
    if kind == "all":
        assert torch.equal(got[tokens], grad)
    if kind in ("none", "padding"):
        assert not bool(got.any())
    # No position at all: zeros, or nothing.
    assert not bool(lce.embedding_backward(grad[:0], tokens[:0], V).any())
    kept = lce.embedding_backward(grad[:0], tokens[:0], V, grad_weight=got.clone(), accumulate=True)
    assert torch.equal(kept, got)


def test_very_wide_rows(lce):
    tokens, weight, grad = _inputs(70, 70005, 3, "bf16")
    _check_rows(lce.embedding_forward(tokens, weight, 2.0), tokens, weight, 2.0)
    _check_gradient(lce.embedding_backward(grad, tokens, 3), grad, tokens, 3)


def test_long_sums(lce):
    """A token at 300000 positions: a chain of fp32 additions would lose all that is added after the first."""
    N = 300000
    grad = torch.full((N, 8), 2.0 ** -24, device="cuda")
    grad[0] = 1.0
    tokens = torch.zeros(N, dtype=torch.int64, device="cuda")
    got = lce.embedding_backward(grad, tokens, 2)
    _check_gradient(got, grad, tokens, 2)
    assert float(got[0, 0]) > 1.017


def test_values_that_are_not_finite(lce):
    """They stay in their tokens' rows; infinities of one sign stay infinite over many chunks."""
    N, V = 300, 10
    tokens = torch.arange(N, device="cuda") % V
    grad = torch.ones((N, 16), device="cuda")
    grad[13, 2], grad[24, 3], grad[7::10, 5] = math.nan, math.inf, -math.inf
    got = lce.embedding_backward(grad, tokens, V)
    want, _ = O.embedding_backward(grad, tokens, V)
    assert torch.equal(got.cpu().double().nan_to_num(5.0, 1e9, -1e9), want.nan_to_num(5.0, 1e9, -1e9)) and torch.equal(got.cpu().isnan(), want.isnan())
    one = torch.full((300,), 4, device="cuda")
    got = lce.embedding_backward(torch.full((300, 8), math.inf, device="cuda"), one, V)
    assert bool(got[4].isposinf().all())
    # Rows of tokens that do not count may hold anything.
    grad[:] = 1.0
    grad[::10] = math.nan
    assert bool(lce.embedding_backward(grad, tokens, V, 1.0, 0).isfinite().all())


def test_gradient_strides(lce):
    tokens, weight, _ = _inputs(300, 300, 40, "bf16")
    wide = torch.randn((300, 700), device="cuda").to(torch.bfloat16)
    for at, H in ((3, 200), (8, 64), (1, 5)):
        grad = wide[:, at:at + H]
        buf = torch.full((40, 500), 7.0, dtype=torch.bfloat16, device="cuda")
        out = buf[:, 2:2 + H]
        lce.embedding_backward(grad.view(3, 100, H), tokens.view(3, 100), 40, grad_weight=out)
        _check_gradient(out, grad, tokens, 40)
        lce.embedding_backward(grad, tokens, 40, grad_weight=out, accumulate=True)
        assert bool((buf[:, :2] == 7).all() and (buf[:, 2 + H:] == 7).all())
    one = wide[:1, :64].expand(300, 64)
    _check_gradient(lce.embedding_backward(one, tokens, 40), one, tokens, 40)


@pytest.mark.parametrize("dtype", list(DT))
def test_autograd(lce, dtype):
    tokens, weight, grad = _inputs(200, 72, 50, dtype)
    weight.requires_grad_()
    out = lce.embedding(tokens.view(4, 50), weight, 3.0, 2)
    _check_rows(out, tokens.view(4, 50), weight, 3.0)
    g, = torch.autograd.grad(out, weight, grad.view(4, 50, 72), retain_graph=True)
    _check_gradient(g, grad, tokens, 50, 3.0, 2)
    # A broadcast upstream gradient, one with other strides, and a lazily negated one.
    row = grad[:1, None].expand(4, 50, 72)
    g, = torch.autograd.grad(out, weight, row, retain_graph=True)
    _check_gradient(g, row, tokens, 50, 3.0, 2)
    g, = torch.autograd.grad(out, weight, grad.view(50, 4, 72).transpose(0, 1), retain_graph=True)
    _check_gradient(g, grad.view(50, 4, 72).transpose(0, 1), tokens, 50, 3.0, 2)
    if dtype == "fp32":
        negated = torch.complex(torch.zeros_like(grad), grad).conj().imag
        g, = torch.autograd.grad(out, weight, negated.view(4, 50, 72), retain_graph=True)
        _check_gradient(g, -grad, tokens, 50, 3.0, 2)
    # Used twice, the weight gets both gradients.
    first = tokens[:7].clamp(0, 49)
    (lce.embedding(first, weight).float().sum() + lce.embedding(first, weight, 2.0).float().sum()).backward()
    ones = torch.ones((7, 72), device="cuda")
    _check_gradient(weight.grad, ones, first, 50, 3.0)
    assert not lce.embedding(tokens, weight.detach()).requires_grad


def test_autograd_refusals(lce):
    tokens, weight, grad = _inputs(20, 16, 50, "fp32", invalid=False)
    weight.requires_grad_()
    out = lce.embedding(tokens, weight)
    dy = grad.clone().requires_grad_()
    g, = torch.autograd.grad(out, weight, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    with pytest.raises((RuntimeError, ValueError)):
        torch.autograd.grad(out, weight, torch.stack([grad, grad]), is_grads_batched=True, retain_graph=True)
    tokens.add_(1)  # the saved tokens
    with pytest.raises(RuntimeError):
        torch.autograd.grad(out, weight, grad)
    with pytest.raises(ValueError):
        lce.embedding(tokens, weight, 1.0, 50)


def test_refusals(lce):
    tokens, weight, grad = _inputs(20, 16, 50, "fp32", invalid=False)
    leaf = weight.clone().requires_grad_()
    for call in (lambda: lce.embedding_forward(tokens.cpu(), weight), lambda: lce.embedding_forward(tokens.float(), weight), lambda: lce.embedding_forward(tokens[::2], weight),
                 lambda: lce.embedding_forward(tokens, weight.double()), lambda: lce.embedding_forward(tokens, weight[0]), lambda: lce.embedding_forward(tokens, weight.t()),
                 lambda: lce.embedding_forward(tokens, weight, math.inf), lambda: lce.embedding_forward(tokens, weight, out=weight[:20, :8]),
                 lambda: lce.embedding_forward(tokens, weight, out=leaf[:20] * 1.0), lambda: lce.embedding_backward(grad[:10], tokens, 50),
                 lambda: lce.embedding_backward(grad, tokens, 0), lambda: lce.embedding_backward(grad, tokens, 50, padding_idx=50),
                 lambda: lce.embedding_backward(grad, tokens, 50, padding_idx=-1), lambda: lce.embedding_backward(grad, tokens, 50, accumulate=True),
                 lambda: lce.embedding_backward(grad, tokens, 50, grad_weight=weight[:40]), lambda: lce.embedding_backward(grad, tokens, 50, grad_weight=weight.half()),
                 lambda: lce.embedding_backward(grad.t(), tokens[:16], 50), lambda: lce.embedding_backward(grad, tokens, 50, workspace=torch.empty(10, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lce.embedding_forward(tokens, weight, out=weight[:20]), lambda: lce.embedding_backward(weight[:20], tokens, 50, grad_weight=weight),
                 lambda: lce.embedding_backward(grad, tokens, 50, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(lce.LCEError):
            call()


def test_given_outputs_are_known_to_autograd(lce):
    tokens, weight, grad = _inputs(20, 16, 50, "fp32", invalid=False)
    x = torch.ones((50, 16), device="cuda", requires_grad=True)
    y = (x * weight).sum()  # saves weight
    lce.embedding_backward(grad, tokens, 50, grad_weight=weight, accumulate=True)
    with pytest.raises(RuntimeError):
        y.backward()


def test_offsets_past_32_bits(lce):
    """A matrix of 2.5 billion values: its last rows looked up, written and added to; all the others zero."""
    V, H = 300001, 8192
    big = torch.empty((V, H), dtype=torch.bfloat16, device="cuda")
    tokens = torch.tensor([V - 1, 0, V - 1, V - 2, 262145], device="cuda")
    grad = torch.randn((5, H), device="cuda").to(torch.bfloat16)
    lce.embedding_backward(grad, tokens, V, grad_weight=big)
    want, _ = O.embedding_backward(grad, torch.tensor([2, 0, 2, 1, 3]), 4)
    rows = torch.tensor([0, V - 2, V - 1, 262145], device="cuda")
    _check_gradient(big[rows], grad, torch.tensor([2, 0, 2, 1, 3]), 4)
    norm = sum(float(b.float().square().sum(dtype=torch.float64)) for b in big.split(20000))
    assert abs(norm - float(big[rows].double().square().sum())) <= 1e-9 * norm
    out = lce.embedding_forward(tokens, big)
    assert torch.equal(out, big[tokens])
    old = big[rows].clone()
    lce.embedding_backward(grad, tokens, V, grad_weight=big, accumulate=True)
    _check_gradient(big[rows], grad, torch.tensor([2, 0, 2, 1, 3]), 4, old=old)


def test_deterministic(lce):
    tokens, _, grad = _inputs(20000, 256, 1000, "fp32")
    first = lce.embedding_backward(grad, tokens, 1000)
    for _ in range(5):
        assert torch.equal(first, lce.embedding_backward(grad, tokens, 1000))


def test_streams_and_graphs(lce):
    """On a side stream; two graphs with a workspace each, replayed in turn on inputs changed in place, with eager work between."""
    N, H, V = 5000, 136, 700
    tokens, weight, grad = _inputs(N, H, V, "bf16", invalid=False)
    need = lce.embedding_workspace_size(N, H)
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    base = torch.randn((V, H), device="cuda").to(torch.bfloat16)

    def everything(ws):
        added = base.clone()
        return (lce.embedding_forward(tokens, weight, 2.0), lce.embedding_backward(grad, tokens, V, workspace=ws),
                lce.embedding_backward(grad, tokens, V, grad_weight=added, accumulate=True, workspace=ws))

    want = everything(spaces[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = everything(spaces[0])
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graphs = []
    for ws in spaces:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs = everything(ws)
        graphs.append((g, outs))
    for k in range(4):
        for g, outs in graphs:
            for t in outs:
                t.zero_()
            g.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), k
        tokens.copy_((tokens * 7 + k) % V)
        grad.mul_(0.5)
        want = [t.clone() for t in everything(spaces[0])]
        torch.cuda.synchronize()


def test_two_streams_at_once(lce):
    tokens, _, grad = _inputs(9000, 512, 3000, "bf16")
    want = lce.embedding_backward(grad, tokens, 3000)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(lce.embedding_backward(grad, tokens, 3000))
    torch.cuda.synchronize()
    assert all(torch.equal(g, want) for g in got)

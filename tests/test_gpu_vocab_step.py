"""The operators on the vocabulary's matrix and logits with those beside them: a training step whose input and output layers
share a weight, and tokens produced one after the other."""
import numpy as np
import pytest
import torch

import oracle
from oracle import ops as RO
from oracle import vocab as O

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


# The step's own bars (of the largest magnitude; fp32 1e-5, bf16 2e-2), and the roundings of what is in front of it, half a step
# each: the embedded rows, the normalised rows, dX, dH, the sum of both gradients.
@pytest.mark.parametrize("dtype,loss_bar,bar", [(torch.float32, 1e-5, 3e-5), (torch.bfloat16, 2e-3, 2e-2 + 5 * 2.0 ** -8)])
@pytest.mark.parametrize("N,H,V", [(300, 136, 1031), (64, 256, 500)])
def test_tied_training_step(lce, dtype, loss_bar, bar, N, H, V):
    g = torch.Generator().manual_seed(N)
    W = (0.3 * torch.randn((V, H), generator=g)).to(dtype)
    gamma = (1.0 + 0.1 * torch.randn(H, generator=g)).to(dtype)
    tokens, labels = torch.randint(0, V, (N,), generator=g), torch.randint(0, V, (N,), generator=g)
    tokens[: N // 4] = 3
    labels[::9] = -100
    scale = 8.0
    x = O.embedding(tokens, W, scale)
    normed, added, r = RO.add_rmsnorm(x, None, gamma, EPS)
    ref = oracle.forward_backward(normed.numpy(), W.double().numpy(), labels)
    dx, dg = RO.add_rmsnorm_backward(torch.from_numpy(ref["dH"]), None, added, gamma, r)
    dW = torch.from_numpy(ref["dW"]) + O.embedding_backward(dx, tokens, V, scale)[0]

    def near(got, want):
        assert float((got.cpu().double() - want).abs().max()) <= bar * float(want.abs().max())

    weight, gain = W.cuda().requires_grad_(), gamma.cuda().requires_grad_()
    t, y = tokens.cuda(), labels.cuda()
    loss = lce.linear_cross_entropy(lce.rmsnorm(lce.embedding(t, weight, scale), gain, EPS), weight, y)
    grads = torch.autograd.grad(loss, (weight, gain))
    assert abs(loss.item() - ref["loss"]) <= loss_bar * abs(ref["loss"])
    near(grads[0], dW)
    near(grads[1], dg)
    # The same by hand: the embedding's gradient added to the one that the output layer left.
    rows = lce.embedding_forward(t, W.cuda(), scale)
    h, _, rstd = lce.add_rmsnorm_forward(rows, None, gamma.cuda(), EPS, return_rstd=True)
    _, dH, grad = lce.forward_backward(h, W.cuda(), y)
    drows, dgain = lce.add_rmsnorm_backward(dH, None, rows, None, gamma.cuda(), rstd)
    assert lce.embedding_backward(drows, t, V, scale, grad_weight=grad, accumulate=True) is grad
    near(grad, dW)
    assert torch.equal(dgain, grads[1])
    norm, clipped = lce.clip_grad_norm([grad, dgain], 0.1)
    assert float(lce.grad_norm(clipped)) <= 0.1 * (1 + 2.0 ** -8)


def test_answers(lce):
    """Tokens one after the other for four requests with settings of their own: embedded, normalised with the residual, multiplied with the
    weight in 4 bits, drawn. Every stage against its definition on what the stage before it gave."""
    N, H, V = 4, 320, 1500
    g = torch.Generator().manual_seed(2)
    W = (torch.randn((V, H), generator=g)).to(torch.bfloat16).cuda()
    gamma = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    codes, scales = lce.mxfp4_quantize(W)
    weight = O.mxfp4_values(codes, scales)
    tokens = torch.tensor([1, 700, 700, 1499], device="cuda")
    residual = torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
    t, k = torch.tensor([0.0, 0.7, 1.0, 1.0], device="cuda"), torch.tensor([0, 20, 0, 5], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 0.9, 0.5, 1.0], device="cuda")
    seen = []
    for step in range(6):
        x = lce.embedding_forward(tokens, W, 0.5)
        assert torch.equal(x.cpu().double(), O.embedding(tokens, W, 0.5))  # (half of a bfloat16 is one)
        normed, residual = lce.add_rmsnorm_forward(x, residual, gamma, EPS)
        logits = lce.mxfp4_linear(normed, codes, scales)
        want = O.mxfp4_values(*lce.mxfp4_quantize(normed)) @ weight.T
        size = O.mxfp4_values(*lce.mxfp4_quantize(normed)).abs() @ weight.abs().T
        assert bool(((logits.cpu().double() - want).abs() <= 2.0 ** -8 * 1.001 * want.abs() + H * 2.0 ** -24 * size).all())
        u = torch.rand(N, generator=g).cuda()
        tokens, logs = lce.sample(logits, u, t, k, p, return_logprobs=True)
        want, want_logs = O.sample(logits, u, t, k, p)
        assert torch.equal(tokens.cpu(), want)
        assert float((logs.cpu().double() - want_logs).abs().max()) <= 1e-6
        seen.append(tokens.tolist())
    assert all(0 <= v < V for row in seen for v in row)


def test_a_row_without_an_answer(lce):
    """A row of NaN gives -1, which embeds to NaN again and leaves the others alone."""
    W = torch.randn((40, 64), device="cuda").to(torch.bfloat16)
    codes, scales = lce.mxfp4_quantize(W)
    x = lce.embedding_forward(torch.tensor([3, -1, 5], device="cuda"), W)
    logits = lce.mxfp4_linear(x, codes, scales)
    tokens = lce.sample(logits, torch.full((3,), 0.5, device="cuda"), temperature=0.0)
    assert bool(logits[1].isnan().all()) and tokens[1] == -1 and bool(logits[[0, 2]].isfinite().all()) and bool((tokens[[0, 2]] >= 0).all())


def test_answers_in_a_graph(lce):
    """One step of it captured with its workspace, the token fed back in place, against the same steps run one by one."""
    N, H, V = 3, 256, 5000
    W = torch.randn((V, H), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    gamma = torch.ones(H, dtype=torch.bfloat16, device="cuda")
    codes, scales = lce.mxfp4_quantize(W.roll(1, 0))  # (another weight than the rows', so that a token does not answer itself)
    tokens, u = torch.zeros(N, dtype=torch.int64, device="cuda"), torch.zeros(N, device="cuda")
    ws = torch.empty(lce.sample_workspace_size(N, V), dtype=torch.uint8, device="cuda")

    def step(tokens, u):
        normed, _ = lce.add_rmsnorm_forward(lce.embedding_forward(tokens, W), None, gamma, EPS)
        return lce.sample(lce.mxfp4_linear(normed, codes, scales), u, 4.0, 100, 0.95, workspace=ws)

    numbers = torch.rand((6, N), generator=torch.Generator().manual_seed(4)).cuda()
    want, now = [], tokens.clone()
    for r in numbers:
        now = step(now, r)
        want.append(now.tolist())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(tokens, u)
    got = []
    for r in numbers:
        u.copy_(r)
        graph.replay()
        tokens.copy_(out)
        got.append(out.tolist())
    assert got == want and len(set(map(tuple, got))) > 1


def test_what_has_no_gradient_says_so(lce):
    """Logits of the 4-bit product and log-probabilities of drawn tokens are not constants to a gradient: asking for it raises."""
    hidden = torch.randn((3, 64), device="cuda", requires_grad=True)
    codes, scales = lce.mxfp4_quantize(torch.randn((40, 64), device="cuda"))
    u = torch.rand(3, device="cuda")
    logits = lce.mxfp4_linear(hidden, codes, scales)
    assert torch.equal(logits, lce.mxfp4_linear(hidden.detach(), codes, scales))
    tokens, logs = lce.sample(logits, u, top_k=5, return_logprobs=True)
    assert not tokens.requires_grad and torch.equal(tokens, lce.sample(logits.detach(), u, top_k=5))
    for value in (logits, logs):
        with pytest.raises(RuntimeError, match="not differentiable"):
            value.sum().backward()
    with pytest.raises(ValueError):
        lce.mxfp4_linear(hidden, codes, scales, out=torch.empty((3, 40), device="cuda"))
    with torch.no_grad():
        assert not lce.mxfp4_linear(hidden, codes, scales).requires_grad
    assert not lce.sample(logits, u).requires_grad
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(hidden.detach(), torch.ones_like(hidden))
        with pytest.raises(RuntimeError):
            lce.mxfp4_linear(dual, codes, scales)


def test_training_in_a_graph(lce):
    """The embedding's lookup and gradient captured together, replayed on tokens and upstream gradients changed in place."""
    V, N, H = 500, 3000, 264
    weight = torch.randn((V, H), device="cuda").to(torch.bfloat16).requires_grad_()
    tokens, dy = torch.randint(0, V, (N,), device="cuda"), torch.randn((N, H), device="cuda").to(torch.bfloat16)

    def step():
        out = lce.embedding(tokens, weight, 2.0, 7)
        return (out.detach(), *torch.autograd.grad(out, weight, dy))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for k in range(4):
        tokens.copy_((tokens * 3 + k) % V)
        dy.mul_(-0.5)
        want = [t.clone() for t in step()]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k


def test_drawn_log_probabilities_are_no_constants_to_their_settings(lce):
    """They depend on the temperature as on the logits: of a setting that autograd follows, asking for its gradient raises too."""
    logits, u = torch.randn((3, 200), device="cuda"), torch.rand(3, device="cuda")
    plain = dict(temperature=torch.full((3,), 0.7, device="cuda"), top_p=torch.full((3,), 0.9, device="cuda"), min_p=torch.full((3,), 0.01, device="cuda"))
    want = lce.sample(logits, u, **plain, return_logprobs=True)
    for name in plain:
        for z in (logits, logits.clone().requires_grad_()):
            settings = plain | {name: plain[name].clone().requires_grad_()}
            tokens, logs = lce.sample(z, u, **settings, return_logprobs=True)
            assert torch.equal(tokens, want[0]) and torch.equal(logs, want[1]) and not tokens.requires_grad
            with pytest.raises(RuntimeError, match="not differentiable"):
                torch.autograd.grad(logs.sum(), settings[name])
            assert not lce.sample(z, u, **settings).requires_grad
            with torch.no_grad():
                assert not lce.sample(z, u, **settings, return_logprobs=True)[1].requires_grad
        with torch.autograd.forward_ad.dual_level():
            dual = torch.autograd.forward_ad.make_dual(plain[name], torch.ones_like(plain[name]))
            with pytest.raises(RuntimeError):
                lce.sample(logits, u, **(plain | {name: dual}), return_logprobs=True)

"""The operators with the output-layer step, as a training program runs them: residual + final norm, the fused
projection and loss, gradients clipped into the buffers that the host optimizer reads, one AdamW step; and as an
evaluation runs them."""
import numpy as np
import pytest
import torch

import oracle
import workloads
from oracle import ops as O

pytestmark = pytest.mark.gpu

EPS = 1e-5


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def _oracle_step(x, res, gamma, W, y):
    normed, added, r = O.add_rmsnorm(x, res, gamma, EPS)
    ref = oracle.forward_backward(normed.numpy(), W.double().numpy(), y)
    dx, dg = O.add_rmsnorm_backward(torch.from_numpy(ref["dH"]), None, added, gamma, r)
    return ref["loss"], dx, dg, torch.from_numpy(ref["dW"])


# The step's own bars (of the largest magnitude): fp32 1e-5 (here: and of dH's two normalisations, 2e-5); bf16 2e-2,
# and three more roundings of half a step each (the normalised rows, the sum, dX): 3 * 2^-8 = 1.2e-2.
@pytest.mark.parametrize("dtype,loss_bar,bar", [("fp32", 1e-5, 2e-5), ("bf16", 1e-3, 3.2e-2)])
@pytest.mark.parametrize("N,H,V", [(300, 136, 4099), (64, 256, 1000)])
def test_training_step(lce, dtype, loss_bar, bar, N, H, V):
    d = workloads.random_case(N, H, V, dtype=dtype, seed=3, w_std=0.3)
    gen = torch.Generator().manual_seed(N)
    res = torch.randn((N, H), generator=gen).to(d["hidden"].dtype)
    gamma = (1.0 + 0.1 * torch.randn(H, generator=gen)).to(res.dtype)
    x, W, y = d["hidden"], d["weight"], d["labels"]
    loss64, dx64, dg64, dW64 = _oracle_step(x, res, gamma, W, y)
    leaves = [t.cuda().requires_grad_() for t in (x, res, gamma, W)]
    normed, added = lce.add_rmsnorm(leaves[0], leaves[1], leaves[2], EPS)
    loss = lce.linear_cross_entropy(normed, leaves[3], y.cuda())
    grads = torch.autograd.grad(loss, leaves)
    assert abs(loss.item() - loss64) <= loss_bar * abs(loss64)
    for got, want in zip(grads, (dx64, dx64, dg64, dW64)):
        assert float((got.cpu().double() - want).abs().max()) <= bar * float(want.abs().max())
    # The model's gradients (of hidden, gamma and W) clipped to a third of their norm, beside the unclipped ones.
    mine = [grads[0], grads[2], grads[3]]
    limit = float(O.grad_norm(mine)) / 3
    norm, clipped = lce.clip_grad_norm(mine, limit)
    wn, wc = O.clip(mine, limit)
    assert abs(float(norm) - float(wn)) <= 2.0 ** -23 * float(wn)
    assert float(lce.grad_norm(clipped)) <= limit * (1 + 2.0 ** -8)
    # One AdamW step of W on the host from its clipped gradient: the first step moves each weight by lr against
    # its gradient's sign, up to eps / |g|.
    master = W.float().clone()
    m, v = torch.zeros_like(master), torch.zeros_like(master)
    lce.host_adam_step(master, clipped[2].cpu(), m, v, step=1, lr=1e-2, eps=1e-12)
    g = clipped[2].cpu().float()
    moved = (master - W.float())[g.abs() > 1e-6]
    assert torch.allclose(moved, -1e-2 * torch.sign(g[g.abs() > 1e-6]), rtol=1e-3, atol=1e-6)


def test_as_the_fused_norm(lce):
    """add_rmsnorm in front of the step gives what the step with its own RMSNorm gives on the rounded sum."""
    d = workloads.make_rmsnorm_inputs("llama3_8b", seed=3, N=70, H=72, V=1031)
    h, gamma, W, y = d["hidden"].cuda(), d["gamma"].cuda(), d["weight"].cuda(), d["labels"].cuda()
    zero = torch.zeros_like(h)
    normed, added = lce.add_rmsnorm_forward(h, zero, gamma, d["eps"])
    assert torch.equal(added, h)
    loss, x = lce.rmsnorm_forward(h, gamma, W, y, d["eps"], return_normed=True)
    # The same fp32 formula up to the order of the sums: a value near a border may round to the other side.
    assert float((normed.float() - x.float()).abs().max()) <= 2.0 ** -7 * float(x.float().abs().max())
    assert float((normed == x).float().mean()) > 0.99
    mine = lce.forward(normed, W, y)
    assert abs(float(mine) - float(loss)) <= 1e-3 * abs(float(loss))


def test_evaluation_in_eight_bits(lce):
    """A prompt's rows in e4m3 with a scale per 64 values, as an 8-bit product reads them: dequantised, their loss
    is the oracle's on the same values."""
    d = workloads.random_case(200, 256, 2000, dtype="bf16", seed=9, w_std=0.3)
    gen = torch.Generator().manual_seed(4)
    res = torch.randn((200, 256), generator=gen).to(torch.bfloat16)
    gamma = (1.0 + 0.1 * torch.randn(256, generator=gen)).to(torch.bfloat16)
    q, scales, added = lce.add_rmsnorm_quant(d["hidden"].cuda(), res.cuda(), gamma.cuda(), EPS, group_size=64)
    rows = (q.float().view(200, 4, 64) * scales[..., None]).view(200, 256).to(torch.bfloat16)
    loss = lce.forward(rows, d["weight"].cuda(), d["labels"].cuda())
    ref = oracle.forward(rows.cpu(), d["weight"], d["labels"])["loss"]
    assert abs(float(loss) - ref) <= 1e-3 * abs(ref)
    y, _, _ = O.add_rmsnorm(d["hidden"], res, gamma, EPS)
    got = rows.cpu().double().numpy()
    assert np.abs(got - y.numpy()).max() <= (2.0 ** -4 + 2.0 ** -8) * np.abs(y.numpy()).max()


def test_outputs_that_autograd_follows(lce):
    """A given output with a graph of its own would say that it is still what that graph computed: refused where
    gradients are recorded, and fine without."""
    x, r, dy = (torch.linspace(-1.0, 2.0, 256, device="cuda").view(4, 64) * k for k in (1.0, 2.0, 3.0))
    gamma, rstd = torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    leaf = x.clone().requires_grad_()

    def followed():
        return leaf * 1.0

    for call in (lambda t: lce.add_rmsnorm_forward(x, r, gamma, EPS, normed=t), lambda t: lce.add_rmsnorm_forward(t, r, gamma, EPS, added=t),
                 lambda t: lce.add_rmsnorm_quant(x, r, gamma, EPS, added=t), lambda t: lce.add_rmsnorm_backward(dy, None, x, r, gamma, rstd, grad_hidden=t),
                 lambda t: lce.clip_grad_norm(x, 1.0, out=t), lambda t: lce.clip_grad_norm([t], 1.0, out=[t])):
        t = followed()
        with pytest.raises(ValueError):
            call(t)
        assert torch.equal(t, x)
        with torch.no_grad():
            call(t)
            assert not torch.equal(t, x)
        call(followed().detach())

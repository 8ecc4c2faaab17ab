"""The float64 definitions of the operators around the step, against independent facts: torch's own
rms_norm with autograd, central differences, and torch's gradient clipping."""
import pytest
import torch

from oracle import ops as O


def _case(N, H, seed=0):
    g = torch.Generator().manual_seed(seed)
    x, res, dy, ds = (torch.randn((N, H), generator=g, dtype=torch.float64) for _ in range(4))
    gamma = 1.0 + 0.2 * torch.randn(H, generator=g, dtype=torch.float64)
    return x, res, gamma, dy, ds


@pytest.mark.parametrize("N,H", [(1, 1), (3, 7), (5, 64)])
def test_rmsnorm_is_torchs_with_its_gradients(N, H):
    x, res, gamma, dy, ds = _case(N, H)
    leaves = [t.clone().requires_grad_() for t in (x, res, gamma)]
    s = leaves[0] + leaves[1]
    y = torch.nn.functional.rms_norm(s, (H,), leaves[2], 1e-5)
    want = torch.autograd.grad((y, s), leaves, (dy, ds))
    normed, added, r = O.add_rmsnorm(x, res, gamma, 1e-5)
    dx, dg = O.add_rmsnorm_backward(dy, ds, added, gamma, r)
    for a, b in ((normed, y), (added, s), (dx, want[0]), (dx, want[1]), (dg, want[2])):
        assert torch.allclose(a, b, rtol=1e-12, atol=1e-12)


def test_gradients_are_the_differences():
    x, res, gamma, dy, ds = _case(3, 5, seed=4)

    def value(x, res, gamma):
        y, s, _ = O.add_rmsnorm(x, res, gamma, 1e-3)
        return float((y * dy).sum() + (s * ds).sum())

    _, s, r = O.add_rmsnorm(x, res, gamma, 1e-3)
    dx, dg = O.add_rmsnorm_backward(dy, ds, s, gamma, r)
    h = 1e-6
    for t, grad, put in ((x, dx, lambda t: (t, res, gamma)), (res, dx, lambda t: (x, t, gamma)), (gamma, dg, lambda t: (x, res, t))):
        for k in range(t.numel()):
            up, down = t.clone(), t.clone()
            up.view(-1)[k] += h
            down.view(-1)[k] -= h
            diff = (value(*put(up)) - value(*put(down))) / (2 * h)
            assert abs(diff - float(grad.reshape(-1)[k])) <= 1e-7 * max(1.0, abs(diff))


def test_scales():
    y = torch.tensor([[1.0, -448.0, 2.0, 0.0, 3.0], [0.0] * 5])
    assert torch.equal(O.group_scales(y, 0), torch.tensor([[1.0], [O.SCALE_MIN]], dtype=torch.float64))
    assert torch.equal(O.group_scales(y, 2), torch.tensor(
        [[1.0, 2.0 / 448, 3.0 / 448], [O.SCALE_MIN] * 3], dtype=torch.float64))


@pytest.mark.parametrize("max_norm", [0.0, 0.3, 5.0, 1e9])
@pytest.mark.parametrize("norm_type", [2.0, float("inf")])
def test_clip_is_torchs(max_norm, norm_type):
    gen = torch.Generator().manual_seed(3)
    params = [torch.nn.Parameter(torch.zeros(s, dtype=torch.float64)) for s in ((), (3,), (4, 5))]
    for p in params:
        p.grad = torch.randn(p.shape, generator=gen, dtype=torch.float64)
    norm, clipped = O.clip([p.grad for p in params], max_norm, norm_type)
    want = torch.nn.utils.clip_grad_norm_(params, max_norm, norm_type)
    assert torch.allclose(norm, want, rtol=1e-14)
    for c, p in zip(clipped, params):
        assert torch.allclose(c, p.grad, rtol=1e-14)

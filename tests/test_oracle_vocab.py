"""The float64 definitions of the operators on the vocabulary's matrix and logits, against independent facts: torch's
embedding with autograd, central differences, the format's values by hand, and frequencies of drawn tokens."""
import math

import pytest
import torch

from oracle import vocab as O


@pytest.mark.parametrize("padding", [None, 2])
def test_embedding_is_torchs_with_its_gradient(padding):
    g = torch.Generator().manual_seed(1)
    W = torch.randn((7, 5), generator=g, dtype=torch.float64, requires_grad=True)
    t = torch.tensor([[0, 2, 6], [2, 2, 1]])
    dy = torch.randn((2, 3, 5), generator=g, dtype=torch.float64)
    out = torch.nn.functional.embedding(t, W, padding_idx=padding) * 1.5
    want, = torch.autograd.grad(out, W, dy)
    assert torch.equal(O.embedding(t, W, 1.5), out.detach())
    assert torch.allclose(O.embedding_backward(dy, t, 7, 1.5, padding)[0], want, rtol=1e-14)


def test_embedding_gradient_is_the_differences():
    W = torch.randn((4, 3), generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    t, dy = torch.tensor([3, 1, 3, -1, 4]), torch.arange(15.0, dtype=torch.float64).view(5, 3)
    grad, size = O.embedding_backward(dy, t, 4, 0.5)

    def value(W):
        out = O.embedding(t, W, 0.5)
        assert out[3:].isnan().all()
        return float((out[:3] * dy[:3]).sum())

    for k in range(12):
        up, down = W.clone(), W.clone()
        up.view(-1)[k] += 1e-3
        down.view(-1)[k] -= 1e-3
        assert abs((value(up) - value(down)) / 2e-3 - float(grad.view(-1)[k])) < 1e-9
    assert bool((size >= grad.abs()).all())


def test_mxfp4_by_hand():
    x = torch.zeros(3, 32)
    x[0, :9] = torch.tensor([6.0, -5.0, 0.25, -0.25, 0.75, 2.5, 3.5, -7.0, 0.26])  # largest 7: 2^2, so a scale of 1
    x[1, 0], x[1, 1] = 2.0 ** -126, math.inf
    codes, scales = O.mxfp4_quantize(x)
    assert scales[:, 0].tolist() == [127, 255, 0]
    #           6  -4 (tie)  0 (tie)  -0   1 (tie)  2 (tie)  4 (tie)  -6  0.5
    assert codes[0, :9].tolist() == [7, 8 + 6, 0, 8, 2, 4, 6, 8 + 7, 1]
    packed = O.mxfp4_pack(codes)
    assert packed[0, 0] == 7 + 16 * 14
    assert O.mxfp4_values(packed, scales)[0, :9].tolist() == [6, -4, 0, 0, 1, 2, 4, -6, 0.5]
    assert O.mxfp4_values(packed, scales)[1].isnan().all()


def test_sampling_by_hand():
    z = torch.log(torch.tensor([[0.1, 0.4, 0.2, 0.3]]))
    draw = lambda u, **kw: int(O.sample(z, torch.tensor([u]), **kw)[0])
    assert [draw(u) for u in (0.0, 0.099, 0.101, 0.499, 0.501, 0.699, 0.701, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert [draw(u, top_k=2) for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert [draw(u, top_p=0.39) for u in (0.0, 0.9)] == [1, 1]
    assert [draw(u, top_p=0.5) for u in (0.0, 0.57, 0.58)] == [1, 1, 3]
    assert [draw(u, min_p=0.45) for u in (0.0, 0.44, 0.45, 0.66, 0.67)] == [1, 1, 2, 2, 3]
    assert draw(0.9, temperature=0.0) == 1 and draw(0.2, temperature=0.1) == 1
    tie = torch.zeros(1, 4)
    assert [int(O.sample(tie, torch.tensor([u]), top_k=3)[0]) for u in (0.0, 0.4, 0.9)] == [0, 1, 2]
    assert float(O.sample(z, torch.tensor([0.3]), top_k=2)[1]) == pytest.approx(math.log(0.4 / 0.7), rel=1e-6)


def test_frequencies():
    z = torch.randn((1, 40), generator=torch.Generator().manual_seed(3), dtype=torch.float64)
    n = 20000
    t, l = O.sample(z.expand(n, 40), (torch.arange(n) + 0.5) / n, temperature=0.7)
    p = torch.softmax(z[0] / torch.tensor(0.7).double(), 0)
    assert bool((torch.bincount(t, minlength=40) - n * p).abs().max() <= 1.01)
    assert torch.allclose(l, p[t].log(), rtol=1e-9)

"""Sampling on the GPU against the definition in float64, sorted and added up in order: the same tokens, and their log-probabilities.

A token can differ where a running sum comes within the rounding of the sums (2^-42 of the largest weight for each, fixed by the
vocabulary's size) of u times the whole; the inputs are fixed and none does. A log-probability is rounded once (2^-24 of it), beside
errors below 1e-9.
"""
import math

import numpy as np
import pytest
import torch

from oracle import vocab as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


@pytest.fixture(scope="module")
def lce():
    import paper_2603_16428_amd as m
    m.load_library()
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    return m


def _logits(N, V, dtype, sharp, seed=0):
    g = torch.Generator().manual_seed(1000 * seed + N + V)
    z = 12 + sharp * (1.2 * torch.randn((N, V), generator=g) - torch.log1p(torch.randperm(V, generator=g).float()))
    return z.to(DT[dtype]).cuda(), torch.rand(N, generator=g).cuda()


def _check(lce, z, u, **settings):
    tokens, logs = lce.sample(z, u, **settings, return_logprobs=True)
    V = z.shape[-1]
    flat = {k: v.reshape(-1) if isinstance(v, torch.Tensor) else v for k, v in settings.items()}
    want, want_logs = O.sample(z.reshape(-1, V), u.reshape(-1), **flat)
    got, got_logs = tokens.cpu().reshape(-1), logs.cpu().double().reshape(-1)
    assert tokens.dtype == torch.int64 and tokens.shape == z.shape[:-1]
    assert torch.equal(got, want), (settings, [(int(i), int(got[i]), int(want[i])) for i in (got != want).nonzero()[:4, 0]])
    assert torch.equal(got_logs.isnan(), want_logs.isnan())
    off = (got_logs - want_logs).abs() - (2.0 ** -24 * 1.01 * want_logs.abs() + 1e-9)
    assert not bool((off.nan_to_num(0.0) > 0).any()), float(off.nan_to_num(0.0).max())
    assert torch.equal(lce.sample(z, u, **settings), tokens)


SETTINGS = [dict(), dict(temperature=0.7), dict(temperature=0.0), dict(top_k=1), dict(top_k=5), dict(top_k=50), dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.05),
            dict(top_k=50, top_p=0.95, temperature=0.8), dict(top_k=400, min_p=0.02), dict(top_p=0.99, min_p=0.001, temperature=1.5), dict(top_k=5000, top_p=0.9),
            dict(top_k=3, top_p=0.9, min_p=0.3), dict(top_p=0.0), dict(min_p=1.0)]


# Vocabularies around the groups' and parts' sizes (64, 4096) and the borders from which groups are 128 and 256.
@pytest.mark.parametrize("N,V", [(1, 1), (3, 2), (2, 7), (3, 8), (2, 9), (4, 63), (4, 64), (4, 65), (5, 1000), (3, 4095), (3, 4096), (3, 4097), (2, 50257), (1, 128256)])
@pytest.mark.parametrize("dtype", list(DT))
def test_settings(lce, N, V, dtype):
    for k, s in enumerate(SETTINGS):
        for sharp in (1.5, 0.3):
            _check(lce, *_logits(N, V, dtype, sharp, k), **s)


@pytest.mark.parametrize("V", [262144, 262145, 524288, 524289, 1 << 20])
def test_large_vocabularies(lce, V):
    for k, s in enumerate([dict(), dict(top_k=50, top_p=0.9), dict(top_p=0.9), dict(temperature=0.0), dict(min_p=0.01)]):
        _check(lce, *_logits(2, V, ("fp32", "bf16")[k % 2], 1.0, k), **s)


@pytest.mark.parametrize("dtype", list(DT))
def test_flat_rows(lce, dtype):
    """More logits in question than the list in LDS holds, many of them equal in 16 bits."""
    for s in (dict(top_p=0.5), dict(top_p=0.9), dict(top_p=0.999), dict(top_k=9000), dict(top_k=9000, top_p=0.8), dict(top_k=30000, top_p=0.9, min_p=0.2), dict(min_p=0.2), dict()):
        for sharp in (0.05, 0.6):
            _check(lce, *_logits(3, 60001, dtype, sharp), **s)


@pytest.mark.parametrize("V", [10, 4096, 70000])
def test_equal_logits(lce, V):
    """All are equal: the kept ones are the first, and each has its share of [0, 1) to the last bit where that is a power of two."""
    z = torch.full((8, V), 3.0, dtype=torch.bfloat16, device="cuda")
    z[:, 1::2] = 3.0
    u = torch.tensor([0.0, 0.125, 0.25, 0.5, 0.75, 0.875, 0.999, 1 - 2.0 ** -24], device="cuda")
    for s in (dict(), dict(top_k=8), dict(top_k=1), dict(top_p=0.5), dict(top_k=8, top_p=0.5), dict(min_p=1.0), dict(temperature=0.0), dict(top_k=V - 1)):
        _check(lce, z, u, **s)
    assert lce.sample(z, u, top_k=8).tolist() == [0, 1, 2, 4, 6, 7, 7, 7]
    assert lce.sample(z, u, top_k=8, top_p=0.5).tolist() == [0, 0, 1, 2, 3, 3, 3, 3]


def test_zeros_of_both_signs_are_equal(lce):
    z = torch.zeros((2, 300), device="cuda")
    z[0, ::2] = -0.0
    z[1, 1::2] = -0.0
    for dtype in DT.values():
        for s in (dict(temperature=0.0), dict(top_k=1), dict(top_k=6), dict(top_p=0.1)):
            _check(lce, z.to(dtype), torch.tensor([0.6, 0.6], device="cuda"), **s)


def test_masked_infinite_and_nan(lce):
    """-inf never comes; nothing else, or a NaN, gives -1; +inf are the largest and equal; so are the type's lowest values among masked ones."""
    for dtype in DT.values():
        z = torch.randn((10, 500), device="cuda").to(dtype)
        z[0, ::2] = -math.inf
        z[1, :] = -math.inf
        z[2, :] = -math.inf
        z[2, 77] = torch.finfo(dtype).min
        z[3, 5] = math.nan
        z[4, 9], z[4, 300] = math.inf, math.inf
        z[5, 9], z[5, 10] = math.inf, math.nan
        z[6, :] = torch.finfo(dtype).min
        z[7, :] = torch.finfo(dtype).min
        z[7, 40:44] = torch.finfo(dtype).max
        z[8, 1:] = -math.inf
        u = torch.full((10,), 0.6, device="cuda")
        for s in SETTINGS + [dict(top_k=400), dict(top_k=499, top_p=0.9)]:
            _check(lce, z, u, **s)
        assert lce.sample(z, u)[[1, 3, 5]].tolist() == [-1, -1, -1] and lce.sample(z, u)[4] == 300


def test_numbers_at_and_past_the_ends(lce):
    z, _ = _logits(1, 3000, "fp32", 1.5)
    u = torch.tensor([0.0, -0.0, -1.0, 2.0 ** -149, 1 - 2.0 ** -24, 1.0, 7.0, math.inf, -math.inf, math.nan], device="cuda")
    z = z.expand(10, 3000)
    for s in (dict(), dict(top_k=7), dict(top_p=0.8), dict(temperature=0.0)):
        got = lce.sample(z, u, **s)
        assert got[9] == -1 and bool((got[:9] >= 0).all())
        assert len(set(got[:3].tolist() + got[8:9].tolist())) == 1 and len(set(got[5:8].tolist())) == 1
    _check(lce, z[:5], u[:5], top_k=7)


def test_temperatures_of_any_size(lce):
    z, u = _logits(4, 2000, "fp32", 1.0)
    for t in (1e-38, 1e-6, 1e-3, 100.0, 1e30):
        for s in (dict(), dict(top_k=10), dict(top_p=0.9), dict(min_p=0.5)):
            _check(lce, z, u, temperature=t, **s)


def test_infinite_temperature(lce):
    """All logits above -inf become equal."""
    z, u = _logits(5, 2000, "fp32", 1.0)
    z[:, ::3] = -math.inf
    for s in (dict(), dict(top_k=10), dict(top_p=0.5), dict(min_p=1.0), dict(top_k=1900, top_p=0.5)):
        _check(lce, z, u, temperature=1e30, **s)
        assert torch.equal(lce.sample(z, u, temperature=math.inf, **s), lce.sample(z, u, temperature=1e30, **s))


def test_settings_of_each_row(lce):
    N, V = 64, 5000
    g = torch.Generator().manual_seed(8)
    z, u = _logits(N, V, "bf16", 1.2)

    def pick(values, dtype=torch.float32):
        return torch.tensor(values, dtype=dtype)[torch.randint(0, len(values), (N,), generator=g)].cuda()

    t, p, m = pick([0.0, 0.5, 1.0, 2.0]), pick([0.3, 0.9, 1.0]), pick([0.0, 0.05, 0.5])
    k = pick([0, 1, 20, 5000, 4999], torch.int32)
    _check(lce, z, u, temperature=t, top_k=k, top_p=p, min_p=m)
    _check(lce, z.view(8, 8, V), u.view(8, 8), temperature=t.view(8, 8), top_k=k.view(8, 8), top_p=0.9)
    # Out of their ranges they are off, or at the nearest end.
    odd = torch.tensor([-1.0, 3.0, math.inf, 0.5] * 16, device="cuda")
    assert torch.equal(lce.sample(z, u, temperature=odd.clamp(max=1.0)), lce.sample(z, u, temperature=odd.clamp(0.0, 1.0)))
    assert torch.equal(lce.sample(z, u, top_p=odd), lce.sample(z, u, top_p=odd.clamp(0.0, 1.0)))
    assert torch.equal(lce.sample(z, u, min_p=odd), lce.sample(z, u, min_p=odd.clamp(0.0, 1.0)))
    assert torch.equal(lce.sample(z, u, top_k=k - 10), lce.sample(z, u, top_k=(k - 10).clamp(min=0)))


def test_rows_of_a_wider_buffer(lce):
    wide, u = _logits(6, 3000, "bf16", 1.0)
    for at, V in ((1, 1000), (3, 2049), (8, 64)):
        _check(lce, wide[:, at:at + V], u, top_k=20)
        _check(lce, wide[:, at:at + V], u, top_p=0.9)
        _check(lce, wide[:, at:at + V], u)
    assert lce.sample(wide[:0], u[:0]).shape == (0,)
    assert lce.sample(wide[0], u[0]).shape == ()


def test_shares(lce):
    """Evenly spaced numbers over one row (shared by all): every kept token comes as often as its share."""
    z, _ = _logits(1, 3000, "fp32", 1.0)
    N = 20000
    u = ((torch.arange(N, device="cuda") + 0.5) / N).float()
    for s in (dict(), dict(top_k=40), dict(top_p=0.8, temperature=1.3)):
        tokens = lce.sample(z.expand(N, 3000), u, **s)
        assert bool((tokens[1:] >= tokens[:-1]).all())
        want, logs = O.sample(z.expand(8, 3000), u[:8], **s)
        p = torch.softmax(z[0].double() / s.get("temperature", 1.0), 0)
        kept = torch.zeros_like(p)
        order = torch.argsort(z[0], descending=True, stable=True)
        n = s.get("top_k", 3000)
        if "top_p" in s:
            n = int((torch.cumsum(p[order], 0) - p[order] < 0.8).sum())
        kept[order[:n]] = p[order[:n]]
        assert bool((torch.bincount(tokens, minlength=3000) - N * kept / kept.sum()).abs().max() <= 1.5)


def test_refusals(lce):
    z, u = _logits(4, 100, "fp32", 1.0)
    k = torch.ones(4, device="cuda")
    for call in (lambda: lce.sample(z.double(), u), lambda: lce.sample(z, u.double()), lambda: lce.sample(z, u[:3]), lambda: lce.sample(z, u.cpu()), lambda: lce.sample(z.t(), u),
                 lambda: lce.sample(z, u, temperature=-1.0), lambda: lce.sample(z, u, temperature=math.nan), lambda: lce.sample(z, u, top_k=-1), lambda: lce.sample(z, u, top_p=-0.5),
                 lambda: lce.sample(z, u, min_p=1.1), lambda: lce.sample(z, u, top_k=k), lambda: lce.sample(z, u, temperature=k[:2]), lambda: lce.sample(z, u, top_p=k.cpu()),
                 lambda: lce.sample(z, u, min_p=torch.ones(8, device="cuda")[::2]), lambda: lce.sample(z, u, workspace=torch.empty(4, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: lce.sample(z, u, workspace=torch.empty(4, dtype=torch.uint8, device="cuda")),
                 lambda: lce.sample(torch.empty((1, (1 << 20) + 1), dtype=torch.bfloat16, device="cuda"), u[:1])):
        with pytest.raises(lce.LCEError):
            call()


def test_streams_and_graphs(lce):
    """On a side stream; two graphs with a workspace each, replayed in turn on logits, numbers and settings changed in place."""
    N, V = 6, 9000
    z, u = _logits(N, V, "bf16", 1.3)
    t, k = torch.full((N,), 0.9, device="cuda"), torch.tensor([0, 1, 5, 50, 0, 0], dtype=torch.int32, device="cuda")
    p = torch.tensor([1.0, 1.0, 0.9, 0.9, 0.9, 0.9999], device="cuda")
    spaces = [torch.empty(lce.sample_workspace_size(N, V), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def everything(ws):
        return lce.sample(z, u, t, k, p, 0.0, True, ws) + (lce.sample(z, u, workspace=ws), lce.sample(z, u, temperature=0.0, workspace=ws))

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
    for r in range(4):
        for g, outs in graphs:
            for o in outs:
                o.zero_()
            g.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            assert all(torch.equal(a, b) for a, b in zip(outs, want)), r
        z.copy_(z.roll(17, 1))
        u.copy_((u + 0.31) % 1.0)
        t.mul_(1.1)
        k.copy_(k.roll(1))
        want = everything(spaces[0])
        torch.cuda.synchronize()


@pytest.mark.parametrize("V", [262144, 300001, 1 << 20])
def test_many_small_weights_together(lce, V):
    """One large logit and a tail whose weights are some 2^-43 of its own each, but count together: u times the whole falls into the token's part, to
    2^-25 of the whole, twice that where top-p's end is looked for as well (exact sums: extended precision, whose own roundings are V 2^-64)."""
    u = torch.tensor([0.0, 1e-8, 2e-8, 5e-8, 0.5, 1 - 2.0 ** -24], device="cuda")
    for tail in (2.0 ** -43.05, 2.0 ** -44.05):
        for large in (0, V // 2, V - 1):
            z = torch.full((V,), math.log(tail), device="cuda")
            z[large] = 0.0
            w = np.exp(z.cpu().double().numpy()).astype(np.longdouble)
            for settings in (dict(), dict(min_p=1e-30), dict(top_k=V - 1), dict(top_p=1 - 2.0 ** -24), dict(top_p=1 - 2.0 ** -24, min_p=1e-30)):
                kept = w.copy()
                if "top_k" in settings:  # all but the last of the equal ones
                    kept[V - 1 if large != V - 1 else V - 2] = 0
                running = np.cumsum(kept)
                if "top_p" in settings:  # the large one and the first of the tail
                    last = int(np.searchsorted(np.cumsum(np.delete(w, large)), settings["top_p"] * running[-1] - 1))
                    kept[np.delete(np.arange(V), large)[last + 1:]] = 0
                    running = np.cumsum(kept)
                off = (2.0 ** -24 if "top_p" in settings else 2.0 ** -25) * running[-1]
                tokens, logs = lce.sample(z.expand(len(u), V), u, **settings, return_logprobs=True)
                for t, log, at in zip(tokens.tolist(), logs.tolist(), u.double().tolist()):
                    case = (V, tail, large, settings, at, t)
                    aim = np.longdouble(at) * running[-1]
                    assert running[t] - w[t] - off <= aim <= running[t] + off, case
                    want = float(z[t].double()) - float(np.log(running[-1]))
                    assert abs(log - want) <= 2.0 ** -24 * 1.01 * abs(want) + off, case


@pytest.mark.parametrize("V", [9000, 100003, 150016])
def test_all_three_settings_beyond_the_groups(lce, V):
    """A top-k above the number of groups (V / 64) with top-p and min-p, peaked and nearly flat: neither tables nor a bound by the groups."""
    for dtype in DT:
        for sharp in (1.5, 0.05):
            _check(lce, *_logits(3, V, dtype, sharp, 5), top_k=3000, top_p=0.9, min_p=0.05)

"""The residual's addition with RMSNorm (rows in their own type and in e4m3) and its backward on the GPU,
against float64.

Bounds, with u = eps / 2 of the type (half a step) and w = 2^-24 (fp32's): an fp32 sum of H terms goes
through at most 32 terms in one thread and 10 joins, so a row's mean square is at most 44 w off and r = 1/sqrt
half of that and 4 w; with the two products and s, normed is at most (22 + 4 + 3) w < 32 w and the output's
rounding u off. In fp16 a value below 2^-14 rounds to a step of 2^-24 (half: 2^-25).
"""
import pytest
import torch

from oracle import ops as O

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
W = 2.0 ** -24
EPS = 1e-5


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


def _inputs(N, H, dtype, seed=0, scale=True):
    g = torch.Generator().manual_seed(1000 * N + H + seed)
    size = torch.exp(torch.empty(N, 1).uniform_(-1.4, 2.8, generator=g)) if scale else 1.0
    x, r = (size * torch.randn((N, H), generator=g) for _ in range(2))
    gamma = 1.0 + 0.2 * torch.randn(H, generator=g)
    dy, ds = (torch.randn((N, H), generator=g) for _ in range(2))
    return tuple(t.to(DT[dtype]).cuda() for t in (x, r, gamma, dy, ds))


def _near(got, want, rel, absolute=0.0):
    """|got - want| <= rel |want| + absolute, element by element (both may be tensors)."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape
    off = (got - want).abs() - (rel * want.abs() + absolute)
    assert bool((off <= 0).all()), f"{float(off.max()):.3g} over the bound at {int(off.argmax())} of {got.numel()}"


def _check_forward(normed, added, rstd, x, residual, gamma, eps=EPS):
    dtype = x.dtype
    y, s, r = O.add_rmsnorm(x, residual, gamma, eps)
    _near(normed, y, _u(dtype) * (1 + 32 * W) + 32 * W, _step(dtype))
    if residual is not None:
        _near(added, s, _u(dtype) + 2 * W, _step(dtype))
    if rstd is not None:
        _near(rstd, r, 28 * W)


# Widths around the borders between the kernel's variants, and ends of rows of every kind.
WIDTHS = [1, 7, 8, 9, 64, 127, 128, 129, 249, 256, 257, 500, 512, 513, 1000, 1024, 1025, 2041, 2048, 2056, 4096, 4097, 6144, 6152, 8192, 8199,
          12288, 12296, 16384, 16385, 32761, 32768]


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("H", WIDTHS)
def test_forward(lce, H, dtype):
    for N in (1, 2, 17, 50):
        x, r, gamma, _, _ = _inputs(N, H, dtype)
        normed, added, rstd = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
        _check_forward(normed, added, rstd, x, r, gamma)
        alone, same = lce.add_rmsnorm_forward(x, None, gamma, EPS)
        assert same is x
        _check_forward(alone, None, None, x, None, gamma)


def test_many_rows(lce):
    for N, H, dtype in ((70001, 128, "bf16"), (5003, 768, "fp16"), (3001, 72, "fp32"), (1500, 4096, "bf16")):
        x, r, gamma, _, _ = _inputs(N, H, dtype)
        _check_forward(*lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True), x, r, gamma)


def test_more_rows_than_a_grid(lce):
    """17 million rows of 8 values: more than one workgroup for 16 rows allows, so the kernel walks on; rows after
    the last one stay."""
    N, H = 17_000_003, 8
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((N, H), generator=g, device="cuda").to(torch.bfloat16)
    gamma = (1 + 0.1 * torch.randn(H, generator=g, device="cuda")).to(torch.bfloat16)
    out = torch.full((N + 50, H), 5.0, dtype=torch.bfloat16, device="cuda")
    lce.add_rmsnorm_forward(x, None, gamma, EPS, normed=out[:N])
    assert bool((out[N:] == 5).all())
    for at in (slice(0, 4000), slice((1 << 24) - 2000, (1 << 24) + 2000), slice(N - 4000, N)):
        _check_forward(out[at], None, None, x[at], None, gamma)
    want = x.double() * (x.double().square().mean(1, keepdim=True) + EPS).rsqrt() * gamma.double()
    # Within one step of bfloat16 (2^-7) everywhere; most exactly its rounding.
    assert bool(((out[:N].double() - want).abs() <= 2.0 ** -8 * 1.001 * want.abs()).all())


def test_no_rows(lce):
    x, r, gamma, _, _ = _inputs(1, 64, "bf16")
    x, r = x[:0], r[:0]
    normed, added, rstd = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
    assert normed.shape == added.shape == (0, 64) and rstd.shape == (0,)
    q, scales, _ = lce.add_rmsnorm_quant(x, r, gamma, EPS, 32)
    assert q.shape == (0, 64) and scales.shape == (0, 2)
    dx, dg = lce.add_rmsnorm_backward(normed, added, x, r, gamma, rstd)
    assert dx.shape == (0, 64) and not dg.any()


@pytest.mark.parametrize("dtype", list(DT))
def test_shapes_strides_and_alignment(lce, dtype):
    """Leading dimensions, rows of wider buffers at any element's alignment, one row for all; outputs in columns
    of a buffer whose other values stay."""
    x, r, gamma, _, _ = _inputs(24, 1000, dtype)
    for H, at in ((200, 1), (519, 3), (128, 8)):
        xs, rs, gs = x.view(4, 6, 1000)[:, :, at:at + H], r.view(4, 6, 1000)[:, :, 2 * at:2 * at + H], gamma[at:at + H]
        buf = torch.full((24, 2000), 7.0, dtype=DT[dtype], device="cuda")
        normed, added = buf[:, 5:5 + H].view(4, 6, H), buf[:, 1001:1001 + H].view(4, 6, H)
        got = lce.add_rmsnorm_forward(xs, rs, gs, EPS, normed=normed, added=added, return_rstd=True)
        assert got[0] is normed and got[1] is added and got[2].shape == (4, 6)
        _check_forward(*(t.reshape(24, -1).squeeze(-1) if t.dim() == 2 else t.reshape(24, H) if t.dim() == 3 else t
                         for t in got[:2]), got[2].reshape(24), xs.reshape(24, H), rs.reshape(24, H), gs)
        rest = torch.ones(2000, dtype=torch.bool, device="cuda")
        rest[5:5 + H] = rest[1001:1001 + H] = False
        assert bool((buf[:, rest] == 7.0).all())
    one = r[:1].expand(24, 1000)
    _check_forward(*lce.add_rmsnorm_forward(x, one, gamma, EPS), None, x, one, gamma)
    row = x[3]
    normed, added = lce.add_rmsnorm_forward(row, r[3], gamma, EPS)
    assert normed.shape == (1000,)
    _check_forward(normed, added, None, row, r[3], gamma)


@pytest.mark.parametrize("H", [128, 1000, 4096, 12288, 32768])
def test_in_place(lce, H):
    x, r, gamma, dy, ds = _inputs(33, H, "bf16")
    want = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
    a, b = x.clone(), r.clone()
    normed, added, rstd = lce.add_rmsnorm_forward(a, b, gamma, EPS, normed=a, added=b, return_rstd=True)
    assert normed is a and added is b
    for got, w in zip((normed, added, rstd), want):
        assert torch.equal(got, w)
    a, b = x.clone(), r.clone()
    lce.add_rmsnorm_forward(a, b, gamma, EPS, normed=b, added=a)
    assert torch.equal(b, want[0]) and torch.equal(a, want[1])
    dx, dg = lce.add_rmsnorm_backward(dy, ds, x, r, gamma, want[2])
    for k in range(4):
        ins = [dy.clone(), ds.clone(), x.clone(), r.clone()]
        got, gg = lce.add_rmsnorm_backward(*ins, gamma, want[2], grad_hidden=ins[k])
        assert got is ins[k] and torch.equal(got, dx) and torch.equal(gg, dg)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H", [5, 129, 257, 513, 1025, 1543, 2049, 4097, 6151, 8199, 12289, 16385, 32761])
def test_in_place_of_odd_widths(lce, H, dtype):
    """A row's last values are loaded with some of the thread's before (of another wave, where H is just above a
    multiple of 512): in place they are the old ones all the same, in both directions, with rows back to back."""
    x, r, gamma, dy, ds = _inputs(33, H, dtype, seed=4)
    want = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
    for k in range(2):
        ins = [x.clone(), r.clone()]
        got = lce.add_rmsnorm_forward(*ins, gamma, EPS, normed=ins[k], added=ins[1 - k])
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    q = lce.add_rmsnorm_quant(x, r, gamma, EPS, 64)
    a = x.clone()
    got = lce.add_rmsnorm_quant(a, r, gamma, EPS, 64, added=a)
    assert got[2] is a and torch.equal(a, q[2]) and torch.equal(got[0].view(torch.uint8), q[0].view(torch.uint8))
    dx, dg = lce.add_rmsnorm_backward(dy, ds, x, r, gamma, want[2])
    for k in range(4):
        ins = [dy.clone(), ds.clone(), x.clone(), r.clone()]
        got, gg = lce.add_rmsnorm_backward(*ins, gamma, want[2], grad_hidden=ins[k])
        assert got is ins[k] and torch.equal(got, dx) and torch.equal(gg, dg)


def test_rows_that_are_not_finite_or_zero(lce):
    x, r, gamma, _, _ = _inputs(12, 1000, "bf16")
    clean = lce.add_rmsnorm_forward(x, r, gamma, EPS)
    x2, r2 = x.clone(), r.clone()
    x2[2, 5] = float("nan")
    x2[4, 7] = float("inf")
    r2[6, 999] = float("-inf")
    x2[8], r2[8] = 0.0, 0.0
    normed, added = lce.add_rmsnorm_forward(x2, r2, gamma, EPS)
    others = [0, 1, 3, 5, 7, 9, 10, 11]
    assert torch.equal(normed[others], clean[0][others]) and torch.equal(added[others], clean[1][others])
    assert normed[2].isnan().all() and not normed[8].any()
    for i, j in ((4, 7), (6, 999)):  # r = 0: the infinite value gives NaN, the others 0
        assert normed[i, j].isnan() and int((normed[i] == 0).sum()) == 999
    q, scales, _ = lce.add_rmsnorm_quant(x2, r2, gamma, EPS, 128)
    qc, sc, _ = lce.add_rmsnorm_quant(x, r, gamma, EPS, 128)
    assert torch.equal(q[others].view(torch.uint8), qc[others].view(torch.uint8)) and torch.equal(scales[others], sc[others])
    assert q[2].float().isnan().all() and scales[2].isnan().all()
    assert scales[4, 0].isnan() and q[4, :128].float().isnan().all() and not q[4, 128:].float().any()
    assert not q[8].float().any() and bool((scales[8] == O.SCALE_MIN).all())
    q, scales, _ = lce.add_rmsnorm_quant(x2, r2, gamma, EPS)
    assert q[2].float().isnan().all() and scales[4, 0].isnan() and q[4].float().isnan().all()
    assert not q[8].float().any() and float(scales[8]) == O.SCALE_MIN


def test_eps_zero_and_tiny_values(lce):
    x, r, gamma, _, _ = _inputs(9, 257, "fp32")
    for scale in (1e-15, 1e15):  # mean squares of 1e-30 and 1e30
        _check_forward(*lce.add_rmsnorm_forward(x * scale, r * scale, gamma, 0.0), None, x * scale, r * scale, gamma, 0.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_sums_of_many_waves(lce, dtype):
    """The 16 waves of the widest rows hold 2^24 and fifteen ones (their squares are exact). Joined in pairs, four
    roundings of w at most: 2 w in r, and 2 w for the rsqrt. Joined in a chain every one is lost: 15 w, 7.5 w in r."""
    x = torch.zeros((3, 32768), dtype=DT[dtype], device="cuda")
    x[:, ::512][:, :16] = 1.0
    x[:, 0] = 4096.0
    gamma = torch.ones(32768, dtype=DT[dtype], device="cuda")
    _, _, r = lce.add_rmsnorm_forward(x, None, gamma, 0.0, return_rstd=True)
    want = ((2.0 ** 24 + 15) / 32768) ** -0.5
    assert bool(((r.cpu().double() - want).abs() <= 4 * W * want).all())


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("H", [1, 8, 31, 33, 100, 128, 129, 136, 250, 256, 512, 520, 1024, 1030, 2048, 4096, 4100, 6000, 8192, 12288, 16384, 20000])
def test_quant(lce, H, group, dtype):
    """A value is at most half a step of e4m3 off: 2^-4 of it, or 2^-10 of the scale where it is below 2^-6 scale
    (and 96 w for the fp32 arithmetic of the value and its scale); each group's largest is 448."""
    N = 19
    x, r, gamma, _, _ = _inputs(N, H, dtype)
    q, scales, added, rstd = lce.add_rmsnorm_quant(x, r, gamma, EPS, group, return_rstd=True)
    y, s, rr = O.add_rmsnorm(x, r, gamma, EPS)
    _near(added, s, _u(x.dtype) + 2 * W, _step(x.dtype))
    _near(rstd, rr, 28 * W)
    want = O.group_scales(y, group)
    sc = scales.view(N, -1)
    assert scales.shape == want.shape and q.dtype == torch.float8_e4m3fn
    _near(sc, want, 36 * W)
    wide = want.repeat_interleave(group or H, 1)[:, :H]
    values = q.float().cpu().double() * sc.cpu().double().repeat_interleave(group or H, 1)[:, :H]
    bound = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * wide) + 96 * W * y.abs()
    assert bool(((values - y).abs() <= bound).all())
    top = torch.nn.functional.pad(q.float().abs(), (0, -H % (group or H))).view(N, -1, group or H).amax(-1)
    assert bool((top == 448).all())
    alone = lce.add_rmsnorm_quant(x, None, gamma, EPS, group)
    assert alone[2] is x
    _near(alone[1].view(N, -1), O.group_scales(O.add_rmsnorm(x, None, gamma, EPS)[0], group), 36 * W)


def test_quant_at_the_smallest_scale(lce):
    """Values around 2^-126 and below (a tiny gain): the scale stays at 2^-126, and fp32's own smallest step, 2^-149,
    is what the arithmetic may be off (a few times)."""
    x, r, gamma, _, _ = _inputs(7, 300, "fp32")
    for group in (0, 32):
        for size in (2.0 ** -122, 2.0 ** -130):
            g = gamma * size
            q, scales, _ = lce.add_rmsnorm_quant(x, r, g, EPS, group)
            y, _, _ = O.add_rmsnorm(x, r, g, EPS)
            assert bool((scales == O.SCALE_MIN).all())
            off = (q.float().cpu().double() * O.SCALE_MIN - y).abs()
            assert bool((off <= torch.clamp(2.0 ** -4 * y.abs(), min=2.0 ** -10 * O.SCALE_MIN) + 96 * W * y.abs() + 8 * 2.0 ** -149).all())
            assert q.float().abs().max() > 0.1


def _check_quant(lce, x, res, gamma, group, eps=EPS):
    """test_quant's bounds, and 8 of fp32's own smallest steps for values next to the smallest scale."""
    q, scales, added = lce.add_rmsnorm_quant(x, res, gamma, eps, group)
    N, H = x.shape
    y, _, _ = O.add_rmsnorm(x, res, gamma, eps)
    want = O.group_scales(y, group)
    _near(scales.view(N, -1), want, 36 * W)
    wide = want.repeat_interleave(group or H, 1)[:, :H]
    values = q.float().cpu().double() * scales.view(N, -1).cpu().double().repeat_interleave(group or H, 1)[:, :H]
    bound = torch.maximum(2.0 ** -4 * y.abs(), 2.0 ** -10 * wide) + 96 * W * y.abs() + 8 * 2.0 ** -149
    assert bool(((values - y).abs() <= bound).all())  # false where a value is NaN
    top = torch.nn.functional.pad(q.float().cpu().abs(), (0, -H % (group or H))).view(N, -1, group or H).amax(-1)
    assert bool((top[want > O.SCALE_MIN * (1 + 36 * W)] == 448).all())


@pytest.mark.parametrize("group", [0, 32, 128])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H", [6, 264, 4096])
def test_quant_of_tiny_groups(lce, H, dtype, group):
    """Finite scales around the least one, in rows of every size: gains that have decayed to almost nothing,
    throughout a row and in one group beside ordinary ones; rows of such values."""
    g = torch.Generator().manual_seed(H + group)
    rms = torch.tensor([1.0, 0.2, 0.02, 0.002]).repeat_interleave(3)[:, None]
    x, res = ((rms * torch.randn((12, H), generator=g) / 2 ** 0.5).to(DT[dtype]).cuda() for _ in range(2))
    gain = 1.0 + 0.2 * torch.randn(H, generator=g)
    for e in range(-132, -100, 2):
        _check_quant(lce, x, res, (gain * 2.0 ** e).to(DT[dtype]).cuda(), group)
        one = gain.clone()
        one[32:64] *= 2.0 ** e
        _check_quant(lce, x, res, one.to(DT[dtype]).cuda(), group)
    sizes = torch.tensor([2e-36, 1e-36, 5e-37, 1e-37, 1e-38, 1e-40])[:, None]
    rows = [(sizes * torch.randn((6, H), generator=g)).to(DT[dtype]).cuda() for _ in range(2)]
    _check_quant(lce, *rows, gain.to(DT[dtype]).cuda(), group)
    _check_quant(lce, rows[0], None, gain.to(DT[dtype]).cuda(), group)


def test_quant_of_any_product(lce):
    """Rows and gains whose products leave fp32 while the normalised values do not."""
    x, res, gamma, _, _ = _inputs(9, 257, "fp32")
    for size, gain in ((1e15, 1e28), (1e15, 1e-35), (1e-15, 1e-30), (1e-15, 1e35)):
        for group in (0, 32):
            _check_quant(lce, x * size, res * size, gamma * gain, group, eps=0.0)


def test_quant_into_a_wider_buffer(lce):
    x, r, gamma, _, _ = _inputs(6, 300, "bf16")
    buf = torch.full((6, 511), 1.0, device="cuda").to(torch.float8_e4m3fn)
    q, scales, _ = lce.add_rmsnorm_quant(x, r, gamma, EPS, 64, quantised=buf[:, 3:303])
    want = lce.add_rmsnorm_quant(x, r, gamma, EPS, 64)
    assert torch.equal(q.contiguous().view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(scales, want[1])
    assert bool((buf[:, :3].float() == 1).all()) and bool((buf[:, 303:].float() == 1).all())


def _check_backward(dx, dg, dy, ds, x, res, gamma, r):
    """From r as the forward left it. dx is at most its rounding off, and the fp32 arithmetic: a row's dot product at most 48 w of its terms'
    magnitudes, times r^3 |s|; a few w of the other terms. dgamma: a chain of at most N / 256 + 100 additions."""
    dtype = x.dtype
    s = x.cpu().double() + (0 if res is None else res.cpu().double())
    want, wg = O.add_rmsnorm_backward(dy, ds, s, gamma, r)
    f = [None if t is None else t.detach().cpu().double().abs() for t in (dy, ds, s, gamma, r)]
    rr = f[4][:, None]
    terms = rr * f[3] * f[0] + (0 if ds is None else f[1])
    dot = rr ** 3 * f[2] * (f[0] * f[3] * f[2]).mean(1, keepdim=True)
    _near(dx, want, _u(dtype), W * (8 * terms + 64 * dot) + _step(dtype))
    if dg is not None:
        _near(dg, wg, _u(dtype), W * (s.shape[0] / 256 + 100) * (f[0] * f[2] * rr).sum(0) + _step(dtype))


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("H", WIDTHS)
def test_backward(lce, H, dtype):
    for N in (1, 2, 19, 50):
        x, res, gamma, dy, ds = _inputs(N, H, dtype, seed=1)
        _, s, r = lce.add_rmsnorm_forward(x, res, gamma, EPS, return_rstd=True)
        _check_backward(*lce.add_rmsnorm_backward(dy, ds, x, res, gamma, r), dy, ds, x, res, gamma, r)
        _check_backward(*lce.add_rmsnorm_backward(dy, ds, s, None, gamma, r), dy, ds, s, None, gamma, r)
        dx, none = lce.add_rmsnorm_backward(dy, None, x, res, gamma, r, need_gamma=False)
        assert none is None
        _check_backward(dx, None, dy, None, x, res, gamma, r)


def test_backward_of_many_rows(lce):
    """More rows than workgroups, in every kind of variant."""
    for N, H, dtype in ((40001, 128, "bf16"), (20001, 200, "bf16"), (9001, 500, "fp16"), (5003, 768, "fp16"), (4099, 2048, "bf16"), (3001, 4096, "bf16"),
                        (1500, 12288, "fp32"), (700, 20000, "bf16")):
        x, res, gamma, dy, ds = _inputs(N, H, dtype, seed=2)
        _, s, r = lce.add_rmsnorm_forward(x, res, gamma, EPS, return_rstd=True)
        ws = torch.full((lce.add_rmsnorm_workspace_size(N, H, DT[dtype]),), 255, dtype=torch.uint8, device="cuda")
        first = lce.add_rmsnorm_backward(dy, ds, x, res, gamma, r, workspace=ws)
        _check_backward(*first, dy, ds, x, res, gamma, r)
        for got, want in zip(lce.add_rmsnorm_backward(dy, ds, x, res, gamma, r), first):
            assert torch.equal(got, want)


def test_backward_strides(lce):
    x, res, gamma, dy, ds = _inputs(18, 999, "bf16", seed=3)
    H = 301
    xs, rs = x[:, 1:1 + H], res[:, 2:2 + H]
    _, _, r = lce.add_rmsnorm_forward(xs, rs, gamma[:H], EPS, return_rstd=True)
    buf = torch.full((18, 640), 3.0, dtype=torch.bfloat16, device="cuda")
    one = dy[:1, 4:4 + H].expand(18, H)
    dx, dg = lce.add_rmsnorm_backward(one, ds[:, 5:5 + H], xs, rs, gamma[:H], r, grad_hidden=buf[:, 7:7 + H])
    _check_backward(dx, dg, one, ds[:, 5:5 + H], xs, rs, gamma[:H], r)
    assert bool((buf[:, :7] == 3).all()) and bool((buf[:, 7 + H:] == 3).all())


@pytest.mark.parametrize("dtype", list(DT))
def test_autograd(lce, dtype):
    x, res, gamma, dy, ds = _inputs(37, 200, dtype, seed=5)
    leaves = [t.requires_grad_() for t in (x, res, gamma)]
    normed, added = lce.add_rmsnorm(*leaves, EPS)
    grads = torch.autograd.grad((normed, added), leaves, (dy, ds), retain_graph=True)
    ins = [t.detach() for t in leaves]
    _, _, r = lce.add_rmsnorm_forward(*ins, EPS, return_rstd=True)
    dx, dg = lce.add_rmsnorm_backward(dy, ds, *ins, r)
    assert torch.equal(grads[0], dx) and torch.equal(grads[1], dx) and torch.equal(grads[2], dg)
    # One output's gradient alone; some inputs alone; gradients that are expanded, transposed, negated, zero.
    only = torch.autograd.grad(added, (x, gamma), ds, retain_graph=True)
    assert torch.equal(only[0], ds) and not only[1].any()
    dx0, dg0 = lce.add_rmsnorm_backward(dy, None, *ins, r)
    assert torch.equal(torch.autograd.grad(normed, gamma, dy, retain_graph=True)[0], dg0)
    assert torch.equal(torch.autograd.grad(normed, res, dy, retain_graph=True)[0], dx0)
    assert torch.equal(torch.autograd.grad(normed, x, dy.t().contiguous().t(), retain_graph=True)[0], dx0)
    want = lce.add_rmsnorm_backward(torch.ones_like(dy), None, *ins, r)[0]
    assert torch.equal(torch.autograd.grad(normed.sum(), x, retain_graph=True)[0], want)
    assert torch.equal(torch.autograd.grad(normed, x, torch._neg_view(-dy), retain_graph=True)[0], dx0)
    zero = torch._efficientzerotensor(dy.shape, dtype=dy.dtype, device="cuda")
    assert not torch.autograd.grad(normed, x, zero, retain_graph=True)[0].any()
    with pytest.raises((RuntimeError, ValueError)):  # batched gradients
        torch.autograd.grad(normed, x, torch.stack([dy, dy]), retain_graph=True, is_grads_batched=True)
    with pytest.raises(RuntimeError):  # once differentiable
        g, = torch.autograd.grad((normed * normed).sum(), x, create_graph=True)
        torch.autograd.grad(g.sum(), x)
    # The norm alone.
    y = lce.rmsnorm(leaves[0], leaves[2], EPS)
    _, same, r1 = lce.add_rmsnorm_forward(x.detach(), None, gamma.detach(), EPS, return_rstd=True)
    want = lce.add_rmsnorm_backward(dy, None, same, None, gamma.detach(), r1)
    for got, w in zip(torch.autograd.grad(y, (x, gamma), dy), want):
        assert torch.equal(got, w)
    with torch.no_grad():
        assert not lce.rmsnorm(x, gamma, EPS).requires_grad
    with torch.inference_mode():
        a, b = x * 1, res * 1
        assert lce.add_rmsnorm_forward(a, b, gamma, EPS, normed=a, added=b)[0] is a


def test_autograd_of_shared_and_broadcast_inputs(lce):
    """One tensor as both addends, one row added to all, no rows, a single row."""
    x, res, gamma, dy, ds = _inputs(30, 136, "fp32", seed=8)
    a = x.clone().requires_grad_()
    got, = torch.autograd.grad(lce.add_rmsnorm(a, a, gamma, EPS), a, (dy, ds))
    _, s, r = lce.add_rmsnorm_forward(x, x, gamma, EPS, return_rstd=True)
    dx, _ = lce.add_rmsnorm_backward(dy, ds, x, x, gamma, r)
    assert torch.equal(got, dx + dx)
    one = res[:1].clone().requires_grad_()
    got, = torch.autograd.grad(lce.add_rmsnorm(x, one.expand(30, 136), gamma, EPS), one, (dy, ds))
    _, s, r = O.add_rmsnorm(x, res[:1], gamma, EPS)
    want, _ = O.add_rmsnorm_backward(dy, ds, s, gamma, r)
    # Each row's gradient as in _check_backward (w for its rounding), and 30 fp32 additions of the rows.
    f = [t.cpu().double().abs() for t in (dy, ds, s, gamma, r[:, None])]
    rows = 8 * (f[4] * f[3] * f[0] + f[1]) + 64 * f[4] ** 3 * f[2] * (f[0] * f[3] * f[2]).mean(1, keepdim=True) + want.abs()
    assert bool(((got[0].cpu().double() - want.sum(0)).abs() <= W * (rows.sum(0) + 30 * want.abs().sum(0))).all())
    empty, g = x[:0].clone().requires_grad_(), gamma.clone().requires_grad_()
    grads = torch.autograd.grad(lce.rmsnorm(empty, g, EPS).sum(), (empty, g))
    assert grads[0].shape == (0, 136) and not grads[1].any()
    row = x[0].clone().requires_grad_()
    got = torch.autograd.grad(lce.rmsnorm(row, g, EPS), (row, g), dy[0])
    _, s, r = lce.add_rmsnorm_forward(x[:1], None, gamma, EPS, return_rstd=True)
    want = lce.add_rmsnorm_backward(dy[:1], None, x[:1], None, gamma, r)
    assert torch.equal(got[0], want[0][0]) and torch.equal(got[1], want[1])


def test_hooks_that_change_what_was_saved(lce):
    """Saved tensors that come back on the host, in another type or shape are refused; copies are fine."""
    x, res, gamma, dy, ds = _inputs(5, 64, "bf16", seed=13)
    leaves = [t.requires_grad_() for t in (x, res, gamma)]
    want = torch.autograd.grad(lce.add_rmsnorm(*leaves, EPS), leaves, (dy, ds))
    with torch.autograd.graph.save_on_cpu():
        outs = lce.add_rmsnorm(*leaves, EPS)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(outs, leaves, (dy, ds)), want))
    for change in (lambda t: t.cpu(), lambda t: t.double(), lambda t: t[..., :1], torch._neg_view):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
            outs = lce.add_rmsnorm(*leaves, EPS)
        with pytest.raises(ValueError):
            torch.autograd.grad(outs, leaves, (dy, ds))


def test_two_streams_at_once(lce):
    """Calls on two streams that run at the same time, each with its own outputs and workspace."""
    sets = [_inputs(2000, 4096, "bf16", seed=k) for k in (20, 21)]
    want = []
    for x, r, g, dy, ds in sets:
        n, a, rs = lce.add_rmsnorm_forward(x, r, g, EPS, return_rstd=True)
        want.append((n, a, *lce.add_rmsnorm_backward(dy, ds, x, r, g, rs), lce.grad_norm([n, a])))
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(3):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                x, r, g, dy, ds = sets[k]
                n, a, rs = lce.add_rmsnorm_forward(x, r, g, EPS, return_rstd=True)
                got[k].append((n, a, *lce.add_rmsnorm_backward(dy, ds, x, r, g, rs), lce.grad_norm([n, a])))
    torch.cuda.synchronize()
    for k in range(2):
        for outs in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(outs, want[k]))


def test_gradients_are_the_forwards_differences(lce):
    """Along random directions, with the outputs' values in float64 from the formula: the derivative of
    <dy, normed> + <ds, added> by central differences (step 1e-6, whose own error is below 1e-8 of the terms)
    against the kernel's fp32 gradients (64 w of the terms' magnitudes)."""
    x, res, gamma, dy, ds = _inputs(6, 130, "fp32", seed=6)
    leaves = [t.requires_grad_() for t in (x, res, gamma)]
    grads = torch.autograd.grad(lce.add_rmsnorm(*leaves, EPS), leaves, (dy, ds))
    at = [t.detach().cpu().double() for t in (x, res, gamma)]
    up = [t.cpu().double() for t in (dy, ds)]

    def value(p):
        y, s, _ = O.add_rmsnorm(*p, EPS)
        return float((y * up[0]).sum() + (s * up[1]).sum())

    gen = torch.Generator().manual_seed(1)
    for k in range(3):
        for _ in range(3):
            d = torch.randn(at[k].shape, generator=gen, dtype=torch.float64)
            a, b = ([t + s * 1e-6 * d if j == k else t for j, t in enumerate(at)] for s in (1, -1))
            diff = (value(a) - value(b)) / 2e-6
            g = grads[k].cpu().double()
            size = float((g.abs() * d.abs()).sum())
            assert abs(float((g * d).sum()) - diff) <= (64 * W + 1e-6) * size


def test_offsets_past_32_bits(lce):
    """Rows 2^30 values apart: the third is 2^32 bytes away."""
    buf = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    x, r, gamma, dy, ds = _inputs(3, 4096, "bf16", seed=7)
    far = buf.as_strided((3, 4096), (1 << 30, 1))
    far.copy_(x)
    want = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
    got = lce.add_rmsnorm_forward(far, r, gamma, EPS, return_rstd=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    lce.add_rmsnorm_forward(x, r, gamma, EPS, normed=far)
    assert torch.equal(far, want[0])
    far.copy_(x)
    a = lce.add_rmsnorm_backward(dy, ds, far, r, gamma, want[2], grad_hidden=far)
    b = lce.add_rmsnorm_backward(dy, ds, x, r, gamma, want[2])
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_refusals(lce):
    x, r, gamma, dy, ds = _inputs(4, 64, "bf16")
    rstd = torch.ones(4, device="cuda")
    bad = [
        lambda: lce.add_rmsnorm_forward(x, r[:, :32], gamma), lambda: lce.add_rmsnorm_forward(x, r.float(), gamma),
        lambda: lce.add_rmsnorm_forward(x, r, gamma[:32]), lambda: lce.add_rmsnorm_forward(x, r, gamma.float()),
        lambda: lce.add_rmsnorm_forward(x.double(), r.double(), gamma.double()), lambda: lce.add_rmsnorm_forward(x.t(), r.t(), x[0, :4]),
        lambda: lce.add_rmsnorm_forward(x, r, gamma, normed=x.float()), lambda: lce.add_rmsnorm_forward(x, None, gamma, added=r),
        lambda: lce.add_rmsnorm_forward(torch._neg_view(x), r, gamma), lambda: lce.add_rmsnorm_forward(x, torch._neg_view(r), gamma),
        lambda: lce.add_rmsnorm_quant(x, r, gamma, quantised=x), lambda: lce.add_rmsnorm_backward(dy[:2], ds, x, r, gamma, rstd),
        lambda: lce.add_rmsnorm_backward(dy, ds, x, r, gamma, rstd[:2]), lambda: lce.add_rmsnorm_backward(dy, ds.cpu(), x, r, gamma, rstd),
        lambda: lce.add_rmsnorm_backward(torch._neg_view(dy), ds, x, r, gamma, rstd), lambda: lce.add_rmsnorm(x, None, gamma),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            print("accepted:", k)
    for call, status in [(lambda: lce.add_rmsnorm_forward(x, r, gamma, -1.0), 1), (lambda: lce.add_rmsnorm_forward(x, r, gamma, normed=x, added=x), 1),
                         (lambda: lce.add_rmsnorm_forward(x[:2], r[:2], gamma, normed=x[1:3]), 1),
                         (lambda: lce.add_rmsnorm_backward(dy, ds, x, r, gamma, rstd, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), 3)]:
        with pytest.raises(lce.LCEError) as e:
            call()
        assert e.value.status == status
    for space in (torch.empty(1 << 22, dtype=torch.uint8), torch.empty(1 << 22, dtype=torch.float32, device="cuda")):
        with pytest.raises(ValueError):
            lce.add_rmsnorm_backward(dy, ds, x, r, gamma, rstd, workspace=space)
    wide = torch.zeros(1, 32776, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(lce.LCEError) as e:
        lce.rmsnorm(wide, wide[0])
    assert e.value.status == 2


def test_lazily_negated_rstd_is_refused(lce):
    """Its bytes have the other sign: the gradients would too."""
    x, r, gamma, dy, ds = _inputs(4, 64, "fp32")
    _, _, rstd = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
    lazy = torch._neg_view(-rstd)
    assert torch.equal(lazy, rstd)
    with pytest.raises(ValueError):
        lce.add_rmsnorm_backward(dy, ds, x, r, gamma, lazy)
    _check_backward(*lce.add_rmsnorm_backward(dy, ds, x, r, gamma, lazy.resolve_neg()), dy, ds, x, r, gamma, rstd)


def test_streams_and_graphs(lce):
    """On a side stream; captured and replayed with eager work between, on inputs changed in place; two graphs
    with a workspace each, replayed in turn."""
    x, r, gamma, dy, ds = _inputs(300, 1000, "bf16", seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def everything(ws):
        normed, added, rstd = lce.add_rmsnorm_forward(x, r, gamma, EPS, return_rstd=True)
        q, scales, _ = lce.add_rmsnorm_quant(x, r, gamma, EPS, 64)
        dx, dg = lce.add_rmsnorm_backward(dy, ds, x, r, gamma, rstd, workspace=ws)
        return normed, added, rstd, q.view(torch.uint8), scales, dx, dg

    need = lce.add_rmsnorm_workspace_size(300, 1000)
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2)]
    want = [t.clone() for t in everything(spaces[0])]
    torch.cuda.synchronize()
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
        x.mul_(0.75)
        want = [t.clone() for t in everything(spaces[0])]
        torch.cuda.synchronize()


def test_autograd_in_a_graph(lce):
    """The forward and the gradients captured together, replayed on inputs changed in place."""
    x, r, gamma, dy, ds = _inputs(100, 520, "bf16", seed=12)
    leaves = [t.requires_grad_() for t in (x, r, gamma)]

    def step():
        return torch.autograd.grad(lce.add_rmsnorm(*leaves, EPS), leaves, (dy, ds))

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
        with torch.no_grad():
            x.mul_(1.25)
        want = [t.clone() for t in step()]
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want)), k

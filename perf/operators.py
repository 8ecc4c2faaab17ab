"""The operators around the output-layer step that are timed: their inputs, plain forms and float64 results.

A case is one call (`kind`) in `dtype`:

  norm    lce.add_rmsnorm_forward: the residual's addition and the RMSNorm of the sum (evaluation, serving)
  train   lce.add_rmsnorm(...) and its backward, both outputs with an upstream gradient
  quant   lce.add_rmsnorm_quant: the same with the normalised rows in 8 bits and a scale per row or group
  gnorm   lce.grad_norm: the 2-norm over all gradients of a model
  clip    lce.clip_grad_norm: the norm and the gradients scaled to `limit` times it, in new memory
  within  lce.clip_grad_norm_: the same in place, the gradients within the limit as at most steps

The rows are [N, H]. The gradients are those of a V x H output layer with its norm's gain and of `layers`
decoder layers of width H, views of one flat buffer per type (as gradient buckets are).
"""
import math

import torch

own = False

EPS = 1e-5
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
FP8 = torch.float8_e4m3fn
FP8_MAX = 448.0
TINY = 2.0 ** -126


def _rows(name, kind, N, H, dtype="bf16", residual=True, group=0):
    c = {"name": name, "kind": kind, "N": N, "H": H, "dtype": dtype, "residual": residual}
    return c | {"group": group} if kind == "quant" else c


def _grads(name, kind, V, H, layers, dtype, limit=0.25):
    return {"name": name, "kind": kind, "V": V, "H": H, "layers": layers, "dtype": dtype, "limit": limit}


def listed():
    return [
        # One token in front of a Llama-3-8B head: the smallest call of a serving program.
        _rows("norm_token", "norm", 1, 4096),
        # A prompt of 4 x 1024 tokens at Mistral-Large's width.
        _rows("norm_prompt", "norm", 4096, 12288),
        # Norms of queries by head, without a residual: 8 x 1024 tokens of 32 heads.
        _rows("norm_heads", "norm", 262144, 128, residual=False),
        # The smallest training workload of the repository, in float32.
        _rows("train_tiny", "train", 256, 256, "fp32"),
        # Ragged sequences, not padded, at the width of GPT-2 small, in float16.
        _rows("train_ragged", "train", 3973, 768, "fp16"),
        # The headline workload's rows: 8 x 1024 tokens, Llama-3-8B.
        _rows("train_llama", "train", 8192, 4096),
        # A batch of single tokens, a scale per row.
        _rows("quant_tokens", "quant", 24, 4096),
        # A prompt of 8 x 1024 tokens, a scale for each 128 values.
        _rows("quant_prompt", "quant", 8192, 4096, group=128),
        # The output layer of the smallest training workload and its norm's gain.
        _grads("clip_tiny", "clip", 4096, 256, 0, "fp32"),
        # A model of GPT-2 small's sizes: 110 tensors, an odd vocabulary, gains in float32, matrices in bfloat16.
        _grads("clip_model", "clip", 50257, 768, 12, "mixed"),
        # The Llama-3-8B output layer and gain in place, within the limit.
        _grads("clip_within", "within", 128256, 4096, 0, "bf16", limit=4.0),
        # The norm alone, Qwen2.5-7B's output layer and one decoder layer: the largest.
        _grads("gnorm_qwen", "gnorm", 152064, 3584, 1, "bf16"),
    ]


def _shapes(case):
    """(shape, type) of each gradient."""
    V, H, mixed = case["V"], case["H"], case["dtype"] == "mixed"
    matrix = torch.bfloat16 if mixed else DTYPES[case["dtype"]]
    gain = torch.float32 if mixed else matrix
    kv, wide = max(1, H // 4), 7 * H // 2
    layer = [((H, H), matrix), ((kv, H), matrix), ((kv, H), matrix), ((H, H), matrix), ((wide, H), matrix),
             ((wide, H), matrix), ((H, wide), matrix), ((H,), gain), ((H,), gain)]
    return layer * case["layers"] + [((H,), gain), ((V, H), matrix)]


def _bytes(case):
    if "V" in case:
        n = sum(math.prod(s) * t.itemsize for s, t in _shapes(case))
        return n + 4 if case["kind"] == "gnorm" else 2 * n + 4
    N, H, size = case["N"], case["H"], DTYPES[case["dtype"]].itemsize
    rows = N * H * size
    reads = rows * (2 if case["residual"] else 1) + H * size
    added = rows if case["residual"] else 0
    if case["kind"] == "norm":
        return reads + rows + added
    if case["kind"] == "quant":
        groups = -(-H // case["group"]) if case["group"] else 1
        return reads + N * H + 4 * N * groups + added
    # Upstream gradients of the outputs in; outputs, the rows' gradient (one for both addends) and the gain's out.
    return reads + rows + added + 2 * rows + added + H * size


def draw(rng):
    top = max(_bytes(c) for c in listed())

    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choices(("norm", "train", "quant", "clip", "within", "gnorm"), (20, 30, 20, 14, 6, 10))[0]
        if kind in ("clip", "within", "gnorm"):
            c = _grads("", kind, log_uniform(256, 152064), log_uniform(64, 4096), rng.choice((0, 0, 1, 2, 8, 24)),
                       rng.choice(("bf16", "bf16", "fp16", "fp32", "mixed")), 4.0 if kind == "within" else rng.choice((0.05, 0.5, 1.5)))
        else:
            # Widths of models are multiples of 8 as a rule; every eighth is any number.
            H = log_uniform(64, 16384) if rng.random() < 0.125 else 8 * log_uniform(8, 2048)
            c = _rows("", kind, log_uniform(64 if kind == "train" else 1, 16384), H, rng.choices(("bf16", "fp16", "fp32"), (60, 20, 20))[0],
                      rng.random() < 0.75, rng.choice((0, 0, 32, 64, 128)))
        del c["name"]
        if _bytes(c) <= top:
            return c


def _inputs(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    if "V" in case:
        shapes = _shapes(case)
        flats = {t: torch.empty(sum(math.prod(s) for s, u in shapes if u == t), dtype=t, device=dev)
                 for t in dict.fromkeys(t for _, t in shapes)}
        at, views = dict.fromkeys(flats, 0), []
        for shape, t in shapes:
            n = math.prod(shape)
            views.append(flats[t][at[t]:at[t] + n].view(shape))
            at[t] += n
            size = math.exp(math.log(1e-5) + math.log(1e3) * float(torch.rand((), generator=g, device=dev)))
            for v in views[-1].reshape(-1).split(1 << 26):
                v.copy_(size * torch.randn(v.numel(), generator=g, device=dev))
        return list(flats.values()), views
    N, H, dtype = case["N"], case["H"], DTYPES[case["dtype"]]

    def rows(scale=1.0):
        return (scale * torch.randn((N, H), generator=g, device=dev)).to(dtype)

    # The residual stream's size varies by token.
    size = torch.exp(math.log(0.25) + math.log(64.0) * torch.rand((N, 1), generator=g, device=dev))
    hidden = rows(size)
    residual = rows(size) if case["residual"] else None
    gamma = (1.0 + 0.1 * torch.randn(H, generator=g, device=dev)).to(dtype)
    return hidden, residual, gamma, rows() if case["kind"] == "train" else None, rows() if case["kind"] == "train" else None


def _sum_squares(flats):
    return sum(f.double().square().sum() for f in flats)


def prepare(case, seed):
    s = dict(case)
    if "V" in case:
        s["flats"], s["grads"] = _inputs(case, seed)
        s["max_norm"] = case["limit"] * math.sqrt(float(_sum_squares(s["flats"])))
        if case["kind"] == "clip":
            s["out_flats"] = [torch.empty_like(f) for f in s["flats"]]
            s["out"] = []
            at = dict.fromkeys((f.dtype for f in s["flats"]), 0)
            for v in s["grads"]:
                flat = next(f for f in s["out_flats"] if f.dtype == v.dtype)
                s["out"].append(flat[at[v.dtype]:at[v.dtype] + v.numel()].view(v.shape))
                at[v.dtype] += v.numel()
        return s
    s["hidden"], s["residual"], s["gamma"], s["grad_normed"], s["grad_added"] = _inputs(case, seed)
    if case["kind"] == "train":
        s["leaves"] = [t.requires_grad_() for t in (s["hidden"], s["residual"], s["gamma"]) if t is not None]
    return s


def _plain_norm(s):
    """(normalised rows, sum) in float32."""
    added = s["hidden"].float()
    if s["residual"] is not None:
        added = added + s["residual"].float()
    return added * torch.rsqrt(added.square().mean(-1, keepdim=True) + EPS) * s["gamma"].float(), added


def _groups(y, group):
    """The rows in groups, the last one filled with zeros: [N, groups, group]."""
    N, H = y.shape
    group = group or H
    y = torch.nn.functional.pad(y, (0, -H % group))
    return y.view(N, -1, group)


def _plain(s):
    kind = s["kind"]
    if kind in ("clip", "within", "gnorm"):
        norm = sum(f.float().square().sum(dtype=torch.float64) for f in s["flats"]).sqrt().float()
        if kind == "gnorm":
            return norm
        factor = torch.clamp(s["max_norm"] / (norm + 1e-6), max=1.0)
        out = s["flats"] if kind == "within" else s["out_flats"]
        return norm, [o.copy_(f.float() * factor) for o, f in zip(out, s["flats"])]
    y, added = _plain_norm(s)
    dtype = s["hidden"].dtype
    if kind == "quant":
        z = _groups(y, s["group"])
        scales = (z.abs().amax(-1, keepdim=True) / FP8_MAX).clamp(min=TINY)
        q = (z / scales).view(len(y), -1)[:, :y.shape[1]].to(FP8)
        return (q, scales[..., 0]) + ((added.to(dtype),) if s["residual"] is not None else ())
    outs = (y.to(dtype),) + ((added.to(dtype),) if s["residual"] is not None else ())
    if kind == "norm":
        return outs
    upstream = (s["grad_normed"], s["grad_added"])[:len(outs)]
    return tuple(o.detach() for o in outs) + torch.autograd.grad(outs, s["leaves"], upstream)


def run(s):
    if not own:
        return _plain(s)
    import paper_2603_16428_amd as lce
    kind = s["kind"]
    if kind == "gnorm":
        return lce.grad_norm(s["grads"])
    if kind == "clip":
        norm, _ = lce.clip_grad_norm(s["grads"], s["max_norm"], out=s["out"])
        return norm, s["out_flats"]
    if kind == "within":
        return lce.clip_grad_norm_(s["grads"], s["max_norm"]), s["flats"]
    hidden, residual, gamma = s["hidden"], s["residual"], s["gamma"]
    if kind == "quant":
        q, scales, added = lce.add_rmsnorm_quant(hidden, residual, gamma, EPS, group_size=s["group"])
        return (q, scales) + ((added,) if residual is not None else ())
    if kind == "norm":
        normed, added = lce.add_rmsnorm_forward(hidden, residual, gamma, EPS)
        return (normed,) + ((added,) if residual is not None else ())
    outs = lce.add_rmsnorm(hidden, residual, gamma, EPS) if residual is not None else (lce.rmsnorm(hidden, gamma, EPS),)
    upstream = (s["grad_normed"], s["grad_added"])[:len(outs)]
    return tuple(o.detach() for o in outs) + torch.autograd.grad(outs, s["leaves"], upstream)


def work(case):
    if "V" in case:
        n = sum(math.prod(s) for s, _ in _shapes(case))
        return {"bytes": _bytes(case), "flops": n * (2 if case["kind"] == "gnorm" else 3)}
    return {"bytes": _bytes(case), "flops": case["N"] * case["H"] * (16 if case["kind"] == "train" else 6)}


def exact(case, seed):
    if "V" in case:
        flats, _ = _inputs(case, seed)
        norm = math.sqrt(float(_sum_squares(flats)))
        total = torch.tensor(norm, dtype=torch.float64)
        if case["kind"] == "gnorm":
            return total
        factor = min(1.0, case["limit"] * norm / (norm + 1e-6))
        return total, [f.double() * factor for f in flats]
    hidden, residual, gamma, dy, ds = _inputs(case, seed)
    N, H = hidden.shape
    x, w = hidden.double(), gamma.double()
    if residual is not None:
        x = x + residual.double()
    r = 1.0 / torch.sqrt((x * x).sum(1, keepdim=True) / H + EPS)
    y = x * r * w
    added = (x,) if residual is not None else ()
    if case["kind"] == "norm":
        return (y, *added)
    if case["kind"] == "quant":
        group = case["group"] or H
        scales = torch.stack([y[:, k:k + group].abs().max(1).values for k in range(0, H, group)], 1) / FP8_MAX
        scales = scales.clamp(min=TINY)
        q = (y / scales.repeat_interleave(group, 1)[:, :H]).to(FP8).double()
        return (q, scales, *added)
    g = dy.double() * w
    dx = r * g - r ** 3 * x * (g * x).sum(1, keepdim=True) / H
    if residual is not None:
        dx = dx + ds.double()
    return (y, *added, dx, *((dx,) if residual is not None else ()), (dy.double() * x * r).sum(0))

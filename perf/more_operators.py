"""The operators on a vocabulary's matrix and logits that are timed: their inputs, plain forms and float64 results.

A case is one call (`kind`) in `dtype`:

  embed   lce.embedding_forward: the rows of a V x H matrix that N tokens name, times a factor
  train   lce.embedding(...) and its gradient, a dense V x H tensor
  tied    lce.embedding_backward into a given gradient (that of an output layer with the same weight), which it adds to
  pack    lce.mxfp4_quantize and lce.mxfp4_dequantize: rows in 4 bits with a scale for each 32 values, and their values
  logits  lce.mxfp4_linear: rows, quantised within the call, times a V x H weight held in 4 bits
  sample  lce.sample: a token for each row of logits, from a given random number

Rows in 4 bits: each group of 32 values of a row has a power of two, its byte the exponent + 127 (255: the group holds a NaN or an
infinity), and codes of 4 bits (sign, two bits of exponent, one of mantissa: 0, 0.5, 1, 1.5, 2, 3, 4, 6), two in a byte, the first
in the low half. The exponent is that of the group's largest magnitude less 2; larger values than 6 become 6.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
GROUP = 32
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _embed(name, kind, N, H, V, dtype="bf16", scale=1.0, padding=False):
    return {"name": name, "kind": kind, "N": N, "H": H, "V": V, "dtype": dtype, "scale": scale, "padding": padding}


def _rows(name, kind, N, H, V=0, dtype="bf16"):
    return {"name": name, "kind": kind, "N": N, "H": H, "dtype": dtype} | ({"V": V} if kind == "logits" else {})


def _sample(name, N, V, dtype, temperature, top_k=0, top_p=1.0, min_p=0.0, by_row=False, flat=False):
    return {"name": name, "kind": "sample", "N": N, "V": V, "dtype": dtype, "temperature": temperature, "top_k": top_k, "top_p": top_p,
            "min_p": min_p, "by_row": by_row, "flat": flat}


def listed():
    return [
        # One token in front of a Llama-3-8B: the smallest call of a serving program.
        _embed("embed_token", "embed", 1, 4096, 128256),
        # A prompt of 8 x 1024 tokens, with the rows scaled by sqrt(H).
        _embed("embed_prompt", "embed", 8192, 4096, 128256, scale=64.0),
        # Ragged sequences at the width of GPT-2 small, in float16, with a padding token and an odd vocabulary.
        _embed("train_ragged", "train", 3973, 768, 50257, "fp16", padding=True),
        # The headline workload's input layer: 8 x 1024 tokens, Llama-3-8B.
        _embed("train_llama", "train", 8192, 4096, 128256),
        # The same with the output layer's weight: added to the gradient that the output layer left.
        _embed("tied_llama", "tied", 8192, 4096, 128256),
        # A prompt's rows of 8 x 1024 tokens.
        _rows("pack_prompt", "pack", 8192, 4096),
        # One token through a Llama-3-8B output layer.
        _rows("logits_token", "logits", 1, 4096, 128256),
        # A batch of single tokens, Mistral-Large's output layer.
        _rows("logits_batch", "logits", 48, 12288, 32768),
        # Scoring a prompt of two sequences, Qwen2.5-7B's output layer: the largest.
        _rows("logits_prompt", "logits", 2048, 3584, 152064),
        # One token's answer with the usual settings.
        _sample("sample_token", 1, 128256, "bf16", 0.8, top_k=50, top_p=0.95),
        # A batch of single tokens whose requests have settings of their own, in float32.
        _sample("sample_batch", 256, 152064, "fp32", 1.0, top_k=200, top_p=0.9, min_p=0.02, by_row=True),
        # A batch drawn from the whole distribution, an odd vocabulary.
        _sample("sample_whole", 64, 50257, "fp16", 1.0),
    ]


def work(case):
    kind, size = case["kind"], DTYPES[case["dtype"]].itemsize
    if kind == "sample":
        # Tokens and log-probabilities out. An exponential and the running sums for each logit.
        return {"bytes": case["N"] * (case["V"] * size + 4 + 8 + 4), "flops": 4 * case["N"] * case["V"]}
    N, H = case["N"], case["H"]
    packed = H // 2 + H // GROUP
    if kind == "pack":
        return {"bytes": N * (2 * H * size + packed), "flops": 4 * N * H}
    V = case["V"]
    if kind == "logits":
        return {"bytes": N * H * size + V * packed + N * V * size, "flops": 2 * N * H * V}
    rows = _different(N, V)
    read = 8 * N + rows * H * size
    if kind == "embed":
        return {"bytes": read + N * H * size, "flops": N * H}
    if kind == "train":
        return {"bytes": read + N * H * size + N * H * size + V * H * size, "flops": 2 * N * H}
    return {"bytes": 8 * N + N * H * size + 2 * rows * H * size, "flops": 2 * N * H}


def _different(N, V):
    """How many of the V tokens N draws name, which are even over the logarithm of their number."""
    rows, k = 0.0, 0
    while k < V:
        step = min(max(1, k // 500), V - k)
        rows += step * (1.0 - (1.0 - math.log1p(step / (k + 1)) / step / math.log1p(V)) ** N)
        k += step
    return round(rows)


def draw(rng):
    largest = [work(c) for c in listed()]
    most = {k: max(w[k] for w in largest) for k in ("bytes", "flops")}

    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        kind = rng.choices(("embed", "train", "tied", "pack", "logits", "sample"), (12, 14, 14, 10, 25, 25))[0]
        dtype = rng.choices(("bf16", "fp16", "fp32"), (60, 20, 20))[0]
        V = log_uniform(256, 152064)
        if kind == "sample":
            c = _sample("", log_uniform(1, 512), V, dtype, rng.choice((0.0, 0.6, 0.8, 1.0, 1.0, 1.3)), rng.choice((0, 0, 1, 20, 50, 400, 3000)),
                        rng.choice((1.0, 1.0, 0.5, 0.8, 0.9, 0.95, 0.99)), rng.choice((0.0, 0.0, 0.0, 0.05, 0.1)), rng.random() < 0.5, rng.random() < 0.15)
        elif kind in ("pack", "logits"):
            c = _rows("", kind, log_uniform(1, 16384 if kind == "pack" else 4096), 32 * log_uniform(2, 384), V, dtype)
        else:
            # Widths of models are multiples of 8 as a rule; every eighth is any number.
            H = log_uniform(64, 8192) if rng.random() < 0.125 else 8 * log_uniform(8, 1024)
            c = _embed("", kind, log_uniform(1 if kind == "embed" else 32, 32768), H, V, dtype, rng.choice((1.0, 1.0, round(math.sqrt(H), 3))), rng.random() < 0.3)
        del c["name"]
        w = work(c)
        if all(w[k] <= most[k] for k in most):
            return c


# ---- inputs ----

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(shape, g, dtype, scale=1.0):
    out = torch.empty(shape, dtype=dtype, device="cuda")
    for rows in out.split(max(1, (1 << 26) // shape[-1])):
        rows.copy_(scale * torch.randn(rows.shape, generator=g, device="cuda"))
    return out


def _inputs(case, seed):
    g, kind, N, dtype = _generator(seed), case["kind"], case["N"], DTYPES[case["dtype"]]
    if kind == "sample":
        V = case["V"]
        # A few frequent tokens and a long tail, as sharp as the row's context makes it.
        rank = torch.randperm(V, generator=g, device="cuda").float()
        lo, hi = (0.7, 1.2) if case["flat"] else (1.3, 3.0)
        sharp = lo + (hi - lo) * torch.rand((N, 1), generator=g, device="cuda")
        logits = torch.empty((N, V), dtype=dtype, device="cuda")
        for z, s in zip(logits.split(64), sharp.split(64)):
            z.copy_(12.0 + s * (1.2 * torch.randn(z.shape, generator=g, device="cuda") - torch.log1p(rank)))
        u = torch.rand(N, generator=g, device="cuda")
        settings = {}
        for name in ("temperature", "top_k", "top_p", "min_p"):
            settings[name] = case[name]
            if case["by_row"]:
                # Half of the requests leave a setting off.
                off = {"temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0}[name]
                t = torch.full((N,), case[name], dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda")
                settings[name] = torch.where(torch.rand(N, generator=g, device="cuda") < 0.5, t, torch.full_like(t, off))
        return logits, u, settings
    H = case["H"]
    if kind in ("pack", "logits"):
        # Rows behind a norm; a few of their values are large, as a model's are.
        hidden = torch.randn((N, H), generator=g, device="cuda")
        hidden = (hidden * torch.where(torch.rand((N, H), generator=g, device="cuda") < 0.001, 20.0, 1.0)).to(dtype)
        if kind == "pack":
            return hidden
        codes = torch.empty((case["V"], H // 2), dtype=torch.uint8, device="cuda")
        scales = torch.empty((case["V"], H // GROUP), dtype=torch.uint8, device="cuda")
        for c, s in zip(codes.split(8192), scales.split(8192)):
            packed, exponents = _plain_pack(0.02 * torch.randn((len(c), H), generator=g, device="cuda"))
            c.copy_(packed)
            s.copy_(exponents)
        return hidden, codes, scales
    V = case["V"]
    tokens = torch.exp(torch.rand(N, generator=g, device="cuda", dtype=torch.float64) * math.log1p(V)).floor().long() - 1
    tokens = tokens.clamp(0, V - 1)
    if case["padding"]:
        tokens[torch.rand(N, generator=g, device="cuda") < 0.1] = 0
    matrix = _randn((V, H), g, dtype, 0.02) if kind != "tied" else _randn((V, H), g, dtype, 1e-3)
    grad = _randn((N, H), g, dtype, 1e-2) if kind != "embed" else None
    return tokens, matrix, grad


def prepare(case, seed):
    s = dict(case)
    kind = case["kind"]
    if kind == "sample":
        s["logits"], s["u"], s["settings"] = _inputs(case, seed)
    elif kind == "pack":
        s["hidden"] = _inputs(case, seed)
    elif kind == "logits":
        s["hidden"], s["codes"], s["scales"] = _inputs(case, seed)
    else:
        s["tokens"], s["matrix"], s["grad"] = _inputs(case, seed)
        s["padding_idx"] = 0 if case["padding"] else None
        if kind == "train":
            s["matrix"].requires_grad_()
    return s


# ---- plain forms ----

def _power(e):
    """2^e in float64, from its bits (exact, as torch's exp2 need not be)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _plain_pack(x):
    """(codes, exponents' bytes) of the rows x in float32."""
    groups = x.float().view(x.shape[0], -1, GROUP)
    top = groups.abs().amax(-1, keepdim=True)
    e = (torch.frexp(top).exponent - 3).clamp(min=-127)  # frexp's mantissa is below 1: floor(log2) is one less
    e = torch.where(top == 0, torch.full_like(e, -127), e)
    y = groups.double() / _power(e)
    a = y.abs()
    # Steps of 0.5 below 2, of 1 below 4, of 2 above, ties to the even code.
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    a = (torch.round(a / step) * step).clamp(max=6.0)
    code = sum((a > v).to(torch.uint8) for v in E2M1[:-1]) | (torch.signbit(y).to(torch.uint8) << 3)
    code = code.view(x.shape[0], -1)
    bad = ~torch.isfinite(top)
    byte = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), byte.view(x.shape[0], -1)


def _plain_values(codes, exponents):
    """The values in float32."""
    code = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1).int()
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    e = exponents.int().repeat_interleave(GROUP, 1)
    value = table[code] * _power(e - 127).float()
    return torch.where(e == 255, torch.full_like(value, math.nan), value)


def _row(v, N):
    """A setting as a float64 column."""
    return (v.double() if isinstance(v, torch.Tensor) else torch.full((N,), v, dtype=torch.float32, device="cuda").double()).view(N, 1)


def _plain_sample(logits, u, settings):
    N, V = logits.shape
    z = logits.double() + 0.0
    T, k, p, least = (_row(settings[n], N) for n in ("temperature", "top_k", "top_p", "min_p"))
    k = torch.where(k <= 0, V, k)
    top = z.amax(1, keepdim=True)
    w = torch.where(z == top, 1.0, torch.exp((z - top) / torch.where(T > 0, T, 1.0)))
    _, order = torch.sort(z, dim=1, descending=True, stable=True)
    falling = w.gather(1, order)
    rank = torch.arange(V, device="cuda").view(1, V)
    falling = torch.where(rank < k, falling, 0.0)
    running = falling.cumsum(1)
    before = torch.nn.functional.pad(running, (1, 0))[:, :-1]
    keep = (rank < k) & ((before < p * running[:, -1:]) | (p >= 1.0) | (rank == 0)) & (falling >= least)
    keep = torch.where(T > 0, keep, rank == 0)
    kept = torch.where(torch.zeros_like(keep).scatter(1, order, keep), w, 0.0)
    running = kept.cumsum(1)
    total = running[:, -1:]
    token = (running <= u.double().view(N, 1) * total).sum(1, keepdim=True)
    return token.view(N), (kept.gather(1, token) / total).log().float().view(N)


def _plain(s):
    kind = s["kind"]
    if kind == "sample":
        return _plain_sample(s["logits"], s["u"], s["settings"])
    if kind == "pack":
        codes, exponents = _plain_pack(s["hidden"])
        return _plain_values(codes, exponents).to(s["hidden"].dtype), exponents
    if kind == "logits":
        rows = _plain_values(*_plain_pack(s["hidden"]))
        return (rows @ _plain_values(s["codes"], s["scales"]).T).to(s["hidden"].dtype)
    tokens, matrix, scale = s["tokens"], s["matrix"].detach(), s["scale"]
    out = (matrix[tokens].float() * scale).to(matrix.dtype)
    if kind == "embed":
        return out
    named = tokens != s["padding_idx"] if s["padding_idx"] is not None else torch.ones_like(tokens, dtype=torch.bool)
    rows, at = torch.unique(tokens, return_inverse=True)
    sums = torch.zeros((len(rows), matrix.shape[1]), device="cuda").index_add_(0, at, torch.where(named[:, None], s["grad"].float() * scale, 0.0))
    if kind == "tied":
        matrix[rows] = (matrix[rows].float() + sums).to(matrix.dtype)
        return matrix
    grad = torch.zeros_like(matrix)
    grad[rows] = sums.to(matrix.dtype)
    return out, grad


def run(s):
    if not own:
        return _plain(s)
    import paper_2603_16428_amd as lce
    kind = s["kind"]
    if kind == "sample":
        return lce.sample(s["logits"], s["u"], **s["settings"], return_logprobs=True)
    if kind == "pack":
        codes, scales = lce.mxfp4_quantize(s["hidden"])
        return lce.mxfp4_dequantize(codes, scales, s["hidden"].dtype), scales
    if kind == "logits":
        return lce.mxfp4_linear(s["hidden"], s["codes"], s["scales"])
    if kind == "embed":
        return lce.embedding_forward(s["tokens"], s["matrix"], s["scale"])
    if kind == "tied":
        return lce.embedding_backward(s["grad"], s["tokens"], s["V"], s["scale"], s["padding_idx"], grad_weight=s["matrix"], accumulate=True)
    out = lce.embedding(s["tokens"], s["matrix"], s["scale"], s["padding_idx"])
    return (out.detach(), *torch.autograd.grad(out, s["matrix"], s["grad"]))


# ---- the definitions in 64 bits ----

def _exact_values(codes, exponents):
    """The values of packed rows, from the bits: (1 + m / 2) 2^(e - 1), or m / 2 where e is 0."""
    out = torch.empty((codes.shape[0], 2 * codes.shape[1]), dtype=torch.float64, device=codes.device)
    for half in range(2):
        c = ((codes >> (4 * half)) & 15).long()
        m, e = (c & 1).double(), (c >> 1) & 3
        out[:, half::2] = torch.where(e == 0, m / 2, (1 + m / 2) * torch.ldexp(torch.ones_like(m), e - 1)) * torch.where(c >= 8, -1.0, 1.0)
    groups = out.view(len(out), -1, GROUP)
    groups *= torch.tensor([2.0 ** (k - 127) for k in range(256)], dtype=torch.float64, device=codes.device)[exponents.long()][..., None]
    return out


def _exact_rounded(x):
    """(values of the rows x rounded to 4 bits with their groups' scales, the scales' bytes)."""
    groups = x.double().reshape(len(x), -1, GROUP)
    powers = torch.tensor([2.0 ** k for k in range(-125, 129)], dtype=torch.float64, device=x.device)
    # The powers up to the largest magnitude say how large it is: its exponent, less 2, is the scale's, from -127 on.
    e = (torch.bucketize(groups.abs().max(-1, keepdim=True).values, powers, right=True) - 128).clamp(min=-127)
    scale = torch.tensor([2.0 ** k for k in range(-127, 129)], dtype=torch.float64, device=x.device)[e + 127]
    unit = groups / scale
    # Borders between neighbours; a value on one goes to the even code.
    borders = torch.tensor([(a + b) / 2 for a, b in zip(E2M1, E2M1[1:])], dtype=torch.float64, device=x.device)
    a = unit.abs()
    up, down = torch.bucketize(a, borders, right=True), torch.bucketize(a, borders)
    code = torch.where(up == down, up, torch.where(up % 2 == 0, up, down))
    value = torch.tensor(E2M1, dtype=torch.float64, device=x.device)[code] * torch.sign(unit) * scale
    return value.reshape(x.shape), (e + 127).to(torch.uint8).reshape(len(x), -1)


def _exact_sample(logits, u, settings):
    z, u = logits.double().cpu().numpy(), u.double().cpu().numpy()
    N, V = z.shape
    T, k, p, least = (_row(settings[n], N).cpu().numpy()[:, 0] for n in ("temperature", "top_k", "top_p", "min_p"))
    tokens, logs = np.empty(N, dtype=np.int64), np.empty(N)
    for i in range(N):
        if not T[i] > 0:
            tokens[i], logs[i] = int(np.argmax(z[i])), 0.0
            continue
        order = np.argsort(-z[i], kind="stable")
        w = np.exp((z[i][order] - z[i].max()) / T[i])
        n = int(min(k[i], V)) if k[i] > 0 else V
        if p[i] < 1.0:
            n = min(n, max(1, int(np.searchsorted(np.cumsum(w[:n]), p[i] * w[:n].sum()) + 1)))
        n = max(1, min(n, int((w >= least[i]).sum())))
        chosen = np.sort(order[:n])
        w = np.exp((z[i][chosen] - z[i].max()) / T[i])
        running = np.cumsum(w)
        at = min(n - 1, int(np.searchsorted(running, u[i] * running[-1], side="right")))
        tokens[i], logs[i] = chosen[at], math.log(w[at] / running[-1])
    return torch.from_numpy(tokens), torch.from_numpy(logs)


def exact(case, seed):
    kind = case["kind"]
    if kind == "sample":
        return _exact_sample(*_inputs(case, seed))
    if kind == "pack":
        return _exact_rounded(_inputs(case, seed))
    if kind == "logits":
        hidden, codes, scales = _inputs(case, seed)
        rows, _ = _exact_rounded(hidden)
        out = torch.empty((len(rows), len(codes)), dtype=torch.float64, device="cuda")
        at = 0
        for c, s in zip(codes.split(16384), scales.split(16384)):
            out[:, at:at + len(c)] = rows @ _exact_values(c, s).T
            at += len(c)
        return out
    tokens, matrix, grad = _inputs(case, seed)
    out = matrix.index_select(0, tokens).double() * case["scale"]
    if kind == "embed":
        return out
    total = matrix.double() if kind == "tied" else torch.zeros(matrix.shape, dtype=torch.float64, device="cuda")
    if case["padding"]:
        grad = grad[tokens != 0]
        tokens = tokens[tokens != 0]
    total.index_put_((tokens,), case["scale"] * grad.double(), accumulate=True)
    return total if kind == "tied" else (out, total)

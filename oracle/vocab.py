"""Float64 definitions of the operators on the vocabulary's matrix and logits (torch and numpy on the CPU).

Every function takes tensors of any type (converted exactly) and gives float64 or whole numbers.
"""
from __future__ import annotations

import math

import numpy as np
import torch

GROUP = 32
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _f64(t):
    return t.detach().cpu().to(torch.float64)


def embedding(tokens, weight, scale=1.0):
    tokens, weight = tokens.cpu().long(), _f64(weight)
    V = len(weight)
    known = (tokens >= 0) & (tokens < V)
    out = weight[tokens.clamp(0, V - 1)] * scale
    return torch.where(known[..., None], out, torch.full_like(out, math.nan))


def embedding_backward(grad, tokens, V, scale=1.0, padding_idx=None):
    """(gradient, sums of the terms' magnitudes), both [V, H]."""
    grad, tokens = _f64(grad), tokens.cpu().long().reshape(-1)
    grad = grad.reshape(len(tokens), grad.shape[-1])
    counts = (tokens >= 0) & (tokens < V)
    if padding_idx is not None:
        counts &= tokens != padding_idx
    total = torch.zeros((V, grad.shape[-1]), dtype=torch.float64)
    size = torch.zeros_like(total)
    total.index_add_(0, tokens[counts], grad[counts] * scale)
    size.index_add_(0, tokens[counts], (grad[counts] * scale).abs())
    return total, size


def mxfp4_quantize(x):
    """(codes [..., H] not packed, scale bytes [..., H / 32])."""
    x = _f64(x).numpy()
    groups = x.reshape(x.shape[:-1] + (-1, GROUP))
    codes = np.zeros(groups.shape, dtype=np.uint8)
    scales = np.zeros(groups.shape[:-1], dtype=np.uint8)
    for at in np.ndindex(scales.shape):
        g = groups[at]
        top = np.abs(g).max()
        if not np.isfinite(g).all():
            scales[at] = 255
            continue
        e = max(-127, math.frexp(top)[1] - 3) if top > 0 else -127
        scales[at] = e + 127
        for j, v in enumerate(g):
            a = abs(v) / 2.0 ** e
            # The nearest value, the even code of two equally near ones (6 for all that is larger).
            best = min(range(8), key=lambda c: (abs(E2M1[c] - min(a, 6.0)), c % 2))
            codes[at][j] = best | (8 if math.copysign(1.0, v) < 0 else 0)
    return torch.from_numpy(codes.reshape(x.shape)), torch.from_numpy(scales)


def mxfp4_pack(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def mxfp4_values(codes, scales):
    """The values of packed codes."""
    codes, scales = codes.cpu(), scales.cpu()
    c = torch.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (-1,)).long()
    value = torch.tensor(E2M1, dtype=torch.float64)[c & 7] * torch.where(c >= 8, -1.0, 1.0)
    power = torch.tensor([2.0 ** (b - 127) for b in range(255)] + [math.nan], dtype=torch.float64)
    return value * power[scales.long()].repeat_interleave(GROUP, -1)


def sample(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(tokens, log-probabilities) of rows [N, V]; settings are numbers or [N]. Sorted, and added up in order."""
    z, u = _f64(logits).numpy(), _f64(uniforms).numpy()
    N, V = z.shape

    def column(v):
        return v.detach().cpu().double().numpy() if isinstance(v, torch.Tensor) else np.full(N, float(np.float32(v)))

    T, K, P, M = map(column, (temperature, top_k, top_p, min_p))
    tokens, logs = np.full(N, -1, dtype=np.int64), np.full(N, np.nan)
    for i in range(N):
        row = z[i] + 0.0
        if np.isnan(row).any() or np.isnan(u[i]) or not row.max() > -np.inf:
            continue
        if not T[i] > 0:
            tokens[i], logs[i] = int(np.argmax(row)), 0.0
            continue
        top = row.max()
        with np.errstate(invalid="ignore", over="ignore"):
            x = np.where(row == top, 0.0, (row - top) / T[i])
        order = np.argsort(-row, kind="stable")
        w = np.exp(x)[order]
        n = int(K[i]) if 0 < K[i] < V else V
        if P[i] < 1.0:
            before, share = 0.0, P[i] * math.fsum(w[:n])
            running = np.concatenate(([0.0], np.cumsum(w[:n])[:-1]))
            n = max(1, int((running < share).sum()))
        n = max(1, min(n, int((w >= min(M[i], 1.0)).sum())))
        chosen = np.sort(order[:n])
        w = np.exp(x)[chosen]
        running = np.cumsum(w)
        at = int((running <= min(max(u[i], 0.0), 1.0) * running[-1]).sum())
        if at >= n:
            at = int(np.flatnonzero(w > 0)[-1])
        tokens[i], logs[i] = chosen[at], x[chosen[at]] - math.log(running[-1])
    return torch.from_numpy(tokens), torch.from_numpy(logs)

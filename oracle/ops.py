"""Float64 definitions of the operators around the output-layer step (torch on the CPU).

rows are [N, H]; every function takes and gives float64 (inputs of other types are converted exactly).
"""
from __future__ import annotations

import torch

FP8_MAX = 448.0
SCALE_MIN = 2.0 ** -126


def _f64(t):
    return None if t is None else t.detach().cpu().to(torch.float64)


def add_rmsnorm(x, residual, gamma, eps):
    """(normed, added, rstd)."""
    x, residual, gamma = _f64(x), _f64(residual), _f64(gamma)
    s = x if residual is None else x + residual
    r = 1.0 / torch.sqrt((s * s).mean(-1) + eps)
    return s * r[..., None] * gamma, s, r


def add_rmsnorm_backward(dy, ds, s, gamma, r):
    """(grad_hidden, grad_gamma) from s and r as the forward left them."""
    dy, ds, s, gamma, r = (_f64(t) for t in (dy, ds, s, gamma, r))
    r = r[..., None]
    g = dy * gamma
    dx = r * g - r ** 3 * s * (g * s).mean(-1, keepdim=True)
    if ds is not None:
        dx = dx + ds
    H = s.shape[-1]
    return dx, (dy * s * r).reshape(-1, H).sum(0)


def group_scales(y, group):
    """[N, groups] scales of the rows y [N, H] (group 0: the whole row)."""
    y = _f64(y)
    H = y.shape[-1]
    group = group or H
    return torch.stack([(y[..., k:k + group].abs().amax(-1) / FP8_MAX).clamp(min=SCALE_MIN)
                        for k in range(0, H, group)], -1)


def grad_norm(grads, norm_type=2.0):
    flat = torch.cat([_f64(g).reshape(-1) for g in grads])
    if norm_type == float("inf"):
        return flat.abs().max() if flat.numel() else torch.zeros((), dtype=torch.float64)
    return flat.square().sum().sqrt()


def clip(grads, max_norm, norm_type=2.0):
    """(norm, clipped gradients)."""
    norm = grad_norm(grads, norm_type)
    factor = 1.0 if max_norm == float("inf") else torch.clamp(max_norm / (norm + 1e-6), max=1.0)
    return norm, [_f64(g) * factor for g in grads]

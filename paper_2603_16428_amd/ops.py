"""Python binding of the operators around the output-layer step (include/lce_ops.h).

In front of the step: the residual's addition with the RMSNorm of the sum, with rows in their own type
or in 8 bits with scales, and its backward. Behind it: the global norm of many gradients, and clipping
by it. Argument marshalling only, as in lce.py: every computation runs in liblce.so's HIP kernels, on
the current stream of the tensors' device, and nothing waits for the GPU.
"""
from __future__ import annotations

import array
import ctypes

import torch

from .lce import DTYPES, LCE_OK, LCEError, _bytes_are_values, _differentiated, load_library

EXPORTED = ("lce_add_rmsnorm_forward", "lce_add_rmsnorm_quant", "lce_add_rmsnorm_workspace_size",
            "lce_add_rmsnorm_backward", "lce_grad_norm_workspace_size", "lce_grad_norm", "lce_clip_grad_norm")
FP8 = torch.float8_e4m3fn
GROUP_SIZES = (0, 32, 64, 128)
NORM_TYPES = {2.0: 0, float("inf"): 1}
_PLAIN = {torch.Tensor}

_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    lib = load_library()
    i64, vp, sz, ci, f32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    rows = [vp, i64, vp, i64, vp, i64, i64, ci, f32]
    for name, args, res in [
            ("lce_add_rmsnorm_forward", rows + [vp, i64, vp, i64, vp, vp], ci),
            ("lce_add_rmsnorm_quant", rows + [ci, vp, i64, vp, vp, i64, vp, vp], ci),
            ("lce_add_rmsnorm_workspace_size", [i64, i64, ci], sz),
            ("lce_add_rmsnorm_backward", [vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, i64, i64, ci, vp, i64, vp, vp, sz, vp], ci),
            ("lce_grad_norm_workspace_size", [i64], sz),
            ("lce_grad_norm", [vp, i64, ci, vp, vp, sz, vp], ci),
            ("lce_clip_grad_norm", [vp, i64, ci, f32, vp, vp, vp, sz, vp], ci)]:
        f = getattr(lib, name)
        f.argtypes, f.restype = args, res
    _lib = lib
    return lib


# The current device and a device's current stream, as numbers. torch's public calls wrap them in objects: 5 us of
# a call whose launch takes 4.
_device_index = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", lambda index: torch.cuda.current_stream(index).cuda_stream)


def _space(workspace, like, nbytes: int):
    """A given workspace (its size is the library's to check), or a new one."""
    if workspace is None:
        return like.new_empty(nbytes, dtype=torch.uint8)
    if workspace.dtype is not torch.uint8 or workspace.device != like.device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous uint8 tensor on the tensors' device")
    return workspace


def _call(name: str, device, *args) -> None:
    """A library call on the current stream of `device`, with that device the current one."""
    f = getattr(_lib or _library(), name)
    index = device.index
    if index == _device_index():
        st = f(*args, _raw_stream(index))
    else:
        with torch.cuda.device(device):
            st = f(*args, _raw_stream(index))
    if st != LCE_OK:
        raise LCEError(st, name)


# ---- the residual's addition and the RMSNorm of the sum --------------------------------------------

def _pitch(t, what: str) -> int:
    """Elements between the rows [N, H] that t's leading dimensions make up, its last one being H."""
    if t.is_contiguous():
        return t.shape[-1]
    if t.is_neg():
        raise ValueError(f"{what} is a lazily negated view: resolve_neg() it first")
    shape, stride = t.shape, t.stride()
    if shape[-1] > 1 and stride[-1] != 1:
        raise ValueError(f"{what}: the values of a row must be consecutive")
    pitch = span = None
    for n, st in zip(reversed(shape[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if pitch is None:
            pitch = st
        elif st != span:
            raise ValueError(f"{what}: the rows must be evenly spaced over the leading dimensions")
        span = n * st
    return shape[-1] if pitch is None else pitch


def _optional(t, what: str):
    """Pointer and pitch of rows that may be absent."""
    return (None, 0) if t is None else (t.data_ptr(), _pitch(t, what))


def _check_rows(hidden, gamma):
    """(N, H, shape, dtype, device) of rows and their gain."""
    if not hidden.is_cuda:
        raise ValueError("hidden must be a device tensor")
    shape, dtype, dev = hidden.shape, hidden.dtype, hidden.device
    if dtype not in DTYPES:
        raise ValueError("hidden must be bfloat16, float16 or float32")
    if not shape or shape[-1] < 1:
        raise ValueError("hidden must be [..., H]")
    H = shape[-1]
    if gamma.shape != (H,) or gamma.dtype is not dtype or gamma.get_device() != dev.index:
        raise ValueError("gamma must be [H] of the hidden dtype, on the hidden's device")
    if not gamma.is_contiguous() or gamma.is_neg() or hidden.is_neg():
        raise ValueError("gamma must be contiguous, and nothing a lazily negated view")
    return hidden.numel() // H, H, shape, dtype, dev


def _check_like(t, shape, dtype, dev, what: str):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev.index:
        raise ValueError(f"{what} must have the hidden's shape, dtype and device")
    if t.is_neg():
        raise ValueError(f"{what} is a lazily negated view: resolve_neg() it first")


def _written(tensors) -> None:
    """Tells autograd that the kernels write these tensors (a saved one of them is then refused in a backward)."""
    try:
        torch.autograd.graph.increment_version(tensors)
    except RuntimeError:  # inference tensors have no version
        torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


def _check_unfollowed(t, what: str) -> None:
    """A given output must not have a graph: it would keep it, and say that it is something else."""
    if t.requires_grad and torch.is_grad_enabled():
        raise ValueError(f"{what} requires a gradient, and this call is not differentiable: give it detached, or call under torch.no_grad()")


def _output(t, like, dtype, what: str):
    """A given output, checked, or a new one (rows of `like`'s shape), and its pitch."""
    if t is None:
        H = like.shape[-1]
        if not like.is_contiguous():
            return like.new_empty(like.shape, dtype=dtype), H
        return torch.empty_like(like) if dtype is like.dtype else torch.empty_like(like, dtype=dtype), H
    _check_like(t, like.shape, dtype, like.device, what)
    _check_unfollowed(t, what)
    _written([t])
    return t, _pitch(t, what)


def _run_forward(hidden, residual, gamma, eps, quant, group_size, normed, added, return_rstd):
    N, H, shape, dtype, dev = _check_rows(hidden, gamma)
    out, out_pitch = _output(normed, hidden, FP8 if quant else dtype, "normed")
    scales = None
    if quant:
        scales = hidden.new_empty(shape[:-1] + (-(-H // group_size) if group_size else 1,), dtype=torch.float32)
    if residual is None:
        if added is not None:
            raise ValueError("without a residual there is no sum: it is hidden itself")
        total, res, res_pitch, total_ptr, total_pitch = hidden, None, 0, None, 0
    else:
        _check_like(residual, shape, dtype, dev, "residual")
        total, total_pitch = _output(added, hidden, dtype, "added")
        res, res_pitch, total_ptr = residual.data_ptr(), _pitch(residual, "residual"), total.data_ptr()
    rstd = hidden.new_empty(shape[:-1], dtype=torch.float32) if return_rstd else None
    if N:
        r = None if rstd is None else rstd.data_ptr()
        if quant:
            _call("lce_add_rmsnorm_quant", dev, hidden.data_ptr(), _pitch(hidden, "hidden"), res, res_pitch, gamma.data_ptr(),
                  N, H, DTYPES[dtype], eps, group_size, out.data_ptr(), out_pitch, scales.data_ptr(), total_ptr, total_pitch, r)
        else:
            _call("lce_add_rmsnorm_forward", dev, hidden.data_ptr(), _pitch(hidden, "hidden"), res, res_pitch, gamma.data_ptr(),
                  N, H, DTYPES[dtype], eps, out.data_ptr(), out_pitch, total_ptr, total_pitch, r)
    outs = (out, scales, total) if quant else (out, total)
    return outs + (rstd,) if return_rstd else outs


def add_rmsnorm_forward(hidden, residual, gamma, eps: float = 1e-5, normed=None, added=None,
                        return_rstd: bool = False):
    """(normed, added[, rstd]): added = hidden + residual and normed = RMSNorm(added) * gamma.

    hidden [..., H] and residual (or None: added is hidden itself) need consecutive values in a row and
    evenly spaced rows, not contiguity. The sum is normalised in fp32, before its rounding. `normed` and
    `added` may be given, and may be hidden or residual themselves (a residual stream updated in place).
    Given outputs, here and in the calls below, must not require a gradient where gradients are recorded.
    rstd [...] (fp32) is 1 / sqrt(mean(added^2) + eps), for add_rmsnorm_backward. Not differentiable, in
    forward mode either: see add_rmsnorm.
    """
    return _run_forward(hidden, residual, gamma, eps, False, 0, normed, added, return_rstd)


def add_rmsnorm_quant(hidden, residual, gamma, eps: float = 1e-5, group_size: int = 0, quantised=None, added=None,
                      return_rstd: bool = False):
    """(quantised, scales, added[, rstd]): as add_rmsnorm_forward, the normalised rows as float8_e4m3fn.

    Each group of `group_size` (32, 64 or 128; 0: the whole row) consecutive values of a row has one fp32
    scale, its largest magnitude / 448: quantised * scale stands for the value. scales is
    [..., ceil(H / group_size)] ([..., 1] with a scale per row). Not differentiable.
    """
    if group_size not in GROUP_SIZES:
        raise ValueError(f"group_size must be one of {GROUP_SIZES}")
    return _run_forward(hidden, residual, gamma, eps, True, group_size, quantised, added, return_rstd)


def add_rmsnorm_workspace_size(N: int, H: int, dtype=torch.bfloat16) -> int:
    return int(_library().lce_add_rmsnorm_workspace_size(N, H, DTYPES[dtype]))


def add_rmsnorm_backward(grad_normed, grad_added, hidden, residual, gamma, rstd, need_gamma: bool = True,
                         grad_hidden=None, workspace: torch.Tensor | None = None):
    """(grad_hidden, grad_gamma) from the upstream gradients of normed and of added (None: there is none).

    hidden, residual (or None) and gamma as the forward call had them; or added and None, where one tensor
    is kept instead of two (the sum then enters with its rounding). grad_hidden is the gradient of hidden
    and of the residual alike; it may be given, and may be grad_normed, grad_added, hidden or residual
    themselves. grad_gamma is None without need_gamma.
    """
    N, H, shape, dtype, dev = _check_rows(hidden, gamma)
    _check_like(grad_normed, shape, dtype, dev, "grad_normed")
    if grad_added is not None:
        _check_like(grad_added, shape, dtype, dev, "grad_added")
    if residual is not None:
        _check_like(residual, shape, dtype, dev, "residual")
    if rstd.shape != shape[:-1] or rstd.dtype != torch.float32 or rstd.device != dev or not rstd.is_contiguous() or rstd.is_neg():
        raise ValueError("rstd must be the forward call's")
    dx, dx_pitch = _output(grad_hidden, hidden, dtype, "grad_hidden")
    dg = ws = None
    size = 0
    if need_gamma:
        dg = torch.empty_like(gamma)
        size = (_lib or _library()).lce_add_rmsnorm_workspace_size(N, H, DTYPES[dtype])
        if size == 0:
            raise LCEError(2, "lce_add_rmsnorm_workspace_size")
        ws = _space(workspace, hidden, size)
        size = ws.numel()
    elif N == 0:
        return dx, None
    _call("lce_add_rmsnorm_backward", dev, grad_normed.data_ptr(), _pitch(grad_normed, "grad_normed"),
          *_optional(grad_added, "grad_added"), hidden.data_ptr(), _pitch(hidden, "hidden"),
          *_optional(residual, "residual"), gamma.data_ptr(), rstd.data_ptr(), N, H, DTYPES[dtype],
          dx.data_ptr(), dx_pitch, None if dg is None else dg.data_ptr(),
          None if ws is None else ws.data_ptr(), size)
    return dx, dg


def _upstream(g):
    """An upstream gradient as rows that the kernels can read: its values in memory, its rows evenly spaced."""
    if g is None or (type(g) is torch.Tensor and g.is_contiguous() and not g.is_neg() and g.data_ptr() != 0):
        return g
    if not _bytes_are_values(g):
        if type(g) is not torch.Tensor:
            raise ValueError("the upstream gradient must be a plain tensor")
        # Lazily negated or zero tensors become memory; batched ones (is_grads_batched) cannot.
        g = torch.zeros(g.shape, dtype=g.dtype, device=g.device).add_(g)
        if not _bytes_are_values(g):
            raise ValueError("the upstream gradient must be a plain tensor")
    try:
        _pitch(g, "grad")
        return g
    except ValueError:
        return g.contiguous()


class AddRMSNorm(torch.autograd.Function):
    """(normed, added) of add_rmsnorm_forward with its gradients; without a residual, normed alone.

    The backward takes the unrounded sum, as the forward did: both addends are kept for it, not their
    rounded sum, which would put a second rounding into every gradient (gamma's 1.5 times as far off).
    """

    @staticmethod
    def forward(ctx, hidden, residual, gamma, eps):
        ctx.set_materialize_grads(False)
        need = True in ctx.needs_input_grad
        normed, added, *rstd = _run_forward(hidden, residual, gamma, eps, False, 0, None, None, need)
        if need:
            ctx.save_for_backward(hidden, residual, gamma, rstd[0])
        return normed if residual is None else (normed, added)

    @staticmethod
    def backward(ctx, grad_normed, grad_added=None):
        # Under create_graph the gradients say so if they are differentiated again; without, that costs nothing.
        if torch.is_grad_enabled():
            return AddRMSNorm._once(ctx, grad_normed, grad_added)
        return AddRMSNorm._gradients(ctx, grad_normed, grad_added)

    @staticmethod
    def _gradients(ctx, grad_normed, grad_added):
        hidden, residual, gamma, rstd = ctx.saved_tensors
        need = ctx.needs_input_grad
        need_gamma = need[2]
        grad_normed, grad_added = _upstream(grad_normed), _upstream(grad_added)
        if grad_normed is None:  # nothing came back through the norm
            grads = grad_added, torch.zeros_like(gamma) if need_gamma else None
        else:
            # All are checked again: hooks may have changed what was saved.
            grads = add_rmsnorm_backward(grad_normed, grad_added, hidden, residual, gamma, rstd, need_gamma)
        return grads[0] if need[0] else None, grads[0] if need[1] else None, grads[1], None

    _once = staticmethod(torch.autograd.function.once_differentiable(_gradients.__func__))


def add_rmsnorm(hidden, residual, gamma, eps: float = 1e-5):
    """(normed, added): added = hidden + residual, normed = RMSNorm(added) * gamma. Differentiable (once)."""
    if residual is None:
        raise ValueError("residual is None: rmsnorm(hidden, gamma, eps) is the norm alone")
    return AddRMSNorm.apply(hidden, residual, gamma, eps)


def rmsnorm(hidden, gamma, eps: float = 1e-5):
    """RMSNorm(hidden) * gamma over the last dimension. Differentiable (once)."""
    return AddRMSNorm.apply(hidden, None, gamma, eps)


# ---- the global norm of many gradients, and clipping -----------------------------------------------

def _dense(t) -> bool:
    """Whether t's values fill one block of memory, each place once, in whatever order of dimensions."""
    if t.is_contiguous():
        return True
    want = 1
    for st, n in sorted((st, n) for n, st in zip(t.shape, t.stride()) if n != 1):
        if st != want:
            return False
        want *= n
    return True


def _check_grads(grads):
    """The gradients that are not None, their device, their lce_tensor_t entries, and whether one requires a gradient."""
    grads = [grads] if isinstance(grads, torch.Tensor) else [g for g in grads if g is not None]
    if not grads:
        raise ValueError("no gradients")
    index, flat = grads[0].get_device(), []
    if index < 0:
        raise ValueError("gradients must be device tensors")
    strided, codes, requires = torch.strided, DTYPES, False
    for g in grads:  # a model has hundreds: half a microsecond for each
        code = codes.get(g.dtype)
        if code is None or g.layout is not strided or g.is_neg():
            raise ValueError("gradients must be dense bfloat16, float16 or float32 tensors, not lazily negated views")
        if g.get_device() != index:
            raise ValueError("gradients must be tensors of one device")
        if not (g.is_contiguous() or g.numel() == 0 or _dense(g)):
            raise ValueError("a gradient's values must fill one block of memory, in any order")
        if g.requires_grad:
            requires = True
        flat += (g.data_ptr(), g.numel(), code)
    return grads, grads[0].device, array.array("q", flat), requires


def _followed(grads, requires) -> bool:
    return (requires or getattr(torch.autograd.forward_ad, "_current_level", 0) >= 0) and _differentiated(grads)


class _Undifferentiated(torch.autograd.Function):
    """What a call gives for tensors that autograd follows: differentiating it raises, instead of finding constants."""

    @staticmethod
    def forward(ctx, call, *followed):
        return call()

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the gradients' norm and clipping are not differentiable: detach() them to use them as constants")

    @staticmethod
    def jvp(ctx, *tangents):
        _Undifferentiated.backward(ctx)


def _norm_type(norm_type):
    if norm_type not in NORM_TYPES:
        raise ValueError("norm_type must be 2.0 or inf")
    return NORM_TYPES[norm_type]


def grad_norm_workspace_size(count: int) -> int:
    """Bytes of workspace for `count` gradients."""
    return int((_lib or _library()).lce_grad_norm_workspace_size(count))


def grad_norm(grads, norm_type: float = 2.0, workspace: torch.Tensor | None = None):
    """The norm (2 or inf) over all values of the gradients: a device scalar in fp32, squares summed in fp64.

    grads: device tensors (Nones among them are left out) of one device and any of the three types, each
    filling one block of memory. Not differentiable: of gradients with a graph of their own (create_graph) the
    norm raises if it is differentiated.
    """
    kind = _norm_type(norm_type)
    grads, dev, table, requires = _check_grads(grads)
    if _followed(grads, requires):
        return _Undifferentiated.apply(lambda: _norm(grads, dev, table, kind, workspace), *grads)
    return _norm(grads, dev, table, kind, workspace)


def _norm(grads, dev, table, norm_type, workspace):
    norm = grads[0].new_empty((), dtype=torch.float32)
    ws = _space(workspace, grads[0], grad_norm_workspace_size(len(grads)))
    _call("lce_grad_norm", dev, table.buffer_info()[0], len(grads), norm_type, norm.data_ptr(), ws.data_ptr(), ws.numel())
    return norm


def _clip(grads, dev, table, max_norm, norm_type, out, workspace):
    kinds = set(map(type, grads))
    if kinds != _PLAIN and any(issubclass(c, torch.nn.Parameter) for c in kinds):  # scaling the weights themselves is never meant
        raise ValueError("clipping takes gradients, not parameters: [p.grad for p in parameters]")
    norm = grads[0].new_empty((), dtype=torch.float32)
    ws = _space(workspace, grads[0], grad_norm_workspace_size(len(grads)))
    outs = None if out is None else array.array("Q", [t.data_ptr() for t in out])
    _written(grads if out is None else out)
    _call("lce_clip_grad_norm", dev, table.buffer_info()[0], len(grads), norm_type, max_norm,
          None if outs is None else outs.buffer_info()[0], norm.data_ptr(),
          ws.data_ptr(), ws.numel())
    return norm


def clip_grad_norm_(grads, max_norm: float, norm_type: float = 2.0, workspace: torch.Tensor | None = None):
    """Scales the gradients in place so that their norm is at most max_norm; returns the norm before.

    The factor is min(1, max_norm / (norm + 1e-6)). Nothing waits for the norm: it and the factor stay on
    the device, and gradients within the limit are not written. A NaN among the gradients makes all NaN.
    Autograd does not see it, as if under torch.no_grad(): the norm is a constant, and gradients with a graph
    of their own keep the one they had.
    """
    kind = _norm_type(norm_type)
    grads, dev, table, requires = _check_grads(grads)
    if requires and any(g.requires_grad and g.is_leaf for g in grads):
        raise ValueError("a leaf that requires a gradient is a weight, not a gradient: [p.grad for p in parameters]")
    return _clip(grads, dev, table, max_norm, kind, None, workspace)


def clip_grad_norm(grads, max_norm: float, norm_type: float = 2.0, out=None, workspace: torch.Tensor | None = None):
    """(norm, clipped): as clip_grad_norm_, with the scaled gradients in other memory.

    out: tensors of the gradients' shapes, strides and types (for instance those that a copy to the host
    reads), one for each gradient that is not None; new ones by default. Not differentiable: of gradients
    with a graph of their own the norm and new tensors raise if they are differentiated.
    """
    kind = _norm_type(norm_type)
    grads, dev, table, requires = _check_grads(grads)
    if out is not None:
        out = [out] if isinstance(out, torch.Tensor) else [t for t in out if t is not None]
        index, same = dev.index, len(out) == len(grads)
        for t, g in zip(out, grads):  # half a microsecond for each, as in _check_grads
            if (t.get_device() != index or t.dtype is not g.dtype or t.shape != g.shape or t.is_neg()
                    or not (t.is_contiguous() and g.is_contiguous() or t.stride() == g.stride() or t.numel() <= 1)):
                same = False
            if t.requires_grad:
                _check_unfollowed(t, "out")
        if not same:
            raise ValueError("out must match the gradients in number, shape, strides, dtype and device")
    if _followed(grads, requires):
        norm, *new = _Undifferentiated.apply(lambda: _clip_into(grads, dev, table, max_norm, kind, out, workspace), *grads)
        return norm, new if out is None else out
    if out is None:
        norm, *out = _clip_into(grads, dev, table, max_norm, kind, None, workspace)
        return norm, out
    return _clip(grads, dev, table, max_norm, kind, out, workspace), out


def _clip_into(grads, dev, table, max_norm, norm_type, out, workspace):
    """The norm, and the clipped gradients where they are new."""
    outs = [torch.empty_like(g) for g in grads] if out is None else out
    norm = _clip(grads, dev, table, max_norm, norm_type, outs, workspace)
    return (norm,) if out is not None else (norm, *outs)

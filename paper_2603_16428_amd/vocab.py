"""Python binding of the operators on the vocabulary's matrix and logits (include/lce_vocab.h).

In front of a model: the rows of its V x H matrix that tokens name, and their gradient, alone or added to that of an output
layer with the same weight. Behind it, when it answers: the output layer's product with a weight in 4 bits, and a token from
logits. Argument marshalling only, as in lce.py and ops.py: every computation runs in liblce.so's HIP
kernels, on the current stream of the tensors' device, and nothing waits for the GPU.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import ops
from .lce import DTYPES, LCEError, _differentiated, load_library
from .ops import _check_unfollowed, _pitch, _space, _upstream, _written

EXPORTED = ("lce_embedding_forward", "lce_embedding_workspace_size", "lce_embedding_backward", "lce_mxfp4_quantize",
            "lce_mxfp4_dequantize", "lce_mxfp4_matmul", "lce_sample_workspace_size", "lce_sample")
_TOKENS = {torch.int64: 8, torch.int32: 4}

class SampleSettings(ctypes.Structure):
    """lce_sample_t."""

    _fields_ = [("temperature", ctypes.c_float), ("top_p", ctypes.c_float), ("min_p", ctypes.c_float), ("top_k", ctypes.c_int32),
                ("temperatures", ctypes.c_void_p), ("top_ps", ctypes.c_void_p), ("min_ps", ctypes.c_void_p), ("top_ks", ctypes.c_void_p)]


_lib = None


def _library() -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    lib = load_library()
    i64, vp, sz, ci, f32 = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_float
    for name, args, res in [
            ("lce_embedding_forward", [vp, ci, i64, vp, i64, i64, i64, ci, f32, vp, i64, vp], ci),
            ("lce_embedding_workspace_size", [i64, i64], sz),
            ("lce_embedding_backward", [vp, i64, vp, ci, i64, i64, i64, ci, f32, i64, vp, i64, ci, vp, sz, vp], ci),
            ("lce_mxfp4_quantize", [vp, i64, i64, i64, ci, vp, vp, vp], ci),
            ("lce_mxfp4_dequantize", [vp, vp, i64, i64, ci, vp, i64, vp], ci),
            ("lce_mxfp4_matmul", [vp, vp, i64, vp, vp, i64, i64, ci, vp, i64, vp], ci),
            ("lce_sample_workspace_size", [i64, i64], sz),
            ("lce_sample", [vp, i64, i64, i64, ci, vp, ctypes.POINTER(SampleSettings), vp, vp, vp, sz, vp], ci)]:
        f = getattr(lib, name)
        f.argtypes, f.restype = args, res
    _lib = lib
    return lib


def _call(name: str, device, *args) -> None:
    if _lib is None:
        _library()
    ops._call(name, device, *args)


def _device_rows(t, what: str):
    """The device of rows in one of the three types."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if t.dtype not in DTYPES:
        raise ValueError(f"{what} must be bfloat16, float16 or float32")
    if t.is_neg():
        raise ValueError(f"{what} is a lazily negated view: resolve_neg() it first")
    return t.device


def _given(t, shape, dtype, dev, what: str):
    """A given output, checked and told to autograd as written."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != dev.index:
        raise ValueError(f"{what} must be {list(shape)} of {dtype} on {dev}")
    if t.is_neg():
        raise ValueError(f"{what} is a lazily negated view: resolve_neg() it first")
    _check_unfollowed(t, what)
    _written([t])
    return t


class _Undifferentiated(torch.autograd.Function):
    """What a call gives for tensors that autograd follows: differentiating it raises, instead of finding constants."""

    @staticmethod
    def forward(ctx, call, *followed):
        return call()

    @staticmethod
    def backward(ctx, *grads):
        raise RuntimeError("the 4-bit product and sampling are not differentiable: detach() their input to use them as constants")

    @staticmethod
    def jvp(ctx, *tangents):
        _Undifferentiated.backward(ctx)


def _followed(t) -> bool:
    return (t.requires_grad or getattr(torch.autograd.forward_ad, "_current_level", 0) >= 0) and _differentiated([t])


# ---- embedding -----------------------------------------------------------------------------------

def _check_tokens(tokens, dev):
    """Bytes of a token."""
    if tokens.get_device() != dev.index:
        raise ValueError("tokens must be on the device of the rows")
    size = _TOKENS.get(tokens.dtype)
    if size is None or not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous int64 or int32")
    return size


def _check_scale(scale):
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")


def embedding_forward(tokens, weight, scale: float = 1.0, out=None):
    """scale * weight[tokens]: [..., H] of weight's type, each value rounded once.

    tokens [...] (int64 or int32, contiguous), weight [V, H] with consecutive values in a row. A token outside [0, V) gives a row
    of NaN. Not differentiable, in forward mode either: see embedding.
    """
    dev = _device_rows(weight, "weight")
    if weight.dim() != 2 or weight.shape[0] < 1 or weight.shape[1] < 1:
        raise ValueError("weight must be [V, H]")
    size = _check_tokens(tokens, dev)
    _check_scale(scale)
    V, H = weight.shape
    shape = tokens.shape + (H,)
    if out is None:
        out, pitch = weight.new_empty(shape), H
    else:
        pitch = _pitch(_given(out, shape, weight.dtype, dev, "out"), "out")
    _call("lce_embedding_forward", dev, tokens.data_ptr(), size, tokens.numel(), weight.data_ptr(), _pitch(weight, "weight"), V, H,
          DTYPES[weight.dtype], scale, out.data_ptr(), pitch)
    return out


def embedding_workspace_size(N: int, H: int) -> int:
    """Bytes of workspace for the gradient of N tokens' rows."""
    return int((_lib or _library()).lce_embedding_workspace_size(N, H))


def embedding_backward(grad, tokens, num_embeddings: int, scale: float = 1.0, padding_idx: int | None = None, grad_weight=None,
                       accumulate: bool = False, workspace: torch.Tensor | None = None):
    """The gradient of the weight, [num_embeddings, H]: for each token, scale times the sum of its rows of grad [..., H].

    Sums are fp32 in an order that the tokens fix, rounded once. grad_weight may be given; with accumulate the sums are added
    to the values there (that of linear_cross_entropy where the output layer has the same weight), and only the rows
    that tokens name are read and written. Rows of padding_idx, and of tokens outside the matrix, count for nothing. tokens are
    contiguous. Not differentiable, in forward mode either.
    """
    dev = _device_rows(grad, "grad")
    size = _check_tokens(tokens, dev)
    _check_scale(scale)
    if grad.dim() < 1 or grad.shape[:-1] != tokens.shape or grad.shape[-1] < 1:
        raise ValueError("grad must be [..., H] with a row for each token")
    if num_embeddings < 1 or (padding_idx is not None and not 0 <= padding_idx < num_embeddings):
        raise ValueError("padding_idx must be a token of the matrix, which has at least one row")
    N, H = tokens.numel(), grad.shape[-1]
    if grad_weight is None:
        if accumulate:
            raise ValueError("accumulate adds to a given grad_weight")
        grad_weight, pitch = grad.new_empty((num_embeddings, H)), H
    else:
        pitch = _pitch(_given(grad_weight, (num_embeddings, H), grad.dtype, dev, "grad_weight"), "grad_weight")
    need = (_lib or _library()).lce_embedding_workspace_size(N, H)
    if need == 0:
        raise LCEError(2, "lce_embedding_workspace_size")
    ws = _space(workspace, grad, need)
    _call("lce_embedding_backward", dev, grad.data_ptr(), _pitch(grad, "grad"), tokens.data_ptr(), size, N, num_embeddings, H,
          DTYPES[grad.dtype], scale, -1 if padding_idx is None else padding_idx, grad_weight.data_ptr(), pitch, int(accumulate),
          ws.data_ptr(), ws.numel())
    return grad_weight


class Embedding(torch.autograd.Function):
    """embedding_forward with the gradient of weight, a dense tensor."""

    @staticmethod
    def forward(ctx, tokens, weight, scale, padding_idx):
        ctx.set_materialize_grads(False)
        if padding_idx is not None and not 0 <= padding_idx < len(weight):
            raise ValueError("padding_idx must be a token of the matrix")
        ctx.save_for_backward(tokens)
        ctx.call = len(weight), scale, padding_idx
        return embedding_forward(tokens, weight, scale)

    @staticmethod
    def backward(ctx, grad):
        if torch.is_grad_enabled():  # under create_graph: the gradient says so if it is differentiated again
            return Embedding._once(ctx, grad)
        return Embedding._gradients(ctx, grad)

    @staticmethod
    def _gradients(ctx, grad):
        if grad is None or not ctx.needs_input_grad[1]:
            return None, None, None, None
        tokens, = ctx.saved_tensors
        return None, embedding_backward(_upstream(grad), tokens, *ctx.call), None, None

    _once = staticmethod(torch.autograd.function.once_differentiable(_gradients.__func__))


def embedding(tokens, weight, scale: float = 1.0, padding_idx: int | None = None):
    """scale * weight[tokens] for contiguous tokens. Differentiable (once) with respect to weight; rows of padding_idx get no gradient.

    The gradient is a tensor of weight's size: where weight is an output layer's too, autograd adds up two of them. (A backward
    written by hand adds the second in place: embedding_backward with accumulate.)
    """
    return Embedding.apply(tokens, weight, scale, padding_idx)


# ---- rows and weights in 4 bits --------------------------------------------------------------------

MXFP4_GROUP = 32


def _check_codes(codes, scales, what: str):
    """The leading shape and H of a matrix in 4 bits."""
    if not codes.is_cuda or codes.dtype is not torch.uint8 or scales.dtype is not torch.uint8 or scales.device != codes.device:
        raise ValueError(f"{what}: codes and scales must be uint8 tensors of one device")
    H = 2 * codes.shape[-1] if codes.dim() else 0
    if H < MXFP4_GROUP or H % MXFP4_GROUP or scales.shape != codes.shape[:-1] + (H // MXFP4_GROUP,):
        raise ValueError(f"{what}: codes must be [..., H/2] and scales [..., H/32], H a multiple of 32")
    if not codes.is_contiguous() or not scales.is_contiguous():
        raise ValueError(f"{what}: codes and scales must be contiguous")
    return codes.shape[:-1], H


def mxfp4_quantize(hidden, codes=None, scales=None):
    """(codes, scales): rows [..., H] (H a multiple of 32) in 4 bits with a power of two for each 32 values (OCP MXFP4).

    codes [..., H/2] (uint8) hold two values a byte, the first in the low half: sign, two bits of exponent, one of mantissa
    (0, 0.5, 1, 1.5, 2, 3, 4, 6). scales [..., H/32] (uint8) hold exponents + 127: that of the group's largest magnitude less 2.
    A group with a NaN or an infinity has scale 255. Both may be given. Not differentiable.
    """
    dev = _device_rows(hidden, "hidden")
    H = hidden.shape[-1] if hidden.dim() else 0
    if H < MXFP4_GROUP or H % MXFP4_GROUP:
        raise ValueError("hidden must be [..., H] with H a multiple of 32")
    pitch, lead = _pitch(hidden, "hidden"), hidden.shape[:-1]
    outs = []
    for t, n, what in ((codes, H // 2, "codes"), (scales, H // MXFP4_GROUP, "scales")):
        if t is None:
            t = hidden.new_empty(lead + (n,), dtype=torch.uint8)
        elif not _given(t, lead + (n,), torch.uint8, dev, what).is_contiguous():
            raise ValueError(f"{what} must be contiguous")
        outs.append(t)
    codes, scales = outs
    _call("lce_mxfp4_quantize", dev, hidden.data_ptr(), pitch, hidden.numel() // H, H, DTYPES[hidden.dtype], codes.data_ptr(), scales.data_ptr())
    return codes, scales


def mxfp4_dequantize(codes, scales, dtype=torch.bfloat16, out=None):
    """The values [..., H] that codes and scales stand for, rounded once to dtype. Not differentiable."""
    lead, H = _check_codes(codes, scales, "mxfp4")
    if dtype not in DTYPES:
        raise ValueError("dtype must be bfloat16, float16 or float32")
    if out is None:
        out, pitch = codes.new_empty(lead + (H,), dtype=dtype), H
    else:
        pitch = _pitch(_given(out, lead + (H,), dtype, codes.device, "out"), "out")
    _call("lce_mxfp4_dequantize", codes.device, codes.data_ptr(), scales.data_ptr(), out.numel() // H, H, DTYPES[dtype], out.data_ptr(), pitch)
    return out


def mxfp4_matmul(codes, scales, weight_codes, weight_scales, dtype=torch.bfloat16, out=None):
    """Rows [..., H] times a weight [V, H], both in 4 bits: [..., V] in dtype, summed in fp32, rounded once. Not differentiable."""
    lead, H = _check_codes(codes, scales, "rows")
    shape, weight_H = _check_codes(weight_codes, weight_scales, "weight")
    if len(shape) != 1 or weight_H != H or weight_codes.device != codes.device:
        raise ValueError("the weight must be [V, H] with the rows' H, on their device")
    if dtype not in DTYPES:
        raise ValueError("dtype must be bfloat16, float16 or float32")
    V = shape[0]
    if out is None:
        out, pitch = codes.new_empty(lead + (V,), dtype=dtype), V
    else:
        pitch = _pitch(_given(out, lead + (V,), dtype, codes.device, "out"), "out")
    _call("lce_mxfp4_matmul", codes.device, codes.data_ptr(), scales.data_ptr(), lead.numel(), weight_codes.data_ptr(), weight_scales.data_ptr(),
          V, H, DTYPES[dtype], out.data_ptr(), pitch)
    return out


def mxfp4_linear(hidden, weight_codes, weight_scales, out=None):
    """hidden [..., H], quantised here, times a weight in 4 bits: [..., V] of hidden's type (an output layer's logits).

    Not differentiable: training keeps the weight in its own type (linear_cross_entropy). Of a hidden that autograd follows the
    result raises if it is differentiated.
    """
    if _followed(hidden):
        if out is not None:
            raise ValueError("hidden requires a gradient, and this call is not differentiable: give it detached, or call under torch.no_grad()")
        return _Undifferentiated.apply(lambda: mxfp4_linear(hidden.detach(), weight_codes, weight_scales), hidden)
    codes, scales = mxfp4_quantize(hidden)
    return mxfp4_matmul(codes, scales, weight_codes, weight_scales, hidden.dtype, out)


# ---- a token from logits ---------------------------------------------------------------------------

def _setting(v, lead, dev, dtype, what: str):
    """(one value, a pointer to each row's)."""
    if not isinstance(v, torch.Tensor):
        return v, None
    if v.shape != lead or v.dtype is not dtype or v.get_device() != dev.index or not v.is_contiguous() or v.is_neg():
        raise ValueError(f"{what} must be a number or a contiguous tensor of {dtype} with one for each row, on the logits' device")
    return 0, v.data_ptr()


def sample_workspace_size(N: int, V: int) -> int:
    """Bytes of workspace for the tokens of N rows of V logits."""
    return int((_lib or _library()).lce_sample_workspace_size(N, V))


def sample(logits, uniforms, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, return_logprobs: bool = False,
           workspace: torch.Tensor | None = None):
    """tokens [...] (int64), or (tokens, logprobs): for each row of logits [..., V] the token that its number in uniforms [...] draws.

    uniforms are fp32 in [0, 1). Logits are divided by temperature (0: the largest logit, the first of equal ones); then top_k keeps that many
    of the largest (0: all; of equal ones the first), top_p of these as many as make up that share, and min_p of these those
    of at least that share of the largest one's probability. The kept ones, in the order of the vocabulary, divide up [0, 1) by their probabilities,
    and the token is the one whose part holds the row's number. Each setting is a number, or a tensor with one for each row (fp32; top_k:
    int32). logprobs (fp32) are the logs of the tokens' probabilities among the kept ones. A row with a NaN, or with
    nothing above -inf, gives -1. Not differentiable: the logprobs of logits or settings that autograd follows raise if they are differentiated.
    """
    if return_logprobs:
        given = logits, temperature, top_p, min_p
        followed = [v for v in given if isinstance(v, torch.Tensor) and _followed(v)]
        if followed:
            z, t, p, m = (v.detach() if isinstance(v, torch.Tensor) else v for v in given)
            return _Undifferentiated.apply(lambda: sample(z, uniforms, t, top_k, p, m, True, workspace), *followed)
    dev = _device_rows(logits, "logits")
    V = logits.shape[-1] if logits.dim() else 0
    if V < 1:
        raise ValueError("logits must be [..., V]")
    lead = logits.shape[:-1]
    if uniforms.shape != lead or uniforms.dtype is not torch.float32 or uniforms.get_device() != dev.index or not uniforms.is_contiguous() or uniforms.is_neg():
        raise ValueError("uniforms must be contiguous float32 with one for each row, on the logits' device")
    t, ts = _setting(temperature, lead, dev, torch.float32, "temperature")
    p, ps = _setting(top_p, lead, dev, torch.float32, "top_p")
    m, ms = _setting(min_p, lead, dev, torch.float32, "min_p")
    k, ks = _setting(top_k, lead, dev, torch.int32, "top_k")
    if not (t >= 0 and p >= 0 and 0 <= m <= 1 and k >= 0):
        raise ValueError("temperature, top_k and top_p must not be negative, min_p must be from 0 to 1")
    N, need = logits.numel() // V, (_lib or _library()).lce_sample_workspace_size(logits.numel() // V, V)
    if need == 0:
        raise LCEError(2, "lce_sample_workspace_size")
    tokens = logits.new_empty(lead, dtype=torch.int64)
    logprobs = logits.new_empty(lead, dtype=torch.float32) if return_logprobs else None
    ws = _space(workspace, logits, need)
    settings = SampleSettings(t, p, m, min(k, V), ts, ps, ms, ks)
    _call("lce_sample", dev, logits.data_ptr(), _pitch(logits, "logits"), N, V, DTYPES[logits.dtype], uniforms.data_ptr(), settings, tokens.data_ptr(),
          None if logprobs is None else logprobs.data_ptr(), ws.data_ptr(), ws.numel())
    return (tokens, logprobs) if return_logprobs else tokens

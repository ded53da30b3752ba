"""The layers beside a sparse product: norms, dropout, the matrix product and the gated feed-forward block, on the dense rows of features.

``SparseOperator`` (``autograd.py``) multiplies by the matrix; a graph network then works on the result row by row.  Here are
these steps as differentiable functions of GPU tensors in float32, bfloat16 or float16, over the HIP library
``libdgsp_layers.so`` (``include/dgsp_layers.h``).  Sums and statistics are held in 32 bits, and the same call gives the same
bits every time.

    s = residual + dropout(A x);  y = layer norm of s:      y, s = add_layer_norm(op(x), x, weight, bias, p=0.1, seed=7, offset=step)
    s + dropout(feed-forward block of y):                    dropout(gated_ff(y, w_gate, w_up, w_down), 0.1, 7, step, residual=s)

    root-mean-square norm, and the product after it:        linear(rms_norm(x, g), w, b, "gelu", residual=x)
    the same with activations kept in 8 bits:               linear(rms_norm(x, g), w, b, "gelu", residual=x, keep_8bit=True)
    and in 8 bits, for serving:                             linear_8bit(rms_norm_8bit(x, g), quantise(w), b, "gelu", residual=x)

Tensors may have any number of leading axes; the last one is the width.  Rows that lie at one distance from each other (a
column slice, a broadcast row) are taken as they are, other orders are copied first.  Work runs on the current stream and can be
captured into a graph.  Wrong arguments raise ``DgspError``.  Gradients of gradients are refused, and so is capturing the gradient
of a leaf while a result made from it on the default stream is still held.

Dropout's random numbers are a function of ``seed``, ``offset`` and the place of the element, and the mask is never stored:
give every call of a step its own ``offset`` (or its own ``seed``), and every step new ones.  ``offset`` may be an int64 GPU
tensor of one element, read when the kernels run: a replayed graph draws new masks if the program advances it in between.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.util
from pathlib import Path
from typing import NamedTuple

from . import binding as dg

LIB_PATH = Path(__file__).resolve().parent / "libdgsp_layers.so"
NATIVE_PATH = LIB_PATH.with_name("_dgsp_layers_torch.so")

F32, BF16, F16 = 0, 1, 2
SILU, GELU, RELU = 0, 1, 2
ACTIVATIONS = {"silu": SILU, "gelu": GELU, "relu": RELU}
NO_ACTIVATION = 3
E4M3, INT8 = 0, 1
KINDS = {"e4m3": E4M3, "int8": INT8}
KEEP_NOTHING, KEEP_WHOLE, KEEP_8BIT = 0, 1, 2

EXPORTS = (
    "dgsp_dropout", "dgsp_layer_norm", "dgsp_layer_norm_backward", "dgsp_layer_norm_backward_workspace_bytes", "dgsp_gated_ff",
    "dgsp_gated_ff_saved_bytes", "dgsp_gated_ff_workspace_bytes", "dgsp_gated_ff_backward",
    "dgsp_gated_ff_backward_workspace_bytes", "dgsp_rms_norm", "dgsp_rms_norm_backward", "dgsp_rms_norm_backward_workspace_bytes",
    "dgsp_quantise", "dgsp_dequantise", "dgsp_rms_norm_8bit", "dgsp_linear", "dgsp_linear_saved_bytes", "dgsp_linear_workspace_bytes",
    "dgsp_linear_backward", "dgsp_linear_backward_workspace_bytes", "dgsp_linear_8bit", "dgsp_linear_8bit_workspace_bytes",
)


class Dropout(ctypes.Structure):
    """``dgsp_dropout_t``"""
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("device_offset", ctypes.c_void_p)]


_lib = None


def lib():
    """The loaded library, for callers of the C entry points (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not LIB_PATH.exists():
            raise dg.DgspError(f"{LIB_PATH} is missing: run `python -m paper_2106_16064_amd.build` (there is no CPU fallback)")
        L = ctypes.CDLL(str(LIB_PATH))
        i64, vp, ci, cf, drop = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.POINTER(Dropout)
        L.dgsp_dropout.argtypes = [i64, i64, ci, drop, vp, i64, vp, i64, vp, i64, vp]
        L.dgsp_layer_norm.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, drop, vp, vp, cf, vp, i64, vp, i64, vp, vp]
        L.dgsp_layer_norm_backward.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, drop, vp, vp, vp, vp, vp, i64, vp]
        matrices = [vp, i64] * 4
        L.dgsp_gated_ff.argtypes = [i64] * 4 + [ci, ci] + matrices + [vp, i64, vp, vp, i64, vp]
        L.dgsp_gated_ff_backward.argtypes = [i64] * 4 + [ci, ci] + matrices + [vp, i64, vp, vp, vp, vp, vp, vp, i64, vp]
        for name in EXPORTS:
            getattr(L, name).restype = i64 if name.endswith("_bytes") else ci
        L.dgsp_layer_norm_backward_workspace_bytes.argtypes = [i64, i64]
        for name in ("saved", "workspace", "backward_workspace"):
            getattr(L, f"dgsp_gated_ff_{name}_bytes").argtypes = [i64, i64, i64, i64, ci]
        L.dgsp_rms_norm.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, drop, vp, cf, vp, i64, vp, i64, vp, vp]
        L.dgsp_rms_norm_backward.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, vp, vp, vp, i64, vp, i64, drop, vp, vp, vp, vp, i64, vp]
        L.dgsp_rms_norm_backward_workspace_bytes.argtypes = [i64, i64]
        L.dgsp_quantise.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, vp, vp]
        L.dgsp_dequantise.argtypes = [i64, i64, ci, ci, vp, i64, vp, vp, i64, vp]
        L.dgsp_rms_norm_8bit.argtypes = [i64, i64, ci, ci, vp, i64, vp, i64, vp, cf, vp, i64, vp, vp, i64, vp]
        L.dgsp_linear.argtypes = [i64] * 3 + [ci] * 4 + [vp, i64, vp, i64, vp, vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, vp]
        L.dgsp_linear_saved_bytes.argtypes = [i64, i64, ci, ci, ci, ci]
        L.dgsp_linear_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.dgsp_linear_backward.argtypes = [i64] * 3 + [ci] * 4 + [vp, i64, vp, vp, i64, vp, vp, i64, vp, vp, vp, vp, i64, vp]
        L.dgsp_linear_backward_workspace_bytes.argtypes = [i64, i64, i64, ci, ci, ci]
        L.dgsp_linear_8bit.argtypes = [i64] * 3 + [ci] * 3 + [vp, i64, vp, vp, i64, vp, vp, vp, i64, vp, i64, vp, i64, vp]
        L.dgsp_linear_8bit_workspace_bytes.argtypes = [i64, i64, i64]
        _lib = L
    return _lib


_native = None


def native():
    """The layers as native functions on tensors (positional arguments; see ``csrc_layers/torch_binding.cpp``)."""
    global _native
    if _native is None:
        import torch  # noqa: F401  (its libraries have to be loaded before the module)
        lib()
        if not NATIVE_PATH.exists():
            raise dg.DgspError(f"{NATIVE_PATH} is missing: run `python -m paper_2106_16064_amd.build`")
        spec = importlib.util.spec_from_file_location("_dgsp_layers_torch", NATIVE_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        module.set_error_type(dg.DgspError)
        _native = module
    return _native


def layer_norm(x, weight=None, bias=None, eps=1e-5):
    """``(x - mean) / sqrt(var + eps) * weight + bias`` over the last axis.  ``weight`` and ``bias``: one axis as long, in the
    type of ``x`` or float32, or None."""
    y = (_native or native()).layer_norm(x, weight, bias, eps)
    return _functions().norm.apply(x, None, weight, bias, eps, 0.0, 0, 0)[0] if y is None else y


def add_layer_norm(x, residual, weight=None, bias=None, eps=1e-5, p=0.0, seed=0, offset=0):
    """``s = residual + dropout(x)`` and the layer norm of ``s``, in one pass; returns ``(y, s)``.  ``s`` is rounded to the type
    of ``x``, ``y`` is made from the sum before that; of 16-bit types the backward pass makes it again and keeps ``x`` and
    ``residual`` for that."""
    out = (_native or native()).add_layer_norm(x, residual, weight, bias, eps, p, seed, offset)
    return _functions().norm.apply(x, residual, weight, bias, eps, p, seed, offset) if out is None else out


def dropout(x, p, seed, offset=0, residual=None):
    """``dropout(x)``, or ``residual + dropout(x)``: each element is dropped with probability ``p`` (in steps of 1/65536) and
    otherwise scaled so that the mean stays.  A dropped element counts as 0 whatever it holds."""
    y = (_native or native()).dropout(x, p, seed, offset, residual)
    return _functions().dropout.apply(x, p, seed, offset, residual) if y is None else y


def gated_ff(x, w_gate, w_up, w_down, activation="silu"):
    """The gated feed-forward block ``(act(x w_gate^T) * (x w_up^T)) w_down^T``; ``activation``: "silu", "gelu" or "relu".
    ``w_gate`` and ``w_up`` are hidden x width, ``w_down`` is out_width x hidden, all in the type of ``x``."""
    try:
        act = ACTIVATIONS[activation]
    except (KeyError, TypeError):
        raise dg.DgspError(f"activation must be one of {', '.join(ACTIVATIONS)}") from None
    y = (_native or native()).gated_ff(x, w_gate, w_up, w_down, act)
    return _functions().gated.apply(x, w_gate, w_up, w_down, act) if y is None else y


def rms_norm(x, weight=None, eps=1e-5):
    """``x / sqrt(mean(x^2) + eps) * weight`` over the last axis.  ``weight``: one axis as long, in the type of ``x`` or float32, or None."""
    y = (_native or native()).rms_norm(x, weight, eps)
    return _functions().rms.apply(x, None, weight, eps, 0.0, 0, 0)[0] if y is None else y


def add_rms_norm(x, residual, weight=None, eps=1e-5, p=0.0, seed=0, offset=0):
    """``s = residual + dropout(x)`` and the root-mean-square norm of ``s``, in one pass; returns ``(y, s)`` as ``add_layer_norm`` does."""
    out = (_native or native()).add_rms_norm(x, residual, weight, eps, p, seed, offset)
    return _functions().rms.apply(x, residual, weight, eps, p, seed, offset) if out is None else out


class Rows8(NamedTuple):
    """Rows in 8 bits: blocks of 32 columns, each with a power of two as its scale.

    ``values``: the rows' elements over their scales, float8_e4m3fn or int8, the last axis filled up with zeros to whole blocks.
    ``scales``: uint8, ``ceil(width / 128) x rows x 4``, byte ``b`` for ``2^(b - 127)``: block ``k`` of row ``r`` at ``[k // 4, r, k % 4]``;
    255 is NaN, and places beyond the last block hold 127.  ``width``: how many columns there are."""
    values: object
    scales: object
    width: int


def quantise(x, kind="e4m3"):
    """``x`` as :class:`Rows8`: "e4m3", which ``linear_8bit`` reads, or "int8", which is nearer to ``x``.  Each element is rounded to the
    nearest value, ties to even; it has no gradient."""
    if kind not in ("e4m3", "int8"):
        raise dg.DgspError(f"kind must be one of {', '.join(KINDS)}")
    return Rows8(*(_native or native()).quantise(x, KINDS[kind]), x.shape[-1])


def dequantise(rows, dtype=None):
    """The numbers that :class:`Rows8` stand for, as a tensor of ``dtype`` (float32 if None, bfloat16 or float16)."""
    values, scales, width = _as_rows8(rows, "rows")
    return (_native or native()).dequantise(values, scales, width, F32 if dtype is None else _type_number(dtype))


def rms_norm_8bit(x, weight=None, eps=1e-5):
    """The root-mean-square norm of ``x`` as :class:`Rows8` in e4m3, rounded once; for serving: it has no gradient."""
    return Rows8(*(_native or native()).rms_norm_8bit(x, None, weight, eps), x.shape[-1])


def add_rms_norm_8bit(x, residual, weight=None, eps=1e-5):
    """``s = residual + x`` and the root-mean-square norm of ``s`` as :class:`Rows8` in e4m3; returns ``(y, s)``.  It has no gradient."""
    _need_tensor(residual, "residual")
    values, scales, s = (_native or native()).rms_norm_8bit(x, residual, weight, eps)
    return Rows8(values, scales, x.shape[-1]), s


def linear(x, weight, bias=None, activation=None, residual=None, keep_8bit=False):
    """``act(x weight^T + bias) + residual`` in one pass; ``activation``: "silu", "gelu", "relu" or None.

    ``weight`` is out_width x width in the type of ``x``; ``bias`` has one axis of out_width, in the type of ``x`` or float32;
    ``residual`` has the shape and type of the result.  ``keep_8bit``: what the backward pass needs of the activations is kept in 8 bits,
    ``x`` as whole numbers with a scale for every 32 columns and the activation's derivative in steps of 1/112.  The result is the same; the
    weight's gradient is that of the ``x`` kept, and those of ``x``, weight and bias are made with the derivative kept.

    Without it ``x`` is kept, and of silu and gelu ``x weight^T + bias`` in the type of ``bias`` (of ``x`` if there is none): a float32 bias of
    16-bit matrices has an exact gradient for twice the memory.  With it the backward pass of 16-bit matrices wider than 128 lays the ``x`` kept
    out in their type while it runs."""
    act = _epilogue(activation)
    y = (_native or native()).linear(x, weight, bias, act, residual, bool(keep_8bit))
    return _functions().linear.apply(x, weight, bias, act, residual, bool(keep_8bit)) if y is None else y


def linear_8bit(x, weight, bias=None, activation=None, residual=None, dtype=None):
    """``linear`` of :class:`Rows8` in e4m3, for serving: products of eight neighbouring columns are added cut off 2^-13 below the power of two of
    the largest, and sums of those in 32 bits.  The result is of ``dtype`` (bfloat16 if None, float32 or float16); ``bias``: of that type or
    float32; ``residual``: of that type.  It has no gradient."""
    act = _epilogue(activation)
    type_number = BF16 if dtype is None else _type_number(dtype)
    return (_native or native()).linear_8bit(*_as_rows8(x, "x"), *_as_rows8(weight, "weight"), bias, act, residual, type_number)


def _epilogue(activation):
    if activation is None:
        return NO_ACTIVATION
    try:
        return ACTIVATIONS[activation]
    except (KeyError, TypeError):
        raise dg.DgspError(f"activation must be None or one of {', '.join(ACTIVATIONS)}") from None


def _as_rows8(rows, name):
    if not isinstance(rows, tuple) or len(rows) != 3:
        raise dg.DgspError(f"{name} must be Rows8: values, scales and width")
    return rows


def _need_tensor(t, name):
    if t is None:
        raise dg.DgspError(f"{name} must be a tensor")


def _type_number(dtype):
    import torch
    try:
        return {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}[dtype]
    except (KeyError, TypeError):
        raise dg.DgspError("dtype must be float32, bfloat16 or float16") from None


@functools.lru_cache(maxsize=None)
def _functions():
    """The layers as ``torch.autograd.Function``, for calls that the native graph nodes do not serve because more than reverse
    mode looks at them (see ``autograd.py``)."""
    import types

    import torch

    def keep(drop, *tensors):
        """What ``save_for_backward`` gets, with dropout's offset last if it is a tensor, and the arguments of dropout without it."""
        p, seed, offset = drop
        return ((*tensors, offset), (p, seed, None)) if isinstance(offset, torch.Tensor) else ((*tensors, None), drop)

    def given(drop, offset):
        return drop if offset is None else (*drop[:2], offset)

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, bias, eps, p, seed, offset):
            y, s, stats = native().layer_norm_forward(x, residual, weight, bias, eps, p, seed, offset)
            ctx.residual = residual is not None
            again = ctx.residual and x.dtype != torch.float32          # the sum is made again where the one written is rounded
            saved, ctx.drop = keep((p, seed, offset), s if ctx.residual and not again else x, residual if again else None, stats, weight, bias)
            ctx.save_for_backward(*saved)
            return (y, s) if ctx.residual else (y,)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, ds=None):
            s, added, stats, weight, bias, offset = ctx.saved_tensors
            dropped = ctx.residual and ctx.drop[0] > 0
            drop = given(ctx.drop, offset)
            dsum, dx, dweight, dbias = native().layer_norm_backward(s, added, stats, weight, bias, dy, ds, int(dropped), *drop)
            return dx if dropped else dsum, dsum if ctx.residual else None, dweight, dbias, None, None, None, None

    class Dropped(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, p, seed, offset, residual):
            ctx.residual = residual is not None
            saved, ctx.drop = keep((p, seed, offset))
            ctx.save_for_backward(*saved)
            return native().dropout_forward(x, p, seed, offset, residual)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            return native().dropout_forward(dy, *given(ctx.drop, *ctx.saved_tensors), None), None, None, None, dy if ctx.residual else None

    class Gated(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w_gate, w_up, w_down, activation):
            y, saved = native().gated_ff_forward(x, w_gate, w_up, w_down, activation)
            ctx.activation = activation
            ctx.save_for_backward(x, w_gate, w_up, w_down, saved)
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            x, w_gate, w_up, w_down, saved = ctx.saved_tensors
            return (*native().gated_ff_backward(x, w_gate, w_up, w_down, ctx.activation, dy, saved), None)

    class Rms(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, residual, weight, eps, p, seed, offset):
            y, s, rstd = native().rms_norm_forward(x, residual, weight, eps, p, seed, offset)
            ctx.residual = residual is not None
            again = ctx.residual and x.dtype != torch.float32
            saved, ctx.drop = keep((p, seed, offset), s if ctx.residual and not again else x, residual if again else None, rstd, weight)
            ctx.save_for_backward(*saved)
            return (y, s) if ctx.residual else (y,)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy, ds=None):
            s, added, rstd, weight, offset = ctx.saved_tensors
            dropped = ctx.residual and ctx.drop[0] > 0
            dsum, dx, dweight = native().rms_norm_backward(s, added, rstd, weight, dy, ds, int(dropped), *given(ctx.drop, offset))
            return dx if dropped else dsum, dsum if ctx.residual else None, dweight, None, None, None, None

    class Linear(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias, activation, residual, keep_8bit):
            y, saved, values, scales = native().linear_forward(x, weight, bias, activation, residual, keep_8bit)
            ctx.activation, ctx.residual = activation, residual is not None
            ctx.save_for_backward(values if keep_8bit else x, scales, weight, bias, saved)
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            x, scales, weight, bias, saved = ctx.saved_tensors
            dx, dweight, dbias = native().linear_backward(x, scales, weight, bias, saved, dy, ctx.activation)
            return dx, dweight, dbias, None, dy if ctx.residual else None, None

    return types.SimpleNamespace(norm=Norm, dropout=Dropped, gated=Gated, rms=Rms, linear=Linear)

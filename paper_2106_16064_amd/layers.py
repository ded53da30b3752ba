"""The layers beside a sparse product: layer norm, dropout and the gated feed-forward block, on the dense rows of features.

``SparseOperator`` (``autograd.py``) multiplies by the matrix; a graph network then works on the result row by row.  Here are
these steps as differentiable functions of GPU tensors in float32, bfloat16 or float16, over the HIP library
``libdgsp_layers.so`` (``include/dgsp_layers.h``).  Sums and statistics are held in 32 bits, and the same call gives the same
bits every time.

    s = residual + dropout(A x);  y = layer norm of s:      y, s = add_layer_norm(op(x), x, weight, bias, p=0.1, seed=7, offset=step)
    s + dropout(feed-forward block of y):                    dropout(gated_ff(y, w_gate, w_up, w_down), 0.1, 7, step, residual=s)

Tensors may have any number of leading axes; the last one is the width.  Rows that lie at one distance from each other (a
column slice, a broadcast row) are taken as they are, other orders are copied first.  Work runs on the current stream and can be
captured into a graph.  Wrong arguments raise ``DgspError``.  Gradients of gradients are refused.

Dropout's random numbers are a function of ``seed``, ``offset`` and the place of the element, and the mask is never stored:
give every call of a step its own ``offset`` (or its own ``seed``), and every step new ones.  ``offset`` may be an int64 GPU
tensor of one element, read when the kernels run: a replayed graph draws new masks if the program advances it in between.
"""
from __future__ import annotations

import ctypes
import functools
import importlib.util
from pathlib import Path

from . import binding as dg

LIB_PATH = Path(__file__).resolve().parent / "libdgsp_layers.so"
NATIVE_PATH = LIB_PATH.with_name("_dgsp_layers_torch.so")

F32, BF16, F16 = 0, 1, 2
SILU, GELU, RELU = 0, 1, 2
ACTIVATIONS = {"silu": SILU, "gelu": GELU, "relu": RELU}

EXPORTS = (
    "dgsp_dropout", "dgsp_layer_norm", "dgsp_layer_norm_backward", "dgsp_layer_norm_backward_workspace_bytes", "dgsp_gated_ff",
    "dgsp_gated_ff_saved_bytes", "dgsp_gated_ff_workspace_bytes", "dgsp_gated_ff_backward",
    "dgsp_gated_ff_backward_workspace_bytes",
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

    return types.SimpleNamespace(norm=Norm, dropout=Dropped, gated=Gated)

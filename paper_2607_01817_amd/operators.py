"""Operators beside the chunk loop: the root-mean-square norm, 8-bit products
and rotary positions, forward and backward (the C ABI's hcms_rms_norm*,
hcms_quantize_fp8, hcms_linear_fp8 and hcms_rope*).

8-bit tensors are ``float8_e4m3fn`` values with power-of-two scales held as
``float8_e8m0fnu``, one for each block of 128 elements of a row or of 128 x 128,
in groups of four blocks: ``[ceil(K / 512)][rows or blocks of rows][4]``.

The tensors are checked, allocated and passed on in ``_hcms_torch.so``
(csrc/torch_ops.cpp), which calls the C ABI and refuses what it refuses with
:class:`HcmsError`; wrong shapes, types and devices are ValueError and TypeError.
Calls run on the current stream, or on ``stream``, to which their outputs and
workspaces then belong.  Tensors given to write to (``out``, ``h_out``) carry no
gradient: one that requires grad is refused where autograd records, and a write to
one that an operator has saved for its backward makes that backward raise, as
PyTorch's own writes in place do.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

from . import _PKG, _check, _gpu_device, _ints, _table_rows, load

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
SCALE_BLOCK = 128
_HALF = {"interleaved": False, "half": True}
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class RopeHeads(ctypes.Structure):
    """hcms_rope_heads of the C ABI."""
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_token", ctypes.c_int64),
                ("x_head", ctypes.c_int64), ("y_token", ctypes.c_int64), ("y_head", ctypes.c_int64),
                ("heads", ctypes.c_int)]


@functools.lru_cache(maxsize=None)
def _ops():
    """The tensor side of the operators (raises if it has not been built)."""
    load()
    if not os.path.exists(os.path.join(_PKG, "_hcms_torch.so")):
        raise RuntimeError("_hcms_torch.so is missing: build it with "
                           "`python -m paper_2607_01817_amd.build` (no CPU fallback exists)")
    from . import _hcms_torch
    return _hcms_torch


def _under(stream, fn, *args):
    """fn(*args) with ``stream`` as the current stream."""
    with torch.cuda.stream(stream):
        return fn(*args)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
             residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
             h_out: torch.Tensor | None = None, *, stream=None):
    """Root-mean-square norm of rows: ``y = h / sqrt(mean(h^2) + eps) * weight``
    with ``h = x + residual``.  Returns y, or (y, h) with a residual, where h is
    the residual stream's next value.  x and residual [M][D] may have any row
    stride (a slice of a projection's output, for a norm of queries)."""
    if stream is not None:
        return _under(stream, rms_norm, x, weight, eps, residual, out, h_out)
    return _ops().rms_norm(x, weight, eps, residual, out, h_out)


def rms_norm_fp8(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
                 residual: torch.Tensor | None = None, h_out: torch.Tensor | None = None, *,
                 stream=None):
    """:func:`rms_norm` with y in 8 bits, as :func:`linear_fp8` reads it: returns
    (q, scale), or (q, scale, h) with a residual.  D must be a multiple of 16."""
    if stream is not None:
        return _under(stream, rms_norm_fp8, x, weight, eps, residual, h_out)
    return _ops().rms_norm_fp8(x, weight, eps, residual, h_out)


def rms_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
                      residual: torch.Tensor | None = None, dh: torch.Tensor | None = None, *,
                      stream=None):
    """Gradients (dx, dw) of :func:`rms_norm` from its inputs: dx is the gradient
    of x and of the residual alike, dh the gradient that reaches h from elsewhere."""
    if stream is not None:
        return _under(stream, rms_norm_backward, dy, x, weight, eps, residual, dh)
    return _ops().rms_norm_backward(dy, x, weight, eps, residual, dh)


class RmsNorm:
    """Autograd over :func:`rms_norm`: ``RmsNorm.apply(x, weight, eps, residual)``
    returns y, or (y, h) with a residual.  x and the residual are kept for the
    backward."""

    @staticmethod
    def apply(x, weight, eps=1e-6, residual=None):
        return _ops().rms_norm_train(x, weight, eps, residual)


def quantize_fp8(x: torch.Tensor, block: int | None = 1, t_block: int | None = None, *, stream=None):
    """x [M][K] in 8 bits, as operands of :func:`linear_fp8`: (q, scale) with one
    scale per row and 128 columns (``block`` 1, an activation) or per 128 x 128
    (``block`` 128, a weight).  ``t_block`` asks for the transpose too (or, with
    ``block`` None, alone): (q, scale, t, t_scale) with t [K][M rounded up to 16],
    padded with zeros, and its scales along M."""
    if stream is not None:
        return _under(stream, quantize_fp8, x, block, t_block)
    return _ops().quantize_fp8(x, block, t_block)


def linear_fp8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
               dtype: torch.dtype = torch.bfloat16, parts: int = 1,
               out: torch.Tensor | None = None, *, stream=None) -> torch.Tensor:
    """8-bit projection: x [M][K] (scales per row and 128 k) times w [N][K] (scales
    per 128 x 128), accumulated in fp32, as ``dtype`` [M][N].  With bfloat16 the
    matrix cores cut each product 13 binary places below the largest of its group of
    8 (1.4e-5 of the sum on normal operands, a hundredth of bfloat16's rounding); with
    float32 they keep it whole, at half the rate.  With ``parts`` the
    columns come as so many tensors, [parts][M][N / parts]: the queries, keys and
    values of a QKV projection.  K must be a multiple of 16 and N / parts of 8."""
    if stream is not None:
        return _under(stream, linear_fp8, x, x_scale, w, w_scale, dtype, parts, out)
    return _ops().linear_fp8(x, x_scale, w, w_scale, dtype, parts, out)


class Fp8Linear:
    """A projection whose three products run in 8 bits: ``Fp8Linear.apply(x, w)``
    is x [M][K] times w [N][K] in their dtype, with activations and gradients
    quantised per row and 128 of the contraction, and weights (and the activations
    of the weight's gradient) per 128 x 128.  K and N must be multiples of 16 (N of
    8 without gradients), each at most 2^20, and M too where w needs a gradient, whose
    contraction runs over the tokens.  What the backward needs is kept in 8 bits.  In
    bfloat16 the gradients' products are cut as :func:`linear_fp8` says."""

    @staticmethod
    def apply(x, w):
        return _ops().fp8_linear_train(x, w)


def rope_frequencies(pairs: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original_length: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(frequencies, magnitude) of ``pairs`` rotated pairs, scaled for contexts
    ``factor`` times longer than ``original_length``: ``scaling`` "none", "linear",
    "ntk" or "yarn" (see hcms.h, hcms_rope_frequencies).  Host only."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_SCALINGS)}")
    (pairs,), _ = _ints([pairs])
    buf = (ctypes.c_double * min(max(pairs, 1), 256))()     # more are refused below
    mag = ctypes.c_double()
    _check(load().hcms_rope_frequencies(pairs, float(base), _SCALINGS[scaling], float(factor),
                                        float(original_length), float(beta_fast), float(beta_slow), buf,
                                        ctypes.byref(mag)))
    return list(buf), mag.value


def rope_table_freqs(grid, axis_pairs, freqs, magnitude: float = 1.0, device="cuda", *,
                     stream=None) -> torch.Tensor:
    """The rotation table (see :func:`rope_table`) of given frequencies, one per
    pair, with every entry times ``magnitude``: float32 [entries][2].  ``device`` is
    the current one (that of ``stream``)."""
    if stream is not None:
        return _under(stream, rope_table_freqs, grid, axis_pairs, freqs, magnitude, device)
    device = _gpu_device(device)
    n = _table_rows(grid, axis_pairs)
    g, na = _ints(grid)
    p, _ = _ints(axis_pairs)
    freqs = [float(f) for f in freqs]
    if len(freqs) != sum(p):
        raise ValueError("one frequency per pair")
    table = torch.empty((n, 2), dtype=torch.float32, device=device)
    _check(load().hcms_rope_table_freqs(table.data_ptr(), g, p, na, (ctypes.c_double * len(freqs))(*freqs),
                                        float(magnitude), torch.cuda.current_stream().cuda_stream))
    return table


def _half(layout: str) -> bool:
    if layout not in _HALF:
        raise ValueError(f"layout must be one of {sorted(_HALF)}")
    return _HALF[layout]


def rope(q: torch.Tensor, k: torch.Tensor | None, table: torch.Tensor, grid, axis_pairs,
         positions: torch.Tensor | None = None, layout: str = "interleaved", inverse: bool = False,
         out=None, *, stream=None):
    """Rotary positions of queries q [S][H][d] and keys k [S][Hk][d] (or None), any
    strides of tokens and heads: the first 2 sum(axis_pairs) elements of each head
    turn by ``table`` (:func:`rope_table` or :func:`rope_table_freqs` of the same
    grid and axis_pairs), pairs (2p, 2p + 1) or, with layout "half", (p, p + their
    number).  ``positions``: int32 or int64 [S] (one axis) or [S][axes]; without,
    token t sits at place t of the row-major grid.  A position outside the grid
    gives NaN.  ``inverse`` turns back (the gradient's rotation).  ``out``: (q, k)
    to write to, which may be the inputs themselves.  Returns (q, k), or q."""
    if stream is not None:
        return _under(stream, rope, q, k, table, grid, axis_pairs, positions, layout, inverse, out)
    return _ops().rope(q, k, table, grid, axis_pairs, positions, _half(layout), bool(inverse), out)


class Rope:
    """Autograd over :func:`rope`: ``Rope.apply(q, k, table, grid, axis_pairs,
    positions, layout)`` returns the rotated (q, k), or q without keys."""

    @staticmethod
    def apply(q, k, table, grid, axis_pairs, positions=None, layout="interleaved"):
        return _ops().rope_train(q, k, table, grid, axis_pairs, positions, _half(layout))

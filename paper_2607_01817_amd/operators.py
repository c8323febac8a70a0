"""Operators beside the chunk loop: the root-mean-square norm, 8-bit products
and rotary positions, forward and backward (the C ABI's hcms_rms_norm*,
hcms_quantize_fp8, hcms_linear_fp8 and hcms_rope*).

8-bit tensors are ``float8_e4m3fn`` values with power-of-two scales held as
``float8_e8m0fnu``, one for each block of 128 elements of a row or of 128 x 128,
in groups of four blocks: ``[ceil(K / 512)][rows or blocks of rows][4]``.
"""
from __future__ import annotations

import contextlib
import ctypes

import torch

from . import _check, _dev, _devs, _dtype, _expect, _ints, _stream, _table_rows, load

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
SCALE_BLOCK = 128
_LAYOUTS = {"interleaved": 0, "half": 1}
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class RopeHeads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_token", ctypes.c_int64),
                ("x_head", ctypes.c_int64), ("y_token", ctypes.c_int64), ("y_head", ctypes.c_int64),
                ("heads", ctypes.c_int)]


def _on(stream):
    """Outputs and workspaces belong to the stream that the call runs on."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


def _rows(t: torch.Tensor, name: str) -> int:
    """The row stride of a 2-D tensor whose rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions (got {t.dim()})")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    M, D = t.shape
    if M > 0 and D > 1 and t.stride(1) != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    if M > 1 and t.stride(0) < D:
        raise ValueError(f"the rows of {name} overlap")
    return t.stride(0) if M > 1 else D


def _ptr(t):
    return None if t is None else t.data_ptr()


def _one_device(x: torch.Tensor, named):
    for t, n in named:
        if t is not None and t.device != x.device:
            raise ValueError(f"{n} is on {t.device}, not on {x.device}")


def _norm_args(x, weight, residual):
    ldx = _rows(x, "x")
    M, D = x.shape
    _dtype(x)
    if not isinstance(weight, torch.Tensor) or weight.shape != (D,):
        raise ValueError("weight must be [D]")
    _dtype(weight)
    _dev(weight, "weight")
    ldr = D
    if residual is not None:
        ldr = _rows(residual, "residual")
        if residual.shape != x.shape or residual.dtype != x.dtype:
            raise ValueError("residual must match x")
    _one_device(x, ((weight, "weight"), (residual, "residual")))
    return M, D, ldx, ldr


def _out(t, shape, dtype, device, name):
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    _expect(t, shape, dtype, name)
    _dev(t, name)
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, not on {device}")
    return t


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
             residual: torch.Tensor | None = None, out: torch.Tensor | None = None,
             h_out: torch.Tensor | None = None, stream=None):
    """Root-mean-square norm of rows: ``y = h / sqrt(mean(h^2) + eps) * weight``
    with ``h = x + residual``.  Returns y, or (y, h) with a residual, where h is
    the residual stream's next value.  x and residual [M][D] may have any row
    stride (a slice of a projection's output, for a norm of queries)."""
    M, D, ldx, ldr = _norm_args(x, weight, residual)
    if residual is None and h_out is not None:
        raise ValueError("h_out is given without a residual")
    with _on(stream):
        y = _out(out, (M, D), x.dtype, x.device, "out")
        h = None if residual is None else _out(h_out, (M, D), x.dtype, x.device, "h_out")
    _check(load().hcms_rms_norm(x.data_ptr(), _ptr(residual), weight.data_ptr(), y.data_ptr(), _ptr(h),
                                M, D, ldx, ldr, eps, _dtype(x), _dtype(weight), _stream(stream)))
    return y if h is None else (y, h)


def rms_norm_fp8(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
                 residual: torch.Tensor | None = None, h_out: torch.Tensor | None = None,
                 stream=None):
    """:func:`rms_norm` with y in 8 bits, as :func:`linear_fp8` reads it: returns
    (q, scale), or (q, scale, h) with a residual.  D must be a multiple of 16."""
    M, D, ldx, ldr = _norm_args(x, weight, residual)
    if residual is None and h_out is not None:
        raise ValueError("h_out is given without a residual")
    with _on(stream):
        q = torch.empty((M, D), dtype=E4M3, device=x.device)
        scale = _scales(M, D, x.device)
        h = None if residual is None else _out(h_out, (M, D), x.dtype, x.device, "h_out")
    _check(load().hcms_rms_norm_fp8(x.data_ptr(), _ptr(residual), weight.data_ptr(), q.data_ptr(),
                                    scale.data_ptr(), _ptr(h), M, D, ldx, ldr, eps, _dtype(x),
                                    _dtype(weight), _stream(stream)))
    return (q, scale) if h is None else (q, scale, h)


def rms_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6,
                      residual: torch.Tensor | None = None, dh: torch.Tensor | None = None, stream=None):
    """Gradients (dx, dw) of :func:`rms_norm` from its inputs: dx is the gradient
    of x and of the residual alike, dh the gradient that reaches h from elsewhere."""
    M, D, ldx, ldr = _norm_args(x, weight, residual)
    for t, n in ((dy, "dy"), (dh, "dh")):
        if t is not None:
            _expect(t, (M, D), x.dtype, n)
            _dev(t, n)
    _one_device(x, ((dy, "dy"), (dh, "dh")))
    lib = load()
    with _on(stream):
        dx = torch.empty((M, D), dtype=x.dtype, device=x.device)
        dw = torch.empty_like(weight)
        partial = torch.empty((_check(lib.hcms_rms_norm_partials(M, D)), D), dtype=torch.float32,
                              device=x.device)
    _check(lib.hcms_rms_norm_backward(dy.data_ptr(), x.data_ptr(), _ptr(residual), _ptr(dh),
                                      weight.data_ptr(), dx.data_ptr(), dw.data_ptr(), partial.data_ptr(),
                                      M, D, ldx, ldr, eps, _dtype(x), _dtype(weight), _stream(stream)))
    return dx, dw


class RmsNorm(torch.autograd.Function):
    """Autograd over :func:`rms_norm`: ``RmsNorm.apply(x, weight, eps, residual)``
    returns y, or (y, h) with a residual.  x and the residual are kept for the
    backward."""

    @staticmethod
    def forward(fctx, x, weight, eps=1e-6, residual=None):
        fctx.set_materialize_grads(False)
        fctx.save_for_backward(x, weight, residual)
        fctx.hcms = eps
        return rms_norm(x, weight, eps, residual)

    @staticmethod
    def backward(fctx, dy, dh=None):
        x, weight, residual = fctx.saved_tensors
        if dy is None:   # only h was used
            return dh, None, None, dh
        dx, dw = rms_norm_backward(dy.contiguous(), x, weight, fctx.hcms, residual,
                                   None if dh is None else dh.contiguous())
        return dx, dw, None, None if residual is None else dx


def _scales(rows: int, K: int, device) -> torch.Tensor:
    """Room for the scales of ``rows`` rows (or blocks of rows) of K elements."""
    return torch.empty((-(-K // (4 * SCALE_BLOCK)), rows, 4), dtype=E8M0, device=device)


def quantize_fp8(x: torch.Tensor, block: int | None = 1, t_block: int | None = None, stream=None):
    """x [M][K] in 8 bits, as operands of :func:`linear_fp8`: (q, scale) with one
    scale per row and 128 columns (``block`` 1, an activation) or per 128 x 128
    (``block`` 128, a weight).  ``t_block`` asks for the transpose too (or, with
    ``block`` None, alone): (q, scale, t, t_scale) with t [K][M rounded up to 16],
    padded with zeros, and its scales along M."""
    ldx = _rows(x, "x")
    if (block is None and t_block is None) or block not in (None, 1, SCALE_BLOCK) \
            or t_block not in (None, 1, SCALE_BLOCK):
        raise ValueError("block and t_block are 1, 128 or None, not both None")
    M, K = x.shape
    q = scale = t = t_scale = None
    with _on(stream):
        if block is not None:
            q = torch.empty((M, K), dtype=E4M3, device=x.device)
            scale = _scales(M if block == 1 else -(-M // SCALE_BLOCK), K, x.device)
        if t_block is not None:
            t = torch.empty((K, -(-M // 16) * 16), dtype=E4M3, device=x.device)
            t_scale = _scales(K if t_block == 1 else -(-K // SCALE_BLOCK), M, x.device)
    if M > 0:
        _check(load().hcms_quantize_fp8(x.data_ptr(), _ptr(q), _ptr(scale), block or 1, _ptr(t),
                                        _ptr(t_scale), t_block or 1, M, K, ldx, _dtype(x),
                                        _stream(stream)))
    if t is None:
        return q, scale
    return (t, t_scale) if q is None else (q, scale, t, t_scale)


def linear_fp8(x: torch.Tensor, x_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
               dtype: torch.dtype = torch.bfloat16, parts: int = 1, out: torch.Tensor | None = None,
               stream=None) -> torch.Tensor:
    """8-bit projection: x [M][K] (scales per row and 128 k) times w [N][K] (scales
    per 128 x 128), accumulated in fp32, as ``dtype`` [M][N].  With ``parts`` the
    columns come as so many tensors, [parts][M][N / parts]: the queries, keys and
    values of a QKV projection.  K must be a multiple of 16 and N / parts of 8."""
    if not (isinstance(x, torch.Tensor) and isinstance(w, torch.Tensor)) or x.dim() != 2 or w.dim() != 2 \
            or x.shape[1] != w.shape[1]:
        raise ValueError("x must be [M][K] and w [N][K]")
    M, K = x.shape
    N = w.shape[0]
    groups = -(-K // (4 * SCALE_BLOCK))
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype}; use bfloat16 or float32")
    parts = int(parts)
    if parts < 1 or N % (8 * parts):
        raise ValueError(f"N = {N} must be {parts} parts of a multiple of 8")
    _expect(x, (M, K), E4M3, "x")
    _expect(x_scale, (groups, M, 4), E8M0, "x_scale")
    _expect(w, (N, K), E4M3, "w")
    _expect(w_scale, (groups, -(-N // SCALE_BLOCK), 4), E8M0, "w_scale")
    _devs(((x, "x"), (x_scale, "x_scale"), (w, "w"), (w_scale, "w_scale")))
    _one_device(x, ((x_scale, "x_scale"), (w, "w"), (w_scale, "w_scale")))
    shape = (M, N) if parts == 1 else (parts, M, N // parts)
    with _on(stream):
        y = _out(out, shape, dtype, x.device, "out")
    _check(load().hcms_linear_fp8(x.data_ptr(), x_scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(),
                                  y.data_ptr(), M, N, K, parts, 0 if dtype == torch.bfloat16 else 1,
                                  _stream(stream)))
    return y


class Fp8Linear(torch.autograd.Function):
    """A projection whose three products run in 8 bits: ``Fp8Linear.apply(x, w)``
    is x [M][K] times w [N][K] in x's dtype, with activations and gradients
    quantised per row and 128 of the contraction, and weights (and the activations
    of the weight's gradient) per 128 x 128.  K, and N where x needs a gradient,
    must be multiples of 16.  What the backward needs is kept in 8 bits."""

    @staticmethod
    def forward(fctx, x, w):
        if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1] or x.dtype != w.dtype:
            raise ValueError("x must be [M][K] and w [N][K] of one dtype")
        dx, dw = fctx.needs_input_grad
        if dx and w.shape[0] % 16:
            raise ValueError(f"N = {w.shape[0]} must be a multiple of 16 for the gradient of x")
        xq, xs, *xt = quantize_fp8(x, 1, SCALE_BLOCK if dw else None)
        wq, ws, *wt = quantize_fp8(w, SCALE_BLOCK, SCALE_BLOCK if dx else None)
        fctx.save_for_backward(*(xt or (None, None)), *(wt or (None, None)))
        fctx.hcms = (x.shape[0], w.dtype)
        return linear_fp8(xq, xs, wq, ws, dtype=x.dtype)

    @staticmethod
    def backward(fctx, dy):
        xt, xts, wt, wts = fctx.saved_tensors
        M, dtype = fctx.hcms
        need_x, need_w = fctx.needs_input_grad
        dy = dy.contiguous()
        if M == 0:
            return (torch.empty((0, wt.shape[0]), dtype=dy.dtype, device=dy.device) if need_x else None,
                    torch.zeros((dy.shape[1], xt.shape[0]), dtype=dtype, device=dy.device) if need_w else None)
        got = list(quantize_fp8(dy, 1 if need_x else None, 1 if need_w else None))
        dx = linear_fp8(got[0], got[1], wt, wts, dtype=dy.dtype) if need_x else None
        dw = linear_fp8(got[-2], got[-1], xt, xts, dtype=dtype) if need_w else None
        return dx, dw


def rope_frequencies(pairs: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0,
                     original_length: float = 0.0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """(frequencies, magnitude) of ``pairs`` rotated pairs, scaled for contexts
    ``factor`` times longer than ``original_length``: ``scaling`` "none", "linear",
    "ntk" or "yarn" (see hcms.h, hcms_rope_frequencies).  Host only."""
    if scaling not in _SCALINGS:
        raise ValueError(f"scaling must be one of {sorted(_SCALINGS)}")
    buf = (ctypes.c_double * max(1, pairs))()
    mag = ctypes.c_double()
    _check(load().hcms_rope_frequencies(pairs, float(base), _SCALINGS[scaling], float(factor),
                                        float(original_length), float(beta_fast), float(beta_slow), buf,
                                        ctypes.byref(mag)))
    return list(buf), mag.value


def rope_table_freqs(grid, axis_pairs, freqs, magnitude: float = 1.0, device="cuda",
                     stream=None) -> torch.Tensor:
    """The rotation table (see :func:`rope_table`) of given frequencies, one per
    pair, with every entry times ``magnitude``: float32 [entries][2]."""
    n = _table_rows(grid, axis_pairs)
    g, na = _ints(grid)
    p, _ = _ints(axis_pairs)
    freqs = [float(f) for f in freqs]
    if len(freqs) != sum(int(x) for x in axis_pairs):
        raise ValueError("one frequency per pair")
    with _on(stream):
        table = torch.empty((n, 2), dtype=torch.float32, device=device)
    _check(load().hcms_rope_table_freqs(table.data_ptr(), g, p, na, (ctypes.c_double * len(freqs))(*freqs),
                                        float(magnitude), _stream(stream)))
    return table


def _heads(x, S, d, dtype, name):
    """Checks a side's heads [S][heads][d] and gives its token and head strides."""
    if not isinstance(x, torch.Tensor) or x.dim() != 3 or x.shape[0] != S or x.shape[2] != d or x.dtype != dtype:
        raise ValueError(f"{name} must be [S][heads][d] of one dtype")
    if not x.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    if x.numel() and d > 1 and x.stride(2) != 1:
        raise ValueError(f"the head vectors of {name} must be contiguous")
    return x.stride(0), x.stride(1)


def rope(q: torch.Tensor, k: torch.Tensor | None, table: torch.Tensor, grid, axis_pairs,
         positions: torch.Tensor | None = None, layout: str = "interleaved", inverse: bool = False,
         out=None, stream=None):
    """Rotary positions of queries q [S][H][d] and keys k [S][Hk][d] (or None), any
    strides of tokens and heads: the first 2 sum(axis_pairs) elements of each head
    turn by ``table`` (:func:`rope_table` or :func:`rope_table_freqs` of the same
    grid and axis_pairs), pairs (2p, 2p + 1) or, with layout "half", (p, p + their
    number).  ``positions``: int32 or int64 [S] (one axis) or [S][axes]; without,
    token t sits at place t of the row-major grid.  A position outside the grid
    gives NaN.  ``inverse`` turns back (the gradient's rotation).  ``out``: (q, k)
    to write to, which may be the inputs themselves.  Returns (q, k), or q."""
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be [S][heads][d]")
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
    S, _, d = q.shape
    _expect(table, (_table_rows(grid, axis_pairs), 2), torch.float32, "table")
    _dev(table, "table")
    g, na = _ints(grid)
    p, _ = _ints(axis_pairs)
    pb = 0
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
            raise TypeError("positions must be an int32 or int64 tensor")
        if tuple(positions.shape) != (S, na) and not (na == 1 and tuple(positions.shape) == (S,)):
            raise ValueError("positions must be [S] or [S][axes]")
        _dev(positions, "positions")
        pb = positions.element_size()
    if out is not None and len(out) != 2:
        raise ValueError("out must be the pair (q, k)")
    ins, outs, sides = (q, k), [], []
    _one_device(q, ((k, "k"), (table, "table"), (positions, "positions")))
    for i, (x, name) in enumerate(zip(ins, ("q", "k"))):
        if x is None:
            outs.append(None)
            sides.append(None)
            continue
        xt, xh = _heads(x, S, d, q.dtype, name)
        if out is None:
            with _on(stream):
                y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        else:
            y = out[i]
            if not isinstance(y, torch.Tensor) or y.shape != x.shape:
                raise ValueError(f"out's {name} must match {name}")
            _one_device(x, ((y, f"out's {name}"),))
        yt, yh = _heads(y, S, d, q.dtype, f"out's {name}")
        outs.append(y)
        sides.append(RopeHeads(x.data_ptr(), y.data_ptr(), xt, xh, yt, yh, x.shape[1]))
    _check(load().hcms_rope(ctypes.byref(sides[0]), None if k is None else ctypes.byref(sides[1]),
                            table.data_ptr(), g, p, na, _ptr(positions), pb, S, d, _LAYOUTS[layout],
                            int(bool(inverse)), _dtype(q), _stream(stream)))
    return outs[0] if k is None else tuple(outs)


class Rope(torch.autograd.Function):
    """Autograd over :func:`rope`: ``Rope.apply(q, k, table, grid, axis_pairs,
    positions, layout)`` returns the rotated (q, k)."""

    @staticmethod
    def forward(fctx, q, k, table, grid, axis_pairs, positions=None, layout="interleaved"):
        fctx.set_materialize_grads(False)
        fctx.save_for_backward(table, positions)
        fctx.hcms = (tuple(grid), tuple(axis_pairs), layout)
        return rope(q, k, table, grid, axis_pairs, positions, layout)

    @staticmethod
    def backward(fctx, dq, dk):
        table, positions = fctx.saved_tensors
        grid, pairs, layout = fctx.hcms
        back = {"positions": positions, "layout": layout, "inverse": True}
        dq, dk = (g if g is None or g.stride(2) == 1 else g.contiguous() for g in (dq, dk))
        if dq is not None and dk is not None:
            dq, dk = rope(dq, dk, table, grid, pairs, **back)
        else:
            dq, dk = (None if g is None else rope(g, None, table, grid, pairs, **back) for g in (dq, dk))
        return dq, dk, None, None, None, None, None

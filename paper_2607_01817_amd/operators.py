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
import functools

import torch

from . import _check, _dev, _devs, _dtype, _expect, _ints, load

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
SCALE_BLOCK = 128
_LAYOUTS = {"interleaved": 0, "half": 1}
_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3}


class RopeHeads(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("x_token", ctypes.c_int64),
                ("x_head", ctypes.c_int64), ("y_token", ctypes.c_int64), ("y_head", ctypes.c_int64),
                ("heads", ctypes.c_int)]


_NO_CONTEXT = contextlib.nullcontext()


def _on(stream):
    """Outputs and workspaces belong to the stream that the call runs on."""
    return _NO_CONTEXT if stream is None else torch.cuda.stream(stream)


def _stream(stream, x: torch.Tensor) -> int:
    """The handle of the stream to launch on, x's device being the current one."""
    if stream is not None:
        return stream.cuda_stream
    device = torch._C._cuda_getDevice()
    if x.device.index != device:
        raise ValueError(f"the tensors are on {x.device}, the current device is {device}")
    return torch._C._cuda_getCurrentRawStream(device)


def _rows(t: torch.Tensor, name: str) -> int:
    """The row stride of a 2-D tensor whose rows are contiguous."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions (got {t.dim()})")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor")
    M, D = t.shape
    if t.is_contiguous():
        return D
    if D > 1 and t.stride(1) != 1:
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


def _out(t, shape, dtype, x, name):
    """The output t, or a new one beside x."""
    if t is None:
        return x.new_empty(shape, dtype=dtype)
    _expect(t, shape, dtype, name)
    _dev(t, name)
    _one_device(x, ((t, name),))
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
        y = _out(out, (M, D), x.dtype, x, "out")
        h = None if residual is None else _out(h_out, (M, D), x.dtype, x, "h_out")
    _check(load().hcms_rms_norm(x.data_ptr(), _ptr(residual), weight.data_ptr(), y.data_ptr(), _ptr(h),
                                M, D, ldx, ldr, eps, _dtype(x), _dtype(weight), _stream(stream, x)))
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
        q = x.new_empty((M, D), dtype=E4M3)
        scale = _scales(M, D, x)
        h = None if residual is None else _out(h_out, (M, D), x.dtype, x, "h_out")
    _check(load().hcms_rms_norm_fp8(x.data_ptr(), _ptr(residual), weight.data_ptr(), q.data_ptr(),
                                    scale.data_ptr(), _ptr(h), M, D, ldx, ldr, eps, _dtype(x),
                                    _dtype(weight), _stream(stream, x)))
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
    return _norm_backward(dy, x, weight, eps, residual, dh, ldx, ldr, stream)


def _norm_backward(dy, x, weight, eps, residual, dh, ldx, ldr, stream=None):
    """The launch of :func:`rms_norm_backward` on tensors that have been checked."""
    M, D = x.shape
    lib = load()
    with _on(stream):
        dx = x.new_empty((M, D))
        dw = torch.empty_like(weight)
        partial = x.new_empty((_check(lib.hcms_rms_norm_partials(M, D)), D), dtype=torch.float32)
    _check(lib.hcms_rms_norm_backward(dy.data_ptr(), x.data_ptr(), _ptr(residual), _ptr(dh),
                                      weight.data_ptr(), dx.data_ptr(), dw.data_ptr(), partial.data_ptr(),
                                      M, D, ldx, ldr, eps, _dtype(x), _dtype(weight), _stream(stream, x)))
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
        # autograd gives gradients of the outputs' shape and type
        M, D = x.shape
        dx, dw = _norm_backward(dy.contiguous(), x, weight, fctx.hcms, residual,
                                None if dh is None else dh.contiguous(), x.stride(0) if M > 1 else D,
                                D if residual is None or M <= 1 else residual.stride(0))
        return dx, dw, None, None if residual is None else dx


def _scales(rows: int, K: int, x: torch.Tensor) -> torch.Tensor:
    """Room for the scales of ``rows`` rows (or blocks of rows) of K elements."""
    return x.new_empty((-(-K // (4 * SCALE_BLOCK)), rows, 4), dtype=E8M0)


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
    return _quantize(x, block, t_block, ldx, stream)


def _quantize(x, block, t_block, ldx, stream=None):
    """The launch of :func:`quantize_fp8` on a tensor that has been checked."""
    M, K = x.shape
    q = scale = t = t_scale = None
    with _on(stream):
        if block is not None:
            q = x.new_empty((M, K), dtype=E4M3)
            scale = _scales(M if block == 1 else -(-M // SCALE_BLOCK), K, x)
        if t_block is not None:
            t = x.new_empty((K, -(-M // 16) * 16), dtype=E4M3)
            t_scale = _scales(K if t_block == 1 else -(-K // SCALE_BLOCK), M, x)
    if M > 0:
        _check(load().hcms_quantize_fp8(x.data_ptr(), _ptr(q), _ptr(scale), block or 1, _ptr(t),
                                        _ptr(t_scale), t_block or 1, M, K, ldx, _dtype(x),
                                        _stream(stream, x)))
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
        y = _out(out, shape, dtype, x, "out")
    return _linear(x, x_scale, w, w_scale, y, parts, stream)


def _linear(x, x_scale, w, w_scale, y, parts=1, stream=None):
    """The launch of :func:`linear_fp8` on tensors that have been checked."""
    M, K = x.shape
    _check(load().hcms_linear_fp8(x.data_ptr(), x_scale.data_ptr(), w.data_ptr(), w_scale.data_ptr(),
                                  y.data_ptr(), M, w.shape[0], K, parts, _dtype(y), _stream(stream, x)))
    return y


class Fp8Linear(torch.autograd.Function):
    """A projection whose three products run in 8 bits: ``Fp8Linear.apply(x, w)``
    is x [M][K] times w [N][K] in x's dtype, with activations and gradients
    quantised per row and 128 of the contraction, and weights (and the activations
    of the weight's gradient) per 128 x 128.  K and N must be multiples of 16 (N of
    8 without gradients).  What the backward needs is kept in 8 bits."""

    @staticmethod
    def forward(fctx, x, w):
        if x.dim() != 2 or w.dim() != 2 or x.shape[1] != w.shape[1] or x.dtype != w.dtype:
            raise ValueError("x must be [M][K] and w [N][K] of one dtype")
        dx, dw = fctx.needs_input_grad
        if w.shape[0] % (16 if dx or dw else 8):
            raise ValueError(f"N = {w.shape[0]} must be a multiple of 16, or of 8 without gradients")
        _one_device(x, ((w, "w"),))
        xq, xs, *xt = quantize_fp8(x, 1, SCALE_BLOCK if dw else None)
        wq, ws, *wt = quantize_fp8(w, SCALE_BLOCK, SCALE_BLOCK if dx else None)
        fctx.save_for_backward(*(xt or (None, None)), *(wt or (None, None)))
        fctx.hcms = (x.shape[0], w.dtype)
        return _linear(xq, xs, wq, ws, x.new_empty((x.shape[0], w.shape[0])))

    @staticmethod
    def backward(fctx, dy):
        xt, xts, wt, wts = fctx.saved_tensors
        M, dtype = fctx.hcms
        need_x, need_w = fctx.needs_input_grad
        dy = dy.contiguous()
        if M == 0:
            return (torch.empty((0, wt.shape[0]), dtype=dy.dtype, device=dy.device) if need_x else None,
                    torch.zeros((dy.shape[1], xt.shape[0]), dtype=dtype, device=dy.device) if need_w else None)
        got = _quantize(dy, 1 if need_x else None, 1 if need_w else None, dy.shape[1])
        dx = dw = None
        if need_x:
            dx = _linear(got[0], got[1], wt, wts, dy.new_empty((M, wt.shape[0])))
        if need_w:
            dw = _linear(got[-2], got[-1], xt, xts, dy.new_empty((dy.shape[1], xt.shape[0]), dtype=dtype))
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


@functools.lru_cache(maxsize=256)
def _axes(grid: tuple, axis_pairs: tuple):
    """The C arrays of a grid and its pair counts, and the table's entries."""
    g, na = _ints(grid)
    p, npairs = _ints(axis_pairs)
    if na != npairs:
        raise ValueError("one pair count per grid axis")
    return g, p, na, _check(load().hcms_rope_table_entries(g, p, na))


def rope_table_freqs(grid, axis_pairs, freqs, magnitude: float = 1.0, device="cuda",
                     stream=None) -> torch.Tensor:
    """The rotation table (see :func:`rope_table`) of given frequencies, one per
    pair, with every entry times ``magnitude``: float32 [entries][2]."""
    g, p, na, n = _axes(tuple(grid), tuple(axis_pairs))
    freqs = [float(f) for f in freqs]
    if len(freqs) != sum(p):
        raise ValueError("one frequency per pair")
    with _on(stream):
        table = torch.empty((n, 2), dtype=torch.float32, device=device)
    _check(load().hcms_rope_table_freqs(table.data_ptr(), g, p, na, (ctypes.c_double * len(freqs))(*freqs),
                                        float(magnitude), _stream(stream, table)))
    return table


def _check_side(x, y, S, d, dtype, name):
    """x and y must be [S][heads][d], any strides of tokens and heads."""
    if x.shape != y.shape or x.shape[0] != S or x.shape[2] != d or not x.dtype == y.dtype == dtype:
        raise ValueError(f"{name} and its output must be [S][heads][d] of one dtype")
    if x.numel() and d > 1 and not x.stride(2) == y.stride(2) == 1:
        raise ValueError(f"the head vectors of {name} must be contiguous")


def _side(x, y):
    """A side's heads as the library takes them."""
    xs, ys = x.stride(), y.stride()
    return RopeHeads(x.data_ptr(), y.data_ptr(), xs[0], xs[1], ys[0], ys[1], x.shape[1])


def _rope(q, k, yq, yk, table, axes, positions, layout, inverse, stream=None):
    """The launch of :func:`rope` on tensors that have been checked."""
    ks = None if k is None else ctypes.byref(_side(k, yk))
    _check(load().hcms_rope(ctypes.byref(_side(q, yq)), ks, table.data_ptr(), axes[0], axes[1], axes[2],
                            _ptr(positions), 0 if positions is None else positions.element_size(),
                            q.shape[0], q.shape[2], _LAYOUTS[layout], 1 if inverse else 0, _dtype(q),
                            _stream(stream, q)))


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
    if k is not None and (not isinstance(k, torch.Tensor) or k.dim() != 3):
        raise ValueError("k must be [S][heads][d]")
    if layout not in _LAYOUTS:
        raise ValueError(f"layout must be one of {sorted(_LAYOUTS)}")
    S, _, d = q.shape
    axes = _axes(tuple(grid), tuple(axis_pairs))
    na = axes[2]
    _expect(table, (axes[3], 2), torch.float32, "table")
    if positions is not None:
        if not isinstance(positions, torch.Tensor) or positions.dtype not in (torch.int32, torch.int64):
            raise TypeError("positions must be an int32 or int64 tensor")
        if tuple(positions.shape) != (S, na) and not (na == 1 and tuple(positions.shape) == (S,)):
            raise ValueError("positions must be [S] or [S][axes]")
        _dev(positions, "positions")
    _dev(table, "table")
    if out is None:
        with _on(stream):
            yq, yk = q.new_empty(q.shape), None if k is None else k.new_empty(k.shape)
    else:
        yq, yk = out
        if not isinstance(yq, torch.Tensor) or not (k is None or isinstance(yk, torch.Tensor)):
            raise TypeError("out must be the tensors (q, k)")
    if not q.is_cuda:
        raise ValueError("q must be a GPU tensor")
    _one_device(q, ((yq, "out's q"), (k, "k"), (None if k is None else yk, "out's k"), (table, "table"),
                    (positions, "positions")))
    _check_side(q, yq, S, d, q.dtype, "q")
    if k is not None:
        _check_side(k, yk, S, d, q.dtype, "k")
    _rope(q, k, yq, yk, table, axes, positions, layout, inverse, stream)
    return yq if k is None else (yq, yk)


class Rope(torch.autograd.Function):
    """Autograd over :func:`rope`: ``Rope.apply(q, k, table, grid, axis_pairs,
    positions, layout)`` returns the rotated (q, k)."""

    @staticmethod
    def forward(fctx, q, k, table, grid, axis_pairs, positions=None, layout="interleaved"):
        fctx.set_materialize_grads(False)
        fctx.save_for_backward(table, positions)
        fctx.hcms = (_axes(tuple(grid), tuple(axis_pairs)), layout)
        return rope(q, k, table, grid, axis_pairs, positions, layout)

    @staticmethod
    def backward(fctx, dq, dk):
        # autograd gives gradients of the outputs' shapes and type
        table, positions = fctx.saved_tensors
        axes, layout = fctx.hcms
        dq, dk = (g if g is None or g.stride(2) == 1 else g.contiguous() for g in (dq, dk))
        gq, gk = (None if g is None else g.new_empty(g.shape) for g in (dq, dk))
        if dq is None and dk is not None:   # one side alone, as the queries' place
            _rope(dk, None, gk, None, table, axes, positions, layout, True)
        elif dq is not None:
            _rope(dq, dk, gq, gk, table, axes, positions, layout, True)
        return gq, gk, None, None, None, None, None

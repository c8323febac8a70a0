"""The operators beside the chunk loop on the CPU: their oracle, and what the C ABI
and the binding refuse.  No call here launches a kernel."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_01817_amd as hcms
from oracle import operators as op
from paper_2607_01817_amd.operators import RopeHeads

OK, ENULL, ESHAPE, EDTYPE, EALIGN, EARG, EALIAS = 0, -1, -2, -4, -5, -7, -8
A, B, C, D, E, F = (0x10000000 * i for i in range(1, 7))   # fake addresses, never dereferenced


@pytest.fixture(scope="module")
def lib():
    return hcms.load()


# ---------------------------------------------------------------------------
# The oracle
# ---------------------------------------------------------------------------
def test_e4m3_is_the_nearest_of_the_representable_values():
    codes = np.arange(256, dtype=np.uint8)
    grid = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    grid = np.unique(grid[np.isfinite(grid)])
    assert grid.max() == 448 and len(grid) == 253
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 4000), np.exp(rng.uniform(-9, 6, 4000)), grid,
                        (grid[1:] + grid[:-1]) / 2])
    got = op.e4m3(x)
    assert np.isin(got, grid).all()
    best = np.abs(x[:, None] - grid).min(1)
    assert (np.abs(x - got) == best).all()
    # ties: torch's cast rounds to even too
    t = torch.from_numpy(x).float()
    assert (t.double().numpy() == x).sum() > 500   # the grid and its midpoints among them
    same = t.double().numpy() == x
    assert (t.to(torch.float8_e4m3fn).double().numpy() == got)[same].all()


@pytest.mark.parametrize("amax,e", [(448.0, 0), (448.5, 1), (224.0, -1), (224.1, 0), (0.0, -126), (1e-40, -126),
                                    (3.0e38, 120), (math.inf, 128), (math.nan, 128)])
def test_scale_exponent(amax, e):
    assert op.scale_exponent(amax) == e


@pytest.mark.parametrize("rows", [1, 128])
def test_quantize_takes_each_block_by_itself(rows):
    rng = np.random.default_rng(3)
    x = rng.standard_normal((150, 300)) * np.exp2(rng.integers(-140, 120, (150, 1)))
    x[7], x[140, 299], x[3, 4] = 0, np.inf, 1e-320
    q, e = op.quantize(x, rows)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            s = slice(i * rows, (i + 1) * rows), slice(j * 128, (j + 1) * 128)
            want = op.scale_exponent(np.abs(x[s]).max())
            assert e[i, j] == want
            if want < 128:
                assert np.array_equal(q[s], op.e4m3(x[s] / 2.0 ** want))
            else:
                assert np.isnan(q[s]).all()


def test_norm_gradient_is_that_of_differences():
    rng = np.random.default_rng(1)
    x, r, dy, dh = rng.standard_normal((4, 3, 10))
    w, eps = rng.standard_normal(10), 1e-3
    dx, dw = op.rms_norm_backward(dy, x, w, eps, r, dh)

    def value(x, w):
        y, h = op.rms_norm(x, w, eps, r)
        return (y * dy).sum() + (h * dh).sum()

    s = 1e-6
    for i in np.ndindex(*x.shape):
        d = np.zeros_like(x)
        d[i] = s
        assert abs((value(x + d, w) - value(x - d, w)) / (2 * s) - dx[i]) < 1e-8
    for i in range(10):
        d = np.zeros(10)
        d[i] = s
        assert abs((value(x, w + d) - value(x, w - d)) / (2 * s) - dw[i]) < 1e-8


@pytest.mark.parametrize("scaling", ["none", "linear", "ntk", "yarn"])
@pytest.mark.parametrize("pairs", [1, 2, 21, 64, 256])
def test_rope_frequencies_match_the_oracle(lib, scaling, pairs):
    args = dict(base=10000.0, scaling=scaling, factor=8.0, original_length=4096.0)
    f, m = hcms.rope_frequencies(pairs, **args)
    want, wm = op.frequencies(pairs, **args)
    assert np.allclose(f, want, rtol=1e-13, atol=0) and abs(m - wm) < 1e-14
    assert (np.diff(f) < 0).all()


def test_scaled_frequencies_slow_the_slowest_pair_by_the_factor(lib):
    plain, _ = hcms.rope_frequencies(64)
    for scaling in ("linear", "ntk", "yarn"):
        f, m = hcms.rope_frequencies(64, scaling=scaling, factor=4.0, original_length=4096.0)
        assert abs(f[-1] * 4 / plain[-1] - 1) < 1e-12
        assert abs(f[0] / plain[0] - (0.25 if scaling == "linear" else 1)) < 1e-12
    assert abs(m - (0.1 * math.log(4) + 1)) < 1e-15


@pytest.mark.parametrize("pairs", [1, 2, 8, 21, 64, 256])
@pytest.mark.parametrize("length", [3.0, 100.0, 4096.0, 65536.0, 262144.0, 1e6, 1e9])
@pytest.mark.parametrize("fast,slow", [(32.0, 1.0), (8.0, 2.0), (4.0, 4.0)])
def test_yarn_slows_pairs_by_their_turns(lib, pairs, length, fast, slow):
    """From each pair's turns over the original length alone: kept from beta_fast on,
    slowed by the factor up to beta_slow, strictly between in between (but for the pair
    of the last whole index up to beta_fast, where the mixture starts)."""
    base, factor = 10000.0, 8.0
    got, m = hcms.rope_frequencies(pairs, base, "yarn", factor, length, fast, slow)
    want, wm = op.frequencies(pairs, base, "yarn", factor, length, fast, slow)
    assert np.allclose(got, want, rtol=1e-12, atol=0) and abs(m - wm) < 1e-14
    plain = base ** (-np.arange(pairs) / pairs)
    turns = length * plain / (2 * math.pi)
    share = np.asarray(got) / plain
    near = 1 + 1e-9
    assert np.allclose(share[turns >= fast * near], 1, rtol=1e-12, atol=0)
    assert np.allclose(share[turns * near <= slow], 1 / factor, rtol=1e-12, atol=0)
    between = (turns * near < fast) & (turns > slow * near)
    assert (share[between] > 1 / factor * near).all() and (share[between] <= 1).all()
    assert (np.diff(share) <= 1e-12).all()


def test_rotation_preserves_scores_of_equal_distance():
    rng = np.random.default_rng(2)
    q, k = rng.standard_normal((2, 1, 1, 16))
    f, _ = op.frequencies(6)
    for layout in ("interleaved", "half"):
        s = [(op.rotate(q, f[None] * a, layout=layout) * op.rotate(k, f[None] * (a + 5), layout=layout)).sum()
             for a in (0, 3, 70)]
        assert np.ptp(s) < 1e-12


# ---------------------------------------------------------------------------
# Refusals of the C ABI
# ---------------------------------------------------------------------------
def test_rms_norm_refusals(lib):
    def call(x=A, r=B, w=C, y=D, h=E, M=4, D_=64, ldx=64, ldr=64, eps=1e-6, dt=0, wdt=0):
        return lib.hcms_rms_norm(x, r, w, y, h, M, D_, ldx, ldr, eps, dt, wdt, None)

    assert call(M=0) == OK and call(M=0, x=None, y=None) == OK
    assert call(M=-1) == ESHAPE and call(D_=7) == ESHAPE and call(D_=16385, ldx=20000, ldr=20000) == ESHAPE
    assert call(ldx=63) == ESHAPE and call(ldr=63) == ESHAPE and call(ldx=-64) == ESHAPE
    assert call(dt=2) == EDTYPE and call(wdt=7) == EDTYPE
    assert call(eps=-1.0) == EARG and call(eps=math.nan) == EARG and call(eps=math.inf) == EARG
    assert call(x=None) == ENULL and call(w=None) == ENULL and call(y=None) == ENULL
    assert call(h=None) == ENULL and call(r=None) == ENULL       # residual and h together
    assert call(x=A + 1) == EALIGN and call(x=A + 2, dt=1) == EALIGN and call(w=C + 2, wdt=1) == EALIGN
    assert call(y=A) == EALIAS and call(h=B + 2) == EALIAS and call(y=E + 8) == EALIAS
    assert call(y=C - 4 * 64 * 2 + 2) == EALIAS
    assert b"overlaps" in lib.hcms_last_error()


def test_rms_norm_fp8_refusals(lib):
    def call(q=D, s=E, M=4, D_=64, h=F):
        return lib.hcms_rms_norm_fp8(A, B, C, q, s, h, M, D_, 128, 128, 1e-6, 0, 0, None)

    assert call(M=0) == OK
    assert call(D_=72) == ESHAPE and call(D_=72, M=0) == ESHAPE
    assert call(q=None) == ENULL and call(s=None) == ENULL
    assert call(q=D + 8) == EALIGN and call(s=E + 4) == EALIGN
    assert call(s=D + 16) == EALIAS and call(h=E) == EALIAS


def test_rms_norm_backward_refusals(lib):
    def call(dy=A, x=B, r=None, dh=None, w=C, dx=D, dw=E, p=F, M=4, ldx=64):
        return lib.hcms_rms_norm_backward(dy, x, r, dh, w, dx, dw, p, M, 64, ldx, 64, 1e-6, 0, 0, None)

    assert call(dw=None) == ENULL and call(p=None) == ENULL and call(x=None) == ENULL
    assert call(ldx=60) == ESHAPE and call(p=F + 2) == EALIGN
    assert call(dx=A) == EALIAS and call(dx=C) == EALIAS and call(p=E) == EALIAS and call(dh=D) == EALIAS
    assert call(r=D + 64) == EALIAS
    assert lib.hcms_rms_norm_partials(0, 64) == 0
    assert lib.hcms_rms_norm_partials(3, 4) == ESHAPE and lib.hcms_rms_norm_partials(-1, 64) == ESHAPE
    assert 1 <= lib.hcms_rms_norm_partials(1, 5120) <= 1


def test_quantize_refusals(lib):
    def call(x=A, q=B, qs=C, qb=1, t=D, ts=E, tb=128, M=40, K=64, ldx=64, dt=0):
        return lib.hcms_quantize_fp8(x, q, qs, qb, t, ts, tb, M, K, ldx, dt, None)

    assert call(M=0) == OK and call(q=None, qs=None, t=None, ts=None) == OK
    assert call(K=24) == ESHAPE and call(K=0) == ESHAPE and call(K=(1 << 20) + 16, ldx=1 << 21) == ESHAPE
    assert call(ldx=48) == ESHAPE and call(M=-1) == ESHAPE
    assert call(qb=64) == EARG and call(tb=0) == EARG and call(dt=5) == EDTYPE
    assert call(qs=None) == ENULL and call(t=None) == ENULL and call(x=None) == ENULL
    assert call(q=B + 8) == EALIGN and call(ts=E + 1) == EALIGN and call(x=A + 1) == EALIGN
    assert call(q=A) == EALIAS and call(t=B) == EALIAS and call(ts=C) == EALIAS
    assert call(ts=D + 48 * 64 - 16) == EALIAS      # t holds 48 (40 rounded up to 16) values a row


def test_linear_fp8_refusals(lib):
    def call(x=A, xs=B, w=C, ws=D, y=E, M=4, N=48, K=64, parts=1, dt=0):
        return lib.hcms_linear_fp8(x, xs, w, ws, y, M, N, K, parts, dt, None)

    assert call(M=0) == OK and call(N=0) == OK
    assert call(K=8) == ESHAPE and call(K=24) == ESHAPE and call(K=(1 << 20) + 16) == ESHAPE
    assert call(N=12) == ESHAPE and call(N=1 << 21) == ESHAPE and call(M=-1) == ESHAPE and call(N=-8) == ESHAPE
    assert call(parts=0) == ESHAPE and call(parts=4) == ESHAPE and call(N=72, parts=2) == ESHAPE
    assert call(dt=3) == EDTYPE and call(xs=None) == ENULL and call(y=None) == ENULL
    assert call(w=C + 8) == EALIGN and call(ws=D + 4) == EALIGN
    assert call(y=A) == EALIAS and call(y=D - 16) == EALIAS


def test_rope_refusals(lib):
    one = (ctypes.c_int * 1)

    def heads(x, y, xt=256, xh=64, yt=256, yh=64, n=4):
        return ctypes.byref(RopeHeads(x, y, xt, xh, yt, yh, n))

    def call(q=heads(A, B), k=None, table=C, grid=(100,), pairs=(32,), pos=None, pb=0, S=10, d=64, layout=0,
             dt=0, axes=None):
        n = len(grid)
        return lib.hcms_rope(q, k, table, (ctypes.c_int * n)(*grid), (ctypes.c_int * n)(*pairs),
                             n if axes is None else axes, pos, pb, S, d, layout, 0, dt, None)

    assert call(S=0) == OK and call(S=0, table=None) == OK and call(q=heads(None, None, n=0)) == OK
    assert call(q=None) == ENULL and call(table=None) == ENULL and call(q=heads(A, None)) == ENULL
    assert call(S=101) == ESHAPE and call(pairs=(33,)) == ESHAPE and call(d=1024) == ESHAPE
    assert call(d=1, pairs=(1,)) == ESHAPE and call(S=-1) == ESHAPE and call(q=heads(A, B, n=-1)) == ESHAPE
    assert call(axes=0) == EARG and call(axes=5) == EARG and call(layout=2) == EARG
    assert call(pos=D, pb=2) == EARG and call(pos=D) == EARG and call(pb=4) == EARG
    assert call(dt=2) == EDTYPE
    assert call(table=C + 4) == EALIGN and call(pos=D + 4, pb=8) == EALIGN and call(q=heads(A + 1, B)) == EALIGN
    assert call(q=heads(A, B, yh=32)) == ESHAPE           # output heads overlap
    assert call(q=heads(A, B, yt=128)) == ESHAPE          # output tokens overlap
    assert call(q=heads(A, B, yt=64, yh=512)) == ESHAPE   # head-major, heads shorter than the tokens
    assert call(q=heads(A, B, xt=-1)) == ESHAPE
    assert call(q=heads(A, A + 64)) == EALIAS and call(q=heads(A, C)) == EALIAS
    assert call(q=heads(A, B), k=heads(D, B + 128)) == EALIAS
    assert call(q=heads(A, B), k=heads(B, D)) == EALIAS            # q's output on k's input
    assert call(q=heads(C + 8, C + 8)) == EALIAS                   # in place over the table
    assert call(q=heads(A, A), k=heads(D, A + 64)) == EALIAS       # one in place, the other's output over it
    assert call(q=heads(A, A, yt=512)) == EALIAS                   # same address, other strides


def test_rope_in_place_refuses_heads_that_overlap(lib):
    """Sides in place (output = input, 4 heads of 64 bf16 in tokens of xt elements)
    whose heads another workgroup reads or writes.  Refused calls only: the addresses
    are no memory."""
    def call(q, k, S=10):
        def heads(x, y, t=512, n=4):
            return ctypes.byref(RopeHeads(x, y, t, 64, t, 64, n))
        one = ctypes.c_int * 1
        return lib.hcms_rope(heads(*q), heads(*k), C, one(100), one(32), 1, None, 0, S, 64, 0, 0, 0, None)

    for S in (1, 10):
        assert call((A, A), (A, A), S) == EALIAS                   # one buffer, turned twice
        assert call((A, A), (A + 3 * 128, A + 3 * 128), S) == EALIAS   # k begins at q's last head
        assert call((A, A), (A + 3 * 128 + 126, A + 3 * 128 + 126), S) == EALIAS   # by one element
        assert call((A, A), (A, D), S) == EALIAS                   # k reads what q turns in place
        assert call((A, D), (A, A), S) == EALIAS and call((A, D), (D, D), S) == EALIAS
    assert call((A, A), (A + 7 * 128, A + 7 * 128)) == EALIAS      # k's second head is the next token's first
    assert call((A, A), (A + 4 * 128, A + 4 * 128, 256)) == EALIAS   # other token strides
    assert b"overlaps" in lib.hcms_last_error()


def test_rope_table_and_frequency_refusals(lib):
    g, p = (ctypes.c_int * 1)(16), (ctypes.c_int * 1)(4)
    f = (ctypes.c_double * 4)(1, 0.5, 0.25, 0.1)
    assert lib.hcms_rope_table_freqs(None, g, p, 1, f, 1.0, None) == ENULL
    assert lib.hcms_rope_table_freqs(A, g, p, 1, None, 1.0, None) == ENULL
    assert lib.hcms_rope_table_freqs(A + 8, g, p, 1, f, 1.0, None) == EALIGN
    assert lib.hcms_rope_table_freqs(A, g, p, 1, f, math.nan, None) == EARG
    assert lib.hcms_rope_table_freqs(A, g, (ctypes.c_int * 1)(257), 1, f, 1.0, None) == ESHAPE
    assert lib.hcms_rope_table_freqs(A, g, p, 1, (ctypes.c_double * 4)(1, math.inf, 0, 0), 1.0, None) == EARG
    for kw in (dict(pairs=0), dict(pairs=257)):
        with pytest.raises(hcms.HcmsError) as e:
            hcms.rope_frequencies(**kw)
        assert e.value.status == ESHAPE
    for kw in (dict(base=1.0), dict(scaling="linear", factor=0.5), dict(scaling="yarn", factor=2.0),
               dict(scaling="yarn", factor=2.0, original_length=10, beta_fast=1, beta_slow=2)):
        with pytest.raises(hcms.HcmsError) as e:
            hcms.rope_frequencies(8, **kw)
        assert e.value.status == EARG
    with pytest.raises(ValueError):
        hcms.rope_frequencies(8, scaling="other")


# ---------------------------------------------------------------------------
# Refusals of the binding (before the library sees a pointer)
# ---------------------------------------------------------------------------
def test_binding_refuses_host_tensors_and_wrong_shapes():
    x, w = torch.zeros(4, 64), torch.zeros(64)
    with pytest.raises(ValueError, match="GPU"):
        hcms.rms_norm(x, w)
    with pytest.raises(ValueError, match="dimensions"):
        hcms.rms_norm(x[0], w)
    with pytest.raises(ValueError, match="GPU"):
        hcms.quantize_fp8(x)
    with pytest.raises(ValueError, match="GPU"):
        hcms.rope(x.view(4, 1, 64), None, torch.zeros(128, 2), [4], [32])
    with pytest.raises(ValueError, match="table"):
        hcms.rope(x.view(4, 1, 64), None, torch.zeros(127, 2), [4], [32])
    with pytest.raises(ValueError, match="layout"):
        hcms.rope(x.view(4, 1, 64), None, torch.zeros(128, 2), [4], [32], layout="other")
    q = torch.zeros(8, 64).to(hcms.E4M3)
    s = torch.zeros(1, 8, 4)
    with pytest.raises(ValueError, match="x_scale"):
        hcms.linear_fp8(q, s, q, s)
    with pytest.raises(ValueError, match="parts"):
        hcms.linear_fp8(q, s, q, s, parts=5)
    with pytest.raises(TypeError, match="dtype"):
        hcms.linear_fp8(q, s, q, s, dtype=torch.float16)


def test_rope_tables_refuse_devices_whose_memory_a_kernel_here_does_not_write(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for make in (lambda dev: hcms.rope_table([4], [2], device=dev),
                 lambda dev: hcms.rope_table_freqs([4], [2], [1.0, 0.1], device=dev)):
        for dev in ("cpu", torch.device("cpu"), None, "meta", "cuda:1", torch.device("cuda", 3)):
            with pytest.raises(ValueError, match="device"):
                make(dev)


def test_rows_and_tokens_that_span_more_than_63_bits_are_refused(lib):
    """Strides whose span wraps would pass for buffers that overlap nothing."""
    M, far = 2 ** 31 - 1, 1 << 40
    def norm(ldx, ldr, M=M):
        return lib.hcms_rms_norm(A, B, C, D, E, M, 8, ldx, ldr, 1e-6, 0, 0, None)

    assert norm(far, 8) == ESHAPE and norm(8, far) == ESHAPE and norm((1 << 29) + 1, 8, (1 << 31) - 1) == ESHAPE
    assert b"span" in lib.hcms_last_error()
    assert lib.hcms_rms_norm_backward(A, B, None, None, C, D, E, F, M, 8, far, 8, 1e-6, 0, 0, None) == ESHAPE
    assert lib.hcms_quantize_fp8(A, B, C, 1, None, None, 1, M, 16, far, 0, None) == ESHAPE
    one = ctypes.c_int * 1
    for xt, yt in ((far, 64), (64, far)):
        q = RopeHeads(A, B, xt, 64, yt, 64, 1)
        assert lib.hcms_rope(ctypes.byref(q), None, C, one(100), one(1), 1, D, 4, M, 64, 0, 0, 0, None) == ESHAPE
        assert b"span" in lib.hcms_last_error()


def test_linear_fp8_refuses_rows_whose_last_tile_passes_32_bits(lib):
    for M in (2 ** 31 - 1, 2 ** 31 - 255):
        assert lib.hcms_linear_fp8(A, B, C, D, E, M, 8, 16, 1, 0, None) == ESHAPE


def test_sizes_past_32_bits_are_refused_and_not_wrapped(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="32 bits"):
        hcms.rope_table([2 ** 32 + 4], [2])
    with pytest.raises(ValueError, match="32 bits"):
        hcms.rope_table_freqs([4], [2 ** 32 + 2], [1.0, 0.1])
    with pytest.raises(ValueError, match="32 bits"):
        hcms.rope_frequencies(2 ** 32 + 8)
    with pytest.raises(hcms.HcmsError) as e:
        hcms.rope_frequencies(2 ** 31 - 1)     # 16 GiB of frequencies
    assert e.value.status == ESHAPE

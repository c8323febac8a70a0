"""The paged 4-bit cache and the head vectors' norm and rotation on the CPU: their oracle,
and what the C ABI and the binding refuse.  No call here launches a kernel."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2607_01817_amd as hcms
from oracle import cache as oc
from paper_2607_01817_amd.operators import KvBatch, KvCachePointers, KvRows, RopeHeads
from tests.cache_util import Batch

OK, ENULL, ESHAPE, EDTYPE, EALIGN, EARG, EALIAS = 0, -1, -2, -4, -5, -7, -8
A, B, C, D, E, F, G, H, I, J, K, L = (0x10000000 * i for i in range(1, 13))   # fake addresses, never dereferenced


@pytest.fixture(scope="module")
def lib():
    return hcms.load()


# ---------------------------------------------------------------------------
# The oracle
# ---------------------------------------------------------------------------
def test_e2m1_is_the_nearest_with_ties_to_even():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-6, 6, 5000), oc.GRID, -oc.GRID])
    got = oc.values(oc.e2m1(x)[:, None].repeat(32, 1), np.zeros((len(x), 1), int))[:, 0]
    full = np.concatenate([oc.GRID, -oc.GRID])
    assert (np.abs(got - x) == np.abs(x[:, None] - full).min(1)).all()
    mid = (oc.GRID[1:] + oc.GRID[:-1]) / 2
    assert oc.e2m1(mid).tolist() == [0, 2, 2, 4, 4, 6, 6] and oc.e2m1(-mid).tolist() == [8, 10, 10, 12, 12, 14, 14]


@pytest.mark.parametrize("amax,e", [(6.0, 0), (6.01, 1), (3.0, -1), (3.01, 0), (0.0, -126), (1e-40, -126), (3.0e38, 126),
                                    (math.inf, 128), (math.nan, 128)])
def test_scale_exponent(amax, e):
    assert oc.scale_exponent(amax) == e


@pytest.mark.parametrize("page", [64, 192])
def test_the_cache_s_layout_holds_what_is_stored(page):
    b = Batch((200, 3), (200, 70), 2, 64, page, seed=1)
    rng = np.random.default_rng(2)
    k, v = rng.standard_normal((2, b.T, 2, 64))
    old = b.read(1)
    b.store(k, v)
    for s, (first, n) in enumerate(((0, 200), (200, 3))):
        got = b.read(s)
        for x, y, was in zip(got, (k, v), old):
            assert np.array_equal(x[-n:], oc.held(y[first:first + n]))
            if s:
                assert np.array_equal(x[:-n], was[:-n])
    t = np.arange(64)
    assert sorted(oc.key_scale_place(t)) == sorted(oc.value_place(t)) == t.tolist()


def test_head_norm_gradient_is_that_of_differences():
    rng = np.random.default_rng(1)
    x, dy = rng.standard_normal((2, 3, 2, 8))
    w, z = rng.standard_normal(8), 1.3 * np.exp(1j * rng.uniform(0, 6, (3, 3)))
    for layout in ("half", "interleaved"):
        dx, dw = oc.head_norm_backward(dy, x, w, 1e-3, z, layout)

        def value(x, w):
            return (oc.head_norm(x, w, 1e-3, z, layout) * dy).sum()

        for var, grad in ((x, dx), (w, dw)):
            for i in np.ndindex(*var.shape):
                d = np.zeros_like(var)
                d[i] = 1e-6
                up, down = (value(x + s * d, w) if var is x else value(x, w + s * d) for s in (1, -1))
                assert abs((up - down) / 2e-6 - grad[i]) < 1e-8


def test_attention_sees_its_window():
    for causal, window in ((True, 0), (True, 3), (False, 4), (False, 0)):
        begin, end = oc.sees(3, 5, causal, window)
        assert end.tolist() == ([3, 4, 5] if causal else [5, 5, 5])
        assert begin.tolist() == [max(0, e - window) if window else 0 for e in end]
    assert oc.sees(3, 1, True, 2)[1].tolist() == [0, 0, 1]


# ---------------------------------------------------------------------------
# Refusals of the C ABI
# ---------------------------------------------------------------------------
def _heads(x, y, xt=256, xh=64, yt=256, yh=64, n=4):
    return ctypes.byref(RopeHeads(x, y, xt, xh, yt, yh, n))


def _ints(*v):
    return (ctypes.c_int * len(v))(*v)


def test_qk_norm_rope_refusals(lib):
    def call(q=_heads(A, B), k=_heads(C, D), qw=E, kw=F, table=G, grid=(100,), pairs=(32,), pos=None, pb=0, S=10, d=64,
             layout=0, eps=1e-6, dt=0, wdt=0):
        return lib.hcms_qk_norm_rope(q, k, qw, kw, table, _ints(*grid), _ints(*pairs), len(grid), pos, pb, S, d, layout,
                                     eps, dt, wdt, None)

    assert call(S=0) == OK and call(S=0, table=None, qw=None) == OK
    assert call(q=_heads(None, None, n=0), k=None, qw=None, kw=None) == OK
    assert call(q=None) == ENULL and call(table=None) == ENULL and call(qw=None) == ENULL and call(kw=None) == ENULL
    assert call(S=101) == ESHAPE and call(pairs=(33,)) == ESHAPE and call(d=514) == ESHAPE and call(S=-1) == ESHAPE
    assert call(layout=2) == EARG and call(eps=-1.0) == EARG and call(eps=math.nan) == EARG and call(pos=H, pb=2) == EARG
    assert call(dt=2) == EDTYPE and call(wdt=9) == EDTYPE
    assert call(table=G + 4) == EALIGN and call(qw=E + 1) == EALIGN and call(kw=F + 2, wdt=1) == EALIGN
    assert call(q=_heads(A + 1, B)) == EALIGN and call(pos=H + 2, pb=4) == EALIGN
    assert call(q=_heads(A, B, yh=32)) == ESHAPE and call(q=_heads(A, B, yt=128)) == ESHAPE
    assert call(q=_heads(A, A + 64)) == EALIAS and call(q=_heads(A, E)) == EALIAS and call(k=_heads(C, F - 64)) == EALIAS
    assert call(k=_heads(C, A)) == EALIAS and call(k=_heads(C, B + 128)) == EALIAS and call(q=_heads(A, G)) == EALIAS
    assert call(q=_heads(A, A), k=_heads(A, A)) == EALIAS                   # one buffer, twice in place


def test_qk_norm_rope_backward_refusals(lib):
    def call(dq=_heads(A, B), dk=_heads(C, D), q=_heads(E, None), k=_heads(F, None), qw=G, kw=H, dqw=I, dkw=J, p=K, table=L,
             S=10, d=64, eps=1e-6, dt=0, wdt=0):
        return lib.hcms_qk_norm_rope_backward(dq, dk, q, k, qw, kw, dqw, dkw, p, table, _ints(100), _ints(32), 1, None, 0,
                                              S, d, 0, eps, dt, wdt, None)

    none = _heads(None, None, n=0)
    assert call(dq=none, dk=none, q=none, k=none, dqw=None, dkw=None, qw=None, kw=None, p=None) == OK
    assert call(dq=None) == ENULL and call(q=None) == ENULL and call(dk=None) == ENULL and call(k=None) == ENULL
    assert call(p=None) == ENULL and call(qw=None) == ENULL and call(q=_heads(None, None)) == ENULL
    assert call(q=_heads(E, None, n=3)) == ESHAPE and call(q=_heads(E, None, xt=-1)) == ESHAPE
    assert call(q=_heads(E + 1, None)) == EALIGN and call(p=K + 2) == EALIGN and call(dqw=I + 1) == EALIGN
    assert call(eps=math.inf) == EARG and call(dt=5) == EDTYPE and call(wdt=5) == EDTYPE
    assert call(dq=_heads(A, E)) == EALIAS and call(dk=_heads(C, E + 64)) == EALIAS      # a gradient over an input
    assert call(dqw=G) == EALIAS and call(dqw=J) == EALIAS and call(p=L) == EALIAS and call(p=E) == EALIAS
    assert call(p=A) == EALIAS and call(p=B + 128) == EALIAS and call(dkw=D) == EALIAS and call(dq=_heads(A, H)) == EALIAS
    assert lib.hcms_qk_norm_rope_partials(-1, 4) == ESHAPE and lib.hcms_qk_norm_rope_partials(4, -1) == ESHAPE
    assert lib.hcms_qk_norm_rope_partials(0, 4) == 0 and 0 < lib.hcms_qk_norm_rope_partials(1, 2) <= 2


def _cache(k=A, v=B, ks=C, vs=D, pages=10, heads=2, d=64, page=64):
    return ctypes.byref(KvCachePointers(k, v, ks, vs, pages, heads, d, page))


def _batch(pages=E, lengths=F, starts=G, B=3, W=2):
    return ctypes.byref(KvBatch(pages, lengths, starts, B, W))


def _rows(x, token=128, head=64):
    return ctypes.byref(KvRows(x, token, head))


def test_append_kv_refusals(lib):
    def call(cache=_cache(), batch=_batch(), k=_rows(H), v=_rows(I), hk=J, hv=K, T=5, table=L, grid=(100,), pairs=(32,),
             pos=None, pb=0, layout=0, dt=0):
        return lib.hcms_append_kv(cache, batch, k, v, hk, hv, T, table, _ints(*grid), _ints(*pairs), len(grid), pos, pb,
                                  layout, dt, None)

    assert call(T=0) == OK and call(batch=_batch(B=0)) == OK and call(T=0, cache=_cache(k=None), k=_rows(None)) == OK
    assert call(cache=None) == ENULL and call(batch=None) == ENULL and call(k=None) == ENULL
    for c in (_cache(k=None), _cache(v=None), _cache(ks=None), _cache(vs=None)):
        assert call(cache=c) == ENULL
    for b in (_batch(pages=None), _batch(lengths=None), _batch(starts=None)):
        assert call(batch=b) == ENULL
    assert call(k=_rows(None)) == ENULL and call(hk=None) == ENULL and call(hv=None) == ENULL
    assert call(table=None, pos=E, pb=4) == ENULL
    for c in (_cache(d=96), _cache(d=0), _cache(page=32), _cache(page=96), _cache(page=0), _cache(pages=0), _cache(heads=0),
              _cache(heads=(1 << 15) + 1), _cache(page=1 << 21)):
        assert call(cache=c) == ESHAPE
    assert call(T=-1) == ESHAPE and call(batch=_batch(B=-1)) == ESHAPE and call(batch=_batch(W=0)) == ESHAPE
    assert call(T=(1 << 22) + 1) == ESHAPE and call(batch=_batch(B=1 << 21)) == ESHAPE
    assert call(batch=_batch(W=1 << 25)) == ESHAPE and call(cache=_cache(page=1 << 20), batch=_batch(W=2048)) == ESHAPE
    assert call(pairs=(33,)) == ESHAPE and call(k=_rows(H, token=-1)) == ESHAPE and call(v=_rows(I, head=1 << 41)) == ESHAPE
    assert call(layout=3) == EARG and call(pos=E, pb=2) == EARG and call(pb=4) == EARG and call(dt=2) == EDTYPE
    assert call(cache=_cache(k=A + 8)) == EALIGN and call(cache=_cache(vs=D + 4)) == EALIGN
    assert call(batch=_batch(starts=G + 2)) == EALIGN and call(k=_rows(H + 1)) == EALIGN and call(hk=J + 1) == EALIGN
    assert call(table=L + 4) == EALIGN and call(pos=0xF0000004, pb=8) == EALIGN
    assert call(hk=H) == EALIAS and call(hk=K) == EALIAS and call(k=_rows(A + 64)) == EALIAS and call(hv=E) == EALIAS
    assert call(cache=_cache(v=A + 16)) == EALIAS and call(cache=_cache(ks=F)) == EALIAS and call(table=D + 64) == EALIAS


def test_cache_attention_refusals(lib):
    def call(cache=_cache(), batch=_batch(), q=_rows(H), out=I, ws=J, T=5, heads=4, scale=0.1, window=0, dt=0):
        return lib.hcms_cache_attention(cache, batch, q, out, ws, T, heads, scale, 1, window, dt, None)

    assert call(T=0) == OK and call(batch=_batch(B=0)) == OK and call(heads=0) == OK
    assert call(q=None) == ENULL and call(q=_rows(None)) == ENULL and call(out=None) == ENULL and call(cache=None) == ENULL
    assert call(heads=3) == ESHAPE and call(heads=-2) == ESHAPE and call(T=1 << 21, heads=512) == ESHAPE
    assert call(batch=_batch(B=1 << 20), cache=_cache(heads=4)) == ESHAPE
    assert call(cache=_cache(d=32)) == ESHAPE and call(batch=_batch(W=0)) == ESHAPE
    assert call(scale=math.nan) == EARG and call(scale=math.inf) == EARG and call(window=-1) == EARG and call(dt=3) == EDTYPE
    assert call(q=_rows(H + 1)) == EALIGN and call(out=I + 1) == EALIGN and call(ws=J + 4) == EALIGN
    assert call(out=H) == EALIAS and call(out=A + 32) == EALIAS and call(out=G) == EALIAS
    far = _batch(W=1000)                                     # long enough to be split
    n = ctypes.c_int64()
    assert lib.hcms_cache_attention_workspace(_cache(), far, 5, 4, 0, 0, ctypes.byref(n)) == OK and n.value > 0
    assert call(batch=far, ws=None) == ENULL and call(batch=far, ws=I) == EALIAS and call(batch=far, ws=H - 16) == EALIAS
    assert lib.hcms_cache_attention_workspace(_cache(), far, 5, 4, 0, 0, None) == ENULL
    assert lib.hcms_cache_attention_workspace(_cache(), far, 5, 3, 0, 0, ctypes.byref(n)) == ESHAPE
    assert lib.hcms_cache_attention_workspace(_cache(), far, 5, 4, -1, 0, ctypes.byref(n)) == EARG
    assert lib.hcms_cache_attention_workspace(_cache(), _batch(W=1), 5, 4, 0, 0, ctypes.byref(n)) == OK and n.value == 0


def test_rows_that_span_more_than_63_bits_are_refused(lib):
    far = _rows(H, token=1 << 40)
    assert lib.hcms_cache_attention(_cache(), _batch(), far, I, J, 1 << 21, 2, 0.1, 0, 0, 0, None) == ESHAPE
    assert b"span" in lib.hcms_last_error()


def test_heads_that_span_more_than_63_bits_are_refused(lib):
    def call(T, heads, token, head, n):
        return lib.hcms_cache_attention(_cache(heads=n), _batch(), _rows(H, token=token, head=head), I, J, T, heads, 0.1, 0, 0,
                                        0, None)

    for args in ((1, 1 << 28, 64, 1 << 40, 2), (1, 1 << 29, 0, 1 << 33, 1), (1 << 20, 4, 1 << 40, 1 << 40, 2),
                 (2, (1 << 20) + 2, 1 << 40, 1 << 40, 2)):
        assert call(*args) == ESHAPE and b"span" in lib.hcms_last_error(), args
    assert call(1, (1 << 20) + 1, 64, 1 << 40, 1) == EALIAS      # 2^60 to the last head: over the cache


def test_caches_whose_bytes_pass_63_bits_are_refused(lib):
    n = ctypes.c_int64()
    for c in (_cache(pages=(1 << 31) - 1, heads=1 << 15, page=1 << 20), _cache(pages=1 << 30, heads=1 << 13, page=64)):
        assert lib.hcms_cache_attention(c, _batch(), _rows(H), I, J, 5, 1 << 15, 0.1, 0, 0, 0, None) == ESHAPE
        assert b"together" in lib.hcms_last_error()
        assert lib.hcms_cache_attention_workspace(c, _batch(), 5, 1 << 15, 0, 0, ctypes.byref(n)) == ESHAPE
        assert lib.hcms_append_kv(c, _batch(), _rows(H), _rows(I), None, None, 5, None, None, None, 0, None, 0, 0, 0,
                                  None) == ESHAPE


# ---------------------------------------------------------------------------
# Refusals of the binding
# ---------------------------------------------------------------------------
def _host_cache(pages=2, heads=2, d=64, page=64):
    def z(*s, dtype=torch.uint8):
        return torch.zeros((pages, heads) + s, dtype=torch.uint8).view(dtype)
    n = page // 64
    return hcms.KvCache(z(page, d // 2), z(n, d // 2, 64), z(n, d // 32, 64, dtype=hcms.E8M0), z(n, d // 32, 64, dtype=hcms.E8M0))


def test_binding_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(3, 2, 64)
    ints = [torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)]
    c = _host_cache()
    with pytest.raises(ValueError, match="GPU"):
        hcms.append_kv(x, x, c, *ints)
    with pytest.raises(ValueError, match="GPU"):
        hcms.cache_attention(x, c, *ints)
    with pytest.raises(ValueError, match="heads"):
        hcms.cache_attention(x[0], c, *ints)
    with pytest.raises(ValueError, match="contiguous"):
        hcms.cache_attention(x.transpose(1, 2), c, *ints)
    with pytest.raises(ValueError, match="layout"):
        hcms.append_kv(x, x, c, *ints, layout="other")
    with pytest.raises(ValueError, match="grid"):
        hcms.append_kv(x, x, c, *ints, table=torch.zeros(4, 2))
    w = torch.ones(64)
    with pytest.raises(ValueError, match="GPU"):
        hcms.qk_norm_rope(x, None, w, None, torch.zeros(96, 2), [3], [32])
    with pytest.raises(ValueError, match="table"):
        hcms.qk_norm_rope(x, None, w, None, torch.zeros(95, 2), [3], [32])
    with pytest.raises(ValueError, match="layout"):
        hcms.QkNormRope.apply(x, None, w, None, torch.zeros(96, 2), [3], [32], None, "other")


def test_kv_cache_refuses_other_sizes_and_devices(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    for bad in ((0, 1, 64), (1, 0, 64), (1, 1, 96), (1, 1, 64, 32), (1, 1, 64, 100)):
        with pytest.raises(ValueError, match="page"):
            hcms.kv_cache(*bad)
    with pytest.raises(ValueError, match="device"):
        hcms.kv_cache(1, 1, 64, device="cpu")
    with pytest.raises(ValueError, match="32 bits"):
        hcms.kv_cache(1 << 32, 1, 64)

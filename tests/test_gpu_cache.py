"""The paged 4-bit cache on the GPU: the append and the attention over it, against the
float64 oracle of ``oracle/cache.py``.

Tolerances, from the arithmetic, with A = sum of p |v| / sum of p of an output element:
  * append: codes, scales and held values equal to the oracle's (rotations in fp64);
  * attention: a score is a sum of d exact products (fp32: of 3 d, of parts of them) in
    fp32, within (3 d + 4) 2^-24 of the row's largest sum of |q k|, times the scale; exp's
    argument and value add 2^-21; each doubles where numerator and denominator both have
    it.  P in bf16 is within 2^-8 of itself (fp32: exact in three parts).  The sums over L
    tokens add one rounding a step of 32 tokens and lanes, of at most L / 16 + 64 steps.
    Numbers below 2^-126 may count as 0 in fp32 and bf16: of a probability (relative to
    one of 1 at least in the sum), of its parts, and of their products, 2^-124 (|v| + 1) a
    token together.  Then the rounding of the output.
"""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.cache_util import Batch, numpy_of, same_values
from tests.gpu_util import bits, log

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32
ROUND = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}


def _f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _randn(seed, *shape, dtype=FP32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


# ---------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------
# rows, lengths, heads, d, page: one token; ragged batches, some empty; whole chunks, and
# chunks that begin or end inside; pages that end inside a run; many sequences.
APPENDS = [((1,), (1,), 1, 64, 64), ((1,), (1000,), 8, 128, 64), ((64,), (64,), 2, 128, 64), ((70,), (200,), 1, 64, 64),
           ((0, 5, 0, 130, 1), (0, 5, 77, 131, 64), 3, 64, 128), ((200, 3), (513, 3), 2, 128, 192),
           ((1,) * 70, tuple(range(1, 71)), 1, 64, 64), ((0, 0), (10, 0), 1, 128, 64)]


def _append_case(hcms, rows, lengths, heads, d, page, dtype, layout, grid, pairs, seed=1):
    b = Batch(rows, lengths, heads, d, page, seed)
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(b.T, 3 * heads * d, generator=g)
    x *= torch.exp2(torch.randint(-6, 6, x.shape, generator=g).float())     # blocks of many sizes
    if b.T > 2:
        x[1, :32], x[2, heads * d:heads * d + 40] = 0, 0
    x = x.to(dtype)
    k, v = x[:, :heads * d].unflatten(1, (heads, d)), x[:, heads * d:2 * heads * d].unflatten(1, (heads, d))
    table = hcms.rope_table(list(grid), list(pairs)) if grid else None
    K = _f64(k)
    if grid and b.T:
        K = oc.turn(K, oc.factors(_f64(table), grid, pairs, oc.coordinates(grid, [p for _, p in b.places()])), layout)
    return b, x, k, v, K, _f64(v), table


def _views(x, heads, d):
    return x[:, :heads * d].unflatten(1, (heads, d)), x[:, heads * d:2 * heads * d].unflatten(1, (heads, d))


@pytest.mark.parametrize("rows,lengths,heads,d,page", APPENDS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("layout,grid,part", [("half", (2048,), 1), ("interleaved", (11, 12, 16), 1), ("half", (2048,), 0.3),
                                              ("interleaved", (2048,), 0.3), ("half", None, 0)])
def test_append(hcms, rows, lengths, heads, d, page, dtype, layout, grid, part):
    pairs = None
    if grid:
        n = max(len(grid), int(d // 2 * part))
        pairs = [n // len(grid) + (a < n % len(grid)) for a in range(len(grid))]
    log(f"[append] rows={rows} lengths={lengths} heads={heads} d={d} page={page} {dtype} {layout} pairs={pairs}")
    b, x, k, v, K, V, table = _append_case(hcms, rows, lengths, heads, d, page, dtype, layout, grid, pairs)
    cache, *batch = b.gpu(hcms)
    gk, gv = _views(x.cuda(), heads, d)
    held = hcms.append_kv(gk, gv, cache, *batch, table=table, grid=grid, axis_pairs=pairs, layout=layout, held=True)
    b.store(K, V)
    got = numpy_of(cache)
    for name, a, w in zip(("k_scale", "v_scale"), got[2:], b.cache[2:]):
        assert np.array_equal(a, w), name
    for name, a, w in zip("kv", got[:2], b.cache[:2]):
        assert same_values(a, w), name
    for name, a, w in zip("kv", held, (K, V)):
        want = torch.from_numpy(oc.held(w)).to(dtype).double().numpy() if b.T else w   # exact in bf16 too
        assert np.array_equal(_f64(a), want), name
    # without the held values: the same cache
    other, *batch = b.gpu(hcms)
    assert hcms.append_kv(gk, gv, other, *batch, table=table, grid=grid, axis_pairs=pairs, layout=layout) is None
    for a, w in zip(numpy_of(other), got):
        assert np.array_equal(a, w)


def test_every_code_and_tie(hcms):
    """Values on and next to each border of two codes, in blocks of every scale."""
    edges = np.array([0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    near = np.concatenate([edges, np.nextafter(edges.astype(np.float32), 9, dtype=np.float32),
                           np.nextafter(edges.astype(np.float32), -9, dtype=np.float32)])[:25].clip(-6, 6)
    row = np.concatenate([near, -near, [6.0] * 14])[:64].astype(np.float32)
    row[31] = row[63] = 6.0
    exps = [-127, -126, -60, -1, 0, 1, 60, 124]
    x = np.stack([np.ldexp(row, e) for e in exps])
    x = np.concatenate([x, np.ldexp(np.where(np.arange(64) % 32 == 5, 3.4e38 / 2 ** 127, 0), 127)[None].astype(np.float32),
                        np.full((1, 64), 1e-45, np.float32)])
    b = Batch((len(x),), (len(x),), 1, 64)
    cache, *batch = b.gpu(hcms)
    t = torch.from_numpy(x)[:, None].cuda()
    hk, hv = hcms.append_kv(t, t, cache, *batch, held=True)
    b.store(_f64(t), _f64(t))
    got = numpy_of(cache)
    assert np.array_equal(got[2], b.cache[2]) and np.array_equal(got[3], b.cache[3])
    assert same_values(got[0], b.cache[0]) and same_values(got[1], b.cache[1])
    with np.errstate(over="ignore"):
        want = oc.held(_f64(t)).astype(np.float32)
    for h in (hk, hv):
        assert np.array_equal(h.cpu().numpy(), want)


@pytest.mark.parametrize("layout,pairs", [("interleaved", 32), ("half", 32), ("interleaved", 27), ("half", 24), ("half", 12)])
def test_turned_keys_next_to_borders(hcms, layout, pairs):
    """Keys that the rotation moves off a border of two codes, or of two scales, by less
    than fp32 can hold, to either side: cos 1 and sin +-2^-28 on edges of at least 0.25,
    whose half steps are 2^-26 at least."""
    edges = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    exps = [-126, -100, 0, 60, 123]
    rows = []
    for e in exps:
        for top in (4.0, 6.0):                     # blocks whose largest value is a code, or the border itself
            for sign in (1.0, -1.0):
                first = np.where(edges[np.arange(pairs) % 8] > top, 3.5, edges[np.arange(pairs) % 8])
                second = sign * np.where(np.arange(pairs) % 2, 1.0, -1.0)
                x = np.zeros(64)
                at = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if layout == "interleaved" else (
                    slice(0, pairs), slice(pairs, 2 * pairs))
                x[at[0]], x[at[1]] = first, second
                rows.append(np.ldexp(x, e))
    x = np.stack(rows).astype(np.float32)
    assert np.array_equal(x.astype(np.float64), np.stack(rows))
    n = len(x)
    table = torch.zeros(n * pairs, 2)
    table[:, 0] = 1.0
    table[:, 1] = 2.0 ** -28 * (1 - 2 * (torch.arange(n * pairs) // 3 % 2)).float()
    b = Batch((n,), (n,), 1, 64)
    cache, *batch = b.gpu(hcms)
    t = torch.from_numpy(x)[:, None].cuda()
    hcms.append_kv(t, t, cache, *batch, table=table.cuda(), grid=[n], axis_pairs=[pairs], layout=layout)
    z = oc.factors(_f64(table), [n], [pairs], np.arange(n)[:, None])
    b.store(oc.turn(_f64(t), z, layout), _f64(t))
    got = numpy_of(cache)
    assert np.array_equal(got[2], b.cache[2]) and np.array_equal(got[3], b.cache[3])
    assert same_values(got[0], b.cache[0]) and same_values(got[1], b.cache[1])


def test_appended_blocks_that_are_not_finite(hcms):
    b = Batch((3,), (3,), 1, 128)
    cache, *batch = b.gpu(hcms)
    k, v = _randn(1, 3, 1, 128), _randn(2, 3, 1, 128)
    k[0, 0, 40], k[1, 0, 3], v[2, 0, 127] = float("nan"), float("inf"), -float("inf")
    hk, hv = hcms.append_kv(k.cuda(), v.cuda(), cache, *batch, held=True)
    got = numpy_of(cache)
    assert got[2][b.page_table[0, 0], 0, 0, 1, oc.key_scale_place(0)] == 255
    assert got[2][b.page_table[0, 0], 0, 0, 0, oc.key_scale_place(1)] == 255
    assert got[3][b.page_table[0, 0], 0, 0, 3, oc.value_place(2)] == 255
    hk, hv = hk.cpu(), hv.cpu()
    assert hk[0, 0, 32:64].isnan().all() and hk[1, 0, :32].isnan().all() and hv[2, 0, 96:].isnan().all()
    assert hk.isnan().sum() == 64 and hv.isnan().sum() == 32


def test_append_at_positions(hcms):
    heads, d, grid, pairs = 2, 128, (9, 40, 40), (22, 21, 21)
    for kind in (torch.int32, torch.int64):
        b = Batch((5, 20), (40, 90), heads, d, seed=3)
        rng = np.random.default_rng(1)
        at = np.stack([rng.integers(0, g, b.T) for g in grid], 1)
        at[7, 1] = 40                                                     # outside the grid
        k, v = _randn(4, b.T, heads, d, dtype=BF16), _randn(5, b.T, heads, d, dtype=BF16)
        table = hcms.rope_table(list(grid), list(pairs))
        cache, *batch = b.gpu(hcms)
        hk, hv = hcms.append_kv(k.cuda(), v.cuda(), cache, *batch, table=table, grid=grid, axis_pairs=pairs,
                                positions=torch.from_numpy(at).to(kind).cuda(), held=True)
        want = oc.held(oc.turn(_f64(k), oc.factors(_f64(table), grid, pairs, at)))
        ok = np.arange(b.T) != 7
        assert np.array_equal(_f64(hk)[ok], want[ok]) and np.isnan(_f64(hk)[7]).all()
        assert np.array_equal(_f64(hv), oc.held(_f64(v)))


def test_append_leaves_what_is_not_the_batch_s(hcms):
    """Rows behind the last sequence, pages that there are not, more rows than tokens,
    a sequence past its pages: nothing but tokens with a place is written."""
    heads, d = 2, 64
    b = Batch((3, 2, 4, 6), (10, 70, 2, 130), heads, d, seed=5, width=2)
    b.page_table[1, 1] = b.pages          # the second sequence's last page is none
    b.page_table[3, :2] = b.page_table[3, :2]
    b.W, b.page_table = 2, np.ascontiguousarray(b.page_table[:, :2])      # 128 of the fourth's 130 tokens have room
    before = [x.copy() for x in b.cache]
    k, v = _randn(1, b.T + 4, heads, d), _randn(2, b.T + 4, heads, d)
    cache, *batch = b.gpu(hcms)
    hcms.append_kv(k.cuda(), v.cuda(), cache, *batch, held=True)
    b.store(_f64(k), _f64(v))
    got = numpy_of(cache)
    for a, w, old in zip(got, b.cache, before):
        assert same_values(a, w) and not np.array_equal(a, old)


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
def _check(got, q, b, dtype, scale, causal, window, what, lost=()):
    got, Q, d = _f64(got), _f64(q), q.shape[2]
    for s in range(len(b.rows)):
        a, e = b.starts[s], b.starts[s + 1]
        if a == e or s in lost:
            continue
        K, V = b.read(s)
        want, A, most = oc.attention(Q[a:e], K, V, scale, causal, window)
        score = abs(scale) * (3 * d + 4) * 2.0 ** -24 * most + 2.0 ** -21
        bound = ROUND[dtype] * np.abs(want) + A * ((2.0 ** -8 if dtype == BF16 else 0) + 2 * score[..., None] +
                                                   (b.lengths[s] / 16 + 64) * 2.0 ** -24) * (1 + 2.0 ** -7) + \
            b.lengths[s] * 2.0 ** -124 * (np.abs(V).max(initial=0) + 1)
        assert np.isfinite(got[a:e]).all(), (what, s)
        worst = float((np.abs(got[a:e] - want) / np.maximum(bound, 1e-300)).max())
        log(f"    {what} sequence {s}: worst error {worst:.3f} of its bound")
        assert worst <= 1.0, (what, s, worst)


# rows, lengths, key heads, queries a key head, d, page
ATTENDS = [((1,), (1,), 1, 1, 64, 64), ((1,), (64,), 2, 5, 128, 64), ((1,), (1001,), 8, 5, 128, 64),
           ((1, 1, 1), (17, 4000, 650), 2, 4, 128, 128), ((3, 0, 1, 2), (3, 500, 0, 129), 3, 3, 64, 192),
           ((17,), (40,), 1, 1, 128, 64), ((40, 7), (300, 7), 2, 2, 64, 64), ((33,), (2100,), 1, 16, 128, 64),
           ((130,), (190,), 1, 3, 64, 64), ((1,) * 67, tuple(range(5, 72)), 1, 2, 64, 64), ((2,), (9000,), 1, 7, 64, 512),
           ((300, 1), (301, 700), 2, 1, 128, 64), ((90, 0, 1, 257, 31), (90, 5, 640, 1000, 700), 1, 2, 64, 128),
           ((128,), (3000,), 1, 2, 128, 64), ((1, 300) + (1,) * 10, (70, 400) + tuple(range(100, 900, 80)), 1, 2, 128, 64),
           ((3,) * 9, tuple(range(200, 1100, 100)), 2, 1, 64, 64)]


@pytest.mark.parametrize("rows,lengths,heads,group,d,page", ATTENDS)
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("causal,window", [(False, 0), (True, 0), (True, 100), (False, 65), (True, 1)])
def test_attention(hcms, rows, lengths, heads, group, d, page, dtype, causal, window):
    log(f"[cache attention] rows={rows} lengths={lengths} heads={heads}x{group} d={d} {dtype} causal={causal} {window}")
    b = Batch(rows, lengths, heads, d, page, seed=sum(lengths) + d)
    q = _randn(7, b.T, heads * group, d, dtype=dtype)
    got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal, window=window)
    _check(got, q, b, dtype, d ** -0.5, causal, window, "out")
    again = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal, window=window)
    assert torch.equal(bits(got), bits(again))


# Pages that sequences may have, of which these have a few: enough for the kernel for many
# rows from some hundred rows on, and for waves alone from some hundred sequences on.
WIDE = 1 << 17


@pytest.mark.parametrize("rows,lengths,heads,group,d,page", [
    ((130,), (190,), 1, 3, 64, 64), ((300, 1), (301, 700), 2, 1, 128, 64), ((128,), (3000,), 1, 2, 128, 64),
    ((90, 0, 1, 257, 31), (90, 5, 640, 1000, 700), 1, 2, 64, 128), ((520, 300), (900, 2500), 2, 4, 128, 192),
    ((257, 70, 64, 65), (2000, 64, 500, 65), 3, 1, 64, 64), ((1, 300) + (1,) * 10, (70, 400) + tuple(range(100, 900, 80)), 1, 2, 128, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("causal", [False, True])
def test_attention_of_many_rows(hcms, rows, lengths, heads, group, d, page, dtype, causal):
    log(f"[many rows] rows={rows} lengths={lengths} heads={heads}x{group} d={d} {dtype} causal={causal}")
    b = Batch(rows, lengths, heads, d, page, seed=sum(lengths) + d, width=WIDE)
    q = _randn(7, b.T, heads * group, d, dtype=dtype)
    got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal)
    _check(got, q, b, dtype, d ** -0.5, causal, 0, "out")
    again = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal)
    assert torch.equal(bits(got), bits(again))


@pytest.mark.parametrize("rows,lengths", [((660,), (700,)), ((403, 3, 0, 300), (600, 3, 70, 500))])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("causal,window", [(True, 0), (True, 100), (False, 65), (True, 1)])
def test_many_rows_on_short_caches_and_in_windows(hcms, rows, lengths, d, dtype, causal, window):
    """A workgroup takes whole tiles of many rows."""
    log(f"[many rows, short] rows={rows} lengths={lengths} d={d} {dtype} causal={causal} {window}")
    b = Batch(rows, lengths, 2, d, 64, seed=sum(lengths) + d)
    q = _randn(7, b.T, 96, d, dtype=dtype)
    got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal, window=window)
    _check(got, q, b, dtype, d ** -0.5, causal, window, "out")


@pytest.mark.parametrize("rows,lengths,heads,group,d", [
    ((1,) * 300, tuple(range(300)), 1, 3, 128), ((1, 0, 3, 1) * 80, (40, 7, 1900, 1) * 80, 2, 8, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 1500)])
def test_attention_of_many_sequences(hcms, rows, lengths, heads, group, d, dtype, causal, window):
    """More tiles than workgroups: waves with pieces of their own."""
    log(f"[many sequences] {len(rows)} heads={heads}x{group} d={d} {dtype} causal={causal} {window}")
    b = Batch(rows, lengths, heads, d, 64, seed=d, width=1000)
    q = _randn(7, b.T, heads * group, d, dtype=dtype)
    got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal, window=window)
    _check(got, q, b, dtype, d ** -0.5, causal, window, "out")


@pytest.mark.parametrize("scale", [0.0, -0.2, 3.0, 1e-3])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("rows,width", [(5, 0), (70, 0), (70, WIDE)])
def test_scales_and_peaked_rows(hcms, scale, dtype, rows, width):
    b = Batch((rows,), (700,), 2, 128, seed=9, width=width)
    b.cache[2][:] = 127
    q = _randn(1, rows, 4, 128, dtype=dtype)
    got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), scale=scale)
    _check(got, q, b, dtype, float(np.float32(scale)), False, 0, f"scale {scale}")


@pytest.mark.parametrize("order", [1, -1])
@pytest.mark.parametrize("rows,width", [(1, 0), (40, 0), (300, WIDE)])
def test_scores_that_rise_and_fall_along_the_cache(hcms, order, rows, width):
    """The running maximum moves in every chunk, or never after the first."""
    b = Batch((rows,), (3000,), 1, 64, seed=4, width=width)
    q = torch.ones(rows, 1, 64)
    K = np.linspace(0, 1, 3000)[::order]
    for p in range(3000):
        k = np.full(64, np.float64(K[p]))
        oc.store(b.cache, b.page_table[0, p // 64], p % 64, 0, k, np.random.default_rng(p).standard_normal(64))
    for dtype in (BF16, FP32):
        got = hcms.cache_attention(q.to(dtype).cuda(), *b.gpu(hcms), scale=2.0)
        _check(got, q.to(dtype), b, dtype, 2.0, False, 0, f"order {order}")


@pytest.mark.parametrize("rows,width", [(1, 0), (5, 8 * 64), (40, 0), (300, WIDE)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("power", [5, 12, 25, 40, 90, 118])
@pytest.mark.parametrize("sign", [1, -1])
def test_scores_of_any_size(hcms, rows, width, dtype, power, sign):
    """Scores of halves up to 6, times 2^power and more, exact in fp32: a row's output is the
    mean of the values of the 12 tokens with the largest one, as the next is 128 and more
    below and its probability 0.  Theirs are equal, at most 2^-13 from 1 (in bf16: rounded to
    1 in the sum over values), so sums and quotient are off by 32 roundings.  With a scale of
    0 it is the mean of all, the powers of two off by 2^-21 and the sums as elsewhere."""
    rng = np.random.default_rng(power + rows)
    b = Batch((rows,), (700,), 1, 64, seed=rows, width=width)
    size = rng.choice([0.5, 1.0, 2.0, 3.0], 700) if sign > 0 else rng.choice([1.5, 2.0, 3.0], 700)
    top = rng.permutation(700)[:12]
    size[top] = 6.0 if sign > 0 else 0.5
    for p in range(700):
        k = np.zeros(64)
        k[0] = sign * size[p]
        oc.store(b.cache, b.page_table[0, p // 64], p % 64, 0, k, rng.standard_normal(64))
    q = torch.zeros(rows, 2, 64)
    q[:, 0, 0], q[:, 1, 0] = 2.0 ** (power + 3), 2.0 ** (power + 2)
    q = q.to(dtype)
    V = b.read(0)[1][:, 0]
    for scale in (1.0, 0.0):
        got = _f64(hcms.cache_attention(q.cuda(), *b.gpu(hcms), scale=scale))
        seen = V[top] if scale else V
        want, mass = seen.mean(0), np.abs(seen).mean(0)
        off = (32 * 2.0 ** -24 + (2.0 ** -13 if dtype == BF16 else 0) if scale else
               2.0 ** -20 + (700 / 16 + 64) * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0))
        bound = ROUND[dtype] * np.abs(want) + mass * off * (1 + 2.0 ** -7)
        worst = float((np.abs(got - want) / bound).max())
        log(f"    rows={rows} {dtype} 2^{power} {sign} scale {scale}: worst error {worst:.3f} of its bound")
        assert worst <= 1.0, (scale, worst)


@pytest.mark.parametrize("rows,width", [(1, 0), (300, WIDE)])
@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 1e-44])
def test_the_largest_and_smallest_scales(hcms, rows, width, scale):
    """Scores of zero, and others times the smallest scales, give the mean of the values."""
    b = Batch((rows,), (700,), 2, 128, seed=9, width=width)
    q = torch.zeros(rows, 4, 128) if abs(scale) > 1 else _randn(1, rows, 4, 128)
    for dtype in (BF16, FP32):
        got = hcms.cache_attention(q.to(dtype).cuda(), *b.gpu(hcms), scale=scale)
        _check(got, q.to(dtype), b, dtype, float(np.float32(scale)), False, 0, f"scale {scale}")


def test_strided_queries_out_and_rows_of_no_sequence(hcms):
    b = Batch((3, 5), (100, 65), 2, 128, seed=6)
    heads, d, extra = 6, 128, 4
    x = _randn(3, b.T + extra, 3 * heads * d + 5, dtype=BF16).cuda()
    q = x[:, 3:3 + heads * d].unflatten(1, (heads, d))
    out = torch.full((b.T + extra, heads, d), 9.0, dtype=BF16, device="cuda")
    got = hcms.cache_attention(q, *b.gpu(hcms), causal=True, out=out)
    assert got.data_ptr() == out.data_ptr() and (out[b.T:] == 9).all()
    want = hcms.cache_attention(q[:b.T].contiguous(), *b.gpu(hcms), causal=True)
    assert torch.equal(bits(out[:b.T]), bits(want))
    by_head = q.transpose(0, 1).contiguous().transpose(0, 1)          # heads outermost
    assert torch.equal(bits(hcms.cache_attention(by_head, *b.gpu(hcms), causal=True)[:b.T]), bits(want))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_many_rows_that_see_nothing(hcms, dtype, d):
    b = Batch((70, 130, 100), (0, 2, 40), 1, d, seed=8, width=WIDE)
    q = _randn(1, b.T, 2, d, dtype=dtype)
    for causal in (True, False):
        got = hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal)
        assert (got[:70] == 0).all() and (not causal or ((got[70:198] == 0).all() and (got[200:260] == 0).all()))
        _check(got, q, b, dtype, d ** -0.5, causal, 0, f"causal={causal}")


def test_rows_that_see_nothing_and_lengths_of_zero(hcms):
    b = Batch((2, 4, 1), (0, 2, 40), 1, 64, seed=8)      # more rows than tokens: the first rows see nothing if causal
    q = _randn(1, b.T, 2, 64, dtype=FP32)
    for causal in (True, False):
        got = _f64(hcms.cache_attention(q.cuda(), *b.gpu(hcms), causal=causal))
        assert (got[:2] == 0).all() and np.isfinite(got).all()
        if causal:
            assert (got[2:4] == 0).all() and (got[4:] != 0).any(-1).all()
        _check(torch.from_numpy(got), q, b, FP32, 0.125, causal, 0, f"causal={causal}")
    cache, pages, lengths, starts = b.gpu(hcms)
    none = torch.zeros(0, 2, 64).cuda()
    assert hcms.cache_attention(none, cache, pages, lengths, torch.zeros_like(starts)).shape == (0, 2, 64)
    left = hcms.cache_attention(q.cuda(), cache, pages[:0], lengths[:0], starts[:1], out=torch.full((b.T, 2, 64), 5.0).cuda())
    assert (left == 5).all()


@pytest.mark.parametrize("group", [2, 20, 12000])   # few rows and many
@pytest.mark.parametrize("d", [64, 128])
def test_values_that_are_not_finite_reach_the_rows_that_see_them_only(hcms, group, d):
    """NaN in keys and values of tokens before a window, after a causal row's place, and
    behind the sequence's end in its last page."""
    for dtype in (BF16, FP32):
        for part in (2, 3):                                       # k_scale, v_scale
            for byte in (255, 254, 253):
                b = Batch((6,), (100,), 1, d, seed=2)
                q = _randn(1, 6, group, d, dtype=dtype).cuda()
                clean = _f64(hcms.cache_attention(q, *b.gpu(hcms), causal=True, window=20))
                place = oc.key_scale_place if part == 2 else oc.value_place
                for p in (97, 78, 100, 127):                      # rows 0 to 5 see [75 + i, 95 + i)
                    b.cache[part][b.page_table[0, p // 64], 0, 0, 1, place(p % 64)] = byte
                got = _f64(hcms.cache_attention(q, *b.gpu(hcms), causal=True, window=20))
                for i in range(6):
                    seen = any(75 + i <= p < 95 + i for p in (97, 78))
                    if not seen:
                        assert np.array_equal(got[i], clean[i]), (dtype, part, byte, i)
                    elif part == 3:
                        bad = slice(32, 64)
                        assert not np.isfinite(got[i][:, bad]).any()
                        got[i][:, bad] = clean[i][:, bad] = 0
                        assert np.array_equal(got[i], clean[i])
                    elif byte == 255:
                        assert np.isnan(got[i]).all()


@pytest.mark.parametrize("rows,width", [(1, 0), (90, 0), (90, 2 * WIDE)])
def test_nan_in_the_middle_of_a_sequence(hcms, rows, width):
    b = Batch((rows, rows), (300, 300), 1, 128, seed=2, width=width)
    b.cache[3][b.page_table[0, 1], 0, 0, 2, oc.value_place(7)] = 255
    b.cache[2][b.page_table[1, 1], 0, 0, 2, oc.key_scale_place(7)] = 255
    got = _f64(hcms.cache_attention(_randn(1, 2 * rows, 1, 128).cuda(), *b.gpu(hcms)))
    first = got[:rows, 0]
    assert np.isnan(first[:, 64:96]).all() and np.isfinite(first[:, :64]).all() and np.isfinite(first[:, 96:]).all()
    assert np.isnan(got[rows:]).all()


@pytest.mark.parametrize("rows,group,width", [(1, 1, 0), (1, 8, 600), (90, 2, 0), (90, 2, 2 * WIDE)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("byte", [252, 253, 254, 255])
def test_scales_from_2_to_the_126_on_are_nan_wherever_their_chunk_lies(hcms, rows, group, width, d, dtype, byte):
    """In chunks that every row sees whole, that a window cuts and that the sequence's end
    cuts; of any codes, zeros and the smallest among them.  Zeros of scale 2^125 are numbers."""
    log(f"[large scales] rows={rows}x{group} width={width} d={d} {dtype} byte={byte}")
    q = _randn(1, 4 * rows, group, d, dtype=dtype).cuda()
    for code in (0x00, 0x11, 0x77):
        for part in (2, 3):
            if byte == 252 and (part == 2 or code):      # sums past fp32's range
                continue
            b = Batch((rows,) * 4, (300,) * 4, 1, d, seed=2, width=width)
            clean = _f64(hcms.cache_attention(q, *b.gpu(hcms), window=250))
            for s, p in enumerate((100, 60, 299)):              # the fourth sequence has none; rows see [50, 300)
                page, t = b.page_table[s, p // 64], p % 64
                if part == 2:
                    b.cache[0][page, 0, t, 16:32] = code
                    b.cache[2][page, 0, 0, 1, oc.key_scale_place(t)] = byte
                else:
                    b.cache[1][page, 0, 0, 16:32, oc.value_place(t)] = code
                    b.cache[3][page, 0, 0, 1, oc.value_place(t)] = byte
            got = _f64(hcms.cache_attention(q, *b.gpu(hcms), window=250))
            bad = np.zeros(got.shape, bool)
            if byte > 252:
                bad[:3 * rows, :, slice(32, 64) if part == 3 else slice(None)] = True
            assert np.array_equal(np.isnan(got), bad) and np.isfinite(got[~bad]).all(), (code, part)
            same = np.ones(got.shape, bool)
            same[:3 * rows, :, slice(32, 64) if part == 3 else slice(None)] = False
            assert np.array_equal(got[same], clean[same]), (code, part)


@pytest.mark.parametrize("rows,width", [(1, 0), (90, 0), (90, 2 * WIDE)])
@pytest.mark.parametrize("x", [1e36, 2.6e38, 3.4e38])
def test_appended_values_next_to_the_largest(hcms, rows, width, x):
    """Past 6 2^125 = 2.55e38 a block's values are NaN to the rows that see them, in a whole
    chunk and in one that the sequence's end cuts; 1e36, 2^-8 of the largest number, is one."""
    b = Batch((rows, rows), (130, 200), 1, 64, seed=2, width=width)
    k, v = _randn(1, 2 * rows, 1, 64), _randn(2, 2 * rows, 1, 64)
    v[0, 0, 3], k[rows, 0, 40] = x, x
    cache, *batch = b.gpu(hcms)
    hcms.append_kv(k.cuda(), v.cuda(), cache, *batch)
    q = _randn(3, 2 * rows, 2, 64)
    q[..., 32:] *= 2.0 ** -20
    got = _f64(hcms.cache_attention(q.cuda(), cache, *batch))
    if x < 2.55e38:
        assert np.isfinite(got[:rows]).all()
    else:
        assert np.isnan(got[:rows, :, :32]).all() and np.isfinite(got[:rows, :, 32:]).all() and np.isnan(got[rows:]).all()


@pytest.mark.parametrize("rows,width", [(1, 0), (90, 0), (90, WIDE)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_appended_nan_comes_out(hcms, rows, dtype, width):
    """A block that was not finite when it was appended (whose codes are zeros) is NaN to
    the rows that see it."""
    b = Batch((rows, rows), (200, 200), 1, 64, seed=2, width=width)
    k, v = _randn(1, 2 * rows, 1, 64, dtype=dtype), _randn(2, 2 * rows, 1, 64, dtype=dtype)
    k[0, 0, 3], v[rows, 0, 40] = float("inf"), float("nan")
    cache, *batch = b.gpu(hcms)
    hcms.append_kv(k.cuda(), v.cuda(), cache, *batch)
    got = _f64(hcms.cache_attention(_randn(3, 2 * rows, 2, 64, dtype=dtype).cuda(), cache, *batch))
    assert np.isnan(got[:rows]).all() and np.isnan(got[rows:, :, 32:]).all() and np.isfinite(got[rows:, :, :32]).all()


@pytest.mark.parametrize("group", [3, 40, 16000])   # few rows and many
def test_pages_that_there_are_not_and_sequences_past_them(hcms, group):
    b = Batch((2, 2, 2), (150, 150, 150), 1, 64, seed=3)
    b.page_table[0, 1], b.page_table[1, 0] = b.pages, -5
    q = _randn(1, 6, group, 64, dtype=BF16)
    cache, pages, lengths, starts = b.gpu(hcms)
    lengths[2] = 3 * 64 + 1
    got = _f64(hcms.cache_attention(q.cuda(), cache, pages, lengths, starts, causal=True))
    assert np.isnan(got).all()
    got = _f64(hcms.cache_attention(q.cuda(), cache, pages, lengths, starts, causal=True, window=10))
    assert np.isfinite(got[:4]).all() and np.isnan(got[4:]).all()      # the lost pages are out of the window


@pytest.mark.parametrize("group,width", [(4, 0), (40, 0), (64, 8 * WIDE)])
def test_queries_that_are_not_finite_stay_in_their_rows(hcms, group, width):
    b = Batch((3,), (200,), 1, 64, seed=3, width=width)
    q = _randn(1, 3, group, 64, dtype=BF16)
    clean = _f64(hcms.cache_attention(q.cuda(), *b.gpu(hcms)))
    q[1, 2, 5] = float("nan")
    got = _f64(hcms.cache_attention(q.cuda(), *b.gpu(hcms)))
    assert np.isnan(got[1, 2]).all()
    clean[1, 2] = got[1, 2] = 0
    assert np.array_equal(got, clean)


# ---------------------------------------------------------------------------
# Together
# ---------------------------------------------------------------------------
def _steps(hcms, cache, table, H, Hk, d, grid, pairs, sizes, seed, stream=None):
    """Pieces of two sequences one behind the other: norm and rotation, append, attention."""
    lengths, out, kept = [0, 0], [], []
    pages = torch.tensor([[3, 0, 5, 6], [1, 4, 2, 7]], dtype=torch.int32).cuda()
    w = (1 + 0.1 * _randn(99, 2, d, dtype=BF16)).cuda()
    for step, rows in enumerate(sizes):
        T = sum(rows)
        lengths = [a + r for a, r in zip(lengths, rows)]
        at = [n - r + i for n, r in zip(lengths, rows) for i in range(r)]
        x = _randn(seed + step, T, (H + 2 * Hk) * d, dtype=BF16).cuda()
        q, k, v = (t.unflatten(1, (-1, d)) for t in x.split((H * d, Hk * d, Hk * d), 1))
        pos = torch.tensor(at, dtype=torch.int32).cuda()
        args = (torch.tensor(lengths, dtype=torch.int32).cuda(),
                torch.tensor([0, rows[0], T], dtype=torch.int32).cuda())
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        q, k = hcms.qk_norm_rope(q, k, w[0], w[1], table, grid, pairs, positions=pos, stream=stream)
        held = hcms.append_kv(k, v, cache, pages, *args, held=True, stream=stream)
        out.append(hcms.cache_attention(q, cache, pages, *args, causal=True, stream=stream))
        kept.append((q, *held))
        if stream is not None:
            torch.cuda.current_stream().wait_stream(stream)
    return out, kept


def test_a_rolling_sequence_equals_attention_over_what_the_cache_holds(hcms):
    """Prompts, then pieces, then tokens: each output against the oracle on the held keys
    and values; and the same on another stream."""
    H, Hk, d, grid, pairs = 4, 2, 64, [256], [32]
    table = hcms.rope_table(grid, pairs)
    sizes = [(100, 30), (1, 1), (1, 1), (40, 0), (1, 64), (1, 1)]
    out, kept = _steps(hcms, hcms.kv_cache(8, Hk, d), table, H, Hk, d, grid, pairs, sizes, 50)
    past = [[np.zeros((0, Hk, d))] * 2, [np.zeros((0, Hk, d))] * 2]
    for rows, o, (q, k, v) in zip(sizes, out, kept):
        first = 0
        for s, n in enumerate(rows):
            part = slice(first, first + n)
            past[s] = [np.concatenate((p, _f64(x)[part])) for p, x in zip(past[s], (k, v))]
            first += n
            if n == 0:
                continue
            want, A, most = oc.attention(_f64(q)[part], *past[s], d ** -0.5, True)
            bound = 2.0 ** -8 * np.abs(want) + A * (2.0 ** -8 + 2.0 ** -14) * (1 + 2.0 ** -7)
            assert (np.abs(_f64(o)[part] - want) <= bound).all()
    other, _ = _steps(hcms, hcms.kv_cache(8, Hk, d), table, H, Hk, d, grid, pairs, sizes, 50, torch.cuda.Stream())
    for a, c in zip(out, other):
        assert torch.equal(bits(a), bits(c))


def test_a_step_in_a_graph_follows_its_lengths(hcms):
    """One captured step of decoding, replayed as the sequences grow, against eager calls;
    eager work of the same operators runs between the replays."""
    H, Hk, d, grid, pairs, n = 8, 2, 128, [4096], [64], 6
    table, page = hcms.rope_table(grid, pairs), 64
    base = Batch((1, 1), (600, 63), Hk, d, page, seed=1, width=12)
    base.page_table[:] = np.arange(24).reshape(2, 12)
    def fresh():
        c = hcms.kv_cache(24, Hk, d, page)
        g = torch.Generator().manual_seed(3)
        for t, first, past in zip(c, (0, 0, 125, 125), (256, 256, 129, 129)):     # any codes, scales near 1
            t.view(torch.uint8).copy_(torch.randint(first, past, t.shape, generator=g).to(torch.uint8))
        return c
    pages = torch.from_numpy(base.page_table).cuda()
    starts = torch.tensor([0, 1, 2], dtype=torch.int32).cuda()
    x = _randn(5, n, 2, (H + 2 * Hk) * d, dtype=BF16).cuda()

    def step(cache, xs, lengths):
        q, k, v = (t.unflatten(1, (-1, d)) for t in xs.split((H * d, Hk * d, Hk * d), 1))
        hcms.append_kv(k, v, cache, pages, lengths, starts, table=table, grid=grid, axis_pairs=pairs, layout="half")
        return hcms.cache_attention(q, cache, pages, lengths, starts, causal=True)

    eager, lengths = fresh(), torch.tensor([600, 63], dtype=torch.int32).cuda()
    want = []
    for i in range(n):
        want.append(step(eager, x[i], lengths).clone())
        lengths += 1
    cache, xs, lengths = fresh(), x[0].clone(), torch.tensor([600, 63], dtype=torch.int32).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(fresh(), xs, lengths)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache, xs, lengths)
    for i in range(n):
        xs.copy_(x[i])
        graph.replay()
        step(fresh(), x[i], lengths)                 # eager, between the replays
        torch.cuda.synchronize()
        assert torch.equal(bits(out), bits(want[i])), i
        lengths += 1
    for a, c in zip(numpy_of(cache), numpy_of(eager)):
        assert np.array_equal(a, c)


def test_two_batches_on_two_streams(hcms):
    """Calls that overlap have workspaces of their own."""
    cases = [Batch((1,), (9000,), 2, 128, seed=i) for i in (1, 2)]
    q = [_randn(i, 1, 8, 128, dtype=BF16).cuda() for i in (3, 4)]
    args = [b.gpu(hcms) for b in cases]
    want = [hcms.cache_attention(x, *a) for x, a in zip(q, args)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [hcms.cache_attention(x, *a, stream=s) for x, a, s in zip(q, args, streams)]
        torch.cuda.synchronize()
        for a, c in zip(got, want):
            assert torch.equal(bits(a), bits(c))


def test_past_32_bits(hcms):
    """A cache of more than 2^31 bytes of keys, whose last pages are used."""
    heads, d, page = 64, 128, 64
    pages = (1 << 31) // (heads * page * d // 2) + 8
    cache = hcms.kv_cache(pages, heads, d, page)
    assert cache.k.numel() > 1 << 31
    k, v = _randn(1, 3, heads, d, dtype=BF16), _randn(2, 3, heads, d, dtype=BF16)
    table = torch.tensor([[pages - 1]], dtype=torch.int32).cuda()
    batch = (table, torch.tensor([3], dtype=torch.int32).cuda(), torch.tensor([0, 3], dtype=torch.int32).cuda())
    hk, hv = hcms.append_kv(k.cuda(), v.cuda(), cache, *batch, held=True)
    q = _randn(3, 3, heads, d, dtype=BF16)
    got = _f64(hcms.cache_attention(q.cuda(), cache, *batch, causal=True))
    want, A, _ = oc.attention(_f64(q), _f64(hk), _f64(hv), d ** -0.5, True)
    assert (np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -14) * (np.abs(want) + A) * (1 + 2.0 ** -7)).all()
    assert int(cache.k[:pages - 1].max()) == 0


def test_more_tiles_than_a_grid_s_axis_has_threads_for(hcms):
    """2^27 query heads on one key head: 2^23 tiles of a workgroup each, all alike."""
    b = Batch((1,), (40,), 1, 64, seed=3)
    args = b.gpu(hcms)
    q, n = _randn(1, 1, 1, 64, dtype=BF16).cuda(), 1 << 27
    one = bits(hcms.cache_attention(q, *args))
    log(f"[grid] {n} heads")
    out = torch.zeros(1, n, 64, dtype=BF16, device="cuda")
    hcms.cache_attention(q.expand(1, n, 64), *args, out=out)
    for part in out.view(torch.int16).split(n // 16, 1):
        assert bool((part == one).all())

"""The norm and rotation of query and key heads in one pass on the GPU, against the
float64 oracle of ``oracle/cache.py``.

Tolerances, from the arithmetic: fp32 statistics, products and rotation.  A head
vector's sum of squares has at most 8 lane steps of 16 terms, so it and what follows are
within 2^-17 of the magnitudes of their terms; the rotation's terms are both elements of
a pair; then the rounding of the storage type.  dw sums over tokens and heads in fp32, in
a tree whose paths have at most S H / 512 + 100 steps, each 2^-24 of the magnitudes.
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import cache as oc
from tests.gpu_util import bits, log

pytestmark = pytest.mark.gpu
BF16, FP32 = torch.bfloat16, torch.float32
ROUND = {BF16: 2.0 ** -8, FP32: 2.0 ** -24}
EPS = 1e-5


def _f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _randn(seed, *shape, dtype=FP32):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def _within(got, want, bound, what):
    got = _f64(got)
    assert got.shape == want.shape and np.isfinite(got).all(), what
    worst = float((np.abs(got - want) / np.maximum(bound, 1e-300)).max()) if got.size else 0.0
    log(f"    {what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0, f"{what}: {worst:.3f} times the bound"


def _spread(x, z, layout):
    """Of each element the magnitudes of the two terms that the rotation adds, at least:
    with c, s >= 0, (a, b) turned either way gives |a c - b s| and a c + b s, of sum
    2 max(a c, b s), and the same of the pair's other element."""
    there, back = (oc.turn(np.abs(x), np.abs(z.real) + i * np.abs(z.imag), layout) for i in (1j, -1j))
    return np.abs(there) + np.abs(back)


# S, H, Hk, d, pairs of each axis, grid, layout: one and many tokens and heads; whole and
# partial rotations; lengths that the wide accesses do not divide; up to four axes.
SHAPES = [(1, 1, 1, 64, (32,), (1,), "half"), (1, 40, 8, 128, (64,), (1,), "half"),
          (7, 5, 5, 128, (22, 21, 21), (2, 2, 2), "interleaved"), (33, 3, 1, 128, (32,), (40,), "half"),
          (50, 2, 2, 128, (24,), (50,), "half"), (129, 4, 2, 64, (8, 8), (13, 10), "interleaved"),
          (9, 3, 2, 32, (4, 4, 4, 4), (2, 2, 2, 2), "half"), (5, 2, 1, 512, (256,), (5,), "interleaved"),
          (5, 2, 1, 512, (256,), (5,), "half"), (6, 1, 2, 256, (64,), (6,), "half"),
          (3, 2, 1, 24, (4,), (3,), "interleaved"), (11, 3, 2, 50, (12,), (11,), "half"),
          (11, 3, 2, 37, (5, 3), (11, 1), "interleaved"), (4, 1, 1, 2, (1,), (4,), "half"),
          (300, 2, 1, 96, (3,), (300,), "interleaved"), (2, 70, 3, 40, (20,), (2,), "interleaved"),
          (1030, 1, 1, 128, (64,), (1030,), "interleaved")]


def _case(S, H, Hk, d, pairs, grid, layout, dtype, seed, hcms):
    qkv = _randn(seed, S, (H + 2 * Hk) * d, dtype=dtype)
    q, k = qkv[:, :H * d].unflatten(1, (H, d)), qkv[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
    wdt = dtype if d % 3 else FP32
    qw, kw = ((1 + 0.3 * _randn(seed + 1 + i, d)).to(wdt) for i in range(2))
    table = hcms.rope_table(list(grid), list(pairs))
    z = oc.factors(_f64(table), grid, pairs, oc.coordinates(grid, np.arange(S)))
    return qkv, q, k, qw, kw, table, z


@pytest.mark.parametrize("S,H,Hk,d,pairs,grid,layout", SHAPES)
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_qk_norm_rope_and_gradients(hcms, S, H, Hk, d, pairs, grid, layout, dtype):
    log(f"[head norm] S={S} H={H},{Hk} d={d} pairs={pairs} {layout} {dtype}")
    qkv, q, k, qw, kw, table, z = _case(S, H, Hk, d, pairs, grid, layout, dtype, S + d, hcms)
    dev = qkv.cuda()
    gq, gk = dev[:, :H * d].unflatten(1, (H, d)), dev[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
    got = hcms.qk_norm_rope(gq, gk, qw.cuda(), kw.cuda(), table, grid, pairs, layout=layout, eps=EPS)
    dys = _randn(5, S, H, d, dtype=dtype), _randn(6, S, Hk, d, dtype=dtype)
    leaves = [t.detach().cuda().requires_grad_(True) for t in (q, k, qw, kw)]
    leaves[0] = gq.detach().requires_grad_(True)     # a strided view of a projection's output
    y = hcms.QkNormRope.apply(*leaves, table, grid, pairs, None, layout, EPS)
    assert torch.equal(bits(y[0]), bits(got[0])) and torch.equal(bits(y[1]), bits(got[1]))
    grads = torch.autograd.grad(y, leaves, [t.cuda() for t in dys])
    for i, (x, w, dy) in enumerate(((q, qw, dys[0]), (k, kw, dys[1]))):
        X, W, DY, side = _f64(x), _f64(w), _f64(dy), "qk"[i]
        want = oc.head_norm(X, W, EPS, z, layout)
        n = np.abs(X) / np.sqrt((X * X).mean(-1, keepdims=True) + EPS)
        _within(got[i], want, ROUND[dtype] * np.abs(want) + 2.0 ** -17 * _spread(n * W, z, layout) + 1e-30, side)
        dx, dw = oc.head_norm_backward(DY, X, W, EPS, z, layout)
        r = 1 / np.sqrt((X * X).mean(-1, keepdims=True) + EPS)
        g = _spread(DY, z, layout)
        gw = g * np.abs(W)
        terms = r * (gw + n * (gw * n).mean(-1, keepdims=True))
        _within(grads[i], dx, ROUND[dtype] * np.abs(dx) + 2.0 ** -17 * terms, "d" + side)
        steps = S * X.shape[1] / 512 + 100
        _within(grads[2 + i], dw, ROUND[w.dtype] * np.abs(dw) +
                (2.0 ** -17 + steps * 2.0 ** -24) * (g * n).sum((0, 1)), "dw" + side)


def test_qk_norm_rope_equals_norm_and_rope_apart_in_fp32(hcms):
    """As the two operators one behind the other, within their roundings."""
    S, H, Hk, d, grid, pairs = 300, 4, 2, 128, [5, 6, 10], [22, 21, 21]
    _, q, k, qw, kw, table, _ = _case(S, H, Hk, d, pairs, grid, "interleaved", FP32, 3, hcms)
    q, k, qw, kw = (t.contiguous().cuda() for t in (q, k, qw, kw))
    got = hcms.qk_norm_rope(q, k, qw, kw, table, grid, pairs)
    nq = hcms.rms_norm(q.view(-1, d), qw).view(S, H, d)
    nk = hcms.rms_norm(k.view(-1, d), kw).view(S, Hk, d)
    for a, b in zip(got, hcms.rope(nq, nk, table, grid, pairs)):
        assert float((a - b).abs().max()) <= 2.0 ** -17 * 8


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,grid,pairs", [(128, (4096,), (64,)), (64, (9, 11, 13), (12, 10, 10)), (50, (4096,), (7,))])
def test_positions(hcms, kind, layout, d, grid, pairs):
    S, H = 21, 3
    table = hcms.rope_table(list(grid), list(pairs))
    rng = np.random.default_rng(2)
    at = np.stack([rng.integers(0, g, S) for g in grid], 1)
    at[3, 0], at[5, -1] = grid[0], -1                      # outside the grid
    x, w = _randn(9, S, H, d), 1 + 0.1 * _randn(10, d)
    pos = torch.from_numpy(at).to(kind).cuda()
    y = hcms.qk_norm_rope(x.cuda(), None, w.cuda(), None, table, grid, pairs, positions=pos, layout=layout, eps=EPS)
    z = oc.factors(_f64(table), grid, pairs, at)
    want = oc.head_norm(_f64(x), _f64(w), EPS, z, layout)
    got, P = _f64(y), sum(pairs)
    turned = np.zeros(d, bool)
    turned[:2 * P] = True
    for t in (3, 5):
        assert np.isnan(got[t][:, turned]).all()
    ok = [t for t in range(S) if t not in (3, 5)]
    assert np.abs(got[ok] - want[ok]).max() <= 2.0 ** -17 * 8
    if len(grid) == 1:
        one = hcms.qk_norm_rope(x.cuda(), None, w.cuda(), None, table, grid, pairs, positions=pos[:, 0].contiguous(),
                                layout=layout, eps=EPS)
        assert torch.equal(bits(one), bits(y))


@pytest.mark.parametrize("d,layout", [(128, "half"), (64, "interleaved"), (50, "half")])
def test_in_place_and_out(hcms, d, layout):
    S, H, Hk, P = 40, 3, 2, d // 4
    qkv, q, k, qw, kw, table, _ = _case(S, H, Hk, d, (P,), (S,), layout, BF16, 8, hcms)
    dev, w = qkv.cuda(), (qw.cuda(), kw.cuda())
    gq, gk = dev[:, :H * d].unflatten(1, (H, d)), dev[:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
    want = hcms.qk_norm_rope(gq, gk, *w, table, [S], [P], layout=layout)
    packed = torch.full((S, (H + Hk) * d + 3), 7.0, dtype=BF16, device="cuda")   # strides that 8 does not divide
    out = packed[:, 1:1 + H * d].unflatten(1, (H, d)), packed[:, 1 + H * d:1 + (H + Hk) * d].unflatten(1, (Hk, d))
    got = hcms.qk_norm_rope(gq, gk, *w, table, [S], [P], layout=layout, out=out)
    for a, b in zip(got, want):
        assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -8 * 8   # another order of the sums: a rounding
    assert (packed[:, 0] == 7).all() and (packed[:, -2:] == 7).all()
    v = dev[:, (H + Hk) * d:].clone()
    again = hcms.qk_norm_rope(gq, gk, *w, table, [S], [P], layout=layout, out=(gq, gk))
    for a, b in zip(again, want):
        assert torch.equal(bits(a), bits(b))
    assert again[0].data_ptr() == dev.data_ptr() and torch.equal(bits(v), bits(dev[:, (H + Hk) * d:]))


def test_gradients_of_one_side_and_no_tokens(hcms):
    S, H, Hk, d = 10, 3, 2, 64
    _, q, k, qw, kw, table, _ = _case(S, H, Hk, d, (32,), (S,), "half", FP32, 4, hcms)
    leaves = [t.detach().contiguous().cuda().requires_grad_(True) for t in (q, k, qw, kw)]
    y = hcms.QkNormRope.apply(*leaves, table, [S], [32], None, "half", EPS)
    dq, dk = torch.randn_like(y[0]), torch.randn_like(y[1])
    whole = torch.autograd.grad(y, leaves, (dq, dk), retain_graph=True)
    a = torch.autograd.grad(y[0], (leaves[0], leaves[2]), dq, retain_graph=True)
    b = torch.autograd.grad(y[1], (leaves[1], leaves[3]), dk, retain_graph=True)
    for g, w in zip((a[0], b[0], a[1], b[1]), whole):
        assert float((g - w).abs().max()) <= 2.0 ** -17 * float(w.abs().max())
    y[1].sum().backward()                                        # an expanded gradient
    assert torch.isfinite(leaves[1].grad).all() and leaves[0].grad is None
    none = [t.detach()[:0].requires_grad_(True) for t in leaves[:2]] + [t.detach().requires_grad_(True) for t in leaves[2:]]
    y = hcms.QkNormRope.apply(*none, table, [S], [32], None, "half", EPS)
    g = torch.autograd.grad(y, none, (dq[:0], dk[:0]))
    assert g[0].shape == (0, H, d) and (g[2] == 0).all() and (g[3] == 0).all()
    alone = leaves[0].detach().requires_grad_(True)
    w = leaves[2].detach().requires_grad_(True)
    y = hcms.QkNormRope.apply(alone, None, w, None, table, [S], [32], None, "half", EPS)
    g = torch.autograd.grad(y, (alone, w), dq)
    assert float((g[0] - whole[0]).abs().max()) <= 2.0 ** -17 * float(whole[0].abs().max())


def test_gradient_matches_differences(hcms):
    S, H, d, grid, pairs = 19, 3, 64, [19], [24]
    table = hcms.rope_table(grid, pairs)
    x, u, dy = (_randn(70 + i, S, H, d).cuda() for i in range(3))
    w, uw = (1 + 0.1 * _randn(80, d)).cuda(), _randn(81, d).cuda()
    leaves = [x.clone().requires_grad_(True), w.clone().requires_grad_(True)]
    y = hcms.QkNormRope.apply(leaves[0], None, leaves[1], None, table, grid, pairs, None, "half", EPS)
    dx, dw = torch.autograd.grad(y, leaves, dy)

    def value(t):
        z = hcms.qk_norm_rope(x + t * u, None, w + t * uw, None, table, grid, pairs, layout="half", eps=EPS)
        return float((z.double() * dy.double()).sum())

    s = 1e-2
    got = (value(s) - value(-s)) / (2 * s)
    want = float((dx.double() * u.double()).sum() + (dw.double() * uw.double()).sum())
    scale = float(dx.double().norm() * u.double().norm() + dw.double().norm() * uw.double().norm())
    log(f"    slope {got:.6g}, gradient {want:.6g}, scale {scale:.4g}")
    assert abs(got - want) <= 1e-3 * scale


def test_extremes_and_a_gradient_of_a_gradient(hcms):
    d = 64
    table = hcms.rope_table([4], [32])
    x = torch.zeros(4, 1, d)
    x[1] = 1e-18
    x[2, 0, 3] = float("nan")
    y = hcms.qk_norm_rope(x.cuda(), None, torch.ones(d).cuda(), None, table, [4], [32]).cpu()
    assert (y[0] == 0).all() and torch.isfinite(y[1]).all() and y[2].isnan().all() and (y[3] == 0).all()
    q = torch.randn(4, 1, d).cuda().requires_grad_(True)
    w = torch.ones(d).cuda().requires_grad_(True)
    out = hcms.QkNormRope.apply(q, None, w, None, table, [4], [32])
    with pytest.raises(RuntimeError, match="once"):
        torch.autograd.grad(out.sum(), (q, w), create_graph=True)
    with torch.no_grad():
        out = hcms.QkNormRope.apply(q, None, w, None, table, [4], [32])
    y = hcms.QkNormRope.apply(q, None, w, None, table, [4], [32])
    with torch.no_grad():
        q.add_(1)                      # what the backward needs
    with pytest.raises(RuntimeError, match="modified"):
        y.sum().backward()


@pytest.mark.parametrize("S,H,Hk,d,pairs,grid,layout", [SHAPES[i] for i in (0, 1, 2, 5, 7, 8, 9, 11, 12, 15)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("eps", [0.0, float(np.float32(1e-40))])
def test_mean_squares_below_2_to_the_minus_126(hcms, S, H, Hk, d, pairs, grid, layout, dtype, eps):
    """Head vectors so small that mean(x^2) + eps is subnormal, and with an eps of its own
    zeros among them, whose outputs are zeros and whose gradients are finite.  Of the mean,
    each square and the product with 1 / d are off by 2^-150 at most, half a step, so it is
    within 2^-149; of r, n and dx that takes at most a half, a half and three halves of the
    relative error, all counted as two."""
    log(f"[head norm, small] S={S} H={H},{Hk} d={d} pairs={pairs} {layout} {dtype} eps={eps}")
    _, q, k, qw, kw, table, z = _case(S, H, Hk, d, pairs, grid, layout, dtype, S + d, hcms)
    q, k = (t * 2.0 ** -66 for t in (q, k))
    assert ((q.double() ** 2).mean(-1) + eps < 2.0 ** -126).all() and ((q.double() ** 2).mean(-1) > 2.0 ** -142).all()
    zero = eps > 0 and S > 1
    if zero:
        q[1], k[1, 0] = 0, 0
    leaves = [t.cuda().requires_grad_(True) for t in (q, k, qw, kw)]
    y = hcms.QkNormRope.apply(*leaves, table, grid, pairs, None, layout, eps)
    dys = _randn(5, S, H, d, dtype=dtype), _randn(6, S, Hk, d, dtype=dtype)
    grads = torch.autograd.grad(y, leaves, [t.cuda() for t in dys])
    if zero:
        assert (y[0][1] == 0).all() and (y[1][1, 0] == 0).all()
    for i, (x, w, dy) in enumerate(((q, qw, dys[0]), (k, kw, dys[1]))):
        X, W, DY, side = _f64(x), _f64(w), _f64(dy), "qk"[i]
        mean = (X * X).mean(-1, keepdims=True) + eps
        n, r = np.abs(X) / np.sqrt(mean), 1 / np.sqrt(mean)
        rel = 2.0 ** -17 + 2 * 2.0 ** -149 / mean
        _within(y[i], oc.head_norm(X, W, eps, z, layout), ROUND[dtype] * np.abs(oc.head_norm(X, W, eps, z, layout)) +
                rel * _spread(n * W, z, layout) + 1e-30, side)
        dx, dw = oc.head_norm_backward(DY, X, W, eps, z, layout)
        g = _spread(DY, z, layout)
        gw = g * np.abs(W)
        _within(grads[i], dx, ROUND[dtype] * np.abs(dx) + rel * r * (gw + n * (gw * n).mean(-1, keepdims=True)), "d" + side)
        _within(grads[2 + i], dw, ROUND[w.dtype] * np.abs(dw) +
                ((rel + (S * X.shape[1] / 512 + 100) * 2.0 ** -24) * g * n).sum((0, 1)), "dw" + side)


@pytest.mark.parametrize("pairs,layout", [(64, "interleaved"), (27, "half")])
def test_past_32_bits(hcms, pairs, layout):
    """More than 2^31 elements: the last tokens bit for bit as alone, both directions."""
    S, H, d, n = 66000, 256, 128, 700
    q = torch.randn(S, H, d, generator=torch.Generator("cuda").manual_seed(1), dtype=BF16, device="cuda")
    assert q.numel() > 1 << 31
    w, table = torch.full((d,), 1.5, dtype=BF16, device="cuda"), hcms.rope_table([50], [pairs])
    at = torch.arange(S, device="cuda") % 50
    log(f"[2^31] {pairs} pairs {layout}")
    with torch.no_grad():
        y = hcms.qk_norm_rope(q, None, w, None, table, [50], [pairs], at, layout)
        alone = hcms.qk_norm_rope(q[-n:], None, w, None, table, [50], [pairs], at[-n:], layout)
    assert torch.equal(bits(y[-n:]), bits(alone))
    log("[2^31] backward")

    def dx(x, dy, places):
        x = x.detach().requires_grad_()
        out = hcms.QkNormRope.apply(x, None, w, None, table, [50], [pairs], places, layout)
        return torch.autograd.grad(out, x, dy)[0]

    assert torch.equal(bits(dx(q, y, at)[-n:]), bits(dx(q[-n:], y[-n:], at[-n:])))


def _step(hcms, leaves, table, dq, dk):
    q, k, qw, kw = leaves
    y = hcms.QkNormRope.apply(q, k, qw, kw, table, [50], [32], None, "half", EPS)
    return [*y, *torch.autograd.grad(y, leaves, (dq, dk))]


def test_a_training_step_in_a_graph(hcms):
    """Forward and backward captured and replayed, bit for bit the eager ones; while an
    eager graph of the same leaves is alive the captured backward is refused, and the
    process and the leaves go on."""
    leaves = [_randn(1, 50, 4, 64, dtype=BF16).cuda(), _randn(2, 50, 2, 64, dtype=BF16).cuda(),
              *(1 + 0.3 * _randn(3 + i, 64, dtype=BF16).cuda() for i in (0, 1))]
    leaves = [t.requires_grad_() for t in leaves]
    dq, dk = _randn(5, 50, 4, 64, dtype=BF16).cuda(), _randn(6, 50, 2, 64, dtype=BF16).cuda()
    table = hcms.rope_table([50], [32])
    _step(hcms, leaves, table, dq, dk)
    torch.cuda.synchronize()
    log("[graph] capture")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _step(hcms, leaves, table, dq, dk)
    for i in range(4):
        with torch.no_grad():
            leaves[0].copy_(_randn(10 + i, 50, 4, 64, dtype=BF16))
            dk.copy_(_randn(20 + i, 50, 2, 64, dtype=BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        for a, b in zip(got, _step(hcms, leaves, table, dq, dk)):
            assert torch.equal(bits(a.detach()), bits(b.detach()))
    del out, got, graph, a, b
    log("[graph] beside an eager graph of the leaves")
    alive = hcms.QkNormRope.apply(*leaves, table, [50], [32], None, "half", EPS)
    torch.cuda.synchronize()
    other, flag = torch.cuda.CUDAGraph(), torch.zeros(1, device="cuda")
    with torch.cuda.graph(other):
        flag.add_(1.0)
        with pytest.raises(RuntimeError, match="drop that graph"):
            _step(hcms, leaves, table, dq, dk)
    other.replay()
    torch.cuda.synchronize()
    assert flag.item() == 1.0
    for t in torch.autograd.grad(alive, leaves, (dq, dk)):
        assert torch.isfinite(t).all()


def test_a_captured_training_step_on_two_streams(hcms):
    """Queries and keys made on two streams of one capture, both directions, bit for bit the
    eager step."""
    S, H, Hk, d = 50, 4, 2, 64
    xq, xk = _randn(1, S, H, d).cuda(), _randn(2, S, Hk, d).cuda()
    leaves = [(1 + 0.3 * _randn(3 + i, *shape)).cuda().requires_grad_()
              for i, shape in enumerate(((S, H, d), (S, Hk, d), (d,), (d,)))]
    dq, dk, table = _randn(7, S, H, d).cuda(), _randn(8, S, Hk, d).cuda(), hcms.rope_table([S], [32])
    side = torch.cuda.Stream()

    def step():
        a, b, qw, kw = leaves
        here = torch.cuda.current_stream()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            k = xk * b
        q = xq * a
        here.wait_stream(side)
        y = hcms.QkNormRope.apply(q, k, qw, kw, table, [S], [32], None, "half", EPS)
        out = [q, k, *y, *torch.autograd.grad(y, leaves, (dq, dk))]
        here.wait_stream(side)
        return [t.detach() for t in out]

    want = step()
    torch.cuda.synchronize()
    log("[graph] capture of two streams")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    log("[graph] replays")
    for i in range(4):
        xk.copy_(_randn(20 + i, S, Hk, d))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(bits(a), bits(b))


def test_the_first_capture_of_a_process_refuses_an_eager_graph_s_leaves():
    """In a process of its own, whose first capture has the first of all ids."""
    code = """
import torch
import paper_2607_01817_amd as hcms
x, w = torch.randn(8, 2, 64, device="cuda", requires_grad=True), torch.ones(64, device="cuda", requires_grad=True)
table, flag = hcms.rope_table([8], [32]), torch.zeros(1, device="cuda")
alive = hcms.QkNormRope.apply(x, None, w, None, table, [8], [32])
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    flag.add_(1.0)
    y = hcms.QkNormRope.apply(x, None, w, None, table, [8], [32])
    try:
        torch.autograd.grad(y, (x, w), torch.ones_like(y))
    except RuntimeError as e:
        assert "drop that graph" in str(e), e
        flag.add_(1.0)
graph.replay()
torch.cuda.synchronize()
assert flag.item() == 2.0
"""
    done = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=100,
                          cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert done.returncode == 0, done.stderr[-2000:]

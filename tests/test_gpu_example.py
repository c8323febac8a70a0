"""examples/fp8_block.py, the operators and the chunk loop together, against the same
block in float64 on the CPU.

Tolerances, relative in the Frobenius norm: rounding to e4m3 changes a value by at
most 2^-4 of itself, at most 2^-4 / sqrt(3) = 3.6 % in the mean over a binade, so a
product of two rounded operands by 5.1 % and the block's two products in sequence,
with what the first one changes in the scores counted once more, by 9 %; twice that
is allowed.  A gradient passes the products' transposes as well: 13 %, twice that.
The serving path rounds the norm to 8 bits at once, the training path to bf16 first,
which moves a value in 2^4 by one step of 8 bits: 2^-4 / 2^2 of a product.
"""
import importlib.util
import os
import sys

import pytest
import torch

from paper_2607_01817_amd import inputs
from tests.gpu_util import log

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example(hcms):
    spec = importlib.util.spec_from_file_location("fp8_block", os.path.join(ROOT, "examples", "fp8_block.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def _plain(block, w, x, residual, weights):
    """The block in float64."""
    norm, q_norm, k_norm, w_qkv, w_o = weights

    def rms(t, g):
        return t * torch.rsqrt(t.square().mean(-1, keepdim=True) + block.eps) * g

    h = x + residual
    q, k, v = (rms(h, norm) @ w_qkv.T).view(w.S, 3, w.H, w.d).unbind(1)
    q, k = rms(q, q_norm), rms(k, k_norm)
    coords = torch.cartesian_prod(*[torch.arange(g, dtype=torch.float64) for g in w.grid])
    ang = torch.cat([coords[:, a:a + 1] * w.base ** (-torch.arange(n, dtype=torch.float64) / n)
                     for a, n in enumerate(w.axis_pairs)], 1)[:, None]

    def turn(t):
        a, b = t[..., 0::2], t[..., 1::2]
        return torch.stack((a * ang.cos() - b * ang.sin(), a * ang.sin() + b * ang.cos()), -1).flatten(-2)

    q, k, v = turn(q).transpose(0, 1), turn(k).transpose(0, 1), v.transpose(0, 1)
    p = torch.softmax(q @ k.transpose(1, 2) * w.scale, -1)
    return (p @ v).transpose(0, 1).reshape(w.S, w.H * w.d) @ w_o.T, h


def _far(got, want):
    return ((got.double().cpu() - want).norm() / want.norm()).item()


@pytest.mark.parametrize("name", ["layer_small", "layer_ragged"])
def test_block(example, name):
    w = inputs.LAYERS[name]
    block = example.Block(w.D, w.H, w.d, w.grid, w.axis_pairs, w.chunkings[-1], P=w.P, seed=w.seed)
    g = torch.Generator().manual_seed(w.seed)
    x, residual, dy = (torch.randn(w.S, w.D, generator=g).to(torch.bfloat16) for _ in range(3))
    leaves = [t.detach().double().requires_grad_() for t in (x, residual, *(p.cpu() for p in (
        block.norm, block.q_norm, block.k_norm, block.w_qkv, block.w_o)))]
    want, want_h = _plain(block, w, leaves[0], leaves[1], leaves[2:])
    want.backward(dy.double())

    served, h = block.prepare().serve(x.cuda(), residual.cuda())
    xg, rg = x.cuda().requires_grad_(), residual.cuda().requires_grad_()
    y, _ = block.train_forward(xg, rg)
    y.backward(dy.cuda())
    log(f"[block] {name}: serving {_far(served, want.detach()):.4f}, training {_far(y.detach(), want.detach()):.4f}, "
        f"apart {_far(served, y.detach().double().cpu()):.4f}")
    assert _far(h, want_h.detach()) <= 2.0 ** -8
    assert _far(served, want.detach()) <= 0.18 and _far(y.detach(), want.detach()) <= 0.18
    assert _far(served, y.detach().double().cpu()) <= 0.0625
    got = [xg.grad, rg.grad] + [p.grad for p in (block.norm, block.q_norm, block.k_norm, block.w_qkv, block.w_o)]
    for n, a, b in zip(("x", "residual", "norm", "q_norm", "k_norm", "w_qkv", "w_o"), got, leaves):
        log(f"[block] {name}: gradient of {n} {_far(a, b.grad):.4f}")
        assert _far(a, b.grad) <= 0.26, n


def test_training_lowers_the_loss(example, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["fp8_block.py", "--steps", "10"])
    example.main()
    lines = capsys.readouterr().out.splitlines()
    first, last = (float(ln.split()[-1]) for ln in lines[:2])
    assert last < first, lines

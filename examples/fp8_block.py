"""An attention block with its norms and 8-bit projections around the chunk loop.

    python examples/fp8_block.py [--workload layer_small|layer_wan_p8] [--steps N]

One pre-norm block of a residual stream, as one GPU of a sequence-parallel group
holds it: D-wide tokens, H local heads of dimension d.

    h     = x + residual                     the residual stream's next value
    q,k,v = norm(h) w_qkv                    8-bit product
    q, k  = rope(norm(q)), rope(norm(k))     norms of each head vector
    y     = attention(q, k, v) w_o           chunk loop, 8-bit product

``serve`` quantises the weights once and each activation where it is made (the
norm writes 8 bits itself); ``train`` runs the same block through autograd, where
the products of both directions are in 8 bits.
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2607_01817_amd as hcms  # noqa: E402
from paper_2607_01817_amd import inputs  # noqa: E402


class Block(torch.nn.Module):
    def __init__(self, D, H, d, grid, axis_pairs, chunk_sizes, P=1, eps=1e-6, seed=0):
        super().__init__()
        self.D, self.H, self.d, self.eps = D, H, d, eps
        self.grid, self.axis_pairs, self.chunk_sizes, self.P = grid, axis_pairs, chunk_sizes, P
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(n, k):
            w = torch.randn(n, k, generator=g, device="cuda") / k ** 0.5
            return torch.nn.Parameter(w.to(torch.bfloat16))

        def ones(n):
            return torch.nn.Parameter(torch.ones(n, dtype=torch.bfloat16, device="cuda"))

        self.norm, self.q_norm, self.k_norm = ones(D), ones(d), ones(d)
        self.w_qkv, self.w_o = weight(3 * H * d, D), weight(D, H * d)
        self.table = hcms.rope_table(grid, axis_pairs)
        self.ctx = hcms.Context()
        self.scale = d ** -0.5

    def prepare(self):
        """The weights in 8 bits, for ``serve`` (again after they have changed)."""
        with torch.no_grad():
            self.qkv8 = hcms.quantize_fp8(self.w_qkv, 128)
            self.o8 = hcms.quantize_fp8(self.w_o, 128)
        return self

    @torch.no_grad()
    def serve(self, x, residual):
        """(y, h) of x and residual [S][D]."""
        S, H, d = x.shape[0], self.H, self.d
        n, n_scale, h = hcms.rms_norm_fp8(x, self.norm, self.eps, residual=residual)
        q, k, v = hcms.linear_fp8(n, n_scale, *self.qkv8, parts=3)
        q = hcms.rms_norm(q.view(S * H, d), self.q_norm, self.eps).view(S, H, d)
        k = hcms.rms_norm(k.view(S * H, d), self.k_norm, self.eps).view(S, H, d)
        hcms.rope(q, k, self.table, self.grid, self.axis_pairs, out=(q, k))
        o = self.ctx.forward(q, k, v.view(S, H, d), self.P, self.scale, self.chunk_sizes)
        return hcms.linear_fp8(*hcms.quantize_fp8(o.view(S, H * d)), *self.o8), h

    def train_forward(self, x, residual):
        """The same with gradients of x, residual and the weights."""
        S, H, d = x.shape[0], self.H, self.d
        n, h = hcms.RmsNorm.apply(x, self.norm, self.eps, residual)
        q, k, v = hcms.Fp8Linear.apply(n, self.w_qkv).view(S, 3, H, d).unbind(1)
        q = hcms.RmsNorm.apply(q.reshape(S * H, d), self.q_norm, self.eps).view(S, H, d)
        k = hcms.RmsNorm.apply(k.reshape(S * H, d), self.k_norm, self.eps).view(S, H, d)
        q, k = hcms.Rope.apply(q, k, self.table, self.grid, self.axis_pairs)
        o = hcms.HcmsAttention.apply(q, k, v, self.ctx, self.P, self.scale, self.chunk_sizes)
        return hcms.Fp8Linear.apply(o.view(S, H * d), self.w_o), h


def time_ms(fn, reps):
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    fn()
    a.record()
    for _ in range(reps):
        fn()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / reps


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="layer_small", choices=sorted(w for w in inputs.LAYERS if w != "layer_fp32"))
    ap.add_argument("--steps", type=int, default=20)
    args = ap.parse_args()
    w = inputs.LAYERS[args.workload]
    block = Block(w.D, w.H, w.d, w.grid, w.axis_pairs, hcms.default_chunks(w.H, min(3, w.H)), seed=w.seed)
    g = torch.Generator(device="cuda").manual_seed(w.seed + 1)
    x, residual, target = (torch.randn(w.S, w.D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))

    opt = torch.optim.SGD(block.parameters(), lr=0.5)
    for step in range(args.steps):
        opt.zero_grad()
        y, _ = block.train_forward(x, residual)
        loss = (y - target).float().square().mean()
        loss.backward()
        opt.step()
        if step in (0, args.steps - 1):
            print(f"step {step}: loss {loss.item():.4f}", flush=True)

    y, h = block.prepare().serve(x, residual)
    with torch.no_grad():
        t, _ = block.train_forward(x, residual)
    print(f"serving and training forward differ by {((y - t).float().norm() / t.float().norm()).item():.1e}")
    print(f"{w.name}: S={w.S} D={w.D} H={w.H}: serving {time_ms(lambda: block.serve(x, residual), 5):.3f} ms, "
          f"chunk loop with bf16 projections alone "
          f"{time_ms(lambda: block.ctx.layer_forward(x, block.w_qkv.data, block.w_o.data, 1, w.H, w.d, block.scale, block.chunk_sizes, block.table, w.grid, w.axis_pairs), 5):.3f} ms")


if __name__ == "__main__":
    main()

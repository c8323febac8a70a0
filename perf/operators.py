"""Timed cases of the operators around the chunk loop of an 8-bit attention layer.

The layer reads the residual stream through a root-mean-square norm, projects it in 8-bit floating
point, rotates queries and keys by their positions, runs the chunk loop and projects back.  The
operators are the norm, the 8-bit product with its quantisation, and the rotation, each forward and
backward.  A case is a dict of plain values; ``kind`` names the calls:

  norm          rms_norm: the residual's addition and the norm, in the storage type
  norm_train    RmsNorm: the same through autograd, with the gradients of x, residual and weight
  norm_linear   rms_norm_fp8 into linear_fp8: the norm's 8-bit output and the projection that reads it
  linear        linear_fp8 on operands that are held in 8 bits
  linear_train  Fp8Linear: a projection and its two gradients, all three products in 8 bits
  rope          rope on queries and keys that are views of one projection's output
  rope_train    Rope: the same through autograd

M tokens, D the model width (what a norm runs over), N and K a projection's output and input width,
H query heads and Hk key heads of dimension d of which the first R elements turn.  8 bits are e4m3
(float8_e4m3fn) with a scale for each block: of 128 consecutive k of one token, or of 128 x 128 of a
weight.  Scales are powers of two, held as their exponent (float8_e8m0fnu), the smallest that brings
the block's magnitudes to at most 448; four blocks' exponents lie side by side, in the shape
[groups of four blocks][tokens, or weight blocks][4].  Activations are standard normal times a per-channel gain, weights standard
normal over the square root of their input width, norm weights near 1, output gradients standard
normal.

Where ``own`` is false the plain forms run: elementary torch operations in float32.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
BASE = 10000.0       # base of the rotary frequencies
BLOCK = 128          # elements that share a scale
FP8_MAX = 448.0      # largest finite e4m3 value


def listed():
    return [
        # One token through a full-width norm with the residual: the smallest call, all latency.
        dict(name="norm_token", kind="norm", M=1, D=5120, dtype="bf16", residual=True),
        # The flagship's tokens (36 latent frames of 1560) through the norm in front of a layer.
        dict(name="norm_wan", kind="norm", M=56160, D=5120, dtype="bf16", residual=True),
        # A training step's norm of a 5-frame clip at the model width.
        dict(name="norm_train_clip", kind="norm_train", M=7800, D=5120, dtype="bf16", residual=True),
        # A still image (one latent frame): the norm in 8 bits and the QKV projection of 5 heads.
        dict(name="norm_qkv_image", kind="norm_linear", M=1560, D=5120, N=1920, dtype="bf16",
             residual=True, parts=3),
        # One token through a full-width projection: the weight's bytes count.
        dict(name="linear_token", kind="linear", M=1, N=5120, K=5120, dtype="bf16", parts=1),
        # One frame through a full-width projection.
        dict(name="linear_image", kind="linear", M=1560, N=5120, K=5120, dtype="bf16", parts=1),
        # The flagship's QKV projection, split into queries, keys and values: the largest product.
        dict(name="linear_wan_qkv", kind="linear", M=56160, N=1920, K=5120, dtype="bf16", parts=3),
        # Odd sizes: tokens, columns and the last block of k end inside a tile; fp32 output.
        dict(name="linear_ragged", kind="linear", M=3001, N=1000, K=1936, dtype="fp32", parts=1),
        # A clip's QKV projection in training: quantisation, three products, both gradients.
        dict(name="linear_train_clip", kind="linear_train", M=7800, N=1920, K=5120, dtype="bf16"),
        # Eight sequences' next tokens far out in a long context: halves layout, 40 query heads on
        # 8 key heads, frequencies interpolated by parts.
        dict(name="rope_tokens", kind="rope", M=8, H=40, Hk=8, d=128, R=128, layout="half",
             dtype="bf16", n=131072, scaling="yarn", grid=""),
        # The flagship's queries and keys on the latent grid, 5 heads, row-major positions.
        dict(name="rope_wan", kind="rope", M=56160, H=5, Hk=5, d=128, R=128, layout="interleaved",
             dtype="bf16", n=0, scaling="none", grid="36,30,52"),
        # Training at an odd length: half of a head of 64 turns, shared key heads, fp32.
        dict(name="rope_train_ragged", kind="rope_train", M=7801, H=16, Hk=2, d=64, R=32,
             layout="half", dtype="fp32", n=16384, scaling="linear", grid=""),
    ]


# ---------------------------------------------------------------------------
# Sizes
# ---------------------------------------------------------------------------
def _ints(text):
    return [int(x) for x in text.split(",")]


def _grid(case):
    """The position grid: the case's, or one axis of n positions."""
    return _ints(case["grid"]) if case["grid"] else [case["n"]]


def _pairs(case):
    """The R / 2 pairs of a head vector in one group per axis, larger groups first."""
    n, p = len(_grid(case)), case["R"] // 2
    return [p // n + (1 if a < p % n else 0) for a in range(n)]


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    k, M = case["kind"], case["M"]
    if k in ("norm", "norm_train"):
        x, r = e * M * case["D"], 1 if case["residual"] else 0
        fwd, w = x * (2 + 2 * r), e * case["D"]
        if k == "norm":
            return {"bytes": fwd + w, "flops": 6 * M * case["D"]}
        # the output's and the residual stream's gradients and the stream in, its gradient out
        return {"bytes": fwd + x * (3 + r) + 3 * w, "flops": 20 * M * case["D"]}
    if k in ("rope", "rope_train"):
        both = 2 if k == "rope_train" else 1
        x = e * M * (case["H"] + case["Hk"]) * case["d"]
        entries = sum(g * p for g, p in zip(_grid(case), _pairs(case)))
        return {"bytes": both * (2 * x + 8 * min(entries, M * case["R"] // 2)), "flops": both * 3 * x / e}
    N, K = case["N"], case.get("K", case.get("D"))
    kb = math.ceil(K / BLOCK)
    held = M * K + N * K + kb * (M + math.ceil(N / BLOCK))
    if k == "linear":
        return {"bytes": held + e * M * N, "flops": 2 * M * N * K}
    if k == "norm_linear":
        x = e * M * K * (3 if case["residual"] else 1)
        return {"bytes": x + e * K + N * K + kb * math.ceil(N / BLOCK) + e * M * N,
                "flops": 2 * M * N * K}
    # x, w and the output's gradient in, the output and two gradients out
    return {"bytes": 2 * e * (M * K + N * K + M * N), "flops": 6 * M * N * K}


def draw(rng):
    """One more case: each kind as often as the others, lengths spread over their logarithm from
    one token on, widths over those of 1 to 40 heads of 64 or 128 and ragged ones beside them."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(ragged=0):
        w = rng.choice((1, 2, 3, 4, 5, 8, 10, 13, 20, 40)) * rng.choice((64, 128))
        return w + (ragged * rng.randint(1, 7) if ragged and rng.random() < 0.4 else 0)

    kind = rng.choice(("norm", "norm_train", "norm_linear", "linear", "linear_train", "rope",
                       "rope_train"))
    top = {n: max(work(c)[n] for c in listed()) for n in ("flops", "bytes")}
    while True:
        case = dict(kind=kind, M=log(1, 60000), dtype=rng.choice(("bf16", "bf16", "fp32")))
        if kind in ("norm", "norm_train"):
            case.update(D=width(1), residual=rng.random() < 0.7)
        elif kind == "norm_linear":
            # fp32 storage of an 8-bit norm's projection would compare 8-bit roundings at 32 bits
            case.update(D=width(16), N=width(8), dtype="bf16", residual=rng.random() < 0.7, parts=1)
        elif kind == "linear":
            case.update(N=width(8), K=width(16), parts=1)
            if case["N"] % 24 == 0:
                case.update(parts=rng.choice((1, 3)))
        elif kind == "linear_train":
            # widths of 16, so that each of the three products has whole 16-byte rows
            case.update(N=width(16), K=width(16), dtype="bf16")
        else:
            d = rng.choice((64, 128))
            H = rng.choice((1, 2, 3, 4, 5, 8, 10, 13, 20, 40))
            case.update(H=H, Hk=rng.choice([h for h in (1, 2, 4, 5, 8, 10, 20, 40) if H % h == 0]),
                        d=d, R=rng.choice((d, d, d // 2, d // 4)),
                        layout=rng.choice(("half", "interleaved")),
                        n=rng.choice((4096, 16384, 131072)), grid="",
                        scaling=rng.choice(("none", "linear", "ntk", "yarn")))
            if rng.random() < 0.3:
                grid = (rng.randint(1, 36), rng.randint(4, 40), rng.randint(4, 52))
                case.update(M=math.prod(grid), grid=",".join(map(str, grid)), n=0, scaling="none")
        w = work(case)
        # half of the bytes: the plain forms of quantisation and gradients move more for the same work
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] / 2:
            return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _randn(g, shape, by=1.0):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    return x if by == 1.0 else x * by


def _tokens(g, M, D, dtype):
    """Activations: standard normal, each channel with a gain of its own."""
    gain = torch.exp(0.5 * _randn(g, (D,)))
    return (_randn(g, (M, D)) * gain).to(dtype)


def _scales(amax):
    """The exponent byte of the smallest power of two s with amax <= 448 s, at least 2^-126, and 1 / s."""
    e = ((amax.view(torch.int32) + 0x1FFFFF >> 23) - 8).clamp_min(1)   # 448 = 1.75 * 2^8
    return e, (254 - e << 23).view(torch.float32)


def _held_scales(e):
    """Exponents [rows][blocks] as the scale operand [groups][rows][4], padded with ones."""
    e = torch.nn.functional.pad(e, (0, -e.shape[1] % 4), value=127).to(torch.uint8)
    return e.unflatten(1, (-1, 4)).transpose(0, 1).contiguous().view(torch.float8_e8m0fnu)


def _rows8(x):
    """e4m3 values of x and the exponents [M][blocks] of their scales, one per token and 128 k."""
    M, K = x.shape
    xb = torch.nn.functional.pad(x.float(), (0, -K % BLOCK)).reshape(M, -1, BLOCK)
    e, by = _scales(xb.abs().amax(-1))
    q = (xb * by[..., None]).to(torch.float8_e4m3fn)
    return q.view(M, -1)[:, :K].contiguous(), e


def _blocks8(w):
    """e4m3 values of w and the exponents [N blocks][K blocks] of their scales, one per 128 x 128."""
    N, K = w.shape
    wb = torch.nn.functional.pad(w.float(), (0, -K % BLOCK, 0, -N % BLOCK))
    wb = wb.reshape(-(-N // BLOCK), BLOCK, -(-K // BLOCK), BLOCK)
    e, by = _scales(wb.abs().amax((1, 3)))
    q = (wb * by[:, None, :, None]).to(torch.float8_e4m3fn)
    return q.view(wb.shape[0] * BLOCK, -1)[:N, :K].contiguous(), e


def _freqs(case):
    """Turns per position of each pair, in float64, and the table's magnitude."""
    kind, factor, length = case["scaling"], 8.0, case["n"] / 8.0
    out, mag = [], 1.0
    for p in _pairs(case):
        i = torch.arange(p, device="cuda", dtype=torch.float64)
        base = BASE * factor ** (p / (p - 1.0)) if kind == "ntk" and p > 1 else BASE
        f = base ** (-i / p)
        if kind == "linear":
            f = f / factor
        elif kind == "yarn":
            # pairs that turn more than 32 times over the trained length keep their frequency, those
            # that turn less than once are slowed by the factor, those between are mixed
            at = [p * math.log(length / (2 * math.pi * r)) / math.log(BASE) for r in (32.0, 1.0)]
            lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), p - 1)
            keep = 1.0 - ((i - lo) / max(hi - lo, 1e-3)).clamp(0.0, 1.0)
            f = f * keep + f / factor * (1.0 - keep)
            mag = 0.1 * math.log(factor) + 1.0
        out.append(f)
    return out, mag


def _table(case):
    """The rotation table a program keeps: (magnitude cos, magnitude sin) of every axis, coordinate
    and pair, axis by axis, float32 [entries][2]."""
    freqs, mag = _freqs(case)
    rows = []
    for n, f in zip(_grid(case), freqs):
        a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * f
        rows.append(torch.stack((a.cos(), a.sin()), -1).mul(mag).float().view(-1, 2))
    return torch.cat(rows).contiguous()


def _inputs(case, seed):
    """The case's input tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    k, M, dt = case["kind"], case["M"], DTYPES[case["dtype"]]
    t = {}
    if k in ("norm", "norm_train", "norm_linear"):
        D = case["D"]
        t["x"] = _tokens(g, M, D, dt)
        t["residual"] = _tokens(g, M, D, dt) if case["residual"] else None
        t["weight"] = (1.0 + 0.1 * _randn(g, (D,))).to(dt)
        if k == "norm_train":
            t["dy"] = _randn(g, (M, D)).to(dt)
            t["dh"] = _randn(g, (M, D)).to(dt) if case["residual"] else None
    if k in ("linear", "linear_train"):
        t["x"] = _tokens(g, M, case["K"], dt)
    if "N" in case:
        K = case.get("K", case.get("D"))
        t["w"] = _randn(g, (case["N"], K), K ** -0.5).to(dt)
        if k == "linear_train":
            t["dy"] = _randn(g, (M, case["N"])).to(dt)
        else:
            t["w8"], e = _blocks8(t.pop("w"))
            t["w_scale"] = _held_scales(e)
    if k == "linear":
        t["x8"], e = _rows8(t.pop("x"))
        t["x_scale"] = _held_scales(e)
    if k in ("rope", "rope_train"):
        H, Hk, d = case["H"], case["Hk"], case["d"]
        t["qkv"] = _randn(g, (M, (H + 2 * Hk) * d)).to(dt)
        t["positions"] = None
        if not case["grid"]:
            first = max(0, case["n"] - M) if k == "rope" else 0
            at = torch.randint(0, case["n"], (M,), generator=g, device="cuda")
            # new tokens of as many sequences, or one sequence from a place of its own on
            at = at if M < 64 else (at[:1] % (first + 1) + torch.arange(M, device="cuda")) % case["n"]
            t["positions"] = at.to(torch.int32)
        if k == "rope_train":
            t["dq"], t["dk"] = _randn(g, (M, H, d)).to(dt), _randn(g, (M, Hk, d)).to(dt)
    return t


def prepare(case, seed):
    t = _inputs(case, seed)
    s = dict(case, t=t)
    if case["kind"] in ("rope", "rope_train"):
        s["table"], s["dims"], s["pairs"] = _table(case), _grid(case), _pairs(case)
        H, Hk, d = case["H"], case["Hk"], case["d"]
        s["q"] = t["qkv"][:, :H * d].unflatten(1, (H, d))
        s["k"] = t["qkv"][:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
        # for the plain form: each pair's axis, entry of coordinate 0, and the axis's pairs and stride
        ax = torch.tensor([a for a, p in enumerate(s["pairs"]) for _ in range(p)], device="cuda")
        off = [sum(g * p for g, p in zip(s["dims"][:a], s["pairs"][:a])) for a in range(len(s["dims"]))]
        s["entry"] = torch.tensor([o + i for o, p in zip(off, s["pairs"]) for i in range(p)], device="cuda")
        s["step"] = torch.tensor(s["pairs"], device="cuda")[ax]
        s["stride"] = torch.tensor([math.prod(s["dims"][a + 1:]) for a in range(len(s["dims"]))], device="cuda")[ax]
        s["size"] = torch.tensor(s["dims"], device="cuda")[ax]
    if case["kind"].endswith("_train"):
        s["leaves"] = [t[n] for n in ("x", "residual", "weight", "w") if t.get(n) is not None]
        if case["kind"] == "rope_train":
            s["q"], s["k"] = s["q"].detach(), s["k"].detach()
            s["leaves"] = [s["q"], s["k"]]
        for x in s["leaves"]:
            x.requires_grad_(True)
    return s


# ---------------------------------------------------------------------------
# Plain forms: elementary operations in float32
# ---------------------------------------------------------------------------
def _norm(x, residual, weight):
    h = x.float() if residual is None else x.float() + residual.float()
    r = torch.rsqrt((h * h).mean(-1, keepdim=True) + EPS)
    return h, r, h * r * weight.float()


def _two_to(e, K):
    """Scales from exponents [rows][blocks] or a scale operand, each for the 128 k of its block."""
    if e.dtype == torch.float8_e8m0fnu:
        e = e.view(torch.uint8).transpose(0, 1).flatten(1)
    return (e.int() << 23).view(torch.float32).repeat_interleave(BLOCK, 1)[:, :K]


def _dequant_rows(q, e):
    return q.float() * _two_to(e, q.shape[1])


def _dequant_blocks(q, e):
    return q.float() * _two_to(e, q.shape[1]).repeat_interleave(BLOCK, 0)[:q.shape[0]]


def _parts(y, parts):
    return y if parts == 1 else y.unflatten(1, (parts, -1)).transpose(0, 1).contiguous()


def _turn(x, cos, sin, R, layout):
    """The first R elements of each head rotated, the others as they are."""
    x = x.float()
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if layout == "interleaved" else (x[..., :R // 2], x[..., R // 2:R])
    u, v = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((u, v), -1).flatten(-2) if layout == "interleaved" else torch.cat((u, v), -1)
    return torch.cat((y, x[..., R:]), -1)


def _cos_sin(s):
    """(cos, sin) [M][1][R / 2] of the tokens' positions."""
    at = s["t"]["positions"]
    if at is None:
        c = torch.arange(s["M"], device="cuda")[:, None] // s["stride"] % s["size"]
    else:
        c = at.long()[:, None]
    cs = s["table"][s["entry"] + c * s["step"]][:, None]
    return cs[..., 0], cs[..., 1]


def _plain(s):
    t, k, dt = s["t"], s["kind"], DTYPES[s["dtype"]]
    if k == "norm":
        h, _, y = _norm(t["x"], t["residual"], t["weight"])
        return (y.to(dt), h.to(dt)) if s["residual"] else y.to(dt)
    if k == "norm_train":
        h, r, y = _norm(t["x"], t["residual"], t["weight"])
        dy, n = t["dy"].float(), h * r
        g = dy * t["weight"].float()
        dx = r * (g - n * (g * n).mean(-1, keepdim=True))
        dw = (dy * n).sum(0).to(dt)
        if not s["residual"]:
            return y.to(dt), dx.to(dt), dw
        dx = (dx + t["dh"].float()).to(dt)
        return y.to(dt), h.to(dt), dx, dx, dw
    if k == "norm_linear":
        h, _, y = _norm(t["x"], t["residual"], t["weight"])
        y = _parts((_dequant_rows(*_rows8(y)) @ _dequant_blocks(t["w8"], t["w_scale"]).t()).to(dt), s["parts"])
        return (y, h.to(dt)) if s["residual"] else y
    if k == "linear":
        y = _dequant_rows(t["x8"], t["x_scale"]) @ _dequant_blocks(t["w8"], t["w_scale"]).t()
        return _parts(y.to(dt), s["parts"])
    if k == "linear_train":
        x, w, dy = t["x"], t["w"], t["dy"]
        w8 = _dequant_blocks(*_blocks8(w))
        y = _dequant_rows(*_rows8(x)) @ w8.t()
        dx = _dequant_rows(*_rows8(dy)) @ w8
        dw = _dequant_rows(*_rows8(dy.t())) @ _dequant_blocks(*_blocks8(x.t())).t()
        return y.to(dt), dx.to(dt), dw.to(dt)
    cos, sin = _cos_sin(s)
    out = [_turn(x, cos, sin, s["R"], s["layout"]).to(dt) for x in (s["q"], s["k"])]
    if k == "rope_train":
        out += [_turn(x, cos, -sin, s["R"], s["layout"]).to(dt) for x in (t["dq"], t["dk"])]
    return tuple(out)


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    if not own:
        with torch.no_grad():
            return _plain(s)
    import paper_2607_01817_amd as hcms
    t, k = s["t"], s["kind"]
    if k == "norm":
        return hcms.rms_norm(t["x"], t["weight"], EPS, residual=t["residual"])
    if k == "norm_train":
        out = hcms.RmsNorm.apply(t["x"], t["weight"], EPS, t["residual"])
        if not s["residual"]:
            return (out.detach(), *torch.autograd.grad(out, (t["x"], t["weight"]), t["dy"]))
        dx, dr, dw = torch.autograd.grad(out, (t["x"], t["residual"], t["weight"]), (t["dy"], t["dh"]))
        return out[0].detach(), out[1].detach(), dx, dr, dw
    if k == "norm_linear":
        q, scale, *h = hcms.rms_norm_fp8(t["x"], t["weight"], EPS, residual=t["residual"])
        y = hcms.linear_fp8(q, scale, t["w8"], t["w_scale"], parts=s["parts"])
        return (y, *h) if h else y
    if k == "linear":
        return hcms.linear_fp8(t["x8"], t["x_scale"], t["w8"], t["w_scale"], dtype=DTYPES[s["dtype"]],
                               parts=s["parts"])
    if k == "linear_train":
        y = hcms.Fp8Linear.apply(t["x"], t["w"])
        return (y.detach(), *torch.autograd.grad(y, (t["x"], t["w"]), t["dy"]))
    if k == "rope":
        return hcms.rope(s["q"], s["k"], s["table"], s["dims"], s["pairs"], positions=t["positions"],
                         layout=s["layout"])
    q, kk = hcms.Rope.apply(s["q"], s["k"], s["table"], s["dims"], s["pairs"], t["positions"], s["layout"])
    return (q.detach(), kk.detach(), *torch.autograd.grad((q, kk), (s["q"], s["k"]), (t["dq"], t["dk"])))


# ---------------------------------------------------------------------------
# 64-bit results from the definitions
# ---------------------------------------------------------------------------
def _two64(e):
    """2^e in float64, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _e4m3(x):
    """Round to 3 bits behind the leading one, from 2^-9 on, ties to even."""
    _, e = torch.frexp(x)
    step = _two64((e - 1).clamp_min(-6) - 3)
    return (x / step).round().mul(step).clamp(-FP8_MAX, FP8_MAX)


def _held(x, rows):
    """The values that x's 8-bit form stands for, blocks of rows x 128."""
    out = torch.empty_like(x)
    for j in range(0, x.shape[1], BLOCK):
        c = x[:, j:j + BLOCK]
        if rows == 1:
            top = c.abs().amax(1, keepdim=True)
        else:
            top = torch.cat([b.abs().max().expand(b.shape[0], 1) for b in c.split(rows)])
        m, e = torch.frexp(top)   # 448 = 0.875 * 2^9
        s = _two64((e - 9 + (m > 0.875).int()).clamp_min(-126))
        out[:, j:j + BLOCK] = _e4m3(c / s) * s
    return out


def _rotated64(x, angle, mag, R, layout):
    x = x.double()
    if layout == "interleaved":
        z = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous())
    else:
        z = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous())
    z = z * torch.polar(torch.full_like(angle, mag), angle)[:, None]
    y = torch.view_as_real(z).flatten(-2) if layout == "interleaved" else torch.cat((z.real, z.imag), -1)
    return torch.cat((y, x[..., R:]), -1)


def exact(case, seed):
    t, k = _inputs(case, seed), case["kind"]
    if k in ("norm", "norm_train", "norm_linear"):
        x = t["x"].double()
        h = x if t["residual"] is None else x + t["residual"].double()
        h = h.requires_grad_(k == "norm_train")
        w = t["weight"].double().requires_grad_(k == "norm_train")
        y = h / (h.square().sum(1, keepdim=True) / case["D"] + EPS).sqrt() * w
        if k == "norm":
            return (y, h) if case["residual"] else y
        if k == "norm_train":
            dx, dw = torch.autograd.grad(y, (h, w), t["dy"].double())
            if not case["residual"]:
                return y.detach(), dx, dw
            dx = dx + t["dh"].double()
            return y.detach(), h.detach(), dx, dx, dw
        t["x8"] = _held(y, 1)
    if k == "linear_train":
        x, w, dy = (t[n].double() for n in ("x", "w", "dy"))
        w = _held(w, BLOCK)
        return (_held(x, 1) @ w.T, _held(dy, 1) @ w,
                _held(dy.T.contiguous(), 1) @ _held(x.T.contiguous(), BLOCK).T)
    if k in ("linear", "norm_linear"):
        y = None
        for j in range(-(-t["w8"].shape[1] // BLOCK)):
            c = slice(j * BLOCK, (j + 1) * BLOCK)
            a, b = t["x8"][:, c].double(), t["w8"][:, c].double()
            if k == "linear":
                a = a * _two64(t["x_scale"].view(torch.uint8)[j // 4, :, j % 4].int() - 127)[:, None]
            by = _two64(t["w_scale"].view(torch.uint8)[j // 4, :, j % 4].int() - 127)
            b = b * by.repeat_interleave(BLOCK)[:b.shape[0], None]
            y = a @ b.T if y is None else y.addmm_(a, b.T)
        y = _parts(y, case["parts"])
        return (y, h) if k == "norm_linear" and case["residual"] else y
    H, Hk, d, R = case["H"], case["Hk"], case["d"], case["R"]
    freqs, mag = _freqs(case)
    rest, coords = torch.arange(case["M"], device="cuda"), []
    for n in reversed(_grid(case)):
        coords.insert(0, rest % n)
        rest = rest // n
    if t["positions"] is not None:
        coords = [t["positions"]]
    angle = torch.cat([c.double()[:, None] * f for c, f in zip(coords, freqs)], 1)
    q, kk = t["qkv"][:, :H * d].unflatten(1, (H, d)), t["qkv"][:, H * d:(H + Hk) * d].unflatten(1, (Hk, d))
    out = [_rotated64(x, angle, mag, R, case["layout"]) for x in (q, kk)]
    if k == "rope_train":
        out += [_rotated64(t[n], -angle, mag, R, case["layout"]) for n in ("dq", "dk")]
    return tuple(out)

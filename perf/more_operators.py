"""Timed cases of attention over a paged cache held in 4 bits, of what fills that cache, and of the
norm and rotation of query and key heads in one pass.

A rolling sequence keeps its past keys and values in a paged cache.  Each step norms and rotates the
heads of the new tokens, appends their keys and values to the cache and attends over it.  A case is a
dict of plain values; ``kind`` names the calls:

  norm_rope         qk_norm_rope: each query and key head vector normed and turned by its position
  norm_rope_train   QkNormRope: the same through autograd, with the gradients of the heads and weights
  append            append_kv: keys turned by their positions, keys and values into the cache in 4 bits,
                    and the values that the cache now holds for them
  attend            cache_attention: the new tokens' queries over the cache
  step              append_kv and then cache_attention, as a step of serving makes them

H query heads and Hk key heads of dimension d, of which the first R elements turn.  A batch of B
sequences: each brings up to ``new`` tokens on top of up to ``context`` that are cached already
(``ragged``: from none on, else all alike).  The tokens lie packed, sequence behind sequence.

4 bits are e2m1 values (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with a scale for each 32
consecutive elements of a head vector: the smallest power of two, from 2^-126 on, that brings their
magnitudes to at most 6, held as its exponent (float8_e8m0fnu); values are rounded to the nearest,
ties to the even code.  A page holds ``page`` tokens of each key head, in chunks of 64:

  k        [pages][Hk][page][d / 2]            two elements in a byte, the first in the low half
  k_scale  [pages][Hk][page / 64][d / 32][64]  token t of a chunk at 4 (t % 16) + t // 16
  v        [pages][Hk][page / 64][d / 2][64]   token t at 16 (t // 4 % 4) + 4 (t // 16) + t % 4
  v_scale  [pages][Hk][page / 64][d / 32][64]  token t as in v

Where ``own`` is false the plain forms run: elementary torch operations in float32, and in float64
what is next to a border of the 4-bit values.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
EPS = 1e-6
BASE = 10000.0                                    # base of the rotary frequencies
BLOCK, CHUNK = 32, 64                             # elements that share a scale; tokens of a chunk
GRID4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of the 4-bit codes


def listed():
    return [
        # One token's heads, far out in a long context: the smallest call, all latency.
        dict(name="norm_rope_token", kind="norm_rope", M=1, H=40, Hk=8, d=128, R=128, layout="half",
             dtype="bf16", grid="131072"),
        # The flagship's queries and keys on the latent grid, 5 heads.
        dict(name="norm_rope_wan", kind="norm_rope", M=56160, H=5, Hk=5, d=128, R=128,
             layout="interleaved", dtype="bf16", grid="36,30,52"),
        # Training on a clip of 5 latent frames, all 40 heads.
        dict(name="norm_rope_train_clip", kind="norm_rope_train", M=7800, H=40, Hk=40, d=128, R=128,
             layout="interleaved", dtype="bf16", grid="5,30,52"),
        # Training at an odd length: half of a head of 64 turns, shared key heads, fp32.
        dict(name="norm_rope_train_ragged", kind="norm_rope_train", M=7801, H=16, Hk=2, d=64, R=32,
             layout="half", dtype="fp32", grid="16384"),
        # One latent frame behind 35 others on the grid: the keys and values of 40 heads.
        dict(name="append_frame", kind="append", B=1, new=1560, context=54600, ragged=False, lay=1,
             Hk=40, d=128, R=128, layout="interleaved", dtype="bf16", page=64, grid="36,30,52"),
        # Prompts of many lengths, some empty, onto caches of any fill: fp32, a part of the head turns.
        dict(name="append_ragged", kind="append", B=29, new=701, context=1003, ragged=True, lay=2,
             Hk=3, d=64, R=32, layout="half", dtype="fp32", page=128, grid="2048"),
        # One sequence's next token on a short context: latency.
        dict(name="step_token", kind="step", B=1, new=1, context=1000, ragged=False, lay=3, H=40, Hk=8,
             d=128, R=128, layout="half", dtype="bf16", page=64, grid="131072", causal=True, window=0),
        # Next tokens of 64 sequences of many lengths.
        dict(name="step_batch", kind="step", B=64, new=1, context=8191, ragged=True, lay=4, H=40, Hk=8,
             d=128, R=128, layout="half", dtype="bf16", page=64, grid="131072", causal=True, window=0),
        # Two sequences far out in a long context: work is split along the cache.
        dict(name="step_long", kind="step", B=2, new=1, context=131071, ragged=False, lay=5, H=40, Hk=8,
             d=128, R=128, layout="half", dtype="bf16", page=256, grid="131072", causal=True, window=0),
        # A new latent frame's queries over the whole rolling cache, frame included: the largest product.
        dict(name="attend_frame", kind="attend", B=1, new=1560, context=54600, ragged=False, lay=6, H=5,
             Hk=5, d=128, dtype="bf16", page=64, causal=False, window=0),
        # A prompt's next pieces, causal, with shared key heads.
        dict(name="attend_chunk", kind="attend", B=2, new=2048, context=14336, ragged=False, lay=7, H=40,
             Hk=8, d=128, dtype="bf16", page=64, causal=True, window=0),
        # Pieces of many lengths, some empty, in a sliding window: fp32, odd numbers everywhere.
        dict(name="attend_ragged", kind="attend", B=11, new=333, context=4001, ragged=True, lay=8, H=9,
             Hk=3, d=64, dtype="fp32", page=192, causal=True, window=1001),
    ]


# ---------------------------------------------------------------------------
# Sizes
# ---------------------------------------------------------------------------
def _grid(case):
    return [int(x) for x in case["grid"].split(",")]


def _pairs(case):
    """The R / 2 pairs of a head vector in one group per axis, larger groups first."""
    n, p = len(_grid(case)), case["R"] // 2
    return [p // n + (1 if a < p % n else 0) for a in range(n)]


def _batch(case):
    """(new tokens, length with them) of each sequence."""
    if not case["ragged"]:
        return [(case["new"], case["context"] + case["new"])] * case["B"]
    rng, out = random.Random(case["lay"]), []
    for b in range(case["B"]):
        n = case["new"] if b == 0 or case["new"] == 1 else rng.randint(0, case["new"])
        out.append((n, n + rng.randint(0, case["context"])))
    return out


def _sees(case, n, length):
    """[begin, end) of the cached tokens that each of a sequence's n queries sees."""
    ends = [length - n + i + 1 if case["causal"] else length for i in range(n)]
    return [(max(0, e - case["window"]) if case["window"] else 0, e) for e in ends]


def _held_bytes(case, tokens):
    """Bytes of so many tokens' keys and values in the cache."""
    return 2 * tokens * case["Hk"] * (case["d"] // 2 + case["d"] // BLOCK)


def work(case):
    e, d, k = 2 if case["dtype"] == "bf16" else 4, case["d"], case["kind"]
    if k.startswith("norm_rope"):
        M, heads = case["M"], case["H"] + case["Hk"]
        x = e * M * heads * d
        entries = sum(g * p for g, p in zip(_grid(case), _pairs(case)))
        table, w = 8 * min(entries, M * case["R"] // 2), 2 * e * d
        if k == "norm_rope":
            return {"bytes": 2 * x + table + w, "flops": M * heads * (4 * d + 3 * case["R"])}
        # the heads and the outputs' gradients in, the outputs and the heads' gradients out
        return {"bytes": 4 * x + 2 * table + 2 * w, "flops": M * heads * (16 * d + 6 * case["R"])}
    batch = _batch(case)
    T, out = sum(n for n, _ in batch), {"bytes": 0, "flops": 0}
    if k in ("append", "step"):
        entries = sum(g * p for g, p in zip(_grid(case), _pairs(case)))
        out["bytes"] += 4 * e * T * case["Hk"] * d + _held_bytes(case, T) + 8 * min(entries, T * case["R"] // 2)
        out["flops"] += T * case["Hk"] * (3 * case["R"] + 4 * d)
    if k in ("attend", "step"):
        seen, pairs = 0, 0
        for n, length in batch:
            see = _sees(case, n, length)
            pairs += sum(b - a for a, b in see)
            seen += max(b for _, b in see) - min(a for a, _ in see) if see else 0
        out["bytes"] += 2 * e * T * case["H"] * d + _held_bytes(case, seen)
        out["flops"] += 4 * pairs * case["H"] * d
    return out


def draw(rng):
    """One more case: each kind as often as the others, lengths spread over their logarithm from one
    token on, heads of 64 or 128, any sharing of key heads, short and long pages."""
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("norm_rope", "norm_rope_train", "append", "attend", "step"))
    top = {n: max(work(c)[n] for c in listed()) for n in ("flops", "bytes")}
    while True:
        d = rng.choice((64, 128))
        Hk = rng.choice((1, 2, 3, 4, 5, 8, 10))
        case = dict(kind=kind, H=Hk * rng.choice((1, 1, 2, 3, 4, 5, 8)), Hk=Hk, d=d,
                    dtype=rng.choice(("bf16", "bf16", "fp32")))
        if kind != "attend":
            case.update(R=rng.choice((d, d, d // 2, d // 4)), layout=rng.choice(("half", "interleaved")),
                        grid=rng.choice(("131072", "131072", "64,40,52")))
        if kind.startswith("norm_rope"):
            case.update(M=log(1, 60000))
        else:
            case.update(B=log(1, 64), new=log(1, 5) if kind == "step" else log(1, 4000),
                        context=log(1, 120000), ragged=rng.random() < 0.6, lay=rng.randint(10, 10 ** 6),
                        page=64 * rng.choice((1, 1, 2, 3, 4, 8)))
            if kind == "append":
                del case["H"]
                case.update(context=log(1, 20000))
            else:
                case.update(causal=rng.random() < 0.7, window=rng.choice((0, 0, log(1, 20000))))
            if case["new"] + case["context"] > 131072 or case["B"] * (case["new"] + case["context"]) > 600000:
                continue
        w = work(case)
        # a quarter of the bytes: the plain forms' copies in 32 bits are eight times those of the cache
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] / 4:
            return case


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _randn(g, shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def _table(case):
    """The rotation table a program keeps: (cos, sin) of every axis, coordinate and pair, axis by
    axis, float32 [entries][2]."""
    rows = []
    for n, p in zip(_grid(case), _pairs(case)):
        f = BASE ** (-torch.arange(p, device="cuda", dtype=torch.float64) / p)
        a = torch.arange(n, device="cuda", dtype=torch.float64)[:, None] * f
        rows.append(torch.stack((a.cos(), a.sin()), -1).float().view(-1, 2))
    return torch.cat(rows).contiguous()


def _codes(x):
    """(codes, exponents of the scales) of x [..., d] in 4 bits; x in float64 where it may lie next to
    a border between two of them."""
    xb = x.unflatten(-1, (-1, BLOCK))
    e = _exponents(xb.abs().amax(-1))
    xb = xb * torch.exp2(-e.to(x.dtype))[..., None]
    a = xb.abs()
    code = sum((a > b if i % 2 == 0 else a >= b).to(torch.uint8)
               for i, b in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)))
    return (code + 8 * (xb < 0).to(torch.uint8)).flatten(-2), e


def _exponents(top):
    """The smallest e >= -126 with top <= 6 * 2^e; 6 = 0.75 * 2^3."""
    m, e = torch.frexp(top)
    return torch.where(top == 0, -126, (e - 3 + (m > 0.75).int()).clamp_min(-126))


def _bytes4(code):
    """Two codes in a byte, the first in the low half."""
    return code[..., 0::2] + 16 * code[..., 1::2]


def _orders():
    """Places of a chunk's tokens in k_scale, and in v and v_scale."""
    t = torch.arange(CHUNK, device="cuda")
    return 4 * (t % 16) + t // 16, 16 * (t // 4 % 4) + 4 * (t // 16) + t % 4


def _fill(g, case, pages):
    """A cache whose pages hold standard normal keys and values, each channel with a gain of its own."""
    Hk, d, page = case["Hk"], case["d"], case["page"]
    cache = dict(k=torch.empty(pages, Hk, page, d // 2, dtype=torch.uint8, device="cuda"),
                 v=torch.empty(pages, Hk, page // CHUNK, d // 2, CHUNK, dtype=torch.uint8, device="cuda"))
    for n in ("k_scale", "v_scale"):
        cache[n] = torch.empty(pages, Hk, page // CHUNK, d // BLOCK, CHUNK, dtype=torch.uint8, device="cuda")
    ks, vs = _orders()
    gain = torch.exp(0.3 * _randn(g, (2, Hk, 1, d)))
    step = max(1, (1 << 26) // (Hk * page * d))
    for p in range(0, pages, step):
        n = min(step, pages - p)
        for i, name in enumerate("kv"):
            code, e = _codes(_randn(g, (n, Hk, page, d)) * gain[i])
            byte, e = _bytes4(code), (e + 127).to(torch.uint8).unflatten(2, (-1, CHUNK)).transpose(-1, -2)
            cache[name + "_scale"][p:p + n, ..., ks if name == "k" else vs] = e
            if name == "k":
                cache["k"][p:p + n] = byte
            else:
                cache["v"][p:p + n, ..., vs] = byte.unflatten(2, (-1, CHUNK)).transpose(-1, -2)
    return cache


def _inputs(case, seed):
    """The case's input tensors, from the seed alone."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, d, t = DTYPES[case["dtype"]], case["d"], {}
    H, Hk = case.get("H", 0), case["Hk"]
    if case["kind"].startswith("norm_rope"):
        M, n = case["M"], math.prod(_grid(case))
        gain = torch.exp(0.5 * _randn(g, (H + Hk, d))).reshape(-1)
        t["qkv"] = torch.cat((_randn(g, (M, (H + Hk) * d)) * gain, _randn(g, (M, Hk * d))), 1).to(dt)
        t["q_weight"], t["k_weight"] = ((1.0 + 0.1 * _randn(g, (d,))).to(dt) for _ in range(2))
        t["positions"] = None
        if M != n:   # new tokens of as many sequences, or one sequence from a place of its own on
            at = torch.randint(0, n, (M,), generator=g, device="cuda")
            at = at if M < 64 else (at[:1] + torch.arange(M, device="cuda")) % n
            axes, rest = [], at
            for size in reversed(_grid(case)):
                axes.insert(0, rest % size)
                rest = rest // size
            t["positions"] = torch.stack(axes, 1).to(torch.int32)
        if case["kind"] == "norm_rope_train":
            t["dq"], t["dk"] = _randn(g, (M, H, d)).to(dt), _randn(g, (M, Hk, d)).to(dt)
        return t
    batch, page = _batch(case), case["page"]
    T = sum(n for n, _ in batch)
    used = [-(-length // page) for _, length in batch]
    pages = sum(used) + 2
    t["lengths"] = torch.tensor([length for _, length in batch], dtype=torch.int32, device="cuda")
    t["starts"] = torch.tensor([sum(n for n, _ in batch[:b]) for b in range(len(batch) + 1)],
                               dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    t["page_table"] = torch.zeros(len(batch), max(used + [1]), dtype=torch.int32, device="cuda")
    for b, n in enumerate(used):
        t["page_table"][b, :n] = order[sum(used[:b]):sum(used[:b]) + n]
    t["cache"] = _fill(g, case, pages)
    gain = torch.exp(0.3 * _randn(g, (H + 2 * Hk, d))).reshape(-1)
    t["qkv"] = (_randn(g, (T, (H + 2 * Hk) * d)) * gain).to(dt)
    return t


def _heads(qkv, H, Hk, d):
    """Queries, keys and values: views of a projection's output."""
    return [x.unflatten(1, (-1, d)) if x.shape[1] else None
            for x in qkv.split((H * d, Hk * d, Hk * d), 1)]


def prepare(case, seed):
    t = _inputs(case, seed)
    s = dict(case, t=t)
    s["q"], s["k"], s["v"] = _heads(t["qkv"], case.get("H", 0), case["Hk"], case["d"])
    if case["kind"] != "attend":
        s["table"], s["dims"], s["pairs"] = _table(case), _grid(case), _pairs(case)
        # for the plain form: each pair's axis, entry of coordinate 0, and the axis's pairs
        s["axis"] = torch.tensor([a for a, p in enumerate(s["pairs"]) for _ in range(p)], device="cuda")
        off = [sum(g * p for g, p in zip(s["dims"][:a], s["pairs"][:a])) for a in range(len(s["dims"]))]
        s["entry"] = torch.tensor([o + i for o, p in zip(off, s["pairs"]) for i in range(p)], device="cuda")
        s["step"] = torch.tensor(s["pairs"], device="cuda")[s["axis"]]
    if case["kind"].startswith("norm_rope"):
        if case["kind"] == "norm_rope_train":
            s["q"], s["k"] = s["q"].detach(), s["k"].detach()
            s["leaves"] = [s["q"], s["k"], t["q_weight"], t["k_weight"]]
            for x in s["leaves"]:
                x.requires_grad_(True)
        return s
    s["batch"] = _batch(case)
    if own:
        import paper_2607_01817_amd as hcms
        c = t["cache"]
        s["cache"] = hcms.KvCache(c["k"], c["v"], c["k_scale"].view(torch.float8_e8m0fnu),
                                  c["v_scale"].view(torch.float8_e8m0fnu))
    return s


# ---------------------------------------------------------------------------
# Plain forms: elementary operations
# ---------------------------------------------------------------------------
def _coords(s, at):
    """Coordinates [n][axes] of places on the row-major grid."""
    out = []
    for size in reversed(s["dims"]):
        out.insert(0, at % size)
        at = at // size
    return torch.stack(out, 1)


def _cos_sin(s, coords):
    """(cos, sin) [M][1][R / 2] of coordinates [M][axes]."""
    cs = s["table"][s["entry"] + coords.long()[:, s["axis"]] * s["step"]][:, None]
    return cs[..., 0], cs[..., 1]


def _turn(x, cos, sin, R, layout):
    """The first R elements of each head rotated, the others as they are."""
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if layout == "interleaved" else (x[..., :R // 2], x[..., R // 2:R])
    u, v = a * cos - b * sin, a * sin + b * cos
    y = torch.stack((u, v), -1).flatten(-2) if layout == "interleaved" else torch.cat((u, v), -1)
    return torch.cat((y, x[..., R:]), -1)


def _norm_rope(s):
    t, dt, R = s["t"], DTYPES[s["dtype"]], s["R"]
    at = t["positions"] if t["positions"] is not None else _coords(s, torch.arange(s["M"], device="cuda"))
    cos, sin = _cos_sin(s, at)
    outs, grads, weights = [], [], []
    for x, w, dy in ((s["q"], t["q_weight"], t.get("dq")), (s["k"], t["k_weight"], t.get("dk"))):
        x, w = x.float(), w.float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        n = x * r
        outs.append(_turn(n * w, cos, sin, R, s["layout"]).to(dt))
        if dy is not None:
            g = _turn(dy.float(), cos, -sin, R, s["layout"])
            weights.append((g * n).sum((0, 1), dtype=torch.float64).to(dt))
            g = g * w
            grads.append((r * (g - n * (g * n).mean(-1, keepdim=True))).to(dt))
    return tuple(outs + grads + weights)


def _places(s):
    """Of the packed tokens: sequence, place in it."""
    seq = [b for b, (n, _) in enumerate(s["batch"]) for _ in range(n)]
    at = [length - n + i for n, length in s["batch"] for i in range(n)]
    return torch.tensor(seq, device="cuda"), torch.tensor(at, device="cuda")


VALUES4 = GRID4 + tuple(-x for x in GRID4)


def _append(s):
    t, c, page, dt = s["t"], s["t"]["cache"], s["page"], DTYPES[s["dtype"]]
    seq, at = _places(s)
    cos, sin = (x.double() for x in _cos_sin(s, _coords(s, at)))
    held, values = [], torch.tensor(VALUES4, device="cuda")
    ks, vs = _orders()
    p, slot = t["page_table"][seq, at // page].long(), at % page
    chunk, lane = slot // CHUNK, slot % CHUNK
    heads = torch.arange(s["Hk"], device="cuda")
    for name, x in (("k", _turn(s["k"].double(), cos, sin, s["R"], s["layout"])), ("v", s["v"].float())):
        code, e = _codes(x)
        byte, order = _bytes4(code), ks if name == "k" else vs
        # advanced indexes apart put their axes first: [tokens][heads][...]
        c[name + "_scale"][p[:, None], heads, chunk[:, None], :, order[lane][:, None]] = (e + 127).to(torch.uint8)
        if name == "k":
            c["k"][p[:, None], heads, slot[:, None]] = byte
        else:
            c["v"][p[:, None], heads, chunk[:, None], :, vs[lane][:, None]] = byte
        by = torch.exp2(e.float()).repeat_interleave(BLOCK, -1)
        held.append((values[code.long()] * by).to(dt))
    return tuple(held)


def _read(s, b, length):
    """Keys and values [Hk][length][d] of sequence b in float32."""
    t, c, out = s["t"], s["t"]["cache"], []
    pages = t["page_table"][b, :-(-length // s["page"])].long()
    values = torch.tensor(VALUES4, device="cuda")
    ks, vs = _orders()
    for name, order in (("k", ks), ("v", vs)):
        byte, e = c[name][pages], c[name + "_scale"][pages][..., order].transpose(-1, -2)
        if name == "v":
            byte = byte[..., vs].transpose(-1, -2)
        byte = byte.flatten(2, -2) if name == "v" else byte      # [pages][Hk][page][d / 2]
        x = values[torch.stack((byte % 16, byte // 16), -1).flatten(-2).int()]
        by = torch.exp2(e.flatten(2, 3).float() - 127)
        x = (x.unflatten(-1, (-1, BLOCK)) * by[..., None]).flatten(-2)
        out.append(x.transpose(0, 1).flatten(1, 2)[:, :length])
    return out


def _attend(s):
    H, Hk, d, dt = s["H"], s["Hk"], s["d"], DTYPES[s["dtype"]]
    T = s["q"].shape[0]
    out = torch.empty(T, H, d, dtype=dt, device="cuda")
    first = 0
    for b, (n, length) in enumerate(s["batch"]):
        if n == 0:
            continue
        K, V = _read(s, b, length)
        K = K.transpose(1, 2).contiguous()
        rows = max(1, (1 << 28) // (H * length))
        for i in range(0, n, rows):
            m = min(rows, n - i)
            q = s["q"][first + i:first + i + m].float() * d ** -0.5
            q = q.view(m, Hk, H // Hk, d).transpose(0, 1).reshape(Hk, -1, d)
            x = torch.bmm(q, K).view(Hk, m, H // Hk, length)
            end = torch.arange(length - n + i, length - n + i + m, device="cuda") + 1
            end = end if s["causal"] else torch.full_like(end, length)
            at = torch.arange(length, device="cuda")
            dark = at >= end[:, None]
            if s["window"]:
                dark |= at < end[:, None] - s["window"]
            x = x.masked_fill(dark[:, None], -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            y = torch.bmm(x.view(Hk, -1, length), V) / x.sum(-1).view(Hk, -1, 1)
            out[first + i:first + i + m] = y.view(Hk, m, H // Hk, d).transpose(0, 1).reshape(m, H, d).to(dt)
        first += n
    return out


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def run(s):
    t, k = s["t"], s["kind"]
    if not own:
        with torch.no_grad():
            if k.startswith("norm_rope"):
                return _norm_rope(s)
            held = _append(s) if k in ("append", "step") else ()
            return (_attend(s), *held) if k in ("attend", "step") else held
    import paper_2607_01817_amd as hcms
    if k == "norm_rope":
        return hcms.qk_norm_rope(s["q"], s["k"], t["q_weight"], t["k_weight"], s["table"], s["dims"], s["pairs"],
                                 positions=t["positions"], layout=s["layout"], eps=EPS)
    if k == "norm_rope_train":
        y = hcms.QkNormRope.apply(s["q"], s["k"], t["q_weight"], t["k_weight"], s["table"], s["dims"], s["pairs"],
                                  t["positions"], s["layout"], EPS)
        return (y[0].detach(), y[1].detach(), *torch.autograd.grad(y, s["leaves"], (t["dq"], t["dk"])))
    batch, held = (t["page_table"], t["lengths"], t["starts"]), ()
    if k in ("append", "step"):
        held = hcms.append_kv(s["k"], s["v"], s["cache"], *batch, table=s["table"], grid=s["dims"],
                              axis_pairs=s["pairs"], layout=s["layout"], held=True)
    if k == "append":
        return held
    return (hcms.cache_attention(s["q"], s["cache"], *batch, causal=s["causal"], window=s["window"]), *held)


# ---------------------------------------------------------------------------
# 64-bit results from the definitions
# ---------------------------------------------------------------------------
def _rotated64(x, z, R, layout):
    """Heads x [M][heads][d] turned by complex factors z [M][R / 2]."""
    x = x.double()
    if layout == "interleaved":
        w = torch.view_as_complex(x[..., :R].reshape(*x.shape[:-1], R // 2, 2).contiguous())
    else:
        w = torch.complex(x[..., :R // 2].contiguous(), x[..., R // 2:R].contiguous())
    w = w * z[:, None]
    y = torch.view_as_real(w).flatten(-2) if layout == "interleaved" else torch.cat((w.real, w.imag), -1)
    return torch.cat((y, x[..., R:]), -1)


def _factors64(case, at):
    """The table's complex factors [M][R / 2] for places or coordinates `at`."""
    table, row, out = _table(case).double(), 0, []
    dims = _grid(case)
    for a, (size, p) in enumerate(zip(dims, _pairs(case))):
        c = at[:, a].long() if at.dim() == 2 else at // math.prod(dims[a + 1:]) % size
        out.append(torch.view_as_complex(table[row:row + size * p].view(size, p, 2))[c])
        row += size * p
    return torch.cat(out, 1)


def _held64(x):
    """The values that x's 4-bit form stands for: the nearest of each block's grid."""
    x = x.double().unflatten(-1, (-1, BLOCK))
    top = x.abs().amax(-1, keepdim=True)
    s = torch.full_like(top, 2.0 ** -126)
    for e in range(-125, 126):
        s = torch.where(top > 6 * 2.0 ** (e - 1), 2.0 ** e, s)
    a = (x / s).abs()
    # steps of a half below 2, of one below 4, of two from there on; ties to the even multiple
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    return ((a / step).round() * step * s * x.sign()).flatten(-2)


def _cached64(case, t, b, head, length):
    """Keys and values [length][d] of one sequence and head."""
    page, c = case["page"], t["cache"]
    at = torch.arange(length, device="cuda")
    p, slot = t["page_table"][b].long()[at // page], at % page
    chunk, u = slot // CHUNK, slot % CHUNK
    place = u // 4 % 4 * 16 + u // 16 * 4 + u % 4
    out = []
    for byte, e in ((c["k"][p, head, slot], c["k_scale"][p, head, chunk, :, u % 16 * 4 + u // 16]),
                    (c["v"][p, head, chunk, :, place], c["v_scale"][p, head, chunk, :, place])):
        code = torch.stack((byte & 15, byte >> 4), -1).flatten(1).long()
        sign, ee, m = 1 - 2.0 * (code >> 3), code >> 1 & 3, (code & 1).double()
        x = sign * torch.where(ee == 0, m / 2, (1 + m / 2) * torch.exp2(ee.double() - 1))
        out.append(x * torch.exp2(e.double() - 127).repeat_interleave(BLOCK, 1))
    return out


def exact(case, seed):
    t, k, d = _inputs(case, seed), case["kind"], case["d"]
    H, Hk = case.get("H", 0), case["Hk"]
    q, kk, v = _heads(t["qkv"], H, Hk, d)
    if k.startswith("norm_rope"):
        at = t["positions"] if t["positions"] is not None else torch.arange(case["M"], device="cuda")
        z = _factors64(case, at)
        outs, grads = [], []
        for x, w, dy in ((q, t["q_weight"], t.get("dq")), (kk, t["k_weight"], t.get("dk"))):
            x, w = (y.double().requires_grad_(dy is not None) for y in (x, w))
            y = _rotated64(x / (x.square().sum(-1, keepdim=True) / d + EPS).sqrt() * w, z, case["R"], case["layout"])
            outs.append(y.detach())
            if dy is not None:
                grads.append(torch.autograd.grad(y, (x, w), dy.double()))
        return (*outs, *(g[0] for g in grads), *(g[1] for g in grads))
    batch, held = _batch(case), ()
    if k in ("append", "step"):
        at = torch.cat([torch.arange(length - n, length, device="cuda") for n, length in batch])
        held = (_held64(_rotated64(kk, _factors64(case, at), case["R"], case["layout"])), _held64(v))
        if k == "append":
            return held
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    first = 0
    for b, (n, length) in enumerate(batch):
        if n == 0:
            continue
        see = torch.tensor(_sees(case, n, length), device="cuda")
        for j in range(Hk):
            K, V = _cached64(case, t, b, j, length)
            for x, h in zip((K, V), held):
                x[length - n:] = h[first:first + n, j]
            rows = max(1, (1 << 27) // length)
            for h in range(j * (H // Hk), (j + 1) * (H // Hk)):
                for i in range(0, n, rows):
                    m = min(rows, n - i)
                    x = q[first + i:first + i + m, h].double() @ K.T / math.sqrt(d)
                    at = torch.arange(length, device="cuda")
                    x[(at < see[i:i + m, :1]) | (at >= see[i:i + m, 1:])] = -math.inf
                    out[first + i:first + i + m, h] = torch.softmax(x, -1) @ V
        first += n
    return (out, *held)

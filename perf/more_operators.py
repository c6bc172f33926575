"""Between a layer's projections and its attention, as timed cases: the norms of queries and keys and their position
rotation (``rope``), the gradient of both (``grad``), writing new tokens into a cache of 8-bit codes with a scale for each
block of tokens and head (``append``), and attention over such a cache (``blocks``).

``listed()`` names the cases, ``draw()`` gives more of the same ranges, ``prepare()`` makes what a program holds before
the call, ``run()`` is one call: in elementary torch operations, or with ``own`` through the library's entry points.
``exact()`` gives the same results in float64.
"""
import math
import random

import numpy as np
import torch

own = False

LOG2E = 1.4426950408889634
TILE = 128  # keys between two moves of the running maximum of the lattice weights
ORDER = {"h15": 1, "sq4": 2, "sq8": 3}  # S(Q_{2^-k}): k
MODES = {"exact": 0, "h15": 1, "sq4": 2, "sq8": 3}  # the library's exp_mode values
EPS = 1e-6
FP8 = torch.float8_e4m3fn


def _rope(name, b, s, hq, hkv, d, rot, inter, norm, out="bf16", start=0, packed=False, kind="rope"):
    # inter: pairs of neighbouring channels, else of the two halves; start: the largest first position of a sequence;
    # packed: each position given, two documents in a sequence
    return {"name": name, "kind": kind, "B": b, "S": s, "Hq": hq, "Hkv": hkv, "d": d, "rot": rot, "inter": inter,
            "norm": norm, "out": out, "start": start, "packed": packed}


def _append(name, b, hkv, n, cap, d, block, fill, ragged=False):
    # fill: the largest number of tokens that a cache holds before; ragged: some sequences bring fewer new tokens
    return {"name": name, "kind": "append", "B": b, "Hkv": hkv, "n": n, "cap": cap, "d": d, "block": block,
            "fill": fill, "ragged": ragged}


def _blocks(name, b, hq, hkv, sq, sk, d, block, mode, sharp=False, cut=0, empty=False):
    # cut: keys of a part (lattice weights are rounded relative to their part's running maximum; the hardware
    # exponential does not depend on it and takes the library's choice)
    return {"name": name, "kind": "blocks", "B": b, "Hq": hq, "Hkv": hkv, "Sq": sq, "Sk": sk, "d": d, "block": block,
            "mode": mode, "sharp": sharp, "cut": cut, "empty": empty}


def listed():
    return [
        # the smallest: a small model's decode step, four chats, no norms; bound by the call and its launch
        _rope("rope_b4h8kv2_s1_d64", 4, 1, 8, 2, 64, 64, False, False, start=1000),
        # prompts of a model with norms, half layout
        _rope("rope_norm_b2h32kv8_s4096", 2, 4096, 32, 8, 128, 128, False, True),
        # an odd chunk far into a long context, a quarter of the head rotated in neighbouring pairs, FP8 attention's operands
        _rope("rope_fp8_b3h24kv8_s1001_rot32", 3, 1001, 24, 8, 128, 32, True, False, "fp8", start=900000),
        # a training step's batch, gradients of the norm weights too
        _rope("grad_norm_b4h32kv8_s2048", 4, 2048, 32, 8, 128, 128, False, True, kind="grad"),
        # a small model, two documents packed in each odd sequence
        _rope("grad_norm_b3h8kv2_s777_d64_rot32", 3, 777, 8, 2, 64, 32, True, True, packed=True, kind="grad"),
        # the token that a decode step adds to each cache of a serving batch
        _append("append_b16kv8_n1", 16, 8, 1, 8192, 128, 64, 8000),
        # the chunk of a prompt that is written at once, behind caches that end inside a block
        _append("append_b4kv8_n4096_ragged", 4, 8, 4096, 8192, 128, 64, 3000, ragged=True),
        # four chats of a small model: short caches, one launch or two
        _blocks("blocks_b4h8kv2_sk500_d64", 4, 8, 2, 1, 500, 64, 32, "exact"),
        # a decode step of a serving batch with caches of up to 8K
        _blocks("blocks_b16h32kv8_sk8192", 16, 32, 8, 1, 8192, 128, 64, "exact", sharp=True),
        # four drafted tokens of an odd batch with the lattice weights, odd lengths, small blocks, one cache still empty
        _blocks("blocks_h15_b7h24kv8_sq4_sk5003", 7, 24, 8, 4, 5003, 128, 16, "h15", True, 512, empty=True),
        # many long caches: one token for each of 64 chats of up to 32K
        _blocks("blocks_b64h32kv8_sk32768", 64, 32, 8, 1, 32768, 128, 128, "exact"),
        # a chunk of 2K tokens of a prompt of 32K, written to the cache before: bound by the matrix core
        _blocks("blocks_b1h32kv8_sq2048_sk32768", 1, 32, 8, 2048, 32768, 128, 64, "exact"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    hkv = rng.choice([1, 2, 3, 4, 8, 8])
    return hkv * rng.choice([1, 2, 3, 4, 4, 8]), hkv


def draw(rng):
    most = {}
    for c in listed():
        w, m = work(c), most.setdefault(c["kind"], {"bytes": 0, "flops": 0})
        most[c["kind"]] = {k: max(m[k], w[k]) for k in m}
    while True:
        kind = rng.choice(["rope", "grad", "append", "blocks", "blocks"])
        hq, hkv = _heads(rng)
        d = rng.choice([64, 128, 128])
        if kind in ("rope", "grad"):
            rot = rng.choice([d, d, d // 2, d // 4, 16 * rng.randint(1, d // 16)])
            s = 1 if kind == "rope" and rng.random() < 0.3 else _log_int(rng, 1, 16384)
            c = _rope("", _log_int(rng, 1, 64), s, hq, hkv, d, rot, rng.random() < 0.4, rng.random() < 0.6,
                      "fp8" if kind == "rope" and rng.random() < 0.3 else "bf16",
                      rng.choice([0, _log_int(rng, 1, 1000000)]), rng.random() < 0.3, kind)
        elif kind == "append":
            block = rng.choice([16, 32, 64, 128])
            n = 1 if rng.random() < 0.3 else _log_int(rng, 1, 16384)
            fill = 0 if rng.random() < 0.2 else _log_int(rng, 1, 32768)
            cap = -(-(n + fill + rng.randint(0, 200)) // block) * block
            c = _append("", _log_int(rng, 1, 64), hkv, n, cap, d, block, fill, rng.random() < 0.4)
        else:
            mode = rng.choice(["exact"] * 5 + ["h15"] * 3 + ["sq4", "sq8"])
            sk = _log_int(rng, 1, 32768)
            sq = rng.choice([1, 1, 1, 2, 4, 7, 16, _log_int(rng, 2, 2048)])
            c = _blocks("", _log_int(rng, 1, 64), hq, hkv, min(sq, sk), sk, d, rng.choice([16, 32, 64, 128]), mode,
                        rng.random() < 0.4, rng.choice([0, 128 * rng.randint(2, 16)]) if mode != "exact" else 0,
                        rng.random() < 0.3)
            if mode != "exact" and c["B"] * hq * c["Sq"] * sk > 1 << 29:
                continue  # (the plain form holds these weights in 64 bits)
        w = work(c)
        if w["bytes"] <= most[kind]["bytes"] and w["flops"] <= most[kind]["flops"]:
            del c["name"]
            return c


def _lens(c):
    """Keys in each sequence's cache: the longest has Sk, the others a fourth of it at least; "empty": one has none."""
    r = random.Random(c["B"] * 1000003 + c["Sk"])
    lens = [c["Sk"]] + [r.randint(max(1, c["Sk"] // 4), c["Sk"]) for _ in range(c["B"] - 1)]
    if c["empty"] and c["B"] > 1:
        lens[1] = 0
    r.shuffle(lens)
    return lens


def _held(c):
    """Tokens that each cache holds before an append, and new ones."""
    r = random.Random(c["B"] * 1000003 + c["fill"])
    held = [c["fill"]] + [r.randint(0, c["fill"]) for _ in range(c["B"] - 1)]
    new = [c["n"]] + [r.randint(0, c["n"]) if c["ragged"] else c["n"] for _ in range(c["B"] - 1)]
    return held, new


def _reach(c):
    """Blocks that n new tokens can lie in."""
    return min((c["n"] + c["block"] - 2) // c["block"] + 1, c["cap"] // c["block"])


def work(case):
    c = case
    if c["kind"] in ("rope", "grad"):
        rows, vrows = c["B"] * c["S"] * float(c["Hq"] + c["Hkv"]), c["B"] * c["S"] * float(c["Hkv"])
        e = 1 if c["out"] == "fp8" else 2
        if c["kind"] == "rope":
            return {"bytes": (rows + vrows) * c["d"] * (2 + e), "flops": rows * c["d"] * 8}
        return {"bytes": (rows * (6 if c["norm"] else 4) + vrows * 4) * c["d"], "flops": rows * c["d"] * 16}
    if c["kind"] == "append":
        tokens = float(sum(_held(c)[1])) * c["Hkv"]
        return {"bytes": 2 * tokens * (c["d"] * 3 + 1.0 / c["block"]), "flops": 4 * tokens * c["d"]}
    lens = _lens(c)
    keys = c["Hkv"] * float(sum(lens))
    rows = c["B"] * c["Hq"] * c["Sq"]
    # row i of a sequence sees its first n - Sq + i + 1 keys
    seen = float(sum(sum(range(max(0, n - c["Sq"] + 1), n + 1)) for n in lens)) * c["Hq"]
    return {"bytes": rows * (4 * c["d"] + 4) + 2.0 * keys * (c["d"] + 1.0 / c["block"]), "flops": 4.0 * c["d"] * seen}


def _scale(c):
    return float(np.float32(1.0 / math.sqrt(c["d"])))


def _least(amax):
    """The exponent byte of the least scale 2^(e - 127) with which values up to amax fit e4m3, 1 at least."""
    m, e = torch.frexp(amax.float() / 448.0)
    return (torch.where(m == 0.5, e - 1, e) + 127).masked_fill(amax == 0, 1).clamp(min=1)


def _power(e):
    """2^(e - 127) of exponent bytes e in 1 .. 254."""
    return (e.int() << 23).view(torch.float32)


def _codes(x):
    return x.clamp(-448, 448).to(FP8)


def _quantized(c, x):
    """Codes and exponent bytes of [B, Hkv, rows, d], the rows a whole number of blocks."""
    b, h, rows, d = x.shape
    x = x.view(b, h, -1, c["block"], d)
    e = _least(x.abs().amax((-1, -2)))
    return _codes(x / _power(e)[..., None, None]).view(b, h, rows, d), e


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    st = {"case": c}
    if c["kind"] in ("rope", "grad"):
        heads = c["Hq"] + 2 * c["Hkv"]
        # one projection's output, a few channels of each head much larger than the others
        x = normal(c["B"], c["S"], heads, c["d"])
        x *= 1.0 + 7.0 * (torch.rand(heads, c["d"], generator=gen, device="cuda") < 0.02)
        st["qkv"] = x.to(torch.bfloat16).view(c["B"], c["S"], heads * c["d"])
        # frequencies in radians a position, those of a long context four times slower
        i = torch.arange(c["rot"] // 2, device="cuda", dtype=torch.float64)
        st["freqs"] = torch.pow(500000.0 if c["start"] > 10000 else 10000.0, -2.0 * i / c["rot"])
        st["amplitude"] = 1.0
        if c["start"] > 10000:
            st["freqs"] /= 4.0
            st["amplitude"] = float(np.float32(0.1 * math.log(4.0) + 1.0))
        first = (torch.rand(c["B"], generator=gen, device="cuda", dtype=torch.float64) * (c["start"] + 1)).int()
        if c["packed"]:
            at = torch.arange(c["S"], device="cuda", dtype=torch.int32)
            st["positions"] = first[:, None] + torch.where(at < c["S"] // 3, at, at - c["S"] // 3)
        else:
            st["positions"] = first  # of a sequence's first row
        st["wq"] = st["wk"] = None
        if c["norm"]:
            st["wq"], st["wk"] = ((1.0 + 0.2 * normal(c["d"])).to(torch.bfloat16) for _ in range(2))
        for x, h in (("q", c["Hq"]), ("k", c["Hkv"]), ("v", c["Hkv"])):
            shape = (c["B"], h, c["S"], c["d"])
            if c["kind"] == "grad":
                st["g" + x] = normal(*shape).to(torch.bfloat16)
            else:
                st[x + "_out"] = torch.empty(shape, dtype=FP8 if c["out"] == "fp8" else torch.bfloat16, device="cuda")
        if c["kind"] == "grad":
            st["dqkv"] = torch.empty_like(st["qkv"])
            st["dwq"], st["dwk"] = (torch.empty(c["d"], device="cuda") if c["norm"] else None for _ in range(2))
        # static descales of the FP8 operands
        st["descale"] = (1 / 16, 1 / 16, 1 / 12) if c["out"] == "fp8" else (1.0, 1.0, 1.0)
        return st
    if c["kind"] == "append":
        held, new = _held(c)
        st["lens"], st["counts"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (held, new))
        shape = (c["B"], c["Hkv"], c["n"], c["d"])
        grow = torch.exp(0.5 * normal(*shape[:3], 1))  # tokens of different sizes
        st["k"], st["v"] = ((normal(*shape) * grow).to(torch.bfloat16) for _ in range(2))
        both = []
        for x in ("kc", "vc"):
            st[x], e = _quantized(c, normal(c["B"], c["Hkv"], c["cap"], c["d"]))
            both.append(e)
        st["scales"] = torch.stack(both, -1).to(torch.uint8).view(torch.float8_e8m0fnu)  # [B, Hkv, blocks, 2]
        st["lens_out"] = torch.empty(c["B"], dtype=torch.int32, device="cuda")
        return st
    st["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda")
    st["scale"] = _scale(c)
    st["q"] = normal(c["B"], c["Hq"], c["Sq"], c["d"]).to(torch.bfloat16)
    rows = -(-c["Sk"] // c["block"]) * c["block"]
    both = []
    for x in ("k", "v"):
        y = normal(c["B"], c["Hkv"], rows, c["d"])
        if x == "k" and c["sharp"]:  # 2% of the keys four times as large: those that many queries look at
            y *= 1.0 + 3.0 * (torch.rand(*y.shape[:3], 1, generator=gen, device="cuda") < 0.02)
        st[x], e = _quantized(c, y)
        del y
        both.append(e)
    st["scales"] = torch.stack(both, -1).to(torch.uint8).view(torch.float8_e8m0fnu)
    st["out"] = torch.empty(st["q"].shape, dtype=torch.bfloat16, device="cuda")
    st["lse"] = torch.empty(st["q"].shape[:3], dtype=torch.float32, device="cuda")
    return st


def _views(c, qkv):
    """Queries, keys and values [B, S, heads, d] of a projection's output."""
    return qkv.view(c["B"], c["S"], -1, c["d"]).split([c["Hq"], c["Hkv"], c["Hkv"]], 2)


# ---- the plain forms ------------------------------------------------------

def _angles(c, st):
    """Cosines and sines [B, S, 1, rot / 2], times the amplitude."""
    p = st["positions"].double()
    if p.dim() == 1:
        p = p[:, None] + torch.arange(c["S"], device="cuda")
    t = p[:, :, None, None] * st["freqs"]
    return (torch.cos(t) * st["amplitude"]).float(), (torch.sin(t) * st["amplitude"]).float()


def _turned(c, x, cos, sin):
    """The first rot channels of x turned by the angles."""
    r = x[..., :c["rot"]]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["inter"] else r.chunk(2, -1)
    pair = (a * cos - b * sin, b * cos + a * sin)
    r = torch.stack(pair, -1).flatten(-2) if c["inter"] else torch.cat(pair, -1)
    return torch.cat((r, x[..., c["rot"]:]), -1)


def _plain_rope(c, st):
    cos, sin = _angles(c, st)
    out = {}
    for x, w, name, s in zip(_views(c, st["qkv"]), (st["wq"], st["wk"], None), "qkv", st["descale"]):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
        x = (_turned(c, x, cos, sin) if name != "v" else x).transpose(1, 2)
        out[name] = (_codes(x / s) if c["out"] == "fp8" else x.to(torch.bfloat16)).contiguous()
    return out


def _plain_grad(c, st):
    cos, sin = _angles(c, st)
    q, k, _ = _views(c, st["qkv"])
    parts, dw = [], []
    for g, x, w in ((st["gq"], q, st["wq"]), (st["gk"], k, st["wk"])):
        dy = _turned(c, g.transpose(1, 2).float(), cos, -sin)
        if w is not None:
            x = x.float()
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
            x = x * r
            dw.append((dy * x).sum((0, 1, 2)))
            dy = dy * w.float()
            dy = r * (dy - x * (dy * x).mean(-1, keepdim=True))
        parts.append(dy.to(torch.bfloat16))
    parts.append(st["gv"].transpose(1, 2))
    return {"dqkv": torch.cat(parts, 2).view(st["qkv"].shape), **dict(zip(("dwq", "dwk"), dw))}


def _plain_append(c, st):
    held, t, reach = st["lens"].long(), c["block"], _reach(c)
    new = torch.minimum(st["counts"].long(), c["cap"] - held)
    b0 = (held // t).clamp(max=c["cap"] // t - reach)  # the first block that is looked at
    slot = b0[:, None] * t + torch.arange(reach * t, device="cuda")  # [B, W]
    mine = ((slot >= held[:, None]) & (slot < (held + new)[:, None]))[:, None, :, None]
    rows = slot[:, None, :, None].expand(-1, c["Hkv"], -1, c["d"])
    source = (slot - held[:, None]).clamp(0, c["n"] - 1)[:, None, :, None].expand_as(rows)
    at = b0[:, None] + torch.arange(reach, device="cuda")  # [B, reach]
    some = mine.view(c["B"], 1, reach, t).any(-1)
    full = (held[:, None] > at * t)[:, None]  # blocks that hold a token already
    scales = st["scales"].view(torch.uint8)
    for i, x in enumerate("kv"):
        cache = st[x + "c"].view(torch.uint8)
        fresh = st[x].gather(2, source).float().masked_fill(~mine, 0.0)
        e_old = scales[..., i].gather(2, at[:, None].expand(-1, c["Hkv"], -1)).int()
        e = torch.maximum(_least(fresh.view(c["B"], c["Hkv"], reach, -1).abs().amax(-1)), torch.where(full, e_old, 1))
        e = torch.where(some, e, e_old)
        wide = lambda y: y.repeat_interleave(t, -1).unsqueeze(-1)  # noqa: E731
        shrink = torch.where(some & full, _power(e_old) / _power(e), 1.0)
        there = cache.gather(2, rows).view(FP8)
        old = torch.where((slot < held[:, None])[:, None, :, None], (there.float() * wide(shrink)).to(FP8).float(),
                          there.float())
        codes = torch.where(mine, _codes(fresh / wide(_power(e))).float(), old).to(FP8)
        cache.scatter_(2, rows, codes.view(torch.uint8))
        scales[..., i].scatter_(2, at[:, None].expand(-1, c["Hkv"], -1), e.to(torch.uint8))
    return {"k": st["kc"], "v": st["vc"], "scales": st["scales"], "lens": (held + new).int()}


def _dequantized(c, st, i, t):
    """Keys (0) or values (1) [B, Hkv, rows, d] as numbers."""
    s = _power(st["scales"].view(torch.uint8)[..., i]).to(t)
    x = st["kv"[i]].to(torch.float32).to(t)
    return (x.view(*s.shape, c["block"], c["d"]) * s[..., None, None]).view(x.shape)


def _lattice(s, cut, c1, k):
    """Weights S(Q_{2^-k}) of logits [..., keys], each relative to the running maximum of its tile within its part, and
    those maxima, one a key."""
    n = s.shape[-1]
    per = -(-min(cut, n) // TILE) if cut else -(-n // TILE)  # tiles of a part
    size = max(1, per) * TILE
    pad = torch.nn.functional.pad(s, (0, -n % size), value=-math.inf)
    tiles = pad.view(*s.shape[:-1], -1, max(1, per), TILE)
    top = tiles.amax(-1).cummax(-1).values.unsqueeze(-1)
    f = float(1 << k)
    c1 = torch.tensor(c1, dtype=s.dtype, device=s.device)
    y = torch.round((tiles - top.masked_fill(top == -math.inf, 0.0)) * c1 * f).clamp(min=-126.0 * f) / f  # halves to even
    w = (y - torch.floor(y) + 1.0) * torch.exp2(torch.floor(y))
    w = w.masked_fill(tiles == -math.inf, 0.0)
    return w.reshape(pad.shape)[..., :n], top.expand_as(tiles).reshape(pad.shape)[..., :n]


def _plain_blocks(c, st):
    t = torch.float32 if c["mode"] == "exact" else torch.float64  # a lattice weight next to a border needs the 64
    c1 = float(np.float32(st["scale"] * LOG2E))
    q = st["q"].to(t).view(c["B"], c["Hkv"], -1, c["d"])
    last = (st["lens"].view(-1, 1) - c["Sq"] + torch.arange(c["Sq"], device="cuda")).repeat(1, c["Hq"] // c["Hkv"])
    s = q @ _dequantized(c, st, 0, t).transpose(-1, -2).contiguous()
    s.masked_fill_((torch.arange(s.shape[-1], device="cuda") > last.unsqueeze(-1)).unsqueeze(1), -math.inf)
    m = s.amax(-1, keepdim=True)
    base = m.masked_fill(m == -math.inf, 0.0)
    if c["mode"] == "exact":
        w = torch.exp2((s - base) * c1)
    else:
        w, a = _lattice(s[..., :c["Sk"]], c["cut"], c1, ORDER[c["mode"]])
        w = torch.nn.functional.pad(w * torch.exp2((a - base) * c1), (0, s.shape[-1] - c["Sk"]))
    total = w.sum(-1, keepdim=True)
    o = torch.where(total > 0, (w @ _dequantized(c, st, 1, t)) / total, 0.0)
    lse = (m * c1 + torch.log2(total)) * math.log(2.0)
    return {"o": o.reshape(st["q"].shape).to(torch.bfloat16), "lse": lse.reshape(st["q"].shape[:3]).float()}


# ---- the library's calls --------------------------------------------------

def _own_rope(c, st):
    import paper_2609_33586_amd as attn
    q, k, v = attn.attn_rope(*_views(c, st["qkv"]), freqs=st["freqs"], positions=st["positions"], interleaved=c["inter"],
                             amplitude=st["amplitude"], q_weight=st["wq"], k_weight=st["wk"], eps=EPS,
                             descale=st["descale"], q_out=st["q_out"], k_out=st["k_out"], v_out=st["v_out"])
    return {"q": q, "k": k, "v": v}


def _own_grad(c, st):
    import paper_2609_33586_amd as attn
    if "plan" not in st:  # a training loop keeps its workspace
        need = attn.attn_rope_bwd_workspace_bytes(c["B"], c["S"], c["Hq"], c["Hkv"], c["d"]) if c["norm"] else 0
        st["plan"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    q, k, _ = _views(c, st["qkv"])
    dq, dk, dv = _views(c, st["dqkv"])
    attn.attn_rope_bwd(st["gq"], st["gk"], st["gv"], q=q, k=k, freqs=st["freqs"], positions=st["positions"],
                       interleaved=c["inter"], amplitude=st["amplitude"], q_weight=st["wq"], k_weight=st["wk"], eps=EPS,
                       dq=dq, dk=dk, dv=dv, dq_weight=st["dwq"], dk_weight=st["dwk"], workspace=st["plan"])
    return {"dqkv": st["dqkv"], **({"dwq": st["dwq"], "dwk": st["dwk"]} if c["norm"] else {})}


def _own_append(c, st):
    import paper_2609_33586_amd as attn
    lens = attn.attn_cache_append(st["k"], st["v"], st["kc"], st["vc"], st["scales"], st["lens"], block=c["block"],
                                  counts=st["counts"], lens_out=st["lens_out"])
    return {"k": st["kc"], "v": st["vc"], "scales": st["scales"], "lens": lens}


def _own_blocks(c, st):
    import paper_2609_33586_amd as attn
    if "plan" not in st:  # a decode loop keeps its cut and its workspace from step to step
        cut = c["cut"]
        if c["mode"] == "exact":
            cut = attn.attn_decode_blocks_split_keys(c["B"], c["Hq"], c["Hkv"], c["Sq"], c["Sk"], c["d"])
        need = attn.attn_decode_blocks_workspace_bytes(c["B"], c["Hq"], c["Sq"], c["Sk"], c["d"], cut)
        st["plan"] = cut, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    cut, ws = st["plan"]
    o, lse = attn.attn_decode_blocks(st["q"], st["k"], st["v"], st["scales"], block=c["block"], Sk=c["Sk"],
                                     lens=st["lens"], causal=True, scale=st["scale"], exp_mode=MODES[c["mode"]],
                                     split_keys=cut, out=st["out"], lse=st["lse"], workspace=ws)
    return {"o": o, "lse": lse}


def run(state):
    c = state["case"]
    if own:
        return {"rope": _own_rope, "grad": _own_grad, "append": _own_append, "blocks": _own_blocks}[c["kind"]](c, state)
    return {"rope": _plain_rope, "grad": _plain_grad, "append": _plain_append, "blocks": _plain_blocks}[c["kind"]](c, state)


# ---- 64 bits --------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    of = {"rope": _exact_rope, "grad": _exact_grad, "append": _exact_append, "blocks": _exact_blocks}
    return of[case["kind"]](case, st)


def _rotation(c, st, i):
    """The complex factors [S, rot / 2] of sequence i."""
    p = st["positions"][i].double()
    p = p + torch.arange(c["S"], device="cuda") if p.dim() == 0 else p
    t = p[:, None] * st["freqs"]
    return torch.polar(torch.full_like(t, st["amplitude"]), t)


def _pairs(c, x):
    """The rotated channels of [S, d] as complex numbers [S, rot / 2]."""
    h = c["rot"] // 2
    if c["inter"]:
        return torch.complex(x[:, 0:c["rot"]:2].contiguous(), x[:, 1:c["rot"]:2].contiguous())
    return torch.complex(x[:, :h].contiguous(), x[:, h:c["rot"]].contiguous())


def _unpaired(c, x, z):
    x, h = x.clone(), c["rot"] // 2
    if c["inter"]:
        x[:, 0:c["rot"]:2], x[:, 1:c["rot"]:2] = z.real, z.imag
    else:
        x[:, :h], x[:, h:c["rot"]] = z.real, z.imag
    return x


def _e4m3(x):
    """The nearest e4m3 value of numbers up to 448, ties to even, in float64."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp(-6, 8) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def _exact_rope(c, st):
    out = {}
    for x, w, name, s in zip(_views(c, st["qkv"]), (st["wq"], st["wk"], None), "qkv", st["descale"]):
        y = torch.empty(c["B"], x.shape[2], c["S"], c["d"], dtype=torch.float64, device="cuda")
        for i in range(c["B"]):
            turn = _rotation(c, st, i)
            for h in range(x.shape[2]):
                z = x[i, :, h].double()
                if w is not None:
                    z = z / torch.sqrt(z.square().sum(-1, keepdim=True) / c["d"] + EPS) * w.double()
                y[i, h] = z if name == "v" else _unpaired(c, z, _pairs(c, z) * turn)
        out[name] = (y / s).clamp(-448, 448) if c["out"] == "fp8" else y
    return out


def _exact_grad(c, st):
    out = torch.empty(c["B"], c["S"], c["Hq"] + 2 * c["Hkv"], c["d"], dtype=torch.float64, device="cuda")
    dws, first = {}, 0
    for g, x, w, name in zip((st["gq"], st["gk"]), _views(c, st["qkv"]), (st["wq"], st["wk"]), ("dwq", "dwk")):
        dw = torch.zeros(c["d"], dtype=torch.float64, device="cuda")
        for i in range(c["B"]):
            back = _rotation(c, st, i).conj()
            for h in range(x.shape[2]):
                dy = g[i, h].double()
                dy = _unpaired(c, dy, _pairs(c, dy) * back)
                if w is not None:
                    z = x[i, :, h].double()
                    n = torch.sqrt(z.square().sum(-1, keepdim=True) / c["d"] + EPS)
                    dw += (dy * z / n).sum(0)
                    dy = dy * w.double()
                    dy = dy / n - z * (dy * z).sum(-1, keepdim=True) / (c["d"] * n ** 3)
                out[i, :, first + h] = dy
        first += x.shape[2]
        if w is not None:
            dws[name] = dw
    out[:, :, first:] = st["gv"].double().transpose(1, 2)
    return {"dqkv": out.view(st["qkv"].shape), **dws}


def _exact_append(c, st):
    held, new = _held(c)
    t, scales = c["block"], st["scales"].view(torch.uint8).clone()
    out = {x: st[x + "c"].double() for x in "kv"}
    for b in range(c["B"]):
        end = min(held[b] + new[b], c["cap"])
        for first in range(held[b] // t * t, end, t):
            lo, hi = max(first, held[b]), min(first + t, end)
            if lo >= hi:
                continue
            for i, x in enumerate("kv"):
                rows = st[x][b, :, lo - held[b]:hi - held[b]].double()  # [Hkv, tokens, d]
                need = torch.ceil(torch.log2(rows.abs().amax((-1, -2)).clamp(min=448 * 2.0 ** -126) / 448.0))
                if lo > first:
                    was = scales[b, :, first // t, i].double() - 127
                    need = torch.maximum(need, was)
                    old = out[x][b, :, first:lo]
                    out[x][b, :, first:lo] = _e4m3(old * torch.exp2(was - need)[:, None, None])
                out[x][b, :, lo:hi] = _e4m3(rows / torch.exp2(need)[:, None, None])
                scales[b, :, first // t, i] = (need + 127).to(torch.uint8)
    return {**out, "scales": torch.exp2(scales.double() - 127),
            "lens": torch.tensor([min(a + b, c["cap"]) for a, b in zip(held, new)], dtype=torch.int32)}


def _exact_blocks(c, st):
    g, lens, t = c["Hq"] // c["Hkv"], _lens(c), c["block"]
    c1 = float(np.float32(st["scale"] * LOG2E))
    factors = torch.exp2(st["scales"].view(torch.uint8).double() - 127)
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c["B"]):
        n = lens[b]
        hide = torch.arange(n, device="cuda") > (torch.arange(c["Sq"], device="cuda") + (n - c["Sq"])).unsqueeze(-1)
        for h in range(c["Hkv"] if n else 0):
            k, v = (st[x][b, h, :n].double() * factors[b, h, :, i].repeat_interleave(t)[:n, None]
                    for i, x in enumerate("kv"))
            for r in range(h * g, (h + 1) * g):
                x = (st["q"][b, r].double() @ k.T * c1).masked_fill(hide, -math.inf)  # base-two exponents
                top = x.amax(-1, keepdim=True)
                base = top.masked_fill(top == -math.inf, 0.0)
                if c["mode"] == "exact":
                    w = torch.exp2(x - base)
                else:
                    w, f = torch.zeros_like(x), 2.0 ** ORDER[c["mode"]]
                    for j in range(0, n, TILE):
                        if j % (c["cut"] or n) == 0:
                            a = torch.full_like(top, -math.inf)
                        y = x[:, j:j + TILE]
                        a = torch.maximum(a, y.amax(-1, keepdim=True))
                        z = torch.round((y - a.masked_fill(a == -math.inf, 0.0)) * f).clamp(min=-126 * f) / f
                        z = torch.exp2(z.floor()) * (1 + z - z.floor()) * torch.exp2(a - base)
                        w[:, j:j + TILE] = torch.where(y == -math.inf, 0.0, z)
                total = w.sum(-1, keepdim=True)
                o[b, r] = torch.where(total > 0, (w @ v) / total, 0.0)
                lse[b, r] = ((top + torch.log2(total)) / LOG2E).squeeze(-1)
    return {"o": o, "lse": lse}

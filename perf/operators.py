"""Serving with a key/value cache that is shared and kept small, as timed cases: attention for a batch that shares a long
prefix (``prefix``), the attention weight that each cached key has received (``weights``), and the eviction of the keys
that received least (``evict``).

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
TYPES = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "fp8": 1}


def _prefix(name, dtype, b, hq, hkv, sq, p, sk, d, mode, sharp=False, p_cut=0, cut=0, empty=False):
    # p_cut, cut: keys of a part, of the prefix and of the own caches (lattice weights are rounded relative to their
    # part's running maximum; the hardware exponential does not depend on them and takes the library's choice)
    return {"name": name, "kind": "prefix", "dtype": dtype, "B": b, "Hq": hq, "Hkv": hkv, "Sq": sq, "P": p, "Sk": sk,
            "d": d, "mode": mode, "sharp": sharp, "p_cut": p_cut, "cut": cut, "empty": empty}


def _weights(name, dtype, b, hq, hkv, sq, sk, d, decay, sharp=False, empty=False):
    return {"name": name, "kind": "weights", "dtype": dtype, "B": b, "Hq": hq, "Hkv": hkv, "Sq": sq, "Sk": sk, "d": d,
            "decay": decay, "sharp": sharp, "empty": empty}


def _evict(name, dtype, b, hkv, sk, keep, recent, d, ties=False, empty=False):
    return {"name": name, "kind": "evict", "dtype": dtype, "B": b, "Hkv": hkv, "Sk": sk, "keep": keep, "recent": recent,
            "d": d, "ties": ties, "empty": empty}


def listed():
    return [
        # a small model's assistant: four chats over one short instruction, bound by the call and its launches
        _prefix("prefix_bf16_b4h8kv2_p500_d64", "bf16", 4, 8, 2, 1, 500, 60, 64, "exact"),
        # a serving batch over one system prompt with examples, each chat with its own turns
        _prefix("prefix_bf16_b32h32kv8_p8192", "bf16", 32, 32, 8, 1, 8192, 1024, 128, "exact", sharp=True),
        # four drafted tokens of an odd batch with the lattice weights, odd lengths, one cache still empty
        _prefix("prefix_fp8_b7h24kv8_sq4_p5003", "fp8", 7, 24, 8, 4, 5003, 777, 128, "h15", True, 1024, 256, empty=True),
        # the largest: a whole document of 32K tokens asked about by 64 chats at once
        _prefix("prefix_fp8_b64h32kv8_p32768", "fp8", 64, 32, 8, 1, 32768, 2048, 128, "exact"),
        # the smallest: one short chat of a small model, one new token
        _weights("weights_bf16_b1h8kv2_sk300_d64", "bf16", 1, 8, 2, 1, 300, 64, 1.0),
        # a decode step of a serving batch: every key of every cache gets its weight
        _weights("weights_bf16_b16h32kv8_sk8192", "bf16", 16, 32, 8, 1, 8192, 128, 1.0, sharp=True),
        # ragged FP8 caches at head dimension 64, older weights fading
        _weights("weights_fp8_b5h24kv8_sk5001_d64", "fp8", 5, 24, 8, 1, 5001, 64, 0.99, empty=True),
        # the last 64 tokens of two long prompts look back, to choose the keys worth keeping
        _weights("weights_fp8_b2h32kv8_sq64_sk16384", "fp8", 2, 32, 8, 64, 16384, 128, 0.0),
        # a whole prompt of 8K tokens, every query counted
        _weights("weights_bf16_b1h32kv8_sq8192", "bf16", 1, 32, 8, 8192, 8192, 128, 0.0),
        # the smallest: a short cache loses two thirds of its keys
        _evict("evict_bf16_b1kv2_sk300_keep100_d64", "bf16", 1, 2, 300, 100, 20, 64),
        # a 32K prompt brought down to 2K keys, many weights equal
        _evict("evict_bf16_b1kv8_sk32768_keep2048", "bf16", 1, 8, 32768, 2048, 64, 128, ties=True),
        # a serving batch whose ragged caches have outgrown their budget
        _evict("evict_fp8_b32kv8_sk5000_keep4096", "fp8", 32, 8, 5000, 4096, 256, 128, empty=True),
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
        kind = rng.choice(["prefix", "weights", "evict"])
        dtype, d = rng.choice(["bf16", "fp8"]), rng.choice([64, 128, 128])
        hq, hkv = _heads(rng)
        sharp, empty = rng.random() < 0.4, rng.random() < 0.3
        if kind == "prefix":
            mode = rng.choice(["exact"] * 5 + ["h15"] * 3 + ["sq4", "sq8"])
            p = 0 if rng.random() < 0.1 else _log_int(rng, 1, 32768)
            sk = _log_int(rng, 1, 4096)
            cuts = [rng.choice([0, 128 * rng.randint(2, 16)]) if mode != "exact" else 0 for _ in range(2)]
            c = _prefix("", dtype, _log_int(rng, 1, 64), hq, hkv, rng.choice([1, 1, 1, 2, 4, 7, 16]), p, sk, d, mode,
                        sharp, cuts[0], cuts[1], empty)
        elif kind == "weights":
            sk = _log_int(rng, 1, 65536)
            sq = rng.choice([1, 1, 1, 4, _log_int(rng, 2, 256), _log_int(rng, 2, 8192)])
            c = _weights("", dtype, _log_int(rng, 1, 64), hq, hkv, min(sq, sk), sk, d, rng.choice([0.0, 1.0, 0.9]), sharp,
                         empty)
        else:
            sk = _log_int(rng, 2, 65536)
            keep = _log_int(rng, 1, sk)
            c = _evict("", dtype, _log_int(rng, 1, 64), hkv, sk, keep, rng.randint(0, keep), d, rng.random() < 0.4, empty)
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


def work(case):
    c, e = case, BYTES[case["dtype"]]
    lens = _lens(c)
    keys = c["Hkv"] * float(sum(lens))
    if c["kind"] == "evict":
        kept = c["Hkv"] * float(sum(min(n, c["keep"]) for n in lens))
        return {"bytes": 4 * keys + kept * (2 * 2 * c["d"] * e + 8), "flops": keys}
    rows = c["B"] * c["Hq"] * c["Sq"]
    # row i of a sequence sees its first n - Sq + i + 1 keys
    seen = float(sum(sum(range(max(0, n - c["Sq"] + 1), n + 1)) for n in lens)) * c["Hq"]
    if c["kind"] == "weights":
        return {"bytes": rows * (c["d"] * e + 4) + keys * (c["d"] * e + (4 if c["decay"] == 0 else 8)),
                "flops": 2.0 * c["d"] * seen}
    return {"bytes": rows * (c["d"] * (e + 2) + 4) + 2.0 * (keys + c["Hkv"] * c["P"]) * c["d"] * e,
            "flops": 4.0 * c["d"] * (seen + float(rows) * c["P"])}


def _scale(c):
    return float(np.float32(1.0 / math.sqrt(c["d"])))


def _stored(c, x):
    """A tensor in the operand type, and its descale (FP8: one scale per tensor, amax / 448)."""
    if c["dtype"] == "bf16" or x.numel() == 0:
        return x.to(TYPES[c["dtype"]]), 1.0
    s = float(x.abs().max()) / 448.0
    return (x / s).to(torch.float8_e4m3fn), s


def _sharpen(c, x, gen):
    """2% of the keys of each head four times as large: the keys that many queries look at."""
    n = int(round(0.02 * x.shape[-2]))
    if c["sharp"] and n:
        at = torch.rand(x.shape[:-1], generator=gen, device="cuda").argsort(dim=-1)[..., :n, None].expand(*x.shape[:-2], n, c["d"])
        x.scatter_(-2, at, 4 * x.gather(-2, at))
    return x


def _limits(c, lens):
    """The last own key that each query row of a sequence sees, -1 for none: [B, Sq]."""
    n = torch.as_tensor(lens, device="cuda").view(-1, 1)
    return (n - c["Sq"] + torch.arange(c["Sq"], device="cuda")).clamp(min=-1)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    lens = _lens(c)
    st = {"case": c, "lens": torch.tensor(lens, dtype=torch.int32, device="cuda"), "scale": _scale(c)}
    own_shape = (c["B"], c["Hkv"], c["Sk"], c["d"])
    if c["kind"] == "evict":
        st["k"], st["v"] = (_stored(c, normal(*own_shape))[0] for _ in range(2))
        # accumulated weights: a few keys have most; "ties": weights that were counted in whole steps
        acc = torch.exp(2.0 * normal(*own_shape[:3]))
        st["acc"] = torch.floor(4.0 * acc) if c["ties"] else acc
        # the compact cache that the kept keys move to, empty so far
        out = (c["B"], c["Hkv"], c["keep"])
        st["k_out"], st["v_out"] = (torch.zeros(*out, c["d"], dtype=torch.uint8, device="cuda").repeat_interleave(BYTES[c["dtype"]], -1)
                                    .view(TYPES[c["dtype"]]) for _ in range(2))
        st["acc_out"] = torch.zeros(out, device="cuda")
        st["index"] = torch.zeros(out, dtype=torch.int32, device="cuda")
        st["lens_out"] = torch.zeros(c["B"], dtype=torch.int32, device="cuda")
        return st
    q, qd = _stored(c, normal(c["B"], c["Hq"], c["Sq"], c["d"]))
    k, v = _sharpen(c, normal(*own_shape), gen), normal(*own_shape)
    if c["kind"] == "prefix":
        kp, vp = (normal(c["Hkv"], c["P"], c["d"]) for _ in range(2))
        kp = _sharpen(c, kp, gen)
        if c["dtype"] == "fp8":  # prefix and own caches have one scale
            kd, vd = (float(max(t.abs().max() for t in pair if t.numel())) / 448.0 for pair in ((k, kp), (v, vp)))
            st["k"], st["v"], st["kp"], st["vp"] = ((t / s).to(torch.float8_e4m3fn) for t, s in ((k, kd), (v, vd), (kp, kd), (vp, vd)))
        else:
            kd = vd = 1.0
            st["k"], st["v"], st["kp"], st["vp"] = (t.to(torch.bfloat16) for t in (k, v, kp, vp))
        st["q"], st["descale"] = q, (qd, kd, vd)
        st["out"] = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
        st["lse"] = torch.empty(q.shape[:3], dtype=torch.float32, device="cuda")
        return st
    st["q"], (st["k"], kd) = q, _stored(c, k)
    st["descale"] = (qd, kd, 1.0)
    # what the attention call before returned: the log-sum of every query row
    lse, limits, g = torch.empty(q.shape[:3], device="cuda"), _limits(c, lens), c["Hq"] // c["Hkv"]
    keys = torch.arange(c["Sk"], device="cuda")
    for b in range(c["B"]):
        hide = keys > limits[b].view(-1, 1)
        for h in range(c["Hq"]):
            s = (q[b, h].float() @ st["k"][b, h // g].float().T) * (st["scale"] * qd * kd)
            lse[b, h] = s.masked_fill_(hide, -math.inf).logsumexp(-1)
    st["lse"] = lse
    st["acc"] = torch.rand(own_shape[:3], generator=gen, device="cuda")
    return st


# ---- the plain forms ------------------------------------------------------

def _hidden(c, st):
    """Own keys that a row does not see: [B, 1, G Sq, Sk]."""
    last = (st["lens"].view(-1, 1) - c["Sq"] + torch.arange(c["Sq"], device="cuda")).repeat(1, c["Hq"] // c["Hkv"])
    return (torch.arange(c["Sk"], device="cuda") > last.unsqueeze(-1)).unsqueeze(1)


def _scores(c, st, t):
    """Raw logits against the prefix and against the own caches, both [B, Hkv, G Sq, keys]."""
    q = st["q"].to(t).view(c["B"], c["Hkv"], -1, c["d"])
    own_s = (q @ st["k"].to(t).transpose(-1, -2)).masked_fill(_hidden(c, st), -math.inf)
    if "kp" not in st:
        return None, own_s
    rows = q.transpose(0, 1).reshape(c["Hkv"], -1, c["d"])  # the prefix meets the rows of all sequences at once
    pre_s = rows @ st["kp"].to(t).transpose(-1, -2)
    return pre_s.view(c["Hkv"], c["B"], -1, c["P"]).transpose(0, 1), own_s


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


def _plain_prefix(c, st):
    t = torch.float32 if c["mode"] == "exact" else torch.float64  # a lattice weight next to a border needs the 64
    qd, kd, vd = st["descale"]
    c1 = float(np.float32(st["scale"] * qd * kd * LOG2E))
    parts = _scores(c, st, t)
    m = torch.cat([x.amax(-1, keepdim=True) for x in parts if x.shape[-1]], -1).amax(-1, keepdim=True)
    base = m.masked_fill(m == -math.inf, 0.0)
    if c["mode"] == "exact":
        pre_w, own_w = (torch.exp2((x - base) * c1) for x in parts)
    else:
        pre, mine = _lattice(parts[0], c["p_cut"], c1, ORDER[c["mode"]]), _lattice(parts[1], c["cut"], c1, ORDER[c["mode"]])
        pre_w, own_w = (w * torch.exp2((a - base) * c1) for w, a in (pre, mine))
    total = pre_w.sum(-1, keepdim=True) + own_w.sum(-1, keepdim=True)
    rows = pre_w.transpose(0, 1).reshape(c["Hkv"], -1, c["P"]) @ st["vp"].to(t)
    o = rows.view(c["Hkv"], c["B"], -1, c["d"]).transpose(0, 1) + own_w @ st["v"].to(t)
    o = torch.where(total > 0, o / total * vd, 0.0)
    lse = (m * c1 + torch.log2(total)) * math.log(2.0)
    return {"o": o.reshape(st["q"].shape).to(torch.bfloat16), "lse": lse.reshape(st["q"].shape[:3]).float()}


def _plain_weights(c, st):
    qd, kd, _ = st["descale"]
    s = _scores(c, st, torch.float32)[1] * (st["scale"] * qd * kd)
    lse = st["lse"].view(c["B"], c["Hkv"], -1, 1)
    got = torch.exp(s - lse).masked_fill(s == -math.inf, 0.0).sum(-2, dtype=torch.float64)
    held = torch.arange(c["Sk"], device="cuda") < st["lens"].view(-1, 1, 1)
    old = c["decay"] * st["acc"] if c["decay"] else torch.zeros_like(st["acc"])
    return st["acc"].copy_(torch.where(held, (old + got).float(), st["acc"]))


def _plain_evict(c, st):
    n = st["lens"].view(-1, 1, 1)
    slot = torch.arange(c["Sk"], device="cuda")
    score = st["acc"].masked_fill(slot >= n - c["recent"], math.inf).masked_fill(slot >= n, -1.0)  # (weights are 0 or more)
    best = score.sort(dim=-1, descending=True, stable=True).indices[..., :c["keep"]]  # equal ones: the lowest first
    best = best.masked_fill(best >= n, c["Sk"]).sort(dim=-1).values
    real = best < c["Sk"]
    at = best.clamp(max=c["Sk"] - 1)
    rows = at.unsqueeze(-1).expand(-1, -1, -1, c["d"] * BYTES[c["dtype"]])
    k, v = (torch.where(real.unsqueeze(-1), st[x].view(torch.uint8).gather(2, rows), st[x + "_out"].view(torch.uint8))
            .view(TYPES[c["dtype"]]) for x in ("k", "v"))
    acc = torch.where(real, st["acc"].gather(2, at), st["acc_out"])
    return {"k": k, "v": v, "acc": acc, "index": torch.where(real, at, -1).int(),
            "lens": st["lens"].clamp(max=c["keep"])}


# ---- the library's calls --------------------------------------------------

def _own_prefix(c, st):
    import paper_2609_33586_amd as attn
    if "plan" not in st:  # a decode loop keeps its cuts and its workspace from step to step
        cuts = (c["p_cut"], c["cut"])
        if c["mode"] == "exact":
            cuts = attn.attn_decode_prefix_split_keys(c["B"], c["Hq"], c["Hkv"], c["Sq"], c["P"], c["Sk"], c["d"],
                                                      attn.ATTN_BF16 if c["dtype"] == "bf16" else attn.ATTN_FP8_E4M3)
        need = attn.attn_decode_prefix_workspace_bytes(c["B"], c["Hq"], c["Sq"], c["P"], c["Sk"], c["d"], *cuts)
        st["plan"] = cuts, torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    (p_cut, cut), ws = st["plan"]
    o, lse = attn.attn_decode_prefix(st["q"], st["kp"], st["vp"], st["k"], st["v"], lens=st["lens"], causal=True,
                                     scale=st["scale"], exp_mode=MODES[c["mode"]], prefix_split_keys=p_cut,
                                     split_keys=cut, descale=st["descale"], out=st["out"], lse=st["lse"], workspace=ws)
    return {"o": o, "lse": lse}


def _own_weights(c, st):
    import paper_2609_33586_amd as attn
    if "plan" not in st:
        need = attn.attn_key_weights_workspace_bytes(c["B"], c["Hq"], c["Hkv"], c["Sq"], c["Sk"], c["d"])
        st["plan"] = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
    return attn.attn_key_weights(st["q"], st["k"], st["lse"], st["acc"], lens=st["lens"], causal=True,
                                 scale=st["scale"], decay=c["decay"], descale=st["descale"], workspace=st["plan"])


def _own_evict(c, st):
    import paper_2609_33586_amd as attn
    k, v, acc, index, lens = attn.attn_evict(st["k"], st["v"], st["acc"], lens=st["lens"], keep=c["keep"],
                                             recent=c["recent"], k_out=st["k_out"], v_out=st["v_out"],
                                             acc_out=st["acc_out"], index=st["index"], lens_out=st["lens_out"])
    return {"k": k, "v": v, "acc": acc, "index": index, "lens": lens}


def run(state):
    c = state["case"]
    if own:
        return {"prefix": _own_prefix, "weights": _own_weights, "evict": _own_evict}[c["kind"]](c, state)
    return {"prefix": _plain_prefix, "weights": _plain_weights, "evict": _plain_evict}[c["kind"]](c, state)


# ---- 64 bits --------------------------------------------------------------

def exact(case, seed):
    return {"prefix": _exact_prefix, "weights": _exact_weights, "evict": _exact_evict}[case["kind"]](case, prepare(case, seed))


def _exact_prefix(c, st):
    g, lens = c["Hq"] // c["Hkv"], _lens(c)
    qd, kd, vd = st["descale"]
    c1 = float(np.float32(st["scale"] * qd * kd * LOG2E))
    o = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(st["q"].shape[:3], dtype=torch.float64, device="cuda")
    for h in range(c["Hkv"]):
        kp, vp = st["kp"][h].double(), st["vp"][h].double()
        for b in range(c["B"]):
            heads = slice(h * g, (h + 1) * g)
            q = st["q"][b, heads].double()  # [g, Sq, d]
            n = lens[b]
            x = torch.cat([q @ kp.T, q @ st["k"][b, h, :n].double().T], -1) * c1  # base-two exponents
            last = torch.arange(c["Sq"], device="cuda") + (c["P"] + n - c["Sq"])
            hide = torch.arange(c["P"] + n, device="cuda") > last.clamp(min=c["P"] - 1).unsqueeze(-1)
            x = x.masked_fill(hide, -math.inf)
            if not x.shape[-1]:
                lse[b, heads] = -math.inf
                continue
            v = torch.cat([vp, st["v"][b, h, :n].double()], 0)
            top = x.amax(-1, keepdim=True)
            dead = top == -math.inf
            if c["mode"] == "exact":
                w = torch.exp2(x - top.masked_fill(dead, 0.0))
            else:
                w = torch.zeros_like(x)
                for start, end, cut in ((0, c["P"], c["p_cut"]), (c["P"], c["P"] + n, c["cut"])):
                    for j in range(start, end, TILE):
                        if (j - start) % (cut or end) == 0:
                            a = torch.full_like(top, -math.inf)
                        t = x[..., j:min(j + TILE, end)]
                        a = torch.maximum(a, t.amax(-1, keepdim=True))
                        f = 2.0 ** ORDER[c["mode"]]
                        y = torch.round((t - a.masked_fill(a == -math.inf, 0.0)) * f).clamp(min=-126 * f) / f
                        y = torch.exp2(y.floor()) * (1 + y - y.floor()) * torch.exp2(a - top.masked_fill(dead, 0.0))
                        w[..., j:min(j + TILE, end)] = torch.where(t == -math.inf, 0.0, y)
            total = w.sum(-1, keepdim=True)
            o[b, heads] = torch.where(dead, 0.0, (w @ v) / total * vd)
            lse[b, heads] = ((top + torch.log2(total)) / LOG2E).squeeze(-1)
    return {"o": o, "lse": lse}


def _exact_weights(c, st):
    g, lens = c["Hq"] // c["Hkv"], _lens(c)
    acc, a = st["acc"].double(), st["scale"] * st["descale"][0] * st["descale"][1]
    for b in range(c["B"]):
        n = lens[b]
        last = torch.arange(c["Sq"], device="cuda") + (n - c["Sq"])
        for h in range(c["Hkv"]):
            k, new = st["k"][b, h, :n].double(), torch.zeros(n, dtype=torch.float64, device="cuda")
            for r in range(h * g, (h + 1) * g):
                x = st["q"][b, r].double() @ k.T * a - st["lse"][b, r].double().unsqueeze(-1)
                new += torch.where(torch.arange(n, device="cuda") <= last.unsqueeze(-1), x.exp(), 0.0).sum(0)
            acc[b, h, :n] = (c["decay"] * acc[b, h, :n] if c["decay"] else 0.0) + new
    return acc


def _exact_evict(c, st):
    out = {x: st[x + "_out"].to(torch.float64) for x in ("k", "v", "acc")}
    index = torch.full(st["index"].shape, -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(_lens(c)):
        for h in range(c["Hkv"]):
            old, late = st["acc"][b, h].double().cpu().numpy(), max(0, n - c["recent"])
            if n <= c["keep"]:
                kept = np.arange(n)
            else:
                first = np.lexsort((np.arange(late), -old[:late]))[:c["keep"] - (n - late)]
                kept = np.sort(np.concatenate([first, np.arange(late, n)]))
            at = torch.from_numpy(kept).to("cuda")
            index[b, h, :len(kept)] = at.int()
            for x in ("k", "v", "acc"):
                out[x][b, h, :len(kept)] = st[x][b, h].double()[at]
    return {**out, "index": index, "lens": torch.tensor([min(n, c["keep"]) for n in _lens(c)], dtype=torch.int32)}

"""Plain float64 forms of the operators over shared and bounded caches, and the
tolerances that follow from the kernels' arithmetic.

Rounding: half a step of BF16 is 2^-8 of a value, of FP32 2^-24.  A logit is a
sum of d products in FP32: off by at most d 2^-24 sum |q k| (e_s).  A weight
2^(c1 (s - m)) is then off by c1 ln2 2 e_s of itself (s and m), by 2^-23 of its
exponent in the fma and by a few 2^-24 in the exponential: rel below.  P is
rounded to BF16 (2^-8) for the hardware exponential, exact for the lattice
weights.  A lattice weight changes, by at most half of itself, where its
exponent lies within what its error can move over a rounding border; the share
of such weights is allowed as a slack."""
import math

import torch

import paper_2609_33586_amd as pkg

TILE = 128
LOG2E = 1.4426950408889634
EXACT, H15, SQ4, SQ8 = pkg.ATTN_EXP_EXACT, pkg.ATTN_EXP_H15, pkg.ATTN_EXP_SQ4, pkg.ATTN_EXP_SQ8
ORDER = {H15: 1, SQ4: 2, SQ8: 3}
BF16, FP8 = torch.bfloat16, torch.float8_e4m3fn


def say(msg):
    print(msg, flush=True)


def scale_of(d):
    return float(torch.tensor(1.0 / math.sqrt(d), dtype=torch.float32))


def randn(shape, seed, dtype, sharp=False):
    """Standard normals in the operand type (every 13th row four times as large if sharp); FP8: 30 times them, up to
    e4m3's largest value (the conversion makes NaN of what lies beyond)."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    x = torch.randn(*shape, generator=gen, device="cuda")
    if sharp:
        x[..., ::13, :] *= 4
    return (x * 30).clamp(-448, 448).to(dtype) if dtype == FP8 else x.to(dtype)


#: descales of the FP8 test operands, which are 30 times normals
DESCALE = (1 / 32, 1 / 30, 1 / 28)


def visible(n, Sq, causal):
    """Own keys that each position sees: [Sq, n]."""
    j, i = torch.arange(n, device="cuda"), torch.arange(Sq, device="cuda")
    return j <= (n - Sq + i).unsqueeze(-1) if causal else torch.ones(Sq, n, dtype=torch.bool, device="cuda")


def prefix_ref(q, kp, vp, k, v, lens, causal, scale, descale, mode, p_cut, cut):
    """O, LSE in float64 and the tolerances of both."""
    B, Hq, Sq, d = q.shape
    Hkv = kp.shape[0] if kp is not None else k.shape[1]
    qd, kd, vd = descale or (1.0, 1.0, 1.0)
    c1 = float(torch.tensor(scale * qd * kd * LOG2E, dtype=torch.float32))
    O = torch.zeros(B, Hq, Sq, d, dtype=torch.float64, device="cuda")
    L = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device="cuda")
    tol_o, tol_l = torch.zeros_like(O), torch.zeros_like(L)
    for b in range(B):
        for h in range(Hq):
            g, qq = h // (Hq // Hkv), q[b, h].double()
            groups = []  # (keys, values, seen, cut)
            if kp is not None and kp.shape[1]:
                groups.append((kp[g].double(), vp[g].double(),
                               torch.ones(Sq, kp.shape[1], dtype=torch.bool, device="cuda"), p_cut))
            n = lens[b] if k is not None else 0
            if n:
                groups.append((k[b, g, :n].double(), v[b, g, :n].double(), visible(n, Sq, causal), cut))
            if not groups:
                continue
            s = [(qq @ kk.T).masked_fill(~see, -math.inf) for kk, _, see, _ in groups]
            vv = torch.cat([x for _, x, _, _ in groups]) * vd
            e_s = d * 2.0 ** -24 * torch.cat([qq.abs() @ kk.abs().T for kk, _, _, _ in groups], -1)
            e_max = e_s.amax(-1, keepdim=True)
            m = torch.cat([x.amax(-1, keepdim=True) for x in s], -1).amax(-1, keepdim=True)
            base = m.masked_fill(m == -math.inf, 0.0)
            w, near = [], []
            for x, (_, _, _, part) in zip(s, groups):
                if mode == EXACT:
                    w.append(torch.exp2((x - base) * c1))
                    near.append(torch.zeros_like(x))
                    continue
                f = 2.0 ** ORDER[mode]
                ws, ns = [], []
                for j in range(0, x.shape[1], TILE):
                    t = x[:, j:j + TILE]
                    if j % (part or x.shape[1]) == 0:
                        a = torch.full_like(m, -math.inf)
                    a = torch.maximum(a, t.amax(-1, keepdim=True))
                    anchor = a.masked_fill(a == -math.inf, 0.0)
                    y = ((t - anchor) * c1 * f).clamp(min=-126 * f)
                    r = torch.round(y) / f
                    ww = torch.exp2(r.floor()) * (1 + r - r.floor()) * torch.exp2((anchor - base) * c1)
                    ww = torch.where(t == -math.inf, 0.0, ww)
                    reach = 2 * c1 * f * e_max + 2.0 ** -22 * (y.abs() + (anchor * c1 * f).abs())
                    ns.append(torch.where((y - y.floor() - 0.5).abs() <= reach, 0.5 * ww, 0.0).nan_to_num(0.0))
                    ws.append(ww)
                w.append(torch.cat(ws, -1))
                near.append(torch.cat(ns, -1))
            w, near, x = torch.cat(w, -1), torch.cat(near, -1), torch.cat(s, -1)
            l = w.sum(-1, keepdim=True)
            live = (l > 0).squeeze(-1)
            o = torch.where(l > 0, (w @ vv) / l, 0.0)
            O[b, h], L[b, h] = o, torch.where(live, ((m * c1 + torch.log2(l)) / LOG2E).squeeze(-1), -math.inf)
            p, slack = (w / l).nan_to_num(0.0), (near / l).nan_to_num(0.0)
            expo = ((x - base).abs() * c1).masked_fill(x == -math.inf, 0.0).amax(-1, keepdim=True)
            tiles = w.shape[-1] / TILE + 64
            rel = 2 * LOG2E * math.log(2) * c1 * e_max + 2.0 ** -23 * (expo + (base * c1).abs()) + tiles * 2.0 ** -24 + 2.0 ** -20
            away = p @ vv.abs()
            tol_o[b, h] = 2.0 ** -8 * o.abs() + away * ((2.0 ** -8 if mode == EXACT else 0.0) + 2 * rel) \
                + 2 * (slack @ vv.abs() + slack.sum(-1, keepdim=True) * o.abs()) + 1e-30
            tol_l[b, h] = (rel + 2 * slack.sum(-1, keepdim=True)).squeeze(-1) + 2.0 ** -22 * (L[b, h].abs().nan_to_num(0.0, posinf=0.0) + 1)
    return O, L, tol_o, tol_l


def check_prefix(o, lse, ref, what):
    O, L, tol_o, tol_l = ref
    dead = L == -math.inf
    assert torch.equal(lse == -math.inf, dead), f"{what}: rows without a key"
    assert bool((o[dead] == 0).all()), f"{what}: O of rows without a key"
    do, dl = (o.double() - O).abs(), (lse.double() - L).abs().masked_fill(dead, 0.0)
    say(f"{what}: max |dO| / tolerance {(do / (tol_o + 1e-30)).max().item():.3f}, |dLSE| {(dl / tol_l).max().item():.3f}")
    assert bool((do <= tol_o).all()) and bool((dl <= tol_l).all()), what


def weights_ref(q, k, lse, acc, lens, causal, scale, descale, decay):
    """acc in float64 and its tolerance."""
    B, Hq, Sq, d = q.shape
    Hkv = k.shape[1]
    qd, kd = (descale or (1.0, 1.0))[:2]
    a = scale * qd * kd
    out, tol = acc.double().clone(), torch.zeros(acc.shape, dtype=torch.float64, device="cuda")
    for b in range(B):
        n = lens[b]
        if not n:
            continue
        see = visible(n, Sq, causal)
        for h in range(Hkv):
            kk = k[b, h, :n].double()
            new, err = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
            for r in range(h * (Hq // Hkv), (h + 1) * (Hq // Hkv)):
                qq, e = q[b, r].double(), lse[b, r].double().unsqueeze(-1)
                x = qq @ kk.T * a
                p = torch.where(see & (e > -math.inf), (x - e).exp(), 0.0)
                # logit, the two products with log2 e, the fma, the exponential
                rel = a * d * 2.0 ** -24 * (qq.abs() @ kk.abs().T) + 2.0 ** -22 * (x.abs() + e.abs().nan_to_num(0.0, posinf=0.0) + 4)
                new += p.sum(0)
                err += (p * rel).sum(0)
            old = decay * out[b, h, :n] if decay else 0.0
            out[b, h, :n] = old + new
            # 16 scores and one running sum a tile of 32 rows, parts, decay
            terms = 16 + Sq * (Hq // Hkv) / 32 + 4
            tol[b, h, :n] = 2 * err + terms * 2.0 ** -24 * (old + new) + 1e-37
    return out, tol


def evict_ref(acc, lens, keep, recent):
    """The indexes that stay, for each (b, h) a list."""
    import numpy as np
    a = acc.cpu().numpy()
    got = []
    for b in range(a.shape[0]):
        for h in range(a.shape[1]):
            n, x = lens[b], a[b, h].astype(np.float64) + 0.0
            if n <= keep:
                got.append(np.arange(n))
                continue
            late = n - min(recent, keep)
            key = np.where(np.isnan(x[:late]), np.inf, x[:late])
            nan = ~np.isnan(x[:late])  # NaN above infinity
            order = np.lexsort((np.arange(late), -key, nan))[:keep - (n - late)]
            got.append(np.sort(np.concatenate([order, np.arange(late, n)])))
    return got

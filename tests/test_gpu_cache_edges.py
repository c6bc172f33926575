"""The operators over shared and bounded caches where rounding cannot hide a
mistake: large logits whose weights and sums are exact, many parts, and values
that are not finite in one sequence of a batch."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import (BF16, DESCALE, EXACT, FP8, H15, SQ4, SQ8, check_prefix, prefix_ref, randn, say, scale_of,
                           weights_ref)

pytestmark = pytest.mark.gpu

LN2 = float(torch.tensor(math.log(2.0), dtype=torch.float32))  # logit scale 1 in base two: 1.0000000027, 1 in FP32

# Exact operands.  Channel 0 gives every logit a common part `base`, channel 1 an
# integer of -8..0 more, the other channels of q are zero: every product and
# partial sum is an integer below 2^24, which FP32 holds.  A weight is then a
# power of two in every mode (the lattice maps hold integers exactly, BF16 holds powers of
# two), and so is every rescale.  What rounds is the sum of weights times V in
# FP32, n terms: n 2^-24 of sum p |v|, the normaliser, its reciprocal and their
# product 2^-22, and O to BF16: 2^-8 of it.


def exact_operands(dt, d, B, Hq, Hkv, Sq, P, Sk, order, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    big = 256.0 if dt == FP8 else 512.0
    q = torch.zeros(B, Hq, Sq, d, device="cuda")
    q[..., 0], q[..., 1] = big, 1.0

    def steps(*shape):
        """Logits above the common part."""
        n = shape[-1]
        if order == "equal":
            return torch.zeros(shape, device="cuda")
        if order == "random":
            return -torch.randint(0, 9, shape, generator=gen, device="cuda").float()
        up = -((n - 1 - torch.arange(n, device="cuda")) * 9 // max(n, 1)).float()  # the maximum moves from tile to tile
        return (up if order == "rising" else up.flip(0)).expand(shape).contiguous()

    def keys(*shape):
        k = torch.randint(-8, 9, (*shape, d), generator=gen, device="cuda").float()
        k[..., 0], k[..., 1] = 256.0, steps(*shape)
        return k.to(dt)

    def values(*shape):
        return torch.randint(-8, 9, (*shape, d), generator=gen, device="cuda").float().add(3.0).to(dt)

    kp = vp = k = v = None
    if P:
        kp, vp = keys(Hkv, P), values(Hkv, P)
    if Sk:
        k, v = keys(B, Hkv, Sk), values(B, Hkv, Sk)
    return q.to(dt), kp, vp, k, v


def exact_ref(q, kp, vp, k, v, lens, causal):
    B, Hq, Sq, d = q.shape
    Hkv = kp.shape[0] if kp is not None else k.shape[1]
    O = torch.zeros(B, Hq, Sq, d, dtype=torch.float64, device="cuda")
    L = torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(O)
    for b in range(B):
        for h in range(Hq):
            g, n = h // (Hq // Hkv), lens[b] if k is not None else 0
            kk = torch.cat([x for x in (kp[g] if kp is not None else None, k[b, g, :n] if n else None) if x is not None]).double()
            vv = torch.cat([x for x in (vp[g] if vp is not None else None, v[b, g, :n] if n else None) if x is not None]).double()
            P = kk.shape[0] - n
            s = q[b, h].double() @ kk.T
            j, i = torch.arange(P + n, device="cuda"), torch.arange(Sq, device="cuda")
            if causal:
                s = s.masked_fill((j >= P) & (j - P > (n - Sq + i).unsqueeze(-1)), -math.inf)
            m = s.amax(-1, keepdim=True)
            w = torch.exp2(s - m)
            l = w.sum(-1, keepdim=True)
            O[b, h], L[b, h] = w @ vv / l, ((m + torch.log2(l)) * math.log(2.0)).squeeze(-1)
            tol[b, h] = 2.0 ** -8 * O[b, h].abs() + ((P + n) * 2.0 ** -24 + 2.0 ** -22) * (w / l @ vv.abs())
    return O, L, tol


def check_exact(got, ref, what):
    o, lse = got
    O, L, tol = ref
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all()), what
    assert (O.abs() > 4 * tol).double().mean().item() > 0.95, "the tolerance has to tell O from zero"
    d, dl = (o.double() - O).abs(), (lse.double() - L).abs()
    say(f"{what}: max |dO| / tolerance {(d / tol).max().item():.3f}, |dLSE| {dl.max().item():.2e}")
    assert bool((d <= tol).all()), what
    assert bool((dl <= 2.0 ** -22 * (L.abs() + 1)).all()), what  # ln 2 (m + log2 l): three roundings


# (B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut): the prefix in blocks of 32 and of 128
# rows, before an own cache, without own caches; own caches alone
EXACT_SHAPES = [
    (4, 1, 1, 1, 300, 130, [130] * 4, 128, 0),
    (50, 1, 1, 1, 300, 130, [130 - i for i in range(50)], 128, 0),
    (40, 4, 1, 1, 700, 70, [70 - i for i in range(40)], 256, 0),       # 160 rows
    (9, 6, 2, 5, 1500, 300, [300, 299, 64, 5, 128, 129, 130, 1, 30], 384, 128),  # 135 rows
    (4, 8, 2, 2, 256, 300, [300, 2, 257, 255], 0, 0),                  # before each own cache
    (3, 12, 4, 16, 0, 600, [600, 16, 257], 0, 128),                    # own caches alone
    (2, 2, 1, 1, 4000, 0, [0, 0], 0, 0),                               # one part of 32 tiles
]


@pytest.mark.parametrize("dt,d", [(BF16, 128), (BF16, 64), (FP8, 128), (FP8, 64)])
@pytest.mark.parametrize("order", ["equal", "random", "rising", "falling"])
def test_large_logits_with_exact_weights(order, dt, d):
    for x, (B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut) in enumerate(EXACT_SHAPES):
        q, kp, vp, k, v = exact_operands(dt, d, B, Hq, Hkv, Sq, P, Sk, order, 20 + x)
        t = torch.tensor(lens, dtype=torch.int32, device="cuda") if Sk else None
        ref = exact_ref(q, kp, vp, k, v, lens, True)
        for mode in (EXACT, H15, SQ4, SQ8):
            got = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=t, causal=True, scale=LN2, exp_mode=mode,
                                         prefix_split_keys=p_cut, split_keys=cut, descale=(1.0, 1.0, 1.0))
            torch.cuda.synchronize()
            check_exact(got, ref, f"{dt} d={d} {order} shape {x} mode {mode}")


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ4, SQ8])
def test_one_key_far_above_the_others(mode, dt):
    # logits are multiples of 2^12, up to 2^17 (e4m3: 2^16): the largest one's key has the weight 1, O is its V.  The
    # others have none, of the lattice's 2^-126 each, the least there is: they move O by |v| <= 11 times that
    for x, (B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut) in enumerate(EXACT_SHAPES):
        d = 128
        q, kp, vp, k, v = exact_operands(dt, d, B, Hq, Hkv, Sq, P, Sk, "equal", 40 + x)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(60 + x)
        for t in (kp, k):
            if t is not None:  # 16 values of either sign below the largest
                t[..., 0] = (16.0 * torch.randint(-15, 15, t.shape[:-1], generator=gen, device="cuda")).to(dt)
        for b in range(B):
            for g in range(Hkv):
                if P == 0 or (Sk and b % 2 and lens[b] >= Sq):
                    k[b, g, (7 * b + 3 * g) % (lens[b] - Sq + 1), 0] = 256.0
                if P:
                    kp[g, (101 * g + 290) % P, 0] = 240.0
        s = torch.tensor(lens, dtype=torch.int32, device="cuda") if Sk else None
        o, lse = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=s, causal=True, scale=LN2, exp_mode=mode,
                                        prefix_split_keys=p_cut, split_keys=cut, descale=(1.0, 1.0, 1.0))
        torch.cuda.synchronize()
        say(f"one key {dt} mode {mode} shape {x}")
        for b in range(B):
            for h in range(Hq):
                g = h // (Hq // Hkv)
                n = lens[b] if Sk else 0
                kk = torch.cat([y for y in (kp[g] if P else None, k[b, g, :n] if n else None) if y is not None])[:, 0].float()
                vv = torch.cat([y for y in (vp[g] if P else None, v[b, g, :n] if n else None) if y is not None])
                at = int(kk.argmax())
                others = kk.clone()
                others[at] = -1e9
                assert others.max() < kk[at]
                away = 0.0 if mode == EXACT else len(kk) * 11 * 2.0 ** -126
                assert bool(((o[b, h].double() - vv[at].double()).abs() <= away).all())
                top = float(q[0, 0, 0, 0]) * float(kk[at]) * math.log(2.0)
                assert bool(((lse[b, h].double() - top).abs() <= 2.0 ** -22 * (abs(top) + 1)).all())


# ---- many parts ---------------------------------------------------------------

# beyond 32 parts, which the merge takes at a time: (B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut)
MANY_PARTS = [
    (2, 4, 2, 1, 128 * 40 + 5, 0, None, 128, 0),                      # 41 parts of the prefix
    (3, 4, 2, 1, 128 * 33, 300, [300, 0, 129], 128, 128),             # 33 and three more, some empty
    (3, 2, 1, 3, 0, 128 * 66, [128 * 66, 0, 100], 0, 128),            # 66 own parts, all of them or all but one empty
    (2, 2, 1, 2, 0, 128 * 35, [1, 128 * 33 + 1], 0, 128),             # a row that sees no key at all; one key in part 34
    (1, 4, 1, 1, 128 * 64, 128 * 32, [128 * 32], 128, 128),           # 96 parts: three turns
    (40, 4, 1, 1, 128 * 34, 200, [5 * i for i in range(40)], 128, 128),  # 160 rows
]


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("x", range(len(MANY_PARTS)))
def test_more_parts_than_the_merge_takes_at_a_time(x, d, dt):
    B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut = MANY_PARTS[x]
    for mode, late in ((EXACT, False), (EXACT, True), (H15, True)):
        q = randn((B, Hq, Sq, d), 300, dt)
        kp, vp = (randn((Hkv, P, d), 301 + i, dt) for i in range(2)) if P else (None, None)
        k, v = (randn((B, Hkv, Sk, d), 303 + i, dt) for i in range(2)) if Sk else (None, None)
        if late:  # the largest logits lie after part 32
            t = kp if P > 33 * 128 else k
            t[..., 33 * 128:, :] = (t[..., 33 * 128:, :].float() * 4).clamp(-448, 448).to(dt)
        t = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None
        descale = DESCALE if dt == FP8 else None
        need = pkg.attn_decode_prefix_workspace_bytes(B, Hq, Sq, P, Sk, d, p_cut, cut)
        room = torch.full((need // 4 + 512,), float("nan"), device="cuda")
        o, lse = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=t, causal=True, scale=scale_of(d), exp_mode=mode,
                                        prefix_split_keys=p_cut, split_keys=cut, descale=descale,
                                        workspace=room[256:-256])
        torch.cuda.synchronize()
        assert bool(room[:256].isnan().all()) and bool(room[-256:].isnan().all())
        ref = prefix_ref(q, kp, vp, k, v, lens or [Sk] * B, True, scale_of(d), descale, mode, p_cut, cut)
        check_prefix(o, lse, ref, f"many parts {dt} d={d} {x} mode {mode} late={late}")
        # the tolerance tells O from zero, unless a row averages thousands of values
        assert (ref[0].abs() > ref[2]).double().mean() > 0.5 or not late


def weight_operands(dt, d, B, Hq, Hkv, Sq, Sk, lens, causal, seed):
    from test_gpu_cache_weights import row_lse
    q, k = randn((B, Hq, Sq, d), seed, dt), randn((B, Hkv, Sk, d), seed + 1, dt, sharp=True)
    descale = DESCALE if dt == FP8 else None
    a = scale_of(d) * (DESCALE[0] * DESCALE[1] if dt == FP8 else 1.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return q, k, row_lse(q, k, lens, causal, a), torch.rand((B, Hkv, Sk), generator=gen, device="cuda"), descale


# query rows in parts, of several batches and KV heads, whose rows see nothing in some parts
@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", [(2, 6, 3, 1100, 900, [900, 40]), (3, 80, 2, 70, 300, [300, 1, 257]),
                                   (2, 10, 1, 700, 1300, [1300, 1100])])
def test_row_parts_of_several_batches_and_heads(shape, d, dt):
    B, Hq, Hkv, Sq, Sk, lens = shape
    need = pkg.attn_key_weights_workspace_bytes(B, Hq, Hkv, Sq, Sk, d)
    assert need > 0
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for causal in (True, False):
        q, k, lse, acc, descale = weight_operands(dt, d, B, Hq, Hkv, Sq, Sk, lens, causal, 500)
        kw = dict(lens=t, causal=causal, scale=scale_of(d), decay=0.75, descale=descale)
        want, tol = weights_ref(q, k, lse, acc, lens, causal, scale_of(d), descale, 0.75)
        room = torch.full((need // 4 + 512,), float("nan"), device="cuda")
        got = acc.clone()
        pkg.attn_key_weights(q, k, lse, got, workspace=room[256:-256], **kw)
        torch.cuda.synchronize()
        diff = (got.double() - want).abs()
        say(f"row parts {dt} d={d} {shape} causal={causal}: {(diff / (tol + 1e-30)).max().item():.3f}")
        assert bool((diff <= tol).all())
        assert bool(room[:256].isnan().all()) and bool(room[-256:].isnan().all())
    # both launches captured, and replayed with other lengths
    g, held, eager = torch.cuda.CUDAGraph(), acc.clone(), acc.clone()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        pkg.attn_key_weights(q, k, lse, held, workspace=room[256:-256], **kw)
    for n in (lens[0], 3, 0, lens[0] // 2):
        t.fill_(n)
        t[0] = lens[0] - n
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        pkg.attn_key_weights(q, k, lse, eager, **kw)
        torch.cuda.synchronize()
        assert torch.equal(held, eager), n


# ---- values that are not finite -------------------------------------------------

@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_a_broken_sequence_leaves_the_others_alone(what, dt):
    # NaN in one sequence of a batch: the rows of the others, in the same workgroups of the prefix, keep every bit
    for B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut in EXACT_SHAPES[:6]:
        d = 128
        q = randn((B, Hq, Sq, d), 700, dt)
        kp, vp = (randn((Hkv, P, d), 701 + i, dt) for i in range(2)) if P else (None, None)
        k, v = (randn((B, Hkv, Sk, d), 703 + i, dt) for i in range(2))
        t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        descale = DESCALE if dt == FP8 else None
        for mode in (EXACT, H15):
            kw = dict(lens=t, causal=True, scale=scale_of(d), exp_mode=mode, prefix_split_keys=p_cut, split_keys=cut,
                      descale=descale)
            clean = pkg.attn_decode_prefix(q, kp, vp, k, v, **kw)
            bad = {"q": q.clone(), "k": k.clone(), "v": v.clone()}
            x = bad[what].float()
            x[1] = math.nan
            bad[what] = x.to(dt)
            o, lse = pkg.attn_decode_prefix(bad["q"], kp, vp, bad["k"], bad["v"], **kw)
            torch.cuda.synchronize()
            rest = [b for b in range(B) if b != 1]
            assert torch.equal(o[rest].view(torch.int16), clean[0][rest].view(torch.int16))
            assert torch.equal(lse[rest], clean[1][rest])
            if what == "v" or mode == EXACT:
                assert bool(o[1, :, -1].isnan().all())


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("Sq", [1, 40, 700])
def test_a_broken_key_or_row_stays_where_it_is(Sq, dt):
    # weights: a key of NaN spoils its own sum, a query row of NaN those of its KV head and batch
    B, Hq, Hkv, Sk, d = 3, 4, 2, 500, 128
    lens = [500, 300, 41]
    q, k, lse, acc, descale = weight_operands(dt, d, B, Hq, Hkv, Sq, Sk, lens, True, 800)
    lse = lse.masked_fill(lse == -math.inf, 9.0)
    kw = dict(lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), causal=True, scale=scale_of(d), descale=descale)
    clean = pkg.attn_key_weights(q, k, lse, acc.clone(), **kw)
    x = k.float()
    x[1, 1, 77] = math.nan
    got = pkg.attn_key_weights(q, x.to(dt), lse, acc.clone(), **kw)
    torch.cuda.synchronize()
    hit = torch.zeros_like(acc, dtype=torch.bool)
    hit[1, 1, 77] = True
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])
    x = q.float()
    x[1, 3, -1] = math.nan  # the last position sees every key
    got = pkg.attn_key_weights(x.to(dt), k, lse, acc.clone(), **kw)
    torch.cuda.synchronize()
    hit[1, 1, :300] = True
    assert bool(got[hit].isnan().all()) and torch.equal(got[~hit], clean[~hit])

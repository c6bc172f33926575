"""The attention weight of each cached key (attn_key_weights) against its
float64 form (cache_helpers.weights_ref)."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import BF16, DESCALE, EXACT, FP8, randn, say, scale_of, visible, weights_ref

pytestmark = pytest.mark.gpu


def row_lse(q, k, lens, causal, a):
    B, Hq, Sq, _ = q.shape
    g = Hq // k.shape[1]
    lse = torch.full((B, Hq, Sq), -math.inf, device="cuda")
    for b in range(B):
        n = lens[b]
        if n:
            for h in range(Hq):
                s = (q[b, h].float() @ k[b, h // g, :n].float().T * a).masked_fill(~visible(n, Sq, causal), -math.inf)
                lse[b, h] = s.logsumexp(-1)
    return lse


def setup(dt, d, B, Hq, Hkv, Sq, Sk, lens, causal, seed, cap=None):
    q, k = randn((B, Hq, Sq, d), seed, dt), randn((B, Hkv, cap or Sk, d), seed + 1, dt, sharp=True)
    descale = DESCALE if dt == FP8 else None
    a = scale_of(d) * (DESCALE[0] * DESCALE[1] if dt == FP8 else 1.0)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    acc = torch.rand((B, Hkv, cap or Sk), generator=gen, device="cuda")
    return q, k, row_lse(q, k, lens, causal, a), acc, descale


# (B, Hq, Hkv, Sq, Sk, lens)
SHAPES = [
    (1, 1, 1, 1, 1, None),
    (3, 4, 2, 1, 300, [300, 0, 257]),       # one new token, an empty cache
    (2, 8, 1, 4, 513, [513, 2]),            # 32 rows packed in one tile, fewer keys than rows
    (2, 6, 2, 11, 100, [100, 5]),           # 33 packed rows: two tiles
    (1, 4, 2, 31, 600, None),
    (2, 4, 2, 32, 300, [300, 40]),          # whole heads, one tile each
    (1, 3, 1, 77, 700, None),               # ragged last tiles
    (1, 2, 1, 500, 500, None),              # a whole prompt
    (2, 2, 2, 400, 300, [300, 20]),         # more rows than keys: the first see none
    (1, 2, 1, 1500, 1300, [1290]),          # 48 tiles of 64 rows: two row parts
    (2, 16, 2, 32, 200, [200, 30]),         # 256 rows: the most that stay in LDS
    (1, 9, 1, 29, 300, None),               # 261 packed rows, positions repeat within a tile
    (1, 40, 1, 70, 500, None),              # 40 heads of two tiles each: two row parts
]


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", [SHAPES[1], SHAPES[3], SHAPES[6], SHAPES[9], SHAPES[10], SHAPES[12]])
def test_rows_without_a_sum_give_nothing_whatever_they_hold(shape, d, dt):
    B, Hq, Hkv, Sq, Sk, lens = shape
    for causal in (True, False):
        q, k, lse, acc, descale = setup(dt, d, B, Hq, Hkv, Sq, Sk, lens or [Sk] * B, causal, 150)
        gen = torch.Generator(device="cuda")
        gen.manual_seed(151)
        out = torch.rand(lse.shape, generator=gen, device="cuda") < 0.2  # padding among the query rows
        out[:, 0] = True
        lse[out] = -math.inf
        say(f"weights, rows left out {dt} d={d} {shape} causal={causal}")
        want, tol = weights_ref(q, k, lse, acc, lens or [Sk] * B, causal, scale_of(d), descale, 0.5)
        bad = q.float()
        bad[out] = math.nan
        q = bad.to(q.dtype)
        t = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None
        pkg.attn_key_weights(q, k, lse, acc, lens=t, causal=causal, scale=scale_of(d), decay=0.5, descale=descale)
        torch.cuda.synchronize()
        assert bool(((acc.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_shapes(shape, d, dt):
    B, Hq, Hkv, Sq, Sk, lens = shape
    for causal in (True, False):
        for decay in (1.0, 0.0, 0.75):
            q, k, lse, acc, descale = setup(dt, d, B, Hq, Hkv, Sq, Sk, lens or [Sk] * B, causal, 100)
            what = f"weights {dt} d={d} {shape} causal={causal} decay={decay}"
            say(what)
            want, tol = weights_ref(q, k, lse, acc, lens or [Sk] * B, causal, scale_of(d), descale, decay)
            t = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None
            got = pkg.attn_key_weights(q, k, lse, acc, lens=t, causal=causal, scale=scale_of(d), decay=decay,
                                       descale=descale)
            torch.cuda.synchronize()
            assert got is acc
            diff = (got.double() - want).abs()
            say(f"  max difference / tolerance {(diff / (tol + 1e-30)).max().item():.3f}")
            assert bool((diff <= tol).all()), what


def test_weights_of_a_row_add_up_to_one():
    # without a mask every row's weights add up to 1; decode's LSE and forward's
    q, k = randn((2, 8, 1, 128), 1, BF16), randn((2, 2, 900, 128), 2, BF16)
    _, lse = pkg.attn_decode(q, k, k, causal=True, scale=scale_of(128), exp_mode=EXACT, split_keys=256)
    acc = pkg.attn_key_weights(q, k, lse, torch.zeros(2, 2, 900, device="cuda"), causal=True, scale=scale_of(128))
    assert torch.allclose(acc.sum(-1), torch.full((2, 2), 4.0, device="cuda"), rtol=1e-5)
    q = randn((1, 4, 333, 64), 3, FP8)
    k = randn((1, 4, 333, 64), 4, FP8)
    _, lse = pkg.attn_fwd_ex(q, k, k, causal=True, scale=scale_of(64), exp_mode=EXACT, descale=DESCALE)
    acc = pkg.attn_key_weights(q, k, lse, torch.zeros(1, 4, 333, device="cuda"), causal=True, scale=scale_of(64),
                               descale=DESCALE)
    # attn_fwd's FP8 logits are off by up to 2^-12 of sum |q k| scale (about 20)
    assert torch.allclose(acc.sum(-1), torch.full((1, 4), 333.0, device="cuda"), rtol=20 * 2.0 ** -12)


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_outside_is_read_or_written(d, dt):
    for B, Hq, Hkv, Sq, Sk, lens in (SHAPES[1], SHAPES[3], SHAPES[8]):
        cap = Sk + 41
        q, k, lse, acc, descale = setup(dt, d, B, Hq, Hkv, Sq, Sk, lens, True, 200, cap)
        t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        kw = dict(lens=t, Sk=Sk, causal=True, scale=scale_of(d), descale=descale)
        clean = pkg.attn_key_weights(q, k, lse, acc.clone(), **kw)
        room = torch.full((acc.numel() + 512,), float("nan"), device="cuda")
        guarded = room[256:-256].view(acc.shape)
        guarded.copy_(acc)
        for b in range(B):
            k.view(torch.uint8)[b, :, lens[b]:] = 0x7F if dt == FP8 else 0xFF
            guarded[b, :, lens[b]:] = float("nan")
        pkg.attn_key_weights(q, k, lse, guarded, **kw)
        torch.cuda.synchronize()
        for b in range(B):
            assert torch.equal(guarded[b, :, :lens[b]], clean[b, :, :lens[b]])
            assert bool(guarded[b, :, lens[b]:].isnan().all())
            assert torch.equal(clean[b, :, lens[b]:], acc[b, :, lens[b]:])
        assert bool(room[:256].isnan().all()) and bool(room[-256:].isnan().all())


def test_old_values_are_not_read_without_decay_and_rows_without_a_sum_give_nothing():
    q, k, lse, acc, _ = setup(BF16, 128, 1, 4, 2, 3, 200, [200], True, 300)
    want = pkg.attn_key_weights(q, k, lse, torch.zeros_like(acc), causal=True, scale=scale_of(128))
    got = pkg.attn_key_weights(q, k, lse, torch.full_like(acc, float("nan")), causal=True, scale=scale_of(128), decay=0.0)
    assert torch.equal(got, want)
    lse.fill_(-math.inf)
    got = pkg.attn_key_weights(q, k, lse, torch.zeros_like(acc), causal=True, scale=scale_of(128))
    assert bool((got == 0).all())


def test_caches_beyond_4_gib_and_graph():
    cap = 1 << 23
    k = torch.empty((5, 1, cap, 128), dtype=FP8, device="cuda")
    for b in range(5):
        k[b, 0, :300] = randn((300, 128), 800 + b, FP8)
    q = randn((5, 2, 1, 128), 810, FP8)
    lens = [300, 7, 0, 129, 250]
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    small = k[:, :, :300].contiguous()
    lse = row_lse(q, small, lens, True, scale_of(128) * DESCALE[0] * DESCALE[1])
    acc = torch.zeros((5, 1, cap), device="cuda")
    kw = dict(lens=t, causal=True, scale=scale_of(128), descale=DESCALE)
    pkg.attn_key_weights(q, k, lse, acc, Sk=300, **kw)
    want = pkg.attn_key_weights(q, small, lse, torch.zeros((5, 1, 300), device="cuda"), **kw)
    assert torch.equal(acc[:, :, :300], want) and bool((acc[:, :, 300:] == 0).all())
    # captured once, replayed: each replay adds what the eager call adds
    held = torch.zeros((5, 1, 300), device="cuda")
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.attn_key_weights(q, small, lse, held, **kw)
    eager = torch.zeros_like(held)
    for n in (300, 3, 0, 200):
        t.fill_(n)
        torch.cuda.synchronize()
        g.replay()
        pkg.attn_key_weights(q, small, lse, eager, **kw)
        torch.cuda.synchronize()
        assert torch.equal(held, eager), n

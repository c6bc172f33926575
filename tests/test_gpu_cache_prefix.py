"""Decode over a shared prefix (attn_decode_prefix) against its float64 form
(cache_helpers.prefix_ref), in both workgroup forms, with and without prefix
and own caches, ragged and empty caches, odd sizes and cuts."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import (BF16, DESCALE, EXACT, FP8, H15, SQ4, SQ8, check_prefix, prefix_ref, randn, say, scale_of)

pytestmark = pytest.mark.gpu


def make(dt, d, B, Hq, Hkv, Sq, P, Sk, seed, cap=None, P_cap=None, sharp=True):
    q = randn((B, Hq, Sq, d), seed, dt)
    kp = vp = k = v = None
    if P:
        kp, vp = randn((Hkv, P_cap or P, d), seed + 1, dt, sharp), randn((Hkv, P_cap or P, d), seed + 2, dt)
    if Sk:
        k, v = randn((B, Hkv, cap or Sk, d), seed + 3, dt, sharp), randn((B, Hkv, cap or Sk, d), seed + 4, dt)
    return q, kp, vp, k, v


def run_and_check(dt, d, B, Hq, Hkv, Sq, P, Sk, lens, mode, p_cut, cut, causal, seed):
    q, kp, vp, k, v = make(dt, d, B, Hq, Hkv, Sq, P, Sk, seed)
    descale = DESCALE if dt == FP8 else None
    what = f"prefix {dt} d={d} B={B} Hq={Hq} Hkv={Hkv} Sq={Sq} P={P} Sk={Sk} lens={lens} mode={mode} cuts={p_cut},{cut} causal={causal}"
    say(what)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens else None
    o, lse = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=t, causal=causal, scale=scale_of(d), exp_mode=mode,
                                    prefix_split_keys=p_cut, split_keys=cut, descale=descale)
    torch.cuda.synchronize()
    check_prefix(o, lse, prefix_ref(q, kp, vp, k, v, lens or [Sk] * B, causal, scale_of(d), descale, mode, p_cut, cut),
                 what)


# (B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut): up to 128 rows of a KV head over the
# batch the keys form of a prefix workgroup, beyond the rows form
SHAPES = [
    (1, 1, 1, 1, 1, 1, None, 0, 0),                       # one key on each side
    (3, 4, 2, 1, 200, 70, [70, 0, 33], 0, 0),             # an empty cache
    (2, 4, 1, 4, 513, 300, [300, 2], 128, 256),           # fewer own keys than rows
    (4, 8, 1, 1, 640, 1, [1, 1, 0, 1], 256, 128),         # 32 rows: a full block of the keys form
    (5, 8, 1, 1, 129, 257, [257, 128, 1, 0, 200], 0, 128),  # 40 rows: two blocks of the keys form
    (9, 6, 2, 5, 700, 65, [65, 64, 63, 0, 4, 5, 6, 1, 30], 384, 0),  # 135 rows: two row blocks, the second ragged
    (2, 12, 4, 16, 300, 260, None, 128, 128),             # 48 rows a sequence: two own row blocks
    (3, 2, 1, 3, 0, 400, [400, 1, 129], 0, 128),          # no prefix
    (3, 2, 1, 3, 0, 100, [100, 0, 2], 0, 0),              # no prefix, one part: O written at once
    (3, 2, 1, 2, 400, 0, None, 128, 0),                   # no own caches
    (40, 2, 1, 1, 150, 0, None, 0, 0),                    # no own caches, one part, 80 rows
    (17, 16, 2, 1, 2000, 40, None, 512, 0),               # 136 rows, several tiles a part
    (32, 4, 1, 1, 600, 20, None, 256, 0),                 # 128 rows: four full blocks of the keys form
    (43, 3, 1, 1, 1, 30, None, 0, 0),                     # 129 rows, one prefix key
    (3, 96, 1, 1, 1300, 70, [70, 0, 1], 1152, 0),         # 288 rows: three row blocks, the last with one wave
    (70, 4, 1, 1, 150, 0, None, 0, 0),                    # 280 rows, one part
    (4, 8, 2, 1, 256, 300, [300, 0, 1, 255], 0, 0),       # a prefix of two rounds, before each own cache
    (4, 8, 2, 2, 512, 129, [129, 0, 1, 128], 0, 0),       # two rounds, or four (BF16, d = 128): not before
    (3, 4, 2, 1, 513, 70, [70, 0, 33], 0, 0),             # more than two rounds: two launches
    (2, 12, 4, 16, 255, 260, [260, 17], 0, 0),            # 48 rows a sequence after the prefix
    (260, 4, 2, 1, 130, 20, [i % 21 for i in range(260)], 0, 0),  # more than 512 own caches: two launches
    (20, 2, 2, 40, 130, 90, [90 - 3 * i for i in range(20)], 0, 0),  # prompts after a prefix, some shorter than theirs
]


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
def test_shapes(shape, d, dt):
    B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut = shape
    for mode in (EXACT, H15):
        run_and_check(dt, d, B, Hq, Hkv, Sq, P, Sk, lens, mode, p_cut, cut, True, 100)


# more ragged own caches than slots, which are taken in the order of their lengths
MANY = [
    (150, 4, 4, 1, 600, 150, [(37 * i) % 151 for i in range(150)], 128, 0),
    (256, 6, 3, 2, 0, 70, [70 if i % 3 else i % 70 for i in range(256)], 0, 0),  # many of one length
    (255, 3, 3, 1, 0, 140, [0] * 254 + [140], 0, 128),
    (99, 12, 3, 16, 200, 30, [30 - i % 31 for i in range(99)], 0, 0),  # two row blocks a cache, the prefix before them
]


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("shape", MANY, ids=[str(i) for i in range(len(MANY))])
def test_long_caches_first(shape, dt):
    B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut = shape
    run_and_check(dt, 64, B, Hq, Hkv, Sq, P, Sk, lens, EXACT, p_cut, cut, True, 700)


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ4, SQ8])
def test_modes_without_causal_mask(mode, dt):
    for shape in (SHAPES[2], SHAPES[5], SHAPES[6]):
        B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut = shape
        run_and_check(dt, 128, B, Hq, Hkv, Sq, P, Sk, lens, mode, p_cut, cut, False, 200)


@pytest.mark.parametrize("dt", [BF16, FP8])
def test_proposed_cuts(dt):
    code = pkg.ATTN_BF16 if dt == BF16 else pkg.ATTN_FP8_E4M3
    for B, Hq, Hkv, Sq, P, Sk in ((1, 8, 2, 1, 5000, 3000), (20, 8, 2, 2, 4100, 129)):
        cuts = pkg.attn_decode_prefix_split_keys(B, Hq, Hkv, Sq, P, Sk, 128, code)
        assert all(c % 128 == 0 for c in cuts)
        run_and_check(dt, 128, B, Hq, Hkv, Sq, P, Sk, None, EXACT, *cuts, True, 300)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ8])
def test_own_caches_alone_are_attn_decode(mode, d):
    # the same logits and weights bit for bit, sums in another order, off by at
    # most 80 roundings of 2^-24 (of max |v|, about 4: 2e-5): O may also round to
    # the neighbouring BF16 value (a step is 2^-7 of it at most)
    B, Hq, Hkv, Sq, Sk = 2, 8, 2, 3, 700
    q, _, _, k, v = make(BF16, d, B, Hq, Hkv, Sq, 0, Sk, 400)
    for cut in (0, 256):
        kw = dict(causal=True, scale=scale_of(d), exp_mode=mode, split_keys=cut)
        o, lse = pkg.attn_decode_prefix(q, None, None, k, v, prefix_split_keys=0, **kw)
        o2, lse2 = pkg.attn_decode(q, k, v, **kw)
        torch.cuda.synchronize()
        assert bool(((o.float() - o2.float()).abs() <= 2.0 ** -7 * o2.float().abs() + 2e-5).all())
        assert bool(((lse - lse2).abs() <= 5e-6 * (1 + lse2.abs())).all())


@pytest.mark.parametrize("dt", [BF16, FP8])
@pytest.mark.parametrize("d", [64, 128])
def test_nothing_outside_is_read_or_written(d, dt):
    # cache rows from lens[b] on, prefix rows from P on and everything around the
    # outputs hold NaN; outputs and workspace are written nowhere else
    for B, Hq, Hkv, Sq, P, Sk, lens, p_cut, cut in (SHAPES[1], SHAPES[4], SHAPES[5], SHAPES[8]):
        q, kp, vp, k, v = make(dt, d, B, Hq, Hkv, Sq, P, Sk, 500, cap=Sk + 37, P_cap=P + 19)
        kw = dict(causal=True, scale=scale_of(d), exp_mode=H15, prefix_split_keys=p_cut, split_keys=cut, Sk=Sk,
                  descale=DESCALE if dt == FP8 else None)
        t = torch.tensor(lens, dtype=torch.int32, device="cuda")
        clean = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=t, P=P if P else None, **kw)
        for x in (k, v):
            for b in range(B):
                x.view(torch.uint8)[b, :, lens[b]:] = 0x7F if dt == FP8 else 0xFF
        for x in (kp, vp) if P else ():
            x.view(torch.uint8)[:, P:] = 0x7F if dt == FP8 else 0xFF
        rows = B * Hq * Sq
        need = pkg.attn_decode_prefix_workspace_bytes(B, Hq, Sq, P, Sk, d, p_cut, cut)
        room = [torch.full((n + 512,), float("nan"), device="cuda") for n in (rows * d // 2, rows, need // 4)]
        out = room[0][256:-256].view(BF16).view(B, Hq, Sq, d)
        lse = room[1][256:-256].view(B, Hq, Sq)
        ws = room[2][256:-256] if need else None
        say(f"guards {dt} d={d} B={B} P={P}")
        pkg.attn_decode_prefix(q, kp, vp, k, v, lens=t, P=P if P else None, out=out, lse=lse, workspace=ws, **kw)
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), clean[0].view(torch.int16)) and torch.equal(lse, clean[1])
        for r in room:
            assert bool(r[:256].isnan().all()) and bool(r[-256:].isnan().all())


def test_lens_out_of_range_count_as_the_nearest():
    q, kp, vp, k, v = make(BF16, 128, 3, 4, 2, 1, 100, 200, 600)
    kw = dict(causal=True, scale=scale_of(128), exp_mode=EXACT, prefix_split_keys=0, split_keys=128, Sk=150)
    wild = torch.tensor([-5, 2 ** 31 - 1, 77], dtype=torch.int32, device="cuda")
    tame = torch.tensor([0, 150, 77], dtype=torch.int32, device="cuda")
    a = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=wild, **kw)
    b = pkg.attn_decode_prefix(q, kp, vp, k, v, lens=tame, **kw)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_extreme_logits():
    # logits of +-2e5 in base two, and equal ones: the weights stay finite
    for P, rows in ((300, 4), (300, 50)):
        q, kp, vp, k, v = make(BF16, 128, rows, 1, 1, 1, P, 130, 700)
        q = q * 300
        kp[0, 5] *= 300
        o, lse = pkg.attn_decode_prefix(q, kp, vp, k, v, causal=True, scale=1.0, exp_mode=EXACT, prefix_split_keys=128,
                                        split_keys=0)
        ref = prefix_ref(q, kp, vp, k, v, [130] * rows, True, 1.0, None, EXACT, 128, 0)
        assert bool(torch.isfinite(o).all())
        check_prefix(o, lse, ref, f"extreme logits, {rows} rows")
        k[:] = k[:, :, :1]
        kp[:] = kp[:, :1]
        o, lse = pkg.attn_decode_prefix(q, kp, vp, k, v, causal=True, scale=1.0, exp_mode=EXACT, prefix_split_keys=128,
                                        split_keys=0)
        check_prefix(o, lse, prefix_ref(q, kp, vp, k, v, [130] * rows, True, 1.0, None, EXACT, 128, 0),
                     f"equal keys, {rows} rows")


def test_caches_beyond_4_gib():
    # five heads of 1 GiB: offsets pass 32 bits; K is V
    cap = 1 << 23
    k = torch.empty((5, 1, cap, 128), dtype=FP8, device="cuda")
    for b in range(5):
        k[b, 0, :300] = randn((300, 128), 800 + b, FP8)
    q = randn((5, 2, 1, 128), 810, FP8)
    lens = [300, 7, 0, 129, 250]
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    kw = dict(causal=True, scale=scale_of(128), descale=DESCALE)
    o, lse = pkg.attn_decode_prefix(q, None, None, k, k, lens=t, Sk=384, exp_mode=EXACT, prefix_split_keys=0, split_keys=128, **kw)
    small = k[:, :, :384].contiguous()
    o2, lse2 = pkg.attn_decode_prefix(q, None, None, small, small, lens=t, exp_mode=EXACT, prefix_split_keys=0,
                                      split_keys=128, **kw)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    check_prefix(o, lse, prefix_ref(q, None, None, small, small, lens, True, scale_of(128), DESCALE, EXACT, 0, 128),
                 "beyond 4 GiB")


def test_side_stream_and_graph_with_growing_caches():
    # captured once, replayed as the caches grow: lens is read on the device
    q, kp, vp, k, v = make(BF16, 128, 12, 8, 2, 1, 500, 300, 900)
    lens = torch.tensor([3] * 12, dtype=torch.int32, device="cuda")
    kw = dict(causal=True, scale=scale_of(128), exp_mode=H15, prefix_split_keys=256, split_keys=128, lens=lens)
    need = pkg.attn_decode_prefix_workspace_bytes(12, 8, 1, 500, 300, 128, 256, 128)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((12, 8, 1), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    pkg.attn_decode_prefix(q, kp, vp, k, v, stream=side, out=out, lse=lse, **kw)  # a workspace of its own
    torch.cuda.current_stream().wait_stream(side)
    eager = pkg.attn_decode_prefix(q, kp, vp, k, v, **kw)
    assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.attn_decode_prefix(q, kp, vp, k, v, out=out, lse=lse, workspace=ws, **kw)
    for n in (3, 128, 0, 300):
        lens.fill_(n)
        lens[5] = 17
        out.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        eager = pkg.attn_decode_prefix(q, kp, vp, k, v, **kw)
        assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1]), n

"""Attention over a cache of 8-bit blocks (attn_decode_blocks) against the
definition in float64."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from qkv_helpers import (BF16, E8M0, EXACT, FP8, H15, SQ4, SQ8, block_cache, blocks_ref, check_prefix, normal, numbers, say,
                         scale_of)

pytestmark = pytest.mark.gpu


def decode(q, cache, block, lens, mode=EXACT, cut=0, causal=True, **kw):
    k, v, scales = cache
    lt = None if lens is None else torch.tensor(lens, dtype=torch.int32, device="cuda")
    return pkg.attn_decode_blocks(q, k, v, scales, block=block, lens=lt, causal=causal, scale=scale_of(q.shape[-1]),
                                  exp_mode=mode, split_keys=cut, **kw)


def run_and_check(B, Hq, Hkv, Sq, cap, d, block, lens, what, mode=EXACT, cut=0, causal=True, seed=1, sharp=True, Sk=None):
    q, cache = normal((B, Hq, Sq, d), seed), block_cache(B, Hkv, cap, d, block, seed + 1, sharp)
    o, lse = decode(q, cache, block, lens, mode, cut, causal, Sk=Sk)
    top = cap if Sk is None else Sk
    n = [top] * B if lens is None else [min(max(x, 0), top) for x in lens]
    check_prefix(o, lse, blocks_ref(q, *cache, block, n, causal, scale_of(d), mode, cut), what)
    return q, cache, o, lse


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ4, SQ8])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_single_tokens(d, mode, block):
    # lengths around a block's, a unit's, a tile's and a round's ends, empty ones and ones out of range
    lens = [0, 1, 15, 64, 65, 127, 128, 129, 256, 257, -3, 400, 333]
    run_and_check(len(lens), 4, 2, 1, 333, d, block, lens, f"{lens}", mode)


@pytest.mark.parametrize("mode", [EXACT, H15, SQ8])
@pytest.mark.parametrize("cut", [128, 256, 512])
def test_parts(mode, cut):
    run_and_check(4, 6, 3, 1, 1500, 128, 64, [1500, 0, 129, 777], f"cut {cut}", mode, cut)
    run_and_check(2, 6, 3, 5, 1500, 64, 16, [3, 1025], f"cut {cut}, 5 positions", mode, cut)


def test_more_than_32_parts():
    run_and_check(1, 2, 1, 1, 128 * 41 + 3, 64, 32, [128 * 41 + 3], "42 parts", EXACT, 128)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ4])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows(d, mode, causal):
    # blocks of 32 rows, of 128, a last one in part, blocks over several heads' positions, more positions than keys
    for i, (Hq, Hkv, Sq, lens, cut) in enumerate([(4, 2, 9, [300, 5], 0), (8, 1, 16, [200, 77], 128), (4, 2, 65, [300, 40], 0),
                                                  (3, 1, 200, [390, 200], 0), (2, 2, 300, [300, 0], 128), (5, 1, 40, [399, 1], 256)]):
        run_and_check(2, Hq, Hkv, Sq, 400, d, [16, 32, 64, 128][i % 4], lens, f"case {i}", mode, cut, causal, 10 + i)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_hundreds_of_rows(d, block, causal):
    # a block of rows over several heads' positions, rows without a key, lengths around a step's and a tile's ends
    for i, (B, Hq, Hkv, Sq, cap, lens, cut) in enumerate([(1, 4, 2, 150, 333, [333], 0), (2, 3, 1, 301, 700, [700, 97], 256),
                                                          (3, 8, 1, 65, 200, [128, 65, 129], 128)]):
        run_and_check(B, Hq, Hkv, Sq, cap, d, block, lens, f"case {i}", EXACT, cut, causal, 20 + i)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_thousands_of_keys_and_rows(d, causal):
    # the form of 512 rows (many caches with room for thousands of keys, mostly empty): lengths around a step's and a
    # tile's ends; blocks of rows over two heads' positions and a last one in part; and a cache in two parts
    lens = [0] * 128
    for b, n in ((0, 1), (1, 63), (5, 64), (6, 65), (17, 127), (18, 128), (40, 129), (41, 1500), (127, 777)):
        lens[b] = n
    run_and_check(128, 2, 1, 450, 8192, d, 16, lens, "two heads of 450 positions", EXACT, 0, causal, 40, sharp=False)
    lens = [8300, 700, 8192, 8193] + [0] * 60
    run_and_check(64, 2, 1, 450, 16384, d, 128, lens, "parts", EXACT, 8192, causal, 41, sharp=False)


def test_anchors_of_many_rows():
    # logits that grow along the keys, so that the running maximum moves far and often; and a tiny scale
    q, (k, v, scales) = normal((1, 2, 600, 64), 30), block_cache(1, 1, 175104, 64, 16, 31)
    n = 900
    scales.view(torch.uint8)[0, 0, :57, 0] = (110 + torch.arange(57, device="cuda") // 3).to(torch.uint8)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for Sk, cut in ((n, 0), (n, 256), (175104, 2176)):  # 128 rows a workgroup, and 512
        for scale in (scale_of(64), 8.0, 1e-38):
            o, lse = pkg.attn_decode_blocks(q, k, v, scales, block=16, causal=True, scale=scale, exp_mode=EXACT, split_keys=cut,
                                            lens=lens, Sk=Sk)
            check_prefix(o, lse, blocks_ref(q, k, v, scales, 16, [n], True, scale, EXACT, cut), f"Sk {Sk} cut {cut} scale {scale}")


@pytest.mark.parametrize("Sk,cut", [(900, 0), (175104, 2176)])  # 128 rows a workgroup, and 512
def test_large_values_under_growing_logits(Sk, cut):
    # logits (base two) that rise by 38 from the first keys to the last, and values of 2^92: neither a row's sums nor what
    # it holds before its maximum moves may overflow
    n, d = 900, 64
    q, (k, v, scales) = normal((1, 2, 600, d), 50), block_cache(1, 1, Sk, d, 64, 51)
    q[..., 0] = 1.0
    k.view(torch.uint8)[0, 0, :n] = 0
    k[0, 0, :n, 0] = (torch.arange(n, device="cuda") / 24).to(FP8)
    scales.view(torch.uint8)[..., 0], scales.view(torch.uint8)[..., 1] = 127, 127 + 90
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    o, lse = pkg.attn_decode_blocks(q, k, v, scales, block=64, causal=True, scale=math.log(2.0), exp_mode=EXACT, split_keys=cut,
                                    lens=lens)
    check_prefix(o, lse, blocks_ref(q, k, v, scales, 64, [n], True, math.log(2.0), EXACT, cut), f"Sk {Sk}")


def test_no_lens_and_Sk():
    run_and_check(2, 4, 4, 1, 200, 64, 64, None, "no lens")
    run_and_check(2, 4, 4, 3, 200, 64, 64, None, "Sk", Sk=130)
    run_and_check(2, 4, 4, 3, 200, 64, 64, [150, 20], "lens beyond Sk", Sk=130)


@pytest.mark.parametrize("rows", [1, 150])
@pytest.mark.parametrize("mode", [EXACT, H15])
def test_what_lies_behind_is_not_read(rows, mode):
    # codes of NaN from lens on, and scales of 255 in the blocks there, in caches that end inside a block and at its end
    B, Hq, Hkv, d, block, cap, lens = 4, 2, 2, 128, 16, 320, [37, 128, 0, 300]
    q, (k, v, scales) = normal((B, Hq, rows, d), 1), block_cache(B, Hkv, cap, d, block, 2)
    cuts = (0, 128)
    clean = [decode(q, (k, v, scales), block, lens, mode, cut) for cut in cuts]
    for b, n in enumerate(lens):
        k.view(torch.uint8)[b, :, n:], v.view(torch.uint8)[b, :, n:] = 0x7F, 0xFF
        scales.view(torch.uint8)[b, :, -(-n // block):] = 255
    for cut, want in zip(cuts, clean):
        got = decode(q, (k, v, scales), block, lens, mode, cut)
        assert bool(torch.isfinite(got[0].float()).all()) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_scale_bytes():
    # scales from 2^-126 to large ones; 0 counts as 1, 255 as 254
    B, d, block, cap = 6, 64, 32, 64
    q, (k, v, scales) = normal((B, 2, 1, d), 3), block_cache(B, 1, cap, d, block, 4)
    sb = scales.view(torch.uint8)
    sb[:, 0, :, 0] = torch.tensor([[1, 0], [100, 120], [127, 127], [130, 110], [117, 127], [0, 1]], dtype=torch.uint8)
    sb[:, 0, :, 1] = torch.tensor([[127, 100], [1, 127], [200, 180], [20, 10], [240, 230], [127, 127]], dtype=torch.uint8)
    o, lse = decode(q, (k, v, scales), block, None)
    # values below 2^-126 count as 0 in the kernel: add what they could give
    ref = list(blocks_ref(q, k, v, scales, block, [cap] * B, True, scale_of(d), EXACT, 0))
    ref[2] = ref[2] + 2.0 ** -126
    check_prefix(o, lse, ref, "scales")


def test_nan_stays_in_its_sequence_and_head():
    q, (k, v, scales) = normal((3, 4, 2, 64), 5), block_cache(3, 2, 200, 64, 64, 6)
    clean = decode(q, (k, v, scales), 64, [200, 150, 100])
    k.view(torch.uint8)[1, 0, 20, 3], v.view(torch.uint8)[1, 1, 30, 5] = 0x7F, 0x7F
    got = decode(q, (k, v, scales), 64, [200, 150, 100])
    for b in (0, 2):
        assert torch.equal(got[0][b], clean[0][b]) and torch.equal(got[1][b], clean[1][b])
    assert bool(got[0][1, :2].isnan().any()) and bool(got[0][1, 2:, :, 5].isnan().all())


def test_large_logits():
    # logits of thousands: the running maximum keeps the sums finite
    q, (k, v, scales) = normal((2, 4, 3, 128), 7) * 40, block_cache(2, 2, 700, 128, 32, 8, True)
    for cut in (0, 256):
        o, lse = decode(q, (k, v, scales), 32, [700, 399], EXACT, cut)
        check_prefix(o, lse, blocks_ref(q, k, v, scales, 32, [700, 399], True, scale_of(128), EXACT, cut), f"cut {cut}")


def test_many_ragged_caches():
    # more workgroups than slots: the longest first; more than 256 sequences: their own order
    for B, Hkv in ((70, 8), (300, 2)):
        lens = [(37 * b) % 200 for b in range(B)]
        run_and_check(B, Hkv, Hkv, 1, 200, 64, 64, lens, f"{B} caches", sharp=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ4, SQ8])
def test_caches_with_room_for_many_keys(d, mode):
    # (the form for more keys than the caches hold goes by the room)
    run_and_check(3, 4, 2, 2, 131072 * 128 // d * 2 // 3, d, 32, [700, 0, 1025], f"{mode}", mode, 256, sharp=False)


def test_equals_decode_of_the_same_numbers():
    # with one scale for all, the BF16 decode of the numbers that the codes stand for, up to the order of sums
    q, (k, v, scales) = normal((2, 8, 4, 128), 9), block_cache(2, 2, 600, 128, 64, 10)
    wide = [numbers(x, scales, 64, i).to(BF16) for i, x in enumerate((k, v))]
    for mode in (EXACT, H15):
        o, lse = decode(q, (k, v, scales), 64, None, mode, 256)
        o2, lse2 = pkg.attn_decode(q, *wide, causal=True, scale=scale_of(128), exp_mode=mode, split_keys=256)
        # each side's P and O are off by 2^-8; a weight at a border may be another lattice point
        assert bool(((o - o2).abs() <= 2.0 ** -6 * o2.abs() + 2.0 ** -5).all()) and bool(((lse - lse2).abs() <= 2e-3).all())


def test_long_cache():
    # offsets beyond 2^31 bytes, the last heads of it against a few keys
    B, Hkv, cap, d, block = 3, 8, 1 << 20, 128, 128
    n = [5000, 1, cap - 2048]
    k, v = (torch.zeros((B, Hkv, cap, d), dtype=torch.uint8, device="cuda").view(FP8) for _ in range(2))
    small = block_cache(B, Hkv, 2048, d, block, 11)
    # the last 2048 slots that are filled differ from zero: keys of zero have the logit 0
    scales = torch.full((B, Hkv, cap // block, 2), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    at = cap - 4096
    for x, y in ((k, small[0]), (v, small[1])):
        x[2, :, at:at + 2048] = y[2]
    scales.view(torch.uint8)[2, :, at // block:at // block + 2048 // block] = small[2].view(torch.uint8)[2]
    q = normal((B, Hkv, 1, d), 12)
    cut = pkg.attn_decode_blocks_split_keys(B, Hkv, Hkv, 1, cap, d)
    o, lse = decode(q, (k, v, scales), block, n, EXACT, cut)
    assert bool((o[:2] == 0).all())
    for b in (0, 1):
        # log of a sum of ones, in FP32
        assert bool(((lse[b].double() - math.log(n[b])).abs() <= 2.0 ** -20 * 16).all())
    kk, vv = (numbers(small[i][2:], small[2][2:], block, i) for i in range(2))
    s = q[2].double() @ kk[0].transpose(-1, -2).contiguous() * scale_of(d)
    rest = cap - 2048 - 2048
    total = s.exp().sum(-1) + rest
    want = (s.exp() @ vv[0]) / total.unsqueeze(-1)
    # P rounds to 2^-8 of each weight, O to 2^-8; FP32 sums over a million keys in parts: 2^-24 of 8192 terms a chain
    size = (s.exp() @ vv[0].abs()) / total.unsqueeze(-1)
    assert bool(((o[2].double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -7 * size).all())
    assert bool(((lse[2].double() - total.log()).abs() <= 2.0 ** -11).all())


def test_streams_and_graph():
    q, cache = normal((3, 8, 1, 128), 13), block_cache(3, 2, 1000, 128, 64, 14)
    lens = torch.tensor([1000, 20, 513], dtype=torch.int32, device="cuda")
    call = lambda **kw: pkg.attn_decode_blocks(q, *cache, block=64, lens=lens, causal=True, scale=0.1, exp_mode=H15,  # noqa: E731
                                               split_keys=256, **kw)
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert call(want_lse=False)[1] is None
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    ws = torch.full((pkg.attn_decode_blocks_workspace_bytes(3, 8, 1, 1000, 128, 256),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out=out, lse=lse, workspace=ws)
    for step in range(3):
        lens -= 9
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), step
    say("replayed")


@pytest.mark.parametrize("causal", [True, False])
def test_more_groups_of_512_rows_than_slots(causal):
    # ragged caches, mostly empty, two blocks of rows each: the longest first, equal lengths in their own order
    lens = [0] * 256
    for b, n in ((0, 1), (1, 64), (2, 700), (3, 700), (100, 65), (128, 1100), (200, 64), (254, 513), (255, 2)):
        lens[b] = n
    run_and_check(256, 2, 1, 512, 8192, 64, 16, lens, "512 rows, longest first", EXACT, 0, causal, 60, sharp=False)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mode", [EXACT, H15, SQ8])
@pytest.mark.parametrize("cut", [0, 256])
def test_more_groups_of_128_rows_than_slots(d, mode, cut):
    # (150 positions of two heads: three blocks of rows, the second over both heads)
    lens = [0] * 100
    for b, n in ((0, 3), (7, 400), (8, 400), (33, 128), (64, 257), (98, 129), (99, 390)):
        lens[b] = n
    for causal in (True, False):
        run_and_check(100, 4, 2, 150, 400, d, 32, lens, f"128 rows, longest first, cut {cut}", mode, cut, causal, 61, sharp=False)



@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
def test_many_rows_with_the_finest_lattice(d, causal):
    for i, (Hq, Hkv, Sq, lens, cut) in enumerate([(4, 2, 9, [300, 5], 0), (4, 2, 65, [300, 40], 0), (3, 1, 200, [390, 200], 0),
                                                  (2, 2, 300, [300, 0], 128), (5, 1, 40, [399, 1], 256)]):
        run_and_check(2, Hq, Hkv, Sq, 400, d, [16, 32, 64, 128][i % 4], lens, f"case {i}", SQ8, cut, causal, 70 + i)


@pytest.mark.parametrize("form,mode", [("keys, streaming", EXACT), ("keys, streaming", H15), ("512 rows", EXACT), ("512 rows, parts", EXACT)])
def test_what_lies_behind_is_not_read_by_the_forms_of_long_caches(form, mode):
    # NaN in every code from lens on and scales of 255 in every block there; lengths inside a block, at its end, at a step's
    # and a tile's
    if form == "keys, streaming":
        B, Hq, Hkv, Sq, cap, d, cut = 4, 4, 2, 2, 65536, 128, 256
        lens = [700, 0, 1025, 512]
    elif form == "512 rows":
        B, Hq, Hkv, Sq, cap, d, cut = 128, 2, 1, 450, 8192, 64, 0
        lens = [0] * 128
        lens[0], lens[3], lens[4], lens[70], lens[127] = 1, 100, 128, 577, 1024
    else:
        B, Hq, Hkv, Sq, cap, d, cut = 1, 2, 1, 600, 175104, 64, 2176
        lens = [2176 + 2045]
    block = 16
    q, (k, v, scales) = normal((B, Hq, Sq, d), 80), block_cache(B, Hkv, cap, d, block, 81)
    want = [decode(q, (k, v, scales), block, lens, mode, cut, causal) for causal in (True, False)]
    for b, n in enumerate(lens):
        k.view(torch.uint8)[b, :, n:], v.view(torch.uint8)[b, :, n:] = 0x7F, 0xFF
        scales.view(torch.uint8)[b, :, -(-n // block):] = 255
    for causal, (o, lse) in zip((True, False), want):
        got = decode(q, (k, v, scales), block, lens, mode, cut, causal)
        assert bool(torch.isfinite(got[0].float()).all()) and torch.equal(got[0], o) and torch.equal(got[1], lse)


@pytest.mark.parametrize("mode", [EXACT, H15])
@pytest.mark.parametrize("B,Hq,Hkv,Sq,cap,cut", [(20, 8, 2, 1, 3000, 0), (3, 8, 2, 1, 3000, 256), (4, 8, 2, 40, 1500, 256), (1, 32, 8, 512, 16384, 2048)])
def test_repeats_itself(B, Hq, Hkv, Sq, cap, cut, mode):
    # no order of workgroups, waves or parts shows in what comes out
    q, cache = normal((B, Hq, Sq, 128), 90), block_cache(B, Hkv, cap, 128, 64, 91, True)
    lens = [cap - 37 * b for b in range(B)]
    want = decode(q, cache, 64, lens, mode, cut)
    for _ in range(5):
        torch.empty_like(want[0]).fill_(1)  # (other work in between)
        got = decode(q, cache, 64, lens, mode, cut)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

"""Writing into a cache of 8-bit blocks (attn_cache_append): codes, scales and
lengths equal the definition's, bit for bit."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from qkv_helpers import BF16, E8M0, FP8, append_ref, block_cache, normal, say

pytestmark = pytest.mark.gpu


def new_rows(B, Hkv, n, d, seed):
    """Rows of sizes that differ by powers of two, so that scales grow and stay."""
    size = torch.exp2(torch.randint(-6, 7, (B, Hkv, n, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).float())
    return [(normal((B, Hkv, n, d), seed + 1 + i, torch.float32) * size).to(BF16) for i in range(2)]


def same_numbers(got, want):
    return torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0))


def append_and_check(k, v, cache, lens, counts, block, what, **kw):
    kc, vc, scales = cache
    cap, i32 = kc.shape[2], torch.int32
    before = [kc.float(), vc.float()]
    bytes_before = scales.view(torch.uint8).clone()
    lt = torch.tensor(lens, dtype=i32, device="cuda")
    ct = None if counts is None else torch.tensor(counts, dtype=i32, device="cuda")
    after = pkg.attn_cache_append(k, v, kc, vc, scales, lt, block=block, counts=ct, **kw)
    for i, (x, codes) in enumerate(((k, kc), (v, vc))):
        out, sc, end = append_ref(x, before[i], bytes_before[..., i], lens, counts, cap, block)
        assert torch.equal(scales.view(torch.uint8)[..., i].int(), sc), f"{what}: scales of {'kv'[i]}"
        assert same_numbers(codes.float().double(), out), f"{what}: codes of {'kv'[i]}"
    assert after.tolist() == end, what
    return end


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_appends_in_turn(d, block):
    # single tokens, a few, whole blocks and chunks, through block borders, over what the cache held before
    B, Hkv, cap = 3, 2, 7 * block + 5
    cache = block_cache(B, Hkv, cap, d, block, 1)
    lens = [0, 3, block - 1]
    for step, n in enumerate([1, 1, 5, block, 1, 2 * block + 3, 1, 7]):
        say(f"step {step}: {n} rows at {lens}")
        lens = append_and_check(*new_rows(B, Hkv, n, d, 100 * step), cache, lens, None, block, f"step {step}")


def test_counts_lengths_and_limits():
    B, Hkv, d, block, cap, n = 8, 1, 64, 32, 100, 40
    cache = block_cache(B, Hkv, cap, d, block, 2)
    lens = [-5, 0, 31, 32, 90, 100, 101, 64]
    counts = [40, 0, 41, -1, 40, 7, 3, 1]
    assert append_and_check(*new_rows(B, Hkv, n, d, 3), cache, lens, counts, block, "limits") == [40, 0, 71, 32, 100, 100, 100, 65]


def test_in_place_lengths():
    k, v = new_rows(2, 2, 3, 64, 4)
    kc, vc, scales = block_cache(2, 2, 64, 64, 16, 5)
    lens = torch.tensor([5, 15], dtype=torch.int32, device="cuda")
    got = pkg.attn_cache_append(k, v, kc, vc, scales, lens, block=16, lens_out=lens)
    assert got is lens and lens.tolist() == [8, 18]


def test_scale_borders():
    # the largest values around 448 * 2^j, the least and the greatest of BF16, zeros
    tops = [448.0, 450.0, 446.0, 224.0, 225.0, 0.0, 2.0 ** -133, 2.0 ** -126, 448 * 2.0 ** -126, 3.3895313892515355e38, 1.0, 1.75]
    B = len(tops)
    k = torch.zeros(B, 1, 2, 64, device="cuda")
    for b, t in enumerate(tops):
        k[b, 0, 0, 17], k[b, 0, 1, 3] = -t, t / 3
    k = k.to(BF16)
    append_and_check(k, -k, block_cache(B, 1, 16, 64, 16, 6), [0] * B, None, 16, "borders")


def test_scales_that_grow_far():
    # codes of a block that must shrink by 1 to 2^40: halved codes stay exact, small ones round, then nothing is left
    kc, vc, scales = cache = block_cache(6, 1, 16, 64, 16, 7)
    scales.view(torch.uint8)[:] = torch.tensor([127, 126, 125, 117, 110, 87], dtype=torch.uint8, device="cuda")[:, None, None, None]
    k = torch.full((6, 1, 1, 64), 300.0, dtype=BF16, device="cuda")
    append_and_check(k, k, cache, [9] * 6, None, 16, "grow")
    # a scale that is larger than needed stays, also 255 (254) and 0 (1)
    scales.view(torch.uint8)[:] = torch.tensor([200, 127, 254, 255, 0, 1], dtype=torch.uint8, device="cuda")[:, None, None, None]
    append_and_check(k, k, cache, [9] * 6, None, 16, "keep")


def test_infinities_and_nan():
    k, v = new_rows(1, 2, 20, 128, 8)
    k[0, 0, 3, 5], k[0, 0, 4, 7], k[0, 1, 15, 0], k[0, 1, 16] = math.inf, -math.inf, math.nan, math.nan
    v[0, 0, 19] = math.inf
    cache = block_cache(1, 2, 32, 128, 16, 9)
    cache[0].view(torch.uint8)[0, 0, 1, 1] = 0x7F  # a NaN among the codes that are there
    append_and_check(k, v, cache, [2], None, 16, "infinities")


def test_nothing_else_is_written():
    # scales and codes of blocks without a new row, and codes behind the last one, keep their bits, NaN patterns included
    kc = torch.full((2, 2, 80, 64), 0xFF, dtype=torch.uint8, device="cuda")
    vc, scales = kc.clone(), torch.full((2, 2, 5, 2), 0xFF, dtype=torch.uint8, device="cuda")
    k, v = new_rows(2, 2, 20, 64, 10)
    pkg.attn_cache_append(k, v, kc.view(FP8), vc.view(FP8), scales.view(E8M0), torch.tensor([16, 48], dtype=torch.int32, device="cuda"),
                          block=16, counts=torch.tensor([20, 0], dtype=torch.int32, device="cuda"))
    for c in (kc, vc):
        assert bool((c[0, :, :16] == 0xFF).all()) and bool((c[0, :, 36:] == 0xFF).all()) and bool((c[1] == 0xFF).all())
        assert not bool((c[0, :, 16:36] == 0xFF).all(-1).any())
    assert bool((scales[0, :, [0, 3, 4]] == 0xFF).all()) and bool((scales[1] == 0xFF).all()) and not bool((scales[0, :, 1:3] == 0xFF).any())


def test_large_caches():
    # offsets beyond 2^31 bytes: the last heads of a large cache
    B, Hkv, cap, d = 9, 8, 1 << 18, 128
    kc, vc = (torch.zeros((B, Hkv, cap, d), dtype=torch.uint8, device="cuda").view(FP8) for _ in range(2))
    scales = torch.full((B, Hkv, cap // 128, 2), 127, dtype=torch.uint8, device="cuda").view(E8M0)
    k, v = new_rows(B, Hkv, 3, d, 11)
    lens = torch.full((B,), cap - 2, dtype=torch.int32, device="cuda")
    after = pkg.attn_cache_append(k, v, kc, vc, scales, lens, block=128)
    assert after.tolist() == [cap] * B
    for i, (x, c) in enumerate(((k, kc), (v, vc))):
        out, sc, _ = append_ref(x[:, :, :2], torch.zeros(B, Hkv, 128, d, device="cuda"),
                                torch.full((B, Hkv, 1), 127, device="cuda"), [126] * B, None, 128, 128)
        assert torch.equal(c[:, :, -128:].float().double(), out)
        assert torch.equal(scales.view(torch.uint8)[:, :, -1, i].int(), sc[..., 0])
        assert not bool(c.view(torch.uint8)[:, :, :-128].any())


def test_captured():
    kc, vc, scales = block_cache(2, 2, 64, 64, 16, 12)
    kc2, vc2, scales2 = kc.clone(), vc.clone(), scales.clone()
    k, v = new_rows(2, 2, 1, 64, 13)
    lens = torch.tensor([3, 14], dtype=torch.int32, device="cuda")
    eager = lens.clone()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        pkg.attn_cache_append(k, v, kc, vc, scales, lens, block=16, lens_out=lens)
    for step in range(20):
        k.mul_(1.3), v.mul_(1.1)
        graph.replay()
        torch.cuda.synchronize()
        eager = pkg.attn_cache_append(k, v, kc2, vc2, scales2, eager, block=16)
        assert lens.tolist() == eager.tolist() == [4 + step, 15 + step]
        assert torch.equal(kc.view(torch.uint8), kc2.view(torch.uint8)) and torch.equal(vc.view(torch.uint8), vc2.view(torch.uint8))
        assert torch.equal(scales.view(torch.uint8), scales2.view(torch.uint8))

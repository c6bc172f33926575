"""Eviction (attn_evict): the indexes that stay against a sort on the CPU, and
their rows bit for bit."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import BF16, FP8, evict_ref, randn, say

pytestmark = pytest.mark.gpu


def check(k, v, acc, lens, keep, recent, Sk=None, out_cap=None, what=""):
    B, Hkv, cap, d = k.shape
    out_cap = out_cap or keep
    fill = lambda *s: torch.full((*s, d * k.element_size()), 0x55, dtype=torch.uint8, device="cuda").view(k.dtype)  # noqa: E731
    k_out, v_out = fill(B, Hkv, out_cap), fill(B, Hkv, out_cap)
    acc_out = torch.full((B, Hkv, out_cap), -7.0, device="cuda")
    t = torch.tensor(lens, dtype=torch.int32, device="cuda") if lens is not None else None
    got = pkg.attn_evict(k, v, acc, lens=t, keep=keep, recent=recent, Sk=Sk, k_out=k_out, v_out=v_out, acc_out=acc_out)
    torch.cuda.synchronize()
    assert got[0] is k_out and got[1] is v_out and got[2] is acc_out
    n = lens if lens is not None else [Sk or cap] * B
    assert got[4].tolist() == [min(x, keep) for x in n]
    for i, want in enumerate(evict_ref(acc, n, keep, recent)):
        b, h, r = i // Hkv, i % Hkv, len(want)
        assert got[3][b, h].tolist() == want.tolist() + [-1] * (keep - r), (what, b, h)
        at = torch.from_numpy(want).cuda()
        for x, y in ((k, k_out), (v, v_out)):
            assert torch.equal(y[b, h, :r].view(torch.uint8), x[b, h][at].view(torch.uint8))
            assert bool((y[b, h, r:].view(torch.uint8) == 0x55).all())
        assert torch.equal(acc_out[b, h, :r].view(torch.int32), acc[b, h][at].view(torch.int32))
        assert bool((acc_out[b, h, r:] == -7.0).all())


def caches(dt, B, Hkv, cap, d, seed):
    k, v = randn((B, Hkv, cap, d), seed, BF16), randn((B, Hkv, cap, d), seed + 1, BF16)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return k.to(dt), v.to(dt), torch.randn((B, Hkv, cap), generator=gen, device="cuda").exp()


@pytest.mark.parametrize("dt,d", [(BF16, 128), (FP8, 128), (BF16, 64), (FP8, 64)])
@pytest.mark.parametrize("n,keep,recent", [(1, 1, 0), (2, 1, 0), (2, 1, 1), (5, 9, 2), (64, 63, 0), (65, 1, 0), (300, 100, 20),
                                           (1024, 1000, 999), (1025, 7, 7), (1025, 7, 50), (5000, 4096, 256),
                                           (20011, 777, 10)])
def test_sizes(n, keep, recent, dt, d):
    k, v, acc = caches(dt, 1, 2, n, d, 10)
    say(f"evict n={n} keep={keep} recent={recent} {dt} d={d}")
    check(k, v, acc, None, keep, recent)


@pytest.mark.parametrize("n,keep,recent", [(32768, 2048, 64), (32769, 32768, 0), (33024, 100, 0), (40000, 20000, 500),
                                           (100003, 5, 1), (70001, 69000, 68999)])
def test_caches_beyond_what_lds_holds(n, keep, recent):
    k, v, acc = caches(FP8, 2, 1, n, 64, 60)
    say(f"evict n={n} keep={keep} recent={recent}")
    check(k, v, acc, None, keep, recent)
    check(k, v, torch.floor(acc), [n, n - 200], keep, recent)  # many equal ones


def test_many_caches_beyond_what_lds_holds():
    k, v, acc = caches(FP8, 35, 2, 33024, 64, 70)  # one workgroup for each
    lens = [33024 - 700 * (b % 7) for b in range(35)]
    check(k, v, acc, lens, 500, 17)
    check(k, v, torch.floor(acc), lens, 33000, 0)


def test_more_heads_than_compute_units():
    k, v, acc = caches(BF16, 75, 4, 500, 64, 80)
    for keep in (90, 400):  # rows copied by the selecting workgroup, and by others
        check(k, v, torch.floor(acc), [500 - 6 * b for b in range(75)], keep, 30)


# (lens, keep, recent) for caches of 30000 keys that eight workgroups share
PARTS = [([30000, 29999, 4096], 1000, 100), ([4097, 4095, 12289], 4096, 0), ([0, 1, 30000], 1, 0), ([20000, 8192, 8193], 8192, 9000),
         ([30000, 20481, 50], 20480, 20479), ([30000, 24577, 12288], 12288, 1)]


@pytest.mark.parametrize("dt,d", [(BF16, 64), (FP8, 128)])
@pytest.mark.parametrize("lens,keep,recent", PARTS)
def test_parts_of_ragged_caches(lens, keep, recent, dt, d):
    k, v, acc = caches(dt, 3, 2, 30100, d, 90)
    for a in (acc, torch.floor(acc), torch.full_like(acc, 0.5), acc.sort(dim=-1)[0], acc.sort(dim=-1, descending=True)[0]):
        say(f"evict parts lens={lens} keep={keep} recent={recent} {dt}")
        check(k, v, a, lens, keep, recent, Sk=30000, out_cap=keep + 3)


def test_parts_with_signs_infinities_and_nan():
    k, v, acc = caches(FP8, 1, 1, 25000, 64, 95)
    a = 1.0 - acc
    a[..., ::3], a[..., 1::50] = math.inf, -math.inf
    a[..., 7::110] = math.nan
    a.view(torch.int32)[..., 9::1100] = -1  # NaN with its sign set
    a[..., 4::9], a[..., 5::9] = 0.0, -0.0
    for keep in (1, 250, 251, 8000, 12000, 24999):
        check(k, v, a, None, keep, 0)
    close = (1.0 + torch.arange(25000, device="cuda").float().flip(0) % 97 * 2.0 ** -23).view(1, 1, -1)
    check(k, v, close, None, 5000, 3)


def test_parts_stay_within_their_workspace_and_replay():
    k, v, acc = caches(BF16, 2, 1, 22000, 64, 97)
    need = pkg.attn_evict_workspace_bytes(2, 1, 22000)
    space = torch.full((need + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    lens = torch.tensor([22000, 21000], dtype=torch.int32, device="cuda")
    out = pkg.attn_evict(k, v, acc, lens=lens, keep=700, recent=50, workspace=space[2048:2048 + need])
    torch.cuda.synchronize()
    assert bool((space[:2048] == 0x5A).all()) and bool((space[2048 + need:] == 0x5A).all())
    kw = dict(zip(("k_out", "v_out", "acc_out", "index", "lens_out"), out))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.attn_evict(k, v, acc, lens=lens, keep=700, recent=50, **kw)
    for n in (22000, 500, 0, 16385):
        lens.fill_(n)
        acc.copy_(torch.rand_like(acc))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for i, want in enumerate(evict_ref(acc, [n] * 2, 700, 50)):
            assert out[3][i, 0].tolist() == want.tolist() + [-1] * (700 - len(want))


def test_ragged_batch_with_room_to_spare():
    k, v, acc = caches(BF16, 6, 3, 700, 128, 20)
    for keep, recent, cap in ((128, 16, 200), (300, 0, 300), (690, 690, 1000)):
        check(k, v, acc, [650, 0, 1, min(keep, 650), min(keep + 1, 650), 649], keep, recent, Sk=650, out_cap=cap)


def test_equal_weights_signs_infinities_and_nan():
    k, v, acc = caches(BF16, 1, 1, 3000, 64, 30)
    for kind in ("equal", "steps", "zeros", "inf", "nan", "negative", "close", "subnormal"):
        a = acc.clone()
        if kind == "equal":
            a.fill_(0.25)
        elif kind == "steps":
            a = torch.floor(a)
        elif kind == "zeros":
            a[..., ::2], a[..., 1::2] = 0.0, -0.0
        elif kind == "inf":
            a[..., ::3], a[..., 1::5] = math.inf, -math.inf
        elif kind == "nan":
            a[..., 7::11] = math.nan
            a[..., 8::11] = math.inf
            a.view(torch.int32)[..., 9::11] = -1  # NaN with its sign set
        elif kind == "negative":
            a = 1.0 - a
        elif kind == "close":  # weights that differ in their lowest bits only
            a = (1.0 + torch.arange(3000, device="cuda").float().flip(0) % 97 * 2.0 ** -23).view(1, 1, -1)
        else:
            a = a * 1e-41
        say(f"evict {kind}")
        for keep, recent in ((1, 0), (100, 0), (1500, 3), (2999, 0)):
            check(k, v, a, None, keep, recent, what=kind)


def test_lens_out_of_range_count_as_the_nearest():
    k, v, acc = caches(BF16, 2, 1, 400, 128, 40)
    wild = torch.tensor([-3, 2 ** 30], dtype=torch.int32, device="cuda")
    index, lens = pkg.attn_evict(k, v, acc, lens=wild, keep=50, recent=5, Sk=300)[3:]
    assert lens.tolist() == [0, 50] and bool((index[0] == -1).all())
    assert index[1, 0].tolist() == evict_ref(acc[1:], [300], 50, 5)[0].tolist()


def test_caches_beyond_4_gib_and_graph():
    cap = 1 << 23
    k = torch.empty((5, 1, cap, 128), dtype=FP8, device="cuda")
    k[:, :, :300] = randn((5, 1, 300, 128), 50, FP8)
    acc = torch.rand((5, 1, cap), device="cuda")
    lens = torch.tensor([300, 7, 0, 129, 250], dtype=torch.int32, device="cuda")
    small, small_acc = k[:, :, :300].contiguous(), acc[:, :, :300].contiguous()
    a = pkg.attn_evict(k, k, acc, lens=lens, keep=100, recent=10, Sk=300)
    b = pkg.attn_evict(small, small, small_acc, lens=lens, keep=100, recent=10)
    for x, y, i in zip(a[0].view(torch.uint8), b[0].view(torch.uint8), lens.tolist()):
        assert torch.equal(x[:, :min(i, 100)], y[:, :min(i, 100)])
    assert torch.equal(a[3], b[3]) and torch.equal(a[4], b[4])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pkg.attn_evict(small, small, small_acc, lens=lens, keep=100, recent=10, k_out=b[0], v_out=b[1], acc_out=b[2],
                       index=b[3], lens_out=b[4])
    for n in (300, 50, 0, 101):
        lens.fill_(n)
        small_acc.copy_(torch.rand_like(small_acc))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert b[4].tolist() == [min(n, 100)] * 5
        for i, want in enumerate(evict_ref(small_acc, [n] * 5, 100, 10)):
            assert b[3][i, 0, :len(want)].tolist() == want.tolist()

"""The C ABI and the binding of the operators over shared and bounded caches
without a GPU: exported names, and refusals before anything is launched."""
import ctypes
import math
import re
from pathlib import Path

import pytest
import torch

import paper_2609_33586_amd as pkg
from paper_2609_33586_amd import cache

HEADER = Path(__file__).resolve().parent.parent / "include" / "h15cache.h"
FAKE = 0x100000  # 16-byte aligned, never dereferenced
INV, UNS = pkg.ATTN_EINVAL, pkg.ATTN_EUNSUPPORTED


@pytest.fixture(scope="module")
def L():
    return cache._lib()


def test_exports_every_declared_symbol(L):
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(attn_\w+)\s*\(", text, flags=re.M))
    assert names == set(cache.EXPORTS)
    for n in names:
        assert hasattr(L, n) and callable(getattr(pkg, n))


def opts(qd=1.0, kd=1.0, vd=1.0, tau=0.0):
    return ctypes.byref(pkg.attn_opts(qd, kd, vd, None, tau, 0))


def prefix(L, q=FAKE, kp=FAKE, vp=FAKE, k=FAKE, v=FAKE, lens=FAKE, o=FAKE, lse=FAKE, B=2, Hq=4, Hkv=2, Sq=1, P=500,
           P_cap=512, Sk=300, cap=320, d=128, causal=1, scale=0.1, dtype=0, mode=1, p_cut=0, cut=0, ws=FAKE,
           wsb=1 << 40, o_=None):
    return L.attn_decode_prefix(q, kp, vp, k, v, lens, o, lse, B, Hq, Hkv, Sq, P, P_cap, Sk, cap, d, causal, scale,
                                dtype, mode, p_cut, cut, ws, wsb, o_)


def test_prefix_refusals(L):
    for name in ("q", "kp", "vp", "k", "v", "o"):
        assert prefix(L, **{name: None}) == INV, name
        assert prefix(L, **{name: FAKE + 8}) == UNS, name
    for kw in ({"B": 0}, {"Hq": 0}, {"Hkv": 0}, {"Hkv": 3}, {"Sq": 0}, {"P": -1}, {"Sk": -1}, {"d": 0}, {"P": 513},
               {"Sk": 321}, {"P": 0, "Sk": 0}, {"p_cut": 100}, {"cut": -128}, {"cut": 64}, {"ws": None}, {"ws": FAKE + 8},
               {"scale": 0.0}, {"scale": math.nan}, {"scale": math.inf}, {"dtype": 1}, {"o_": opts(tau=-1.0)}):
        assert prefix(L, **kw) == INV, kw
    for kw in ({"d": 96}, {"dtype": 2}, {"mode": pkg.ATTN_EXP_ROWMAX_POT}, {"mode": 7}, {"lens": FAKE + 2},
               {"lse": FAKE + 1}, {"o_": opts(tau=8.0)}, {"B": 1 << 15, "Hq": 1 << 14, "Sq": 4}, {"P_cap": 1 << 24},
               {"cap": 1 << 24}, {"B": 1 << 12, "Hq": 1 << 13, "Hkv": 1 << 13}, {"B": 1 << 13, "Hq": 1 << 13, "Hkv": 1}):
        assert prefix(L, **kw) == UNS, kw
    for bad in ((0.0, 1.0, 1.0), (1.0, math.inf, 1.0), (1.0, 1.0, -1.0)):
        assert prefix(L, dtype=1, o_=opts(*bad)) == INV
    need = pkg.attn_decode_prefix_workspace_bytes(2, 4, 1, 500, 300, 128, 128, 256)
    assert need == 2 * 4 * (4 + 2) * (128 + 2) * 4
    assert prefix(L, p_cut=128, cut=256, wsb=need - 1) == INV


def test_prefix_sizes(L):
    ws = pkg.attn_decode_prefix_workspace_bytes
    assert ws(2, 4, 1, 500, 0, 128, 0, 0) == ws(2, 4, 1, 0, 500, 128, 0, 512) == 0  # one part
    assert ws(2, 4, 1, 500, 300, 64, 0, 0) == 2 * 4 * 2 * 66 * 4
    assert ws(0, 4, 1, 500, 300, 64, 0, 0) == ws(1, 4, 1, -1, 300, 64, 0, 0) == ws(1, 4, 1, 5, 300, 64, -1, 0) == 0
    for args in ((1, 32, 8, 1, 32768, 4096), (64, 32, 8, 1, 32768, 2048), (7, 24, 8, 4, 5003, 777), (1, 1, 1, 1, 1, 0),
                 (64, 64, 1, 16, 0, 65536)):
        a, b = pkg.attn_decode_prefix_split_keys(*args, 128, 0)
        assert a >= 0 and b >= 0 and a % 128 == 0 and b % 128 == 0
    cuts = pkg.attn_decode_prefix_split_keys
    assert cuts(16, 32, 8, 1, 0, 8192, 128, 0) == (0, 2048) and cuts(16, 32, 8, 1, 300, 8192, 128, 0) == (0, 4096)
    # next to a prefix in parts: own caches in as many parts as workgroups are left of 512, of two tiles or more
    assert cuts(7, 24, 8, 4, 5003, 777, 128, 1) == (512, 384) and cuts(24, 32, 8, 1, 8192, 1024, 128, 1) == (768, 0)
    assert cuts(64, 32, 8, 1, 32768, 2048, 128, 0) == (2048, 0) and cuts(1, 8, 1, 4096, 8192, 512, 128, 0)[1] == 0
    assert pkg.attn_decode_prefix_split_keys(0, 32, 8, 1, 100, 100, 128, 0) == (0, 0)
    assert pkg.attn_decode_prefix_split_keys(1, 32, 7, 1, 100000, 100000, 128, 0) == (0, 0)
    assert L.attn_decode_prefix_split_keys(1, 32, 8, 1, 100, 100, 128, 0, None, None) == INV


def weights(L, q=FAKE, k=FAKE, lse=FAKE, lens=FAKE, acc=FAKE, B=2, Hq=4, Hkv=2, Sq=1, Sk=300, cap=320, d=128, causal=1,
            scale=0.1, decay=1.0, dtype=0, ws=None, wsb=0, o_=None):
    return L.attn_key_weights(q, k, lse, lens, acc, B, Hq, Hkv, Sq, Sk, cap, d, causal, scale, decay, dtype, ws, wsb, o_)


def test_weights_refusals(L):
    for name in ("q", "k", "lse", "acc"):
        assert weights(L, **{name: None}) == INV, name
    for name, off in (("q", 8), ("k", 8), ("lse", 2), ("acc", 2), ("lens", 2)):
        assert weights(L, **{name: FAKE + off}) == UNS, name
    for kw in ({"B": 0}, {"Hq": 0}, {"Hkv": 0}, {"Hkv": 3}, {"Sq": 0}, {"Sk": 0}, {"Sk": 321}, {"d": 0}, {"scale": -1.0},
               {"decay": -0.5}, {"decay": math.nan}, {"decay": math.inf}, {"dtype": 1}, {"Sq": 4096}):
        assert weights(L, **kw) == INV, kw  # (Sq 4096: a workspace is wanted)
    for kw in ({"d": 96}, {"dtype": 2}, {"o_": opts(tau=1.0)}, {"cap": 1 << 24}, {"Sq": 1 << 23},
               {"B": 1 << 12, "Hq": 1 << 12, "Hkv": 1 << 12}):
        assert weights(L, **kw) == UNS, kw
    need = pkg.attn_key_weights_workspace_bytes(2, 4, 2, 4096, 300, 128)
    assert need > 0 and need % (2 * 2 * 300 * 4) == 0
    assert weights(L, Sq=4096, ws=FAKE, wsb=need - 1) == INV and weights(L, Sq=4096, ws=FAKE + 4, wsb=need) == INV
    assert pkg.attn_key_weights_workspace_bytes(2, 4, 2, 1, 300, 128) == 0
    assert pkg.attn_key_weights_workspace_bytes(2, 4, 3, 4096, 300, 128) == 0


def spread(n):
    """Addresses 64 TiB apart: none overlaps another."""
    return [0x100000 + (i << 46) for i in range(n)]


def evict(L, at=None, lens=None, B=2, Hkv=2, Sk=300, cap=320, out_cap=128, d=128, keep=100, recent=10, dtype=0,
          ws=None, wsb=0):
    k, v, acc, ko, vo, ao, ix, lo = at or spread(8)
    return L.attn_evict(k, v, acc, lens, ko, vo, ao, ix, lo, B, Hkv, Sk, cap, out_cap, d, keep, recent, dtype, ws, wsb,
                        None)


def test_evict_refusals(L):
    for i in range(8):
        at = spread(8)
        at[i] = None
        assert evict(L, at) == INV, i
        at = spread(8)
        at[i] += 8 if i in (0, 1, 3, 4) else 2
        assert evict(L, at) == UNS, i
    for kw in ({"B": 0}, {"Hkv": 0}, {"Sk": 0}, {"Sk": 321}, {"out_cap": 99}, {"keep": 0}, {"recent": -1}, {"d": 0}):
        assert evict(L, **kw) == INV, kw
    for kw in ({"d": 96}, {"dtype": 2}, {"lens": FAKE + 2}, {"B": 1 << 14, "Hkv": 1 << 14, "keep": 200, "out_cap": 200},
               {"B": 1 << 11, "Hkv": 1 << 11, "keep": 1, "recent": 0}):
        assert evict(L, **kw) == UNS, kw
    for i in range(3, 8):  # an output on an input or on another output, from its first or up to its last byte
        for j in range(8):
            if i != j:
                at = spread(8)
                at[i] = at[j]
                assert evict(L, at) == INV, (i, j)
    at = spread(8)
    at[3] = at[0] + 2 * 2 * 320 * 256 - 16
    assert evict(L, at) == INV
    at = spread(8)
    assert evict(L, at, lens=at[7]) == INV  # new lens over the old ones
    big = (1 << 31) - 1
    assert evict(L, Sk=big, cap=big, ws=FAKE, wsb=1 << 60) == UNS
    assert evict(L, Sk=big, cap=big, keep=big, out_cap=big) == UNS


def test_evict_workspace(L):
    need = pkg.attn_evict_workspace_bytes(2, 2, 40000)
    assert need > 0 and need % 16 == 0 and pkg.attn_evict_workspace_bytes(2, 2, 300) == 0
    assert pkg.attn_evict_workspace_bytes(0, 2, 40000) == pkg.attn_evict_workspace_bytes(2, 2, 0) == 0
    at = spread(9)
    for ws, wsb in ((None, need), (at[8], need - 1), (at[8] + 8, need)):
        assert evict(L, at[:8], Sk=40000, cap=40000, ws=ws, wsb=wsb) == INV
    for i in range(8):
        assert evict(L, at[:8], Sk=40000, cap=40000, ws=at[i], wsb=need) == INV, i
    assert evict(L, at[:8], lens=at[8] + need - 4, Sk=40000, cap=40000, ws=at[8], wsb=need) == INV


def test_binding_refuses_host_tensors():
    q, kp = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16), torch.zeros(2, 5, 64, dtype=torch.bfloat16)
    k, f = torch.zeros(1, 2, 5, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 5)
    with pytest.raises(ValueError, match="current GPU"):
        pkg.attn_decode_prefix(q, kp, kp, k, k, causal=True, scale=0.1, exp_mode=0, prefix_split_keys=0, split_keys=0)
    for kv in ((kp, None, k, k), (None, kp, k, k), (kp, kp, k, None), (kp, kp, None, k)):
        with pytest.raises(ValueError, match="both or neither"):
            pkg.attn_decode_prefix(q, *kv, causal=True, scale=0.1, exp_mode=0, prefix_split_keys=0, split_keys=0)
    with pytest.raises(ValueError, match="current GPU"):
        pkg.attn_key_weights(q, k, f[..., :1], f, causal=True, scale=0.1)
    with pytest.raises(ValueError, match="current GPU"):
        pkg.attn_evict(k, k, f, keep=2, recent=1)


def test_binding_checks_shapes_and_types(L):
    good = torch.zeros(2, 3, 4)  # (device -1: the host)
    assert cache._tensor("x", good, (2, 3, 4), -1, torch.float32) is good
    for bad in (torch.zeros(2, 3, 5), torch.zeros(2, 3), torch.zeros(2, 4, 3).transpose(1, 2),
                torch.zeros(2, 3, 4, dtype=torch.int32)):
        with pytest.raises(ValueError, match=r"x must be a contiguous tensor \[2x3x4\] of torch.float32"):
            cache._tensor("x", bad, (2, 3, 4), -1, torch.float32)
    with pytest.raises(ValueError, match="GPU 0"):
        cache._tensor("x", good, (2, 3, 4), 0)
    k = torch.zeros(2, dtype=torch.uint8)
    assert cache._operand("k", k, (2,), -1, torch.float8_e4m3fn, pkg.ATTN_FP8_E4M3) is k  # e4m3 codes as bytes
    with pytest.raises(TypeError, match="k and the first operand"):
        cache._operand("k", k, (2,), -1, torch.bfloat16, pkg.ATTN_BF16)
    with pytest.raises(ValueError, match="4-D"):
        cache._four("k", k)
    c = torch.zeros(2, 3, 5, 64, dtype=torch.uint8)
    assert cache._cache("k", c, 2, 64, -1, torch.float8_e4m3fn, pkg.ATTN_FP8_E4M3) == (3, 5)
    for bad in (c[:1], c[..., :32].contiguous(), c[0], c.unsqueeze(0), c.transpose(1, 2), c[0, 0, 0], c[0, 0]):
        with pytest.raises(ValueError, match="k must be a contiguous tensor"):
            cache._cache("k", bad, 2, 64, -1, torch.uint8, pkg.ATTN_FP8_E4M3)
    with pytest.raises(ValueError, match="GPU 0"):
        cache._cache("k", c, 2, 64, 0, torch.uint8, pkg.ATTN_FP8_E4M3)
    with pytest.raises(TypeError, match="k and the first operand"):
        cache._cache("k", c, 2, 64, -1, torch.bfloat16, pkg.ATTN_BF16)
    assert cache._lens_ptr(None, 2, -1) is None
    for bad in (torch.zeros(2, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)):
        with pytest.raises(ValueError, match="lens"):
            cache._lens_ptr(bad, 2, -1)
    with pytest.raises(ValueError, match="workspace"):
        cache._space(torch.zeros(4, 4).t(), lambda: 8, -1, None)
    assert cache._space(None, lambda: 0, -1, None) == (None, 0, None)

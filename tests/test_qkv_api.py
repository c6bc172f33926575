"""The C ABI and the binding of the operators between projections and attention
without a GPU: exported names, refusals before anything is launched, frequencies."""
import ctypes
import math
import re
from pathlib import Path

import pytest
import torch

import paper_2609_33586_amd as pkg
from paper_2609_33586_amd import qkv

HEADER = Path(__file__).resolve().parent.parent / "include" / "h15qkv.h"
INV, UNS = pkg.ATTN_EINVAL, pkg.ATTN_EUNSUPPORTED


def at(i):
    """Addresses 64 TiB apart, 16-byte aligned, never dereferenced: none overlaps another."""
    return 0x100000 + (i << 46)


@pytest.fixture(scope="module")
def L():
    return qkv._lib()


def opts(qd=1.0, kd=1.0, vd=1.0, tau=0.0):
    return ctypes.byref(pkg.attn_opts(qd, kd, vd, None, tau, 0))


def test_exports_every_declared_symbol(L):
    text = re.sub(r"/\*.*?\*/", "", HEADER.read_text(), flags=re.S)
    names = set(re.findall(r"^\s*(?:int|size_t)\s+(attn_\w+)\s*\(", text, flags=re.M))
    assert names == set(qkv.EXPORTS)
    for n in names:
        assert hasattr(L, n) and callable(getattr(pkg, n))


SPEC = dict(positions=at(10), each=0, freqs=at(11), rot=64, inter=0, amplitude=1.0, qw=at(12), kw=at(13), wt=0, eps=1e-6)


def spec(**kw):
    return ctypes.cast(ctypes.pointer(qkv.attn_rope_spec(*{**SPEC, **kw}.values())), ctypes.c_void_p)


def strides(*nine):
    return None if not nine else ctypes.cast((ctypes.c_int64 * 9)(*nine), ctypes.c_void_p)


def rope(L, q=at(0), k=at(1), v=at(2), st=None, qo=at(3), ko=at(4), vo=at(5), B=2, S=30, Hq=4, Hkv=2, d=128, dtype=0, o_=None, **s):
    return L.attn_rope(q, k, v, st, spec(**s), qo, ko, vo, B, S, Hq, Hkv, d, dtype, o_)


def backward(L, gq=at(0), gk=at(1), gv=at(2), q=at(3), k=at(4), st=None, dq=at(5), dk=at(6), dv=at(7), gst=None, wq=at(8),
             wk=at(9), B=2, S=30, Hq=4, Hkv=2, d=128, ws=at(14), wsb=1 << 40, **s):
    return L.attn_rope_bwd(gq, gk, gv, q, k, st, spec(**s), dq, dk, dv, gst, wq, wk, B, S, Hq, Hkv, d, ws, wsb, None)


BAD_SPEC_INV = ({"rot": -16}, {"rot": 144}, {"freqs": None}, {"amplitude": 0.0}, {"amplitude": math.nan}, {"amplitude": math.inf},
                {"eps": 0.0}, {"eps": -1.0}, {"eps": math.nan}, {"eps": math.inf}, {"eps": 2.0 ** -127})
BAD_SPEC_UNS = ({"rot": 8}, {"rot": 126}, {"wt": 1}, {"wt": 3}, {"positions": at(10) + 2}, {"freqs": at(11) + 4}, {"qw": at(12) + 8},
                {"kw": at(13) + 8})
BAD_SIZES_INV = ({"B": 0}, {"S": 0}, {"d": 0}, {"Hq": 0}, {"Hkv": 0}, {"Hq": -1})
BAD_SIZES_UNS = ({"d": 96}, {"d": 256}, {"B": 1 << 16, "S": 1 << 15}, {"B": 1 << 14, "S": 1 << 14, "Hq": 8}, {"Hq": 1 << 20, "Hkv": 1 << 20},
                 {"B": 1 << 15, "S": 1 << 15, "Hq": 1, "Hkv": 1}, {"B": 1, "S": 32 * (2 ** 24 - 1) + 1, "Hq": 1, "Hkv": 1},
                 {"B": 1, "S": 1, "Hq": 65534, "Hkv": 1})


def test_rope_refusals(L):
    for kw in BAD_SPEC_INV + BAD_SIZES_INV:
        assert rope(L, **kw) == INV, kw
    for kw in BAD_SPEC_UNS + BAD_SIZES_UNS + ({"dtype": 2},):
        assert rope(L, **kw) == UNS, kw
    assert L.attn_rope(at(0), at(1), at(2), None, None, at(3), at(4), at(5), 2, 30, 4, 2, 128, 0, None) == INV
    names = ("q", "k", "v", "qo", "ko", "vo")
    for i, name in enumerate(names):
        assert rope(L, **{name: None}) == INV, name  # an input without its output, or the reverse
        assert rope(L, **{name: at(i) + 8}) == UNS, name
    assert rope(L, **dict.fromkeys(names)) == INV
    assert rope(L, q=None, qo=None, Hkv=0) == INV
    # FP8 takes descales
    assert rope(L, dtype=1) == INV
    for bad in ((0.0, 1.0, 1.0), (1.0, math.inf, 1.0), (1.0, 1.0, -1.0), (1e-45, 1.0, 1.0)):
        assert rope(L, dtype=1, o_=opts(*bad)) == INV, bad
    # strides: multiples of 8, not negative
    good = (30 * 512, 512, 128) + (30 * 256, 256, 128) * 2
    for i in range(9):
        for bad in (-8, 4, 1 << 60):
            assert rope(L, st=strides(*good[:i], bad, *good[i + 1:])) == UNS, (i, bad)
    # an output on an input or on another output, from its first or up to its last byte
    inputs = {"q": 2 * 30 * 4 * 256, "k": 2 * 30 * 2 * 256, "v": 2 * 30 * 2 * 256}
    for out in ("qo", "ko", "vo"):
        for i, name in enumerate(names):
            if name != out:
                assert rope(L, **{out: at(i)}) == INV, (out, name)
                if name in inputs:
                    assert rope(L, **{out: at(i) + inputs[name] - 16}) == INV, (out, name)
        for i in range(10, 14):
            assert rope(L, **{out: at(i)}) == INV, (out, i)
    # the last stride that sizes allow, and the next (in elements; an output beyond 2^63 bytes is an address of no one)
    assert rope(L, q=at(0), B=1, S=3, st=strides(0, (2 ** 59 - 1) // 3 // 8 * 8 + 8, 128, *good[3:])) == UNS
    # a projection's batches further apart than 2^29 elements are taken: this call is refused for its output alone
    assert rope(L, qo=at(0) + 2 * (1 << 33), st=strides(1 << 33, 512, 128, *good[3:])) == INV
    assert rope(L, qo=at(0) + 2 * 100, st=strides(1 << 20, 512, 128, *good[3:])) == UNS
    assert rope(L, qo=at(0) + 2 * (1 << 20), st=strides(1 << 20, 512, 128, *good[3:])) == INV


def test_rope_bwd_refusals(L):
    for kw in BAD_SPEC_INV + BAD_SIZES_INV:
        assert backward(L, **kw) == INV, kw
    for kw in BAD_SPEC_UNS + BAD_SIZES_UNS:
        assert backward(L, **kw) == UNS, kw
    for i, name in enumerate(("gq", "gk", "gv", "q", "k", "dq", "dk", "dv", "wq", "wk")):
        assert backward(L, **{name: None}) == INV, name
        assert backward(L, **{name: at(i) + (2 if name in ("wq", "wk") else 8)}) == UNS, name
    assert backward(L, gq=None, gk=None, gv=None, dq=None, dk=None, dv=None) == INV
    need = pkg.attn_rope_bwd_workspace_bytes(2, 30, 4, 2, 128)
    assert need > 0 and need % 512 == 0
    for ws, wsb in ((None, need), (at(14) + 8, need), (at(14), need - 1)):
        assert backward(L, ws=ws, wsb=wsb) == INV
    good = (30 * 512, 512, 128) + (30 * 256, 256, 128) * 2
    for i in range(9):
        for bad in (-8, 4):
            assert backward(L, gst=strides(*good[:i], bad, *good[i + 1:])) == UNS, (i, bad)
            if i < 6:
                assert backward(L, st=strides(*good[:i], bad, *good[i + 1:])) == UNS, (i, bad)
    for out in ("dq", "dk", "dv", "wq", "wk", "ws"):  # outputs and the workspace on inputs, weights, or each other
        for i in (0, 1, 2, 3, 4, 10, 11, 12, 13):
            assert backward(L, **{out: at(i)}) == INV, (out, i)
    for out, other in (("dq", 8), ("dk", 9), ("dv", 14), ("wq", 9), ("wk", 14)):
        assert backward(L, **{out: at(other)}) == INV, (out, other)


def test_rope_bwd_workspace(L):
    ws = pkg.attn_rope_bwd_workspace_bytes
    for bad in ((0, 5, 4, 2, 128), (1, 0, 4, 2, 128), (1, 5, -1, 2, 128), (1, 5, 0, 0, 128), (1, 5, 4, 2, 96), (1 << 16, 1 << 15, 4, 2, 64)):
        assert ws(*bad) == 0, bad
    assert ws(64, 8192, 64, 8, 128) < 1 << 23 and ws(1, 1, 4, 2, 64) > 0


def append(L, k=at(0), v=at(1), kc=at(2), vc=at(3), sc=at(4), lens=at(5), counts=at(6), out=at(7), B=2, Hkv=2, n=5, cap=100, d=128,
           block=32):
    return L.attn_cache_append(k, v, kc, vc, sc, lens, counts, out, B, Hkv, n, cap, d, block, None)


def test_append_refusals(L):
    for i, name in enumerate(("k", "v", "kc", "vc", "sc", "lens", "counts", "out")):
        if name != "counts":
            assert append(L, **{name: None}) == INV, name
        if name != "sc":
            assert append(L, **{name: at(i) + (8 if i < 4 else 2)}) == UNS, name
    for kw in ({"B": 0}, {"Hkv": 0}, {"n": 0}, {"cap": 0}, {"d": 0}):
        assert append(L, **kw) == INV, kw
    for kw in ({"d": 96}, {"block": 0}, {"block": 8}, {"block": 48}, {"block": 256}, {"cap": 1 << 24}, {"n": 1 << 23},
               {"B": 1 << 12, "Hkv": 1 << 12}, {"B": 1 << 10, "Hkv": 1 << 10, "n": 300, "cap": 3000}):
        assert append(L, **kw) == UNS, kw
    for i, out in ((2, "kc"), (3, "vc"), (4, "sc"), (7, "out")):
        for j in range(8):
            if j != i and (out, j) != ("out", 5):  # (the new lengths may go over the old ones)
                assert append(L, **{out: at(j)}) == INV, (out, j)
    assert append(L, out=at(5) + 4) == INV  # not in part
    assert append(L, kc=at(0) + 2 * 2 * 5 * 256 - 16) == INV


def blocks(L, q=at(0), k=at(1), v=at(2), sc=at(3), lens=at(4), o=at(5), lse=at(6), B=2, Hq=4, Hkv=2, Sq=1, Sk=300, cap=320, d=128,
           block=64, causal=1, scale=0.1, mode=1, cut=0, ws=at(7), wsb=1 << 40, o_=None):
    return L.attn_decode_blocks(q, k, v, sc, lens, o, lse, B, Hq, Hkv, Sq, Sk, cap, d, block, causal, scale, mode, cut, ws, wsb, o_)


def test_blocks_refusals(L):
    for i, name in enumerate(("q", "k", "v", "sc", "lens", "o", "lse")):
        if name not in ("lens", "lse"):
            assert blocks(L, **{name: None}) == INV, name
        assert blocks(L, **{name: at(i) + (8 if name in "qkvo" else 2 if name != "sc" else 1)}) == UNS, name
    for kw in ({"B": 0}, {"Hq": 0}, {"Hkv": 0}, {"Hkv": 3}, {"Sq": 0}, {"Sk": 0}, {"Sk": -1}, {"Sk": 321}, {"d": 0}, {"cut": 100},
               {"cut": -128}, {"cut": 64}, {"scale": 0.0}, {"scale": math.nan}, {"scale": math.inf}, {"o_": opts(tau=-1.0)}):
        assert blocks(L, **kw) == INV, kw
    for kw in ({"d": 96}, {"block": 0}, {"block": 8}, {"block": 96}, {"block": 256}, {"mode": pkg.ATTN_EXP_ROWMAX_POT}, {"mode": 9},
               {"o_": opts(tau=8.0)}, {"cap": 1 << 24}, {"B": 1 << 15, "Hq": 1 << 14, "Sq": 4}, {"B": 1 << 12, "Hq": 1 << 13, "Hkv": 1 << 13},
               {"B": 1 << 13, "Hq": 1 << 13, "Hkv": 1, "cut": 128}, {"B": 1, "Hq": 2 ** 26 - 3, "Hkv": 1, "cut": 128},
               {"B": 1 << 12, "Hq": 1, "Hkv": 1, "Sq": 512, "Sk": 1 << 19, "cap": 1 << 19, "cut": 128, "mode": 0}):
        assert blocks(L, **kw) == UNS, kw
    need = pkg.attn_decode_blocks_workspace_bytes(2, 4, 1, 300, 128, 128)
    assert need == 2 * 4 * 3 * (128 + 2) * 4
    for ws, wsb in ((None, need), (at(7) + 8, need), (at(7), need - 1)):
        assert blocks(L, cut=128, ws=ws, wsb=wsb) == INV
    # an output or the workspace on an input or another output, from its first or up to its last byte
    sizes = (2 * 4 * 256, 2 * 2 * 320 * 128, 2 * 2 * 320 * 128, 2 * 2 * 5 * 2, 8, 2 * 4 * 256, 2 * 4 * 4, need)
    for out, i in (("o", 5), ("lse", 6), ("ws", 7)):
        for j in range(8):
            if j != i:
                assert blocks(L, cut=128, **{out: at(j)}) == INV, (out, j)
                assert blocks(L, cut=128, **{out: at(j) + (sizes[j] - 1) // 16 * 16}) == INV, (out, j)


def test_blocks_sizes(L):
    ws = pkg.attn_decode_blocks_workspace_bytes
    assert ws(2, 4, 1, 300, 128, 0) == ws(2, 4, 1, 300, 128, 384) == ws(0, 4, 1, 300, 128, 128) == ws(2, 4, 1, 300, 128, -1) == 0
    cut = pkg.attn_decode_blocks_split_keys
    for args in ((0, 32, 8, 1, 100), (1, 32, 7, 1, 100000), (1, 32, 8, 0, 100), (1, 32, 8, 1, 0), (64, 32, 8, 1, 8192)):
        assert cut(*args, 128) == 0, args
    for args in ((1, 32, 8, 1, 32768), (16, 32, 8, 1, 8192), (1, 8, 8, 300, 65536), (3, 24, 8, 4, 5003), (64, 32, 8, 1, 16384)):
        assert cut(*args, 128) > 0 and cut(*args, 128) % 128 == 0, args


def test_binding_refuses_host_tensors_and_nothing():
    x, c = torch.zeros(1, 5, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 5, 64, dtype=torch.uint8)
    n = torch.zeros(1, dtype=torch.int32)
    for call in (lambda: pkg.attn_rope(x), lambda: pkg.attn_rope_bwd(x), lambda: pkg.attn_cache_append(x, x, c, c, c, n, block=16),
                 lambda: pkg.attn_decode_blocks(x, c, c, c, block=16, causal=True, scale=0.1, exp_mode=0, split_keys=0)):
        with pytest.raises(ValueError, match="current GPU"):
            call()
    for call in (lambda: pkg.attn_rope(None), lambda: pkg.attn_rope_bwd(None)):
        with pytest.raises(ValueError, match="one at least"):
            call()


def test_binding_checks_of_tensors(L):
    x = torch.zeros(2, 5, 3, 64, dtype=torch.bfloat16)  # (device -1: the host)
    assert qkv._strided("x", x, 2, 5, 64, -1) == (3, 5 * 3 * 64, 3 * 64, 64)
    assert qkv._strided("x", x[:1, :1, :1], 1, 1, 64, -1) == (1, 0, 0, 0)
    for bad in (x.float(), x[0], x[:, :4], x[..., :32], x[:1]):
        with pytest.raises(ValueError, match="x must be"):
            qkv._strided("x", bad, 2, 5, 64, -1)
    with pytest.raises(ValueError, match="rows of x"):
        qkv._strided("x", torch.zeros(2, 5, 64, 64, dtype=torch.bfloat16).transpose(2, 3), 2, 5, 64, -1)
    def apart(y):
        n, *st = qkv._strided("x", y, *y.shape[:2], 64, -1)
        return qkv._apart("x", *y.shape[:2], n, 64, *st)

    for good in (x, x[:, ::2], x.transpose(1, 2), x.transpose(0, 1), x.transpose(0, 2)[:, ::2], x[:1].expand(1, 5, 3, 64),
                 x.as_strided((2, 5, 1, 64), (960, 64, 0, 1))):
        apart(good)
    for bad in (x[:1].expand(2, 5, 3, 64), x.as_strided((2, 5, 3, 64), (960, 64, 64, 1)),
                x.as_strided((2, 5, 3, 64), (320, 64, 320, 1)), x.as_strided((2, 5, 3, 64), (960, 192, 56, 1))):
        with pytest.raises(ValueError, match="overlap"):
            apart(bad)
    f, w = torch.zeros(16, dtype=torch.float64), torch.zeros(64)
    good = dict(freqs=f, positions=None, interleaved=False, amplitude=1.0, q_weight=w, k_weight=None, eps=1e-6)
    s = qkv.attn_rope_spec.from_buffer_copy(qkv._spec(2, 5, 64, -1, **good))  # (packed as the C struct lies)
    assert abs(s.eps - 1e-6) < 1e-12 and s.amplitude == 1.0 and s.freqs == f.data_ptr() and s.q_weight == w.data_ptr()
    assert s.rot == 32 and s.weight_dtype == pkg.ATTN_FP32 and s.k_weight is None
    s = qkv.attn_rope_spec.from_buffer_copy(qkv._spec(2, 5, 64, -1, **{**good, "positions": torch.zeros(2, 5, dtype=torch.int32), "q_weight": w.bfloat16()}))
    assert s.each_position == 1 and s.weight_dtype == pkg.ATTN_BF16
    for kw in ({"freqs": f.float()}, {"positions": torch.zeros(2, 5)}, {"positions": torch.zeros(5, dtype=torch.int32)},
               {"positions": torch.zeros(2, 4, dtype=torch.int32)}, {"q_weight": w[:32]}):
        with pytest.raises(ValueError):
            qkv._spec(2, 5, 64, -1, **{**good, **kw})
    for kw in ({"q_weight": w.half()}, {"k_weight": w.bfloat16()}):
        with pytest.raises(TypeError):
            qkv._spec(2, 5, 64, -1, **{**good, **kw})
    side = type("Stream", (), {"cuda_stream": 0x1234500000})
    for o, want in ((qkv._opts(side), (1.0, 1.0, 1.0)), (qkv._opts(side, (0.5, 2, 4.0)), (0.5, 2.0, 4.0))):
        o = pkg.attn_opts.from_buffer_copy(o)
        assert (o.q_descale, o.k_descale, o.v_descale) == want and o.stream == 0x1234500000
        assert o.rescale_threshold == 0.0 and o.rescale_per_wave == 0
    c, sc = torch.zeros(1, 2, 70, 64, dtype=torch.uint8), torch.zeros(1, 2, 3, 2, dtype=torch.uint8)
    assert qkv._codes("k", c, 1, 2, 64, -1) == 70 and qkv._scales(sc, 1, 2, 70, 32, -1) == sc.data_ptr()
    for bad in (c[0], c.to(torch.bfloat16)):
        with pytest.raises(TypeError):
            qkv._codes("k", bad, 1, 2, 64, -1)
    for bad in (c[..., :32].contiguous(), c[:, :1]):
        with pytest.raises(ValueError):
            qkv._codes("k", bad, 1, 2, 64, -1)
    with pytest.raises(TypeError):
        qkv._scales(sc.float(), 1, 2, 70, 32, -1)
    for block in (16, 64, 0, -32, 2 ** 32 + 32):
        with pytest.raises(ValueError):
            qkv._scales(sc, 1, 2, 70, block, -1)


def test_frequencies():
    f, a = pkg.attn_rope_frequencies(128)
    j = torch.arange(64, dtype=torch.float64)
    plain = torch.exp(-j / 64 * math.log(10000.0))
    assert f.dtype == torch.float64 and a == 1.0 and torch.allclose(f, plain, rtol=1e-14)
    f, a = pkg.attn_rope_frequencies(128, scaling="linear", factor=8.0)
    assert torch.allclose(f, plain / 8, rtol=1e-14) and a == 1.0
    f, _ = pkg.attn_rope_frequencies(128, scaling="base", factor=8.0)
    assert f[0] == 1.0 and abs(f[-1] / (plain[-1] / 8) - 1) < 1e-12
    # the fast pairs are kept, the slow ones interpolated, and those between lie between, in order
    for kw in (dict(scaling="ramp", factor=8.0, original=4096), dict(scaling="smooth", factor=8.0, original=4096, fast=4.0)):
        f, a = pkg.attn_rope_frequencies(128, **kw)
        turns = 4096 * plain / (2 * math.pi)
        assert a == (0.1 * math.log(8.0) + 1.0 if kw["scaling"] == "ramp" else 1.0)
        # (a ramp's ends are rounded outwards to whole pairs)
        kept = pkg.attn_rope_frequencies(128)[0]
        assert torch.equal(f[turns > 40], kept[turns > 40]) and torch.allclose(f[turns < 0.8], plain[turns < 0.8] / 8, rtol=1e-14)
        assert bool((f <= plain * (1 + 1e-15)).all()) and bool((f >= plain / 8 * (1 - 1e-15)).all()) and bool((f.diff() < 0).all())
    f, _ = pkg.attn_rope_frequencies(64, 500000.0, scaling="smooth", factor=4.0, original=8192, fast=4.0)
    p = torch.pow(500000.0, -2.0 * torch.arange(32, dtype=torch.float64) / 64)
    turns = 8192 * p / (2 * math.pi)
    mid = (turns > 1) & (turns < 4)
    keep = (turns - 1) / 3
    assert bool(mid.any()) and torch.allclose(f[mid], (p * keep + p / 4 * (1 - keep))[mid], rtol=1e-13)
    for bad in (dict(rot=3), dict(rot=0), dict(rot=64, base=0.0), dict(rot=64, scaling="other"), dict(rot=64, scaling="linear", factor=0.5),
                dict(rot=64, scaling="ramp", factor=2.0),
                dict(rot=64, base=1.0, scaling="ramp", factor=2.0, original=100), dict(rot=64, scaling="smooth", factor=2.0, original=100, slow=4.0, fast=1.0),
                dict(rot=2, scaling="base", factor=2.0)):
        with pytest.raises(ValueError):
            pkg.attn_rope_frequencies(bad.pop("rot"), bad.pop("base", 10000.0), **bad)

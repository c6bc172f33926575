"""Norms and position rotation (attn_rope) against the formula in float64."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from qkv_helpers import BF16, FP8, bf16_tolerance, check, large_rows, normal, projection, rope_ref, say

pytestmark = pytest.mark.gpu


def freqs_of(rot, base=10000.0, **kw):
    return pkg.attn_rope_frequencies(rot, base, device="cuda", **kw)


def run_and_check(q, k, v, what, *, freqs=None, positions=None, inter=False, amplitude=1.0, wq=None, wk=None, eps=1e-6, **kw):
    got = pkg.attn_rope(q, k, v, freqs=freqs, positions=positions, interleaved=inter, amplitude=amplitude, q_weight=wq,
                        k_weight=wk, eps=eps, **kw)
    for name, x, w, y in (("q", q, wq, got[0]), ("k", k, wk, got[1]), ("v", v, None, got[2])):
        if x is None:
            assert y is None
        elif name == "v":
            assert y.is_contiguous() and torch.equal(y, x.transpose(1, 2))
        else:
            z, tol = rope_ref(x, w, freqs, positions, inter, amplitude, eps)
            check(y, z, bf16_tolerance(z, tol), f"{what} {name}")
    return got


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_layouts_parts_and_sizes(d, inter, norm):
    # (every part of the head, positions of both forms, sizes around a workgroup's positions)
    for i, (B, S, Hq, Hkv, rot) in enumerate([(1, 1, 1, 1, d), (2, 33, 8, 2, d // 2), (3, 64, 5, 5, d // 4), (1, 257, 6, 3, 0),
                                               (5, 1, 32, 8, d), (2, 130, 9, 1, 16), (1, 65, 3, 1, d - 16)]):
        say(f"d {d} inter {inter} norm {norm} case {i}")
        q, k, v = projection(B, S, Hq, Hkv, d, 10 + i)
        w = [(1 + 0.3 * normal((d,), 20 + j, torch.float32)).to(BF16 if i % 2 else torch.float32) if norm else None for j in range(2)]
        pos = [None, torch.arange(B, dtype=torch.int32, device="cuda") * 97,
               torch.randint(0, 5000, (B, S), dtype=torch.int32, device="cuda")][i % 3]
        run_and_check(q, k, v, f"case {i}", freqs=freqs_of(rot)[0] if rot else None, positions=pos, inter=inter,
                      amplitude=1.0 if i % 2 else 1.25, wq=w[0], wk=w[1])


def test_only_some_tensors():
    q, k, v = projection(2, 40, 4, 2, 128, 1)
    f = freqs_of(128)[0]
    w = 1 + 0.3 * normal((128,), 2, torch.float32)
    run_and_check(q, None, None, "q alone", freqs=f, wq=w)
    run_and_check(None, k, None, "k alone", freqs=f, wk=w)
    run_and_check(None, None, v, "v alone")
    run_and_check(q, k, None, "q with a norm, k without", freqs=f, wq=w)
    run_and_check(q, k, v, "k with a norm, q without", freqs=f, wk=w)


def test_strides():
    f = freqs_of(64)[0]
    x = normal((2, 7, 45, 3 * 64), 3)  # [B, H, S, ...]: heads outside positions, rows inside wider ones
    run_and_check(x[..., 64:128].transpose(1, 2), None, None, "heads outermost", freqs=f)
    run_and_check(x.transpose(1, 2)[:, 3:44:2, 1:7:3, 8:72], None, None, "steps", freqs=f)
    run_and_check(x[:1, :, :1, :64].transpose(1, 2).expand(3, 5, 7, 64), None, None, "one row of each head for all", freqs=f)
    one = normal((1, 1, 1, 64), 4).as_strided((1, 1, 1, 64), (13, 5, 3, 1))
    run_and_check(one, None, None, "strides of one element", freqs=f)


def test_batches_far_apart():
    # (as those of long projections: beyond 2^31 elements)
    far = 2 ** 31 + 64
    x = torch.empty((far + 5 * 6 * 64,), dtype=BF16, device="cuda")
    view = x.as_strided((2, 5, 6, 64), (far, 6 * 64, 64, 1))
    view.copy_(normal((2, 5, 6, 64), 5))
    run_and_check(*view.split([4, 1, 1], 2), "far apart", freqs=freqs_of(64)[0], wq=1 + 0.3 * normal((64,), 6, torch.float32))


@pytest.mark.parametrize("inter", [False, True])
def test_far_positions(inter):
    # (angles of 2^31 radians: reduced in 64 bits, they are as exact as FP64 has them)
    for top in (10 ** 6, 2 ** 24 + 1, 2 ** 31 - 40):
        pos = torch.tensor([top, -top, 0], dtype=torch.int32, device="cuda")
        q, k, v = projection(3, 37, 2, 1, 128, 5)
        f, a = freqs_of(128, 500000.0, scaling="ramp", factor=8.0, original=8192)
        run_and_check(q, k, v, f"at {top}", freqs=f, positions=pos, inter=inter, amplitude=a)


def test_sums_of_positions_beyond_32_bits():
    # the first position + i leaves 32 bits, as the formula's number does
    pos = torch.tensor([2 ** 31 - 3], dtype=torch.int32, device="cuda")
    run_and_check(*projection(1, 9, 2, 1, 64, 6), "beyond", freqs=freqs_of(64)[0], positions=pos)


@pytest.mark.parametrize("kw", [{}, {"scaling": "linear", "factor": 4.0}, {"scaling": "base", "factor": 4.0},
                                {"scaling": "ramp", "factor": 16.0, "original": 4096},
                                {"scaling": "smooth", "factor": 8.0, "original": 8192, "fast": 4.0}])
def test_scaled_frequencies(kw):
    f, a = freqs_of(128, **kw)
    q, k, v = projection(1, 100, 3, 1, 128, 7)
    run_and_check(q, k, v, str(kw), freqs=f, amplitude=a, positions=torch.tensor([30000], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("d", [64, 128])
def test_fp8_outputs(d):
    q, k, v = projection(2, 75, 6, 2, d, 8)
    f, descale = freqs_of(d)[0], (1 / 16, 1 / 7, 1 / 100)  # (v's large channels reach the limit)
    w = 1 + 0.3 * normal((d,), 9, torch.float32)
    got = pkg.attn_rope(q, k, v, freqs=f, q_weight=w, descale=descale, out_dtype=FP8)
    for x, weight, y, s, turn in ((q, w, got[0], descale[0], f), (k, None, got[1], descale[1], f), (v, None, got[2], descale[2], None)):
        z, tol = rope_ref(x, weight, turn, None, False, 1.0, 1e-6)
        # (1 / descale and the product: 2^-23)
        z, tol = z / s, (tol + 2.0 ** -23 * z.abs()) / s
        held = z.clamp(-448, 448)
        check(y.float(), held, 2.0 ** -4 * held.abs() + 2 * tol + 2.0 ** -10, f"fp8 d {d}")
    assert bool((got[2].float().abs() == 448).any())
    # what it returns is what the FP8 attention takes
    o, _ = pkg.attn_fwd_ex(*got, causal=True, scale=d ** -0.5, exp_mode=pkg.ATTN_EXP_EXACT, descale=descale)
    assert bool(torch.isfinite(o.float()).all())


def test_infinities_nan_and_zeros_stay_in_their_row():
    q, k, v = (x.clone() for x in projection(1, 20, 2, 2, 128, 10))
    f, w = freqs_of(64)[0], torch.ones(128, device="cuda")
    clean = pkg.attn_rope(q, k, v, freqs=f, q_weight=w)
    q[0, 3, 0, 5], q[0, 4, 1, 100], q[0, 5] = math.inf, math.nan, 0.0
    k[0, 6, 0, 100], k[0, 7, 1, 2], v[0, 8, 0, 0] = -math.inf, math.nan, math.inf
    got = pkg.attn_rope(q, k, v, freqs=f, q_weight=w)
    same = torch.ones(1, 2, 20, dtype=torch.bool, device="cuda")
    same[0, 0, 3] = same[0, 1, 4] = same[0, :, 5] = False
    assert torch.equal(got[0][same], clean[0][same]) and bool((got[0][0, :, 5] == 0).all())
    assert bool(got[0][0, 0, 3].isnan().any()) and bool(got[0][0, 1, 4].isnan().all())
    # without a norm only the pair is reached: channels 2 and 34; those beyond rot by themselves alone
    assert got[1][0, 0, 6, 100] == -math.inf and got[1][0, 1, 7].isnan().nonzero().flatten().tolist() == [2, 34]
    at = torch.ones(128, dtype=torch.bool, device="cuda")
    at[100] = False
    assert torch.equal(got[1][0, 0, 6][at], clean[1][0, 0, 6][at]) and got[2][0, 0, 8, 0] == math.inf
    # FP8: infinities become the largest value, NaN stays
    got = pkg.attn_rope(q, k, v, freqs=f, out_dtype=FP8, descale=(1.0, 1.0, 1.0))
    assert got[2][0, 0, 8, 0].float() == 448 and got[1][0, 0, 6, 100].float() == -448 and bool(got[1][0, 1, 7, 2].float().isnan())


def test_many_heads_and_positions():
    # runs of heads, and more workgroups than fit at once
    q, k, v = projection(1, 3001, 40, 5, 64, 11)
    w = (1 + 0.3 * normal((64,), 12, torch.float32)).to(BF16)
    run_and_check(q, k, v, "many", freqs=freqs_of(64)[0], wq=w, wk=w, inter=True)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", [BF16, FP8])
@pytest.mark.parametrize("tokens", [1, 5, 9, 17, 40, 63, 65, 97])
def test_nothing_behind_the_last_position_is_written(d, dtype, tokens):
    # (a wave's threads also load and store rows of other positions than their own)
    q, k, v = projection(1, tokens, 3, 1, d, 14)
    whole = torch.full((3 * tokens * d + 128 * d,), 7.0, device="cuda").to(dtype)
    out = whole[:3 * tokens * d].view(1, 3, tokens, d)
    f, kw = freqs_of(d)[0], dict(out_dtype=dtype) if dtype is FP8 else {}
    pkg.attn_rope(q, freqs=f, q_out=out, **kw)
    assert bool((whole[3 * tokens * d:].float() == 7).all())
    assert torch.equal(out.float(), pkg.attn_rope(q, freqs=f, **kw)[0].float())
    if dtype is FP8:
        return
    g = normal((1, 3, tokens, d), 15)
    pkg.attn_rope_bwd(g, freqs=f, dq=whole[:3 * tokens * d].view(1, tokens, 3, d))
    assert bool((whole[3 * tokens * d:].float() == 7).all())


def test_other_stream_and_graph():
    q, k, v = projection(2, 50, 4, 2, 128, 13)
    f, pos = freqs_of(128)[0], torch.tensor([3, 400], dtype=torch.int32, device="cuda")
    want = pkg.attn_rope(q, k, v, freqs=f, positions=pos)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.attn_rope(q, k, v, freqs=f, positions=pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    out = [torch.zeros_like(x) for x in want]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.attn_rope(q, k, v, freqs=f, positions=pos, q_out=out[0], k_out=out[1], v_out=out[2])
    for step in range(3):
        pos += 7  # the graph reads the positions when it runs
        graph.replay()
        torch.cuda.synchronize()
        want = pkg.attn_rope(q, k, v, freqs=f, positions=pos)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), step


@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (64, 32, True), (128, 128, False), (128, 32, False), (128, 64, True), (128, 0, False)])
def test_large_rows_have_their_norm(d, rot, inter):
    # the squares of values beyond 2^64 leave FP32, those of the largest rows with every factor that keeps small rows in it
    q, k, w = large_rows(2, 40, 3, d, 30), large_rows(2, 40, 2, d, 31), 1 + 0.3 * normal((d,), 32, torch.float32)
    f = freqs_of(rot)[0] if rot else None
    run_and_check(q, k, None, "large", freqs=f, inter=inter, amplitude=1.25, wq=w, wk=w.to(BF16).float())
    # (an eps that is itself of the size of the squares, and the largest: mean + eps leaves FP32, too)
    for eps in (2.0 ** 126, torch.finfo(torch.float32).max):
        run_and_check(q, None, None, f"eps {eps}", freqs=f, inter=inter, wq=w, eps=eps)


def test_large_rows_as_fp8():
    q, w, descale = large_rows(1, 40, 3, 128, 33), 1 + 0.3 * normal((128,), 34, torch.float32), (1 / 64, 1.0, 1.0)
    got = pkg.attn_rope(q, freqs=freqs_of(128)[0], q_weight=w, descale=descale, out_dtype=FP8)[0]
    z, tol = rope_ref(q, w, freqs_of(128)[0], None, False, 1.0, 1e-6)
    z, tol = z * 64, (tol + 2.0 ** -23 * z.abs()) * 64
    held = z.clamp(-448, 448)
    check(got.float(), held, 2.0 ** -4 * held.abs() + 2 * tol + 2.0 ** -10, "large rows as fp8")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inter", [False, True])
def test_an_infinity_makes_a_row_with_a_norm_nan(d, inter):
    # all of it, in the channels that are rotated and in those that are not, and no other row
    q, k, v = (x.clone() for x in projection(2, 20, 3, 2, d, 36))
    f, w = freqs_of(d // 2)[0], 1 + 0.3 * normal((d,), 37, torch.float32)
    w[3] = 0.0
    kw = dict(freqs=f, interleaved=inter, q_weight=w, k_weight=w)
    for out in ({}, dict(out_dtype=FP8, descale=(1 / 32, 1 / 32, 1 / 32))):
        clean = pkg.attn_rope(q, k, v, **kw, **out)
        x, y = q.clone(), k.clone()
        x[0, 3, 0, 5], x[1, 4, 1, d - 1], x[1, 19, 2, 0], x[1, 19, 2, 1] = math.inf, -math.inf, math.inf, -math.inf
        x[0, 7, 2, ::2], x[0, 7, 2, 9] = 1e38, math.inf
        y[0, 0, 1, d // 2] = math.inf
        got = pkg.attn_rope(x, y, v, **kw, **out)
        for new, old, rows in ((got[0], clean[0], [(0, 0, 3), (1, 1, 4), (1, 2, 19), (0, 2, 7)]), (got[1], clean[1], [(0, 1, 0)])):
            hit = torch.zeros(new.shape[:3], dtype=torch.bool, device="cuda")
            for at in rows:
                hit[at] = True
            assert bool(new.float()[hit].isnan().all()) and torch.equal(new.float()[~hit], old.float()[~hit])


def test_the_weight_of_an_absent_tensor_says_nothing():
    q, k, v = projection(2, 40, 4, 2, 128, 40)
    f, w, other = freqs_of(64)[0], 1 + 0.3 * normal((128,), 41, torch.float32), torch.full((128,), math.nan, device="cuda")
    assert torch.equal(pkg.attn_rope(None, k, v, freqs=f, q_weight=other, k_weight=w)[1], pkg.attn_rope(None, k, v, freqs=f, k_weight=w)[1])
    assert torch.equal(pkg.attn_rope(q, None, v, freqs=f, q_weight=w, k_weight=other)[0], pkg.attn_rope(q, None, v, freqs=f, q_weight=w)[0])
    assert torch.equal(pkg.attn_rope(None, None, v, freqs=f, q_weight=other, k_weight=other)[2], v.transpose(1, 2))

"""The gradient of norms and rotation (attn_rope_bwd) against the formula in
float64, and against differences of attn_rope's own definition."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from qkv_helpers import BF16, angles, check, grad_ref, inverse_rms, large_rows, normal, projection, say, turned

pytestmark = pytest.mark.gpu


def gradients(B, S, Hq, Hkv, d, seed):
    return [normal((B, h, S, d), seed + i) for i, h in enumerate((Hq, Hkv, Hkv))]


def run_and_check(x, g, what, *, freqs=None, positions=None, inter=False, amplitude=1.0, wq=None, wk=None, eps=1e-6, **kw):
    got = pkg.attn_rope_bwd(*g, q=x[0], k=x[1], freqs=freqs, positions=positions, interleaved=inter, amplitude=amplitude,
                            q_weight=wq, k_weight=wk, eps=eps, **kw)
    for i, (name, w) in enumerate((("q", wq), ("k", wk), ("v", None))):
        if g[i] is None:
            assert got[i] is None
            continue
        if name == "v":
            assert torch.equal(got[2], g[2].transpose(1, 2))
            continue
        dx, tol, dw, tol_w = grad_ref(g[i], x[i], w, freqs, positions, inter, amplitude, eps)
        check(got[i], dx, tol, f"{what} d{name}")
        if w is None:
            assert got[3 + i] is None
        else:
            check(got[3 + i], dw, tol_w, f"{what} d{name}_weight")
    return got


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("norm", [False, True])
def test_layouts_parts_and_sizes(d, inter, norm):
    for i, (B, S, Hq, Hkv, rot) in enumerate([(1, 1, 1, 1, d), (2, 33, 8, 2, d // 2), (3, 64, 5, 5, d // 4), (1, 257, 6, 3, 0),
                                               (5, 1, 32, 8, d), (1, 65, 3, 1, d - 16)]):
        say(f"d {d} inter {inter} norm {norm} case {i}")
        x, g = projection(B, S, Hq, Hkv, d, 10 + i), gradients(B, S, Hq, Hkv, d, 40 + i)
        w = [(1 + 0.3 * normal((d,), 20 + j, torch.float32)).to(BF16 if i % 2 else torch.float32) if norm else None for j in range(2)]
        pos = [None, torch.arange(B, dtype=torch.int32, device="cuda") * 97,
               torch.randint(0, 5000, (B, S), dtype=torch.int32, device="cuda")][i % 3]
        f = pkg.attn_rope_frequencies(rot, device="cuda")[0] if rot else None
        run_and_check(x, g, f"case {i}", freqs=f, positions=pos, inter=inter, amplitude=1.0 if i % 2 else 1.25, wq=w[0], wk=w[1])


def test_many_positions_and_a_fused_gradient():
    # several tiles a workgroup, gradients written into parts of one tensor, the rest of it left alone
    B, S, Hq, Hkv, d = 2, 5000, 12, 2, 64
    x, g = projection(B, S, Hq, Hkv, d, 1), gradients(B, S, Hq, Hkv, d, 2)
    w = [1 + 0.3 * normal((d,), 20 + j, torch.float32) for j in range(2)]
    whole = torch.full((B, S, Hq + 2 * Hkv + 1, d), 7.0, dtype=BF16, device="cuda")
    dq, dk, dv, _ = whole.split([Hq, Hkv, Hkv, 1], 2)
    f = pkg.attn_rope_frequencies(d, device="cuda")[0]
    ws = torch.full((pkg.attn_rope_bwd_workspace_bytes(B, S, Hq, Hkv, d),), 255, dtype=torch.uint8, device="cuda")
    got = run_and_check(x, g, "fused", freqs=f, wq=w[0], wk=w[1], dq=dq, dk=dk, dv=dv, workspace=ws)
    assert got[0] is dq and bool((whole[:, :, -1] == 7).all())
    again = pkg.attn_rope_bwd(*g, q=x[0], k=x[1], freqs=f, q_weight=w[0], k_weight=w[1])
    assert all(torch.equal(a, b) for a, b in zip(got, again))  # (a fixed order of sums)


def test_batches_far_apart():
    # (as those of long projections: beyond 2^31 elements, those of a fused gradient too)
    far = 2 ** 31 + 64
    x, out = (torch.empty((far + 5 * 6 * 64,), dtype=BF16, device="cuda").as_strided((2, 5, 6, 64), (far, 6 * 64, 64, 1))
              for _ in range(2))
    x.copy_(normal((2, 5, 6, 64), 5))
    w = 1 + 0.3 * normal((64,), 6, torch.float32)
    dq, dk, dv = out.split([4, 1, 1], 2)
    run_and_check(x.split([4, 1, 1], 2), gradients(2, 5, 4, 1, 64, 7), "far apart", freqs=pkg.attn_rope_frequencies(64, device="cuda")[0],
                  wq=w, wk=w, dq=dq, dk=dk, dv=dv)


def test_only_some_tensors():
    x, g = projection(2, 40, 4, 2, 128, 3), gradients(2, 40, 4, 2, 128, 4)
    f, w = pkg.attn_rope_frequencies(128, device="cuda")[0], 1 + 0.3 * normal((128,), 5, torch.float32)
    run_and_check((x[0], None), [g[0], None, None], "q alone", freqs=f, wq=w)
    run_and_check((None, x[1]), [None, g[1], None], "k alone", freqs=f, wk=w)
    run_and_check((None, None), [None, None, g[2]], "v alone")
    run_and_check((None, x[1]), g, "k with a norm, q without", freqs=f, wk=w)
    # a weight whose tensor has no gradient here is not asked for
    run_and_check((None, x[1]), [None, g[1], None], "q's weight unused", freqs=f, wq=None, wk=w)


def test_zero_rows():
    x, g = [y.clone() for y in projection(1, 9, 2, 1, 64, 6)], gradients(1, 9, 2, 1, 64, 7)
    x[0][0, 4], x[1][0, 2] = 0.0, 0.0
    w = torch.ones(64, device="cuda")
    # (1 / sqrt(eps) multiplies what comes in)
    run_and_check(x, g, "zero rows", freqs=pkg.attn_rope_frequencies(64, device="cuda")[0], wq=w, wk=w, eps=1e-6)


def test_against_differences():
    """The sum of g times attn_rope's definition, in float64, moves with each input as the kernel's gradient says."""
    B, S, H, d, eps, amp = 1, 3, 2, 64, 1e-5, 1.2
    x, g = projection(B, S, H, 1, d, 8)[0], normal((B, H, S, d), 9)
    f, w = pkg.attn_rope_frequencies(32, device="cuda")[0], 1 + 0.3 * normal((d,), 10, torch.float32)
    dx, _, _, dw, _ = pkg.attn_rope_bwd(g, q=x, freqs=f, q_weight=w, eps=eps, amplitude=amp)
    t, gd = angles(f, None, B, S), g.double().transpose(1, 2)

    def value(xx, ww):
        return (gd * turned(xx * inverse_rms(xx, eps) * ww, t, 32, False, amp)[0]).sum().item()

    xd, wd, step = x.double(), w.double(), 1e-4
    for c in range(0, d, 5):
        e = torch.zeros_like(wd)
        e[c] = step
        slope = (value(xd, wd + e) - value(xd, wd - e)) / (2 * step)
        # (central differences: linear in w; the FP32 sums)
        assert abs(slope - dw[c].item()) <= 1e-5 * (gd.abs() * 10).sum(), c
        for s, h in ((0, 0), (2, 1)):
            e = torch.zeros_like(xd)
            e[0, s, h, c] = step
            slope = (value(xd + e, wd) - value(xd - e, wd)) / (2 * step)
            # half a step of the BF16 gradient, and the differences' own error
            assert abs(slope - dx[0, s, h, c].item()) <= 2.0 ** -8 * abs(slope) + 1e-4, (s, h, c)


def test_captured_beside_eager_calls():
    x, g = projection(2, 70, 4, 2, 128, 11), gradients(2, 70, 4, 2, 128, 12)
    f, w = pkg.attn_rope_frequencies(128, device="cuda")[0], 1 + 0.3 * normal((128,), 13, torch.float32)
    kw = dict(q=x[0], k=x[1], freqs=f, q_weight=w, k_weight=w)
    out = pkg.attn_rope_bwd(*g, **kw)
    ws = torch.empty(pkg.attn_rope_bwd_workspace_bytes(2, 70, 4, 2, 128), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pkg.attn_rope_bwd(*g, **kw, dq=out[0], dk=out[1], dv=out[2], dq_weight=out[3], dk_weight=out[4], workspace=ws)
    for step in range(3):
        g[0].mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        want = pkg.attn_rope_bwd(*g, **kw)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), step
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pkg.attn_rope_bwd(*g, **kw, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("d,rot,inter", [(64, 64, False), (64, 32, True), (128, 128, False), (128, 32, False), (128, 64, True), (128, 0, False)])
def test_large_rows_have_their_gradient(d, rot, inter):
    # (rows whose squares leave FP32: dx is small, the weights' gradient has every row's part)
    x, g = (large_rows(2, 40, 3, d, 30), large_rows(2, 40, 2, d, 31), None), gradients(2, 40, 3, 2, d, 32)
    w = 1 + 0.3 * normal((d,), 35, torch.float32)
    f = pkg.attn_rope_frequencies(rot, device="cuda")[0] if rot else None
    run_and_check(x, g, "large", freqs=f, inter=inter, amplitude=1.25, wq=w, wk=w)
    for eps in (2.0 ** 126, torch.finfo(torch.float32).max):
        run_and_check(x, g, f"eps {eps}", freqs=f, inter=inter, wq=w, wk=w, eps=eps)
    # gradients large enough that the largest rows' dx are ordinary numbers again
    g = [(y.float() * 2.0 ** 100).to(BF16) for y in g]
    dx = pkg.attn_rope_bwd(*g, q=x[0], k=x[1], freqs=f, interleaved=inter, q_weight=w, k_weight=w)
    for i in range(2):
        want, tol, _, _ = grad_ref(g[i], x[i], w, f, None, inter, 1.0, 1e-6)
        check(dx[i], want, tol, f"large gradients {i}")


@pytest.mark.parametrize("d", [64, 128])
def test_an_infinity_makes_its_row_and_the_weights_gradient_nan(d):
    x, g = [y.clone() for y in projection(2, 20, 3, 2, d, 36)], gradients(2, 20, 3, 2, d, 37)
    f, w = pkg.attn_rope_frequencies(d // 2, device="cuda")[0], 1 + 0.3 * normal((d,), 38, torch.float32)
    clean = pkg.attn_rope_bwd(*g, q=x[0], k=x[1], freqs=f, q_weight=w, k_weight=w)
    x[0][0, 3, 0, 5], x[0][1, 4, 1, d - 1] = math.inf, -math.inf
    got = pkg.attn_rope_bwd(*g, q=x[0], k=x[1], freqs=f, q_weight=w, k_weight=w)
    hit = torch.zeros(2, 20, 3, dtype=torch.bool, device="cuda")
    hit[0, 3, 0] = hit[1, 4, 1] = True
    assert bool(got[0][hit].isnan().all()) and torch.equal(got[0][~hit], clean[0][~hit])
    assert bool(got[3].isnan().all())
    assert all(torch.equal(got[i], clean[i]) for i in (1, 2, 4))


def test_a_weight_whose_tensor_has_no_gradient_is_not_asked_for():
    # (its tensor may be given, too: it is not read)
    x, g = projection(2, 40, 4, 2, 128, 3), gradients(2, 40, 4, 2, 128, 4)
    f, w, other = pkg.attn_rope_frequencies(128, device="cuda")[0], 1 + 0.3 * normal((128,), 5, torch.float32), torch.full((128,), 7.0, device="cuda")
    for q in (None, x[0]):
        run_and_check((q, x[1]), [None, g[1], g[2]], "q's weight without gq", freqs=f, wq=other, wk=w)
        got = pkg.attn_rope_bwd(None, g[1], g[2], q=q, k=x[1], freqs=f, q_weight=other, k_weight=w)
        want = pkg.attn_rope_bwd(None, g[1], g[2], k=x[1], freqs=f, k_weight=w)
        assert got[0] is None and got[3] is None and all(torch.equal(got[i], want[i]) for i in (1, 2, 4))
    for k in (None, x[1]):
        run_and_check((x[0], k), [g[0], None, None], "k's weight without gk", freqs=f, wq=w, wk=other)
        got = pkg.attn_rope_bwd(g[0], None, g[2], q=x[0], k=k, freqs=f, q_weight=w, k_weight=other)
        want = pkg.attn_rope_bwd(g[0], None, g[2], q=x[0], freqs=f, q_weight=w)
        assert got[1] is None and got[4] is None and all(torch.equal(got[i], want[i]) for i in (0, 2, 3))

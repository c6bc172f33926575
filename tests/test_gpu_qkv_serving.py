"""A layer as it serves: prompts through the projection's output, rotation and
norms, the cache of 8-bit blocks and attention over it, then single tokens,
against the same in float64 that keeps the codes the kernels wrote."""
import pytest
import torch

import paper_2609_33586_amd as pkg
from qkv_helpers import (BF16, E8M0, EXACT, FP8, H15, append_ref, bf16_tolerance, block_cache, blocks_ref, check, check_prefix, normal,
                         projection, rope_ref, say, scale_of)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,block,mode,inter", [(128, 64, EXACT, False), (64, 16, H15, True)])
def test_prompt_then_tokens(d, block, mode, inter):
    B, Hq, Hkv, S, cap, sc = 3, 8, 2, 150, 256, scale_of(d)
    f, amplitude = pkg.attn_rope_frequencies(d, scaling="ramp", factor=4.0, original=64, device="cuda")
    w = [(1 + 0.2 * normal((d,), 1 + i, torch.float32)).to(BF16) for i in range(2)]
    kc, vc = (torch.zeros((B, Hkv, cap, d), dtype=torch.uint8, device="cuda").view(FP8) for _ in range(2))
    scales = torch.zeros((B, Hkv, -(-cap // block), 2), dtype=torch.uint8, device="cuda").view(E8M0)
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    n = [0] * B
    # a padded batch of prompts, then tokens one by one and a few drafted ones at once
    for step, (s, counts) in enumerate([(S, [150, 31, 97]), (1, None), (1, None), (4, None), (1, None), (16, [16, 0, 3])]):
        x = projection(B, s, Hq, Hkv, d, 50 + step)
        q, k, v = pkg.attn_rope(*x, freqs=f, positions=lens, interleaved=inter, amplitude=amplitude, q_weight=w[0], k_weight=w[1])
        for y, xx, ww in ((q, x[0], w[0]), (k, x[1], w[1])):
            z, tol = rope_ref(xx, ww, f, lens, inter, amplitude, 1e-6)
            check(y, z, bf16_tolerance(z, tol), f"step {step}")
        before = [kc.float(), vc.float()]
        was = scales.view(torch.uint8).clone()
        ct = None if counts is None else torch.tensor(counts, dtype=torch.int32, device="cuda")
        lens = pkg.attn_cache_append(k, v, kc, vc, scales, lens, block=block, counts=ct)
        for i, (rows, codes) in enumerate(((k, kc), (v, vc))):
            out, sb, end = append_ref(rows, before[i], was[..., i], n, counts, cap, block)
            assert torch.equal(codes.float().double(), out) and torch.equal(scales.view(torch.uint8)[..., i].int(), sb)
        n = end
        assert lens.tolist() == n
        cut = pkg.attn_decode_blocks_split_keys(B, Hq, Hkv, s, cap, d)
        if counts is not None:
            # each sequence's own last rows: the padded ones' outputs are not looked at
            for b in range(B):
                if not counts[b]:
                    continue
                one = slice(b, b + 1)
                qb = q[one, :, :counts[b]].contiguous()
                o, lse = pkg.attn_decode_blocks(qb, kc[one], vc[one], scales[one], block=block, lens=lens[one], causal=True,
                                                scale=sc, exp_mode=mode, split_keys=cut)
                check_prefix(o, lse, blocks_ref(qb, kc[one], vc[one], scales[one], block, [n[b]], True, sc, mode, cut), f"step {step} b {b}")
        else:
            o, lse = pkg.attn_decode_blocks(q, kc, vc, scales, block=block, lens=lens, causal=True, scale=sc, exp_mode=mode, split_keys=cut)
            check_prefix(o, lse, blocks_ref(q, kc, vc, scales, block, n, True, sc, mode, cut), f"step {step}")
    say("served")


def test_training_step():
    """Rotation and norms into a plain causal attention and back: the projection's and the weights' gradients equal
    those of the whole in float64, up to what BF16 queries, keys and gradients round."""
    B, S, Hq, Hkv, d, eps = 1, 24, 4, 2, 64, 1e-6
    x = normal((B, S, (Hq + 2 * Hkv) * d), 1)
    w = [1 + 0.2 * normal((d,), 2 + i, torch.float32) for i in range(2)]
    f = pkg.attn_rope_frequencies(d, device="cuda")[0]
    views = lambda t: t.view(B, S, -1, d).split([Hq, Hkv, Hkv], 2)  # noqa: E731
    target = normal((B, Hq, S, d), 5, torch.float64)
    hide = torch.ones(S, S, dtype=torch.bool, device="cuda").triu(1)

    def loss(q, k, v):
        k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
        p = ((q @ k.transpose(-1, -2).contiguous()) * d ** -0.5).masked_fill(hide, -torch.inf).softmax(-1)
        return ((p @ v) * target).sum()

    q, k, v = pkg.attn_rope(*views(x), freqs=f, q_weight=w[0], k_weight=w[1], eps=eps)
    leaves = [t.double().requires_grad_() for t in (q, k, v)]
    g = [t.to(BF16) for t in torch.autograd.grad(loss(*leaves), leaves)]
    dx = torch.zeros_like(x)
    dq, dk, dv = views(dx)
    *_, dwq, dwk = pkg.attn_rope_bwd(*g, q=views(x)[0], k=views(x)[1], freqs=f, q_weight=w[0], k_weight=w[1], eps=eps, dq=dq, dk=dk, dv=dv)

    from qkv_helpers import angles, inverse_rms, turned
    whole = [x.double().requires_grad_(), *(t.double().requires_grad_() for t in w)]
    t = angles(f, None, B, S)
    parts = []
    for y, ww in zip(views(whole[0]), (whole[1], whole[2], None)):
        if ww is not None:
            y = turned(y * inverse_rms(y, eps) * ww, t, d, False, 1.0)[0]
        parts.append(y.transpose(1, 2))
    want = torch.autograd.grad(loss(*parts), whole)
    # operands off by 2^-9 rms each, products of a few of them: 2% of the norm is ten times that
    for got, ref, what in ((dx, want[0], "projection"), (dwq, want[1], "q_weight"), (dwk, want[2], "k_weight")):
        err = ((got.double() - ref).norm() / ref.norm()).item()
        say(f"{what}: {err:.2e}")
        assert err <= 2.0 ** -9 * 10, what


@pytest.mark.parametrize("mode", [EXACT, H15])
@pytest.mark.parametrize("S", [7, 70])
def test_padded_batch_with_its_rows_moved_behind_the_padding(mode, S):
    # attn_cache_append takes a sequence's rows before its padding, attn_decode_blocks after it: moved there, a padded batch's
    # queries go through one call
    B, Hq, Hkv, d, block, cap = 4, 8, 2, 128, 16, 256
    counts, n = [S, 1, 0, S // 2], [3, 40, 17, 0]
    f = pkg.attn_rope_frequencies(d, device="cuda")[0]
    k0, v0, scales = block_cache(B, Hkv, cap, d, block, 70)
    lens, ct = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (n, counts))
    q, k, v = pkg.attn_rope(*projection(B, S, Hq, Hkv, d, 71), freqs=f, positions=lens)
    after = pkg.attn_cache_append(k, v, k0, v0, scales, lens, block=block, counts=ct)
    ends = [a + c for a, c in zip(n, counts)]
    assert after.tolist() == ends
    # row i of the batch's first counts[b] goes to S - counts[b] + i, padding to the rows before
    at = (torch.arange(S, device="cuda") + ct[:, None]) % S
    moved = q.gather(2, at[:, None, :, None].expand_as(q))
    o, lse = pkg.attn_decode_blocks(moved, k0, v0, scales, block=block, lens=after, causal=True, scale=scale_of(d), exp_mode=mode, split_keys=0)
    for b in range(B):
        if not counts[b]:
            continue
        rows = slice(S - counts[b], S)
        one = slice(b, b + 1)
        assert torch.equal(moved[b, :, rows], q[b, :, :counts[b]])
        ref = blocks_ref(q[one, :, :counts[b]], k0[one], v0[one], scales[one], block, [ends[b]], True, scale_of(d), mode, 0)
        check_prefix(o[one, :, rows], lse[one, :, rows], ref, f"b {b}")

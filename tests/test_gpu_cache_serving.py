"""The operators over shared and bounded caches as a serving loop runs them:
prompts through the forward, the weights their last queries gave, eviction,
then steps of decode over a shared prefix with the compact caches, the weights
of every step, and another eviction, against the same loop in float64 that
keeps the keys the kernels chose."""
import math

import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import BF16, EXACT, FP8, DESCALE, H15, check_prefix, prefix_ref, randn, say, scale_of, weights_ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt,d,mode", [(BF16, 128, EXACT), (BF16, 64, H15), (FP8, 128, EXACT)])
def test_prompt_evict_decode_evict(dt, d, mode):
    B, Hq, Hkv, S, W, P, keep, cap = 3, 8, 2, 400, 48, 300, 96, 128
    sc, descale = scale_of(d), DESCALE if dt == FP8 else None
    kp, vp = randn((Hkv, P, d), 1, dt), randn((Hkv, P, d), 2, dt)
    q = randn((B, Hq, S, d), 3, dt)
    k, v = randn((B, Hkv, S, d), 4, dt, sharp=True), randn((B, Hkv, S, d), 5, dt)
    # the prompts' own attention, and what their last W queries gave each key
    _, lse = pkg.attn_fwd_ex(q, k, v, causal=True, scale=sc, exp_mode=EXACT, descale=descale)
    tail, tail_lse = q[:, :, -W:].contiguous(), lse[:, :, -W:].contiguous()
    acc = pkg.attn_key_weights(tail, k, tail_lse, torch.zeros(B, Hkv, S, device="cuda"), causal=True, scale=sc,
                               descale=descale)
    want, tol = weights_ref(tail, k, tail_lse, torch.zeros_like(acc), [S] * B, True, sc, descale, 1.0)
    assert bool(((acc.double() - want).abs() <= tol).all())
    # compact caches with room for new keys
    room = lambda: torch.zeros((B, Hkv, cap, d * q.element_size()), dtype=torch.uint8, device="cuda").view(dt)  # noqa: E731
    kc, vc, ac = room(), room(), torch.zeros((B, Hkv, cap), device="cuda")
    _, _, _, index, lens = pkg.attn_evict(k, v, acc, keep=keep, recent=W // 2, k_out=kc, v_out=vc, acc_out=ac)
    at = index.long().unsqueeze(-1).expand(-1, -1, -1, d * q.element_size())
    assert torch.equal(kc[:, :, :keep].view(torch.uint8), k.view(torch.uint8).gather(2, at))
    n = [keep] * B
    cuts = pkg.attn_decode_prefix_split_keys(B, Hq, Hkv, 1, P, cap, d, pkg.ATTN_BF16 if dt == BF16 else pkg.ATTN_FP8_E4M3)
    for step in range(cap - keep):
        # a new key and value of each sequence, then its query row
        x = randn((B, Hkv, 2, d), 100 + step, dt)
        kc[:, :, n[0]] = x[:, :, 0]
        vc[:, :, n[0]] = x[:, :, 1]
        n = [i + 1 for i in n]
        lens += 1
        q1 = randn((B, Hq, 1, d), 200 + step, dt)
        o, lse1 = pkg.attn_decode_prefix(q1, kp, vp, kc, vc, lens=lens, causal=True, scale=sc, exp_mode=mode,
                                         prefix_split_keys=cuts[0], split_keys=cuts[1], descale=descale)
        before = ac.clone()
        pkg.attn_key_weights(q1, kc, lse1, ac, lens=lens, causal=True, scale=sc, descale=descale, decay=0.9)
        if step % 8 == 0:
            check_prefix(o, lse1, prefix_ref(q1, kp, vp, kc, vc, n, True, sc, descale, mode, *cuts), f"step {step}")
            want, tol = weights_ref(q1, kc, lse1, before, n, True, sc, descale, 0.9)
            assert bool(((ac.double() - want).abs() <= tol).all())
    k2, v2, a2, index, lens2 = pkg.attn_evict(kc, vc, ac, lens=lens, keep=keep, recent=10)
    assert lens2.tolist() == [keep] * B
    late = torch.arange(cap - 10, cap, device="cuda", dtype=torch.int32)
    assert bool((index[..., -10:] == late).all())
    dropped = ac.scatter(2, index.long(), -1.0)[..., :cap - 10].amax(-1)  # none that went had more than one that stayed
    stayed = torch.where(index < cap - 10, a2, math.inf).amin(-1)
    assert bool((dropped <= stayed).all())
    q1 = randn((B, Hq, 1, d), 999, dt)
    o, lse1 = pkg.attn_decode_prefix(q1, kp, vp, k2, v2, lens=lens2, causal=True, scale=sc, exp_mode=mode,
                                     prefix_split_keys=0, split_keys=0, descale=descale)
    say("after the second eviction")
    check_prefix(o, lse1, prefix_ref(q1, kp, vp, k2, v2, [keep] * B, True, sc, descale, mode, 0, 0), "compact caches")

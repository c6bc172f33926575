"""Calls on a side stream, in no order with the current one, while the current
stream still uses memory that was let go: workspaces and outputs that a call
takes for itself are not that memory."""
import pytest
import torch

import paper_2609_33586_amd as pkg
from cache_helpers import BF16, H15, randn, say, scale_of

pytestmark = pytest.mark.gpu


def prefix(stream):
    q, kp, vp, k, v = OPERANDS["prefix"]
    return pkg.attn_decode_prefix(q, kp, vp, k, v, causal=True, scale=scale_of(128), exp_mode=H15, prefix_split_keys=128,
                                  split_keys=128, stream=stream)


def decode(stream):
    q, _, _, k, v = OPERANDS["prefix"]
    return pkg.attn_decode(q, k, v, causal=True, scale=scale_of(128), exp_mode=H15, split_keys=128, stream=stream)


def forward(stream):
    q = OPERANDS["forward"]
    return pkg.attn_fwd_ex(q, q, q, causal=True, scale=scale_of(128), exp_mode=H15, stream=stream)


def weights(stream):
    q, k, lse = OPERANDS["weights"]
    acc = torch.zeros(k.shape[:3], device="cuda")
    torch.cuda.synchronize()
    if stream is not None:
        acc.record_stream(stream)  # given by the caller, who lets it go below
    return (pkg.attn_key_weights(q, k, lse, acc, causal=True, scale=scale_of(128), stream=stream),)


def evict(stream):
    k, acc = OPERANDS["evict"]
    return pkg.attn_evict(k, k, acc, keep=9000, recent=10, stream=stream)


OPERANDS = {}


@pytest.fixture(scope="module", autouse=True)
def operands():
    OPERANDS["prefix"] = (randn((16, 8, 4, 128), 1, BF16), randn((2, 1024, 128), 2, BF16), randn((2, 1024, 128), 3, BF16),
                          randn((16, 2, 512, 128), 4, BF16), randn((16, 2, 512, 128), 5, BF16))
    OPERANDS["forward"] = randn((4, 8, 512, 128), 6, BF16)
    q, k = randn((2, 8, 1024, 128), 7, BF16), randn((2, 2, 40000, 128), 8, BF16)
    OPERANDS["weights"] = (q, k, torch.full((2, 8, 1024), 12.0, device="cuda"))
    OPERANDS["evict"] = (randn((1, 4, 40000, 128), 9, BF16), torch.rand((1, 4, 40000), device="cuda"))
    yield
    OPERANDS.clear()


@pytest.mark.parametrize("call", [prefix, decode, forward, weights, evict], ids=lambda f: f.__name__)
def test_pending_work_of_the_current_stream_keeps_its_memory(call):
    want = call(None)
    side, a = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    # the sizes that the call will ask for, among them its workspace
    need = {prefix: pkg.attn_decode_prefix_workspace_bytes(16, 8, 4, 1024, 512, 128, 128, 128),
            decode: pkg.attn_decode_workspace_bytes(16, 8, 4, 512, 128, 128),
            weights: pkg.attn_key_weights_workspace_bytes(2, 8, 2, 1024, 40000, 128),
            evict: pkg.attn_evict_workspace_bytes(1, 4, 40000)}.get(call, 0)
    assert call is forward or need > 0
    sizes = [n for n in [need] + [t.numel() * t.element_size() for t in want] if n]
    blocks = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes]
    say(f"{call.__name__}: blocks of {sizes} bytes")
    for _ in range(40):  # keeps the current stream busy
        a = a @ a * 1e-3
    copies = [b.clone() for b in blocks]
    del blocks
    got = call(side)
    torch.cuda.synchronize()
    for c in copies:
        assert bool((c == 7).all())
    for x, y in zip(got, want):
        assert torch.equal(x, y)
    # outputs that are let go while the side stream still writes them go back to its pool
    out = call(side)
    del out
    fresh = [torch.full((n,), 9, dtype=torch.uint8, device="cuda") for n in sizes]
    torch.cuda.synchronize()
    for b in fresh:
        assert bool((b == 9).all())


def test_attn_fwd_runs_on_the_default_stream_with_memory_of_its_own():
    q = OPERANDS["forward"]
    kw = dict(causal=True, scale=scale_of(128), exp_mode=H15)
    want = pkg.attn_fwd(q, q, q, **kw)
    side, a = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")
    sizes = [t.numel() * t.element_size() for t in want]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        blocks = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes]
        for _ in range(40):  # keeps the side stream busy
            a = a @ a * 1e-3
        copies = [b.clone() for b in blocks]
        del blocks
        got = pkg.attn_fwd(q, q, q, **kw)
    torch.cuda.synchronize()
    assert all(bool((c == 7).all()) for c in copies)
    assert all(torch.equal(x, y) for x, y in zip(got, want))

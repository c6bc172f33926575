"""As tests/test_cache_streams.py for the operators between projections and
attention: memory that a call takes for itself comes from the stream's pool that
it runs on, and sizes and streams that do not fit are refused."""
import pytest
import torch

import paper_2609_33586_amd as pkg
from paper_2609_33586_amd import cache, qkv
from test_cache_streams import Library, Stream, Tensor, pool  # noqa: F401 (pool: the fixture)


class Strided(Tensor):
    def stride(self):
        s = [1]
        for n in reversed(self.shape[1:]):
            s.insert(0, s[0] * n)
        return tuple(s)


@pytest.fixture
def bound():
    """The binding's own library, before another stands in for the package's."""
    return qkv._lib()


@pytest.fixture(autouse=True)
def library(bound, pool, monkeypatch):  # noqa: F811
    monkeypatch.setattr(qkv, "_bound", Library())
    empty = torch.empty

    def strided(*shape, dtype=None, device=None):
        t = empty(*shape, dtype=dtype, device=device)
        t.__class__ = Strided
        return t

    monkeypatch.setattr(torch, "empty", strided)
    monkeypatch.setattr(torch, "empty_strided", lambda shape, strides, **kw: strided(shape, **kw))


Q, KV = Strided(2, 5, 4, 64), Strided(2, 5, 2, 64)  # [B, S, H, d]
GQ, GKV = Strided(2, 4, 5, 64), Strided(2, 2, 5, 64)  # [B, H, S, d]
W, F = Strided(64, dtype=torch.float32), Strided(32, dtype=torch.float64)
C, N = Strided(2, 2, 300, 64, dtype=torch.float8_e4m3fn), Strided(2, dtype=torch.int32)
SC = Strided(2, 2, 19, 2, dtype=torch.uint8)
CALLS = {
    "attn_rope": (lambda s: pkg.attn_rope(Q, KV, KV, freqs=F, q_weight=W, stream=s), 3),
    "attn_rope_bwd": (lambda s: pkg.attn_rope_bwd(GQ, GKV, GKV, q=Q, k=KV, freqs=F, q_weight=W, k_weight=W, stream=s), 5),
    "attn_cache_append": (lambda s: pkg.attn_cache_append(GKV, GKV, C, C, SC, N, block=16, stream=s), 1),
    "attn_decode_blocks": (lambda s: pkg.attn_decode_blocks(GQ, C, C, SC, block=16, causal=True, scale=0.1, exp_mode=1,
                                                            split_keys=128, stream=s), 2),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_comes_from_the_stream_that_the_call_runs_on(pool, name):  # noqa: F811
    side = Stream(2)
    call, outputs = CALLS[name]
    got = call(side)
    assert len(pool) >= outputs and all(t.owner is side for t in pool)
    returned = [t for t in (got if isinstance(got, tuple) else (got,)) if t.owner is not None]
    assert len(returned) == outputs and all(t.waits == [pool.current] for t in returned)


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_the_current_stream_take_its_memory(pool, name):  # noqa: F811
    CALLS[name][0](None)
    assert len(pool) > 0 and all(t.owner is pool.current and t.waits == [] for t in pool)


@pytest.mark.parametrize("name", CALLS)
def test_streams_of_another_device_are_refused(pool, name):  # noqa: F811
    with pytest.raises(ValueError, match="stream must belong to GPU 0"):
        CALLS[name][0](Stream(3, device=1))
    assert not pool


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(pool, monkeypatch, name):  # noqa: F811
    monkeypatch.setattr(cache, "_device", lambda: 1)
    with pytest.raises(ValueError, match="current GPU"):
        CALLS[name][0](None)


@pytest.mark.parametrize("name", ["Sk", "split_keys"])
def test_sizes_beyond_32_bits_are_refused(pool, name):  # noqa: F811
    kw = dict(block=16, causal=True, scale=0.1, exp_mode=1, split_keys=0)
    for x in (2 ** 31, 2 ** 32, 2 ** 32 + 128, -2 ** 31 - 1):
        with pytest.raises(ValueError, match=f"^{name} "):
            pkg.attn_decode_blocks(GQ, C, C, SC, **{**kw, name: x})


def test_outputs_with_nothing_to_write(pool):  # noqa: F811
    for call in (lambda: pkg.attn_rope(Q, v_out=GKV), lambda: pkg.attn_rope_bwd(GQ, dv=KV), lambda: pkg.attn_rope_bwd(GQ, dq_weight=W),
                 lambda: pkg.attn_rope_bwd(GQ, q_weight=W)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        pkg.attn_rope(Q, out_dtype=torch.float16)
    with pytest.raises(ValueError, match="same heads"):
        pkg.attn_rope(Q, KV, Q)
    with pytest.raises(ValueError, match="same heads"):
        pkg.attn_rope_bwd(GQ, GKV, GQ)

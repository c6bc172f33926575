"""Memory that a call takes for itself when it is given a stream: it has to come
from that stream's pool.  A block of the current stream's pool may be one that
was let go a moment ago and that a kernel still running there reads or writes.
The allocator, the library and the tensors are stood in for here (no GPU)."""
import contextlib

import pytest
import torch

import paper_2609_33586_amd as pkg
from paper_2609_33586_amd import cache


class Stream:
    def __init__(self, handle, device=0):
        self.cuda_stream, self.device_index = handle, device


class Tensor:
    """A contiguous tensor on GPU 0: under which stream it was taken, and the other streams its release waits for."""

    def __init__(self, *shape, dtype=torch.bfloat16, owner=None):
        self.shape, self.dtype, self.owner, self.waits = torch.Size(shape), dtype, owner, []
        self.device, self.is_cuda = "cuda:0", True

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def get_device(self):
        return 0

    def data_ptr(self):
        return 0x1000

    def record_stream(self, stream):
        self.waits.append(stream)


class Library:
    """Every call succeeds, every workspace has 512 bytes."""

    def __getattr__(self, name):
        return lambda *a: 512 if name.endswith("_bytes") else pkg.ATTN_OK


class Pool(list):
    """The tensors taken so far; current: the current stream."""
    current = Stream(1)


@pytest.fixture
def pool(monkeypatch):
    pool = Pool()

    @contextlib.contextmanager
    def on(stream):
        before, pool.current = pool.current, stream
        yield
        pool.current = before

    def empty(*shape, dtype=None, device=None):
        shape = shape[0] if not isinstance(shape[0], int) else shape
        pool.append(Tensor(*shape, dtype=dtype, owner=pool.current))
        return pool[-1]

    cache._lib()  # (binds torch)
    monkeypatch.setattr(pkg, "_lib", Library())
    monkeypatch.setattr(pkg, "_raw_stream", lambda: pool.current.cuda_stream)
    monkeypatch.setattr(cache, "_bound", Library())
    monkeypatch.setattr(cache, "_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: pool.current)
    monkeypatch.setattr(torch, "empty", empty)
    return pool


Q, KV, P = Tensor(2, 4, 1, 64), Tensor(2, 2, 300, 64), Tensor(2, 200, 64)
LSE, ACC = Tensor(2, 4, 1, dtype=torch.float32), Tensor(2, 2, 300, dtype=torch.float32)
KW = dict(causal=True, scale=0.1)
# the calls, and how many of the tensors they take are their outputs (the first ones)
CALLS = {
    "attn_fwd_ex": (lambda s: pkg.attn_fwd_ex(Q, Q, Q, exp_mode=1, stream=s, **KW), 2),
    "attn_fwd_probe": (lambda s: pkg.attn_fwd_probe(Q, Q, Q, exp_mode=1, b=0, h=0, row0=0, nrows=1, stream=s, **KW), 5),
    "attn_decode": (lambda s: pkg.attn_decode(Q, KV, KV, exp_mode=1, split_keys=128, stream=s, **KW), 2),
    "attn_decode_noalloc": (lambda s: pkg.attn_decode_noalloc(Q, KV, KV, exp_mode=1, split_keys=128, stream=s, **KW), 2),
    "attn_decode_probe": (lambda s: pkg.attn_decode_probe(Q, KV, KV, exp_mode=1, split_keys=128, b=0, h=0, i=0, stream=s,
                                                          **KW), 5),
    "attn_decode_prefix": (lambda s: pkg.attn_decode_prefix(Q, P, P, KV, KV, exp_mode=1, prefix_split_keys=128,
                                                            split_keys=0, stream=s, **KW), 2),
    "attn_key_weights": (lambda s: pkg.attn_key_weights(Q, KV, LSE, ACC, stream=s, **KW), 0),
    "attn_evict": (lambda s: pkg.attn_evict(KV, KV, ACC, keep=20, recent=3, stream=s), 5),
}


@pytest.mark.parametrize("name", CALLS)
def test_memory_comes_from_the_stream_that_the_call_runs_on(pool, name):
    side = Stream(2)
    call, outputs = CALLS[name]
    got = call(side)
    assert len(pool) >= outputs and len(pool) > 0
    assert all(t.owner is side for t in pool)
    # the caller's stream has the outputs next: their release waits for what it does with them by then
    returned = [t for t in (got if isinstance(got, tuple) else (got,)) if t.owner is not None]
    assert len(returned) == outputs
    assert all(t.waits == [pool.current] for t in returned)


@pytest.mark.parametrize("name", CALLS)
def test_calls_on_the_current_stream_take_its_memory(pool, name):
    CALLS[name][0](None)
    assert len(pool) > 0 and all(t.owner is pool.current and t.waits == [] for t in pool)


# (as h15cache.h counts them, in 32 bits: a number beyond would come out as another one)
@pytest.mark.parametrize("name,call", [
    ("P", lambda x: pkg.attn_decode_prefix(Q, P, P, KV, KV, exp_mode=1, prefix_split_keys=0, split_keys=0, P=x, **KW)),
    ("Sk", lambda x: pkg.attn_decode_prefix(Q, P, P, KV, KV, exp_mode=1, prefix_split_keys=0, split_keys=0, Sk=x, **KW)),
    ("prefix_split_keys", lambda x: pkg.attn_decode_prefix(Q, P, P, KV, KV, exp_mode=1, prefix_split_keys=x, split_keys=0,
                                                           **KW)),
    ("split_keys", lambda x: pkg.attn_decode_prefix(Q, P, P, KV, KV, exp_mode=1, prefix_split_keys=0, split_keys=x, **KW)),
    ("Sk", lambda x: pkg.attn_key_weights(Q, KV, LSE, ACC, Sk=x, **KW)),
    ("Sk", lambda x: pkg.attn_evict(KV, KV, ACC, keep=20, recent=3, Sk=x)),
    ("keep", lambda x: pkg.attn_evict(KV, KV, ACC, keep=x, recent=3)),
    ("recent", lambda x: pkg.attn_evict(KV, KV, ACC, keep=20, recent=x)),
])
def test_sizes_beyond_32_bits_are_refused(pool, name, call):
    for x in (2 ** 31, 2 ** 32, 2 ** 32 + 128, -2 ** 31 - 1, -2 ** 32 + 5):
        with pytest.raises(ValueError, match=f"^{name} "):
            call(x)
    call(128)
    assert all(t.shape.numel() < 2 ** 31 for t in pool)


def test_attn_fwd_takes_its_outputs_where_it_runs(pool, monkeypatch):
    # on the default stream, whatever the current one is
    default = Stream(0)
    monkeypatch.setattr(torch.cuda, "default_stream", lambda *a: default)
    for t in pkg.attn_fwd(Q, Q, Q, exp_mode=1, **KW):
        assert t.owner is default and t.waits == [pool.current]
    pool.current = default
    assert all(t.owner is default for t in pkg.attn_fwd(Q, Q, Q, exp_mode=1, **KW))


@pytest.mark.parametrize("name", ["attn_decode_prefix", "attn_key_weights", "attn_evict"])
def test_streams_of_another_device_are_refused(pool, name):
    with pytest.raises(ValueError, match="stream must belong to GPU 0"):
        CALLS[name][0](Stream(3, device=1))
    assert not pool  # before anything is taken

"""The operators between a layer's projections and its attention
(``include/h15qkv.h``): norms of queries and keys with their position rotation,
its gradient, writing into a cache of 8-bit blocks, and attention over such a
cache.  The functions carry the C names and are reached as those of the
package; like them they raise and never compute anything another way.
"""
from __future__ import annotations

import ctypes
import math
import struct

from . import ATTN_BF16, ATTN_FP8_E4M3, ATTN_OK, AttnError, _dtype_of, _new, _outputs, cache, lib
from .cache import _current_gpu, _current_stream, _four, _lens_ptr, _refuse, _space, _tensor

ATTN_FP32 = 2  # type of norm weights, next to ATTN_BF16

# every symbol h15qkv.h declares
EXPORTS = ("attn_rope", "attn_rope_bwd", "attn_rope_bwd_workspace_bytes", "attn_cache_append", "attn_decode_blocks",
           "attn_decode_blocks_workspace_bytes", "attn_decode_blocks_split_keys")


class attn_rope_spec(ctypes.Structure):
    _fields_ = [("positions", ctypes.c_void_p), ("each_position", ctypes.c_int), ("freqs", ctypes.c_void_p),
                ("rot", ctypes.c_int), ("interleaved", ctypes.c_int), ("amplitude", ctypes.c_float),
                ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("weight_dtype", ctypes.c_int),
                ("eps", ctypes.c_float)]


_bound = None
_torch = None
_bf16 = _f32 = _f64 = _i32 = _fp8 = _e8m0 = None  # torch's types, bound with the library


def _lib() -> ctypes.CDLL:
    """The library with the argument types of these functions, bound on first use."""
    global _bound, _torch, _bf16, _f32, _f64, _i32, _fp8, _e8m0
    if _bound is not None:
        return _bound
    L = lib()
    P, I, F, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
    O = P  # (structures are given as the bytes that they consist of)
    for name, args, res in (
            ("attn_rope", [P] * 8 + [I] * 6 + [O], I),
            ("attn_rope_bwd", [P] * 13 + [I] * 5 + [P, S, O], I),
            ("attn_rope_bwd_workspace_bytes", [I] * 5, S),
            ("attn_cache_append", [P] * 8 + [I] * 6 + [O], I),
            ("attn_decode_blocks", [P] * 7 + [I] * 9 + [F, I, I, P, S, O], I),
            ("attn_decode_blocks_workspace_bytes", [I] * 6, S),
            ("attn_decode_blocks_split_keys", [I] * 6, I)):
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, res
    import torch
    _torch = torch
    _bf16, _f32, _f64, _i32, _fp8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.float8_e4m3fn
    _e8m0 = torch.float8_e8m0fnu
    cache._lib()  # (its checks use its own binding of torch)
    _bound = L
    return L


# ---- frequencies ------------------------------------------------------------

def attn_rope_frequencies(rot: int, base: float = 10000.0, *, scaling: str | None = None, factor: float = 1.0,
                          original: int | None = None, slow: float = 1.0, fast: float = 32.0, device=None):
    """(freqs, amplitude) for attn_rope: radians a position of each pair, float64 [rot / 2], and the factor of the
    rotated channels.

    Unscaled: f_j = base^(-2 j / rot), amplitude 1.  A context `factor` times as
    long as the `original` one that a model was trained for, by `scaling`:
      "linear"  f_j / factor: positions are interpolated;
      "base"    the base times factor^(rot / (rot - 2)): the slowest pair is
                interpolated, the fastest kept;
      "ramp"    f_j kept for pairs that turn more than `fast` times over the
                original context, divided by factor for those that turn less
                than `slow` times, and in between a mixture linear in the pair's
                index; amplitude 0.1 ln(factor) + 1;
      "smooth"  the same ends (usual: slow 1, fast 4), the mixture linear in the
                number of turns; amplitude 1."""
    import torch
    if rot <= 0 or rot % 2 or not base > 0:
        raise ValueError("rot must be even and positive, base positive")
    if scaling not in (None, "linear", "base", "ramp", "smooth") or not factor >= 1.0:
        raise ValueError("scaling must be None, 'linear', 'base', 'ramp' or 'smooth', factor 1 or more")
    if scaling == "base":
        if rot < 4:
            raise ValueError("scaling 'base' takes two pairs or more")
        base = base * factor ** (rot / (rot - 2))
    j = torch.arange(rot // 2, dtype=torch.float64)
    f = torch.pow(torch.tensor(float(base), dtype=torch.float64), -2.0 * j / rot)
    amplitude = 1.0
    if scaling == "linear":
        f = f / factor
    elif scaling in ("ramp", "smooth"):
        if original is None or original <= 0 or not 0 < slow < fast or not base > 1:
            raise ValueError(f"scaling '{scaling}' takes the original context's length, 0 < slow < fast, and a base above 1")
        turns = original * f / (2 * math.pi)
        if scaling == "smooth":
            keep = ((turns - slow) / (fast - slow)).clamp(0.0, 1.0)
        else:
            # the pair's index at which a pair turns `n` times: base^(-2 j / rot) original = 2 pi n
            at = lambda n: rot * math.log(original / (2 * math.pi * n)) / (2 * math.log(base))  # noqa: E731
            first, last = max(math.floor(at(fast)), 0), min(math.ceil(at(slow)), rot - 1)
            keep = 1.0 - ((j - first) / max(last - first, 1e-3)).clamp(0.0, 1.0)
            amplitude = 0.1 * math.log(factor) + 1.0
        f = f * keep + f / factor * (1.0 - keep)
    return f.to(device), amplitude


# ---- norms and rotation -------------------------------------------------------

# (The smallest calls are bound by these checks: a decode step's rotation of four
# chats takes the GPU 4 us.)
def _fresh(a, b, c, d, dtype, first, stream):
    """A new contiguous tensor [a,b,c,d], as _new makes it (given its strides, torch takes 1.3 us for it, else 1.6)."""
    if stream is not None:
        return _new((a, b, c, d), dtype, first.device, stream)
    return _torch.empty_strided((a, b, c, d), (b * c * d, c * d, d, 1), dtype=dtype, device=first.device)


def _strided(name, t, B, S, d, dev):
    """Heads and the three strides of a bf16 tensor [B,S,H,d] whose rows are contiguous."""
    shape = t.shape
    if len(shape) != 4 or t.dtype is not _bf16 or t.get_device() != dev:
        raise ValueError(f"{name} must be a bfloat16 tensor [{B}x{S}xHx{d}] on GPU {dev}")
    b, s, H, e = shape
    if b != B or s != S or e != d:
        raise ValueError(f"{name} must be a bfloat16 tensor [{B}x{S}xHx{d}] on GPU {dev}")
    sb, ss, sh, sd = t.stride()
    if sd != 1:
        raise ValueError(f"the rows of {name} must be contiguous")
    # (the stride of a dimension of one element says nothing)
    return H, sb if B > 1 else 0, ss if S > 1 else 0, sh if H > 1 else 0


def _apart(name, B, S, H, d, sb, ss, sh):
    """An output of these sizes and strides must not lie over itself: its dimensions, the smallest stride first, each
    beyond the ones before."""
    row = (H - 1) * sh + d
    if (sh >= d or H == 1) and (ss >= row or S == 1) and (sb >= (S - 1) * ss + row or B == 1):
        return  # batches outside positions outside heads
    end = d
    for stride, n in sorted(((sb, B), (ss, S), (sh, H))):
        if n > 1 and stride < end:
            raise ValueError(f"rows of {name} overlap")
        end += stride * (n - 1)


# Structures that a call reads before it returns, as their bytes: a third of the time of ctypes' own.
_pack_spec = struct.Struct("@PiPiifPPif").pack  # attn_rope_spec
_pack_strides = struct.Struct("@9q").pack  # attn_strides of three tensors
_pack_opts = struct.Struct("@fffPfi").pack  # attn_opts


def _opts(stream, descale=(1.0, 1.0, 1.0)):
    qd, kd, vd = descale
    return _pack_opts(qd, kd, vd, stream.cuda_stream if stream is not None else _current_stream(), 0.0, 0)


def _spec(B, S, d, dev, freqs, positions, interleaved, amplitude, q_weight, k_weight, eps):
    pptr = fptr = rot = each = 0
    if freqs is not None:
        rot = 2 * freqs.numel()
        if freqs.dtype is not _f64 or freqs.dim() != 1 or not freqs.is_contiguous() or freqs.get_device() != dev:
            _tensor("freqs", freqs, (rot // 2,), dev, _f64)
        fptr = freqs.data_ptr()
    if positions is not None:
        each = 1 if len(positions.shape) == 2 else 0
        pptr = _tensor("positions", positions, (B, S) if each else (B,), dev, _i32).data_ptr()
    wq = wk = 0
    wt = ATTN_BF16
    if q_weight is not None or k_weight is not None:
        kind = (k_weight if q_weight is None else q_weight).dtype
        if kind is not _bf16 and kind is not _f32 or k_weight is not None and k_weight.dtype is not kind:
            raise TypeError("q_weight and k_weight must be bfloat16, or both float32")
        if q_weight is not None:
            wq = _tensor("q_weight", q_weight, (d,), dev).data_ptr()
        if k_weight is not None:
            wk = _tensor("k_weight", k_weight, (d,), dev).data_ptr()
        wt = ATTN_FP32 if kind is _f32 else ATTN_BF16
    return _pack_spec(pptr, each, fptr, rot, 1 if interleaved else 0, amplitude, wq, wk, wt, eps)


def attn_rope(q, k=None, v=None, *, freqs=None, positions=None, interleaved: bool = False, amplitude: float = 1.0,
              q_weight=None, k_weight=None, eps: float = 1e-6, descale=None, out_dtype=None, q_out=None, k_out=None,
              v_out=None, stream=None):
    """Norms of queries and keys for each head, their position rotation, and the attention's layout (see
    include/h15qkv.h, attn_rope).

    q: [B,S,Hq,d], k, v: [B,S,Hkv,d] bf16, views of any strides (multiples of 8)
    with contiguous rows, such as parts of one projection's output; each may be
    None.  freqs: float64 [rot / 2] (attn_rope_frequencies; None: no rotation);
    positions: int32 [B,S], or [B]: those of the first rows (None: from 0).
    q_weight, k_weight: [d] bf16 or fp32 (None: no norm).  Returns (q_out
    [B,Hq,S,d], k_out, v_out [B,Hkv,S,d]): the given tensors, or new ones of
    out_dtype (bfloat16, the default, or float8_e4m3fn with descale = (q, k, v)
    factors, as attn_fwd_ex takes them).  torch records nothing of the call, as
    of the package's others: attn_rope_bwd is its gradient."""
    L = _lib()
    first = q if q is not None else k if k is not None else v
    if first is None:
        raise ValueError("q, k and v: one at least")
    dev = _current_gpu("q", first, stream)
    if len(first.shape) != 4:
        raise ValueError("q must be a 4-D tensor [B,S,H,d]")
    B, S, _, d = first.shape
    given = q_out if q_out is not None else k_out if k_out is not None else v_out
    dtype = given.dtype if given is not None else _bf16 if out_dtype is None else out_dtype
    if dtype is not _bf16 and dtype is not _fp8 or out_dtype is not None and out_dtype is not dtype:
        raise TypeError("attn_rope writes bfloat16 or float8_e4m3fn, all outputs the same")
    Hq = Hkv = a = b = c = e = f = g = h = i = j = 0
    qp = kp = vp = qo = ko = vo = None
    if q is not None:
        Hq, a, b, c = _strided("q", q, B, S, d, dev)
        qp = q.data_ptr()
        q_out = _fresh(B, Hq, S, d, dtype, first, stream) if q_out is None else \
            _tensor("q_out", q_out, (B, Hq, S, d), dev, dtype)
        qo = q_out.data_ptr()
    elif q_out is not None:
        raise ValueError("q_out without q")
    if k is not None:
        Hkv, e, f, g = _strided("k", k, B, S, d, dev)
        kp = k.data_ptr()
        k_out = _fresh(B, Hkv, S, d, dtype, first, stream) if k_out is None else \
            _tensor("k_out", k_out, (B, Hkv, S, d), dev, dtype)
        ko = k_out.data_ptr()
    elif k_out is not None:
        raise ValueError("k_out without k")
    if v is not None:
        n, h, i, j = _strided("v", v, B, S, d, dev)
        if k is not None and n != Hkv:
            raise ValueError("k and v must have the same heads")
        Hkv, vp = n, v.data_ptr()
        v_out = _fresh(B, Hkv, S, d, dtype, first, stream) if v_out is None else \
            _tensor("v_out", v_out, (B, Hkv, S, d), dev, dtype)
        vo = v_out.data_ptr()
    elif v_out is not None:
        raise ValueError("v_out without v")
    spec = _spec(B, S, d, dev, freqs, positions, interleaved, amplitude, q_weight, k_weight, eps)
    rc = L.attn_rope(qp, kp, vp, _pack_strides(a, b, c, e, f, g, h, i, j), spec, qo, ko, vo, B, S, Hq, Hkv, d,
                     ATTN_BF16 if dtype is _bf16 else ATTN_FP8_E4M3, _opts(stream) if descale is None else _opts(stream, descale))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_rope")
    return q_out, k_out, v_out


def attn_rope_bwd_workspace_bytes(B: int, S: int, Hq: int, Hkv: int, d: int) -> int:
    return int(_lib().attn_rope_bwd_workspace_bytes(int(B), int(S), int(Hq), int(Hkv), int(d)))


def _grad(gname, g, dname, out, B, S, d, dev, first, stream):
    """Heads of a gradient g [B,H,S,d], the tensor [B,S,H,d] for what it becomes, and that one's strides."""
    shape = g.shape
    if len(shape) != 4 or g.dtype is not _bf16 or not g.is_contiguous() or g.get_device() != dev:
        raise ValueError(f"{gname} must be a contiguous bfloat16 tensor [{B}xHx{S}x{d}] on GPU {dev}")
    b, H, s, e = shape
    if b != B or s != S or e != d:
        raise ValueError(f"{gname} must be a contiguous bfloat16 tensor [{B}xHx{S}x{d}] on GPU {dev}")
    if out is None:
        out = _fresh(B, S, H, d, _bf16, first, stream)
    n, sb, ss, sh = _strided(dname, out, B, S, d, dev)
    if n != H:
        raise ValueError(f"{dname} must have {gname}'s heads")
    _apart(dname, B, S, H, d, sb, ss, sh)
    return H, out, sb, ss, sh


def _with_weight(name, x, wname, dw, B, S, H, d, dev, first, stream):
    """The tensor for a weight's gradient, and the strides of the rows x that it takes."""
    if x is None:
        raise ValueError(f"{name} is required with {name}_weight")
    n, sb, ss, sh = _strided(name, x, B, S, d, dev)
    if n != H:
        raise ValueError(f"{name} must have g{name}'s heads")
    dw = _new((d,), _f32, first.device, stream) if dw is None else _tensor(wname, dw, (d,), dev, _f32)
    return dw, sb, ss, sh


def attn_rope_bwd(gq, gk=None, gv=None, *, q=None, k=None, freqs=None, positions=None, interleaved: bool = False,
                  amplitude: float = 1.0, q_weight=None, k_weight=None, eps: float = 1e-6, dq=None, dk=None, dv=None,
                  dq_weight=None, dk_weight=None, workspace=None, stream=None):
    """The gradient of attn_rope (see include/h15qkv.h, attn_rope_bwd).

    gq: [B,Hq,S,d], gk, gv: [B,Hkv,S,d] bf16, the gradients of attn_rope's
    outputs; each may be None.  q, k: its inputs, required with their weights.
    The other arguments are attn_rope's.  Returns (dq [B,S,Hq,d], dk, dv
    [B,S,Hkv,d] bf16, dq_weight, dk_weight [d] fp32 or None): the given tensors
    (dq, dk, dv may be views, such as parts of one gradient), or new ones."""
    L = _lib()
    first = gq if gq is not None else gk if gk is not None else gv
    if first is None:
        raise ValueError("gq, gk and gv: one at least")
    dev = _current_gpu("gq", first, stream)
    B, _, S, d = _four("gq", first)
    a = b = c = e = f = g = r = s = t = u = w = x = y = z = o = 0  # strides of q, k; dq, dk, dv
    qp = kp = qd = kd = vd = wqp = wkp = None
    Hq = Hkv = 0
    if gq is not None:
        Hq, dq, r, s, t = _grad("gq", gq, "dq", dq, B, S, d, dev, first, stream)
        if q_weight is not None:
            dq_weight, a, b, c = _with_weight("q", q, "dq_weight", dq_weight, B, S, Hq, d, dev, first, stream)
            qp, wqp = q.data_ptr(), dq_weight.data_ptr()
        elif dq_weight is not None:
            raise ValueError("dq_weight without q_weight")
        qd = dq.data_ptr()
    elif dq is not None or dq_weight is not None:
        raise ValueError("dq or dq_weight without gq")
    if gk is not None:
        Hkv, dk, u, w, x = _grad("gk", gk, "dk", dk, B, S, d, dev, first, stream)
        if k_weight is not None:
            dk_weight, e, f, g = _with_weight("k", k, "dk_weight", dk_weight, B, S, Hkv, d, dev, first, stream)
            kp, wkp = k.data_ptr(), dk_weight.data_ptr()
        elif dk_weight is not None:
            raise ValueError("dk_weight without k_weight")
        kd = dk.data_ptr()
    elif dk is not None or dk_weight is not None:
        raise ValueError("dk or dk_weight without gk")
    if gv is not None:
        n, dv, y, z, o = _grad("gv", gv, "dv", dv, B, S, d, dev, first, stream)
        if gk is not None and n != Hkv:
            raise ValueError("gk and gv must have the same heads")
        Hkv, vd = n, dv.data_ptr()
    elif dv is not None:
        raise ValueError("dv without gv")
    spec = _spec(B, S, d, dev, freqs, positions, interleaved, amplitude, q_weight, k_weight, eps)
    wptr = wbytes = 0
    if wqp is not None or wkp is not None:
        wptr, wbytes, workspace = _space(workspace, lambda: L.attn_rope_bwd_workspace_bytes(B, S, Hq, Hkv, d), dev,
                                         stream)
    rc = L.attn_rope_bwd(None if gq is None else gq.data_ptr(), None if gk is None else gk.data_ptr(),
                         None if gv is None else gv.data_ptr(), qp, kp, _pack_strides(a, b, c, e, f, g, 0, 0, 0), spec,
                         qd, kd, vd, _pack_strides(r, s, t, u, w, x, y, z, o), wqp, wkp, B, S, Hq, Hkv, d, wptr, wbytes,
                         _opts(stream))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_rope_bwd")
    return dq, dk, dv, dq_weight, dk_weight


# ---- a cache of 8-bit blocks ----------------------------------------------------

def _bf16_rows(name, t):
    """The sizes of a contiguous bf16 tensor [.,.,.,d]."""
    shape = _four(name, t)
    if t.dtype is not _bf16:
        raise ValueError(f"{name} must be a bfloat16 tensor")
    return shape


def _codes(name, t, B, Hkv, d, dev):
    """Rows of a cache of e4m3 codes [B,Hkv,rows,d]."""
    shape = t.shape
    if len(shape) != 4 or t.dtype is not _fp8 and _dtype_of(t) != ATTN_FP8_E4M3:
        raise TypeError(f"{name} must be a 4-D tensor of float8_e4m3fn")
    b, h, rows, e = shape
    if b != B or h != Hkv or e != d or not t.is_contiguous() or t.get_device() != dev:
        _tensor(name, t, (B, Hkv, rows, d), dev)
    return rows


def _scales(t, B, Hkv, cap, block, dev):
    if t.dtype is not _e8m0 and t.dtype is not _torch.uint8:
        raise TypeError("scales must be float8_e8m0fnu (or uint8, their bytes)")
    if not 0 < block < 2 ** 31:
        raise ValueError(f"block is out of range: {block}")
    return _tensor("scales", t, (B, Hkv, -(-cap // block), 2), dev).data_ptr()


def attn_cache_append(k, v, k_cache, v_cache, scales, lens, *, block: int, counts=None, lens_out=None, stream=None):
    """Write new keys and values into a cache of 8-bit blocks (see include/h15qkv.h, attn_cache_append).

    k, v: [B,Hkv,n,d] bf16; k_cache, v_cache: [B,Hkv,cap,d] float8_e4m3fn and
    scales: [B,Hkv,ceil(cap / block),2] float8_e8m0fnu (K's, V's), updated in
    place; lens: int32 [B], the slots filled before; counts: int32 [B], the new
    rows of each sequence, its first of the n (default n).  Returns lens_out,
    int32 [B], the slots filled after: the given tensor, which may be lens, or a
    new one.  attn_decode_blocks takes a padded batch's queries the other way
    round, behind their padding."""
    L = _lib()
    B, Hkv, n, d = shape = _bf16_rows("k", k)
    dev = _current_gpu("k", k, stream)
    _tensor("v", v, shape, dev, _bf16)
    cap = _codes("k_cache", k_cache, B, Hkv, d, dev)
    if _codes("v_cache", v_cache, B, Hkv, d, dev) != cap:
        raise ValueError("k_cache and v_cache must have the same rows")
    sptr = _scales(scales, B, Hkv, cap, block, dev)
    lptr = _tensor("lens", lens, (B,), dev, _i32).data_ptr()
    cptr = None if counts is None else _tensor("counts", counts, (B,), dev, _i32).data_ptr()
    lens_out = _new((B,), _i32, k.device, stream) if lens_out is None else \
        _tensor("lens_out", lens_out, (B,), dev, _i32)
    rc = L.attn_cache_append(k.data_ptr(), v.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), sptr, lptr, cptr,
                             lens_out.data_ptr(), B, Hkv, n, cap, d, block, _opts(stream))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_cache_append")
    return lens_out


def attn_decode_blocks_split_keys(B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d: int) -> int:
    """The library's proposed cut for attn_decode_blocks (0: one part)."""
    return int(_lib().attn_decode_blocks_split_keys(int(B), int(Hq), int(Hkv), int(Sq), int(Sk), int(d)))


def attn_decode_blocks_workspace_bytes(B: int, Hq: int, Sq: int, Sk: int, d: int, split_keys: int) -> int:
    return int(_lib().attn_decode_blocks_workspace_bytes(int(B), int(Hq), int(Sq), int(Sk), int(d), int(split_keys)))


def attn_decode_blocks(q, k, v, scales, *, block: int, causal: bool, scale: float, exp_mode: int, split_keys: int,
                       lens=None, Sk: int | None = None, stream=None, out=None, lse=None, want_lse: bool = True,
                       workspace=None):
    """Attention over a cache of 8-bit blocks (see include/h15qkv.h, attn_decode_blocks).

    q: [B,Hq,Sq,d] bf16; k, v: [B,Hkv,Sk_cap,d] float8_e4m3fn and scales:
    [B,Hkv,ceil(Sk_cap / block),2] float8_e8m0fnu, as attn_cache_append writes
    them, whose first lens[b] slots (int32 [B]; default Sk, default all) are
    filled.  When causal, a sequence's last query row sees its last key: of a
    batch appended with counts, a sequence's c = counts[b] queries are moved to
    its last c rows before (there the padding comes first), or it has a call of
    its own with Sq = c.  Returns (O [B,Hq,Sq,d] bf16, LSE [B,Hq,Sq] fp32 or
    None)."""
    L = _lib()
    B, Hq, Sq, d = shape = _bf16_rows("q", q)
    dev = _current_gpu("q", q, stream)
    Hkv = _four("k", k)[1]
    cap = _codes("k", k, B, Hkv, d, dev)
    if _codes("v", v, B, Hkv, d, dev) != cap:
        raise ValueError("k and v must have the same rows")
    sptr = _scales(scales, B, Hkv, cap, block, dev)
    Sk = cap if Sk is None else int(Sk)
    if (Sk | split_keys) >> 31:
        _refuse(Sk=Sk, split_keys=split_keys)
    if out is None or lse is None:
        out, lse = _outputs(q, out, lse, want_lse, stream)
    else:
        _tensor("out", out, shape, dev, _bf16)
        _tensor("lse", lse, shape[:3], dev, _f32)
    wptr, wbytes, workspace = _space(workspace, lambda: L.attn_decode_blocks_workspace_bytes(B, Hq, Sq, Sk, d,
                                                                                            split_keys), dev, stream)
    rc = L.attn_decode_blocks(q.data_ptr(), k.data_ptr(), v.data_ptr(), sptr, _lens_ptr(lens, B, dev), out.data_ptr(),
                              lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, Sk, cap, d, block,
                              1 if causal else 0, scale, exp_mode, split_keys, wptr, wbytes, _opts(stream))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_decode_blocks")
    return out, lse

"""The operators for serving with shared and bounded key/value caches
(``include/h15cache.h``): decode over a shared prefix, the attention weight of
each cached key, and eviction.  The functions carry the C names and are
reached as those of the package; like them they raise and never compute
anything another way.
"""
from __future__ import annotations

import ctypes

from . import ATTN_OK, AttnError, _current_stream, _dtype_of, _new, _new_workspace, _outputs, attn_opts, lib

# every symbol h15cache.h declares
EXPORTS = ("attn_decode_prefix", "attn_decode_prefix_workspace_bytes", "attn_decode_prefix_split_keys",
           "attn_key_weights", "attn_key_weights_workspace_bytes", "attn_evict", "attn_evict_workspace_bytes")

_bound = None
_device = None  # the number of the current device
_torch = None


def _lib() -> ctypes.CDLL:
    """The library with the argument types of these functions (bound on first
    use, so that a build of the h15attn.h entry points alone still loads)."""
    global _bound, _device, _torch
    if _bound is not None:
        return _bound
    L = lib()
    P, I, F, S, O = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(attn_opts)
    IP = ctypes.POINTER(ctypes.c_int)
    for name, args, res in (
            ("attn_decode_prefix", [P] * 8 + [I] * 10 + [F] + [I] * 4 + [P, S, O], I),
            ("attn_decode_prefix_workspace_bytes", [I] * 8, S),
            ("attn_decode_prefix_split_keys", [I] * 8 + [IP, IP], I),
            ("attn_key_weights", [P] * 5 + [I] * 8 + [F, F, I, P, S, O], I),
            ("attn_key_weights_workspace_bytes", [I] * 6, S),
            ("attn_evict", [P] * 9 + [I] * 9 + [P, S, O], I),
            ("attn_evict_workspace_bytes", [I] * 3, S)):
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, res
    import torch
    _torch = torch
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _bound = L
    return L


# Checks are on the path of every call, and the smallest calls are bound by it:
# shapes are compared whole and devices by number, and the workspace of a caller
# who gives one is sized by the library alone.
def _tensor(name, t, shape, dev, dtype=None):
    """A contiguous tensor of this shape on device number dev."""
    if t.shape != shape or not t.is_contiguous() or t.get_device() != dev or (dtype is not None and t.dtype != dtype):
        want = "x".join(map(str, shape))
        raise ValueError(f"{name} must be a contiguous tensor [{want}]{f' of {dtype}' if dtype else ''} on "
                         f"{f'GPU {dev}' if dev >= 0 else 'the host'}")
    return t


def _operand(name, t, shape, dev, first, dt):
    """A tensor as _tensor, of the operand type dt that the first operand has."""
    _tensor(name, t, shape, dev)
    if t.dtype != first and _dtype_of(t) != dt:
        raise TypeError(f"{name} and the first operand must share one operand type")
    return t


def _current_gpu(name, t, stream) -> int:
    """The number of t's device, which has to be the current one, and the stream's, if one is given."""
    dev = t.get_device()
    if dev < 0 or dev != _device():
        raise ValueError(f"{name} must be on the current GPU")
    if stream is not None and stream.device_index != dev:
        raise ValueError(f"stream must belong to GPU {dev}")
    return dev


def _four(name, t):
    shape = t.shape
    if len(shape) != 4 or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous 4-D device tensor")
    return shape


def _cache(name, t, B, d, dev, first, dt):
    """KV heads and rows of a cache [B,Hkv,rows,d] on device number dev, of the first operand's type."""
    shape = t.shape
    if len(shape) != 4 or shape[0] != B or shape[3] != d or not t.is_contiguous() or t.get_device() != dev:
        _tensor(name, t, (B, *shape[1:3], d), dev)
    if t.dtype != first and _dtype_of(t) != dt:
        raise TypeError(f"{name} and the first operand must share one operand type")
    return shape[1], shape[2]


def _call_opts(descale, stream):
    handle = stream.cuda_stream if stream is not None else _current_stream()
    if descale is None:
        return attn_opts(1.0, 1.0, 1.0, handle, 0.0, 0)
    qd, kd, vd = descale
    return attn_opts(float(qd), float(kd), float(vd), handle, 0.0, 0)


def _refuse(**sizes):
    """Sizes go to the library in 32 bits, and ctypes cuts off what lies beyond (negative ones the library refuses)."""
    for name, n in sizes.items():
        if not -2 ** 31 <= n < 2 ** 31:
            raise ValueError(f"{name} is out of range: {n}")


def _lens_ptr(lens, B, dev):
    return None if lens is None else _tensor("lens", lens, (B,), dev, _torch.int32).data_ptr()


def _space(workspace, need, dev, stream):
    """Pointer and size of the caller's workspace, or of a new one of need() bytes, which comes third."""
    if workspace is None:
        n = need()
        if not n:
            return None, 0, None
        workspace = _new_workspace(n, f"cuda:{dev}", stream)
        return workspace.data_ptr(), n, workspace
    if not workspace.is_contiguous() or workspace.get_device() != dev:
        raise ValueError(f"workspace must be a contiguous tensor on GPU {dev}")
    return workspace.data_ptr(), workspace.numel() * workspace.element_size(), workspace


def attn_decode_prefix_split_keys(B: int, Hq: int, Hkv: int, Sq: int, P: int, Sk: int, d: int,
                                  dtype: int) -> tuple[int, int]:
    """The library's proposed cuts (prefix_split_keys, split_keys) for attn_decode_prefix."""
    a, b = ctypes.c_int(0), ctypes.c_int(0)
    _lib().attn_decode_prefix_split_keys(int(B), int(Hq), int(Hkv), int(Sq), int(P), int(Sk), int(d), int(dtype),
                                         ctypes.byref(a), ctypes.byref(b))
    return a.value, b.value


def attn_decode_prefix_workspace_bytes(B: int, Hq: int, Sq: int, P: int, Sk: int, d: int, prefix_split_keys: int,
                                       split_keys: int) -> int:
    return int(_lib().attn_decode_prefix_workspace_bytes(int(B), int(Hq), int(Sq), int(P), int(Sk), int(d),
                                                         int(prefix_split_keys), int(split_keys)))


def attn_decode_prefix(q, kp, vp, k, v, *, causal: bool, scale: float, exp_mode: int, prefix_split_keys: int,
                       split_keys: int, lens=None, P: int | None = None, Sk: int | None = None, descale=None,
                       stream=None, out=None, lse=None, want_lse: bool = True, workspace=None):
    """Decode for a batch that shares a prefix (see include/h15cache.h, attn_decode_prefix).

    q: [B,Hq,Sq,d]; kp, vp: [Hkv,P_cap,d] whose first P rows (default all) are
    the prefix, or None for none; k, v: [B,Hkv,Sk_cap,d] the own caches, whose
    first lens[b] rows (int32 [B]; default Sk, default all) are filled, or None
    for none.  Returns (O [B,Hq,Sq,d] bf16, LSE [B,Hq,Sq] fp32 or None)."""
    L = _lib()
    if (k is None) != (v is None) or (kp is None) != (vp is None):
        raise ValueError("k and v, kp and vp: both or neither")
    B, Hq, Sq, d = shape = _four("q", q)
    dev, first = _current_gpu("q", q, stream), q.dtype
    dt = _dtype_of(q)
    Hkv = P_cap = Sk_cap = 0
    kptr = vptr = kpptr = vpptr = None
    if k is not None:
        Hkv, Sk_cap = _cache("k", k, B, d, dev, first, dt)
        kptr = k.data_ptr()
        vptr = _operand("v", v, k.shape, dev, first, dt).data_ptr()
    if kp is not None:
        if k is None:
            Hkv = kp.shape[0]
        P_cap = kp.shape[1] if len(kp.shape) > 1 else 0
        shape = (Hkv, P_cap, d)
        kpptr = _operand("kp", kp, shape, dev, first, dt).data_ptr()
        vpptr = _operand("vp", vp, shape, dev, first, dt).data_ptr()
    P = P_cap if P is None else int(P)
    Sk = Sk_cap if Sk is None else int(Sk)
    if (P | Sk | prefix_split_keys | split_keys) >> 31:
        _refuse(P=P, Sk=Sk, prefix_split_keys=prefix_split_keys, split_keys=split_keys)
    if out is None or lse is None:
        out, lse = _outputs(q, out, lse, want_lse, stream)
    else:
        _tensor("out", out, q.shape, dev, _torch.bfloat16)
        _tensor("lse", lse, q.shape[:3], dev, _torch.float32)
    wptr, wbytes, workspace = _space(workspace, lambda: L.attn_decode_prefix_workspace_bytes(
        B, Hq, Sq, P, Sk, d, prefix_split_keys, split_keys), dev, stream)
    opts = _call_opts(descale, stream)
    rc = L.attn_decode_prefix(q.data_ptr(), kpptr, vpptr, kptr, vptr, _lens_ptr(lens, B, dev), out.data_ptr(),
                              lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, P, P_cap, Sk, Sk_cap, d,
                              1 if causal else 0, scale, dt, exp_mode, prefix_split_keys, split_keys, wptr, wbytes,
                              ctypes.byref(opts))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_decode_prefix")
    return out, lse


def attn_key_weights_workspace_bytes(B: int, Hq: int, Hkv: int, Sq: int, Sk: int, d: int) -> int:
    return int(_lib().attn_key_weights_workspace_bytes(int(B), int(Hq), int(Hkv), int(Sq), int(Sk), int(d)))


def attn_key_weights(q, k, lse, acc, *, causal: bool, scale: float, decay: float = 1.0, lens=None,
                     Sk: int | None = None, descale=None, stream=None, workspace=None):
    """Add to acc the attention weight that each cached key received (see include/h15cache.h, attn_key_weights).

    q: [B,Hq,Sq,d]; k: [B,Hkv,Sk_cap,d]; lse: [B,Hq,Sq] fp32 as the attention
    call over q returned it; acc: [B,Hkv,Sk_cap] fp32, updated in place and
    returned.  descale: (q, k) or (q, k, v) factors of FP8 operands."""
    L = _lib()
    B, Hq, Sq, d = shape = _four("q", q)
    dev = _current_gpu("q", q, stream)
    dt = _dtype_of(q)
    Hkv, cap = _cache("k", k, B, d, dev, q.dtype, dt)
    _tensor("lse", lse, (B, Hq, Sq), dev, _torch.float32)
    _tensor("acc", acc, (B, Hkv, cap), dev, _torch.float32)
    Sk = cap if Sk is None else int(Sk)
    if Sk >> 31:
        _refuse(Sk=Sk)
    wptr, wbytes, workspace = _space(workspace, lambda: L.attn_key_weights_workspace_bytes(B, Hq, Hkv, Sq, Sk, d), dev,
                                     stream)
    if descale is not None:
        descale = (descale[0], descale[1], 1.0)
    opts = _call_opts(descale, stream)
    rc = L.attn_key_weights(q.data_ptr(), k.data_ptr(), lse.data_ptr(), _lens_ptr(lens, B, dev), acc.data_ptr(), B,
                            Hq, Hkv, Sq, Sk, cap, d, 1 if causal else 0, scale, decay, dt, wptr, wbytes,
                            ctypes.byref(opts))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_key_weights")
    return acc


def attn_evict_workspace_bytes(B: int, Hkv: int, Sk: int) -> int:
    return int(_lib().attn_evict_workspace_bytes(int(B), int(Hkv), int(Sk)))


def attn_evict(k, v, acc, *, keep: int, recent: int, lens=None, Sk: int | None = None, stream=None, k_out=None,
               v_out=None, acc_out=None, index=None, lens_out=None, workspace=None):
    """Keep min(lens[b], keep) keys of every cache, the last `recent` and those with the largest acc (see
    include/h15cache.h, attn_evict).

    k, v: [B,Hkv,Sk_cap,d]; acc: [B,Hkv,Sk_cap] fp32.  Returns (k_out, v_out
    [B,Hkv,out_cap,d], acc_out [B,Hkv,out_cap], index [B,Hkv,keep] int32,
    lens_out [B] int32): the given tensors, or new ones with out_cap = keep.
    Rows of the outputs from lens_out[b] on are left as they were."""
    L = _lib()
    B, Hkv, cap, d = shape = _four("k", k)
    dev, first, f32, i32 = _current_gpu("k", k, stream), k.dtype, _torch.float32, _torch.int32
    dt = _dtype_of(k)
    _operand("v", v, shape, dev, first, dt)
    _tensor("acc", acc, (B, Hkv, cap), dev, f32)
    Sk, keep, recent = cap if Sk is None else int(Sk), int(keep), int(recent)
    if (Sk | keep | recent) >> 31:
        _refuse(Sk=Sk, keep=keep, recent=recent)
    rows = max(keep, 1)
    given = k_out if k_out is not None else v_out
    out_cap = rows if given is None else _four("k_out", given)[2]
    shape = (B, Hkv, out_cap, d)
    new = lambda size, dtype: _new(size, dtype, k.device, stream)  # noqa: E731
    k_out = new(shape, first) if k_out is None else _operand("k_out", k_out, shape, dev, first, dt)
    v_out = new(shape, first) if v_out is None else _operand("v_out", v_out, shape, dev, first, dt)
    shape = (B, Hkv, out_cap)
    acc_out = new(shape, f32) if acc_out is None else _tensor("acc_out", acc_out, shape, dev, f32)
    shape = (B, Hkv, rows)
    index = new(shape, i32) if index is None else _tensor("index", index, shape, dev, i32)
    lens_out = new((B,), i32) if lens_out is None else _tensor("lens_out", lens_out, (B,), dev, i32)
    wptr, wbytes, workspace = _space(workspace, lambda: L.attn_evict_workspace_bytes(B, Hkv, Sk), dev, stream)
    opts = _call_opts(None, stream)
    rc = L.attn_evict(k.data_ptr(), v.data_ptr(), acc.data_ptr(), _lens_ptr(lens, B, dev), k_out.data_ptr(),
                      v_out.data_ptr(), acc_out.data_ptr(), index.data_ptr(), lens_out.data_ptr(), B, Hkv, Sk, cap,
                      out_cap, d, keep, recent, dt, wptr, wbytes, ctypes.byref(opts))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_evict")
    return k_out, v_out, acc_out, index, lens_out

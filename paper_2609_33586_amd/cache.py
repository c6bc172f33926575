"""The operators for serving with shared and bounded key/value caches
(``include/h15cache.h``): decode over a shared prefix, the attention weight of
each cached key, and eviction.  The functions carry the C names and are
reached as those of the package; like them they raise and never compute
anything another way.
"""
from __future__ import annotations

import ctypes

from . import ATTN_OK, AttnError, _dtype_of, _opts, _outputs, attn_opts, lib

# every symbol h15cache.h declares
EXPORTS = ("attn_decode_prefix", "attn_decode_prefix_workspace_bytes", "attn_decode_prefix_split_keys",
           "attn_key_weights", "attn_key_weights_workspace_bytes", "attn_evict")

_bound = None
_device = None


def _lib() -> ctypes.CDLL:
    """The library with the argument types of these functions (bound on first
    use, so that a build of the h15attn.h entry points alone still loads)."""
    global _bound, _device
    L = lib()
    if _bound is L:
        return L
    P, I, F, S, O = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(attn_opts)
    IP = ctypes.POINTER(ctypes.c_int)
    for name, args, res in (
            ("attn_decode_prefix", [P] * 8 + [I] * 10 + [F] + [I] * 4 + [P, S, O], I),
            ("attn_decode_prefix_workspace_bytes", [I] * 8, S),
            ("attn_decode_prefix_split_keys", [I] * 8 + [IP, IP], I),
            ("attn_key_weights", [P] * 5 + [I] * 8 + [F, F, I, P, S, O], I),
            ("attn_key_weights_workspace_bytes", [I] * 6, S),
            ("attn_evict", [P] * 9 + [I] * 9 + [O], I)):
        fn = getattr(L, name)
        fn.argtypes, fn.restype = args, res
    import torch
    _device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    _bound = L
    return L


def _tensor(name, t, shape, device, dtype=None):
    """A contiguous tensor of this shape (None: any size) on the device."""
    if t.device != device or not t.is_contiguous() or (dtype is not None and t.dtype != dtype) \
            or len(t.shape) != len(shape) or any(w is not None and s != w for s, w in zip(t.shape, shape)):
        want = "x".join("?" if w is None else str(w) for w in shape)
        raise ValueError(f"{name} must be a contiguous tensor [{want}]{f' of {dtype}' if dtype else ''} on {device}")
    return t


def _on_current_device(t, name):
    if not t.is_cuda or t.get_device() != _device():
        raise ValueError(f"{name} must be on the current GPU")
    return t.device


def _lens_ptr(lens, B, device):
    if lens is None:
        return None
    import torch
    return _tensor("lens", lens, (B,), device, torch.int32).data_ptr()


def _space(workspace, need, device, stream):
    """The caller's workspace or a new one, its pointer and size."""
    if workspace is None:
        if not need:
            return None, None, 0
        import torch
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        if stream is not None:
            workspace.record_stream(stream)  # it is let go before the work on that stream is done
    elif not workspace.is_contiguous() or workspace.device != device:
        raise ValueError(f"workspace must be a contiguous tensor on {device}")
    return workspace, workspace.data_ptr(), workspace.numel() * workspace.element_size()


def _same_type(dt, **tensors):
    for t in tensors.values():
        if _dtype_of(t) != dt:
            raise TypeError(f"{', '.join(tensors)} and the first operand must share one operand type")


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
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous 4-D device tensor [B,Hq,Sq,d]")
    dev = _on_current_device(q, "q")
    B, Hq, Sq, d = q.shape
    dt = _dtype_of(q)
    Hkv = kp.shape[0] if kp is not None else k.shape[1] if k is not None else 0
    P_cap = Sk_cap = 0
    if kp is not None:
        P_cap = kp.shape[1]
        _tensor("kp", kp, (Hkv, P_cap, d), dev)
        _tensor("vp", vp, (Hkv, P_cap, d), dev)
        _same_type(dt, kp=kp, vp=vp)
    if k is not None:
        Sk_cap = k.shape[2]
        _tensor("k", k, (B, Hkv, Sk_cap, d), dev)
        _tensor("v", v, (B, Hkv, Sk_cap, d), dev)
        _same_type(dt, k=k, v=v)
    P = P_cap if P is None else int(P)
    Sk = Sk_cap if Sk is None else int(Sk)
    out, lse = _outputs(q, out, lse, want_lse)
    need = L.attn_decode_prefix_workspace_bytes(B, Hq, Sq, P, Sk, d, prefix_split_keys, split_keys)
    ws, wptr, wbytes = _space(workspace, need, dev, stream)
    opts = _opts(descale, stream)
    rc = L.attn_decode_prefix(q.data_ptr(), kp.data_ptr() if kp is not None else None,
                              vp.data_ptr() if kp is not None else None, k.data_ptr() if k is not None else None,
                              v.data_ptr() if k is not None else None, _lens_ptr(lens, B, dev), out.data_ptr(),
                              lse.data_ptr() if lse is not None else None, B, Hq, Hkv, Sq, P, P_cap, Sk, Sk_cap, d,
                              int(bool(causal)), float(scale), dt, int(exp_mode), int(prefix_split_keys),
                              int(split_keys), wptr, wbytes, ctypes.byref(opts))
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
    import torch
    L = _lib()
    if q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous 4-D device tensor [B,Hq,Sq,d]")
    dev = _on_current_device(q, "q")
    B, Hq, Sq, d = q.shape
    dt = _dtype_of(q)
    _tensor("k", k, (B, None, None, d), dev)
    _same_type(dt, k=k)
    Hkv, cap = k.shape[1], k.shape[2]
    _tensor("lse", lse, (B, Hq, Sq), dev, torch.float32)
    _tensor("acc", acc, (B, Hkv, cap), dev, torch.float32)
    Sk = cap if Sk is None else int(Sk)
    need = L.attn_key_weights_workspace_bytes(B, Hq, Hkv, Sq, Sk, d)
    ws, wptr, wbytes = _space(workspace, need, dev, stream)
    if descale is not None:
        descale = (descale[0], descale[1], 1.0)
    opts = _opts(descale, stream)
    rc = L.attn_key_weights(q.data_ptr(), k.data_ptr(), lse.data_ptr(), _lens_ptr(lens, B, dev), acc.data_ptr(), B,
                            Hq, Hkv, Sq, Sk, cap, d, int(bool(causal)), float(scale), float(decay), dt, wptr, wbytes,
                            ctypes.byref(opts))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_key_weights")
    return acc


def attn_evict(k, v, acc, *, keep: int, recent: int, lens=None, Sk: int | None = None, stream=None, k_out=None,
               v_out=None, acc_out=None, index=None, lens_out=None):
    """Keep min(lens[b], keep) keys of every cache, the last `recent` and those with the largest acc (see
    include/h15cache.h, attn_evict).

    k, v: [B,Hkv,Sk_cap,d]; acc: [B,Hkv,Sk_cap] fp32.  Returns (k_out, v_out
    [B,Hkv,out_cap,d], acc_out [B,Hkv,out_cap], index [B,Hkv,keep] int32,
    lens_out [B] int32): the given tensors, or new ones with out_cap = keep.
    Rows of the outputs from lens_out[b] on are left as they were."""
    import torch
    L = _lib()
    dev = _on_current_device(k, "k")
    if k.dim() != 4:
        raise ValueError("k must be a contiguous 4-D device tensor [B,Hkv,Sk_cap,d]")
    B, Hkv, cap, d = k.shape
    dt = _dtype_of(k)
    _tensor("k", k, (B, Hkv, cap, d), dev)
    _tensor("v", v, (B, Hkv, cap, d), dev)
    _same_type(dt, v=v)
    _tensor("acc", acc, (B, Hkv, cap), dev, torch.float32)
    Sk, keep = cap if Sk is None else int(Sk), int(keep)
    rows = max(keep, 1)
    if k_out is None:
        k_out = torch.empty((B, Hkv, v_out.shape[2] if v_out is not None else rows, d), dtype=k.dtype, device=dev)
    if k_out.dim() != 4:
        raise ValueError("k_out must be a contiguous 4-D device tensor [B,Hkv,out_cap,d]")
    out_cap = k_out.shape[2]
    if v_out is None:
        v_out = torch.empty((B, Hkv, out_cap, d), dtype=v.dtype, device=dev)
    if acc_out is None:
        acc_out = torch.empty((B, Hkv, out_cap), dtype=torch.float32, device=dev)
    if index is None:
        index = torch.empty((B, Hkv, rows), dtype=torch.int32, device=dev)
    if lens_out is None:
        lens_out = torch.empty(B, dtype=torch.int32, device=dev)
    _tensor("k_out", k_out, (B, Hkv, out_cap, d), dev)
    _tensor("v_out", v_out, (B, Hkv, out_cap, d), dev)
    _same_type(dt, k_out=k_out, v_out=v_out)
    _tensor("acc_out", acc_out, (B, Hkv, out_cap), dev, torch.float32)
    _tensor("index", index, (B, Hkv, rows), dev, torch.int32)
    _tensor("lens_out", lens_out, (B,), dev, torch.int32)
    opts = _opts(None, stream)
    rc = L.attn_evict(k.data_ptr(), v.data_ptr(), acc.data_ptr(), _lens_ptr(lens, B, dev), k_out.data_ptr(),
                      v_out.data_ptr(), acc_out.data_ptr(), index.data_ptr(), lens_out.data_ptr(), B, Hkv, Sk, cap,
                      out_cap, d, keep, int(recent), dt, ctypes.byref(opts))
    if rc != ATTN_OK:
        raise AttnError(rc, "attn_evict")
    return k_out, v_out, acc_out, index, lens_out

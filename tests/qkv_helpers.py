"""Plain float64 forms of the operators between projections and attention, and
the tolerances that follow from the kernels' arithmetic.

Rounding: half a step of BF16 is 2^-8 of a value, of e4m3 2^-4 (2^-10 below its
least normal value 2^-6), of FP32 2^-24.

A rotation: the sine and cosine instructions are off by 1.3e-7 (2^-22.8), the
angle's last rounding by 2^-26 of a turn (2^-23.3 radians), the amplitude and the
two products by 2^-24 each: 2^-21 of |y_a| + |y_b|.  Far positions add the FP64
product's 2^-52 of the angle on either side.  A norm: 16 squares in four chains
and four sums of lanes, halved by the root, whose instruction is off by 2^-23,
and two products: 2^-21 of the value."""
import math

import torch

import paper_2609_33586_amd as pkg
from cache_helpers import BF16, EXACT, FP8, H15, SQ4, SQ8, check_prefix, prefix_ref, say, scale_of, visible  # noqa: F401

E8M0 = torch.float8_e8m0fnu


def normal(shape, seed, dtype=BF16, device="cuda"):
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    return torch.randn(*shape, generator=gen, device=device).to(dtype)


def projection(B, S, Hq, Hkv, d, seed):
    """Queries, keys and values as views of one projection's output, some channels large."""
    x = normal((B, S, Hq + 2 * Hkv, d), seed, torch.float32)
    x[..., ::11] *= 6
    return x.to(BF16).split([Hq, Hkv, Hkv], 2)


def large_rows(B, S, H, d, seed):
    """Rows of sizes from 2^50 to the type's largest, ordinary ones among them, one of a single large channel, one whose
    channels are all the largest value; zeros and channels far below the others in between."""
    top = torch.finfo(BF16).max
    x = normal((B, S, H, d), seed, torch.float32).double()
    e = torch.tensor([0, 50, 61, 64, 66, 90, 100, 126], dtype=torch.float64, device="cuda")
    x = x * torch.exp2(e[torch.arange(S, device="cuda") % 8])[:, None, None]
    x[:, 9], x[:, 9, :, 17] = x[:, 9] * 2.0 ** -61, 1e20
    x[:, 10] = torch.where(x[:, 10] < 0, -top, top)
    x[:, 11, :, ::3], x[:, 12, :, 1::2] = 0.0, x[:, 12, :, 1::2] * 2.0 ** -90
    return x.clamp(-top, top).to(BF16)


def angles(freqs, positions, B, S):
    """[B, S, 1, rot / 2] in float64."""
    at = torch.arange(S, device=freqs.device, dtype=torch.float64)
    if positions is None:
        p = at.expand(B, S)
    elif positions.dim() == 1:
        p = positions.double()[:, None] + at
    else:
        p = positions.double()
    return p[:, :, None, None] * freqs


def pairs(x, rot, inter):
    r = x[..., :rot]
    return (r[..., 0::2], r[..., 1::2]) if inter else (r[..., :rot // 2], r[..., rot // 2:])


def joined(x, rot, inter, a, b):
    out = x.clone()
    if inter:
        out[..., 0:rot:2], out[..., 1:rot:2] = a, b
    else:
        out[..., :rot // 2], out[..., rot // 2:rot] = a, b
    return out


def turned(x, t, rot, inter, amplitude, back=False):
    """The rotation of [B, S, H, d] and, in each channel, |a| + |b| of its pair times the amplitude (|x| elsewhere)."""
    if not rot:
        return x, x.abs()
    a, b = pairs(x, rot, inter)
    c, s = t.cos() * amplitude, t.sin() * (-amplitude if back else amplitude)
    m = (a.abs() + b.abs()) * amplitude
    return joined(x, rot, inter, a * c - b * s, b * c + a * s), joined(x.abs(), rot, inter, m, m)


def inverse_rms(x, eps):
    return 1.0 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)


def far(t):
    """What FP64 angles may be off by, on either side, relative to the pair: [B, S, 1, 1]."""
    return 2 * 2.0 ** -52 * t.abs().amax(-1, keepdim=True) if t is not None and t.numel() else 0.0


def rope_ref(x, w, freqs, positions, inter, amplitude, eps):
    """attn_rope of one tensor [B, S, H, d] in float64, as [B, H, S, d], and its tolerance before the last rounding."""
    B, S = x.shape[:2]
    x = x.double()
    rot = 0 if freqs is None else 2 * freqs.numel()
    t = angles(freqs, positions, B, S) if rot else None
    if w is not None:
        x = x * inverse_rms(x, eps) * w.double()
    z, m = turned(x, t, rot, inter, amplitude)
    tol = m * (2.0 ** -21 + far(t) + (2.0 ** -21 if w is not None else 0.0))
    return z.transpose(1, 2), tol.transpose(1, 2)


def bf16_tolerance(z, tol):
    return 2.0 ** -8 * z.abs() + 2 * tol + 2.0 ** -133


def check(got, want, tol, what):
    bad = (got.double() - want).abs()
    assert bool(torch.isfinite(got.double()).all()), f"{what}: not finite"
    say(f"{what}: max error / tolerance {(bad / tol).max().item():.3f}")
    assert bool((bad <= tol).all()), what


def grad_ref(g, x, w, freqs, positions, inter, amplitude, eps):
    """The gradients of one tensor: dx [B, S, H, d] and dweight (or None), each with its tolerance."""
    g = g.double().transpose(1, 2)  # [B, S, H, d]
    B, S = g.shape[:2]
    rot = 0 if freqs is None else 2 * freqs.numel()
    t = angles(freqs, positions, B, S) if rot else None
    h, m = turned(g, t, rot, inter, amplitude, back=True)
    rel = 2.0 ** -21 + far(t)
    if w is None:
        return h, 2.0 ** -8 * h.abs() + 2 * m * rel + 2.0 ** -133, None, None
    x, w = x.double(), w.double()
    r = inverse_rms(x, eps)
    u = x * r
    e, me = h * w, m * w.abs()
    mean = (e * u).mean(-1, keepdim=True)
    dx = r * (e - u * mean)
    # u is off by 2^-21, e by rel of the pair's, their mean by both and 24 sums, and then four roundings
    size = r * (me + u.abs() * (me * u.abs()).mean(-1, keepdim=True))
    tol = 2.0 ** -8 * dx.abs() + 2 * size * (rel + 2.0 ** -19) + 2.0 ** -133
    terms = (m * u.abs()).sum((0, 1, 2))
    # a thread's chain of terms, the workgroup's 64 threads of a channel, the workgroups' parts
    rows = B * S * g.shape[2]
    chain = min(rows, 8 * 64) + 64 + rows / 32 / 32 + 32
    return dx, tol, (h * u).sum((0, 1, 2)), terms * (rel + 2.0 ** -20 + chain * 2.0 ** -24) + 1e-30


# ---- caches of 8-bit blocks -----------------------------------------------------

def power(e):
    """2^(e - 127) in float64 of exponent bytes (0 counts as 1, 255 as 254)."""
    return torch.exp2(e.clamp(1, 254).double() - 127)


def e4m3(x):
    """The nearest e4m3 value, ties to even, of numbers held to +-448, in float64 (NaN stays)."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(2.0 ** -6, 448))) - 3)
    return (torch.round(x / step) * step).clamp(-448, 448)


def append_ref(x, cache, scales, lens, counts, cap, block):
    """One tensor's cache (as numbers) and scale bytes after an append, from the definition."""
    out, scales = cache.double(), scales.int()
    B, n = x.shape[0], x.shape[2]
    after = []
    for b in range(B):
        held = min(max(lens[b], 0), cap)
        end = min(held + (n if counts is None else min(max(counts[b], 0), n)), cap)
        after.append(end)
        for first in range(held // block * block, end, block):
            lo, hi = max(first, held), min(first + block, end)
            if lo >= hi:
                continue
            rows = x[b, :, lo - held:hi - held].double()
            top = torch.where(rows.isfinite(), rows.abs(), 0.0).amax((-1, -2))
            need = torch.ceil(torch.log2(top.clamp(min=448 * 2.0 ** -126) / 448.0)) + 127
            if lo > first:
                was = scales[b, :, first // block].clamp(1, 254).double()
                need = torch.maximum(need, was)
                out[b, :, first:lo] = e4m3(out[b, :, first:lo] * torch.exp2(was - need)[:, None, None])
            out[b, :, lo:hi] = e4m3(rows / torch.exp2(need - 127)[:, None, None])
            scales[b, :, first // block] = need.int()
    return out, scales, after


def block_cache(B, Hkv, cap, d, block, seed, sharp=False):
    """Codes of K and V and their scales, of blocks of different sizes."""
    both, codes = [], []
    for i in range(2):
        x = normal((B, Hkv, cap, d), seed + i, torch.float32)
        if sharp and i == 0:
            x[:, :, ::13] *= 4
        e = torch.randint(123, 131, (B, Hkv, -(-cap // block)), device="cuda",
                          generator=torch.Generator(device="cuda").manual_seed(seed + 10 + i))
        wide = power(e).float().repeat_interleave(block, -1)[:, :, :cap, None]
        codes.append((x / wide).clamp(-448, 448).to(FP8))
        both.append(e)
    return codes[0], codes[1], torch.stack(both, -1).to(torch.uint8).view(E8M0)


def numbers(codes, scales, block, i):
    """What a cache's codes stand for, float64."""
    s = power(scales.view(torch.uint8)[..., i]).repeat_interleave(block, -1)[:, :, :codes.shape[2], None]
    return codes.float().double() * s


def blocks_ref(q, k, v, scales, block, lens, causal, scale, mode, cut):
    return prefix_ref(q, None, None, numbers(k, scales, block, 0), numbers(v, scales, block, 1), lens, causal, scale,
                      None, mode, 0, cut)

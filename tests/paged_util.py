"""64-bit references of rotary positions and of attention over pages, and how far a kernel's fp32 arithmetic may be from them."""
import math

import torch

LAYOUTS = ("half", "interleaved")
U = 2.0 ** -24                                    # half a step of fp32, relative


def half_step(dtype):
    """Rounding to a type, relative and absolute (below its normal range)."""
    return {torch.float16: (2.0 ** -11, 2.0 ** -25), torch.bfloat16: (2.0 ** -8, 2.0 ** -134), torch.float32: (2.0 ** -24, 2.0 ** -150)}[dtype]


def pairs(D, rot, layout):
    i = torch.arange(rot // 2)
    return (i, i + rot // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rope64(x, positions, freqs, layout, gain, sign=1.0):
    """x [B,H,N,D], positions [B,N]: the turned heads in fp64, and a bound on the error of the fp32 arithmetic before the rounding.

    cos and sin: 3e-8 from the polynomials' ends, their argument (at most pi/4) two roundings, four more in the sum of terms that fall
    off fast: 3.1e-7 in all, so 6e-7 with the roundings of gain, both products and their sum (1 U each of at most |x0| + |x1|).  An angle
    of a radians carries three fp64 roundings in the kernel and two here."""
    x, a = x.double(), positions.double().unsqueeze(-1) * freqs
    i0, i1 = (i.to(x.device) for i in pairs(x.shape[-1], 2 * freqs.numel(), layout))
    c, s = gain * a.cos().unsqueeze(1), gain * sign * a.sin().unsqueeze(1)
    x0, x1 = x[..., i0], x[..., i1]
    y, err = x.clone(), torch.zeros_like(x)
    y[..., i0], y[..., i1] = x0 * c - x1 * s, x1 * c + x0 * s
    e = (x0.abs() + x1.abs()) * abs(gain) * (6e-7 + 5 * 2.0 ** -53 * a.abs().unsqueeze(1))
    err[..., i0] = err[..., i1] = e
    return y, err


def check_rounded(got, want, err):
    rel, least = half_step(got.dtype)
    off = (got.double() - want).abs() - (err + rel * (want.abs() + err) + least)
    assert bool((off <= 0).all()), float(off.max())


def tokens(pages, table, n):
    """The first n tokens of one sequence: [Hkv, n, D]."""
    page = pages.shape[2]
    held = table[: -(-n // page)].long()
    return pages[held].transpose(0, 1).reshape(pages.shape[1], -1, pages.shape[3])[:, :n]


def attention64(q, k_pages, v_pages, table, lens, scale):
    """out, lse in fp64 and bounds on the error of the kernel's fp32 arithmetic.

    A score is a sum of D products of 16-bit numbers in fp32: D + 3 roundings (with the scale) of at most sum |q k|.  A
    probability then is off by twice that (itself and the maximum), by 4 U of the exponentials and their arguments' rounding
    (|s| U), and by 2^-16 where it is held in two 16-bit pieces; a sum over n keys adds n U."""
    B, Hq, D = q.shape
    Hkv = k_pages.shape[1]
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=q.device)
    eo, el = torch.zeros_like(out), torch.zeros_like(lse)
    for b, n in enumerate(lens):
        if n <= 0:
            continue
        k, v = (tokens(p, table[b], n).double() for p in (k_pages, v_pages))
        x = q[b].double().view(Hkv, Hq // Hkv, D)
        s = (x @ k.transpose(1, 2).contiguous()) * scale
        bound = (x.abs() @ k.abs().transpose(1, 2).contiguous()).amax(-1) * abs(scale)
        d = (D + 3) * U * bound + 4 * U * s.abs().amax(-1)                       # [Hkv, G]
        p = torch.softmax(s, -1)
        out[b], lse[b] = (p @ v).view(Hq, D), torch.logsumexp(s, -1).view(Hq)
        rel = (2 * (2 * d + 8 * U + n * U) + 2.0 ** -16).view(Hq, 1)
        eo[b] = rel * (p @ v.abs()).view(Hq, D)
        el[b] = (d + (n + 8) * U).view(Hq) + U * lse[b].abs()
    return out, lse, eo, el

"""The 8-bit paged cache in 64 bits, and attention over common starts of sequences."""
import math

import torch

from tests.paged_util import attention64, half_step, tokens


def exponent64(a):
    """The least e with a <= 448 * 2^e, held within -100 .. 120; 0 for 0."""
    f, e = torch.frexp(a.double())
    return torch.where(a == 0, 0, (e.long() - 9 + (f > 0.875)).clamp(-100, 120))


def power64(e):
    """2^e, from its bits: a device's pow is not exact."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def codes64(y):
    """Nearest E4M3 codes of y (|y| <= 448; NaN and infinities: NaN), ties to the even code."""
    mag = torch.where(y.isfinite(), y.abs(), 0.0).double()
    b = torch.where(mag == 0, -6, (torch.frexp(mag)[1].long() - 1).clamp(min=-6))
    n = torch.round(mag * power64(3 - b)).long()
    code = torch.where(y.isfinite(), 8 * (b + 6) + n, 127)
    return (code + 128 * torch.signbit(y).long()).to(torch.uint8)


def quantise64(x):
    """x [..., D] -> (codes, scale bytes, e)."""
    e = exponent64(torch.where(x.isfinite(), x.abs(), 0.0).amax(-1))
    return codes64(x.double() * power64(-e).unsqueeze(-1)), (e + 127).to(torch.uint8), e


def values64(codes, scales):
    b = codes.long()
    power, digits = (b >> 3) & 15, (b & 7).double()
    x = torch.where(power > 0, (8.0 + digits) * power64(power - 10), digits * 2.0 ** -9)
    x = torch.where((b & 127) == 127, math.nan, torch.where(b >= 128, -x, x))
    return x if scales is None else x * power64(scales.long() - 127).unsqueeze(-1)


def cache8(k_pages, v_pages):
    """16-bit pages in 8 bits: (k_codes, k_scales, v_codes, v_scales)."""
    (k, ks, _), (v, vs, _) = quantise64(k_pages), quantise64(v_pages)
    return k, ks, v, vs


def prefix64(q, k_pages, v_pages, table, lens, shared, scale, dtype):
    """attention64, and what it adds to the bound that the probabilities of the first shared[b] tokens are rounded to dtype once."""
    out, lse, eo, el = attention64(q, k_pages, v_pages, table, lens, scale)
    B, Hq, D = q.shape
    Hkv = k_pages.shape[1]
    for b, n in enumerate(lens):
        if shared[b] <= 0 or n <= 0:
            continue
        k, v = (tokens(p, table[b], n).double() for p in (k_pages, v_pages))
        s = (q[b].double().view(Hkv, Hq // Hkv, D) @ k.transpose(1, 2).contiguous()) * scale
        p = torch.softmax(s, -1)[:, :, :shared[b]].contiguous()
        eo[b] += half_step(dtype)[0] * (p @ v[:, :shared[b]].abs().contiguous()).view(Hq, D)
    return out, lse, eo, el

"""Timing cases of the 8-bit paged cache, of reading pages back, and of attention over shared prefixes, and their plain forms.

Four kinds of work, named by a case's "kind":

  append8  queries and keys of new tokens are rotated, keys and values are written into their pages in 8 bits (thrift_paged_append8)
  paged8   attention of one new token per sequence over the 8-bit cache (thrift_paged_decode8)
  read     the tokens that sequences have in pages, of 16 or 8 bits, laid out as rows of 16 bits (thrift_paged_read, thrift_paged_read8)
  prefix   attention of one new token per sequence where sequences start with the same pages (thrift_paged_decode_prefix,
           thrift_paged_decode_prefix8)

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits (angles and what is rounded to 8 bits in 64), otherwise
it makes the calls a program makes of the library.  Head counts and the longest contexts are those of
paper_2605_23081_amd/workloads.py and perf/operators.py.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = 1e6            # rotary base of long-context models
ORIGINAL = 32768      # tokens a model was trained on before its positions are scaled
_DT = {"f16": torch.float16, "bf16": torch.bfloat16}
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu


def _append8(name, T, Hq, Hkv, dtype, page, pad=0, rot=128, layout="half", factor=1.0, D=128):
    return dict(name=name, kind="append8", T=T, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page, pad=pad, rot=rot, layout=layout, factor=factor)


def _paged8(name, B, Hq, Hkv, tokens, dtype, page, spread, D=128, pad=0):
    return dict(name=name, kind="paged8", B=B, Hq=Hq, Hkv=Hkv, D=D, tokens=tokens, dtype=dtype, page=page, spread=spread, pad=pad)


def _read(name, B, Hkv, tokens, dtype, page, spread, bits, D=128):
    return dict(name=name, kind="read", B=B, Hkv=Hkv, D=D, tokens=tokens, dtype=dtype, page=page, spread=spread, bits=bits)


def _prefix(name, B, Hq, Hkv, prefix, most, dtype, page, bits=16, groups=1, alone=0, pad=0, D=128):
    return dict(name=name, kind="prefix", B=B, Hq=Hq, Hkv=Hkv, D=D, prefix=prefix, most=most, dtype=dtype, page=page, bits=bits,
                groups=groups, alone=alone, pad=pad)


def listed():
    return [
        # a decode step's tokens of sixteen users, in a batch padded to 24 rows
        _append8("append8_16", 24, 32, 8, "bf16", 16, pad=8),
        # a step's worth of prompt pieces, eight query heads per KV head
        _append8("append8_8k", 8192, 64, 8, "bf16", 64, layout="interleaved", factor=4.0),
        # one user, a short conversation
        _paged8("paged8_1x1k", 1, 32, 8, 1000, "bf16", 16, 1.0),
        # many conversations from a few tokens to some thousands, one KV head per query head, padded to 64 rows
        _paged8("paged8_64x4k_mha", 64, 16, 16, 4096, "f16", 16, 64.0, pad=3),
        # sixteen sequences at the longest context
        _paged8("paged8_16x131k", 16, 32, 8, 131072, "f16", 64, 1.0),
        # keys and values in front of a piece of one user's prompt, for the prefill kernel
        _read("read_1x30k", 1, 8, 30720, "bf16", 64, 1.0, 16),
        # the same for a few uneven sequences of an 8-bit cache, one KV head per query head
        _read("read8_5x3001", 5, 16, 3001, "f16", 16, 4.0, 8),
        # six users of an assistant, a short system prompt
        _prefix("prefix_6x2k", 6, 32, 8, 2000, 120, "bf16", 16),
        # questions of many users about one long document, eight query heads per KV head
        _prefix("prefix_64x32k_g8", 64, 64, 8, 32768, 1000, "bf16", 64),
        # three assistants on one server and users of none, one KV head per query head
        _prefix("prefix_40x8k_three", 40, 16, 16, 8192, 4096, "f16", 16, groups=3, alone=5, pad=3),
        # many samples of one long prompt from an 8-bit cache
        _prefix("prefix8_96x16k", 96, 32, 8, 16384, 500, "bf16", 32, bits=8),
    ]


_HEADS = ((32, 8), (64, 8), (16, 16), (32, 8))


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("append8", "read", "paged8", "paged8", "prefix", "prefix"))
    Hq, Hkv = rng.choice(_HEADS)
    dtype = rng.choice(("bf16", "f16"))
    D = rng.choice((128, 128, 128, 64, 256))
    page = rng.choice((16, 32, 64, 128))
    spread = rng.choice((1.0, 2.0, 16.0))
    if kind == "append8":
        T = _log_uniform(rng, 1, 32768)
        c = _append8("", T, Hq, Hkv, dtype, page, pad=rng.choice((0, T // 4)), rot=rng.choice((D, D, D // 2)),
                     layout=rng.choice(("half", "interleaved")), factor=rng.choice((1.0, 1.0, 4.0)), D=D)
    elif kind == "read":
        tokens = _log_uniform(rng, 1, 131072)
        B = _log_uniform(rng, 1, max(1, min(64, 131072 * 8 * 128 // (tokens * Hkv * D))))
        c = _read("", B, Hkv, tokens, dtype, page, spread, rng.choice((16, 8)), D=D)
    elif kind == "paged8":
        tokens = _log_uniform(rng, 8, 131072)
        B = _log_uniform(rng, 1, max(1, min(256, 16 * 131072 * 8 * 128 // (2 * tokens * Hkv * D))))
        c = _paged8("", B, Hq, Hkv, tokens, dtype, page, spread, D=D, pad=rng.choice((0, 0, B // 8)))
    else:
        B = _log_uniform(rng, 2, 128)
        groups = rng.randrange(1, max(1, min(4, B // 4)) + 1)
        most = _log_uniform(rng, 1, max(2, 4096 // max(1, B // 16)))
        prefix = _log_uniform(rng, 64, max(128, min(65536, 64 * 64 * 32768 // (B * Hq * groups))))
        c = _prefix("", B, Hq, Hkv, prefix, most, dtype, page, bits=rng.choice((16, 16, 8)), groups=groups,
                    alone=rng.choice((0, 0, B // 8)), pad=rng.choice((0, 0, B // 8)), D=D)
    del c["name"]
    return c


# ---- inputs ----

def frequencies(rot, factor, device):
    """Radians per position of every pair, fp64, and the gain; scaled by parts where factor > 1: pairs that turn less than once
    in the original length are slowed down by the factor, those that turn more than 32 times are left, the rest in between."""
    i = torch.arange(rot // 2, dtype=torch.float64, device=device)
    theta = BASE ** (-2.0 * i / rot)
    if factor == 1.0:
        return theta, 1.0
    w = ((ORIGINAL * theta / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
    return theta * ((1.0 - w) / factor + w), 0.1 * math.log(factor) + 1.0


def _randn(g, *shape, dtype):
    return torch.randn(*shape, generator=g, dtype=dtype, device=g.device)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 7919 + 29)
    return _PREPARE[case["kind"]](case, g)


def _exponent(a):
    """The least e with a <= 448 * 2^e; -100 .. 120, and 0 where a is 0."""
    f, e = torch.frexp(a)                                               # a = f 2^e, f in [1/2, 1)
    e = (e - 9 + (f > 0.875).to(e.dtype)).clamp(-100, 120)
    return torch.where(a == 0, torch.zeros_like(e), e)


def _power(e):
    """2^e in fp32, exactly: e in -126 .. 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _in_8_bits(x):
    """x [..., D] as codes (e4m3 in bytes) and one scale byte (exponent + 127) for the last axis."""
    e = _exponent(x.abs().amax(-1))
    return (x * _power(-e).unsqueeze(-1)).to(torch.float32).to(_E4M3).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    return codes.view(_E4M3).float() * _power(scales.to(torch.int32) - 127).unsqueeze(-1)


def _pool(g, case, n_pages, bits):
    """Keys and values of n_pages pages; tokens' magnitudes differ as those of a model's do."""
    shape = (n_pages, case["Hkv"], case["page"], case["D"])
    pages = []
    for _ in range(2):
        x = _randn(g, *shape, dtype=_DT[case["dtype"]])
        pages.append(x * torch.exp(0.3 * _randn(g, *shape[:3], 1, dtype=torch.float32)).to(x.dtype))
    if bits == 16:
        return dict(k_pages=pages[0], v_pages=pages[1])
    (k, ks), (v, vs) = (_in_8_bits(x.float()) for x in pages)
    return dict(k_codes=k, k_scales=ks, v_codes=v, v_scales=vs)


def _lengths(g, B, tokens, spread):
    n = tokens * torch.exp(-math.log(spread) * torch.rand(B, generator=g, device=g.device, dtype=torch.float64))
    return n.round().clamp(1, tokens).to(torch.int32)


def _queries(g, case, B):
    """[B,Hq,D]; the heads of a group share a direction."""
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    u = _randn(g, B, Hkv, 1, D, dtype=torch.float32)
    return (_randn(g, B, Hkv, Hq // Hkv, D, dtype=torch.float32) + u).view(B, Hq, D).to(_DT[case["dtype"]])


def _prepare_append8(case, g):
    T, Hq, Hkv, D, page, dt = (case[x] for x in ("T", "Hq", "Hkv", "D", "page", "dtype"))
    dt, dev = _DT[dt], g.device
    n_pages = -(-2 * T // page)
    x = _randn(g, T, Hq + 2 * Hkv, D, dtype=dt)                         # the output of one projection
    freqs, gain = frequencies(case["rot"], case["factor"], dev)
    slots = torch.randperm(n_pages * page, generator=g, device=dev)[:T].to(torch.int32)
    if case["pad"]:
        slots[T - case["pad"]:] = -1                                    # rows that pad the batch
    positions = torch.randint(0, 131072, (T,), generator=g, device=dev).to(torch.int32)
    return dict(case=case, q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:], slots=slots, positions=positions, freqs=freqs, gain=gain,
                q_out=torch.zeros(T, Hq, D, dtype=dt, device=dev), **_pool(g, case, n_pages, 8))


def _prepare_paged8(case, g):
    B, tokens, page, dev = case["B"], case["tokens"], case["page"], g.device
    max_pages = -(-tokens // page)
    n_pages = B * max_pages + 1
    table = torch.randperm(n_pages, generator=g, device=dev)[:B * max_pages].view(B, max_pages).to(torch.int32)
    lens = _lengths(g, B, tokens, case["spread"])
    if case["pad"]:
        lens[B - case["pad"]:] = 0
    return dict(case=case, q=_queries(g, case, B), table=table, seqlens=lens, **_pool(g, case, n_pages, 8))


def _prepare_read(case, g):
    B, tokens, page, dev = case["B"], case["tokens"], case["page"], g.device
    max_pages = -(-tokens // page)
    n_pages = B * max_pages + 1
    table = torch.randperm(n_pages, generator=g, device=dev)[:B * max_pages].view(B, max_pages).to(torch.int32)
    lens = _lengths(g, B, tokens, case["spread"])
    lens[0] = tokens
    return dict(case=case, table=table, seqlens=lens, **_pool(g, case, n_pages, case["bits"]))


def _prepare_prefix(case, g):
    B, page, groups, dev = case["B"], case["page"], case["groups"], g.device
    whole = max(1, case["prefix"] // page)                              # pages of the longest prefix
    rest = -(-case["most"] // page)                                     # pages of a sequence's own tokens at most
    max_pages = whole + rest
    n_pages = groups * whole + B * max_pages + 1
    pages = torch.randperm(n_pages, generator=g, device=dev)
    shared = (whole * (1.0 - 0.3 * torch.rand(groups, generator=g, device=dev))).round().clamp(min=1).long()
    shared[0] = whole
    # the sequences of a group stand anywhere in the batch; the last rows pad it, some in front of them are of no group
    of = torch.arange(B, device=dev) % groups
    of[B - case["pad"] - case["alone"]:] = -1
    busy = B - case["pad"]
    of[:busy] = of[:busy][torch.randperm(busy, generator=g, device=dev)]
    held = torch.where(of >= 0, shared[of.clamp(min=0)], 0)             # pages in front that a sequence shares
    j = torch.arange(max_pages, device=dev)
    prefixes = pages[:groups * whole].view(groups, whole)[of.clamp(min=0)]
    table = pages[groups * whole:groups * whole + B * max_pages].view(B, max_pages).clone()
    table[:, :whole] = torch.where(j[:whole] < held.unsqueeze(1), prefixes, table[:, :whole])
    lens = held * page + _lengths(g, B, case["most"], 16.0)
    lens[busy:] = 0
    return dict(case=case, q=_queries(g, case, B), table=table.to(torch.int32), seqlens=lens.to(torch.int32), group_of=of.to(torch.int32),
                group_lens=(shared * page).to(torch.int32), **_pool(g, case, n_pages, case["bits"]))


_PREPARE = {"append8": _prepare_append8, "paged8": _prepare_paged8, "read": _prepare_read, "prefix": _prepare_prefix}


# ---- one pass ----

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def _rotated(x, cos, sin, rot, layout, gain):
    """x [..., D] in cos's type with the first rot channels of each head turned; cos, sin [..., rot/2] broadcast against it."""
    x = x.to(cos.dtype)
    t = x[..., :rot]
    a, b = (t[..., :rot // 2], t[..., rot // 2:]) if layout == "half" else (t[..., ::2], t[..., 1::2])
    ya, yb = (a * cos - b * sin) * gain, (b * cos + a * sin) * gain
    y = torch.cat([ya, yb], -1) if layout == "half" else torch.stack([ya, yb], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _cache8(s):
    """What an 8-bit cache holds: codes and scales as the numbers they stand for."""
    return dict(k=s["k_codes"].view(_E4M3), k_scale=s["k_scales"].view(_E8M0), v=s["v_codes"].view(_E4M3), v_scale=s["v_scales"].view(_E8M0))


def _plain_append8(s):
    c = s["case"]
    a = s["positions"].double().unsqueeze(-1) * s["freqs"]
    cos, sin = a.cos().unsqueeze(1), a.sin().unsqueeze(1)
    q = _rotated(s["q"], cos.float(), sin.float(), c["rot"], c["layout"], s["gain"]).to(s["q"].dtype)
    k = _rotated(s["k"], cos, sin, c["rot"], c["layout"], s["gain"])
    keep = (s["slots"] >= 0).nonzero().squeeze(1)
    slot = s["slots"].long()[keep]
    page, at = slot // c["page"], slot % c["page"]
    s["k_codes"][page, :, at], s["k_scales"][page, :, at] = _in_8_bits(k[keep])
    s["v_codes"][page, :, at], s["v_scales"][page, :, at] = _in_8_bits(s["v"][keep].float())
    s["q_out"][keep] = q[keep]
    return dict(q=s["q_out"], **_cache8(s))


def _gathered(s, side, table):
    """The tokens of table's pages [n, pages] in 32 bits: [n, Hkv, tokens, D]."""
    if "k_pages" in s:
        x = s[side + "_pages"][table].float()
    else:
        x = _values(s[side + "_codes"][table], s[side + "_scales"][table])
    n, _, Hkv, _, D = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, Hkv, -1, D)


def _plain_paged8(s):
    c = s["case"]
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    table = s["table"].long()
    q = s["q"].float().view(B, Hkv, Hq // Hkv, D) * (1.0 / math.sqrt(D))
    score = torch.matmul(q, _gathered(s, "k", table).transpose(-1, -2))
    seen = torch.arange(score.shape[-1], device=q.device) < s["seqlens"].view(B, 1, 1, 1)
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _gathered(s, "v", table)) / total.masked_fill(total == 0, 1.0)
    lse = (top + total.log()).masked_fill(total == 0, -math.inf)
    return out.reshape(B, Hq, D).to(s["q"].dtype), lse.reshape(B, Hq)


def _plain_read(s):
    c = s["case"]
    table = s["table"].long()
    past = torch.arange(c["tokens"], device=table.device) >= s["seqlens"].unsqueeze(1)
    # in fp16 the largest codes at the largest scale stand for the largest finite number
    most = torch.finfo(_DT[c["dtype"]]).max
    return [_gathered(s, x, table)[:, :, :c["tokens"]].masked_fill(past[:, None, :, None], 0.0).clamp(-most, most).to(_DT[c["dtype"]]) for x in "kv"]


def _plain_prefix(s):
    c = s["case"]
    B, Hq, Hkv, D, page, groups = (c[x] for x in ("B", "Hq", "Hkv", "D", "page", "groups"))
    G = Hq // Hkv
    table, lens, of = s["table"].long(), s["seqlens"].long(), s["group_of"].long()
    whole = max(1, c["prefix"] // page)
    member = of == torch.arange(groups, device=of.device).unsqueeze(1)                # [groups, B]
    held = torch.where(of >= 0, s["group_lens"].long()[of.clamp(min=0)], 0)           # tokens in front that a sequence shares
    q = s["q"].float().view(B, Hkv, G, D) * (1.0 / math.sqrt(D))
    # every group's prefix once, from its first sequence's pages: all queries against all prefixes, those of other groups masked
    first = table[member.int().argmax(1), :whole]
    k, v = (_gathered(s, x, first).transpose(0, 1).reshape(Hkv, groups * whole * page, D) for x in "kv")
    j = torch.arange(whole * page, device=of.device)
    seen = (member.t().unsqueeze(2) & (j < s["group_lens"].long().unsqueeze(1))).reshape(B, 1, 1, -1)
    s1 = torch.matmul(q.transpose(0, 1).reshape(Hkv, B * G, D), k.transpose(1, 2)).view(Hkv, B, G, -1).transpose(0, 1).masked_fill(~seen, -math.inf)
    # the tokens behind, every sequence's own
    rest = -(-c["most"] // page)
    mine = table.gather(1, (held // page).unsqueeze(1) + torch.arange(rest, device=of.device))
    seen = torch.arange(rest * page, device=of.device) < (lens - held).view(B, 1, 1, 1)
    s2 = torch.matmul(q, _gathered(s, "k", mine).transpose(-1, -2)).masked_fill(~seen, -math.inf)
    top = torch.maximum(s1.amax(-1, keepdim=True), s2.amax(-1, keepdim=True))
    zero = top.masked_fill(top == -math.inf, 0.0)
    p1, p2 = torch.exp(s1 - zero), torch.exp(s2 - zero)
    total = p1.sum(-1, keepdim=True) + p2.sum(-1, keepdim=True)
    out = torch.matmul(p1.transpose(0, 1).reshape(Hkv, B * G, -1), v).view(Hkv, B, G, D).transpose(0, 1) + torch.matmul(p2, _gathered(s, "v", mine))
    out = out / total.masked_fill(total == 0, 1.0)
    lse = (top + total.log()).masked_fill(total == 0, -math.inf)
    return out.reshape(B, Hq, D).to(s["q"].dtype), lse.reshape(B, Hq)


_PLAIN = {"append8": _plain_append8, "paged8": _plain_paged8, "read": _plain_read, "prefix": _plain_prefix}


def _library():
    from paper_2605_23081_amd import binding
    return binding


def _pages8(s):
    return s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"]


def _own_append8(s):
    _library().thrift_paged_append8(s["k"], s["v"], s["slots"], *_pages8(s), q=s["q"], q_out=s["q_out"], positions=s["positions"],
                                    freqs=s["freqs"], layout=s["case"]["layout"], gain=s["gain"])
    return dict(q=s["q_out"], **_cache8(s))


def _own_paged8(s):
    return _library().thrift_paged_decode8(s["q"], *_pages8(s), s["table"], s["seqlens"], return_lse=True)


def _own_read(s):
    c = s["case"]
    if c["bits"] == 16:
        return _library().thrift_paged_read(s["k_pages"], s["v_pages"], s["table"], s["seqlens"], c["tokens"])
    return _library().thrift_paged_read8(*_pages8(s), s["table"], s["seqlens"], c["tokens"], _DT[c["dtype"]])


def _own_prefix(s):
    if s["case"]["bits"] == 16:
        return _library().thrift_paged_decode_prefix(s["q"], s["k_pages"], s["v_pages"], s["table"], s["seqlens"], s["group_of"], s["group_lens"],
                                                     return_lse=True)
    return _library().thrift_paged_decode_prefix8(s["q"], *_pages8(s), s["table"], s["seqlens"], s["group_of"], s["group_lens"], return_lse=True)


_OWN = {"append8": _own_append8, "paged8": _own_paged8, "read": _own_read, "prefix": _own_prefix}


# ---- what a pass cannot do without, and its results in 64 bits ----

def _mean_length(tokens, spread):
    return tokens * (1.0 if spread == 1.0 else (1.0 - 1.0 / spread) / math.log(spread))


def work(case):
    kind, Hkv, D, page = case["kind"], case["Hkv"], case["D"], case["page"]
    if kind == "append8":
        n, Hq = case["T"] - case["pad"], case["Hq"]
        return dict(bytes=n * (4 * Hq * D + 2 * Hkv * (3 * D + 1) + 4) + 4 * case["T"] + 4 * case["rot"], flops=3 * n * (Hq + Hkv) * case["rot"])
    if kind == "read":
        tokens = case["tokens"] + (case["B"] - 1) * _mean_length(case["tokens"], case["spread"])
        held = 4 * D if case["bits"] == 16 else 2 * (D + 1)
        return dict(bytes=tokens * (Hkv * held + 4.0 / page) + case["B"] * case["tokens"] * Hkv * 4 * D, flops=0)
    B, Hq = case["B"], case["Hq"]
    if kind == "paged8":
        keys = (B - case["pad"]) * _mean_length(case["tokens"], case["spread"])
        return dict(bytes=keys * (2 * Hkv * (D + 1) + 4.0 / page) + B * Hq * (4 * D + 4) + 4 * B, flops=4 * keys * Hq * D)
    alone = (B - case["pad"]) * _mean_length(case["most"], 16.0)
    shared = max(1, case["prefix"] // page) * page * (1.0 + 0.85 * (case["groups"] - 1))
    members = (B - case["pad"] - case["alone"]) / case["groups"]
    held = 4 * D if case["bits"] == 16 else 2 * (D + 1)
    return dict(bytes=(alone + shared) * (Hkv * held + 4.0 / page) + B * Hq * (4 * D + 4) + 8 * B, flops=4 * (alone + shared * members) * Hq * D)


def exact(case, seed):
    s = prepare(case, seed)
    return _EXACT[case["kind"]](s)


def _nearest8(x):
    """x [..., D] in 64 bits to (the numbers that e4m3 codes stand for, scales): the 8-bit grid has steps of 2^(b-3) in the binade of 2^b, and of
    2^-9 below 2^-6."""
    top = x.abs().amax(-1)
    scale = torch.exp2(torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(-100, 120))
    scale = torch.where(top > 448.0 * scale, 2 * scale, torch.where(top <= 224.0 * scale, scale / 2, scale)).clamp(2.0 ** -100, 2.0 ** 120)
    scale = torch.where(top == 0, torch.ones_like(scale), scale).unsqueeze(-1)
    y = x / scale
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step, scale.squeeze(-1)


def _numbers8(s, side):
    """What the bytes of an 8-bit cache stand for, in 64 bits, from their bits."""
    b = s[side + "_codes"].to(torch.int64)
    power, digits = (b >> 3) & 15, (b & 7).double()
    x = torch.where(power > 0, (8.0 + digits) * torch.exp2(power.double() - 10), digits * 2.0 ** -9)
    return torch.where(b >= 128, -x, x)


def _exact_append8(s):
    case = s["case"]
    turn = torch.polar(torch.tensor(s["gain"], dtype=torch.float64, device=s["freqs"].device).expand(s["positions"].shape + s["freqs"].shape).contiguous(),
                       s["positions"].double().unsqueeze(-1) * s["freqs"]).unsqueeze(1)

    def turned(x):
        y = x.double().clone()
        n = case["rot"]
        even, odd = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * turn
        y[..., even], y[..., odd] = z.real, z.imag
        return y

    live = s["slots"] >= 0
    to = s["slots"][live].long()
    q_out = s["q_out"].double()
    q_out[live] = turned(s["q"])[live]
    found = dict(q=q_out)
    for side, x in (("k", turned(s["k"])), ("v", s["v"].double())):
        codes, scales = _numbers8(s, side).transpose(1, 2).contiguous(), torch.exp2(s[side + "_scales"].double() - 127).transpose(1, 2).contiguous()
        flat, flat_scales = codes.view(-1, case["Hkv"], case["D"]), scales.view(-1, case["Hkv"])
        flat[to], flat_scales[to] = _nearest8(x[live])
        found[side], found[side + "_scale"] = codes.transpose(1, 2), scales.transpose(1, 2)
    return found


def _tokens64(s, side, pages, head):
    if "k_pages" in s:
        return s[side + "_pages"][pages, head].double().reshape(-1, s["case"]["D"])
    part = {side + "_codes": s[side + "_codes"][pages, head]}
    return (_numbers8(part, side) * torch.exp2(s[side + "_scales"][pages, head].double() - 127).unsqueeze(-1)).reshape(-1, s["case"]["D"])


def _exact_attention(s):
    c = s["case"]
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(s["seqlens"].tolist()):
        if n == 0:
            continue
        held = s["table"][b, :-(-n // c["page"])].long()
        for h in range(Hkv):
            keys, values = (_tokens64(s, x, held, h)[:n] for x in "kv")
            rows = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            score = s["q"][b, rows].double() @ keys.t().contiguous() / math.sqrt(D)
            lse[b, rows] = torch.logsumexp(score, -1)
            out[b, rows] = torch.softmax(score, -1) @ values
    return out, lse


def _exact_read(s):
    c = s["case"]
    found = [torch.zeros(c["B"], c["Hkv"], c["tokens"], c["D"], dtype=torch.float64, device=s["table"].device) for _ in "kv"]
    for b, n in enumerate(s["seqlens"].tolist()):
        held = s["table"][b, :-(-n // c["page"])].long()
        for h in range(c["Hkv"]):
            for x, y in zip(found, "kv"):
                x[b, h, :n] = _tokens64(s, y, held, h)[:n]
    return found


_EXACT = {"append8": _exact_append8, "paged8": _exact_attention, "read": _exact_read, "prefix": _exact_attention}

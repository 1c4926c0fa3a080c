"""Timing cases of the operators around a paged 16-bit key-value cache, and their plain forms.

Five kinds of work, named by a case's "kind":

  rope     rotary positions of the query and key heads of a batch (thrift_rope)
  grad     the gradient of that with respect to its inputs (thrift_rope_backward)
  map      one scheduling step of a server: every request's new tokens get pages, block-table entries, slots and
           positions from the requests' lengths (thrift_page_map)
  append   queries and keys of new tokens are rotated, keys and values are written into their pages (thrift_paged_append)
  paged    attention of one new token per sequence over the paged cache (thrift_paged_decode)

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits (angles in 64), otherwise it makes
the calls a program makes of the library.  Head counts and the longest contexts are those of
paper_2605_23081_amd/workloads.py and perf/cases.py.
"""
from __future__ import annotations

import math

import torch

own = False

BASE = 1e6            # rotary base of long-context models
ORIGINAL = 32768      # tokens a model was trained on before its positions are scaled
_DT = {"f16": torch.float16, "bf16": torch.bfloat16}


def _rope(name, kind, B, N, Hq, Hkv, dtype, rot=128, layout="half", factor=1.0, fused=False, D=128):
    return dict(name=name, kind=kind, B=B, N=N, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, rot=rot, layout=layout, factor=factor, fused=fused)


def _map(name, B, page, max_pages, rows, cached, new, pool):
    return dict(name=name, kind="map", B=B, page=page, max_pages=max_pages, rows=rows, cached=cached, new=new, pool=pool)


def _append(name, T, Hq, Hkv, dtype, page, pad=0, rot=128, layout="half", factor=1.0, D=128):
    return dict(name=name, kind="append", T=T, Hq=Hq, Hkv=Hkv, D=D, dtype=dtype, page=page, pad=pad, rot=rot, layout=layout, factor=factor)


def _paged(name, B, Hq, Hkv, tokens, dtype, page, spread, D=128, pad=0):
    return dict(name=name, kind="paged", B=B, Hq=Hq, Hkv=Hkv, D=D, tokens=tokens, dtype=dtype, page=page, spread=spread, pad=pad)


def listed():
    return [
        # the token just sampled for each of sixteen users: latency is all there is
        _rope("rope_16x1", "rope", 16, 1, 32, 8, "bf16"),
        # a layer over the longest prompt of the benchmark, positions scaled beyond the trained length
        _rope("rope_131k", "rope", 1, 131072, 32, 8, "f16", layout="interleaved", factor=4.0),
        # backward pass over an ordinary prompt; q and k lie in the output of one fused projection
        _rope("grad_3001", "grad", 1, 3001, 32, 8, "bf16", fused=True),
        # backward pass over a batch, one KV head per query head, half of each head rotated
        _rope("grad_2x8k_partial", "grad", 2, 8192, 16, 16, "f16", rot=64, layout="interleaved"),
        # a decode step of a server with 256 running requests: one token each, some requests need a new page
        _map("map_256_step", 256, 16, 2048, 256, 8192, 1, 65536),
        # 64 prompts admitted at once, uneven lengths, in a row buffer of fixed size
        _map("map_64_prompts", 64, 64, 512, 262144, 2048, 8192, 16384),
        # a decode step's tokens of sixteen users, in a batch padded to 24 rows
        _append("append_16", 24, 32, 8, "bf16", 16, pad=8),
        # a step's worth of prompt pieces, eight query heads per KV head
        _append("append_8k", 8192, 64, 8, "bf16", 64, layout="interleaved", factor=4.0),
        # one user, a short conversation
        _paged("paged_1x1k", 1, 32, 8, 1000, "bf16", 16, 1.0),
        # a batch of users with uneven long documents, eight query heads per KV head
        _paged("paged_8x32k_g8", 8, 64, 8, 32768, "bf16", 64, 2.0),
        # many conversations from a few tokens to some thousands, one KV head per query head, padded to 64 rows
        _paged("paged_64x4k_mha", 64, 16, 16, 4096, "f16", 16, 64.0, pad=3),
        # sixteen sequences at the longest context
        _paged("paged_16x131k", 16, 32, 8, 131072, "f16", 64, 1.0),
    ]


_HEADS = ((32, 8), (64, 8), (16, 16), (32, 8))


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "grad", "map", "append", "paged", "paged", "paged"))
    Hq, Hkv = rng.choice(_HEADS)
    dtype = rng.choice(("bf16", "f16"))
    D = rng.choice((128, 128, 128, 64, 256))
    rot = rng.choice((D, D, D // 2))
    layout = rng.choice(("half", "interleaved"))
    factor = rng.choice((1.0, 1.0, 4.0))
    page = rng.choice((16, 32, 64, 128))
    if kind in ("rope", "grad"):
        N = _log_uniform(rng, 1, 60000)
        B = _log_uniform(rng, 1, max(1, min(32, 120000 // N)))
        c = _rope("", kind, B, N, Hq, Hkv, dtype, rot=rot, layout=layout, factor=factor, fused=rng.random() < 0.5, D=D)
    elif kind == "map":
        B = _log_uniform(rng, 1, 1024)
        new = _log_uniform(rng, 1, 8192)
        cached = _log_uniform(rng, 1, 16384)
        max_pages = 2 * (new + cached) // page + 1
        rows = min(1 << 18, max(B, B * new // 2 + rng.randrange(1, 64)))
        pool = max(64, int(B * (cached + new) / page * rng.choice((0.4, 1.2))))
        c = _map("", B, page, max_pages, rows, cached, new, pool)
    elif kind == "append":
        T = _log_uniform(rng, 1, 32768)
        c = _append("", T, Hq, Hkv, dtype, page, pad=rng.choice((0, T // 4)), rot=rot, layout=layout, factor=factor, D=D)
    else:
        tokens = _log_uniform(rng, 8, 131072)
        B = _log_uniform(rng, 1, max(1, min(256, 16 * 131072 * 8 * 128 // (2 * tokens * Hkv * D))))
        c = _paged("", B, Hq, Hkv, tokens, dtype, page, rng.choice((1.0, 2.0, 16.0)), D=D, pad=rng.choice((0, 0, B // 8)))
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
    g.manual_seed(int(seed) * 7919 + 17)
    return _PREPARE[case["kind"]](case, g)


def _heads(case, g, B, N):
    """q and k [B,H,N,D]: contiguous, or views of one projection's output [B,N,(Hq + 2 Hkv) D]."""
    Hq, Hkv, D, dt = case["Hq"], case["Hkv"], case["D"], _DT[case["dtype"]]
    if case["fused"]:
        x = _randn(g, B, N, Hq + 2 * Hkv, D, dtype=dt).transpose(1, 2)
        return x[:, :Hq], x[:, Hq:Hq + Hkv]
    return _randn(g, B, Hq, N, D, dtype=dt), _randn(g, B, Hkv, N, D, dtype=dt)


def _prepare_rope(case, g):
    B, N = case["B"], case["N"]
    q, k = _heads(case, g, B, N)
    freqs, gain = frequencies(case["rot"], case["factor"], g.device)
    # every sequence continues at a place of its own, up to the longest context
    first = torch.randint(0, max(1, 131072 - N) + 1, (B, 1), generator=g, device=g.device)
    positions = (first + torch.arange(N, device=g.device)).to(torch.int32)
    return dict(case=case, q=q, k=k, freqs=freqs, gain=gain, positions=positions)


def _prepare_map(case, g):
    B, page, pool = case["B"], case["page"], case["pool"]
    dev, i32 = g.device, torch.int32
    cap = case["max_pages"] * page
    lens = torch.randint(0, case["cached"] + 1, (B,), generator=g, device=dev).clamp(max=cap)
    new = torch.randint(1, case["new"] + 1, (B,), generator=g, device=dev)
    pages = torch.randperm(2 * pool, generator=g, device=dev)
    held = (lens + page - 1) // page
    # the pages that requests hold are drawn from the second half of the pool, the free ones are the first
    j = torch.arange(case["max_pages"], device=dev)
    at = (held.cumsum(0) - held).unsqueeze(1) + j
    table = torch.where(j < held.unsqueeze(1), pages[pool + at % pool], -1).to(i32)
    free = pages[:pool].to(i32)
    return dict(case=case, seqlens=lens.to(i32), new_lens=new.to(i32), table=table, free=free, n_pages=2 * pool,
                free_count=torch.tensor([pool - pool // 7], dtype=i32, device=dev))


def _prepare_append(case, g):
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
                k_pages=_randn(g, n_pages, Hkv, page, D, dtype=dt), v_pages=_randn(g, n_pages, Hkv, page, D, dtype=dt),
                q_out=torch.zeros(T, Hq, D, dtype=dt, device=dev))


def _prepare_paged(case, g):
    B, Hq, Hkv, D, tokens, page = (case[x] for x in ("B", "Hq", "Hkv", "D", "tokens", "page"))
    dt, dev = _DT[case["dtype"]], g.device
    max_pages = -(-tokens // page)
    n_pages = B * max_pages + 1
    table = torch.randperm(n_pages, generator=g, device=dev)[:B * max_pages].view(B, max_pages)
    lens = (tokens * torch.exp(-math.log(case["spread"]) * torch.rand(B, generator=g, device=dev, dtype=torch.float64))).round()
    lens = lens.clamp(1, tokens).to(torch.int32)
    if case["pad"]:
        lens[B - case["pad"]:] = 0
    k_pages = _randn(g, n_pages, Hkv, page, D, dtype=dt)
    v_pages = _randn(g, n_pages, Hkv, page, D, dtype=dt)
    q = _randn(g, B, Hkv, Hq // Hkv, D, dtype=torch.float32)
    # the heads of a group share a direction; the first tokens (sinks) and a few others have keys along it
    u = _randn(g, B, Hkv, D, dtype=torch.float32)
    q = (q + u.unsqueeze(2)).view(B, Hq, D).to(dt)
    at = torch.cat([torch.arange(4, device=dev).expand(B, 4), torch.randint(0, tokens, (B, 4), generator=g, device=dev)], 1) % tokens
    sink = (0.6 * u + 0.5 * _randn(g, B, Hkv, D, dtype=torch.float32)).to(dt)
    k_pages[table.gather(1, at // page), :, at % page] = sink.unsqueeze(1).expand(B, 8, Hkv, D)
    return dict(case=case, q=q, k_pages=k_pages, v_pages=v_pages, table=table.to(torch.int32).contiguous(), seqlens=lens)


_PREPARE = {"rope": _prepare_rope, "grad": _prepare_rope, "map": _prepare_map, "append": _prepare_append, "paged": _prepare_paged}


# ---- one pass ----

def run(state):
    return (_OWN if own else _PLAIN)[state["case"]["kind"]](state)


def _rotated(x, cos, sin, rot, layout, gain):
    """x [..., D] in 32 bits with the first rot channels of each head turned; cos, sin [..., rot/2] broadcast against it."""
    x = x.float()
    t = x[..., :rot]
    a, b = (t[..., :rot // 2], t[..., rot // 2:]) if layout == "half" else (t[..., ::2], t[..., 1::2])
    ya, yb = (a * cos - b * sin) * gain, (b * cos + a * sin) * gain
    y = torch.cat([ya, yb], -1) if layout == "half" else torch.stack([ya, yb], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_rope(s, sign=1.0):
    c = s["case"]
    a = s["positions"].double().unsqueeze(-1) * s["freqs"]                            # angles of far positions need 64 bits
    cos, sin = a.cos().float().unsqueeze(1), (sign * a.sin()).float().unsqueeze(1)
    return [_rotated(x, cos, sin, c["rot"], c["layout"], s["gain"]).to(x.dtype).contiguous() for x in (s["q"], s["k"])]


def _plain_map(s):
    c = s["case"]
    page, rows, table = c["page"], c["rows"], s["table"]
    cap, B = c["max_pages"] * page, c["B"]
    i32 = torch.int32
    lens, new = s["seqlens"].long().clamp(0, cap), s["new_lens"].long().clamp(0, rows)
    ends = new.cumsum(0).clamp(max=rows)
    starts = torch.cat([ends.new_zeros(1), ends])
    fit = torch.minimum(ends - starts[:-1], cap - lens)
    old = (lens + page - 1) // page
    want = (lens + fit + page - 1) // page - old
    avail = s["free_count"].long().clamp(0, s["free"].numel())
    first = want.cumsum(0) - want
    got = torch.minimum((avail - first).clamp(min=0), want)
    placed = torch.minimum(fit, (old + got) * page - lens)
    # the pages taken, in sequence order from the top of the stack
    j = torch.arange(c["max_pages"], device=table.device) - old.unsqueeze(1)
    take = (j >= 0) & (j < got.unsqueeze(1))
    place = (avail - 1 - first.unsqueeze(1) - j).clamp(0, s["free"].numel() - 1)
    table.copy_(torch.where(take, s["free"][place], table))
    row = torch.arange(rows, device=table.device)
    b = torch.searchsorted(ends, row, right=True)
    used = b < B
    b = b.clamp(max=B - 1)
    i = row - starts[b]
    pos = lens[b] + i
    held = table[b, (pos // page).clamp(max=c["max_pages"] - 1)].long()
    slots = torch.where(used & (i < placed[b]) & (held >= 0) & (held < s["n_pages"]), held * page + pos % page, -1)
    return dict(table=table, slots=slots.to(i32), positions=torch.where(used, pos, 0).to(i32), starts=starts.to(i32),
                seqlens=(lens + placed).to(i32), free_count=(avail - torch.minimum(want.sum(), avail)).to(i32))


def _plain_append(s):
    c = s["case"]
    a = s["positions"].double().unsqueeze(-1) * s["freqs"]
    cos, sin = a.cos().float().unsqueeze(1), a.sin().float().unsqueeze(1)
    q, k = (_rotated(x, cos, sin, c["rot"], c["layout"], s["gain"]).to(x.dtype) for x in (s["q"], s["k"]))
    keep = (s["slots"] >= 0).nonzero().squeeze(1)
    slot = s["slots"].long()[keep]
    s["k_pages"][slot // c["page"], :, slot % c["page"]] = k[keep]
    s["v_pages"][slot // c["page"], :, slot % c["page"]] = s["v"][keep]
    s["q_out"][keep] = q[keep]
    return s["q_out"], s["k_pages"], s["v_pages"]


def _plain_paged(s):
    c = s["case"]
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]

    def gathered(pages):
        x = pages[s["table"].long()]                                                  # [B, pages, Hkv, page, D]
        return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, D).float()

    q = s["q"].float().view(B, Hkv, Hq // Hkv, D) * (1.0 / math.sqrt(D))
    score = torch.matmul(q, gathered(s["k_pages"]).transpose(-1, -2))
    seen = torch.arange(score.shape[-1], device=q.device) < s["seqlens"].view(B, 1, 1, 1)
    score = score.masked_fill(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.masked_fill(top == -math.inf, 0.0))
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, gathered(s["v_pages"])) / total.masked_fill(total == 0, 1.0)
    lse = (top + total.log()).masked_fill(total == 0, -math.inf)
    return out.reshape(B, Hq, D).to(s["q"].dtype), lse.reshape(B, Hq)


_PLAIN = {"rope": _plain_rope, "grad": lambda s: _plain_rope(s, -1.0), "map": _plain_map, "append": _plain_append, "paged": _plain_paged}


def _library():
    from paper_2605_23081_amd import binding
    return binding


def _own_rope(s):
    c = s["case"]
    return _library().thrift_rope(s["q"], s["k"], s["freqs"], s["positions"], layout=c["layout"], gain=s["gain"])


def _own_grad(s):
    c = s["case"]
    return _library().thrift_rope_backward(s["q"], s["k"], s["freqs"], s["positions"], layout=c["layout"], gain=s["gain"])


def _own_map(s):
    c = s["case"]
    slots, positions, starts, seqlens, free_count = _library().thrift_page_map(
        s["seqlens"], s["new_lens"], s["table"], s["free"], s["free_count"], c["page"], s["n_pages"], c["rows"])
    return dict(table=s["table"], slots=slots, positions=positions, starts=starts, seqlens=seqlens, free_count=free_count)


def _own_append(s):
    _library().thrift_paged_append(s["k"], s["v"], s["slots"], s["k_pages"], s["v_pages"], q=s["q"], q_out=s["q_out"],
                                   positions=s["positions"], freqs=s["freqs"], layout=s["case"]["layout"], gain=s["gain"])
    return s["q_out"], s["k_pages"], s["v_pages"]


def _own_paged(s):
    return _library().thrift_paged_decode(s["q"], s["k_pages"], s["v_pages"], s["table"], s["seqlens"], return_lse=True)


_OWN = {"rope": _own_rope, "grad": _own_grad, "map": _own_map, "append": _own_append, "paged": _own_paged}


# ---- what a pass cannot do without, and its results in 64 bits ----

def work(case):
    kind = case["kind"]
    if kind in ("rope", "grad"):
        n = case["B"] * case["N"]
        heads = case["Hq"] + case["Hkv"]
        return dict(bytes=n * (4 * heads * case["D"] + 4) + 4 * case["rot"], flops=3 * n * heads * case["rot"])
    if kind == "map":
        B, rows = case["B"], min(case["rows"], case["B"] * (1 + case["new"]) // 2)
        return dict(bytes=20 * B + 8 * (rows // case["page"] + 1) + 8 * case["rows"], flops=0)
    if kind == "append":
        n, Hq, Hkv, D = case["T"] - case["pad"], case["Hq"], case["Hkv"], case["D"]
        return dict(bytes=n * (4 * (Hq + 2 * Hkv) * D + 4) + 4 * case["T"] + 4 * case["rot"], flops=3 * n * (Hq + Hkv) * case["rot"])
    B, Hq, Hkv, D = case["B"], case["Hq"], case["Hkv"], case["D"]
    spread = case["spread"]
    mean = case["tokens"] * (1.0 if spread == 1.0 else (1.0 - 1.0 / spread) / math.log(spread))
    keys = (B - case["pad"]) * mean
    return dict(bytes=keys * (4 * Hkv * D + 4.0 / case["page"]) + B * Hq * (4 * D + 4) + 4 * B, flops=4 * keys * Hq * D)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "map":
        return None
    if kind == "paged":
        return _exact_paged(s)
    turn = torch.polar(torch.tensor(s["gain"], dtype=torch.float64, device=s["freqs"].device).expand(s["positions"].shape + s["freqs"].shape).contiguous(),
                       s["positions"].double().unsqueeze(-1) * s["freqs"])
    if kind == "grad":
        turn = turn.conj()

    def turned(x, turn):
        y = x.double().clone()
        n = case["rot"]
        even, odd = (slice(0, n // 2), slice(n // 2, n)) if case["layout"] == "half" else (slice(0, n, 2), slice(1, n, 2))
        z = torch.complex(y[..., even].contiguous(), y[..., odd].contiguous()) * turn
        y[..., even], y[..., odd] = z.real, z.imag
        return y

    if kind in ("rope", "grad"):
        return [turned(x, turn.unsqueeze(1)) for x in (s["q"], s["k"])]
    q, k, v = turned(s["q"], turn.unsqueeze(1)), turned(s["k"], turn.unsqueeze(1)), s["v"].double()
    pages = [s["k_pages"].double(), s["v_pages"].double()]
    flat = [p.transpose(1, 2).reshape(-1, case["Hkv"], case["D"]) for p in pages]
    q_out = s["q_out"].double()
    live = s["slots"] >= 0
    for f, x in zip(flat, (k, v)):
        f[s["slots"][live].long()] = x[live]
    q_out[live] = q[live]
    back = [f.view(p.shape[0], case["page"], case["Hkv"], case["D"]).transpose(1, 2).contiguous() for f, p in zip(flat, pages)]
    return q_out, back[0], back[1]


def _exact_paged(s):
    c = s["case"]
    B, Hq, Hkv, D = c["B"], c["Hq"], c["Hkv"], c["D"]
    out = torch.zeros(B, Hq, D, dtype=torch.float64, device=s["q"].device)
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device=s["q"].device)
    for b, n in enumerate(s["seqlens"].tolist()):
        if n == 0:
            continue
        held = s["table"][b, :-(-n // c["page"])].long()
        for h in range(Hkv):
            keys = s["k_pages"][held, h].reshape(-1, D)[:n].double()
            values = s["v_pages"][held, h].reshape(-1, D)[:n].double()
            rows = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            score = s["q"][b, rows].double() @ keys.t().contiguous() / math.sqrt(D)
            lse[b, rows] = torch.logsumexp(score, -1)
            out[b, rows] = torch.softmax(score, -1) @ values
    return out, lse

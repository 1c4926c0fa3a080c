"""The paged cache on the GPU: page maps and releases against plain loops, appends bit for bit, attention against 64 bits, and a
server's steps with all of them."""
import math
import random

import pytest
import torch

from tests.paged_util import LAYOUTS, attention64, check_rounded, rope64, tokens

pytestmark = pytest.mark.gpu
DTYPES = (torch.float16, torch.bfloat16)
I32 = torch.int32


@pytest.fixture(scope="module")
def T():
    from paper_2605_23081_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


def _randn(*shape, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _ints(x):
    return torch.tensor(x, dtype=I32, device="cuda")


# ---- page maps ----

def page_map(lens, new, table, free, count, page, n_pages, rows):
    """include/thrift.h in plain steps, on lists: (table, slots, positions, starts, lens, count)."""
    table = [list(r) for r in table]
    width = len(table[0])
    count = min(len(free), max(0, count))
    slots, positions, starts, after = [], [], [0], []
    for b, n in enumerate(new):
        length = placed = min(width * page, max(0, lens[b]))
        here = min(max(0, n), rows - starts[-1])
        starts.append(starts[-1] + here)
        for p in range(length, length + here):
            positions.append(p)
            held = p // page < -(-placed // page)                        # the token's page is the sequence's already
            if p != placed or p >= width * page or (not held and count == 0):
                slots.append(-1)
                continue
            if not held:
                count -= 1
                table[b][p // page] = free[count]
            placed += 1
            name = table[b][p // page]
            slots.append(name * page + p % page if 0 <= name < n_pages else -1)
        after.append(placed)
    pad = rows - len(slots)
    return table, slots + [-1] * pad, positions + [0] * pad, starts, after, count


def _check_map(T, lens, new, table, free, count, page, n_pages, rows):
    t = _ints(table)
    got = T.thrift_page_map(_ints(lens), _ints(new), t, _ints(free), _ints([count]), page, n_pages, rows)
    want = page_map(lens, new, table, free, count, page, n_pages, rows)
    for name, g, w in zip(("table", "slots", "positions", "starts", "lens", "count"), (t, *got), want):
        assert g.tolist() == (w if isinstance(w, list) else [w]), name


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("B", [1, 2, 63, 64, 65, 256, 257])
def test_page_map_against_plain_steps(T, page, B):
    rng = random.Random(page * 1000 + B)
    for trial in range(4):
        print(f"page_map page={page} B={B} trial={trial}", flush=True)
        width = rng.randint(1, 6)
        n_pages = B * width + 3
        lens = [rng.choice((0, 1, page - 1, page, rng.randint(0, width * page), width * page)) for _ in range(B)]
        new = [rng.choice((0, 1, 1, 1, page, rng.randint(0, 2 * page), -3)) for _ in range(B)]
        order = list(range(n_pages))
        rng.shuffle(order)
        table = [[order.pop() if j < -(-n // page) else -1 for j in range(width)] for n in map(lambda x: min(x, width * page), lens)]
        total = sum(max(0, n) for n in new)
        rows = max(1, rng.choice((total, total + 5, total // 2, total + 300)))
        count = rng.choice((len(order), len(order) // 2, 0, len(order) + 9, -1))
        _check_map(T, lens, new, table, order or [0], count if order else 0, page, n_pages, rows)


def test_page_map_refuses_bad_pages_and_lengths_on_the_device(T):
    # pages outside the pool, in the table and on the stack; lengths outside the table
    _check_map(T, [3, 40, -5, 16], [2, 9, 3, 4], [[-1, 0], [2, 99], [-1, -1], [5, -1]], [7, 100, 1, -4], 4, 16, 8, 20)
    _check_map(T, [1000, 5], [4, 40], [[0, 1], [2, -1]], [3, 4, 5], 3, 16, 8, 50)
    # counts whose sums pass 32 bits
    _check_map(T, [0] * 5, [2 ** 31 - 1] * 5, [[-1] * 3 for _ in range(5)], list(range(20)), 20, 16, 20, 77)


def test_page_map_of_the_largest_batch(T):
    B, page, width = 4096, 16, 4
    rng = random.Random(1)
    lens = [rng.randint(0, width * page) for _ in range(B)]
    new = [rng.randint(0, 3) for _ in range(B)]
    pages = list(range(2 * B * width))
    rng.shuffle(pages)
    table = [[pages.pop() if j < -(-n // page) else -7 for j in range(width)] for n in lens]
    _check_map(T, lens, new, table, pages, len(pages), page, 2 * B * width, sum(new) + 11)


def test_release_against_plain_steps(T):
    rng = random.Random(2)
    for B in (1, 3, 64, 300, 4096):
        page, width = 32, 5
        n_pages = B * width
        lens = [rng.choice((0, 1, 31, 32, 33, width * page, 10 ** 6, -4)) for _ in range(B)]
        drop = [rng.choice((0, 1, 5, -1)) for _ in range(B)]
        table = [[rng.choice((-1, n_pages, rng.randrange(n_pages))) if rng.random() < 0.2 else rng.randrange(n_pages) for _ in range(width)] for _ in range(B)]
        for capacity, count in ((B * width + 50, 40), (max(1, B), 0), (B * width + 50, -9)):
            print(f"release B={B} capacity={capacity} count={count}", flush=True)
            free = [1000 + i for i in range(capacity)]
            stack = _ints(free)
            after, left = T.thrift_page_release(_ints(lens), _ints(drop), _ints(table), stack, _ints([count]), page, n_pages)
            have, want = min(max(0, count), capacity), list(free)
            for b in range(B):
                if drop[b]:
                    for p in table[b][: -(-min(max(0, lens[b]), width * page) // page)]:
                        if 0 <= p < n_pages and have < capacity:
                            want[have] = p
                            have += 1
            assert stack.tolist() == want and left.tolist() == [have]
            assert after.tolist() == [0 if d else n for d, n in zip(drop, lens)]


def test_map_and_release_keep_the_pool_whole(T):
    """Hundreds of steps of arrivals, tokens and departures: no page is held twice and none is lost."""
    table = T.PageTable(24, 12, 16, 150, "cuda")
    rng = random.Random(3)
    held = [0] * 24
    for step in range(120):
        new = [rng.choice((0, 1, 1, rng.randint(1, 60))) if rng.random() < 0.7 else 0 for _ in range(24)]
        table.map(_ints(new), sum(new) + 1)
        if step % 3 == 0:
            table.release(_ints([int(rng.random() < 0.3) for _ in range(24)]))
        lens, count = table.seqlens.tolist(), int(table.free_count)
        held = [p for b, n in enumerate(lens) for p in table.block_table[b, :-(-n // 16)].tolist()]
        assert sorted(held + table.free_pages[:count].tolist()) == list(range(150)), step
    assert any(n > 0 for n in table.seqlens.tolist())


# ---- appends ----

@pytest.mark.parametrize("T_,Hq,Hkv,D,rot,page", [(1, 32, 8, 128, 128, 16), (37, 6, 2, 128, 64, 32), (5, 3, 3, 64, 64, 256), (130, 8, 1, 256, 256, 64), (9, 2, 1, 96, 40, 16),
                                                  (70, 4, 4, 128, 0, 16), (3, 2, 2, 30, 14, 16), (300, 64, 8, 128, 128, 64), (5003, 2, 1, 128, 64, 16), (1100, 3, 1, 64, 64, 32), (2100, 1, 2, 48, 16, 16), (2, 1, 1, 2, 2, 16), (4, 2, 1, 1024, 512, 16)])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_against_64_bits(T, T_, Hq, Hkv, D, rot, page, layout, dtype):
    print(f"append T={T_} Hq={Hq} Hkv={Hkv} D={D} rot={rot} page={page} {layout} {dtype}", flush=True)
    n_pages = 2 * T_ // page + 3
    fused = _randn(T_, Hq + 2 * Hkv, D, dtype=dtype)
    q, k, v = fused[:, :Hq], fused[:, Hq:Hq + Hkv], fused[:, Hq + Hkv:]
    g = torch.Generator().manual_seed(T_)
    slots = torch.randperm(n_pages * page, generator=g)[:T_].to(I32)
    slots[::5] = torch.tensor([-1, n_pages * page, -2 ** 31, 2 ** 31 - 1], dtype=I32)[torch.arange(len(slots[::5])) % 4]
    slots = slots.cuda()
    pos = torch.randint(0, 262144, (T_,), dtype=I32, device="cuda")
    freqs, gain = T.rope_frequencies(rot, 1e6, "by_parts", 4.0, 32768, device="cuda") if rot else (None, 1.0)
    for inputs in ((q, k, v), (q.contiguous(), k.contiguous(), v.contiguous())):
        kp, vp = (torch.full((n_pages, Hkv, page, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
        qo = torch.full((T_, Hq, D), 9.0, dtype=dtype, device="cuda")
        out = T.thrift_paged_append(inputs[1], inputs[2], slots, kp, vp, inputs[0], qo, pos, freqs, layout, gain)
        assert out is qo
        live = (slots >= 0) & (slots < n_pages * page)
        at = slots[live].long()
        flat = lambda p: p.transpose(1, 2).reshape(-1, Hkv, D)
        assert torch.equal(flat(vp)[at], v[live])
        if rot:
            for got, x in ((qo[live], q[live]), (flat(kp)[at], k[live])):
                if len(x):
                    want, err = rope64(x.transpose(0, 1).unsqueeze(0), pos[live].unsqueeze(0), freqs, layout, gain)
                    check_rounded(got.transpose(0, 1).unsqueeze(0), want, err)
        else:
            assert torch.equal(qo[live], q[live]) and torch.equal(flat(kp)[at], k[live])
        assert bool((qo[~live] == 9.0).all())
        rest = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
        rest[at] = False
        assert bool(torch.isnan(flat(kp)[rest]).all()) and bool(torch.isnan(flat(vp)[rest]).all())
    # without queries, the same pages; and the queries in place
    kp2, vp2 = (torch.full_like(kp, float("nan")) for _ in range(2))
    assert T.thrift_paged_append(k, v, slots, kp2, vp2, positions=pos, freqs=freqs, layout=layout, gain=gain) is None
    assert torch.equal(torch.nan_to_num(kp2), torch.nan_to_num(kp)) and torch.equal(torch.nan_to_num(vp2), torch.nan_to_num(vp))
    mine = q.contiguous()
    T.thrift_paged_append(k, v, slots, kp2, vp2, mine, mine, pos, freqs, layout, gain)
    assert torch.equal(mine[live], qo[live]) and torch.equal(mine[~live], q[~live])


def test_append_is_the_rotation_of_the_batch(T):
    """Rows of an append have the bits that thrift_rope gives the same heads."""
    q, k = _randn(1, 8, 50, 128, dtype=torch.bfloat16), _randn(1, 2, 50, 128, dtype=torch.bfloat16, seed=1)
    freqs, gain = T.rope_frequencies(128, 1e4, "by_parts", 2.0, 1000, device="cuda")
    for layout in LAYOUTS:
        a, b = T.thrift_rope(q, k, freqs, None, layout, gain)
        kp, vp = (torch.zeros(4, 2, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        n = torch.arange(50, dtype=I32, device="cuda")
        got = T.thrift_paged_append(k[0].transpose(0, 1), k[0].transpose(0, 1), n, kp, vp, q[0].transpose(0, 1), None, n, freqs, layout, gain)
        assert torch.equal(got, a[0].transpose(0, 1))
        assert torch.equal(kp.transpose(0, 1).reshape(2, -1, 128)[:, :50], b[0])


# ---- attention ----

def _cache(B, Hkv, D, page, width, dtype, lens, seed=0, garbage=float("nan"), spare=3):
    """Pages in random order; whatever lies past the lengths is `garbage`, table entries past them name nothing."""
    g = torch.Generator().manual_seed(seed)
    n_pages = B * width + spare
    table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).to(I32)
    kp, vp = _randn(n_pages, Hkv, page, D, dtype=dtype, seed=seed), _randn(n_pages, Hkv, page, D, dtype=dtype, seed=seed + 1)
    live = torch.zeros(n_pages, page, dtype=torch.bool)
    for b, n in enumerate(lens):
        n = min(max(n, 0), width * page)
        for j in range(-(-n // page)):
            live[table[b, j], :min(page, n - j * page)] = True
        table[b, -(-n // page):] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, n_pages], dtype=I32)[torch.arange(width - -(-n // page)) % 4]
    dead = ~live.cuda()
    for p in (kp, vp):
        p.transpose(1, 2)[dead] = garbage
    return kp, vp, table.cuda()


def _check_attention(T, q, kp, vp, table, lens, scale=0.0):
    B, Hq, D = q.shape
    sl = _ints(lens)
    real = scale if scale > 0 else 1 / math.sqrt(D)
    lens = [min(max(n, 0), table.shape[1] * kp.shape[2]) for n in lens]
    want, lse, eo, el = attention64(q, kp, vp, table, lens, real)
    for dt in (torch.float32, q.dtype):
        got, glse = T.thrift_paged_decode(q, kp, vp, table, sl, scale, out_dtype=dt, return_lse=True)
        check_rounded(got, want, eo)
        finite = torch.isfinite(lse)
        assert torch.equal(finite, torch.isfinite(glse)) and bool((glse[~finite] == -math.inf).all())
        assert bool(((glse.double() - lse)[finite].abs() <= el[finite]).all())
    return got


LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 255, 256, 257, 300]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (32, 4), (7, 1), (32, 1), (3, 3), (40, 2), (17, 1)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("room", [300, 1300])                  # of the block table: a workgroup per row, or shares
def test_attention_against_64_bits(T, D, Hq, Hkv, dtype, room):
    for page in (16, 64, 256):
        print(f"paged D={D} Hq={Hq} Hkv={Hkv} page={page} room={room} {dtype}", flush=True)
        width = -(-room // page)
        kp, vp, table = _cache(len(LENS), Hkv, D, page, width, dtype, LENS, seed=page)
        q = _randn(len(LENS), Hq, D, dtype=dtype, seed=9)
        _check_attention(T, q, kp, vp, table, LENS)


@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -65504.0])
@pytest.mark.parametrize("width", [2, 40])
def test_what_lies_past_the_length_reaches_no_result(T, page, garbage, width):
    for lens in ([1], [page + 1, width * page - 1], [0, 0, 0], [2 * page, 10 ** 9, -1]):
        kp, vp, table = _cache(len(lens), 2, 128, page, width, torch.float16, lens, seed=page, garbage=garbage)
        q = _randn(len(lens), 8, 128, dtype=torch.float16, seed=3)
        print(f"past the length page={page} lens={lens} garbage={garbage}", flush=True)
        _check_attention(T, q, kp, vp, table, lens)


@pytest.mark.parametrize("B,Hq,Hkv,top", [(1, 32, 8, 5000), (1, 8, 8, 20000), (2, 64, 8, 9000), (5, 16, 16, 3000), (33, 8, 1, 2000), (1, 1, 1, 70000), (300, 4, 2, 100), (1, 32, 1, 33000)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_ragged_and_long_sequences(T, B, Hq, Hkv, top, dtype):
    rng = random.Random(B * top)
    lens = [top] + [int(math.exp(rng.uniform(0, math.log(top)))) for _ in range(B - 1)]
    page = rng.choice((16, 32, 64))
    print(f"ragged B={B} Hq={Hq} Hkv={Hkv} page={page} lens={lens[:8]} {dtype}", flush=True)
    kp, vp, table = _cache(B, Hkv, 128, page, -(-top // page) + 2, dtype, lens, seed=B, spare=1)
    _check_attention(T, _randn(B, Hq, 128, dtype=dtype, seed=4), kp, vp, table, lens)


def _few_lengths(B, kind):
    if kind == "one far behind":                          # nothing in front of it
        return [0] * (B - 2) + [40, 0]
    if kind == "the last":
        return [0] * (B - 1) + [41]
    if kind == "gaps":                                    # some sequences with tokens, hundreds without between them
        return [(33 if b % 700 in (5, 6) else 0) for b in range(B)]
    return [(b * 7) % 41 for b in range(B)]               # all kinds of short ones


@pytest.mark.parametrize("B", [64, 65, 129, 4096, 4097, 9000])
@pytest.mark.parametrize("kind", ["one far behind", "the last", "gaps", "short"])
def test_many_sequences(T, B, kind):
    lens = _few_lengths(B, kind)
    print(f"many sequences B={B} {kind}", flush=True)
    page, Hkv, D = 16, 1, 64
    k, v = _randn(8, Hkv, page, D, dtype=torch.float16), _randn(8, Hkv, page, D, dtype=torch.float16, seed=1)
    table = (torch.arange(B * 3, device="cuda").view(B, 3) * 5 % 8).to(I32)
    q = _randn(B, 2, D, dtype=torch.float16, seed=2)
    got, lse = T.thrift_paged_decode(q, k, v, table, _ints(lens), out_dtype=torch.float32, return_lse=True)
    n = torch.tensor(lens, device="cuda")
    keys, values = (p[table.long()].transpose(1, 2).reshape(B, 3 * page, D).double() for p in (k, v))
    s = torch.bmm(q.double(), keys.transpose(1, 2).contiguous()) / math.sqrt(D)
    s = s.masked_fill(torch.arange(3 * page, device="cuda") >= n.view(B, 1, 1), -math.inf)
    live = n > 0
    want = torch.bmm(torch.softmax(s[live], -1), values[live])
    # as in attention64: scores of 64 products below 30, 40 keys
    assert bool(((got[live].double() - want).abs() <= 2 ** -15 * values.abs().amax()).all())
    assert bool(((lse[live].double() - torch.logsumexp(s[live], -1)).abs() <= 2 ** -15).all())
    assert bool((got[~live] == 0).all()) and bool((lse[~live] == -math.inf).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gain", [0.01, 30.0])
@pytest.mark.parametrize("lens", [[700, 64, 1, 333], [500, 64, 1, 333]])
def test_flat_and_peaked_scores(T, dtype, gain, lens):
    kp, vp, table = _cache(4, 2, 128, 32, -(-lens[0] // 32), dtype, lens, seed=6)
    q = (_randn(4, 8, 128, dtype=torch.float32, seed=7) * gain).to(dtype)
    _check_attention(T, q, kp, vp, table, lens)
    _check_attention(T, q, kp, vp, table, lens, scale=0.3)
    # scores that fall and that rise along the sequence, by far more than exp can hold
    for sign in (1.0, -1.0):
        kp2 = kp.clone()
        for b, n in enumerate(lens):
            held = table[b, :-(-n // 32)].long()
            ramp = sign * torch.arange(len(held) * 32, device="cuda").view(-1, 1, 32, 1) / 8.0
            kp2[held] = (ramp * torch.ones(128, device="cuda") / 8.0).to(dtype).expand(-1, 2, -1, -1)
            live = torch.arange(len(held) * 32, device="cuda").view(-1, 1, 32, 1) < n
            kp2[held] = torch.where(live, kp2[held], float("nan"))
        _check_attention(T, q.abs(), kp2, vp, table, lens)


@pytest.mark.parametrize("width", [6, 60])
def test_the_largest_values(T, width):
    """Values near the end of bfloat16's range: a mean of them is one of them, whatever the sums are scaled by in between."""
    kp, vp, table = _cache(1, 1, 128, 16, width, torch.bfloat16, [90], seed=8)
    live = ~torch.isnan(vp)
    vp[live] = torch.where(vp[live] > 0, 1.0, -1.0).to(torch.bfloat16) * 2.0 ** 120
    q = _randn(1, 2, 128, dtype=torch.bfloat16, seed=3)
    _check_attention(T, q, kp, vp, table, [90])


@pytest.mark.parametrize("width", [6, 60])
def test_scores_of_minus_infinity_weigh_nothing(T, width):
    """Keys whose product with the query overflows downwards, a whole step of them first."""
    kp, vp, table = _cache(1, 1, 128, 16, width, torch.bfloat16, [90], seed=8)
    q = torch.ones(1, 2, 128, dtype=torch.bfloat16, device="cuda")
    for j in range(4):
        kp[table[0, j].long()] = -3e37
    out, lse = T.thrift_paged_decode(q, kp, vp, table, _ints([90]), out_dtype=torch.float32, return_lse=True)
    k, v = (tokens(p, table[0], 90)[0, 64:].double() for p in (kp, vp))
    s = (q[0].double() @ k.t().contiguous()) / math.sqrt(128)
    want = torch.softmax(s, -1) @ v
    # fp32 sums of 128 products of about 1 (attention64 gives 2^-15 of the values)
    assert bool(((out[0].double() - want).abs() <= 2 ** -14 * v.abs().amax()).all())
    assert bool(((lse[0].double() - torch.logsumexp(s, -1)).abs() <= 2 ** -14).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [6, 60])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("a", [900.0, 1100.0, 2000.0, 4000.0, 28672.0])
def test_scores_past_24_bits(T, dtype, width, sign, a):
    """Scores from 2^23 to 2^33 (in powers of two), where fp32's neighbours are up to hundreds apart: keys with the largest one share the
    weight, the others have none."""
    lens, D, Hkv = [90, 1, 33, 64], 128, 2
    kp, vp, table = _cache(4, Hkv, D, 16, width, dtype, lens, seed=12)
    a = float(torch.tensor(a).to(dtype))
    q = torch.full((4, 2 * Hkv, D), a, dtype=dtype, device="cuda")
    winners = [[0, 31, 32, 77, 89], [0], [32], list(range(64))]
    low, high = (a / 2, a) if sign > 0 else (-a, -a / 2)
    want = torch.empty(4, Hkv, D, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        held = table[b, : -(-n // 16)].long()
        place = torch.arange(len(held) * 16, device="cuda")
        best = torch.isin(place, torch.tensor(winners[b], device="cuda"))
        rows = torch.where(best, high, low).where(place < n, float("nan")).to(dtype)
        kp[held] = rows.view(-1, 1, 16, 1).expand(-1, Hkv, -1, D)
        want[b] = tokens(vp, table[b], n).double()[:, winners[b]].mean(1)
    out, lse = T.thrift_paged_decode(q, kp, vp, table, _ints(lens), out_dtype=torch.float32, return_lse=True)
    # a^2 has at most 17 bits from its first to its last one, so that every sum of up to 128 of them is an fp32 number: the largest scores are
    # equal in the kernel, and the others 2^22 and more below.  P is 1 or 0; at most 64 values are added, each partial sum off by half a
    # step of at most 64 times the largest, and the reciprocal of their number and the product with it follow: 66 U of the largest
    top = vp[~torch.isnan(vp)].double().abs().max()
    assert bool(((out.view(4, Hkv, 2, D).double() - want.unsqueeze(2)).abs() <= 66 * 2.0 ** -24 * top).all())
    # eight roundings: root and quotient of the scale, log2(e), their product, the score's product, the sum with log2(n), ln 2, its product
    n = torch.tensor([len(w) for w in winners], dtype=torch.float64, device="cuda")
    exact = D * a * high / math.sqrt(D) + n.log()
    assert bool(((lse.double() - exact.unsqueeze(1)).abs() <= 8 * 2.0 ** -24 * exact.abs().unsqueeze(1)).all())


def test_the_same_page_twice(T):
    """Sequences that share their first pages, and a table that names a page twice."""
    kp, vp, table = _cache(3, 2, 128, 16, 6, torch.bfloat16, [96, 96, 96], seed=8)
    table[1, :3] = table[0, :3]
    table[2, 4] = table[2, 1]
    _check_attention(T, _randn(3, 8, 128, dtype=torch.bfloat16, seed=8), kp, vp, table, [90, 77, 96])


def test_bad_table_entries_are_not_followed(T):
    """Entries within the length that name no page: any numbers, but nothing outside the pages is read."""
    kp, vp, table = _cache(2, 2, 128, 16, 6, torch.float16, [96, 96], seed=9)
    table[0, 2], table[1, 0], table[1, 5] = -1, 2 ** 31 - 1, -2 ** 31
    out = T.thrift_paged_decode(_randn(2, 8, 128, dtype=torch.float16), kp, vp, table, _ints([96, 96]))
    assert out.shape == (2, 8, 128)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [6, 60])
def test_bad_table_entries_are_clamped(T, dtype, width):
    """The result is that of the table with its entries clamped to the pages, bit for bit, in both forms."""
    lens = [96, 90, 17]
    kp, vp, table = _cache(3, 2, 128, 16, width, dtype, lens, seed=9, garbage=0.5)
    table[0, 2], table[1, 0], table[1, 5], table[2, 1] = -1, 2 ** 31 - 1, -2 ** 31, kp.shape[0]
    q = _randn(3, 8, 128, dtype=dtype)
    print(f"bad entries width={width} {dtype}", flush=True)
    got = T.thrift_paged_decode(q, kp, vp, table, _ints(lens), out_dtype=torch.float32, return_lse=True)
    want = T.thrift_paged_decode(q, kp, vp, table.clamp(0, kp.shape[0] - 1), _ints(lens), out_dtype=torch.float32, return_lse=True)
    assert all(torch.equal(a, b) and bool(torch.isfinite(a).all()) for a, b in zip(got, want))


def test_offsets_past_32_bits(T):
    """Pages whose elements lie past 2^31 (and bytes past 2^32)."""
    Hkv, page, D = 8, 128, 128
    n_pages = (2 ** 31 + 2 ** 29) // (Hkv * page * D)
    kp, vp = (torch.empty(n_pages, Hkv, page, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    far = torch.tensor([n_pages - 1, n_pages - 3, 0, 2 ** 31 // (Hkv * page * D)], device="cuda")
    kp[far], vp[far] = _randn(4, Hkv, page, D, dtype=torch.bfloat16), _randn(4, Hkv, page, D, dtype=torch.bfloat16, seed=1)
    table = far.to(I32).view(1, 4)
    q = _randn(1, 16, D, dtype=torch.bfloat16, seed=2)
    _check_attention(T, q, kp, vp, table, [4 * page - 5])
    k, v = _randn(4, Hkv, D, dtype=torch.bfloat16, seed=3), _randn(4, Hkv, D, dtype=torch.bfloat16, seed=4)
    T.thrift_paged_append(k, v, (far * page + 7).to(I32), kp, vp)
    assert torch.equal(kp[far, :, 7], k) and torch.equal(vp[far, :, 7], v)
    _check_attention(T, q, kp, vp, table, [4 * page])


@pytest.mark.parametrize("dtype,lens", [(torch.bfloat16, [2 ** 31 - 16 - 15, 37]), (torch.float16, [70, 2 ** 31 - 1])])
def test_the_longest_block_table(T, dtype, lens):
    """A table of 2^31 - 16 tokens that names four pages over and over; lengths whose last steps end past 2^31, a short sequence beside."""
    D, page, width = 64, 16, 2 ** 27 - 1
    kp = _randn(4, 1, page, D, dtype=dtype)
    vp = torch.randint(-4, 5, (4, 1, page, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    table = torch.arange(width, dtype=I32, device="cuda").remainder_(4).expand(2, width).contiguous()
    print(f"longest table {dtype} {lens}", flush=True)
    # queries of 0 weigh all keys alike: a wavefront's sums of 2^21 values of at most 4 are exact
    out, lse = T.thrift_paged_decode(torch.zeros(2, 1, D, dtype=dtype, device="cuda"), kp, vp, table, _ints(lens), out_dtype=torch.float32, return_lse=True)
    for b, n in enumerate(min(n, width * page) for n in lens):
        count = torch.tensor([n // 64 + (j < n % 64) for j in range(64)], dtype=torch.float64, device="cuda")
        want = (count.unsqueeze(1) * vp.view(64, D).double()).sum(0) / n
        # the parts of 4 wavefronts and 256 shares: 260 additions each in the sums of values (half a step of at most 4 n) and of weights
        assert bool(((out[b, 0].double() - want).abs() <= 4 * (2 * 260 + 4) * 2.0 ** -24).all())
        assert abs(float(lse[b, 0]) - math.log(n)) <= (260 + 4 * math.log(n)) * 2.0 ** -24


def test_streams_workspaces_and_replays(T):
    """Calls at the same time on two streams with workspaces of their own; a captured call replayed between eager ones with other
    lengths; two captured calls that share one workspace, replayed in turn."""
    lens = [900, 3, 0, 517]
    kp, vp, table = _cache(4, 2, 128, 16, 60, torch.float16, [960] * 4, seed=11)
    q = _randn(4, 8, 128, dtype=torch.float16, seed=12)
    sl = _ints(lens)
    one = lambda **kw: T.thrift_paged_decode(q, kp, vp, table, sl, **kw)
    want = one()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            results.append([one() for _ in range(20)])
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for rs in results for r in rs)
    size = T.paged_decode_workspace_bytes(4, 8, 2, 60, 16, 128)
    assert size > 0
    shared = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        out = torch.empty(4, 8, 128, dtype=torch.float16, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            one(out=out, workspace=shared)
        graphs.append(g), outs.append(out)
    for i, lens in enumerate(([900, 3, 0, 517], [1, 960, 33, 0], [0, 0, 0, 0], [960, 959, 16, 17])):
        sl.copy_(_ints(lens))
        want = one()
        torch.cuda.synchronize()
        for g, out in zip(graphs, outs):
            out.fill_(3)
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs), i


# ---- all together ----

def test_a_captured_step_replayed(T):
    """Map, append and attention of one token per request captured once; every replay moves the pool on as an eager step on a copy of
    it does, with eager work in between, until pages run out."""
    B, Hq, Hkv, D, page, dtype = 5, 8, 2, 128, 16, torch.float16
    freqs, gain = T.rope_frequencies(D, 1e4, device="cuda")

    class Server:
        def __init__(self):
            self.table = T.PageTable(B, 80, page, 21, "cuda")             # 21 pages: a few steps in, some request gets none
            self.cache = T.PagedKVCache(self.table, Hkv, D, dtype)
            self.x = torch.empty(B, Hq + 2 * Hkv, D, dtype=dtype, device="cuda")
            self.new = torch.ones(B, dtype=I32, device="cuda")
            self.seqlens, self.count = _ints([30, 0, 47, 79, 111]), _ints([0])
            held = [2, 0, 3, 5, 7]
            pages = list(range(20, -1, -1))
            for b, n in enumerate(held):
                self.table.block_table[b, :n] = _ints([pages.pop() for _ in range(n)])
            self.table.free_pages[:len(pages)] = _ints(pages)
            self.count.fill_(len(pages))
            for i, p in enumerate((self.cache.k_pages, self.cache.v_pages)):
                p.copy_(_randn(*p.shape, dtype=dtype, seed=40 + i))

        def step(self):
            t = self.table
            t.seqlens, t.free_count = self.seqlens, self.count
            m = t.map(self.new, B + 3)
            x = torch.cat([self.x, torch.zeros(3, Hq + 2 * Hkv, D, dtype=dtype, device="cuda")])
            q = self.cache.append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], m, x[:, :Hq], freqs, "half", gain, q_out=torch.zeros(B + 3, Hq, D, dtype=dtype, device="cuda"))
            out, lse = self.cache.decode(q[:B], return_lse=True)
            self.seqlens.copy_(m.seqlens)
            self.count.copy_(m.free_count)
            return [out, lse, m.slots, m.positions, m.starts]

        def state(self):
            return [self.seqlens, self.count, self.table.block_table, self.cache.k_pages, self.cache.v_pages]

    eager, captured = Server(), Server()
    eager.x.copy_(_randn(*eager.x.shape, dtype=dtype, seed=1)), captured.x.copy_(eager.x)
    eager.step(), captured.step()                                         # (the capture's warm-up)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results = captured.step()
    refused = 0
    for i in range(24):
        x = _randn(*eager.x.shape, dtype=dtype, seed=100 + i)
        eager.x.copy_(x), captured.x.copy_(x)
        want = eager.step()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results + captured.state(), want + eager.state()):
            assert torch.equal(a, b), i
        refused += int((want[2][:B] < 0).sum())
    assert refused > 0 and int(eager.count) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
def test_a_servers_steps(T, dtype, layout):
    """Prompts of several requests, then tokens one by one, requests that end and others that take their pages: the attention of every
    step is that over the tokens the request has had, and that of the prompts' last rows is thrift_attention's at a 16-bit budget."""
    B, Hq, Hkv, D, page = 4, 8, 2, 128, 16
    table = T.PageTable(B, 40, page, 90, "cuda")
    cache = T.PagedKVCache(table, Hkv, D, dtype)
    cache.k_pages.fill_(float("nan")), cache.v_pages.fill_(float("nan"))
    freqs, gain = T.rope_frequencies(D, 1e4, "by_parts", 2.0, 512, device="cuda")
    rng = random.Random(5)
    past = [None] * B                                     # (q, k, v) [H, n, D] as given, unrotated
    for step in range(14):
        new = [rng.randint(100, 300) if past[b] is None else (0 if step == 7 and b == 2 else 1) for b in range(B)]
        rows = sum(new) + rng.choice((0, 7))
        x = _randn(rows, Hq + 2 * Hkv, D, dtype=dtype, seed=step)
        m = table.map(_ints(new), rows)
        q = cache.append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], m, x[:, :Hq], freqs, layout, gain, q_out=torch.zeros(rows, Hq, D, dtype=dtype, device="cuda"))
        starts = m.starts.tolist()
        assert starts == [sum(new[:b]) for b in range(B + 1)]
        last = (m.starts[1:].long() - 1).clamp(min=0)
        lens = table.seqlens.tolist()
        out = cache.decode(q[last], out_dtype=torch.float32)
        for b in range(B):
            own = [t[starts[b]:starts[b + 1]].transpose(0, 1) for t in (x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])]
            past[b] = own if past[b] is None else [torch.cat([p, t], 1) for p, t in zip(past[b], own)]
            n = past[b][1].shape[1]
            assert lens[b] == n, (step, b)
            if new[b] == 0:
                continue
            qr, kr = T.thrift_rope(past[b][0].unsqueeze(0).contiguous(), past[b][1].unsqueeze(0).contiguous(), freqs, None, layout, gain)
            v = past[b][2].unsqueeze(0).contiguous()
            # the heads have the same bits on both ways, so only the attention's arithmetic is left (one page of n tokens here)
            want, _, bound, _ = attention64(qr[:, :, -1], kr, v, _ints([[0]]), [n], 1 / math.sqrt(D))
            check_rounded(out[b:b + 1], want, bound)
            if new[b] > 1:
                full = T.thrift_attention(qr, kr, v, budget=1.0, out_dtype=torch.float32)[0, :, -1]
                assert float((full - out[b]).abs().max()) <= 2e-3, (step, b)           # its tolerance for all-16-bit runs
        drop = [int(step % 4 == 3 and rng.random() < 0.5) for _ in range(B)]
        table.release(_ints(drop))
        for b in range(B):
            if drop[b]:
                past[b] = None


def test_the_general_path_gives_the_same_results(T, monkeypatch):
    """Without the module _call, and for what it does not serve, the calls go through ctypes."""
    q, k = _randn(2, 4, 9, 128, dtype=torch.float16), _randn(2, 2, 9, 128, dtype=torch.float16, seed=1)
    freqs, gain = T.rope_frequencies(64, 1e4, "by_parts", 2.0, 512, device="cuda")
    rows = k.transpose(1, 2).reshape(18, 2, 128)
    lens = _ints([0, 40])

    def results():
        table = T.PageTable(2, 8, 16, 16, "cuda")
        cache = T.PagedKVCache(table, 2, 128, torch.float16)
        m = table.map(_ints([9, 9]), 20)
        rest = torch.zeros(2, 2, 128, dtype=torch.float16, device="cuda")
        x = torch.cat([rows, rest])
        kq = cache.append(x, x, m, x, freqs, "interleaved", gain, q_out=torch.zeros(20, 2, 128, dtype=torch.float16, device="cuda"))
        assert cache.append(x, x, m, None, freqs, "half", gain) is None
        out, lse = cache.decode(q[:, :, 0].contiguous(), return_lse=True)
        own = torch.empty(2, 4, dtype=torch.float32, device="cuda")
        again = cache.decode(q[:, :, 0].contiguous(), out=torch.empty(2, 4, 128, dtype=torch.float32, device="cuda"), lse=own)
        into = torch.empty(2, 9, 4, 128, dtype=torch.float16, device="cuda").transpose(1, 2)
        return [*T.thrift_rope(q, k, freqs, None, "half", gain), *T.thrift_rope_backward(q, k, freqs, lens[:1].expand(9).contiguous(), "interleaved", gain, q_out=into),
                T.thrift_rope(q, None, freqs)[0], *m, kq, out, lse, again, own, table.seqlens, table.free_count]

    want = results()
    monkeypatch.setattr(T, "_call", T._General)
    for i, (a, b) in enumerate(zip(results(), want)):
        assert torch.equal(a, b), i
    with pytest.raises(AssertionError):
        T.thrift_rope(q, k.float(), freqs)


def test_the_module_leaves_other_arguments_to_the_general_path(T):
    m = T._native()
    q = torch.zeros(1, 2, 3, 128, dtype=torch.float16, device="cuda")
    freqs = torch.zeros(64, dtype=torch.float64, device="cuda")
    one = lambda **kw: m.rope(*{**dict(backward=0, q=q, k=None, freqs=freqs, positions=None, layout=0, gain=1.0, qo=None, ko=None, device=0, stream=0), **kw}.values())
    assert isinstance(one(), tuple)
    for bad in (dict(device=1), dict(q=q.float()), dict(q=q.cpu()), dict(q=q[0]), dict(k=q[:, :, :2]), dict(freqs=freqs.float()), dict(positions=torch.zeros(2, dtype=I32, device="cuda")),
                dict(qo=q[:, :1].expand(1, 2, 3, 128)), dict(qo=q.bfloat16()), dict(ko=q), dict(q=q.transpose(2, 3)), dict(layout="half"), dict(q=q[:0])):
        assert one(**bad) is None, bad
    assert one(layout=5) == 2 and one(freqs=torch.zeros(65, dtype=torch.float64, device="cuda")) == 2
    pages = torch.zeros(4, 2, 16, 128, dtype=torch.float16, device="cuda")
    k, slots, table, lens = torch.zeros(3, 2, 128, dtype=torch.float16, device="cuda"), _ints([0, 1, 2]), _ints([[0], [1], [2]]), _ints([1, 1, 1])
    assert m.paged_append(k, k, slots, pages, pages, None, None, None, None, 0, 1.0, 0, 0) is True
    assert m.paged_append(k, k, slots, pages, pages, None, None, None, None, 0, 1.0, 1, 0) is None
    assert m.paged_append(k, k, slots, pages, pages[:, :1], None, None, None, None, 0, 1.0, 0, 0) is None
    assert m.paged_append(k, k, slots.long(), pages, pages, None, None, None, None, 0, 1.0, 0, 0) is None
    assert m.paged_append(k, k, slots, pages, pages, None, None, None, freqs, 0, 1.0, 0, 0) is None
    assert m.paged_decode(k, pages, pages, table, lens, 0.0, None, None, 0, None, 1, 0) is None
    assert m.paged_decode(k, pages, pages, table[:2], lens, 0.0, None, None, 0, None, 0, 0) is None
    wide = torch.zeros(3, 100, dtype=I32, device="cuda")
    assert m.paged_decode(k, pages, pages, wide, lens, 0.0, None, None, 0, torch.empty(16, dtype=torch.uint8, device="cuda"), 0, 0) == 5
    assert m.paged_decode(k, pages, pages, table, lens, 0.0, None, None, 0, torch.empty(0, dtype=torch.uint8, device="cuda"), 0, 0).shape == (3, 2, 128)
    assert m.page_map(lens, lens, table, slots, lens[:1], 16, 4, 3, 1, 0) is None and m.page_map(lens, lens, table, slots, lens, 16, 4, 3, 0, 0) is None
    assert m.page_map(lens, lens, table, slots, lens[:1], 17, 4, 3, 0, 0) == 2 and len(m.page_map(lens, lens, table, slots, lens[:1], 16, 4, 3, 0, 0)) == 5


def test_the_steps_that_the_readme_shows(T):
    import os
    readme = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = readme.split("```python\n")[1].split("```")[0]
    B, Hq, Hkv, D, rows = 3, 8, 2, 128, 3
    names = dict(T=T, torch=torch, B=B, max_pages=8, page_size=16, n_pages=30, Hkv=Hkv, D=D, rows=rows, new_lens=torch.ones(B, dtype=I32, device="cuda"),
                 q=_randn(rows, Hq, D, dtype=torch.bfloat16), k=_randn(rows, Hkv, D, dtype=torch.bfloat16), v=_randn(rows, Hkv, D, dtype=torch.bfloat16, seed=1),
                 ended=_ints([0, 1, 0]))
    exec(code, names)
    # the first token of every request attends to itself alone
    assert torch.equal(names["out"], names["v"].repeat_interleave(Hq // Hkv, 1))
    assert names["table"].seqlens.tolist() == [1, 0, 1] and names["table"].free_count.tolist() == [28]

"""The 8-bit paged cache on the GPU: appends against the format in 64 bits, rows read back bit for bit, attention against 64 bits, and a
server's steps with all of them."""
import math

import pytest
import torch

from tests.paged8_util import cache8, exponent64, codes64, power64, quantise64, values64
from tests.paged_util import LAYOUTS, attention64, check_rounded, half_step, rope64
from tests.test_gpu_paged import DTYPES, I32, LENS, _cache, _few_lengths, _ints, _randn

pytestmark = pytest.mark.gpu
U8 = torch.uint8


@pytest.fixture(scope="module")
def T():
    from paper_2605_23081_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


# ---- appends ----

def _pages8(n_pages, Hkv, page, D, fill=0xab):
    return [torch.full(s, fill, dtype=U8, device="cuda") for s in ((n_pages, Hkv, page, D), (n_pages, Hkv, page)) * 2]


def _check_codes(codes, scales, want, err):
    """The bytes of heads `want` [..., D] known up to err: a scale between those of the ends, and codes between those of the ends at it."""
    assert bool(((scales.long() - 127 >= exponent64((want.abs() - err).amax(-1))) & (scales.long() - 127 <= exponent64((want.abs() + err).amax(-1)))).all())
    inv = power64(127 - scales.long()).unsqueeze(-1)
    value = values64(codes, None)
    low, high = (values64(codes64(((want + s * err) * inv).clamp(-448, 448)), None) for s in (-1, 1))
    assert bool(((value >= low) & (value <= high)).all())


@pytest.mark.parametrize("T_,Hq,Hkv,D,rot,page", [(1, 32, 8, 128, 128, 16), (37, 6, 2, 128, 64, 32), (5, 3, 3, 64, 64, 256), (130, 8, 1, 256, 256, 64), (9, 2, 1, 96, 40, 16),
                                                  (7, 4, 2, 128, 0, 16), (3, 1, 1, 2, 2, 16), (6, 2, 2, 1024, 512, 16), (11, 2, 2, 34, 6, 32), (600, 8, 2, 128, 128, 128),
                                                  (2, 5, 5, 16, 16, 16), (40, 1, 1, 512, 48, 16), (33, 2, 3, 32, 32, 64), (8, 2, 2, 144, 144, 16)])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_append_against_64_bits(T, T_, Hq, Hkv, D, rot, page, layout, dtype):
    print(f"append8 T={T_} Hq={Hq} Hkv={Hkv} D={D} rot={rot} page={page} {layout} {dtype}", flush=True)
    n_pages = -(-2 * T_ // page) + 1
    g = torch.Generator().manual_seed(T_)
    x = _randn(T_, Hq + 2 * Hkv, D, dtype=dtype, seed=T_) * _randn(T_, Hq + 2 * Hkv, 1, dtype=dtype, seed=7).exp()
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    slots = torch.randperm(n_pages * page, generator=g)[:T_].to(I32)
    slots[T_ // 3::5] = torch.tensor([-1, n_pages * page, -2 ** 31, 2 ** 31 - 1], dtype=I32)[torch.arange(len(slots[T_ // 3::5])) % 4]
    if T_ == 1:
        slots[0] = 5
    live = ((slots >= 0) & (slots < n_pages * page)).cuda()
    positions = torch.randint(0, 131072, (T_,), generator=g).to(I32).cuda()
    freqs, gain = T.rope_frequencies(rot, 1e4, "by_parts", 2.0, 4096, device="cuda") if rot else (None, 1.0)
    pages = _pages8(n_pages, Hkv, page, D)
    before = torch.full((T_, Hq, D), 3.0, dtype=dtype, device="cuda")
    q_out = T.thrift_paged_append8(k, v, slots.cuda(), *pages, q=q, q_out=before.clone(), positions=positions, freqs=freqs, layout=layout, gain=gain)
    assert torch.equal(q_out[~live], before[~live])
    none = torch.zeros(rot // 2, dtype=torch.float64, device="cuda") if rot == 0 else freqs
    wq, eq = rope64(q.transpose(0, 1).unsqueeze(0), positions.unsqueeze(0), none, layout, gain)
    wk, ek = rope64(k.transpose(0, 1).unsqueeze(0), positions.unsqueeze(0), none, layout, gain)
    if rot == 0:
        assert torch.equal(q_out[live], q[live])
    else:
        check_rounded(q_out[live], wq[0].transpose(0, 1)[live], eq[0].transpose(0, 1)[live])
    to = slots.cuda()[live].long()
    rows = [p.transpose(1, 2).reshape(n_pages * page, Hkv, *p.shape[3:]) for p in pages]
    _check_codes(rows[0][to], rows[1][to], wk[0].transpose(0, 1)[live], ek[0].transpose(0, 1)[live])
    codes, scales, _ = quantise64(v[live])                                   # what is not turned has one answer
    assert torch.equal(rows[2][to], codes) and torch.equal(rows[3][to], scales)
    rest = torch.ones(n_pages * page, dtype=torch.bool, device="cuda")
    rest[to] = False
    assert all(bool((p[rest] == 0xab).all()) for p in rows)


@pytest.mark.parametrize("T_,Hq,Hkv,D,rot,page", [(2100, 1, 1, 16, 16, 16), (5000, 2, 1, 32, 16, 32), (4097, 1, 2, 64, 64, 64), (1500, 8, 2, 128, 128, 16), (9001, 3, 1, 16, 0, 16), (2049, 4, 4, 256, 128, 16)])
@pytest.mark.parametrize("layout", LAYOUTS)
def test_append_of_many_tokens(T, T_, Hq, Hkv, D, rot, page, layout):
    """Workgroups of one token and, where its heads are few, of several."""
    test_append_against_64_bits(T, T_, Hq, Hkv, D, rot, page, layout, DTYPES[T_ % 2])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [128, 96])
def test_the_largest_the_smallest_and_no_numbers(T, dtype, D):
    """Zeros, numbers below the range of the scale, the largest, ties, infinities and NaN: the bytes of the reference."""
    finfo = torch.finfo(dtype)
    x = torch.zeros(12, 2, D, dtype=torch.float64)
    x[1] = finfo.smallest_normal / 4
    x[2, 0, 3] = finfo.max
    x[3, :, ::2] = -finfo.max
    x[4] = torch.linspace(-1, 1, D) * finfo.max
    x[5] = torch.arange(D) / 64 - 0.5                                        # ties among them
    x[6, 0, 5], x[6, 1, 0] = math.inf, -math.inf
    x[7, 0] = math.nan
    x[8], x[8, 1, 1] = 448.0, -1.0
    x[9], x[9, 0, 0] = 449.0, 2.0 ** -14
    x[10] = -0.0
    x[11] = 2.0 ** -12 * torch.arange(D)
    x = x.to(dtype).cuda()
    pages = _pages8(1, 2, 16, D)
    T.thrift_paged_append8(x, x, _ints(list(range(12))), *pages)
    codes, scales, _ = quantise64(x)
    for c, s in (pages[:2], pages[2:]):
        got, gs = c[0].transpose(0, 1)[:12], s[0].transpose(0, 1)[:12]
        assert torch.equal(gs, scales)
        nan = ~x.isfinite()
        assert torch.equal((got & 127) == 127, nan) and torch.equal(got[~nan], codes[~nan])
    # and back: what passes the type's range becomes its largest number
    k, v = T.thrift_paged_read8(*pages, _ints([[0]]), _ints([12]), 12, dtype)
    want = values64(codes, scales).clamp(-finfo.max, finfo.max).transpose(0, 1).unsqueeze(0)
    for y in (k, v):
        fine = ~want.isnan()
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y[fine].double(), want[fine].to(dtype).double())
        back = y[0].transpose(0, 1)
        err = (2.0 ** -4 + half_step(dtype)[0]) * x.double().abs() + torch.exp2(scales.double() - 127 - 10).unsqueeze(-1)
        sure = x.isfinite() & (x.double().abs() <= finfo.max / 2)
        assert bool(((back.double() - x.double()).abs() <= err)[sure].all())


def test_offsets_past_32_bits(T):
    """A cache whose last pages lie past 2^32 bytes: appended to, read back and attended to as a small one."""
    Hkv, D, page, n_pages = 8, 128, 64, 70000                                # 4.6 GB of codes each
    big, small = _pages8(n_pages, Hkv, page, D, 0), _pages8(6, Hkv, page, D, 0)
    k, v = (_randn(70, Hkv, D, dtype=torch.bfloat16, seed=i) for i in (1, 2))
    at = torch.arange(70)
    names = torch.tensor([n_pages - 1, n_pages - 5])
    T.thrift_paged_append8(k, v, (names[at // page] * page + at % page).to(I32).cuda(), *big)
    T.thrift_paged_append8(k, v, (torch.tensor([5, 1])[at // page] * page + at % page).to(I32).cuda(), *small)
    lens, q = _ints([70]), _randn(1, 16, D, dtype=torch.bfloat16, seed=3)
    tables = [names.to(I32).unsqueeze(0).cuda(), _ints([[5, 1]])]
    a, b = (T.thrift_paged_read8(*p, t, lens, 80) for p, t in zip((big, small), tables))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and bool(a[0].any())
    a, b = (T.thrift_paged_decode8(q, *p, t, lens) for p, t in zip((big, small), tables))
    assert torch.equal(a, b)
    zero = _ints([0])
    a, b = (T.thrift_paged_decode_prefix8(q, *p, t, lens, zero, lens) for p, t in zip((big, small), tables))
    assert torch.equal(a, b)


# ---- reading back ----

def _read64(pages, table, lens, first, N):
    """Tokens by plain indexing: [B, Hkv, N, ...], zeros where there is none."""
    n_pages, Hkv, page = pages.shape[:3]
    B, width = table.shape
    p = torch.arange(N, device="cuda") + torch.tensor([max(0, f) for f in first], device="cuda").unsqueeze(1)
    there = p < torch.tensor([min(max(n, 0), width * page) for n in lens], device="cuda").unsqueeze(1)
    names = table.long().gather(1, (p // page).clamp(max=width - 1))
    there &= (names >= 0) & (names < n_pages)
    rows = pages[names.clamp(0, n_pages - 1), :, p % page].transpose(1, 2)
    return torch.where(there.view(B, 1, N, *[1] * (rows.dim() - 3)), rows, 0)


@pytest.mark.parametrize("D", [128, 2, 6, 8, 64, 72, 256, 1000, 1024])
@pytest.mark.parametrize("N", [1, 7, 64, 301])
@pytest.mark.parametrize("page", [16, 128])
def test_read_is_a_copy(T, D, N, page):
    lens = [0, 1, page, page + 1, 300, -5, 10 ** 6]
    first = [0, 0, page - 1, 3, 17, 2, -4]
    Hkv, width = 3, -(-320 // page)
    for dtype in DTYPES:
        print(f"read D={D} N={N} page={page} {dtype}", flush=True)
        kp, vp, table = _cache(len(lens), Hkv, D, page, width, dtype, lens, seed=D)
        table[4, 1] = kp.shape[0]                                            # names no page: zeros
        for f in (None, first):
            k, v = T.thrift_paged_read(kp, vp, table, _ints(lens), N, None if f is None else _ints(f))
            for got, pages in ((k, kp), (v, vp)):
                want = _read64(pages.view(torch.int16), table, lens, f or [0] * len(lens), N)
                assert got.dtype == dtype and torch.equal(got.view(torch.int16), want)
        codes = [torch.randint(0, 256, s, dtype=U8, device="cuda") for s in ((*kp.shape,), (*kp.shape[:3],)) * 2]
        codes[1].clamp_(118, 136), codes[3].clamp_(100, 135)
        k, v = T.thrift_paged_read8(*codes, table, _ints(lens), N, dtype, _ints(first))
        for got, c, s in ((k, *codes[:2]), (v, *codes[2:])):
            want = _read64(values64(c, s), table, lens, first, N)
            fine = ~want.isnan()
            assert torch.equal(got.isnan(), ~fine)
            most = torch.finfo(dtype).max
            assert torch.equal(got[fine], want[fine].clamp(-most, most).to(dtype))


def test_read_takes_any_alignment_and_the_ends_of_its_range(T):
    D, Hkv, page = 64, 2, 16
    space = torch.zeros(2 * 5 * Hkv * page * D + 16, dtype=torch.float16, device="cuda")
    kp = space[3:3 + 5 * Hkv * page * D].view(5, Hkv, page, D)
    kp.copy_(_randn(*kp.shape, dtype=torch.float16))
    vp = kp.clone()
    table, lens = _ints([[3, 0], [1, 4]]), _ints([20, 32])
    out = torch.full((2 * 2 * 9 * D + 16,), 7.0, dtype=torch.float16, device="cuda")
    into = out[5:5 + 2 * 2 * 9 * D].view(2, 2, 9, D)
    for f in ([0, 0], [12, 30], [2 ** 31 - 1, -2 ** 31], [20, 32]):
        k, v = T.thrift_paged_read(kp, vp, table, lens, 9, _ints(f), k_out=into)
        want = _read64(kp, table, [20, 32], f, 9)
        assert k.data_ptr() == into.data_ptr() and torch.equal(into, want) and torch.equal(v, want)
        assert bool((out[:5] == 7).all()) and bool((out[-11:] == 7).all())
    codes, scales = torch.zeros(5 * Hkv * page * D + 8, dtype=U8, device="cuda"), torch.full((5, Hkv, page), 127, dtype=U8, device="cuda")
    odd = codes[1:1 + 5 * Hkv * page * D].view(5, Hkv, page, D)
    odd.copy_(torch.randint(0, 127, odd.shape, dtype=U8, device="cuda"))
    k, v = T.thrift_paged_read8(odd, scales, odd, scales, table, lens, 9, torch.float16)
    assert torch.equal(k.double(), _read64(values64(odd, scales), table, [20, 32], [0, 0], 9)) and torch.equal(k, v)


# ---- attention ----

def _cache_and_values(B, Hkv, D, page, width, lens, seed=0, garbage=True):
    """An 8-bit cache and the numbers it holds; past the lengths codes are NaN and scales stand for nothing."""
    kp, vp, table = _cache(B, Hkv, D, page, width, torch.bfloat16, lens, seed=seed, garbage=float("nan") if garbage else 1.0)
    for i, p in enumerate((kp, vp)):
        p.mul_((2 * _randn(*p.shape[:3], 1, dtype=torch.bfloat16, seed=seed + 5 + i)).exp() if i else (0.3 * _randn(*p.shape[:3], 1, dtype=torch.bfloat16, seed=seed + 5)).exp())
    pages = list(cache8(kp, vp))
    if garbage:
        for p, c, s in ((kp, 0, 1), (vp, 2, 3)):
            dead = p[..., 0].isnan()
            pages[c][dead], pages[s][dead] = 0x7f, 255
    return pages, values64(*pages[:2]), values64(*pages[2:]), table


def _check_attention(T, q, pages, kv, vv, table, lens, scale=0.0):
    D = q.shape[2]
    real = scale if scale > 0 else 1 / math.sqrt(D)
    clamped = [min(max(n, 0), table.shape[1] * kv.shape[2]) for n in lens]
    want, lse, eo, el = attention64(q, kv, vv, table, clamped, real)
    for dt in (torch.float32, q.dtype):
        got, glse = T.thrift_paged_decode8(q, *pages, table, _ints(lens), scale, out_dtype=dt, return_lse=True)
        check_rounded(got, want, eo)
        finite = torch.isfinite(lse)
        assert torch.equal(finite, torch.isfinite(glse)) and bool((glse[~finite] == -math.inf).all())
        assert bool(((glse.double() - lse)[finite].abs() <= el[finite]).all())
    return got


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (32, 4), (7, 1), (32, 1), (3, 3), (40, 2), (17, 1)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("room", [300, 2600])                  # of the block table
def test_attention_against_64_bits(T, D, Hq, Hkv, dtype, room):
    for page in (16, 64, 256):
        print(f"paged8 D={D} Hq={Hq} Hkv={Hkv} page={page} room={room} {dtype}", flush=True)
        width = -(-room // page)
        pages, kv, vv, table = _cache_and_values(len(LENS), Hkv, D, page, width, LENS, seed=page)
        _check_attention(T, _randn(len(LENS), Hq, D, dtype=dtype, seed=9), pages, kv, vv, table, LENS)


@pytest.mark.parametrize("B,Hq,Hkv,top", [(1, 32, 8, 5000), (1, 8, 8, 20000), (2, 64, 8, 9000), (5, 16, 16, 3000), (33, 8, 1, 2000), (1, 1, 1, 70000), (300, 4, 2, 100), (1, 32, 1, 33000)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_ragged_and_long_sequences(T, B, Hq, Hkv, top, dtype):
    print(f"paged8 ragged B={B} Hq={Hq} Hkv={Hkv} top={top} {dtype}", flush=True)
    g = torch.Generator().manual_seed(B)
    lens = [top] + torch.randint(0, top + 1, (B - 1,), generator=g).tolist()
    D, page = 128, 32
    pages, kv, vv, table = _cache_and_values(B, Hkv, D, page, -(-top // page), lens, seed=B)
    _check_attention(T, _randn(B, Hq, D, dtype=dtype, seed=9), pages, kv, vv, table, lens)


@pytest.mark.parametrize("B", [64, 65, 4097])
@pytest.mark.parametrize("kind", ["one far behind", "the last", "gaps", "short"])
def test_many_sequences(T, B, kind):
    lens = _few_lengths(B, kind)
    print(f"paged8 many B={B} {kind}", flush=True)
    D, page = 64, 16
    width = -(-max(lens) // page) + 1
    pages = 40                                                               # shared by all: what is read is the same wherever the pages are
    table = torch.randint(0, pages, (B, width), generator=torch.Generator().manual_seed(B)).to(I32).cuda()
    kp, vp = (_randn(pages, 1, page, D, dtype=torch.float16, seed=i) for i in (1, 2))
    bytes8 = cache8(kp, vp)
    q = _randn(B, 2, D, dtype=torch.float16, seed=3)
    got = T.thrift_paged_decode8(q, *bytes8, table, _ints(lens), out_dtype=torch.float32)
    some = sorted({0, 1, B // 2, B - 2, B - 1} | {b for b, n in enumerate(lens) if n > 0 and (b % 97 == 0 or n == max(lens))})
    want, _, eo, _ = attention64(q[some], values64(*bytes8[:2]), values64(*bytes8[2:]), table[some], [lens[b] for b in some], 1 / math.sqrt(D))
    check_rounded(got[some], want, eo)
    empty = torch.tensor(lens, device="cuda") <= 0
    assert bool((got[empty] == 0).all()) and bool(torch.isfinite(got).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [6, 200])
def test_scales_far_apart(T, dtype, width):
    """Keys and values whose scales lie 2^60 apart, and the ends of the range."""
    page, D, lens = 16, 128, [90, 33, 64, 1]
    pages, _, _, table = _cache_and_values(4, 2, D, page, width, lens, seed=2, garbage=False)
    g = torch.Generator(device="cuda").manual_seed(4)
    pages[1].copy_(torch.randint(60, 122, pages[1].shape, generator=g, device="cuda").to(U8))
    for low, high in ((90, 150), (27, 30), (200, 236)):
        pages[3].copy_(torch.randint(low, high + 1, pages[3].shape, generator=g, device="cuda").to(U8))
        pages[0][(pages[0] & 127) == 127], pages[2][(pages[2] & 127) == 127] = 0, 0
        kv, vv = values64(*pages[:2]), values64(*pages[2:])
        q = _randn(4, 8, D, dtype=dtype, seed=9)
        want, lse, eo, el = attention64(q, kv, vv, table, lens, 1 / math.sqrt(D))
        got, glse = T.thrift_paged_decode8(q, *pages, table, _ints(lens), out_dtype=torch.float32, return_lse=True)
        check_rounded(got, want, eo + 2.0 ** -126 * D)                       # pieces below 2^-126 may be lost
        assert bool(((glse.double() - lse).abs() <= el).all())


@pytest.mark.parametrize("width", [6, 200])
def test_a_code_without_a_number_gives_nan(T, width):
    page, D, lens = 16, 64, [90, 90]
    pages, _, _, table = _cache_and_values(2, 2, D, page, width, lens, seed=2)
    q = _randn(2, 4, D, dtype=torch.float16, seed=9)
    pages[2][table[0, 2].long(), 1, 3, 17] = 0xff                            # one value of sequence 0, KV head 1
    out = T.thrift_paged_decode8(q, *pages, table, _ints(lens))
    nan = out.isnan()
    assert bool(nan[0, 2:, 17].all()) and int(nan.sum()) == 2
    pages[0][table[1, 1].long(), 0, 0, 0] = 0x7f                             # one key of sequence 1, KV head 0
    out = T.thrift_paged_decode8(q, *pages, table, _ints(lens))
    assert bool(out[1, :2].isnan().all()) and not bool(out[1, 2:].isnan().any())


@pytest.mark.parametrize("width", [6, 200])
def test_bad_table_entries_are_clamped(T, width):
    page, lens = 16, [90, 33]
    pages, _, _, table = _cache_and_values(2, 2, 128, page, width, lens, seed=2, garbage=False)
    n = pages[0].shape[0]
    table[0, 1], table[1, 0], table[0, 4] = -7, n, 2 ** 31 - 1
    q = _randn(2, 8, 128, dtype=torch.float16, seed=9)
    got = T.thrift_paged_decode8(q, *pages, table, _ints(lens))
    assert torch.equal(got, T.thrift_paged_decode8(q, *pages, table.clamp(0, n - 1), _ints(lens))) and bool(torch.isfinite(got).all())


def test_streams_workspaces_and_replays(T):
    """Calls at the same time on two streams; captured calls that share one workspace, replayed between eager ones with other lengths."""
    lens, width = [900, 3, 0, 517], 200
    pages, _, _, table = _cache_and_values(4, 2, 128, 16, width, [width * 16] * 4, seed=11)
    q = _randn(4, 8, 128, dtype=torch.float16, seed=12)
    sl = _ints(lens)
    one = lambda **kw: T.thrift_paged_decode8(q, *pages, table, sl, **kw)
    want = one()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            results.append([one() for _ in range(20)])
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for rs in results for r in rs)
    shared = torch.full((max(256, T.paged_decode8_workspace_bytes(4, 8, 2, width, 16, 128)),), 255, dtype=U8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        out = torch.empty(4, 8, 128, dtype=torch.float16, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            one(out=out, workspace=shared)
        graphs.append(g), outs.append(out)
    for i, lens in enumerate(([900, 3, 0, 517], [1, 3200, 33, 0], [0, 0, 0, 0], [960, 959, 16, 17])):
        sl.copy_(_ints(lens))
        want = one()
        torch.cuda.synchronize()
        for g, out in zip(graphs, outs):
            out.fill_(3)
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs), i


# ---- all together ----

@pytest.mark.parametrize("dtype", DTYPES)
def test_a_servers_steps(T, dtype):
    """Prompts, then tokens one by one and requests that end, on a 16-bit and an 8-bit cache of one page table: the 8-bit one holds the 16-bit one's
    tokens to its rounding, attends as the numbers it holds do, and gives the prefill kernel the rows of a chunk."""
    B, Hq, Hkv, D, page = 4, 8, 2, 128, 16
    table = T.PageTable(B, 40, page, 90, "cuda")
    cache, cache16 = T.PagedKVCache8(table, Hkv, D, dtype), T.PagedKVCache(table, Hkv, D, dtype)
    for p in cache.pages:
        p.fill_(255)
    freqs, gain = T.rope_frequencies(D, 1e4, device="cuda")
    for step in range(8):
        new = [[150, 33, 0, 260], [1, 1, 1, 1], [1, 0, 64, 1], [1, 1, 1, 1]][min(step, 3)]
        rows = sum(new) + 5
        x = _randn(rows, Hq + 2 * Hkv, D, dtype=dtype, seed=step)
        m = table.map(_ints(new), rows)
        args = (x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], m, x[:, :Hq], freqs, "half", gain)
        q = cache.append(*args, q_out=torch.zeros(rows, Hq, D, dtype=dtype, device="cuda"))
        assert torch.equal(q, cache16.append(*args, q_out=torch.zeros(rows, Hq, D, dtype=dtype, device="cuda")))
        last = (m.starts[1:].long() - 1).clamp(min=0)
        lens = table.seqlens.tolist()
        out, lse = cache.decode(q[last], return_lse=True, out_dtype=torch.float32)
        want, wl, eo, el = attention64(q[last], values64(cache.k_codes, cache.k_scales), values64(cache.v_codes, cache.v_scales), table.block_table.clamp(min=0), lens, 1 / math.sqrt(D))
        check_rounded(out, want, eo)
        N = max(lens)
        k8, v8 = cache.read(N)
        k16, v16 = cache16.read(N)
        for a, b in ((k8, k16), (v8, v16)):
            # a step of 2^-4 on either side of the 16-bit rounding, and of elements far below the largest 2^-10 of the scale, which is at most the largest / 224
            assert bool(((a.double() - b.double()).abs() <= (2.0 ** -4 + 2 * half_step(dtype)[0]) * b.double().abs() + b.double().abs().amax(-1, keepdim=True) * 2.0 ** -17).all())
        if step == 0:
            # the rows that were read are what the prefill kernels take: the last query over them, all keys in 16 bits
            n = lens[3]
            full = T.thrift_attention(q[:n].new_zeros(1, Hq, n, D).index_copy_(2, torch.tensor([n - 1], device="cuda"), q[last[3]].view(1, Hq, 1, D)),
                                      k8[3:4, :, :n].contiguous(), v8[3:4, :, :n].contiguous(), budget=1.0, out_dtype=torch.float32)[0, :, -1]
            assert float((full - out[3]).abs().max()) <= 2e-3                # its tolerance for all-16-bit runs
        if step == 4:
            table.release(_ints([0, 1, 0, 0]))
            assert table.seqlens.tolist()[1] == 0


def test_the_general_path_gives_the_same_results(T, monkeypatch):
    x = _randn(20, 2, 128, dtype=torch.float16)
    freqs, gain = T.rope_frequencies(64, 1e4, device="cuda")

    def results():
        table = T.PageTable(2, 8, 16, 16, "cuda")
        cache, cache16 = T.PagedKVCache8(table, 2, 128, torch.float16), T.PagedKVCache(table, 2, 128, torch.float16)
        for p in cache.pages:
            p.zero_()
        m = table.map(_ints([9, 9]), 20)
        q = cache.append(x, x, m, x, freqs, "interleaved", gain, q_out=torch.zeros_like(x))
        cache16.append(x, x, m)
        assert cache.append(x, x, m, None, freqs, "half", gain) is None
        out, lse = cache.decode(q[:2], return_lse=True)
        own = torch.empty(2, 2, dtype=torch.float32, device="cuda")
        again = cache.decode(q[:2], out=torch.empty(2, 2, 128, dtype=torch.float32, device="cuda"), lse=own)
        g = _ints([0, 0])
        both = [*cache.decode_prefix(q[:2], g, g[:1], return_lse=True), cache16.decode_prefix(q[:2], g, g[:1])]
        return [q, out, lse, again, own, *cache.read(12), *cache16.read(12, _ints([3, 0])), *both, *cache.pages]

    want = results()
    monkeypatch.setattr(T, "_call", T._General)
    for i, (a, b) in enumerate(zip(results(), want)):
        assert torch.equal(a, b), i


def test_the_module_leaves_other_arguments_to_the_general_path(T):
    m = T._native()
    k, slots, table, lens = torch.zeros(3, 2, 128, dtype=torch.float16, device="cuda"), _ints([0, 1, 2]), _ints([[0], [1], [2]]), _ints([1, 1, 1])
    p = _pages8(4, 2, 16, 128, 0)
    one = lambda **kw: m.paged_append8(*{**dict(k=k, v=k, slots=slots, a=p[0], b=p[1], c=p[2], d=p[3], q=None, qo=None, pos=None, freqs=None, layout=0, gain=1.0, device=0, stream=0), **kw}.values())
    assert one() is True
    for bad in (dict(device=1), dict(k=k.float()), dict(v=k.bfloat16()), dict(k=k[:2]), dict(slots=slots.long()), dict(a=p[1]), dict(b=p[0]), dict(c=p[2][:, :1]), dict(d=p[3].float()),
                dict(a=p[0].cpu()), dict(qo=k), dict(q=k[:2]), dict(freqs=torch.zeros(64, dtype=torch.float64, device="cuda")), dict(layout="half")):
        assert one(**bad) is None, bad
    assert one(pos=slots, freqs=torch.zeros(65, dtype=torch.float64, device="cuda")) == 2
    for f, pages in ((m.paged_decode8, p), (m.paged_decode_prefix8, p), (m.paged_decode_prefix, [k.new_zeros(4, 2, 16, 128)] * 2)):
        groups = dict(of=slots, gl=lens) if f is not m.paged_decode8 else {}
        one = lambda **kw: f(*{**dict(q=k, **{f"p{i}": x for i, x in enumerate(pages)}, table=table, lens=lens, **groups, scale=0.0, out=None, lse=None, rl=0, ws=None, device=0, stream=0), **kw}.values())
        assert one().shape == (3, 2, 128)
        for bad in (dict(device=1), dict(q=k.float()), dict(table=table[:2]), dict(lens=lens.long()), dict(p0=pages[0][:, :1]), dict(p1=pages[0].cpu()), dict(out=k[:2]), dict(lse=k),
                    dict(ws=k), *([dict(of=slots[:2]), dict(gl=lens.long()), dict(gl=table), dict(of=None)] if groups else [])):
            assert one(**bad) is None, bad
        wide = torch.zeros(3, 100, dtype=I32, device="cuda")
        assert one(table=wide, ws=torch.empty(16, dtype=U8, device="cuda")) == 5
    assert all(f() is None for f in (m.paged_append8, m.paged_decode8, m.paged_decode_prefix, m.paged_decode_prefix8))


def test_the_module_leaves_other_reads_to_the_general_path(T, monkeypatch):
    m = T._native()
    table, lens = _ints([[0, 1], [2, 3], [3, 0]]), _ints([20, 3, 0])
    p8, p16 = _pages8(4, 2, 16, 128, 0x38), [_randn(4, 2, 16, 128, dtype=torch.bfloat16, seed=i) for i in (1, 2)]
    out = torch.zeros(3, 2, 24, 128, dtype=torch.bfloat16, device="cuda")
    for f, pages in ((m.paged_read, p16), (m.paged_read8, p8)):
        last = dict(dt=T.BF16) if len(pages) == 4 else {}
        one = lambda **kw: f(*{**dict({f"p{i}": x for i, x in enumerate(pages)}, table=table, lens=lens, n=24, first=None, ko=None, vo=None, **last, device=0, stream=0), **kw}.values())
        k, v = one()
        assert k.shape == v.shape == out.shape and one(ko=out)[0].data_ptr() == out.data_ptr()
        for bad in (dict(device=1), dict(table=table[:2]), dict(table=lens), dict(lens=lens.long()), dict(n=0), dict(n=-3), dict(n=2 ** 40), dict(n=24.0), dict(first=lens[:2]), dict(ko=out[:2]),
                    dict(vo=out.float()), dict(ko=out.half()), dict(vo=out.transpose(0, 1)), dict(p0=pages[0][:, :1]), dict(p1=pages[1].cpu()), dict(n=2 ** 31 - 1, table=table.expand(3, 2)[:0]),
                    *([dict(dt=T.F32), dict(dt=7), dict(p1=pages[0])] if last else [dict(p0=pages[0].float())])):
            assert one(**bad) is None, bad
        assert f() is None
    assert m.paged_read(*p16, table, lens, 1 << 22, None, out, out, 0, 0) is None
    with pytest.raises(T.ThriftError):
        T.thrift_paged_read(torch.zeros(4, 2, 20, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 2, 20, 128, dtype=torch.bfloat16, device="cuda"), table, lens, 24)
    calls = lambda: [*T.thrift_paged_read(*p16, table, lens, 24, first=_ints([0, 2, -5])), *T.thrift_paged_read8(*p8, table, lens, 7, torch.float16),
                     *T.thrift_paged_read8(*p8, table, lens, 24, k_out=out.clone())]
    want = calls()
    monkeypatch.setattr(T, "_call", T._General)
    assert all(torch.equal(x, y) for x, y in zip(calls(), want))

"""Attention over common starts of sequences on the GPU against 64 bits, in 16 and 8 bits: any grouping, lengths and sizes."""
import math

import pytest
import torch

from tests.paged8_util import cache8, prefix64, values64
from tests.paged_util import check_rounded, tokens
from tests.test_gpu_paged import DTYPES, I32, _ints, _randn

pytestmark = pytest.mark.gpu
U8 = torch.uint8


@pytest.fixture(scope="module")
def T():
    from paper_2605_23081_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


class Batch:
    """Sequences of groups: `of` [B], group_lens in tokens (as given to the call), lens [B].  Pages behind the lengths hold NaN."""

    def __init__(self, of, group_lens, lens, Hkv, D, page, width, dtype, bits, seed=0, narrow=False):
        self.of, self.group_lens, self.lens, self.bits, self.dtype = of, group_lens, lens, bits, dtype
        g = torch.Generator().manual_seed(seed)
        B = len(of)
        # whole pages that members share, whatever the call says of lengths below or above that
        whole = [max(0, min(n, width * page)) // page for n in group_lens]
        self.shared = [whole[o] * page if 0 <= o < len(group_lens) and n >= whole[o] * page else 0 for o, n in zip(of, lens)]
        n_pages = sum(whole) + B * width + 3
        names = torch.randperm(n_pages, generator=g)
        table = names[sum(whole):sum(whole) + B * width].view(B, width).clone()
        starts = [sum(whole[:i]) for i in range(len(whole))]
        live = torch.zeros(n_pages, page, dtype=torch.bool)
        for b, n in enumerate(lens):
            n = min(max(n, 0), width * page)
            if self.shared[b]:
                o = of[b]
                table[b, :whole[o]] = names[starts[o]:starts[o] + whole[o]]
            for j in range(-(-n // page)):
                live[table[b, j], :min(page, n - j * page)] = True
            table[b, -(-n // page):] = torch.tensor([-1, 2 ** 31 - 1, -2 ** 31, n_pages], dtype=torch.long)[torch.arange(width - -(-n // page)) % 4]
        if not narrow:
            # room for more than 128 MB, below which every sequence is read by itself
            more = -(-(130 << 20) // (B * Hkv * page * D * (4 if bits == 16 else 2)))
            table = torch.cat([table, torch.full((B, more), -1)], 1)
        self.table = table.to(I32).cuda()
        dead = ~live.cuda()
        kp, vp = (_randn(n_pages, Hkv, page, D, dtype=dtype, seed=seed + i) for i in (0, 1))
        if bits == 16:
            for p in (kp, vp):
                p.transpose(1, 2)[dead] = float("nan")
            self.pages, self.values = (kp, vp), (kp, vp)
        else:
            kp.mul_((0.3 * _randn(*kp.shape[:3], 1, dtype=dtype, seed=seed + 5)).exp())
            vp.mul_((2 * _randn(*vp.shape[:3], 1, dtype=dtype, seed=seed + 6)).exp())
            self.pages = cache8(kp, vp)
            for p in self.pages:
                p.transpose(1, 2)[dead] = 0x7f if p.dim() == 4 else 255
            self.values = values64(*self.pages[:2]), values64(*self.pages[2:])

    def call(self, T, q, **kw):
        f = T.thrift_paged_decode_prefix if self.bits == 16 else T.thrift_paged_decode_prefix8
        return f(q, *self.pages, self.table, _ints(self.lens), _ints(self.of), _ints(self.group_lens), **kw)

    def check(self, T, q, scale=0.0):
        B, Hq, D = q.shape
        clamped = [min(max(n, 0), self.table.shape[1] * self.values[0].shape[2]) for n in self.lens]
        real = scale if scale > 0 else 1 / math.sqrt(D)
        want, lse, eo, el = prefix64(q, *self.values, self.table, clamped, self.shared, real, self.dtype if self.bits == 16 else torch.bfloat16)
        for dt in (torch.float32, q.dtype):
            got, glse = self.call(T, q, softmax_scale=scale, out_dtype=dt, return_lse=True)
            check_rounded(got, want, eo)
            finite = torch.isfinite(lse)
            assert torch.equal(finite, torch.isfinite(glse)) and bool((glse[~finite] == -math.inf).all())
            assert bool(((glse.double() - lse)[finite].abs() <= el[finite]).all())
        return got


def _mixed(page):
    """Three groups of different sizes anywhere in the batch, sequences of none, empty ones, members without tokens of their own, members
    shorter than their group's start."""
    of = [0, 1, -1, 0, 2, 1, 0, 7, 0, 1, -2 ** 31, 0, 2, 0, 1, 2 ** 31 - 1, 0]
    group_lens = [5 * page + 3, 9 * page, 2 * page]
    own = [1, 20, 77, 0, 5, 3 * page, page, 0, 2 * page + 1, 1, 9, -5 * page - 2, 33, 17, 0, 40, 64]
    start = [group_lens[o] // page * page if 0 <= o < 3 else 0 for o in of]
    return of, group_lens, [s + n for s, n in zip(start, own)]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(4, 4), (8, 2), (32, 4), (7, 1), (32, 1), (40, 2), (17, 1)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_against_64_bits(T, D, Hq, Hkv, dtype, bits):
    for page, narrow in ((16, False), (64, False), (256, False), (32, True)):
        print(f"prefix D={D} Hq={Hq} Hkv={Hkv} page={page} bits={bits} narrow={narrow} {dtype}", flush=True)
        of, group_lens, lens = _mixed(page)
        b = Batch(of, group_lens, lens, Hkv, D, page, 13, dtype, bits, seed=page, narrow=narrow)
        b.check(T, _randn(len(of), Hq, D, dtype=dtype, seed=9))


@pytest.mark.parametrize("B,Hq,Hkv,prefix,own", [(2, 32, 8, 5000, 100), (130, 8, 2, 1000, 40), (64, 16, 16, 512, 200), (33, 8, 1, 20000, 10), (300, 4, 1, 640, 70), (7, 64, 8, 3000, 1),
                                                 (1000, 2, 2, 64, 20)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_one_group(T, B, Hq, Hkv, prefix, own, dtype, bits):
    print(f"prefix one group B={B} Hq={Hq} Hkv={Hkv} prefix={prefix} own={own} bits={bits} {dtype}", flush=True)
    page = 32
    g = torch.Generator().manual_seed(B)
    start = prefix // page * page
    lens = [start + n for n in torch.randint(0, own + 1, (B,), generator=g).tolist()]
    b = Batch([0] * B, [prefix], lens, Hkv, 128, page, -(-(start + own) // page), dtype, bits, seed=B)
    b.check(T, _randn(B, Hq, 128, dtype=dtype, seed=9))


@pytest.mark.parametrize("bits", [16, 8])
def test_many_groups(T, bits):
    """Pairs, groups of one, and groups that nobody is in, at the largest numbers of both."""
    B, page, D = 4096, 16, 64
    of = [(b * 2048 + b // 2) % 4096 if b % 3 else b % 50 for b in range(B)]
    group_lens = [16 * (1 + o % 5) for o in range(4096)]
    lens = [group_lens[o] + (b * 7) % 30 for b, o in enumerate(of)]
    b = Batch(of, group_lens, lens, 1, D, page, 8, torch.float16, bits, seed=1)
    b.check(T, _randn(B, 2, D, dtype=torch.float16, seed=9))


@pytest.mark.parametrize("Hkv,page", [(1, 64), (3, 16)])
@pytest.mark.parametrize("bits", [16, 8])
def test_more_tiles_than_workgroups(T, Hkv, page, bits):
    """Three hundred groups of three, of 600 to 1200 tokens, and one of a hundred: workgroups have several parts of tiles each."""
    D = 64
    of = [b % 300 for b in range(900)] + [300] * 100
    group_lens = [600 + 2 * o for o in range(300)] + [2000]
    start = [n // page * page for n in group_lens]
    lens = [start[o] + (b * 7) % 50 for b, o in enumerate(of)]
    print(f"prefix many tiles Hkv={Hkv} page={page} bits={bits}", flush=True)
    b = Batch(of, group_lens, lens, Hkv, D, page, -(-2100 // page), torch.bfloat16, bits, seed=1)
    b.check(T, _randn(1000, 2 * Hkv, D, dtype=torch.bfloat16, seed=9))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("gain", [0.01, 30.0])
def test_flat_and_peaked_scores(T, bits, dtype, gain):
    page, D = 32, 128
    lens = [640, 700, 641, 650, 900]
    b = Batch([0, 0, 0, 0, 0], [640], lens, 2, D, page, 30, dtype, bits, seed=6)
    q = (_randn(5, 8, D, dtype=torch.float32, seed=7) * gain).to(dtype)
    b.check(T, q)
    b.check(T, q, scale=0.3)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("where", ["start", "own"])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_ramps(T, bits, where, sign):
    """Scores that fall or rise along the tokens by far more than exp can hold: all weight in the common tokens, or in a sequence's own."""
    page, D, start = 16, 64, 400
    lens = [start + n for n in (0, 1, 50, 100)]
    b = Batch([0] * 4, [start], lens, 2, D, page, 40, torch.bfloat16, bits, seed=3)
    if bits == 16:
        k = b.pages[0]
    else:
        k = torch.zeros(b.values[0].shape, dtype=torch.bfloat16, device="cuda")
    for i, n in enumerate(lens):
        for j in range(-(-n // page)):
            if where == "own" and j * page < start:
                ramp = torch.zeros(page, device="cuda")
            else:
                ramp = sign * (torch.arange(page, device="cuda") + j * page) / 8.0
            live = (torch.arange(page, device="cuda") + j * page < n).view(1, page, 1)
            name = int(b.table[i, j])
            k[name] = torch.where(live, (ramp.view(1, page, 1) / 8.0).expand(2, page, D).to(torch.bfloat16), k[name])
    if bits == 16:
        b.values = (k, b.values[1])
    else:
        codes = cache8(k, k)[:2]
        dead = b.pages[1] == 255
        codes[0][dead], codes[1][dead] = 0x7f, 255
        b.pages = (*codes, *b.pages[2:])
        b.values = (values64(*codes), b.values[1])
    b.check(T, _randn(4, 8, D, dtype=torch.bfloat16, seed=7).abs())


@pytest.mark.parametrize("bits", [16, 8])
def test_groups_that_share_nothing(T, bits):
    """Lengths of groups below a page, of 0 and below: the result of the attention without groups, to the last bit of its sums' order."""
    page, D = 64, 128
    for group_lens in ([63, 0], [-1, -2 ** 31]):
        b = Batch([0, 1, 0, 1, 1], group_lens, [100, 0, 64, 63, 500], 2, D, page, 9, torch.float16, bits, seed=2)
        b.check(T, _randn(5, 8, D, dtype=torch.float16, seed=7))
    # and a group whose start is longer than the table is wide: everything there is, or more than anybody has
    for narrow in (True, False):
        b = Batch([0, 0, 0], [2 ** 31 - 1], [9 * page, 9 * page, 100], 2, D, page, 9, torch.float16, bits, seed=2, narrow=narrow)
        b.check(T, _randn(3, 8, D, dtype=torch.float16, seed=7))


@pytest.mark.parametrize("bits", [16, 8])
def test_one_sequence_and_none(T, bits):
    page, D = 16, 128
    for lens in ([50], [0], [16], [1]):
        Batch([0], [16], lens, 2, D, page, 9, torch.float16, bits, seed=2).check(T, _randn(1, 8, D, dtype=torch.float16, seed=7))
    b = Batch([0, 0, -1], [16], [0, 0, 0], 2, D, page, 9, torch.float16, bits, seed=2)
    assert not bool(b.check(T, _randn(3, 8, D, dtype=torch.float16, seed=7)).any())


@pytest.mark.parametrize("bits", [16, 8])
def test_bad_table_entries_are_not_followed(T, bits):
    page, D = 16, 128
    b = Batch([0, 0, 0], [64], [64, 90, 70], 2, D, page, 9, torch.float16, bits, seed=2)
    pages = [torch.zeros_like(p) if p.dim() == 4 else torch.full_like(p, 127) if p.dtype == U8 else p for p in b.pages]
    b.pages = tuple(pages)
    n = pages[0].shape[0]
    b.table[:, 1], b.table[1, 5], b.table[2, 4], b.table[0, 0] = n, -9, 2 ** 31 - 1, -2 ** 31
    assert bool(torch.isfinite(b.call(T, _randn(3, 8, D, dtype=torch.float16, seed=9))).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_streams_workspaces_and_replays(T, bits):
    """Calls at the same time on two streams; captured calls that share one workspace, replayed between eager ones with other lengths and groups."""
    page, D, width = 16, 128, 100
    b = Batch([0, 0, 0, 1, 1], [640, 320], [1600] * 5, 2, D, page, width, torch.float16, bits, seed=4)
    q = _randn(5, 8, D, dtype=torch.float16, seed=12)
    lens, of, group_lens = _ints(b.lens), _ints(b.of), _ints(b.group_lens)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    one = lambda **kw: f(q, *b.pages, b.table, lens, of, group_lens, **kw)
    want = one()
    streams = [torch.cuda.Stream() for _ in range(2)]
    results = []
    torch.cuda.synchronize()
    for s in streams:
        with torch.cuda.stream(s):
            results.append([one() for _ in range(20)])
    torch.cuda.synchronize()
    assert all(torch.equal(r, want) for rs in results for r in rs)
    shared = torch.full((T.paged_decode_prefix_workspace_bytes(bits, 5, 8, 2, 2, b.table.shape[1], page, D),), 255, dtype=U8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):
        out = torch.empty(5, 8, D, dtype=torch.float16, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            one(out=out, workspace=shared)
        graphs.append(g), outs.append(out)
    for i, (ln, o, gl) in enumerate((([1600] * 5, [0, 0, 0, 1, 1], [640, 320]), ([700, 640, 641, 0, 1600], [0, 0, 0, -1, -1], [640, 0]), ([0] * 5, [0] * 5, [640, 320]),
                                     ([5, 900, 33, 320, 330], [1, 0, 0, 1, 1], [16, 320]), ([1599, 1600, 1, 900, 320], [-1] * 5, [640, 320]))):
        lens.copy_(_ints(ln)), of.copy_(_ints(o)), group_lens.copy_(_ints(gl))
        want = one()
        torch.cuda.synchronize()
        for g, out in zip(graphs, outs):
            out.fill_(3)
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, want) for x in outs), i


@pytest.mark.parametrize("bits", [16, 8])
def test_a_server_whose_requests_share_a_prompt(T, bits):
    """A prompt in whole pages that one sequence holds, requests that start with its pages and go on by themselves: every step's attention is that
    of the cache without groups."""
    B, Hq, Hkv, D, page, dtype = 6, 8, 2, 128, 16, torch.bfloat16
    table = T.PageTable(B, 2800, page, 200, "cuda")                          # room for more than 128 MB
    cache = (T.PagedKVCache if bits == 16 else T.PagedKVCache8)(table, Hkv, D, dtype)
    freqs, gain = T.rope_frequencies(D, 1e4, device="cuda")

    def step(new, seed):
        rows = sum(new)
        x = _randn(rows, Hq + 2 * Hkv, D, dtype=dtype, seed=seed)
        m = table.map(_ints(new), rows)
        q = cache.append(x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], m, x[:, :Hq], freqs, "half", gain)
        return q[(m.starts[1:].long() - 1).clamp(min=0)]

    start = 20 * page
    step([start, 0, 0, 0, 0, 0], 0)
    table.block_table[1:5, :20] = table.block_table[0, :20]
    table.seqlens = torch.where(torch.arange(B, device="cuda") < 5, start, 0).to(I32)
    of, group_lens = _ints([0] * 5 + [-1]), _ints([start])
    for i, new in enumerate(([0, 30, 5, 17, 1, 50], [1] * 6, [1, 1, 1, 0, 1, 1], [1] * 6)):
        q = step(new, 1 + i)
        got, lse = cache.decode_prefix(q, of, group_lens, out_dtype=torch.float32, return_lse=True)
        want, wl = cache.decode(q, out_dtype=torch.float32, return_lse=True)
        # probabilities of common tokens rounded once, half a step of bf16 of values of at most 6
        assert float((got - want).abs().max()) <= 2.0 ** -8 * 6 and float((lse - wl).abs().max()) <= 2e-5
        assert not torch.equal(got, torch.zeros_like(got))


def _with_keys(b, rows):
    """The batch with every key of token j of its pages replaced by rows(sequence, tokens) in all channels; what is behind the lengths stays NaN."""
    page = b.values[0].shape[2]
    k = b.pages[0].clone() if b.bits == 16 else torch.zeros(b.values[0].shape, dtype=b.dtype, device="cuda")
    for i, n in enumerate(b.lens):
        held = b.table[i, :-(-n // page)].long()
        place = torch.arange(len(held) * page, device="cuda")
        new = rows(i, place).to(b.dtype).view(-1, 1, page, 1).expand(-1, k.shape[1], -1, k.shape[3])
        k[held] = torch.where((place < n).view(-1, 1, page, 1), new, k[held])
    if b.bits == 16:
        b.pages, b.values = (k, b.pages[1]), (k, b.values[1])
        return b
    codes = cache8(k, k)[:2]
    dead = b.pages[1] == 255
    codes[0][dead], codes[1][dead] = 0x7f, 255
    b.pages, b.values = (*codes, *b.pages[2:]), (values64(*codes), b.values[1])
    return b


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("a", [896.0, 1024.0, 2048.0, 4096.0, 28672.0])
def test_scores_past_24_bits(T, bits, dtype, sign, a):
    """Scores from 2^23 to 2^33 (in powers of two): keys with the largest one, among the common tokens or a sequence's own, share the weight."""
    lens, D, Hkv, common = [690, 640, 665, 700], 128, 2, 640
    b = Batch([0] * 4, [common], lens, Hkv, D, 16, 44, dtype, bits, seed=12)
    shared = [0, 63, 64, 130, 511, 639]
    winners = [shared + [641, 689], shared, shared + [664], shared + list(range(640, 680))]
    low, high = (a / 2, a) if sign > 0 else (-a, -a / 2)
    _with_keys(b, lambda i, place: torch.where(torch.isin(place, torch.tensor(winners[i], device="cuda")), high, low))
    q = torch.full((4, 2 * Hkv, D), a, dtype=dtype, device="cuda")
    out, lse = b.call(T, q, out_dtype=torch.float32, return_lse=True)
    v = b.values[1]
    want = torch.stack([tokens(v, b.table[i], n).double()[:, winners[i]].mean(1) for i, n in enumerate(lens)])
    # the scores are fp32 numbers (a^2 has few bits), so that P is 1 or 0 in either type; at most 46 values are added and parts joined, each partial
    # sum off by half a step of at most 64 times the largest: 66 U of it
    top = v[~torch.isnan(v)].double().abs().max()
    assert bool(((out.view(4, Hkv, 2, D).double() - want.unsqueeze(2)).abs() <= 66 * 2.0 ** -24 * top).all())
    n = torch.tensor([len(w) for w in winners], dtype=torch.float64, device="cuda")
    exact = D * a * high / math.sqrt(D) + n.log()
    assert bool(((lse.double() - exact.unsqueeze(1)).abs() <= 8 * 2.0 ** -24 * exact.abs().unsqueeze(1)).all())


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dead", [64, 100, 640])
def test_scores_of_minus_infinity_weigh_nothing(T, bits, dead):
    """Keys whose product with the query overflows downwards: the first block of the common tokens, more than it, all of them."""
    lens, D, Hkv, common = [690, 641, 665, 700], 128, 2, 640
    b = Batch([0] * 4, [common], lens, Hkv, D, 16, 44, torch.bfloat16, bits, seed=12)
    _with_keys(b, lambda i, place: torch.where(place < dead, -3e37, (place % 13).float() / 64))
    q = torch.ones(4, 2 * Hkv, D, dtype=torch.bfloat16, device="cuda")
    out, lse = b.call(T, q, out_dtype=torch.float32, return_lse=True)
    for i, n in enumerate(lens):
        k, v = (tokens(p, b.table[i], n)[:, dead:].double() for p in b.values)
        s = k.sum(-1) / math.sqrt(D)
        p = torch.softmax(s, -1)
        want = (p.unsqueeze(-1) * v).sum(1)
        # the common tokens' probabilities are rounded to bf16 (2^-8 of each), beside them fp32 sums
        bound = (2.0 ** -8 + 2.0 ** -14) * (p.unsqueeze(-1) * v.abs()).sum(1) + 2.0 ** -14 * v.abs().amax(1)
        assert bool(((out[i].view(Hkv, 2, D).double() - want.unsqueeze(1)).abs() <= bound.unsqueeze(1)).all())
        assert bool(((lse[i].view(Hkv, 2).double() - torch.logsumexp(s, -1).unsqueeze(1)).abs() <= 2.0 ** -14).all())


@pytest.mark.parametrize("bits", [16, 8])
def test_the_largest_values(T, bits):
    """Values near the end of bfloat16's range, scores that rise a little: a mean of them is one of them, whatever the sums are scaled by in between."""
    lens, D = [690, 640, 665, 700], 128
    b = Batch([0] * 4, [640], lens, 2, D, 16, 44, torch.bfloat16, bits, seed=12)
    _with_keys(b, lambda i, place: torch.floor(place.float() / 100) / 8)
    if bits == 16:
        v = b.pages[1]
        live = ~torch.isnan(v)
        v[live] = torch.where(v[live] > 0, 1.0, -1.0).to(torch.bfloat16) * 2.0 ** 120
        b.values = (b.values[0], v)
    else:
        codes, scales = (x.clone() for x in b.pages[2:])
        live = scales != 255
        scales[live] = 247                                                   # 2^120, codes of 1 and -1
        codes[live] = (codes[live] & 128) | 0x38
        b.pages = (*b.pages[:2], codes, scales)
        b.values = (b.values[0], values64(codes, scales))
    b.check(T, torch.full((4, 4, D), 0.5, dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", DTYPES)
def test_bad_common_entries_are_clamped(T, dtype, bits):
    """In common pages and in a sequence's own: the result of the table with its entries clamped to the pages, bit for bit."""
    b = Batch([0] * 4, [640], [690, 640, 665, 700], 2, 128, 16, 44, dtype, bits, seed=2)
    pages = [torch.nan_to_num(p, 0.5) if p.dtype == dtype else torch.where(p == 255, 127, p) if p.dim() == 3 else torch.where(p == 0x7f, 0, p) for p in b.pages]
    n, q = pages[0].shape[0], _randn(4, 8, 128, dtype=dtype, seed=9)
    for entry, j in ((-1, 0), (n, 7), (-2 ** 31, 21), (2 ** 31 - 1, 39)):
        b.table[:, j] = entry
    b.table[0, 41], b.table[3, 43] = -9, n + 3
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    got, want = (f(q, *pages, t, _ints(b.lens), _ints(b.of), _ints(b.group_lens), out_dtype=torch.float32, return_lse=True) for t in (b.table, b.table.clamp(0, n - 1)))
    assert all(torch.equal(x, y) and bool(torch.isfinite(x).all()) for x, y in zip(got, want))


@pytest.mark.parametrize("bits", [16, 8])
def test_offsets_past_32_bits(T, bits):
    """Common pages whose elements lie past 2^31 and whose bytes lie past 2^32."""
    Hkv, page, D, dtype = 8, 128, 128, torch.bfloat16
    n_pages = (2 ** 31 + 2 ** 29) // (Hkv * page * D) * (1 if bits == 16 else 2)
    names = [n_pages - 1, n_pages - 3, 0, n_pages * 4 // 5, 5, n_pages - 2, n_pages - 7]
    far = torch.tensor(names, device="cuda")
    some = [_randn(7, Hkv, page, D, dtype=dtype, seed=i) for i in (0, 1)]
    some = some if bits == 16 else cache8(*some)
    pages = [torch.empty(n_pages, *p.shape[1:], dtype=p.dtype, device="cuda") for p in some]
    for p, x in zip(pages, some):
        p[far] = x
    few, full = torch.tensor([[0, 1, 2, 3, 4], [0, 1, 2, 3, 5], [0, 1, 2, 3, 6]], dtype=I32, device="cuda"), torch.full((3, 230), -1, dtype=I32, device="cuda")      # room for more than 128 MB
    full[:, :5] = far[few.long()].to(I32)
    lens, of, group_lens = _ints([512 + 100, 512, 512 + 128]), _ints([0, 0, 0]), _ints([512])
    q = _randn(3, 4 * Hkv, D, dtype=dtype, seed=5)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    got = f(q, *pages, full, lens, of, group_lens, out_dtype=torch.float32)
    del pages
    few = torch.cat([few, torch.full((3, 225), -1, dtype=I32, device="cuda")], 1)
    assert torch.equal(got, f(q, *some, few, lens, of, group_lens, out_dtype=torch.float32))


def test_the_largest_batch(T):
    """4096 sequences of one group, and one more is refused."""
    B, page, D = 4096, 16, 64
    b = Batch([0] * B, [80], [80 + i % 3 for i in range(B)], 1, D, page, 6, torch.float16, 16, seed=3)
    q = _randn(B, 1, D, dtype=torch.float16, seed=5)
    b.check(T, q)
    with pytest.raises(Exception):
        T.thrift_paged_decode_prefix(torch.cat([q, q[:1]]), *b.pages, torch.cat([b.table, b.table[:1]]), _ints(b.lens + [80]), _ints([0] * (B + 1)), _ints([80]))


def test_the_steps_that_the_readme_shows(T):
    import os
    readme = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code = readme.split("```python\n")[2].split("```")[0]
    B, Hq, Hkv, D, page, pages, dtype = 4, 8, 2, 128, 16, 40, torch.bfloat16
    for kind in (T.PagedKVCache, T.PagedKVCache8):
        table = T.PageTable(B, 2800, page, 100, "cuda")                      # room for more than 128 MB
        cache = kind(table, Hkv, D, dtype)
        freqs, gain = T.rope_frequencies(D, 1e4, device="cuda")
        prompt = _randn(pages * page, 2 * Hkv, D, dtype=dtype)
        cache.append(prompt[:, :Hkv], prompt[:, Hkv:], table.map(_ints([pages * page, 0, 0, 0]), pages * page), prompt[:, :Hkv].repeat(1, Hq // Hkv, 1), freqs, "half", gain)
        names = dict(torch=torch, B=B, pages=pages, page_size=page, table=table, cache=cache, freqs=freqs, gain=gain, rows=7, new_lens=_ints([1, 3, 2, 1]),
                     q=_randn(7, Hq, D, dtype=dtype, seed=1), k=_randn(7, Hkv, D, dtype=dtype, seed=2), v=_randn(7, Hkv, D, dtype=dtype, seed=3), ended=_ints([0, 1, 0, 0]))
        code_to, code_end = code.split("table.block_table[ended")
        exec(code_to, names)
        want = cache.decode(names["q"][names["last"]], out_dtype=torch.float32)
        # probabilities of common tokens rounded once, half a step of bf16 of values of at most 6, and the output rounded
        assert float((names["out"].float() - want).abs().max()) <= 2.0 ** -8 * (6 + float(want.abs().max()))
        assert table.free_count.tolist() == [100 - pages - 4]
        exec("table.block_table[ended" + code_end, names)
        assert table.free_count.tolist() == [100 - pages - 3] and table.seqlens.tolist() == [pages * page + 1, 0, pages * page + 2, pages * page + 1]


@pytest.mark.parametrize("dtype,lens,start", [(torch.bfloat16, [2 ** 31 - 16, 2 ** 31 - 1], 2 ** 31 - 1), (torch.float16, [2 ** 31 - 16 - 15, 2 ** 30 + 77], 2 ** 30)])
@pytest.mark.parametrize("bits", [16, 8])
def test_the_longest_block_table(T, dtype, lens, start, bits):
    """A table of 2^31 - 16 tokens that names four pages over and over, all of it common or half; blocks that end past 2^31."""
    D, page, width = 64, 16, 2 ** 27 - 1
    kp = _randn(4, 1, page, D, dtype=dtype)
    vp = torch.randint(-4, 5, (4, 1, page, D), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(dtype)
    pages = (kp, vp) if bits == 16 else cache8(kp, vp)
    table = torch.arange(width, dtype=I32, device="cuda").remainder_(4).expand(2, width).contiguous()
    print(f"longest prefix {dtype} {lens} {start} {bits}", flush=True)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    # queries of 0 weigh all keys alike: P is a power of two, and sums of 2^23 values, whose means over 64 tokens are below 2, are exact
    assert float(vp.view(64, D).float().mean(0).abs().max()) < 2
    out, lse = f(torch.zeros(2, 1, D, dtype=dtype, device="cuda"), *pages, table, _ints(lens), _ints([0, 0]), _ints([start]), out_dtype=torch.float32, return_lse=True)
    for b, n in enumerate(min(n, width * page) for n in lens):
        count = torch.tensor([n // 64 + (j < n % 64) for j in range(64)], dtype=torch.float64, device="cuda")
        want = (count.unsqueeze(1) * vp.view(64, D).double()).sum(0) / n
        # the parts of 256 tiles, and those of 4 wavefronts and 512 shares of the own tokens: 772 additions each in the sums of values (half a step of at
        # most 4 n) and of weights
        assert bool(((out[b, 0].double() - want).abs() <= 4 * (2 * 772 + 4) * 2.0 ** -24).all())
        assert abs(float(lse[b, 0]) - math.log(n)) <= (772 + 4 * math.log(n)) * 2.0 ** -24


@pytest.mark.parametrize("bits", [16, 8])
def test_a_captured_step_replayed(T, bits):
    """Append with the queries rotated in place, attention with and without common starts, and rows read back in one graph; replayed with other tokens, slots,
    lengths and groups, each replay against the same calls made one by one on another cache."""
    B, Hq, Hkv, D, page, width, dtype = 5, 8, 2, 128, 16, 2800, torch.float16
    n_pages = 300
    shapes = [(n_pages, Hkv, page, D)] * 2 if bits == 16 else [(n_pages, Hkv, page, D), (n_pages, Hkv, page)] * 2
    caches = [[torch.zeros(s, dtype=dtype if bits == 16 else U8, device="cuda") for s in shapes] for _ in range(2)]
    append, decode, prefix, read = (T.thrift_paged_append, T.thrift_paged_decode, T.thrift_paged_decode_prefix, T.thrift_paged_read) if bits == 16 else \
        (T.thrift_paged_append8, T.thrift_paged_decode8, T.thrift_paged_decode_prefix8, T.thrift_paged_read8)
    table = torch.full((B, width), -1, dtype=I32)
    table[:, :40] = torch.arange(40)
    table[:, 40:80] = 40 + torch.arange(B * 40).view(B, 40)
    table = table.cuda()
    lens, of, group_lens, slots, positions = _ints([1] * B), _ints([0] * B), _ints([640]), _ints([-1] * 80), _ints([0] * 80)
    q, k, v = (torch.zeros(80, h, D, dtype=dtype, device="cuda") for h in (Hq, Hkv, Hkv))
    freqs, gain = T.rope_frequencies(D, 1e4, device="cuda")
    more = {} if bits == 16 else dict(dtype=dtype)

    def step(cache, q):
        append(k, v, slots, *cache, q=q, q_out=q, positions=positions, freqs=freqs, gain=gain)
        return [q, decode(q[:B], *cache, table, lens), *prefix(q[:B], *cache, table, lens, of, group_lens, return_lse=True), *read(*cache, table, lens, 48, first=positions[:B], **more)]

    step(caches[0], q), step(caches[1], q.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(caches[0], q)
    names = torch.arange(n_pages * page)
    for i, (n, groups, start) in enumerate((([690, 641, 700, 640, 655], [0] * 5, 640), ([700, 0, 1, 640, 1200], [0, 0, 0, 0, -1], 320), ([1280] * 5, [0, 0, 0, -1, -1], 500), ([3] * 5, [0] * 5, 640))):
        g = torch.Generator().manual_seed(i)
        q.copy_(_randn(80, Hq, D, dtype=dtype, seed=3 * i)), k.copy_(_randn(80, Hkv, D, dtype=dtype, seed=3 * i + 1)), v.copy_(_randn(80, Hkv, D, dtype=dtype, seed=3 * i + 2))
        slots.copy_(names[torch.randperm(240 * page, generator=g)[:80]].to(I32).cuda()), positions.copy_(torch.randint(0, 5000, (80,), generator=g).to(I32).cuda())
        slots[7::9] = -1
        lens.copy_(_ints(n)), of.copy_(_ints(groups)), group_lens.copy_(_ints([start]))
        want = [x.clone() for x in step(caches[1], q.clone())]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for j, (x, y) in enumerate(zip(outs, want)):
            assert torch.equal(x, y), (i, j)
        assert all(torch.equal(x, y) for x, y in zip(*caches))

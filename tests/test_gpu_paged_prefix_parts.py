"""Attention over common starts whose tiles are cut into long parts, every page a different one, against 64 bits."""
import math

import pytest
import torch

from tests.paged8_util import cache8, prefix64, values64
from tests.paged_util import attention64, check_rounded
from tests.test_gpu_paged import DTYPES, I32, _ints, _randn
from tests.test_gpu_paged_prefix import T  # noqa: F401

pytestmark = pytest.mark.gpu

SHARES = 256                              # parts that all tiles are cut into
HKV = 64                                  # KV heads: with one tile each, a part has a quarter of a head's blocks


def _problem(D, G, blocks, dtype, bits, members=3):
    """Sequences of one group of 64 KV heads.  Where a head is one tile, its blocks of 64 tokens come in four parts of `blocks` each (the last one lacks a page);
    where it is two, in two parts and one, or more."""
    page = 16
    start = 64 * blocks * SHARES // HKV - page                                # the last block lacks a page
    shared = start // page
    own = [0, 1, 40] + [page] * (members - 3)
    lens = [start + n for n in own]
    g = torch.Generator().manual_seed(D + blocks)
    n_pages = shared + 3 * members + 1
    names = torch.randperm(n_pages, generator=g)
    # room for more than 128 MB, below which every sequence is read by itself
    table = torch.full((members, shared + 3 + (130 << 20) // (members * HKV * page * D * 2)), -1, dtype=I32)
    table[:, :shared] = names[:shared]
    for b in range(members):
        table[b, shared:shared + 3] = names[shared + 3 * b:shared + 3 * b + 3]
    kp, vp = (_randn(n_pages, HKV, page, D, dtype=dtype, seed=i) for i in (0, 1))
    # queries of which some hundred tokens have most of the weight: a block of other tokens in the place of one is seen in most rows
    q = (_randn(members, HKV * G, D, dtype=torch.float32, seed=9) * 2.5).to(dtype)
    if bits == 16:
        pages, values = (kp, vp), (kp, vp)
    else:
        vp.mul_((2 * _randn(n_pages, HKV, page, 1, dtype=dtype, seed=6)).exp())
        pages = cache8(kp, vp)
        values = values64(*pages[:2]), values64(*pages[2:])
    return q, pages, values, table.cuda(), lens, start


# 4 x 3 rows of a tile: wavefronts take half a block's keys each; 32 x 5: whole blocks (256 channels: one tile of 128 rows with whole blocks, one of 32 with halves)
@pytest.mark.parametrize("D,blocks", [(D, n) for D in (64, 128, 256) for n in (9, 17, 33, 65)] + [(64, 129)])
@pytest.mark.parametrize("G,members", [(4, 3), (32, 5)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_long_parts(T, D, blocks, G, members, dtype, bits):  # noqa: F811
    print(f"prefix parts D={D} blocks={blocks} G={G} members={members} bits={bits} {dtype}", flush=True)
    q, pages, values, table, lens, start = _problem(D, G, blocks, dtype, bits, members)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    got, lse = f(q, *pages, table, _ints(lens), _ints([0] * members), _ints([start]), out_dtype=torch.float32, return_lse=True)
    # some KV heads in 64 bits: the first, the last and two between
    heads = [0, 21, 42, HKV - 1]
    rows = [h * G + i for h in heads for i in range(G)]
    few = [p[:, heads].contiguous() for p in values]
    want, wl, eo, el = prefix64(q[:, rows].contiguous(), *few, table, lens, [start] * members, 1 / math.sqrt(D), dtype if bits == 16 else torch.bfloat16)
    check_rounded(got[:, rows], want, eo)
    assert bool(((lse[:, rows].double() - wl).abs() <= el).all())


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("Hq,Hkv", [(16, 4), (128, 4)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_probabilities_of_common_tokens_hold_two_pieces(T, D, Hq, Hkv, dtype, bits):  # noqa: F811
    """Exact scores of which a few tokens have the weight: fp32 results are as near to 64 bits over common tokens as over a sequence's own."""
    page, start, members, scale = 16, 256, 5, 0.25
    lens = [start, start + 1, start + 7, start + 16, start + 40]
    shared = start // page
    n_pages = shared + 3 * members + 1
    g = torch.Generator(device="cuda").manual_seed(D + Hq)
    # products and their sums are whole numbers
    k = torch.randint(-1, 2, (n_pages, Hkv, page, D), generator=g, device="cuda").to(dtype)
    q = (2 * torch.randint(-1, 2, (members, Hq, D), generator=g, device="cuda")).to(dtype)
    v = torch.randn(n_pages, Hkv, page, D, generator=g, device="cuda").to(dtype)
    pages = (k, v) if bits == 16 else cache8(k, v)
    values = (k, v) if bits == 16 else (values64(*pages[:2]), values64(*pages[2:]))
    table = torch.full((members, shared + 3 + (130 << 20) // (members * Hkv * page * D * 2)), -1, dtype=I32, device="cuda")
    table[:, :shared] = torch.arange(shared)
    table[:, shared:shared + 3] = shared + torch.arange(3 * members).view(members, 3)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    got, lse = f(q, *pages, table, _ints(lens), _ints([0] * members), _ints([start]), softmax_scale=scale, out_dtype=torch.float32, return_lse=True)
    want, wl, _, _ = attention64(q, *values, table, lens, scale)
    weights = torch.stack([attention64(q[b:b + 1], values[0], values[1].abs(), table[b:b + 1], [n], scale)[0][0] for b, n in enumerate(lens)])
    # Of a weight: 2^-16 by its two pieces; the factor of the scores (rounded once, U of at most 64 binades that matter) and the difference to the reference
    # (the same), 8 U for the exponential and the joins, all of it twice, in the weight and in their sum; and a sum over at most 296 tokens, of weights and of values.
    U = 2.0 ** -24
    rel = 2.0 ** -16 + (2 * (64 + 64 + 8) + 2 * 296) * U
    assert bool(((got.double() - want).abs() <= rel * weights).all())
    assert bool(((lse.double() - wl).abs() <= (2 * (64 + 64 + 8) + 296 + wl.abs()) * U).all())


@pytest.mark.parametrize("members,G", [(2, 1), (5, 32)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
def test_the_longest_start_with_a_few_tokens_that_count(T, members, G, dtype, bits):  # noqa: F811
    """2^31 - 16 common tokens in four pages over and over, and five pages at odd places whose scores are far above all others: keys and values there have to be
    each other's."""
    D, page, width = 64, 16, 2 ** 27 - 1
    places = [3, 12345, 2 ** 26 - 1, 2 ** 26 + 4097, width - 1]
    g = torch.Generator(device="cuda").manual_seed(5)
    kp, vp = (torch.randn(9, 1, page, D, generator=g, device="cuda") for _ in range(2))
    q = torch.randn(members, G, D, generator=g, device="cuda") * 0.25
    q[:, :, 0] = 16.0                                                        # channel 0: 16 * 32 / 8 = 64 above the rest, which has a few units
    kp[:, :, :, 0] = 0.0
    kp[4:, :, :, 0] = 32.0
    kp, vp, q = kp.to(dtype), vp.to(dtype), q.to(dtype)
    pages = (kp, vp) if bits == 16 else cache8(kp, vp)
    kv, vv = (kp, vp) if bits == 16 else (values64(*pages[:2]), values64(*pages[2:]))
    table = torch.arange(width, dtype=I32, device="cuda").remainder_(4)
    table[torch.tensor(places, device="cuda")] = torch.arange(4, 9, dtype=I32, device="cuda")
    table = table.expand(members, width).contiguous()
    print(f"longest start with a few tokens {members} {G} {bits} {dtype}", flush=True)
    f = T.thrift_paged_decode_prefix if bits == 16 else T.thrift_paged_decode_prefix8
    got, lse = f(q, *pages, table, _ints([2 ** 31 - 1] * members), _ints([0] * members), _ints([2 ** 31 - 1]), out_dtype=torch.float32, return_lse=True)
    # the 80 tokens alone: 2^31 others of a score that is at least 50 lower weigh 2^31 e^-50 < 2^-41
    few = torch.arange(4, 9, dtype=I32, device="cuda").expand(members, 5)
    want, wl, eo, el = attention64(q, kv, vv, few, [80] * members, 1 / math.sqrt(D))
    assert bool(((got.double() - want).abs() <= eo + 2.0 ** -30 * vv.double().abs().max()).all())
    assert bool(((lse.double() - wl).abs() <= el + 2.0 ** -30).all())

"""NaN and infinities among common tokens, and groups of which nothing is saved, against the attention without groups."""
import math

import pytest
import torch

from tests.test_gpu_paged import DTYPES, _ints, _randn
from tests.test_gpu_paged_prefix import Batch, T  # noqa: F401

pytestmark = pytest.mark.gpu
HKV, PAGE = 3, 16


def _plain(T, b, q, **kw):  # noqa: F811
    return (T.thrift_paged_decode if b.bits == 16 else T.thrift_paged_decode8)(q, *b.pages, b.table, _ints(b.lens), **kw)


def _near(got, want, n):
    """Both are within 2^-16 (two pieces of a probability), n U (sums) and what scores differ by: the same products, summed over D <= 256 channels in another order,
    which is at most 256 U of |q| |k| <= 40, twice.  Values are at most 6."""
    U = 2.0 ** -24
    return bool(((got - want).abs() <= 2 * 6 * (2.0 ** -16 + 2 * n * U + 2 * 256 * 40 * U)).all())


# starts that end inside a block of 64 keys, after whole pages; the odd token lies in the last block, in a row that stands for none behind the end, or in front
@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("G", [2, 32])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("token", [0, 37, 641, 655])
def test_odd_common_tokens(T, D, G, dtype, bits, token):  # noqa: F811
    start, odd = 656, 1                                                       # the KV head with the odd token
    lens = [start, start + 1, start + 40, start + 16, start, 700]
    of = [0, 0, 0, 0, 0, -1]
    q = _randn(6, HKV * G, D, dtype=dtype, seed=9)
    rows = slice(odd * G, (odd + 1) * G)
    kinds = [("key", math.nan), ("value", math.nan)] + ([("value", math.inf)] if bits == 16 else [])
    for what, x in kinds:
        print(f"prefix odd D={D} G={G} bits={bits} token={token} {what} {x} {dtype}", flush=True)
        b = Batch(of, [start], lens, HKV, D, PAGE, 45, dtype, bits, seed=3)
        page, at, channel = int(b.table[0, token // PAGE]), token % PAGE, 5
        clean = b.call(T, q, out_dtype=torch.float32, return_lse=True)
        assert all(bool(torch.isfinite(y).all()) for y in clean)
        side = b.pages[0 if what == "key" else bits // 16 if bits == 16 else 2]
        side[page, odd, at, channel] = 0x7f if bits == 8 else x
        out, lse = b.call(T, q, out_dtype=torch.float32, return_lse=True)
        touched = torch.zeros_like(out, dtype=torch.bool)
        if what == "key":
            touched[:5, rows] = True
        else:
            touched[:5, rows, channel] = True
        # an infinite value times the two pieces of a probability: NaN where the second is 0 or below, otherwise infinite
        wrong = (lambda y: ~torch.isfinite(y)) if x == math.inf else torch.isnan
        assert torch.equal(wrong(out), touched)
        assert torch.equal(out[~touched], clean[0][~touched])
        key = touched.all(-1)
        assert torch.equal(lse.isnan(), key) and torch.equal(lse[~key], clean[1][~key])
        plain, pl = _plain(T, b, q, out_dtype=torch.float32, return_lse=True)
        assert torch.equal(wrong(plain), touched) and torch.equal(pl.isnan(), key)


@pytest.mark.parametrize("bits", [16, 8])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("of,group_lens,lens", [([0, 1, 0, 1, 1], [63, 0], [100, 0, 64, 63, 500]), ([0, 1, 0, 1, 1], [-1, -2 ** 31], [100, 0, 64, 63, 500]),
                                                ([0, 1, 2, -1, 7], [512, 512, 512], [600, 512, 700, 513, 30]),         # one member each
                                                ([0, 0, 0, 0, 0], [128], [500, 128, 200, 129, 140])])                  # 512 tokens saved: tiles
def test_small_groups_against_the_attention_without(T, of, group_lens, lens, dtype, bits):  # noqa: F811
    b = Batch(of, group_lens, lens, 2, 128, 64, 12, dtype, bits, seed=2)
    q = _randn(5, 8, 128, dtype=dtype, seed=7)
    got, want = (f(q, out_dtype=torch.float32, return_lse=True) for f in (lambda *a, **k: b.call(T, *a, **k), lambda *a, **k: _plain(T, b, *a, **k)))
    live = torch.isfinite(want[1])
    scale = max(1.0, float(torch.nan_to_num(b.values[1].double()).abs().max()) / 6)
    assert _near(got[0] / scale, want[0] / scale, 500)
    assert torch.equal(live, torch.isfinite(got[1])) and bool(((got[1] - want[1])[live].abs() <= (500 + 2 * 256 * 40 + 16) * 2.0 ** -24).all())
    assert not bool(got[0][~live.any(-1)].any())

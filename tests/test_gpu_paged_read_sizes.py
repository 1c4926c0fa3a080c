"""Pages read back at sizes whose elements, heads or rows pass what one launch or 31 bits hold."""
import pytest
import torch

from tests.paged8_util import cache8
from tests.test_gpu_paged import I32, _ints, _randn
from tests.test_gpu_paged_prefix import T  # noqa: F401

pytestmark = pytest.mark.gpu
DT = torch.bfloat16


@pytest.fixture(autouse=True)
def give_memory_back():
    yield
    torch.cuda.empty_cache()


def _same_rows(rows, pages, names, step):
    """rows [N,D] are those of the pages [n,page,D] named names, compared in pieces."""
    N, page = rows.shape[0], pages.shape[1]
    flat = pages.reshape(-1, pages.shape[2])
    for at in range(0, N, step):
        n = torch.arange(at, min(N, at + step), device="cuda")
        assert torch.equal(rows[at:at + step], flat[names[n // page].long() * page + n % page]), at


@pytest.mark.parametrize("bits", [16, 8])
def test_more_elements_than_a_launch_has_threads(T, bits):  # noqa: F811
    """Heads of 6 channels are moved an element at a time: 2^32 and some of them."""
    D, page, N = 6, 256, (2 ** 32 // 6 // 2) + 1000
    width = -(-N // page)
    names = torch.randint(0, 7, (2, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=I32)
    kp, vp = (_randn(7, 1, page, D, dtype=DT, seed=i) for i in (0, 1))
    lens = _ints([N, N - 77])
    if bits == 16:
        k, v = T.thrift_paged_read(kp, vp, names, lens, N)
        want = kp, vp
    else:
        codes = cache8(kp, vp)
        few = torch.arange(7, dtype=I32, device="cuda").view(7, 1)
        want = [x.reshape(7, 1, page, D) for x in T.thrift_paged_read8(*codes, few, _ints([page] * 7), page, DT)]
        k, v = T.thrift_paged_read8(*codes, names, lens, N, DT)
    for got, pages in zip((k, v), want):
        _same_rows(got[0, 0], pages[:, 0], names[0], 1 << 25)
        _same_rows(got[1, 0, :N - 77], pages[:, 0], names[1], 1 << 25)
        assert not bool(got[1, 0, N - 77:].any())


@pytest.mark.parametrize("bits", [16, 8])
def test_more_heads_than_a_launch_has_workgroups(T, bits):  # noqa: F811
    """One token of 2^24 heads and more."""
    B, Hkv, D, page = 2 ** 20 + 3, 16, 8, 16
    kp, vp = (_randn(5, Hkv, page, D, dtype=DT, seed=i) for i in (0, 1))
    g = torch.Generator(device="cuda").manual_seed(2)
    names = torch.randint(0, 5, (B, 1), generator=g, device="cuda", dtype=I32)
    lens, first = (torch.randint(0, page, (B,), generator=g, device="cuda", dtype=I32) for _ in range(2))
    if bits == 16:
        k, v = T.thrift_paged_read(kp, vp, names, lens, 1, first=first)
        want = kp, vp
    else:
        codes = cache8(kp, vp)
        want = T.thrift_paged_read8(*codes, torch.arange(5, dtype=I32, device="cuda").view(5, 1), _ints([page] * 5), page, DT)
        k, v = T.thrift_paged_read8(*codes, names, lens, 1, DT, first=first)
    for got, pages in zip((k, v), want):
        rows = pages[names[:, 0].long(), :, first.long()]
        rows[first >= lens] = 0
        assert torch.equal(got[:, :, 0], rows)


def test_the_longest_rows(T):  # noqa: F811
    """2^31 - 1 tokens of one head, of which the sequence has all but the last 255."""
    D, page, N = 8, 256, 2 ** 31 - 1
    width = 2 ** 23 - 1                                                      # 2^31 - 256 tokens
    names = torch.randint(0, 7, (1, width), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=I32)
    kp, vp = (_randn(7, 1, page, D, dtype=DT, seed=i) for i in (0, 1))
    k, v = T.thrift_paged_read(kp, vp, names, _ints([2 ** 31 - 1]), N)
    for got, pages in ((k, kp), (v, vp)):
        _same_rows(got[0, 0, :width * page], pages[:, 0], names[0], 1 << 24)
        assert not bool(got[0, 0, width * page:].any())

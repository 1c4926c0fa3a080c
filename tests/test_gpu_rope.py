"""Rotary positions on the GPU against 64 bits: layouts, parts of the head, strides, alignment, far positions, and the gradient."""
import pytest
import torch

from tests.paged_util import LAYOUTS, check_rounded, rope64

pytestmark = pytest.mark.gpu
DTYPES = (torch.float16, torch.bfloat16)


@pytest.fixture(scope="module")
def T():
    from paper_2605_23081_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


def _randn(*shape, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def _positions(T, B, N, positions):
    if positions is None:
        return torch.arange(N, device="cuda").expand(B, N)
    return positions.expand(B, N) if positions.dim() == 1 else positions


def _check(T, q, k, freqs, positions, layout, gain, got, sign=1.0):
    for x, y in zip((q, k), got):
        if x is not None:
            want, err = rope64(x, _positions(T, x.shape[0], x.shape[2], positions), freqs, layout, gain, sign)
            check_rounded(y, want, err)


# sizes on both sides of the 16-byte accesses: heads of 2 to 256 channels, parts of them, one token to some hundreds
SIZES = [(1, 1, 1, 1, 128, 128), (3, 1, 32, 8, 128, 128), (2, 7, 4, 2, 128, 64), (1, 130, 8, 8, 64, 64), (2, 33, 6, 3, 256, 256), (1, 19, 5, 1, 96, 48),
         (1, 5, 2, 2, 128, 6), (2, 9, 3, 1, 80, 80), (1, 3, 2, 1, 2, 2), (1, 4, 3, 2, 30, 14), (1, 257, 40, 8, 128, 128), (5, 1, 3, 2, 1024, 1024), (1, 2, 64, 8, 128, 32),
         (1, 5003, 2, 1, 128, 128), (3, 1501, 2, 1, 64, 32), (1, 9001, 1, 1, 48, 16), (2, 1050, 3, 2, 256, 256), (1, 1100, 9, 4, 16, 16), (1, 700, 40, 8, 512, 256)]


@pytest.mark.parametrize("B,N,Hq,Hkv,D,rot", SIZES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_against_64_bits(T, B, N, Hq, Hkv, D, rot, layout, dtype):
    print(f"rope B={B} N={N} Hq={Hq} Hkv={Hkv} D={D} rot={rot} {layout} {dtype}", flush=True)
    q, k = _randn(B, Hq, N, D, dtype=dtype), _randn(B, Hkv, N, D, dtype=dtype, seed=1)
    freqs, _ = T.rope_frequencies(rot, 1e6, device="cuda")
    pos = torch.randint(0, 262144, (B, N), dtype=torch.int32, device="cuda")
    kept = q.clone(), k.clone()
    for p, gain in ((None, 1.0), (pos, 1.1386), (pos[0].contiguous(), 1.0)):
        for f, sign in ((T.thrift_rope, 1.0), (T.thrift_rope_backward, -1.0)):
            _check(T, q, k, freqs, p, layout, gain, f(q, k, freqs, p, layout, gain), sign)
    got, none = T.thrift_rope(q, None, freqs, pos, layout)
    assert none is None
    _check(T, q, None, freqs, pos, layout, 1.0, (got, None))
    assert torch.equal(q, kept[0]) and torch.equal(k, kept[1])


@pytest.mark.parametrize("layout", LAYOUTS)
def test_far_and_negative_positions(T, layout):
    q = _randn(1, 2, 6, 128, dtype=torch.float16)
    freqs, _ = T.rope_frequencies(128, 1e4, device="cuda")
    pos = torch.tensor([[0, 2 ** 31 - 1, -1, -2 ** 31, 10 ** 7, -262143]], dtype=torch.int32, device="cuda")
    _check(T, q, None, freqs, pos, layout, 1.0, T.thrift_rope(q, None, freqs, pos, layout))


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rot", [128, 64, 20])
def test_quarter_turns_are_exact(T, layout, rot):
    """Multiples of a quarter of a turn: cos and sin are 0 and +-1 but for the rounding of the frequency itself."""
    x = _randn(1, 3, 8, 128, dtype=torch.bfloat16)
    freqs = torch.full((rot // 2,), 1.5707963267948966, dtype=torch.float64, device="cuda")
    got, _ = T.thrift_rope(x, None, freqs, layout=layout)
    _check(T, x, None, freqs, None, layout, 1.0, (got, None))
    assert torch.equal(got[:, :, 0], x[:, :, 0]) and torch.equal(got[:, :, 4], x[:, :, 4])
    assert torch.equal(got[:, :, 2, :rot], -x[:, :, 2, :rot]) and torch.equal(got[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("shift", [0, 1, 4, 8])
def test_views_of_a_fused_projection(T, dtype, layout, shift):
    """q and k inside [B,N,heads,D] at an offset that does or does not keep 16-byte alignment; results into such a tensor and
    in place; what lies between the heads is left alone."""
    B, N, Hq, Hkv, D = 2, 21, 6, 2, 128
    n = N * (Hq + 2 * Hkv) * D
    buf = _randn(B * n + 64, dtype=dtype)
    view = lambda t: t[shift:shift + B * n].view(B, N, Hq + 2 * Hkv, D).transpose(1, 2)
    q, k = view(buf)[:, :Hq], view(buf)[:, Hq:Hq + Hkv]
    freqs, gain = T.rope_frequencies(64, 1e4, "by_parts", 4.0, 4096, device="cuda")
    want = T.thrift_rope(q.contiguous(), k.contiguous(), freqs, None, layout, gain)
    _check(T, q, k, freqs, None, layout, gain, want)
    for a, b in zip(T.thrift_rope(q, k, freqs, None, layout, gain), want):
        assert a.is_contiguous() and torch.equal(a, b)
    out = torch.full_like(buf, 7.0)
    qo, ko = view(out)[:, :Hq], view(out)[:, Hq:Hq + Hkv]
    T.thrift_rope(q, k, freqs, None, layout, gain, qo, ko)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    rest = torch.ones_like(out, dtype=torch.bool)
    view(rest)[:, :Hq + Hkv] = False
    assert bool((out[rest] == 7.0).all())
    before = buf.clone()
    T.thrift_rope(q, k, freqs, None, layout, gain, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(buf[rest], before[rest])


def test_repeated_inputs_and_odd_strides(T):
    freqs, _ = T.rope_frequencies(128, 1e4, device="cuda")
    one = _randn(1, 1, 9, 128, dtype=torch.float16)
    wide = one.expand(3, 5, 9, 128)
    got, _ = T.thrift_rope(wide, None, freqs)
    assert torch.equal(got, T.thrift_rope(one, None, freqs)[0].expand(3, 5, 9, 128))
    loose = _randn(2, 3, 9, 131, dtype=torch.float16)[..., :128]                        # rows of 131 elements
    assert torch.equal(T.thrift_rope(loose, None, freqs)[0], T.thrift_rope(loose.contiguous(), None, freqs)[0])


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("rot", [128, 48])
def test_gradient_against_differences(T, layout, rot):
    """The rotation is linear: the difference of two outputs is the output of the difference, so that <g, f(x + d) - f(x)> has to be
    <backward(g), d>.  Small whole numbers keep x and x + d exact in 16 bits; what is left are the roundings of three outputs."""
    B, H, N, D = 2, 3, 17, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randint(-8, 9, (B, H, N, D), generator=g, device="cuda").half()
    freqs, gain = T.rope_frequencies(rot, 1e4, "by_parts", 8.0, 2048, device="cuda")
    pos = torch.randint(0, 100000, (B, N), dtype=torch.int32, device="cuda")
    f = lambda t: T.thrift_rope(t, None, freqs, pos, layout, gain)[0].double()
    grad = _randn(B, H, N, D, dtype=torch.float16, seed=2)
    back = T.thrift_rope_backward(grad, None, freqs, pos, layout, gain)[0].double()
    for c in (0, 1, rot // 2, rot - 1, rot, D - 1):
        if c >= D:
            continue
        d = torch.zeros_like(x)
        d[..., c] = 4
        change = f(x + d) - f(x)
        # a head's outputs are at most 12 * sqrt(2) * gain < 32: half a step is 2^-7 at most, in both outputs, at the two channels that move
        lhs, rhs = (grad.double() * change).sum(-1), 4 * back[..., c]
        tol = 2 * 2.0 ** -7 * grad.double().abs().sort(-1).values[..., -2:].sum(-1) + 2.0 ** -11 * rhs.abs() + 1e-4
        assert bool(((lhs - rhs).abs() <= tol).all()), (c, float((lhs - rhs).abs().max()))


def test_nan_and_infinity_pass_through(T):
    x = _randn(1, 1, 4, 128, dtype=torch.bfloat16)
    x[0, 0, 1, 3], x[0, 0, 2, 70], x[0, 0, 3, 127] = float("nan"), float("inf"), float("nan")
    freqs, _ = T.rope_frequencies(64, 1e4, device="cuda")
    got, _ = T.thrift_rope(x, None, freqs, positions=torch.full((4,), 3, dtype=torch.int32, device="cuda"))
    bad = ~torch.isfinite(got[0, 0])
    assert bad.nonzero().tolist() == [[1, 3], [1, 35], [2, 70], [3, 127]]


def test_another_stream_and_replays(T):
    q, k = _randn(2, 4, 33, 128, dtype=torch.float16), _randn(2, 2, 33, 128, dtype=torch.float16, seed=1)
    freqs, _ = T.rope_frequencies(128, 1e4, device="cuda")
    want = T.thrift_rope(q, k, freqs)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = T.thrift_rope(q, k, freqs)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = T.thrift_rope(q, k, freqs)
    for i in range(3):
        q.copy_(_randn(2, 4, 33, 128, dtype=torch.float16, seed=10 + i))
        want = T.thrift_rope(q, k, freqs)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))

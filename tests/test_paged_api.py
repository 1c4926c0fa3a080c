"""Rotary positions and the paged cache on the CPU: frequencies, and everything that is refused before a launch."""
import ctypes as C
import math

import pytest
import torch

from paper_2605_23081_amd import binding as T

NULL, SHAPE, DTYPE, WORKSPACE, ARCH = 1, 2, 3, 5, 6
FAKE = C.c_void_p(0x1000)      # never followed: every call below must be refused first


def test_plain_linear_and_ntk_frequencies():
    for rot, base in ((128, 1e4), (64, 1e6), (2, 500.0), (96, 1e4), (1024, 1e5)):
        f, gain = T.rope_frequencies(rot, base)
        assert f.dtype == torch.float64 and gain == 1.0 and f.numel() == rot // 2
        for i in range(rot // 2):
            assert math.isclose(f[i], base ** (-2 * i / rot), rel_tol=1e-14)
        linear, gain = T.rope_frequencies(rot, base, "linear", 8.0)
        assert gain == 1.0 and torch.allclose(linear, f / 8, rtol=1e-14, atol=0)
        if rot > 2:
            ntk, gain = T.rope_frequencies(rot, base, "ntk", 8.0)
            assert gain == 1.0 and ntk[0] == 1.0 and math.isclose(ntk[-1], f[-1] / 8, rel_tol=1e-12)
            assert bool((ntk <= f).all()) and bool((ntk >= f / 8 * (1 - 1e-12)).all())


def test_frequencies_by_parts():
    rot, base, factor, original = 128, 1e6, 4.0, 32768
    f, _ = T.rope_frequencies(rot, base)
    got, gain = T.rope_frequencies(rot, base, "by_parts", factor, original)
    assert math.isclose(gain, 0.1 * math.log(4.0) + 1.0, rel_tol=1e-7)
    kept = slowed = 0
    for theta, g in zip(f.tolist(), got.tolist()):
        turns = original * theta / (2 * math.pi)
        if turns >= 32:
            assert g == theta
            kept += 1
        elif turns <= 1:
            assert math.isclose(g, theta / factor, rel_tol=1e-14)
            slowed += 1
        else:
            assert theta / factor < g < theta
    assert kept and slowed
    # a factor of 1 changes nothing
    same, gain = T.rope_frequencies(rot, base, "by_parts", 1.0, original)
    assert gain == 1.0 and torch.allclose(same, f, rtol=1e-15, atol=0)


@pytest.mark.parametrize("kw", [dict(rot=0), dict(rot=-2), dict(rot=3), dict(rot=1026), dict(base=1.0), dict(base=math.inf), dict(base=math.nan),
                                dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=math.nan), dict(scaling="ntk", rot=2, factor=2.0),
                                dict(scaling="ntk", factor=math.inf), dict(scaling="by_parts", factor=2.0), dict(scaling="by_parts", factor=2.0, original=math.inf),
                                dict(scaling="by_parts", factor=2.0, original=4096, slow=32.0), dict(scaling="by_parts", factor=2.0, original=4096, slow=-1.0)])
def test_frequencies_refuse(kw):
    with pytest.raises(T.ThriftError) as e:
        T.rope_frequencies(**{**dict(rot=64), **kw})
    assert e.value.code == SHAPE
    assert T.lib().thrift_rope_frequencies(64, 1e4, 4, 1.0, 0.0, 1.0, 32.0, (C.c_double * 32)(), None) == SHAPE
    assert T.lib().thrift_rope_frequencies(64, 1e4, 0, 1.0, 0.0, 1.0, 32.0, None, None) == NULL


@pytest.mark.parametrize("name", ["thrift_rope", "thrift_rope_backward"])
def test_rope_refuses_before_a_launch(name):
    def call(q=FAKE, qo=FAKE, Hq=4, k=FAKE, ko=FAKE, Hkv=2, dt=0, freqs=FAKE, rot=128, layout=0, B=1, N=8, D=128):
        return getattr(T.lib(), name)(q, None, qo, None, Hq, k, None, ko, None, Hkv, dt, None, 0, freqs, rot, layout, 1.0, B, N, D, None)
    assert call(q=None) == NULL and call(qo=None) == NULL and call(k=None) == NULL and call(ko=None) == NULL and call(freqs=None) == NULL
    assert call(dt=2) == DTYPE and call(dt=7) == DTYPE
    for bad in (dict(Hq=0), dict(Hkv=0), dict(rot=0), dict(rot=3), dict(rot=130), dict(rot=-2), dict(layout=2), dict(layout=-1), dict(B=0), dict(N=0),
                dict(D=0), dict(D=127, rot=126), dict(D=1026), dict(B=1 << 16, N=1 << 16), dict(Hq=1 << 30)):
        assert call(**bad) == SHAPE, bad
    if not torch.cuda.is_available():
        assert call() == ARCH and call(k=None, ko=None, Hkv=0) == ARCH


def test_page_calls_refuse_before_a_launch():
    L = T.lib()
    other = C.c_void_p(0x2000)

    def page_map(sl=FAKE, new=FAKE, B=4, ps=16, n=64, bt=FAKE, mp=8, fp=FAKE, cap=64, fc=FAKE, rows=32, slots=FAKE, pos=FAKE, st=FAKE, so=other, fo=other):
        return L.thrift_page_map(sl, new, B, ps, n, bt, mp, fp, cap, fc, rows, slots, pos, st, so, fo, None)
    for bad in ("sl", "new", "bt", "fp", "fc", "slots", "pos", "st", "so", "fo"):
        assert page_map(**{bad: None}) == NULL, bad
    for bad in (dict(B=0), dict(B=4097), dict(ps=8), dict(ps=24), dict(ps=512), dict(ps=0), dict(n=0), dict(mp=0), dict(cap=0), dict(rows=0), dict(so=FAKE),
                dict(fo=FAKE), dict(n=1 << 28), dict(mp=1 << 28), dict(mp=(1 << 27) - 1, rows=64)):
        assert page_map(**bad) == SHAPE, bad

    def release(sl=FAKE, drop=FAKE, B=4, ps=16, n=64, bt=FAKE, mp=8, fp=FAKE, cap=64, fc=FAKE, so=other, fo=other):
        return L.thrift_page_release(sl, drop, B, ps, n, bt, mp, fp, cap, fc, so, fo, None)
    for bad in ("sl", "drop", "bt", "fp", "fc", "so", "fo"):
        assert release(**{bad: None}) == NULL, bad
    for bad in (dict(B=0), dict(B=4097), dict(ps=8), dict(n=0), dict(mp=0), dict(cap=0), dict(so=FAKE), dict(fo=FAKE)):
        assert release(**bad) == SHAPE, bad

    def append(q=FAKE, qo=FAKE, Hq=4, k=FAKE, v=FAKE, Hkv=2, dt=0, T_=8, slots=FAKE, pos=FAKE, freqs=FAKE, rot=128, layout=0, kp=FAKE, vp=FAKE, n=8, ps=16, D=128):
        return L.thrift_paged_append(q, None, qo, Hq, k, None, v, None, Hkv, dt, T_, slots, pos, freqs, rot, layout, 1.0, kp, vp, n, ps, D, None)
    for bad in ("qo", "k", "v", "slots", "pos", "freqs", "kp", "vp"):
        assert append(**{bad: None}) == NULL, bad
    assert append(dt=2) == DTYPE
    for bad in (dict(Hq=0), dict(Hkv=0), dict(T_=0), dict(rot=3), dict(rot=130), dict(layout=2), dict(n=0), dict(ps=8), dict(ps=48), dict(D=0), dict(D=2048),
                dict(D=127, rot=126), dict(n=1 << 28)):
        assert append(**bad) == SHAPE, bad

    def decode(q=FAKE, dt=0, kp=FAKE, vp=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, B=2, Hq=4, Hkv=2, D=128, ps=16, out=FAKE, odt=0, ws=FAKE, size=1 << 40):
        return L.thrift_paged_decode(q, dt, kp, vp, n, bt, mp, sl, B, Hq, Hkv, D, ps, 0.0, out, odt, None, ws, size, None)
    for bad in ("q", "kp", "vp", "bt", "sl", "out"):
        assert decode(**{bad: None}) == NULL, bad
    assert decode(dt=2) == DTYPE and decode(odt=3) == DTYPE
    for bad in (dict(B=0), dict(Hq=0), dict(Hkv=0), dict(Hq=5), dict(Hq=66), dict(D=96), dict(D=512), dict(ps=8), dict(ps=20), dict(mp=0), dict(n=0),
                dict(n=1 << 28), dict(mp=1 << 28), dict(B=1 << 20, Hq=32, Hkv=8)):
        assert decode(**bad) == SHAPE, bad
    for bad in ("q", "kp", "vp", "out"):
        assert decode(**{bad: C.c_void_p(0x1008)}) == SHAPE, bad
    need = L.thrift_paged_decode_workspace(2, 4, 2, 800, 16, 128)
    assert need > 0 and L.thrift_paged_decode_workspace(2, 4, 2, 8, 16, 128) == 0            # a workgroup per row needs none
    assert decode(mp=800, ws=None) == WORKSPACE and decode(mp=800, size=need - 1) == WORKSPACE and decode(mp=800, ws=C.c_void_p(0x1008)) == WORKSPACE
    assert L.thrift_paged_decode_workspace(2, 5, 2, 8, 16, 128) == 0 and L.thrift_paged_decode_workspace(2, 4, 2, 8, 16, 96) == 0
    if not torch.cuda.is_available():
        assert page_map() == ARCH and release() == ARCH and append() == ARCH and append(q=None, qo=None, Hq=0) == ARCH and decode() == ARCH
        assert append(rot=0, pos=None, freqs=None) == ARCH


def test_sizes_past_32_bits_are_refused():
    """Sizes whose low 32 bits would be accepted."""
    L, other, over = T.lib(), C.c_void_p(0x2000), 2 ** 32
    page_map = lambda B=4, ps=16, n=64, mp=8, rows=32: L.thrift_page_map(FAKE, FAKE, B, ps, n, FAKE, mp, FAKE, 64, FAKE, rows, FAKE, FAKE, FAKE, other, other, None)
    release = lambda B=4, ps=16, n=64, mp=8: L.thrift_page_release(FAKE, FAKE, B, ps, n, FAKE, mp, FAKE, 64, FAKE, other, other, None)
    append = lambda Hq=4, Hkv=2, T_=8, rot=128, layout=0, n=8, ps=16, D=128: L.thrift_paged_append(
        FAKE, None, FAKE, Hq, FAKE, None, FAKE, None, Hkv, 0, T_, FAKE, FAKE, FAKE, rot, layout, 1.0, FAKE, FAKE, n, ps, D, None)
    decode = lambda n=8, mp=8, B=2, Hq=4, Hkv=2, D=128, ps=16: L.thrift_paged_decode(
        FAKE, 0, FAKE, FAKE, n, FAKE, mp, FAKE, B, Hq, Hkv, D, ps, 0.0, FAKE, 0, None, FAKE, 1 << 40, None)
    rope = lambda Hq=4, Hkv=2, rot=128, layout=0, B=1, N=8, D=128: L.thrift_rope(
        FAKE, None, FAKE, None, Hq, FAKE, None, FAKE, None, Hkv, 0, None, 0, FAKE, rot, layout, 1.0, B, N, D, None)
    for call in (page_map, release, append, decode, rope):
        for name, value in zip(call.__code__.co_varnames, call.__defaults__):
            assert call(**{name: value + over}) == SHAPE and call(**{name: value - over}) == SHAPE, (call, name)
    assert L.thrift_paged_decode_workspace(2, 4, 2, 800 + over, 16, 128) == 0
    assert append(rot=over) == SHAPE                                                     # whose low bits say that nothing is rotated
    with pytest.raises(T.ThriftError) as e:
        T.rope_frequencies(64 + over)
    assert e.value.code == SHAPE


def test_binding_refuses_what_the_kernels_cannot_index():
    h, i32, f64 = torch.float16, torch.int32, torch.float64
    q, k = torch.zeros(2, 4, 8, 128, dtype=h), torch.zeros(2, 2, 8, 128, dtype=h)
    freqs = torch.zeros(64, dtype=f64)
    with pytest.raises(AssertionError, match="current device"):
        T.thrift_rope(q, k, freqs)                                                       # host tensors
    with pytest.raises(AssertionError, match="contiguous"):
        T.thrift_rope(q.transpose(2, 3), None, freqs)
    with pytest.raises(AssertionError, match="coincide"):
        T.thrift_rope(q, None, freqs, q_out=torch.zeros(1, 1, 1, 128, dtype=h).expand(2, 4, 8, 128))
    for bad in (dict(q=q.float()), dict(k=k.bfloat16()), dict(k=k[:1]), dict(freqs=freqs.float()), dict(positions=torch.zeros(8)), dict(positions=torch.zeros(7, dtype=i32)),
                dict(q_out=q[:, :2]), dict(k_out=k.float()), dict(k=None, k_out=k)):
        with pytest.raises(AssertionError):
            T.thrift_rope(**{**dict(q=q, k=k, freqs=freqs), **bad})
    ints = dict(seqlens=torch.zeros(3, dtype=i32), new_lens=torch.zeros(3, dtype=i32), block_table=torch.zeros(3, 5, dtype=i32),
                free_pages=torch.zeros(9, dtype=i32), free_count=torch.zeros(1, dtype=i32))
    for bad in (dict(seqlens=torch.zeros(4, dtype=i32)), dict(new_lens=torch.zeros(3)), dict(block_table=torch.zeros(5, 3, dtype=i32).t()),
                dict(free_pages=torch.zeros(18, dtype=i32)[::2]), dict(free_count=torch.zeros(2, dtype=i32)), dict()):
        with pytest.raises(AssertionError):
            T.thrift_page_map(**{**ints, **bad}, page_size=16, n_pages=9, rows=4)
    pages = torch.zeros(9, 2, 16, 128, dtype=h)
    kv = torch.zeros(4, 2, 128, dtype=h)
    slots = torch.zeros(4, dtype=i32)
    for bad in (dict(k=kv.bfloat16()), dict(v=kv[:3]), dict(slots=slots[:3]), dict(slots=slots.long()), dict(k_pages=pages[:, :1]), dict(v_pages=pages.bfloat16()),
                dict(q=torch.zeros(3, 4, 128, dtype=h)), dict(freqs=freqs), dict(freqs=freqs, positions=slots[:2]), dict(q_out=kv), dict()):
        with pytest.raises(AssertionError):
            T.thrift_paged_append(**{**dict(k=kv, v=kv, slots=slots, k_pages=pages, v_pages=pages), **bad})
    ok = dict(q=torch.zeros(3, 4, 128, dtype=h), k_pages=pages, v_pages=pages, block_table=torch.zeros(3, 5, dtype=i32), seqlens=torch.zeros(3, dtype=i32))
    for bad in (dict(q=torch.zeros(3, 4, 64, dtype=h)), dict(q=ok["q"].bfloat16()), dict(block_table=ok["block_table"][:2]), dict(seqlens=ok["seqlens"].long()), dict()):
        with pytest.raises(AssertionError):
            T.thrift_paged_decode(**{**ok, **bad})


def test_only_32_heads_of_256_channels_reload_registers_in_the_walk(tmp_path):
    """Keys and values are in flight during the walk over a row's steps, and a reload of a spilled register waits for them."""
    import os
    import subprocess
    from paper_2605_23081_amd import build
    source, listing = "thrift_paged_decode.hip", tmp_path / "paged.s"
    subprocess.run(["hipcc", *build.flags(source), "-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", str(listing)],
                   check=True, capture_output=True)
    assert all("paged_decode_kernel" in k and "Li256ELi2E" in k for k in build.scratch_in_loops(listing.read_text()))


def test_elements_that_coincide_are_seen():
    x = torch.zeros(4, 6, 8)
    assert T._apart(x) and T._apart(x.transpose(0, 2)) and T._apart(x[:, ::2]) and T._apart(x[:1].expand(1, 6, 8)) and T._apart(torch.zeros(5, 1, 3))
    assert not T._apart(x[:1].expand(4, 6, 8)) and not T._apart(x.as_strided((4, 8), (4, 1))) and T._apart(x.as_strided((4, 8), (8, 1)))


def test_tensors_without_storage_are_left_to_the_general_path():
    """Under a transform a tensor has sizes but no data pointer; refusing it must not end the process."""
    from torch._subclasses.fake_tensor import FakeTensorMode
    m = T._native()
    h, i32 = torch.float16, torch.int32
    with FakeTensorMode():
        z = lambda *s, dt=h: torch.zeros(*s, dtype=dt, device="cuda")
        q, freqs, k, pages = z(1, 2, 3, 128), z(64, dt=torch.float64), z(3, 2, 128), z(4, 2, 16, 128)
        ints, table, ws = z(3, dt=i32), z(3, 1, dt=i32), z(1 << 20, dt=torch.uint8)
        out, lse = z(3, 2, 128), z(3, 2, dt=torch.float32)
    seen = []

    def served(q, k):
        seen.append(m.rope(0, q, None, freqs, None, 0, 1.0, q, None, 0, 0))
        seen.append(m.page_map(ints, ints, table, ints, ints[:1], 16, 4, 3, 0, 0))
        seen.append(m.paged_append(k, k, ints, pages, pages, None, None, None, None, 0, 1.0, 0, 0))
        seen.append(m.paged_decode(k, pages, pages, table, ints, 0.0, out, lse, 1, ws, 0, 0))
        return q

    torch.vmap(served)(q.unsqueeze(0), k.unsqueeze(0))
    assert seen == [None] * 4
    assert m.rope() is None and m.page_map() is None and m.paged_append() is None and m.paged_decode() is None

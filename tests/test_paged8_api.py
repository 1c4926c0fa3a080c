"""The 8-bit paged cache, reading pages back and attention over common starts on the CPU: everything that is refused before a launch."""
import ctypes as C

import pytest
import torch

from paper_2605_23081_amd import binding as T
from tests.paged8_util import codes64, quantise64, values64

NULL, SHAPE, DTYPE, WORKSPACE, ARCH = 1, 2, 3, 5, 6
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1008)      # never followed: every call below must be refused first
OVER = 2 ** 32


def append8(q=FAKE, qo=FAKE, Hq=4, k=FAKE, v=FAKE, Hkv=2, dt=0, T_=8, slots=FAKE, pos=FAKE, freqs=FAKE, rot=128, layout=0, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE,
            n=8, ps=16, D=128):
    return T.lib().thrift_paged_append8(q, None, qo, Hq, k, None, v, None, Hkv, dt, T_, slots, pos, freqs, rot, layout, 1.0, kc, ks, vc, vs, n, ps, D, None)


def decode8(q=FAKE, dt=0, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, B=2, Hq=4, Hkv=2, D=128, ps=16, out=FAKE, odt=0, ws=FAKE, size=1 << 40):
    return T.lib().thrift_paged_decode8(q, dt, kc, ks, vc, vs, n, bt, mp, sl, B, Hq, Hkv, D, ps, 0.0, out, odt, None, ws, size, None)


def read(kp=FAKE, vp=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, B=2, Hkv=2, N=40, D=128, ps=16, ko=FAKE, vo=FAKE):
    return T.lib().thrift_paged_read(kp, vp, n, bt, mp, None, sl, B, Hkv, N, D, ps, ko, vo, None)


def read8(kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, B=2, Hkv=2, N=40, D=128, ps=16, ko=FAKE, vo=FAKE, dt=0):
    return T.lib().thrift_paged_read8(kc, ks, vc, vs, n, bt, mp, None, sl, B, Hkv, N, D, ps, ko, vo, dt, None)


def prefix(q=FAKE, dt=0, kp=FAKE, vp=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, go=FAKE, gl=FAKE, ng=2, B=2, Hq=4, Hkv=2, D=128, ps=16, out=FAKE, odt=0, ws=FAKE,
           size=1 << 40):
    return T.lib().thrift_paged_decode_prefix(q, dt, kp, vp, n, bt, mp, sl, go, gl, ng, B, Hq, Hkv, D, ps, 0.0, out, odt, None, ws, size, None)


def prefix8(q=FAKE, dt=0, kc=FAKE, ks=FAKE, vc=FAKE, vs=FAKE, n=8, bt=FAKE, mp=8, sl=FAKE, go=FAKE, gl=FAKE, ng=2, B=2, Hq=4, Hkv=2, D=128, ps=16, out=FAKE,
            odt=0, ws=FAKE, size=1 << 40):
    return T.lib().thrift_paged_decode_prefix8(q, dt, kc, ks, vc, vs, n, bt, mp, sl, go, gl, ng, B, Hq, Hkv, D, ps, 0.0, out, odt, None, ws, size, None)


CALLS = (append8, decode8, read, read8, prefix, prefix8)
NULLABLE = {"q": (append8,), "ws": (decode8, prefix, prefix8)}     # q None leaves q_out unused; a workspace has a status of its own


def _defaults(call):
    return zip(call.__code__.co_varnames, call.__defaults__)


@pytest.mark.parametrize("call", CALLS)
def test_null_pointers_types_and_sizes_are_refused(call):
    for name, value in _defaults(call):
        if value is FAKE and call not in NULLABLE.get(name, ()):
            assert call(**{name: None}) == NULL, name
    names = dict(_defaults(call))
    if "dt" in names:
        assert call(dt=2) == DTYPE and call(dt=7) == DTYPE and call(dt=-1) == DTYPE
    if "odt" in names:
        assert call(odt=3) == DTYPE
    bad = dict(Hq=(0, 5, 66, -4), Hkv=(0, -1), T_=(0, -1, 1 << 23), rot=(3, 130, -2), layout=(2,), n=(0, 1 << 28), ps=(8, 20, 0, 512), D=(0, 127, 2048, 1026),
               mp=(0, 1 << 28), B=(0, -1), N=(0, -1, 1 << 30), ng=(0, -1, 4097))
    if call is append8:
        bad["Hq"] = (0, -4, 1 << 30)
    if call in (decode8, prefix, prefix8):
        bad["D"] += (96, 32, 512)
    if call in (prefix, prefix8):
        bad["B"] += (4097,)
    for name, values in bad.items():
        for value in values if name in names else ():
            assert call(**{name: value}) == SHAPE, (name, value)
    if call in (decode8, prefix, prefix8):
        for name in ("q", "kc", "ks", "vc", "vs", "kp", "vp", "out"):
            assert name not in names or call(**{name: ODD}) == SHAPE, name
    if not torch.cuda.is_available():
        assert call() == ARCH


@pytest.mark.parametrize("call", CALLS)
def test_sizes_past_32_bits_are_refused(call):
    """Sizes whose low 32 bits would be accepted."""
    for name, value in _defaults(call):
        if isinstance(value, int) and name not in ("dt", "odt", "size"):
            assert call(**{name: value + OVER}) == SHAPE and call(**{name: value - OVER}) == SHAPE, name


def test_rows_past_what_a_grid_reaches_are_refused():
    for call in (read, read8):
        assert call(B=1 << 20, Hkv=16, N=255) == SHAPE                                     # 2^31 and more rows
        assert call(B=1 << 10, Hkv=1 << 10, N=2047, D=1024) == SHAPE                       # 2^41 elements


def test_workspaces():
    L = T.lib()
    for size, call in ((lambda **k: L.thrift_paged_decode8_workspace(*{**dict(B=2, Hq=4, Hkv=2, mp=800, ps=16, D=128), **k}.values()), decode8),
                       (lambda **k: L.thrift_paged_decode_prefix_workspace(16, *{**dict(B=2, Hq=4, Hkv=2, ng=2, mp=800, ps=16, D=128), **k}.values()), prefix),
                       (lambda **k: L.thrift_paged_decode_prefix_workspace(8, *{**dict(B=2, Hq=4, Hkv=2, ng=2, mp=800, ps=16, D=128), **k}.values()), prefix8)):
        need = size()
        if need:
            assert call(mp=800, ws=None) == WORKSPACE and call(mp=800, size=need - 1) == WORKSPACE and call(mp=800, ws=ODD) == WORKSPACE
        else:
            assert call is decode8
        assert size(Hq=5) == 0 and size(D=96) == 0 and size(ps=24) == 0 and size(B=0) == 0 and size(mp=800 + OVER) == 0
    assert L.thrift_paged_decode_prefix_workspace(12, 2, 4, 2, 2, 800, 16, 128) == 0
    for bad in (dict(B=4097), dict(ng=0), dict(ng=4097)):
        assert L.thrift_paged_decode_prefix_workspace(16, *{**dict(B=2, Hq=4, Hkv=2, ng=2, mp=800, ps=16, D=128), **bad}.values()) == 0


def test_binding_refuses_what_the_kernels_cannot_index():
    h, i32, u8 = torch.float16, torch.int32, torch.uint8
    codes, scales, kv = torch.zeros(9, 2, 16, 128, dtype=u8), torch.zeros(9, 2, 16, dtype=u8), torch.zeros(4, 2, 128, dtype=h)
    slots, table, lens = torch.zeros(4, dtype=i32), torch.zeros(3, 5, dtype=i32), torch.zeros(3, dtype=i32)
    pages = dict(k_codes=codes, k_scales=scales, v_codes=codes, v_scales=scales)
    wrong_pages = (dict(k_codes=codes[:, :1]), dict(k_codes=codes.to(torch.int8)), dict(v_codes=codes[..., :64]), dict(k_scales=scales[..., :8]), dict(v_scales=scales.float()),
                   dict(k_scales=codes), dict(v_codes=codes.transpose(1, 2)), dict())      # (the last: host tensors)
    freqs = torch.zeros(64, dtype=torch.float64)
    for bad in wrong_pages + (dict(k=kv.float()), dict(v=kv[:3]), dict(v=kv.bfloat16()), dict(slots=slots.long()), dict(q=kv[:3]), dict(freqs=freqs),
                              dict(freqs=freqs, positions=slots[:2]), dict(q_out=kv), dict(k=kv[..., :64], v=kv[..., :64])):
        with pytest.raises(AssertionError):
            T.thrift_paged_append8(**{**dict(k=kv, v=kv, slots=slots, **pages), **bad})
    q = torch.zeros(3, 4, 128, dtype=h)
    for bad in wrong_pages + (dict(q=q.float()), dict(q=q[..., :64]), dict(block_table=table[:2]), dict(seqlens=lens.long()), dict(q=q[:2])):
        with pytest.raises(AssertionError):
            T.thrift_paged_decode8(**{**dict(q=q, block_table=table, seqlens=lens, **pages), **bad})
        with pytest.raises(AssertionError):
            T.thrift_paged_decode_prefix8(**{**dict(q=q, block_table=table, seqlens=lens, group_of=lens, group_lens=lens[:1], **pages), **bad})
    p16 = torch.zeros(9, 2, 16, 128, dtype=h)
    for bad in (dict(group_of=lens[:2]), dict(group_of=lens.long()), dict(group_lens=lens.float()), dict(group_lens=lens[::2]), dict(q=q.bfloat16()), dict()):
        with pytest.raises(AssertionError):
            T.thrift_paged_decode_prefix(**{**dict(q=q, k_pages=p16, v_pages=p16, block_table=table, seqlens=lens, group_of=lens, group_lens=lens), **bad})
    out = torch.zeros(3, 2, 7, 128, dtype=h)
    for bad in wrong_pages + (dict(N=8, k_out=out), dict(first=lens[:2]), dict(first=lens.long()), dict(v_out=out.float()), dict(dtype=torch.float32), dict(seqlens=lens[:2])):
        with pytest.raises(AssertionError):
            T.thrift_paged_read8(**{**dict(block_table=table, seqlens=lens, N=7, dtype=h, **pages), **bad})
    for bad in (dict(k_out=out[:2]), dict(v_out=out.transpose(1, 2)), dict(k_pages=p16.float()), dict(v_pages=p16.bfloat16()), dict()):
        with pytest.raises(AssertionError):
            T.thrift_paged_read(**{**dict(k_pages=p16, v_pages=p16, block_table=table, seqlens=lens, N=7), **bad})


def test_the_format_on_the_cpu():
    """The reference of the format against torch's own type, over all codes and their ties."""
    every = torch.arange(256, dtype=torch.uint8)
    values = values64(every, None)
    assert torch.equal(values.isnan(), every.view(torch.float8_e4m3fn).float().isnan())
    fine = ~values.isnan()
    assert torch.equal(values[fine], every[fine].view(torch.float8_e4m3fn).double())
    y = values[:127]
    halves = (y[1:] + y[:-1]) / 2
    for x in (y, -y, halves, -halves, halves * (1 + 1e-6), halves * (1 - 1e-6), torch.linspace(-448, 448, 9999, dtype=torch.float64)):
        assert torch.equal(codes64(x), x.float().to(torch.float8_e4m3fn).view(torch.uint8))
    for a, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (224.001, 0), (1.0, -8), (0.0, 0), (2.0 ** -120, -100), (3.3e38, 120), (65504.0, 8)):
        assert quantise64(torch.tensor([[a, 0.0]], dtype=torch.float64))[2].item() == e, a

"""Thin ctypes binding of the C ABI in include/thrift.h: argument marshalling only.

Every step of the path runs in the HIP kernels of libthrift_hip.so; PyTorch is used for device
memory and for the current stream.  There is no CPU fallback: if the library has not been built
(``python -m paper_2605_23081_amd.build``) importing a function from here raises.
"""
from __future__ import annotations

import ctypes as C
import math
import operator
import os
import warnings
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libthrift_hip.so")

F16, BF16, F32 = 0, 1, 2
_DT = {torch.float16: F16, torch.bfloat16: BF16, torch.float32: F32}

EXPORTS = (
    "thrift_status_string", "thrift_row_budget", "thrift_visible_blocks", "thrift_budget_to_global_k",
    "thrift_select_kmax", "thrift_block_means", "thrift_select_topk", "thrift_select_topk_shared", "thrift_select_ablation", "thrift_quantize_mxfp4", "thrift_prefill_prepass",
    "thrift_attn_prefill_workspace", "thrift_attn_prefill", "thrift_attn_prefill_chunk", "thrift_attn_prefill_ordered",
    "thrift_attn_decode_workspace", "thrift_attn_decode_least_workspace", "thrift_attn_decode", "thrift_attn_decode_shared", "thrift_attn_decode_static",
    "thrift_kv_cache_append", "thrift_kv_cache_append_advance",
    "thrift_attention_forward_workspace", "thrift_attention_forward",
    "thrift_rope_frequencies", "thrift_rope", "thrift_rope_backward", "thrift_page_map", "thrift_page_release",
    "thrift_paged_append", "thrift_paged_decode_workspace", "thrift_paged_decode", "thrift_paged_read",
    "thrift_paged_append8", "thrift_paged_decode8_workspace", "thrift_paged_decode8", "thrift_paged_read8",
    "thrift_paged_decode_prefix_workspace", "thrift_paged_decode_prefix", "thrift_paged_decode_prefix8", "thrift_peak_probe",
)

_lib = None


class ThriftError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: status {code} ({status_string(code)})")


class _Int:
    """A C int that keeps to its range: ctypes alone would take the low 32 bits of a larger size, which then might be an accepted one.  The
    ends of the range are refused by every call's limits."""

    @staticmethod
    def from_param(x):
        return C.c_int(max(-2 ** 31, min(2 ** 31 - 1, operator.index(x))))


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2605_23081_amd.build` "
                               "(there is no fallback path)")
        L = C.CDLL(LIB_PATH)
        i, d, f, p, sz = C.c_int, C.c_double, C.c_float, C.c_void_p, C.c_size_t
        L.thrift_status_string.restype = C.c_char_p
        L.thrift_status_string.argtypes = [i]
        L.thrift_row_budget.argtypes = [i, d, i]
        L.thrift_visible_blocks.argtypes = [i] * 6
        L.thrift_budget_to_global_k.argtypes = [i, d]
        L.thrift_select_kmax.argtypes = [i, i, i, i, i, d, i, i]
        L.thrift_block_means.argtypes = [p, i, i, i, i, i, i, p, p]
        L.thrift_select_topk.argtypes = [p, p, i, i, i, i, i, i, i, i, i, d, i, i, p, p, i, p]
        L.thrift_select_topk_shared.argtypes = L.thrift_select_topk.argtypes
        L.thrift_select_ablation.argtypes = [i, C.c_uint64, i, i, i, i, i, i, i, d, i, i, p, p, i, p]
        L.thrift_quantize_mxfp4.argtypes = [p, i, i, i, i, i, i, p, p, p]
        L.thrift_prefill_prepass.argtypes = [p, p, p, i, i, i, i, i, i, i, i, p, p, p, p, p, p, p, p, p]
        L.thrift_attn_prefill_workspace.restype = sz
        L.thrift_attn_prefill_workspace.argtypes = [i] * 8
        L.thrift_attn_prefill.argtypes = [p, p, p, i, p, p, p, p, p, p, p, p, i, i, i, i, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_attn_prefill_chunk.argtypes = [p, p, p, i, p, p, p, p, p, p, p, p, i, i, i, i, i, i, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_attn_prefill_ordered.argtypes = [p, p, p, i, p, p, p, p, p, p, p, p, i, i, i, i, i, i, i, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_attn_decode_workspace.restype = L.thrift_attn_decode_least_workspace.restype = sz
        L.thrift_attn_decode_workspace.argtypes = L.thrift_attn_decode_least_workspace.argtypes = [i] * 7
        L.thrift_attn_decode.argtypes = [p, i, p, p, p, p, p, p, p, p, i, i, i, i, i, i, d, i, i, f, p, i, p, p, i, p, sz, p]
        L.thrift_attn_decode_shared.argtypes = L.thrift_attn_decode.argtypes
        L.thrift_attn_decode_static.argtypes = [p, i, p, p, p, p, p, p, p, p, i, i, i, i, i, i, d, i, i, f, p, i, p, p, i, p]
        L.thrift_kv_cache_append.argtypes = [p, p, i, i, p, p, p, p, p, p, p, p, p, i, i, i, i, i, p]
        L.thrift_attention_forward_workspace.restype = sz
        L.thrift_attention_forward_workspace.argtypes = [i, i, i, i, i, i, i, i, d, i]
        L.thrift_attention_forward.argtypes = [p, p, p, i, i, i, i, i, i, i, i, i, d, i, i, f, p, i, p, p, sz, p]
        L.thrift_kv_cache_append_advance.argtypes = [p, p, i, i, p, p, p, p, p, p, p, p, p, p, i, i, i, i, i, p]
        i64, i = C.c_int64, _Int
        L.thrift_rope_frequencies.argtypes = [i, d, i, d, d, d, d, C.POINTER(d), C.POINTER(f)]
        L.thrift_rope.argtypes = [p, p, p, p, i, p, p, p, p, i, i, p, i64, p, i, i, f, i, i, i, p]
        L.thrift_rope_backward.argtypes = L.thrift_rope.argtypes
        L.thrift_page_map.argtypes = [p, p, i, i, i, p, i, p, i, p, i, p, p, p, p, p, p]
        L.thrift_page_release.argtypes = [p, p, i, i, i, p, i, p, i, p, p, p, p]
        L.thrift_paged_append.argtypes = [p, p, p, i, p, p, p, p, i, i, i, p, p, p, i, i, f, p, p, i, i, i, p]
        L.thrift_paged_decode_workspace.restype = sz
        L.thrift_paged_decode_workspace.argtypes = [i] * 6
        L.thrift_paged_decode.argtypes = [p, i, p, p, i, p, i, p, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_paged_read.argtypes = [p, p, i, p, i, p, p, i, i, i, i, i, p, p, p]
        L.thrift_paged_append8.argtypes = [p, p, p, i, p, p, p, p, i, i, i, p, p, p, i, i, f, p, p, p, p, i, i, i, p]
        L.thrift_paged_decode8_workspace.restype = L.thrift_paged_decode_prefix_workspace.restype = sz
        L.thrift_paged_decode8_workspace.argtypes = [i] * 6
        L.thrift_paged_decode8.argtypes = [p, i, p, p, p, p, i, p, i, p, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_paged_read8.argtypes = [p, p, p, p, i, p, i, p, p, i, i, i, i, i, p, p, i, p]
        L.thrift_paged_decode_prefix_workspace.argtypes = [i] * 8
        L.thrift_paged_decode_prefix.argtypes = [p, i, p, p, i, p, i, p, p, p, i, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_paged_decode_prefix8.argtypes = [p, i, p, p, p, p, i, p, i, p, p, p, i, i, i, i, i, i, f, p, i, p, p, sz, p]
        L.thrift_peak_probe.argtypes = [C.c_int, C.c_int, C.c_int, p, sz, C.POINTER(C.c_double), p]
        _lib = L
    return _lib


_call = None


class _General:
    """Stands in for the module _call where it cannot be loaded: leaves every call to the general path."""

    @staticmethod
    def decode(*_):
        return None

    append = attention = rope = page_map = paged_append = paged_decode = paged_append8 = paged_decode8 = paged_decode_prefix = paged_decode_prefix8 = paged_read = paged_read8 = decode


def _native():
    """The module that makes the calls of a serving loop without ctypes (csrc/thrift_call.cpp).  It is compiled against the
    headers of one torch; under another one, or without it, the calls take their general path, 20 us of host time each."""
    global _call
    if _call is None:
        lib()
        try:
            from . import _call as module
        except ImportError as e:
            warnings.warn(f"the module _call cannot be loaded ({e}); build it with `python -m paper_2605_23081_amd.build`", RuntimeWarning)
            module = _General
        _call = module
    return _call


def _raw_stream() -> int:
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except RuntimeError:                                    # no device: no device tensors either, the general path says so
        return 0


def _here_now() -> Tuple[int, int]:
    """The current device and its current stream."""
    try:
        device = torch._C._cuda_getDevice()
        return device, torch._C._cuda_getCurrentRawStream(device)
    except RuntimeError:
        return -1, 0


def _result(r, where: str):
    """What a function of _native() returned: the result, or the status of the C call."""
    if r.__class__ is int:
        raise ThriftError(r, where)
    return r


def status_string(code: int) -> str:
    return lib().thrift_status_string(int(code)).decode()


def _check(code: int, where: str) -> None:
    if code != 0:
        raise ThriftError(code, where)


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream() -> C.c_void_p:
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dev(t: torch.Tensor, dtype=None) -> torch.Tensor:
    assert t.is_cuda and t.is_contiguous(), "device-resident contiguous tensors only"
    if dtype is not None:
        assert t.dtype == dtype, (t.dtype, dtype)
    return t


def _prefill_shapes(q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt, Bq: int) -> None:
    """The C side sees pointers only: check here that every tensor has the dtype and the exact shape the kernel indexes."""
    B, Hq, Nq, D = q.shape
    _, Hkv, Nkv, _ = k.shape
    assert q.dtype == k.dtype == v.dtype and q.dtype in (torch.float16, torch.bfloat16), (q.dtype, k.dtype, v.dtype)
    assert k.shape == v.shape == (B, Hkv, Nkv, D), (k.shape, v.shape)
    Tq, Tv = -(-Nq // Bq), -(-Nkv // 64)
    u8, i32 = torch.uint8, torch.int32
    for name, t, shape, dt in (("q4", q4, (B, Hq, Nq, D // 2), u8), ("qs", qs, (B, Hq, Nq, D // 32), u8),
                               ("k4", k4, (B, Hkv, Nkv, D // 2), u8), ("ks", ks, (B, Hkv, Nkv, D // 32), u8),
                               ("v4", v4, (B, Hkv, Tv, D, 32), u8), ("vs", vs, (B, Hkv, 2 * Tv, D), u8),
                               ("cnt", cnt, (B, Hq, Tq), i32)):
        assert tuple(t.shape) == shape and t.dtype == dt, (name, tuple(t.shape), shape, t.dtype)
    assert idx.dtype == i32 and idx.dim() == 4 and tuple(idx.shape[:3]) == (B, Hq, Tq) and idx.shape[3] >= 1, tuple(idx.shape)


def _cache_shapes(k16, v16, k4, ks, v4, vs, kmean, Bk: int) -> None:
    B, Hkv, Nkv, D = k16.shape
    assert k16.dtype == v16.dtype and k16.dtype in (torch.float16, torch.bfloat16) and v16.shape == k16.shape
    u8 = torch.uint8
    for name, t, shape, dt in (("k4", k4, (B, Hkv, Nkv, D // 2), u8), ("ks", ks, (B, Hkv, Nkv, D // 32), u8),
                               ("v4", v4, (B, Hkv, Nkv // 64, D, 32), u8), ("vs", vs, (B, Hkv, Nkv // 32, D), u8),
                               ("kmean", kmean, (B, Hkv, Nkv // Bk, D), torch.float32)):
        assert tuple(t.shape) == shape and t.dtype == dt, (name, tuple(t.shape), shape, t.dtype)


# ---- host helpers ----

def row_budget(visible: int, budget: float, fixed_k: int = -1) -> int:
    return int(lib().thrift_row_budget(int(visible), float(budget), int(fixed_k)))


def visible_blocks(i: int, Tk: int, Bq: int, Bk: int, causal: bool, q_block_offset: int = 0) -> int:
    return int(lib().thrift_visible_blocks(i, Tk, Bq, Bk, int(causal), q_block_offset))


def budget_to_global_k(n_blocks: int, fraction: float) -> int:
    return int(lib().thrift_budget_to_global_k(int(n_blocks), float(fraction)))


def select_kmax(Tq: int, Tk: int, Bq: int, Bk: int, causal: bool, budget: float, fixed_k: int = -1,
                q_block_offset: int = 0) -> int:
    return int(lib().thrift_select_kmax(Tq, Tk, Bq, Bk, int(causal), float(budget), int(fixed_k), q_block_offset))


# ---- the five compute calls ----

def thrift_block_means(x: torch.Tensor, block: int, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    _dev(x)
    B, H, N, D = x.shape
    if out is None:
        out = torch.empty(B, H, -(-N // max(block, 1)), D, dtype=torch.float32, device=x.device)
    _check(lib().thrift_block_means(_ptr(x), _DT[x.dtype], B, H, N, D, block, _ptr(out), _stream()), "thrift_block_means")
    return out


def thrift_select_topk(qmean: torch.Tensor, kmean: torch.Tensor, Bq: int, Bk: int, causal: bool, budget: float,
                       fixed_k: int = -1, q_block_offset: int = 0, kmax: Optional[int] = None,
                       idx: Optional[torch.Tensor] = None, cnt: Optional[torch.Tensor] = None,
                       group_shared: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    _dev(qmean, torch.float32), _dev(kmean, torch.float32)
    B, Hq, Tq, D = qmean.shape
    _, Hkv, Tk, _ = kmean.shape
    if kmax is None:
        kmax = max(1, select_kmax(Tq, Tk, Bq, Bk, causal, budget, fixed_k, q_block_offset))
    if idx is None:
        idx = torch.empty(B, Hq, Tq, kmax, dtype=torch.int32, device=qmean.device)
        cnt = torch.empty(B, Hq, Tq, dtype=torch.int32, device=qmean.device)
    fn = lib().thrift_select_topk_shared if group_shared else lib().thrift_select_topk
    _check(fn(_ptr(qmean), _ptr(kmean), B, Hq, Hkv, Tq, Tk, D, Bq, Bk, int(causal), float(budget),
              int(fixed_k), int(q_block_offset), _ptr(idx), _ptr(cnt), int(kmax), _stream()),
           "thrift_select_topk_shared" if group_shared else "thrift_select_topk")
    return idx, cnt


SELECT_RANDOM, SELECT_DIAGONAL = 1, 2


def thrift_select_ablation(selector: int, seed: int, B: int, Hq: int, Tq: int, Tk: int, Bq: int, Bk: int, causal: bool,
                           budget: float, fixed_k: int = -1, q_block_offset: int = 0, kmax: Optional[int] = None,
                           device=None, idx: Optional[torch.Tensor] = None, cnt: Optional[torch.Tensor] = None
                           ) -> Tuple[torch.Tensor, torch.Tensor]:
    device = torch.device("cuda", torch.cuda.current_device()) if device is None else device
    if kmax is None:
        kmax = max(1, select_kmax(Tq, Tk, Bq, Bk, causal, budget, fixed_k, q_block_offset))
    if idx is None:
        idx = torch.empty(B, Hq, Tq, kmax, dtype=torch.int32, device=device)
        cnt = torch.empty(B, Hq, Tq, dtype=torch.int32, device=device)
    _check(lib().thrift_select_ablation(int(selector), int(seed) & (2 ** 64 - 1), B, Hq, Tq, Tk, Bq, Bk, int(causal), float(budget),
                                        int(fixed_k), int(q_block_offset), _ptr(idx), _ptr(cnt), int(kmax), _stream()),
           "thrift_select_ablation")
    return idx, cnt


def thrift_quantize_mxfp4(x: torch.Tensor, axis: int, codes: Optional[torch.Tensor] = None,
                          scales: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    _dev(x)
    B, H, N, D = x.shape
    if codes is None:
        if axis == 0:
            codes = torch.empty(B, H, N, D // 2, dtype=torch.uint8, device=x.device)
            scales = torch.empty(B, H, N, D // 32, dtype=torch.uint8, device=x.device)
        else:
            codes = torch.empty(B, H, -(-N // 64), D, 32, dtype=torch.uint8, device=x.device)
            scales = torch.empty(B, H, 2 * -(-N // 64), D, dtype=torch.uint8, device=x.device)
    _check(lib().thrift_quantize_mxfp4(_ptr(x), _DT[x.dtype], B, H, N, D, int(axis), _ptr(codes), _ptr(scales), _stream()),
           "thrift_quantize_mxfp4")
    return codes, scales


def thrift_prefill_prepass(q, k, v, Bq: int, Bk: int, qmean, kmean, q4, qs, k4, ks, v4, vs) -> None:
    """Block means of q and k and the MXFP4 codes of q, k (axis 0) and v (axis 1) in one launch, into the given tensors."""
    for t in (q, k, v, qmean, kmean, q4, qs, k4, ks, v4, vs):
        _dev(t)
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    Tq, Tk, Tv = -(-N // max(Bq, 1)), -(-N // max(Bk, 1)), -(-N // 64)
    u8, f32 = torch.uint8, torch.float32
    assert q.dtype == k.dtype == v.dtype and k.shape == v.shape == (B, Hkv, N, D), (q.dtype, k.dtype, v.dtype, k.shape, v.shape)
    for name, t, shape, dt in (("qmean", qmean, (B, Hq, Tq, D), f32), ("kmean", kmean, (B, Hkv, Tk, D), f32),
                               ("q4", q4, (B, Hq, N, D // 2), u8), ("qs", qs, (B, Hq, N, D // 32), u8),
                               ("k4", k4, (B, Hkv, N, D // 2), u8), ("ks", ks, (B, Hkv, N, D // 32), u8),
                               ("v4", v4, (B, Hkv, Tv, D, 32), u8), ("vs", vs, (B, Hkv, 2 * Tv, D), u8)):
        assert tuple(t.shape) == shape and t.dtype == dt, (name, tuple(t.shape), shape, t.dtype)
    _check(lib().thrift_prefill_prepass(_ptr(q), _ptr(k), _ptr(v), _DT[q.dtype], B, Hq, Hkv, N, D, Bq, Bk, _ptr(qmean), _ptr(kmean),
                                        _ptr(q4), _ptr(qs), _ptr(k4), _ptr(ks), _ptr(v4), _ptr(vs), _stream()), "thrift_prefill_prepass")


def thrift_attn_prefill(q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt, Bq: int, Bk: int, causal: bool,
                        softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                        out_dtype: Optional[torch.dtype] = None, lse: Optional[torch.Tensor] = None) -> torch.Tensor:
    for t in (q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt):
        _dev(t)
    _prefill_shapes(q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt, Bq)
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    if out is None:
        out = torch.empty(B, Hq, N, D, dtype=out_dtype or q.dtype, device=q.device)
    assert tuple(out.shape) == (B, Hq, N, D) and (lse is None or (tuple(lse.shape) == (B, Hq, N) and lse.dtype == torch.float32))
    kmax = idx.shape[-1]
    ws_bytes = lib().thrift_attn_prefill_workspace(B, Hq, Hkv, N, D, Bq, Bk, kmax)
    ws = torch.empty(ws_bytes, dtype=torch.uint8, device=q.device) if ws_bytes else None
    _check(lib().thrift_attn_prefill(_ptr(q), _ptr(k), _ptr(v), _DT[q.dtype], _ptr(q4), _ptr(qs), _ptr(k4), _ptr(ks),
                                     _ptr(v4), _ptr(vs), _ptr(idx), _ptr(cnt), kmax, B, Hq, Hkv, N, D, Bq, Bk,
                                     int(causal), float(softmax_scale), _ptr(out), _DT[out.dtype], _ptr(lse), _ptr(ws),
                                     ws_bytes, _stream()), "thrift_attn_prefill")
    return out


def thrift_attn_prefill_chunk(q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt, Bq: int, Bk: int, causal: bool, q_block_offset: int,
                              softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                              out_dtype: Optional[torch.dtype] = None, lse: Optional[torch.Tensor] = None,
                              tile_order: int = 0) -> torch.Tensor:
    """q, q4, qs: the chunk's Nq tokens; k, v and their codes: the whole key range.  tile_order 1: Sec. 3.3's order;
    2 / 3: ascending order with the staging schedule fixed (see include/thrift.h)."""
    for t in (q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt):
        _dev(t)
    _prefill_shapes(q, k, v, q4, qs, k4, ks, v4, vs, idx, cnt, Bq)
    B, Hq, Nq, D = q.shape
    Hkv, Nkv = k.shape[1], k.shape[2]
    if out is None:
        out = torch.empty(B, Hq, Nq, D, dtype=out_dtype or q.dtype, device=q.device)
    assert tuple(out.shape) == (B, Hq, Nq, D) and (lse is None or (tuple(lse.shape) == (B, Hq, Nq) and lse.dtype == torch.float32))
    kmax = idx.shape[-1]
    _check(lib().thrift_attn_prefill_ordered(_ptr(q), _ptr(k), _ptr(v), _DT[q.dtype], _ptr(q4), _ptr(qs), _ptr(k4), _ptr(ks),
                                             _ptr(v4), _ptr(vs), _ptr(idx), _ptr(cnt), kmax, B, Hq, Hkv, Nq, int(q_block_offset),
                                             Nkv, D, Bq, Bk, int(causal), int(tile_order), float(softmax_scale), _ptr(out),
                                             _DT[out.dtype], _ptr(lse), None, 0, _stream()), "thrift_attn_prefill_ordered")
    return out


def decode_workspace_bytes(B: int, Hq: int, Hkv: int, Nkv: int, D: int, Bk: int, split_blocks: int) -> int:
    return int(lib().thrift_attn_decode_workspace(B, Hq, Hkv, Nkv, D, Bk, split_blocks))


def decode_least_workspace_bytes(B: int, Hq: int, Hkv: int, Nkv: int, D: int, Bk: int, split_blocks: int) -> int:
    return int(lib().thrift_attn_decode_least_workspace(B, Hq, Hkv, Nkv, D, Bk, split_blocks))


def thrift_attn_decode(q, k16, v16, k4, ks, v4, vs, kmean, Bk: int, budget: float, fixed_k: int = -1,
                       split_blocks: int = 256, softmax_scale: float = 0.0, seqlens: Optional[torch.Tensor] = None,
                       out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                       workspace: Optional[torch.Tensor] = None, return_selection: bool = False,
                       group_shared: bool = False):
    if not return_selection and (out is not None or out_dtype is None):
        r = (_call or _native()).decode(q, k16, v16, k4, ks, v4, vs, kmean, Bk, budget, fixed_k, split_blocks, softmax_scale,
                                        seqlens, out, workspace, bool(group_shared), _raw_stream())
        if r is not None:
            return _result(r, "thrift_attn_decode_shared" if group_shared else "thrift_attn_decode")
    for t in (q, k16, v16, k4, ks, v4, vs, kmean):
        _dev(t)
    _cache_shapes(k16, v16, k4, ks, v4, vs, kmean, Bk)
    B, Hq, D = q.shape
    _, Hkv, Nkv, _ = k16.shape
    assert q.dtype == k16.dtype and k16.shape[0] == B and k16.shape[3] == D
    if seqlens is not None:
        _dev(seqlens, torch.int32)
        assert tuple(seqlens.shape) == (B,)
    if out is None:
        out = torch.empty(B, Hq, D, dtype=out_dtype or q.dtype, device=q.device)
    assert tuple(out.shape) == (B, Hq, D)
    if workspace is None:
        size = B, Hq, Hkv, Nkv, D, Bk, split_blocks
        n, least = decode_workspace_bytes(*size), decode_least_workspace_bytes(*size)
        try:
            workspace = torch.empty(max(n, 16), dtype=torch.uint8, device=q.device)
        except torch.OutOfMemoryError:                      # the two-pass form's scores do not fit: the one-pass form
            if least == n:
                raise
            workspace = torch.empty(max(least, 16), dtype=torch.uint8, device=q.device)
    idx = cnt = None
    kmax = 0
    if return_selection:
        kmax = max(1, row_budget(Nkv // Bk, budget, fixed_k))
        idx = torch.empty(B, Hq, kmax, dtype=torch.int32, device=q.device)
        cnt = torch.empty(B, Hq, dtype=torch.int32, device=q.device)
    fn = lib().thrift_attn_decode_shared if group_shared else lib().thrift_attn_decode
    _check(fn(_ptr(q), _DT[q.dtype], _ptr(k16), _ptr(v16), _ptr(k4), _ptr(ks), _ptr(v4), _ptr(vs),
              _ptr(kmean), _ptr(seqlens), B, Hq, Hkv, Nkv, D, Bk, float(budget), int(fixed_k),
              int(split_blocks), float(softmax_scale), _ptr(out), _DT[out.dtype], _ptr(idx), _ptr(cnt),
              kmax, _ptr(workspace), workspace.numel(), _stream()),
           "thrift_attn_decode_shared" if group_shared else "thrift_attn_decode")
    return (out, idx, cnt) if return_selection else out


DECODE_STATIC_SCRATCH_BYTES = 32 << 20


def thrift_attn_decode_static(q, k16, v16, k4, ks, v4, vs, kmean, Bk: int, budget: float, out: torch.Tensor,
                              fixed_k: int = -1, split_blocks: int = 256, softmax_scale: float = 0.0,
                              seqlens: Optional[torch.Tensor] = None, idx: Optional[torch.Tensor] = None,
                              cnt: Optional[torch.Tensor] = None) -> torch.Tensor:
    """thrift_attn_decode on the library's static scratch: the caller passes every buffer (out, and idx / cnt if it
    wants the selection back); neither this wrapper nor the C call allocates."""
    for t in (q, k16, v16, k4, ks, v4, vs, kmean, out):
        _dev(t)
    _cache_shapes(k16, v16, k4, ks, v4, vs, kmean, Bk)
    B, Hq, D = q.shape
    _, Hkv, Nkv, _ = k16.shape
    assert q.dtype == k16.dtype and k16.shape[0] == B and k16.shape[3] == D and tuple(out.shape) == (B, Hq, D)
    if seqlens is not None:
        _dev(seqlens, torch.int32)
        assert tuple(seqlens.shape) == (B,)
    if idx is not None:
        assert idx.dtype == torch.int32 and tuple(idx.shape[:2]) == (B, Hq) and cnt is not None and tuple(cnt.shape) == (B, Hq)
    kmax = 0 if idx is None else idx.shape[-1]
    _check(lib().thrift_attn_decode_static(_ptr(q), _DT[q.dtype], _ptr(k16), _ptr(v16), _ptr(k4), _ptr(ks), _ptr(v4), _ptr(vs),
                                           _ptr(kmean), _ptr(seqlens), B, Hq, Hkv, Nkv, D, Bk, float(budget), int(fixed_k),
                                           int(split_blocks), float(softmax_scale), _ptr(out), _DT[out.dtype], _ptr(idx), _ptr(cnt),
                                           kmax, _stream()), "thrift_attn_decode_static")
    return out


class KVCache:
    """Device buffers of the dual cache (Sec. 4.1, Sec. 5): 16-bit K/V, MXFP4 K/V and the key-block means."""

    def __init__(self, B, Hkv, Nkv, D, Bk, dtype, device, fill: Optional[int] = None):
        assert Nkv % Bk == 0
        u8 = torch.uint8

        def mk(*shape, dtype):
            # fill: a byte pattern for every buffer (tests poison the cache to show that nothing unwritten is read)
            if fill is None:
                return torch.empty(shape, dtype=dtype, device=device)
            nbytes = math.prod(shape) * torch.empty((), dtype=dtype).element_size()
            return torch.full((nbytes,), fill, dtype=u8, device=device).view(dtype).view(shape)

        self.B, self.Hkv, self.Nkv, self.D, self.Bk = B, Hkv, Nkv, D, Bk
        self.k16 = mk(B, Hkv, Nkv, D, dtype=dtype)
        self.v16 = mk(B, Hkv, Nkv, D, dtype=dtype)
        self.k4 = mk(B, Hkv, Nkv, D // 2, dtype=u8)
        self.ks = mk(B, Hkv, Nkv, D // 32, dtype=u8)
        self.v4 = mk(B, Hkv, Nkv // 64, D, 32, dtype=u8)
        self.vs = mk(B, Hkv, Nkv // 32, D, dtype=u8)
        self.kmean = mk(B, Hkv, Nkv // Bk, D, dtype=torch.float32)
        self.seqlens = torch.zeros(B, dtype=torch.int32, device=device)

    def append(self, k_new, v_new, new_lens: Optional[torch.Tensor] = None):
        """Append k_new, v_new [B,Hkv,n,D] (all n tokens, or new_lens[b] of them) and advance seqlens (a new tensor)."""
        r = (_call or _native()).append(k_new, v_new, self.seqlens, new_lens, self.k16, self.v16, self.k4, self.ks, self.v4, self.vs,
                                        self.kmean, self.Bk, _raw_stream())
        if r is not None:
            self.seqlens = _result(r, "thrift_kv_cache_append")
            return
        after = torch.empty_like(self.seqlens)
        thrift_kv_cache_append(k_new, v_new, self.seqlens, self.k16, self.v16, self.k4, self.ks, self.v4, self.vs,
                               self.kmean, self.Bk, new_lens, after)
        self.seqlens = after


def thrift_kv_cache_append(k_new, v_new, seqlens, k16, v16, k4, ks, v4, vs, kmean, Bk: int,
                           new_lens: Optional[torch.Tensor] = None, seqlens_out: Optional[torch.Tensor] = None) -> None:
    for t in (k_new, v_new, k16, v16, k4, ks, v4, vs, kmean):
        _dev(t)
    _dev(seqlens, torch.int32)
    if new_lens is not None:
        _dev(new_lens, torch.int32)
    assert k_new.shape == v_new.shape and k_new.dtype == v_new.dtype == k16.dtype == v16.dtype
    _cache_shapes(k16, v16, k4, ks, v4, vs, kmean, Bk)
    B, Hkv, n_new, D = k_new.shape
    _, _, Nkv, _ = k16.shape
    assert tuple(k16.shape[:2]) == (B, Hkv) and k16.shape[3] == D and tuple(seqlens.shape) == (B,)
    assert new_lens is None or tuple(new_lens.shape) == (B,)
    assert seqlens_out is None or (tuple(_dev(seqlens_out, torch.int32).shape) == (B,))
    _check(lib().thrift_kv_cache_append_advance(_ptr(k_new), _ptr(v_new), _DT[k_new.dtype], n_new, _ptr(seqlens), _ptr(new_lens),
                                        _ptr(seqlens_out), _ptr(k16), _ptr(v16), _ptr(k4), _ptr(ks), _ptr(v4), _ptr(vs), _ptr(kmean),
                                        B, Hkv, Nkv, D, Bk, _stream()), "thrift_kv_cache_append")


PEAK_MFMA_MXFP4, PEAK_MFMA_16, PEAK_HBM_READ, PEAK_VALU_SOFTMAX, PEAK_TILE_MIX = range(5)


def thrift_peak_probe(kind: int, buffer: torch.Tensor, iters: int = 2000, dtype: torch.dtype = torch.bfloat16) -> float:
    """Enqueue one measurement microbenchmark (see include/thrift.h) on the current stream; returns the work of the
    launch (flops, bytes or wave-tiles).  The caller times it."""
    _dev(buffer, torch.uint8)
    work = C.c_double(0.0)
    _check(lib().thrift_peak_probe(int(kind), _DT[dtype], int(iters), _ptr(buffer), buffer.numel(), C.byref(work), _stream()),
           "thrift_peak_probe")
    return float(work.value)


# ---- around the attention: rotary positions and the paged cache ----

ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "by_parts": 3}


def rope_frequencies(rot: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, original: float = 0.0,
                     slow: float = 1.0, fast: float = 32.0, device=None) -> Tuple[torch.Tensor, float]:
    """Radians per position of the rot/2 pairs (fp64, on `device`) and the gain, for the scalings of include/thrift.h."""
    freqs, gain = (C.c_double * max(min(rot // 2, 512), 1))(), C.c_float()               # more are refused
    _check(lib().thrift_rope_frequencies(int(rot), float(base), ROPE_SCALINGS[scaling], float(factor), float(original), float(slow),
                                         float(fast), freqs, C.byref(gain)), "thrift_rope_frequencies")
    return torch.tensor(list(freqs), dtype=torch.float64, device=device), float(gain.value)


def _here(*tensors: Optional[torch.Tensor]) -> None:
    """Device tensors, all on the current device: the calls run on its current stream."""
    current = torch.cuda.current_device() if torch.cuda.is_available() else -1
    for t in tensors:
        if t is not None:
            assert t.is_cuda and t.device.index == current, f"a tensor on {t.device}; the current device is {current}"


def _apart(t: torch.Tensor) -> bool:
    """No two elements of t share an address (sufficient: every stride passes what the smaller ones reach)."""
    reach = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz > 1):
        if stride < reach:
            return False
        reach = stride * (size - 1) + reach
    return True


def _strides(t: torch.Tensor, dims) -> C.Array:
    return (C.c_int64 * len(dims))(*[t.stride(d) for d in dims])


def _heads(t: torch.Tensor, shape, dtype) -> None:
    assert tuple(t.shape) == tuple(shape) and t.dtype == dtype, (tuple(t.shape), tuple(shape), t.dtype, dtype)
    assert t.stride(-1) == 1 or t.shape[-1] == 1, "the channels of a head are contiguous"


def _rope(name: str, q, k, freqs, positions, layout: str, gain: float, q_out, k_out):
    assert q.dtype in (torch.float16, torch.bfloat16), q.dtype
    B, Hq, N, D = q.shape
    _heads(q, q.shape, q.dtype)
    if k is None:
        assert k_out is None
    else:
        _heads(k, (B, k.shape[1], N, D), q.dtype)
        if k_out is None:
            k_out = torch.empty(k.shape, dtype=k.dtype, device=k.device)
        _heads(k_out, k.shape, k.dtype)
    if q_out is None:
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    _heads(q_out, q.shape, q.dtype)
    assert _apart(q_out) and (k_out is None or _apart(k_out)), "elements of an output coincide"
    assert freqs.dtype == torch.float64 and freqs.dim() == 1 and freqs.is_contiguous(), (freqs.dtype, tuple(freqs.shape))
    step = 0
    if positions is not None:
        assert positions.dtype == torch.int32 and tuple(positions.shape) in ((N,), (B, N)) and (N == 1 or positions.stride(-1) == 1), tuple(positions.shape)
        step = positions.stride(0) if positions.dim() == 2 else 0
    _here(q, k, q_out, k_out, freqs, positions)
    s = lambda t: None if t is None else _strides(t, (0, 1, 2))
    _check(getattr(lib(), name)(_ptr(q), s(q), _ptr(q_out), s(q_out), Hq, _ptr(k), s(k), _ptr(k_out), s(k_out), 0 if k is None else k.shape[1],
                                _DT[q.dtype], _ptr(positions), step, _ptr(freqs), 2 * freqs.numel(), ROPE_LAYOUTS[layout], float(gain), B, N, D,
                                _stream()), name)
    return q_out, k_out


def thrift_rope(q, k, freqs, positions: Optional[torch.Tensor] = None, layout: str = "half", gain: float = 1.0,
                q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """q [B,Hq,N,D] and k [B,Hkv,N,D] (or None) with their first 2 * len(freqs) channels turned to positions ([B,N] or [N], default
    0 .. N-1): (q_out, k_out), contiguous unless given.  Inputs and outputs may be views (a fused projection's [B,N,H,D]).  Nothing is
    recorded for autograd: the gradient is thrift_rope_backward."""
    r = (_call or _native()).rope(0, q, k, freqs, positions, ROPE_LAYOUTS[layout], gain, q_out, k_out, *_here_now())
    if r is not None:
        return _result(r, "thrift_rope")
    return _rope("thrift_rope", q, k, freqs, positions, layout, gain, q_out, k_out)


def thrift_rope_backward(q, k, freqs, positions: Optional[torch.Tensor] = None, layout: str = "half", gain: float = 1.0,
                         q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """Gradients of thrift_rope's inputs from those of its outputs, q and k (or None); arguments as thrift_rope."""
    r = (_call or _native()).rope(1, q, k, freqs, positions, ROPE_LAYOUTS[layout], gain, q_out, k_out, *_here_now())
    if r is not None:
        return _result(r, "thrift_rope_backward")
    return _rope("thrift_rope_backward", q, k, freqs, positions, layout, gain, q_out, k_out)


class PageMap(NamedTuple):
    """Places of a step's new tokens (include/thrift.h, thrift_page_map).  The five share one allocation, which lives as long as any of them
    (8 bytes a row: a PageTable holds it until its next step)."""
    slots: torch.Tensor        # [rows] int32
    positions: torch.Tensor    # [rows] int32
    starts: torch.Tensor       # [B+1] int32
    seqlens: torch.Tensor      # [B] int32, after the call
    free_count: torch.Tensor   # [1] int32, after the call


def _ints(shape, *tensors: torch.Tensor) -> None:
    for t in tensors:
        assert t.dtype == torch.int32 and t.is_contiguous() and tuple(t.shape) == tuple(shape), (t.dtype, tuple(t.shape), tuple(shape))


def _pool(seqlens, block_table, free_pages, free_count) -> Tuple[int, int]:
    assert block_table.dim() == 2 and free_pages.dim() == 1, (tuple(block_table.shape), tuple(free_pages.shape))
    B, max_pages = block_table.shape
    _ints((B, max_pages), block_table), _ints((B,), seqlens), _ints(free_pages.shape, free_pages), _ints((1,), free_count)
    return B, max_pages


def thrift_page_map(seqlens, new_lens, block_table, free_pages, free_count, page_size: int, n_pages: int, rows: int) -> PageMap:
    """Pages, block-table entries (written into block_table), slots and positions of new_lens [B] new tokens per sequence."""
    r = (_call or _native()).page_map(seqlens, new_lens, block_table, free_pages, free_count, page_size, n_pages, rows, *_here_now())
    if r is not None:
        return PageMap._make(_result(r, "thrift_page_map"))
    B, max_pages = _pool(seqlens, block_table, free_pages, free_count)
    _ints((B,), new_lens)
    _here(seqlens, new_lens, block_table, free_pages, free_count)
    sizes = (rows, rows, B + 1, B, 1)
    ends = [sum(-(-n // 4) * 4 for n in sizes[:i + 1]) for i in range(5)]
    space = torch.empty(ends[-1], dtype=torch.int32, device=seqlens.device)
    m = PageMap(*(space[e - -(-n // 4) * 4:][:n] for e, n in zip(ends, sizes)))
    _check(lib().thrift_page_map(_ptr(seqlens), _ptr(new_lens), B, int(page_size), int(n_pages), _ptr(block_table), max_pages,
                                 _ptr(free_pages), free_pages.numel(), _ptr(free_count), int(rows), *(_ptr(t) for t in m), _stream()),
           "thrift_page_map")
    return m


def thrift_page_release(seqlens, drop, block_table, free_pages, free_count, page_size: int, n_pages: int) -> Tuple[torch.Tensor, torch.Tensor]:
    """Puts the pages of the sequences with drop [B] != 0 back on the stack: (seqlens, free_count) after the call."""
    B, max_pages = _pool(seqlens, block_table, free_pages, free_count)
    _ints((B,), drop)
    _here(seqlens, drop, block_table, free_pages, free_count)
    after, count = torch.empty_like(seqlens), torch.empty_like(free_count)
    _check(lib().thrift_page_release(_ptr(seqlens), _ptr(drop), B, int(page_size), int(n_pages), _ptr(block_table), max_pages,
                                     _ptr(free_pages), free_pages.numel(), _ptr(free_count), _ptr(after), _ptr(count), _stream()),
           "thrift_page_release")
    return after, count


def _pages(k_pages, v_pages) -> None:
    assert k_pages.dim() == 4 and k_pages.dtype in (torch.float16, torch.bfloat16), (tuple(k_pages.shape), k_pages.dtype)
    assert k_pages.shape == v_pages.shape and k_pages.dtype == v_pages.dtype and k_pages.is_contiguous() and v_pages.is_contiguous()


def _pages8(k_codes, k_scales, v_codes, v_scales) -> None:
    assert k_codes.dim() == 4 and k_codes.shape == v_codes.shape and k_scales.shape == v_scales.shape == k_codes.shape[:3], \
        (tuple(k_codes.shape), tuple(k_scales.shape), tuple(v_codes.shape), tuple(v_scales.shape))
    assert all(t.dtype == torch.uint8 and t.is_contiguous() for t in (k_codes, k_scales, v_codes, v_scales))


def _paged_append(name: str, k, v, slots, pages, dtype, q, q_out, positions, freqs, layout: str, gain: float):
    """pages: the tensors of the cache, the first of them [n_pages,Hkv,page_size,D]."""
    T, Hkv, D = k.shape
    n_pages, _, page_size, _ = pages[0].shape
    _heads(k, (T, Hkv, D), dtype), _heads(v, (T, Hkv, D), dtype), _ints((T,), slots)
    assert pages[0].shape[1] == Hkv and pages[0].shape[3] == D, (tuple(pages[0].shape), tuple(k.shape))
    rot = 0
    if freqs is not None:
        assert freqs.dtype == torch.float64 and freqs.dim() == 1 and freqs.is_contiguous() and freqs.numel() > 0, (freqs.dtype, tuple(freqs.shape))
        assert positions is not None
        _ints((T,), positions)
        rot = 2 * freqs.numel()
    if q is None:
        assert q_out is None
    else:
        _heads(q, (T, q.shape[1], D), dtype)
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        assert q_out.shape == q.shape and q_out.dtype == q.dtype and q_out.is_contiguous(), (tuple(q_out.shape), q_out.dtype)
    _here(k, v, slots, *pages, q, q_out, positions, freqs)
    s = lambda t: None if t is None else _strides(t, (0, 1))
    _check(getattr(lib(), name)(_ptr(q), s(q), _ptr(q_out), 0 if q is None else q.shape[1], _ptr(k), s(k), _ptr(v), s(v), Hkv,
                                _DT[k.dtype], T, _ptr(slots), _ptr(positions), _ptr(freqs), rot, ROPE_LAYOUTS[layout], float(gain),
                                *(_ptr(t) for t in pages), n_pages, page_size, D, _stream()), name)
    return q_out


def thrift_paged_append(k, v, slots, k_pages, v_pages, q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
                        positions: Optional[torch.Tensor] = None, freqs: Optional[torch.Tensor] = None, layout: str = "half",
                        gain: float = 1.0) -> Optional[torch.Tensor]:
    """k, v [T,Hkv,D] into the pages [n_pages,Hkv,page_size,D] at slots [T]; with freqs, k and q [T,Hq,D] are rotated to
    positions [T].  Returns q_out (contiguous; rows of skipped tokens are left as they were)."""
    r = (_call or _native()).paged_append(k, v, slots, k_pages, v_pages, q, q_out, positions, freqs, ROPE_LAYOUTS[layout], gain, *_here_now())
    if r is not None:
        return None if r is True else _result(r, "thrift_paged_append")
    _pages(k_pages, v_pages)
    return _paged_append("thrift_paged_append", k, v, slots, (k_pages, v_pages), k_pages.dtype, q, q_out, positions, freqs, layout, gain)


def thrift_paged_append8(k, v, slots, k_codes, k_scales, v_codes, v_scales, q: Optional[torch.Tensor] = None,
                         q_out: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None,
                         freqs: Optional[torch.Tensor] = None, layout: str = "half", gain: float = 1.0) -> Optional[torch.Tensor]:
    """thrift_paged_append into the 8-bit cache: codes [n_pages,Hkv,page_size,D] and scales [n_pages,Hkv,page_size], bytes."""
    pages = (k_codes, k_scales, v_codes, v_scales)
    r = (_call or _native()).paged_append8(k, v, slots, *pages, q, q_out, positions, freqs, ROPE_LAYOUTS[layout], gain, *_here_now())
    if r is not None:
        return None if r is True else _result(r, "thrift_paged_append8")
    _pages8(*pages)
    assert k.dtype in (torch.float16, torch.bfloat16), k.dtype
    return _paged_append("thrift_paged_append8", k, v, slots, pages, k.dtype, q, q_out, positions, freqs, layout, gain)


def _paged_read(name: str, pages, block_table, seqlens, N: int, dtype, first, k_out, v_out, *last):
    assert block_table.dim() == 2, tuple(block_table.shape)
    B, max_pages = block_table.shape
    n_pages, Hkv, page_size, D = pages[0].shape
    _ints((B, max_pages), block_table), _ints((B,), seqlens)
    if first is not None:
        _ints((B,), first)
    out = [torch.empty(B, Hkv, max(N, 0), D, dtype=dtype, device=block_table.device) if x is None else x for x in (k_out, v_out)]
    for x in out:
        assert tuple(x.shape) == (B, Hkv, N, D) and x.dtype == dtype and x.is_contiguous(), (tuple(x.shape), x.dtype)
    _here(*pages, block_table, seqlens, first, *out)
    _check(getattr(lib(), name)(*(_ptr(t) for t in pages), n_pages, _ptr(block_table), max_pages, _ptr(first), _ptr(seqlens), B, Hkv, N, D,
                                page_size, *(_ptr(t) for t in out), *last, _stream()), name)
    return tuple(out)


def thrift_paged_read(k_pages, v_pages, block_table, seqlens, N: int, first: Optional[torch.Tensor] = None,
                      k_out: Optional[torch.Tensor] = None, v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Tokens first[b] .. first[b] + N - 1 (default: from 0) of every sequence as rows (k, v) [B,Hkv,N,D]; 0 past the lengths."""
    r = (_call or _native()).paged_read(k_pages, v_pages, block_table, seqlens, N, first, k_out, v_out, *_here_now())
    if r is not None:
        return _result(r, "thrift_paged_read")
    _pages(k_pages, v_pages)
    return _paged_read("thrift_paged_read", (k_pages, v_pages), block_table, seqlens, N, k_pages.dtype, first, k_out, v_out)


def thrift_paged_read8(k_codes, k_scales, v_codes, v_scales, block_table, seqlens, N: int, dtype: torch.dtype = torch.bfloat16,
                       first: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None,
                       v_out: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """thrift_paged_read of the 8-bit cache, in dtype."""
    r = (_call or _native()).paged_read8(k_codes, k_scales, v_codes, v_scales, block_table, seqlens, N, first, k_out, v_out, _DT.get(dtype, F32), *_here_now())
    if r is not None:
        return _result(r, "thrift_paged_read8")
    _pages8(k_codes, k_scales, v_codes, v_scales)
    assert dtype in (torch.float16, torch.bfloat16), dtype
    return _paged_read("thrift_paged_read8", (k_codes, k_scales, v_codes, v_scales), block_table, seqlens, N, dtype, first, k_out, v_out, _DT[dtype])


def paged_decode_workspace_bytes(B: int, Hq: int, Hkv: int, max_pages: int, page_size: int, D: int) -> int:
    return int(lib().thrift_paged_decode_workspace(B, Hq, Hkv, max_pages, page_size, D))


def paged_decode8_workspace_bytes(B: int, Hq: int, Hkv: int, max_pages: int, page_size: int, D: int) -> int:
    return int(lib().thrift_paged_decode8_workspace(B, Hq, Hkv, max_pages, page_size, D))


def paged_decode_prefix_workspace_bytes(bits: int, B: int, Hq: int, Hkv: int, n_groups: int, max_pages: int, page_size: int, D: int) -> int:
    return int(lib().thrift_paged_decode_prefix_workspace(bits, B, Hq, Hkv, n_groups, max_pages, page_size, D))


def _paged_decode(name: str, q, pages, block_table, seqlens, groups, need, softmax_scale: float, out, out_dtype, lse, return_lse: bool, workspace):
    """groups: () or (group_of, group_lens); need(B, Hq, Hkv, max_pages, page_size, D): bytes of workspace."""
    B, Hq, D = q.shape
    n_pages, Hkv, page_size, _ = pages[0].shape
    assert _dev(q).dtype in (torch.float16, torch.bfloat16) and pages[0].shape[3] == D, (q.dtype, tuple(q.shape), tuple(pages[0].shape))
    assert block_table.dim() == 2, tuple(block_table.shape)
    max_pages = block_table.shape[1]
    _ints((B, max_pages), block_table), _ints((B,), seqlens)
    if groups:
        _ints((B,), groups[0]), _ints((groups[1].numel(),), groups[1])
    if out is None:
        out = torch.empty(B, Hq, D, dtype=out_dtype or q.dtype, device=q.device)
    assert tuple(_dev(out).shape) == (B, Hq, D) and out.dtype in _DT, (tuple(out.shape), out.dtype)
    if lse is None and return_lse:
        lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device)
    assert lse is None or tuple(_dev(lse, torch.float32).shape) == (B, Hq)
    if workspace is None:
        workspace = torch.empty(need(B, Hq, Hkv, max_pages, page_size, D), dtype=torch.uint8, device=q.device)
    _dev(workspace, torch.uint8)
    _here(q, *pages, block_table, seqlens, *groups, out, lse, workspace)
    more = (_ptr(groups[0]), _ptr(groups[1]), groups[1].numel()) if groups else ()
    _check(getattr(lib(), name)(_ptr(q), _DT[q.dtype], *(_ptr(t) for t in pages), n_pages, _ptr(block_table), max_pages, _ptr(seqlens), *more,
                                B, Hq, Hkv, D, page_size, float(softmax_scale), _ptr(out), _DT[out.dtype], _ptr(lse),
                                _ptr(workspace), workspace.numel(), _stream()), name)
    return (out, lse) if return_lse else out


def thrift_paged_decode(q, k_pages, v_pages, block_table, seqlens, softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None,
                        out_dtype: Optional[torch.dtype] = None, lse: Optional[torch.Tensor] = None, return_lse: bool = False,
                        workspace: Optional[torch.Tensor] = None):
    """Attention of q [B,Hq,D] over the first seqlens [B] tokens of each sequence's pages: out, or (out, lse) with return_lse."""
    if out is not None or out_dtype is None:
        r = (_call or _native()).paged_decode(q, k_pages, v_pages, block_table, seqlens, softmax_scale, out, lse, int(bool(return_lse)), workspace,
                                              *_here_now())
        if r is not None:
            return _result(r, "thrift_paged_decode")
    _pages(k_pages, v_pages)
    assert q.dtype == k_pages.dtype, (q.dtype, k_pages.dtype)
    return _paged_decode("thrift_paged_decode", q, (k_pages, v_pages), block_table, seqlens, (), paged_decode_workspace_bytes, softmax_scale,
                         out, out_dtype, lse, return_lse, workspace)


def thrift_paged_decode8(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, softmax_scale: float = 0.0,
                         out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None, lse: Optional[torch.Tensor] = None,
                         return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """thrift_paged_decode over the 8-bit cache."""
    if out is not None or out_dtype is None:
        r = (_call or _native()).paged_decode8(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, softmax_scale, out, lse, int(bool(return_lse)), workspace,
                                                     *_here_now())
        if r is not None:
            return _result(r, "thrift_paged_decode8")
    _pages8(k_codes, k_scales, v_codes, v_scales)
    return _paged_decode("thrift_paged_decode8", q, (k_codes, k_scales, v_codes, v_scales), block_table, seqlens, (),
                         paged_decode8_workspace_bytes, softmax_scale, out, out_dtype, lse, return_lse, workspace)


def thrift_paged_decode_prefix(q, k_pages, v_pages, block_table, seqlens, group_of, group_lens, softmax_scale: float = 0.0,
                               out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                               lse: Optional[torch.Tensor] = None, return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """thrift_paged_decode where the sequences of group g (group_of [B] == g) have the same pages for their first group_lens [n_groups] [g]
    tokens, which are read once for all of them."""
    if out is not None or out_dtype is None:
        r = (_call or _native()).paged_decode_prefix(q, k_pages, v_pages, block_table, seqlens, group_of, group_lens, softmax_scale, out, lse, int(bool(return_lse)), workspace,
                                                           *_here_now())
        if r is not None:
            return _result(r, "thrift_paged_decode_prefix")
    _pages(k_pages, v_pages)
    assert q.dtype == k_pages.dtype, (q.dtype, k_pages.dtype)
    need = lambda B, Hq, Hkv, *sizes: paged_decode_prefix_workspace_bytes(16, B, Hq, Hkv, group_lens.numel(), *sizes)
    return _paged_decode("thrift_paged_decode_prefix", q, (k_pages, v_pages), block_table, seqlens, (group_of, group_lens), need, softmax_scale,
                         out, out_dtype, lse, return_lse, workspace)


def thrift_paged_decode_prefix8(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, group_of, group_lens,
                                softmax_scale: float = 0.0, out: Optional[torch.Tensor] = None, out_dtype: Optional[torch.dtype] = None,
                                lse: Optional[torch.Tensor] = None, return_lse: bool = False, workspace: Optional[torch.Tensor] = None):
    """thrift_paged_decode_prefix over the 8-bit cache."""
    if out is not None or out_dtype is None:
        r = (_call or _native()).paged_decode_prefix8(q, k_codes, k_scales, v_codes, v_scales, block_table, seqlens, group_of, group_lens, softmax_scale, out, lse, int(bool(return_lse)), workspace,
                                                            *_here_now())
        if r is not None:
            return _result(r, "thrift_paged_decode_prefix8")
    _pages8(k_codes, k_scales, v_codes, v_scales)
    need = lambda B, Hq, Hkv, *sizes: paged_decode_prefix_workspace_bytes(8, B, Hq, Hkv, group_lens.numel(), *sizes)
    return _paged_decode("thrift_paged_decode_prefix8", q, (k_codes, k_scales, v_codes, v_scales), block_table, seqlens, (group_of, group_lens),
                         need, softmax_scale, out, out_dtype, lse, return_lse, workspace)


class PageTable:
    """Block tables, lengths and the stack of free pages of up to B sequences; one serves the caches of all layers."""

    def __init__(self, B: int, max_pages: int, page_size: int, n_pages: int, device):
        i32 = torch.int32
        self.B, self.max_pages, self.page_size, self.n_pages = B, max_pages, page_size, n_pages
        self.block_table = torch.full((B, max_pages), -1, dtype=i32, device=device)
        self.seqlens = torch.zeros(B, dtype=i32, device=device)
        self.free_pages = torch.arange(n_pages - 1, -1, -1, dtype=i32, device=device)       # page 0 is taken first
        self.free_count = torch.full((1,), n_pages, dtype=i32, device=device)

    def map(self, new_lens, rows: int) -> PageMap:
        """Gives new_lens [B] new tokens their places; seqlens and free_count advance (new tensors)."""
        m = thrift_page_map(self.seqlens, new_lens, self.block_table, self.free_pages, self.free_count, self.page_size, self.n_pages, rows)
        self.seqlens, self.free_count = m.seqlens, m.free_count
        return m

    def release(self, drop) -> None:
        """Ends the sequences with drop [B] != 0: their pages are free again, their lengths 0."""
        self.seqlens, self.free_count = thrift_page_release(self.seqlens, drop, self.block_table, self.free_pages, self.free_count,
                                                            self.page_size, self.n_pages)


class PagedKVCache:
    """16-bit pages of one layer; the places of tokens come from a PageTable."""

    def __init__(self, table: PageTable, Hkv: int, D: int, dtype):
        shape = (table.n_pages, Hkv, table.page_size, D)
        self.table = table
        self.k_pages = torch.empty(shape, dtype=dtype, device=table.block_table.device)
        self.v_pages = torch.empty(shape, dtype=dtype, device=table.block_table.device)

    def append(self, k, v, m: PageMap, q: Optional[torch.Tensor] = None, freqs: Optional[torch.Tensor] = None, layout: str = "half",
               gain: float = 1.0, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """k, v [T,Hkv,D] of the step's rows into the pages, rotated with q [T,Hq,D] where freqs is given; returns the rotated q."""
        return thrift_paged_append(k, v, m.slots, self.k_pages, self.v_pages, q, q_out, m.positions, freqs, layout, gain)

    def decode(self, q, softmax_scale: float = 0.0, **kw):
        """Attention of q [B,Hq,D], the newest token of every sequence (thrift_paged_decode)."""
        return thrift_paged_decode(q, self.k_pages, self.v_pages, self.table.block_table, self.table.seqlens, softmax_scale, **kw)

    def read(self, N: int, first: Optional[torch.Tensor] = None, **kw) -> Tuple[torch.Tensor, torch.Tensor]:
        """N tokens of every sequence as dense rows (thrift_paged_read)."""
        return thrift_paged_read(self.k_pages, self.v_pages, self.table.block_table, self.table.seqlens, N, first, **kw)

    def decode_prefix(self, q, group_of, group_lens, softmax_scale: float = 0.0, **kw):
        """decode where the sequences of a group start with the same pages (thrift_paged_decode_prefix)."""
        return thrift_paged_decode_prefix(q, self.k_pages, self.v_pages, self.table.block_table, self.table.seqlens, group_of, group_lens,
                                          softmax_scale, **kw)


class PagedKVCache8:
    """8-bit pages of one layer, with the methods of PagedKVCache; dtype: of the keys and values that are read back."""

    def __init__(self, table: PageTable, Hkv: int, D: int, dtype):
        u8, dev = torch.uint8, table.block_table.device
        shape = (table.n_pages, Hkv, table.page_size)
        self.table, self.dtype = table, dtype
        self.k_codes, self.v_codes = (torch.empty(*shape, D, dtype=u8, device=dev) for _ in range(2))
        self.k_scales, self.v_scales = (torch.empty(shape, dtype=u8, device=dev) for _ in range(2))

    @property
    def pages(self) -> Tuple[torch.Tensor, ...]:
        return self.k_codes, self.k_scales, self.v_codes, self.v_scales

    def append(self, k, v, m: PageMap, q: Optional[torch.Tensor] = None, freqs: Optional[torch.Tensor] = None, layout: str = "half",
               gain: float = 1.0, q_out: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """k, v [T,Hkv,D] of the step's rows into the pages, rotated with q [T,Hq,D] where freqs is given; returns the rotated q."""
        return thrift_paged_append8(k, v, m.slots, *self.pages, q, q_out, m.positions, freqs, layout, gain)

    def decode(self, q, softmax_scale: float = 0.0, **kw):
        """Attention of q [B,Hq,D], the newest token of every sequence (thrift_paged_decode8)."""
        return thrift_paged_decode8(q, *self.pages, self.table.block_table, self.table.seqlens, softmax_scale, **kw)

    def read(self, N: int, first: Optional[torch.Tensor] = None, **kw) -> Tuple[torch.Tensor, torch.Tensor]:
        """N tokens of every sequence as dense rows of the cache's dtype (thrift_paged_read8)."""
        return thrift_paged_read8(*self.pages, self.table.block_table, self.table.seqlens, N, self.dtype, first, **kw)

    def decode_prefix(self, q, group_of, group_lens, softmax_scale: float = 0.0, **kw):
        """decode where the sequences of a group start with the same pages (thrift_paged_decode_prefix8)."""
        return thrift_paged_decode_prefix8(q, *self.pages, self.table.block_table, self.table.seqlens, group_of, group_lens, softmax_scale, **kw)


# ---- Alg. 1 end to end: the user-level form of the paper's signature ----

class PrefillPlan:
    """Buffers of one prefill problem, allocated once so that repeated steps do not allocate."""

    def __init__(self, B, Hq, Hkv, N, D, Bq, Bk, causal, budget, dtype, device, fixed_k=-1, out_dtype=None,
                 selector: int = 0, seed: int = 0, tile_order: int = 0):
        self.args = (B, Hq, Hkv, N, D, Bq, Bk, causal, budget, fixed_k)
        self.tile_order = tile_order                        # 0: Alg. 1's ascending order; 1: the order of the kernel in Sec. 3.3
        self.selector, self.seed = selector, seed           # 0: the paper's heuristic; else an App. A ablation selector
        dev = device
        u8, f32, i32 = torch.uint8, torch.float32, torch.int32
        Tq, Tk = -(-N // Bq), -(-N // Bk)                   # N need not be a multiple of the blocks
        self.Tq, self.Tk = Tq, Tk
        self.qmean = torch.empty(B, Hq, Tq, D, dtype=f32, device=dev)
        self.kmean = torch.empty(B, Hkv, Tk, D, dtype=f32, device=dev)
        self.kmax = max(1, select_kmax(Tq, Tk, Bq, Bk, causal, budget, fixed_k))
        self.idx = torch.empty(B, Hq, Tq, self.kmax, dtype=i32, device=dev)
        self.cnt = torch.empty(B, Hq, Tq, dtype=i32, device=dev)
        self.q4 = torch.empty(B, Hq, N, D // 2, dtype=u8, device=dev)
        self.qs = torch.empty(B, Hq, N, D // 32, dtype=u8, device=dev)
        self.k4 = torch.empty(B, Hkv, N, D // 2, dtype=u8, device=dev)
        self.ks = torch.empty(B, Hkv, N, D // 32, dtype=u8, device=dev)
        self.v4 = torch.empty(B, Hkv, -(-N // 64), D, 32, dtype=u8, device=dev)
        self.vs = torch.empty(B, Hkv, 2 * -(-N // 64), D, dtype=u8, device=dev)
        self.out = torch.empty(B, Hq, N, D, dtype=out_dtype or dtype, device=dev)

    def run(self, q, k, v, softmax_scale: float = 0.0, prepass: bool = True, attention: bool = True) -> torch.Tensor:
        B, Hq, Hkv, N, D, Bq, Bk, causal, budget, fixed_k = self.args
        if prepass:
            if Bk == 64 and Bq in (64, 128) and q.dtype == k.dtype == v.dtype:
                thrift_prefill_prepass(q, k, v, Bq, Bk, self.qmean, self.kmean, self.q4, self.qs, self.k4, self.ks, self.v4, self.vs)
            else:                                           # blocks and mixed types that only the single calls take
                thrift_block_means(q, Bq, out=self.qmean)
                thrift_block_means(k, Bk, out=self.kmean)
                thrift_quantize_mxfp4(q, 0, self.q4, self.qs)
                thrift_quantize_mxfp4(k, 0, self.k4, self.ks)
                thrift_quantize_mxfp4(v, 1, self.v4, self.vs)
            if self.selector == 0:
                thrift_select_topk(self.qmean, self.kmean, Bq, Bk, causal, budget, fixed_k, kmax=self.kmax, idx=self.idx, cnt=self.cnt)
            else:
                thrift_select_ablation(self.selector, self.seed, B, Hq, self.Tq, self.Tk, Bq, Bk, causal, budget, fixed_k,
                                       kmax=self.kmax, idx=self.idx, cnt=self.cnt)
        if attention:
            thrift_attn_prefill_chunk(q, k, v, self.q4, self.qs, self.k4, self.ks, self.v4, self.vs, self.idx, self.cnt, Bq, Bk,
                                      causal, 0, softmax_scale, out=self.out, tile_order=self.tile_order)
        return self.out


def thrift_attention(q, k, v, causal: bool = True, Bq: int = 128, Bk: int = 64, budget: float = 0.05,
                     fixed_k: int = -1, softmax_scale: float = 0.0, out_dtype=None,
                     workspace: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                     lse: Optional[torch.Tensor] = None, tile_order: int = 0) -> torch.Tensor:
    """Alg. 1: Q, K, V, block sizes and FP16 budget in, attention output out (thrift_attention_forward: one C call)."""
    if out is not None or out_dtype is None:
        r = (_call or _native()).attention(q, k, v, int(causal), Bq, Bk, budget, fixed_k, softmax_scale, workspace, out, lse, tile_order,
                                           _raw_stream())
        if r is not None:
            return _result(r, "thrift_attention_forward")
    for t in (q, k, v):
        _dev(t)
    B, Hq, N, D = q.shape
    Hkv = k.shape[1]
    assert q.dtype == k.dtype == v.dtype and k.shape == v.shape == (B, Hkv, N, D), (q.dtype, k.dtype, v.dtype, k.shape, v.shape)
    need = int(lib().thrift_attention_forward_workspace(B, Hq, Hkv, N, D, Bq, Bk, int(causal), float(budget), int(fixed_k)))
    if workspace is None:
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty(B, Hq, N, D, dtype=out_dtype or q.dtype, device=q.device)
    _check(lib().thrift_attention_forward(_ptr(q), _ptr(k), _ptr(v), _DT[q.dtype], B, Hq, Hkv, N, D, Bq, Bk, int(causal),
                                          float(budget), int(fixed_k), int(tile_order), float(softmax_scale), _ptr(out), _DT[out.dtype],
                                          _ptr(lse), _ptr(workspace), workspace.numel(), _stream()), "thrift_attention_forward")
    return out

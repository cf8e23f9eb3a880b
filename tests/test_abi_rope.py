"""Host checks of the rotary encoding's entry points, made before any device
memory is touched (no GPU; pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2601_09083_amd import srt as S
from tests.test_abi_quant_rules import P, built_library  # noqa: F401

ODD = ctypes.c_void_p(4104)  # not 16-byte aligned


def rope(inv_freq=4096, rot=128, interleaved=0, factor=1.0, reserved=0):
    return S.RopeArgs(inv_freq, rot, interleaved, factor, reserved)


def append(r=None, B=4, T=8, Hq=4, Hkv=2, d=128, page=16, max_pages=8, num_pages=9, q=P, ldq=512, k=P, v=P, ldkv=256, depth=P,
           counts=P, q_out=P, kc=P, vc=P, bt=P, ctx=P):
    return S.lib().srt_rope_append(ctypes.byref(r or rope()), B, T, Hq, Hkv, d, page, max_pages, num_pages, q, ldq, k, v, ldkv,
                                   depth, counts, q_out, kc, vc, bt, ctx, None)


def rows(r=None, B=4, T=8, Hq=4, Hkv=2, d=128, q=P, ldq=512, k=P, ldk=256, depth=P, counts=P, ctx=P, q_out=P, k_out=P, ldo=256):
    return S.lib().srt_rope_rows(ctypes.byref(r or rope()), B, T, Hq, Hkv, d, q, ldq, k, ldk, depth, counts, ctx, q_out, k_out,
                                 ldo, None)


@pytest.mark.parametrize("call", [append, rows])
def test_bad_encodings_and_sizes_are_refused(call):
    bad, un = S.SRT_ERR_INVALID, S.SRT_ERR_UNSUPPORTED
    for kw in (dict(rot=0), dict(rot=144), dict(interleaved=2), dict(factor=float("nan")), dict(factor=float("inf")),
               dict(reserved=1), dict(inv_freq=None)):
        assert call(rope(**kw)) == bad, kw
    for kw in (dict(B=-1), dict(T=0), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(ldq=504), dict(ldq=516), dict(q=None),
               dict(k=None), dict(counts=None), dict(ctx=None), dict(q_out=None), dict(q=ODD), dict(k=ODD), dict(q_out=ODD)):
        assert call(**kw) == bad, kw
    assert call(rope(rot=24)) == un and call(rope(rot=8)) == un
    assert call(d=132, ldq=1024, ldkv=1024) == un if call is append else call(d=132, ldq=1024, ldk=1024, ldo=1024) == un
    assert call(d=520, ldq=1 << 20) == un and call(Hq=(1 << 16) + 1, ldq=1 << 30) == un
    assert call(B=0) == S.SRT_OK
    assert S.lib().srt_rope_append(None, 4, 8, 4, 2, 128, 16, 8, 9, P, 512, P, P, 256, P, P, P, P, P, P, P, None) == bad


def test_bad_caches_and_rows_are_refused():
    for kw in (dict(page=0), dict(max_pages=0), dict(num_pages=0), dict(ldkv=248), dict(ldkv=260), dict(v=None), dict(kc=None),
               dict(vc=None), dict(bt=None), dict(v=ODD), dict(kc=ODD), dict(vc=ODD)):
        assert append(**kw) == S.SRT_ERR_INVALID, kw
    for kw in (dict(ldk=248), dict(ldo=248), dict(ldo=260), dict(k_out=None), dict(k_out=ODD)):
        assert rows(**kw) == S.SRT_ERR_INVALID, kw


def test_batches_beyond_a_launch_are_refused():
    assert append(B=1 << 16, T=1 << 12) == S.SRT_ERR_UNSUPPORTED
    assert rows(B=(1 << 31) - 1, T=(1 << 31) - 1) == S.SRT_ERR_UNSUPPORTED


def test_an_encoding_needs_device_memory():
    with pytest.raises(ValueError):
        S.Rope(torch.zeros(64))

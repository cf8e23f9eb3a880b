"""Sizes whose launch would have 2^32 threads or more are refused on the host (no
GPU; pointers are never followed)."""
import ctypes

from paper_2601_09083_amd import srt as S
from tests.test_abi_quant_rules import P, append, built_library, commit, kv  # noqa: F401


def rules(B, V, sampled=False):
    noise = P if sampled else None
    return S.lib().srt_accept_rules(B, 8, V, 4, P, noise, 1.0, ctypes.byref(S.RulesArgs()), P, P, P, P, P, P, None, P, 1 << 45,
                                    None)


def seen(B, V, stride, reset):
    return S.lib().srt_seen_add(P, B, V, P, P, stride, 0, reset, None)


def test_batches_beyond_a_launch_are_refused():
    one = kv(Hkv=1, d=64)
    assert append(one, B=1 << 16, T=4096) == S.SRT_ERR_UNSUPPORTED       # 2^16 x 257 workgroups of 512 threads
    assert append(one, B=1 << 23, T=1) == S.SRT_ERR_UNSUPPORTED
    assert append(kv(Hkv=255), B=(1 << 31) - 1, T=(1 << 31) - 1, ld=1 << 20) == S.SRT_ERR_UNSUPPORTED
    assert commit(one, B=1 << 23) == S.SRT_ERR_UNSUPPORTED
    between = 0xFFFFFFFF // 576 + 1  # too many with the wave of the draft inputs
    assert commit(one, B=between, tail=P, length=P) == S.SRT_ERR_UNSUPPORTED
    assert commit(one, B=between, acc=None) == S.SRT_ERR_INVALID  # (further on, without them)
    assert rules(1 << 24, 1000) == S.SRT_ERR_UNSUPPORTED
    assert rules(1 << 22, 4000) == S.SRT_ERR_UNSUPPORTED
    assert rules(1 << 19, 152064, sampled=True) == S.SRT_ERR_UNSUPPORTED
    assert seen(1 << 22, 100, 100, 0) == S.SRT_ERR_UNSUPPORTED
    assert seen(1 << 20, 152064, 13, 1) == S.SRT_ERR_UNSUPPORTED
    assert seen((1 << 26) - 2, 100, 13, 0) == S.SRT_ERR_UNSUPPORTED

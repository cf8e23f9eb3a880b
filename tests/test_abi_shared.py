"""Host checks of the shared-prefix attention, made before any device memory is
touched (no GPU; pointers are never followed)."""
import ctypes

import pytest

from paper_2601_09083_amd import srt as S
from tests.test_abi_quant_rules import P, built_library  # noqa: F401


def attn(B=4, N=8, Hq=4, Hkv=2, d=128, page=16, max_pages=40, num_pages=100, n_groups=2, q=P, k=P, v=P, bt=P, ctx=P, par=P, n=P,
         ids=P, prefix=P, scale=0.1, out=P, scratch=P, size=1 << 40):
    return S.lib().srt_tree_attn_shared(B, N, Hq, Hkv, d, page, max_pages, num_pages, n_groups, q, k, v, bt, ctx, par, n, ids,
                                        prefix, scale, out, scratch, size, None)


def need(B=4, N=8, Hq=4, Hkv=2, d=128, page=16, max_pages=40, n_groups=2):
    return S.srt_tree_attn_shared_scratch_bytes(B, N, Hq, Hkv, d, page, max_pages, n_groups)


def test_sizes():
    bad, un = S.SRT_ERR_INVALID, S.SRT_ERR_UNSUPPORTED
    for kw, st in ((dict(B=-1), bad), (dict(N=0), bad), (dict(N=257), bad), (dict(Hq=0), bad), (dict(Hkv=0), bad),
                   (dict(Hq=5), bad), (dict(page=0), bad), (dict(max_pages=0), bad), (dict(n_groups=-1), bad), (dict(d=96), un),
                   (dict(page=8), un), (dict(page=24), un), (dict(B=65536), un), (dict(n_groups=4097), un),
                   (dict(Hkv=256, Hq=256), un), (dict(max_pages=(1 << 26) + 1), un), (dict(B=65535, N=256, Hq=2), un)):
        assert attn(**kw) == st and need(**kw) == 0, kw
    assert attn(num_pages=0) == bad and attn(scale=float("nan")) == bad and attn(scale=float("inf")) == bad
    assert attn(B=0) == S.SRT_OK and need() > 0


def test_pointers_and_scratch():
    for name in ("q", "k", "v", "bt", "ctx", "par", "n", "ids", "prefix", "out"):
        assert attn(**{name: None}) == S.SRT_ERR_INVALID, name
    assert attn(scratch=None) == S.SRT_ERR_CAPACITY and attn(size=need() - 1) == S.SRT_ERR_CAPACITY
    assert attn(scratch=ctypes.c_void_p(4096 + 16)) == S.SRT_ERR_INVALID
    assert attn(n_groups=0, ids=None, prefix=None, size=0) == S.SRT_ERR_CAPACITY  # (further on, without groups)


@pytest.mark.parametrize("n_groups", [0, 2])
def test_calls_that_the_plain_attention_refuses(n_groups):
    """Some calls go to srt_tree_attn: what it cannot pack is refused by both, before anything is read."""
    for B, pages in ((4, 1 << 22), (1, 1 << 22), (512, 1 << 22)):
        assert S.srt_tree_attn_scratch_bytes(B, 8, 4, 2, 128, 16, pages) > 0
        assert need(B=B, max_pages=pages, n_groups=n_groups) == 0
        assert attn(B=B, max_pages=pages, n_groups=n_groups) == S.SRT_ERR_UNSUPPORTED
    # (4095 splits of 8192 positions are the most that one packs)
    assert need(B=4, max_pages=4095 * 512, n_groups=n_groups) > 0 and need(B=4, max_pages=4095 * 512 + 1, n_groups=n_groups) == 0

"""Host checks of the 8-bit cache's and the sampling rules' entry points, made
before any device memory is touched (no GPU; pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2601_09083_amd import srt as S

P = ctypes.c_void_p(4096)


@pytest.fixture(autouse=True)
def built_library():
    import os
    if not os.path.exists(S.LIB_PATH):
        from paper_2601_09083_amd import build as B
        B.build()


def kv(**kw):
    a = dict(kv_type=0, Hkv=2, d=128, page=16, max_pages=40, reserved=0, num_pages=100)
    a.update({k: 4096 for k in ("k_pages", "v_pages", "k_scale", "v_scale", "k_tail", "v_tail", "block_table", "ctx_len")})
    a.update(kw)
    return S.KvQuantArgs(**a)


BAD_CACHES = [
    (dict(kv_type=2), S.SRT_ERR_INVALID), (dict(kv_type=-1), S.SRT_ERR_INVALID), (dict(Hkv=0), S.SRT_ERR_INVALID),
    (dict(max_pages=0), S.SRT_ERR_INVALID), (dict(num_pages=0), S.SRT_ERR_INVALID), (dict(reserved=1), S.SRT_ERR_INVALID),
    (dict(page=0), S.SRT_ERR_INVALID), (dict(Hkv=256), S.SRT_ERR_UNSUPPORTED), (dict(d=96), S.SRT_ERR_UNSUPPORTED),
    (dict(page=8), S.SRT_ERR_UNSUPPORTED), (dict(page=24), S.SRT_ERR_UNSUPPORTED), (dict(page=512), S.SRT_ERR_UNSUPPORTED),
    (dict(page=256, max_pages=1 << 22), S.SRT_ERR_UNSUPPORTED),
    (dict(k_pages=None), S.SRT_ERR_INVALID), (dict(v_scale=None), S.SRT_ERR_INVALID), (dict(ctx_len=None), S.SRT_ERR_INVALID),
    (dict(v_pages=4104), S.SRT_ERR_INVALID), (dict(k_tail=4104), S.SRT_ERR_INVALID),
]


def attn(c, B=4, N=8, Hq=4, q=P, k=P, v=P, ld=256, par=P, n=P, scale=0.1, out=P, scratch=P, size=1 << 30):
    return S.lib().srt_tree_attn_quant(ctypes.byref(c), B, N, Hq, q, k, v, ld, par, n, scale, out, scratch, size, None)


def append(c, B=4, T=8, k=P, v=P, ld=256, counts=P):
    return S.lib().srt_kv_append(ctypes.byref(c), B, T, k, v, ld, counts, None)


def commit(c, B=4, N=8, k=P, v=P, ld=256, Dmax=4, acc=P, tok=P, nod=P, Q=8, tail=None, length=None):
    return S.lib().srt_commit_quant(ctypes.byref(c), B, N, k, v, ld, Dmax, acc, tok, nod, Q, tail, length, None)


def read(c, B=4, T=8, start=P, k=P, v=P):
    return S.lib().srt_kv_read(ctypes.byref(c), B, T, start, k, v, None)


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(bad, status):
    for call in (attn, append, commit, read):
        assert call(kv(**bad)) == status, call.__name__
    if "page" in bad or "d" in bad or "kv_type" in bad:
        assert S.lib().srt_tree_attn_quant_scratch_bytes(ctypes.byref(kv(**bad)), 4, 8, 4) == 0


@pytest.mark.parametrize("call", [append, commit, attn])
def test_bad_new_vectors(call):
    c = kv()
    assert call(c, k=None) == S.SRT_ERR_INVALID and call(c, v=None) == S.SRT_ERR_INVALID
    assert call(c, ld=255) == S.SRT_ERR_INVALID       # less than a token's heads
    assert call(c, ld=260) == S.SRT_ERR_INVALID       # not a multiple of 8
    assert call(c, k=ctypes.c_void_p(4104)) == S.SRT_ERR_INVALID
    assert call(c, B=-1) == S.SRT_ERR_INVALID
    assert call(c, B=0) == S.SRT_OK


def test_attention_arguments():
    c = kv()
    for kw in (dict(N=0), dict(N=257), dict(Hq=0), dict(Hq=5), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(q=None), dict(out=None), dict(par=None), dict(n=None), dict(q=ctypes.c_void_p(4100)),
               dict(scratch=ctypes.c_void_p(4096 + 16))):
        assert attn(c, **kw) == S.SRT_ERR_INVALID, kw
    need = S.lib().srt_tree_attn_quant_scratch_bytes(ctypes.byref(c), 4, 8, 4)
    assert need > 0 and need % 4 == 0
    assert attn(c, size=16) == S.SRT_ERR_CAPACITY and attn(c, scratch=None) == S.SRT_ERR_CAPACITY
    assert attn(c, B=65536) == S.SRT_ERR_UNSUPPORTED
    assert attn(c, N=256, Hq=1 << 30) == S.SRT_ERR_UNSUPPORTED
    assert S.lib().srt_tree_attn_quant_scratch_bytes(ctypes.byref(c), 4, 256, 1 << 30) == 0
    assert attn(kv(page=256, max_pages=1 << 21)) == S.SRT_ERR_UNSUPPORTED  # more than 4095 splits
    assert S.lib().srt_tree_attn_quant_scratch_bytes(None, 4, 8, 4) == 0
    assert S.lib().srt_tree_attn_quant(None, 4, 8, 4, P, P, P, 256, P, P, 0.1, P, P, 1 << 30, None) == S.SRT_ERR_INVALID


def test_write_and_read_arguments():
    c = kv()
    assert append(c, T=0) == S.SRT_ERR_INVALID and append(c, counts=None) == S.SRT_ERR_INVALID
    assert append(c, B=1 << 20, T=1 << 30) == S.SRT_ERR_UNSUPPORTED
    for kw in (dict(N=0), dict(N=257), dict(Dmax=-1), dict(Dmax=64), dict(tail=P), dict(length=P), dict(tail=P, length=P, Q=0),
               dict(tail=P, length=P, Q=65), dict(acc=None), dict(tok=None), dict(nod=None)):
        assert commit(c, **kw) == S.SRT_ERR_INVALID, kw
    for kw in (dict(T=0), dict(B=-1), dict(start=None), dict(k=None), dict(v=ctypes.c_void_p(4104))):
        assert read(c, **kw) == S.SRT_ERR_INVALID, kw
    assert read(c, B=0) == S.SRT_OK


def test_rules_arguments():
    L = S.lib()
    none = S.RulesArgs()

    def walk(r=none, B=4, N=8, V=100, D=4, logits=P, tok=P, n=P, scratch=P, size=1 << 20, invT=1.0):
        return L.srt_accept_rules(B, N, V, D, logits, None, invT, ctypes.byref(r), tok, P, n, P, P, P, None, scratch, size, None)

    for kw in (dict(B=-1), dict(N=0), dict(N=257), dict(V=0), dict(D=64), dict(logits=None), dict(tok=None), dict(n=None),
               dict(invT=float("nan")), dict(scratch=ctypes.c_void_p(4112)), dict(r=S.RulesArgs(reserved=1)),
               dict(r=S.RulesArgs(n_bias=-1)), dict(r=S.RulesArgs(bias_tokens=4096, n_bias=1)),
               dict(r=S.RulesArgs(bias_offsets=4096, n_bias=1))):
        assert walk(**kw) == S.SRT_ERR_INVALID, kw
    assert walk(size=8) == S.SRT_ERR_CAPACITY and walk(scratch=None) == S.SRT_ERR_CAPACITY
    assert walk(V=(1 << 21) + 1) == S.SRT_ERR_UNSUPPORTED
    assert walk(B=0) == S.SRT_OK
    assert L.srt_accept_rules(4, 8, 100, 4, P, None, 1.0, None, P, P, P, P, P, P, None, P, 1 << 20, None) == S.SRT_ERR_INVALID


def test_seen_arguments():
    def add(seen=P, B=4, V=100, tok=P, n=P, stride=3, prompt=0, reset=0):
        return S.lib().srt_seen_add(seen, B, V, tok, n, stride, prompt, reset, None)

    for kw in (dict(B=-1), dict(V=0), dict(stride=0), dict(prompt=2), dict(reset=-1), dict(seen=None), dict(tok=None),
               dict(n=None)):
        assert add(**kw) == S.SRT_ERR_INVALID, kw
    assert add(B=0) == S.SRT_OK
    assert add(B=1 << 30, V=1 << 30) == S.SRT_ERR_UNSUPPORTED


def test_binding_refuses_tensors_that_do_not_fit():
    f8 = torch.zeros((3, 2, 16, 64), dtype=torch.uint8).view(torch.float8_e4m3fn)
    sc, tail = torch.zeros(3, 2), torch.zeros((1, 2, 16, 64), dtype=torch.bfloat16)
    bt, ln = torch.zeros((1, 3), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="float8_e4m3fn or torch.int8"):
        S.KvQuant(f8.view(torch.uint8), f8, sc, sc, tail, tail, bt, ln)
    with pytest.raises(ValueError, match="shape"):
        S.KvQuant(f8, f8, sc[:2], sc, tail, tail, bt, ln)
    with pytest.raises(ValueError, match="tails"):
        S.KvQuant(f8, f8, sc, sc, tail[:, :, :8], tail, bt, ln)
    with pytest.raises(ValueError, match="block_table"):
        S.KvQuant(f8, f8, sc, sc, tail, tail, bt[0], ln)
    with pytest.raises(ValueError, match="CUDA"):
        S.KvQuant(f8, f8, sc, sc, tail, tail, bt, ln)
    with pytest.raises(ValueError, match="no such rule"):
        S.Rules(temperature=sc)
    with pytest.raises(ValueError, match="bias lists"):
        S.Rules(bias_tokens=ln)

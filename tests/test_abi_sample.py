"""Host checks of the sampling walk, made before any device memory is touched (no
GPU; pointers are never followed)."""
import ctypes

import pytest
import torch

from paper_2601_09083_amd import srt as S
from tests.test_abi_quant_rules import P, built_library  # noqa: F401


def walk(B=4, N=8, V=100, Dmax=4, logits=P, gumbel=P, reserved=0, rules=None, tok=P, par=P, n=P, acc=P, out=P, nodes=P, em=P):
    s = S.SamplingArgs(reserved=reserved)
    r = ctypes.byref(rules) if rules is not None else None
    return S.lib().srt_accept_sample(B, N, V, Dmax, logits, gumbel, ctypes.byref(s), r, tok, par, n, acc, out, nodes, em, None)


def test_sizes_and_pointers():
    bad, un = S.SRT_ERR_INVALID, S.SRT_ERR_UNSUPPORTED
    for kw in (dict(B=-1), dict(N=0), dict(N=257), dict(V=0), dict(Dmax=-1), dict(Dmax=64), dict(logits=None), dict(tok=None),
               dict(par=None), dict(n=None), dict(acc=None), dict(out=None), dict(nodes=None), dict(reserved=1)):
        assert walk(**kw) == bad, kw
    assert walk(V=(1 << 21) + 1) == un and walk(B=1 << 24) == un and walk(B=1 << 23, V=9000) == un
    assert walk(B=0) == S.SRT_OK
    assert S.lib().srt_accept_sample(4, 8, 100, 4, P, P, None, None, P, P, P, P, P, P, P, None) == bad


def test_rules():
    bad, un = S.SRT_ERR_INVALID, S.SRT_ERR_UNSUPPORTED
    assert walk(rules=S.RulesArgs(reserved=1)) == bad and walk(rules=S.RulesArgs(n_bias=-1)) == bad
    assert walk(rules=S.RulesArgs(bias_tokens=4096)) == bad and walk(rules=S.RulesArgs(bias_offsets=4096, n_bias=3)) == bad
    assert walk(V=(1 << 18) + 1, rules=S.RulesArgs()) == un


def test_parameters_keep_their_tensors():
    s = S.Sampling(top_k=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(TypeError):
        s.tensors["top_p"] = torch.zeros(3)
    for kw in (dict(top_k=torch.zeros(3)), dict(top_p=torch.zeros(3, dtype=torch.float64)), dict(min_p=torch.zeros(6)[::2])):
        with pytest.raises(ValueError):
            S.Sampling(**kw)

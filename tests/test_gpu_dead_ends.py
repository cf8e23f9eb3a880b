"""Walks that end without a token (every token forbidden): what they leave to the
steps that follow."""
import numpy as np
import pytest
import torch

from oracle import commit as CO
from paper_2601_09083_amd import srt
from tests.quant_util import new_cache

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("qmax", [1, 4, 8, 64])
def test_commit_advances_the_draft_inputs_by_the_emitted_tokens(quant, qmax):
    """Every accepted length with and without a bonus token behind it."""
    rng = np.random.default_rng(qmax)
    N, dmax, hkv, page, d = 8, 5, 1, 16, 64
    k = np.repeat(np.arange(dmax + 1), 2)
    B = len(k)
    bonus = np.arange(B) % 2 == 0
    t = rng.integers(0, 12, B)
    tail = np.full((B, qmax), -1, np.int32)
    toks = np.full((B, dmax + 1), -1, np.int32)
    nodes = np.full((B, dmax + 1), -1, np.int32)
    for b in range(B):
        h = min(int(t[b]), qmax)
        tail[b, qmax - h:] = rng.integers(0, 1000, h)
        toks[b, :k[b] + bonus[b]] = rng.integers(0, 1000, k[b] + bonus[b])
        nodes[b, :k[b]] = np.arange(1, k[b] + 1)
    tail_dev, t_dev = i32(tail), i32(t)
    if quant:
        c = new_cache(B, hkv, page, d, "e4m3", 4, "cuda", ctx=t)
        new = torch.zeros((B, N, hkv, d), dtype=torch.bfloat16, device="cuda")
        srt.srt_commit_quant(c, new, new, i32(k), i32(toks), i32(nodes), ctx_tail=tail_dev, draft_len=t_dev)
        ctx = c.ctx_len
    else:
        cache = torch.zeros((B * 4, hkv, page, d), dtype=torch.bfloat16, device="cuda")
        ctx = i32(t)
        srt.srt_commit(cache, cache.clone(), i32(np.arange(B * 4).reshape(B, 4)), ctx, i32(k), i32(toks), i32(nodes), N,
                       ctx_tail=tail_dev, draft_len=t_dev)
    assert ctx.tolist() == (t + k + 1).tolist()  # the root and the accepted nodes have vectors
    for b in range(B):
        want, n = CO.commit_tail(tail[b], int(t[b]), toks[b, :k[b] + bonus[b]])
        assert tail_dev[b].tolist() == want.tolist() and int(t_dev[b]) == n, (b, int(k[b]), bool(bonus[b]))

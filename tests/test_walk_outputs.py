"""Outputs that a walk is given: ones of another walk's sizes are refused before
anything is enqueued (the kernels write B rows of max_depth + 1 entries)."""
import pytest
import torch

from paper_2601_09083_amd import srt as S

B, N, V, D = 4, 8, 100, 3


def arguments():
    i = torch.zeros((B, N), dtype=torch.int32)
    return torch.zeros((B, N, V)), i, i, torch.ones(B, dtype=torch.int32)


def outputs(**other):
    sizes = dict(n_accepted=(B,), out_tokens=(B, D + 1), out_nodes=(B, D + 1), n_emitted=(B,))
    sizes.update(other)
    return {k: torch.zeros(s, dtype=torch.int32) for k, s in sizes.items()}


BAD = [dict(out_tokens=(B, D)), dict(out_nodes=(B - 1, D + 1)), dict(n_accepted=(B - 1,)), dict(n_emitted=(1,))]


@pytest.mark.parametrize("bad", BAD)
def test_rules_walk_refuses_outputs_of_other_sizes(bad):
    logits, tok, par, n = arguments()
    with pytest.raises(ValueError, match=f"out: {list(bad)[0]}"):
        S.srt_accept_rules(logits, None, 1.0, S.Rules(), tok, par, n, D, out=outputs(**bad))


SMALL = [dict(out_tokens=(B, D)), dict(out_nodes=(B - 1, D + 1)), dict(n_accepted=(B - 1,)), dict(n_emitted=(1,))]


@pytest.mark.parametrize("small", SMALL)
@pytest.mark.parametrize("walk", ["accept", "noalloc", "lmhead"])
def test_walks_refuse_outputs_without_room(walk, small):
    logits, tok, par, n = arguments()
    out = outputs(**small)
    with pytest.raises(ValueError, match=f"out: {list(small)[0]}"):
        if walk == "accept":
            S.srt_accept(logits, None, 1.0, tok, par, n, D, out=out)
        elif walk == "noalloc":
            S.srt_accept_noalloc(logits, None, 1.0, tok, par, n, D, out)
        else:
            bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16)
            S.srt_accept_lmhead(bf(B, N, 64), bf(V, 64), None, 1.0, tok, par, n, D, out=out)


@pytest.mark.gpu
def test_rules_walk_keeps_the_scratch_it_is_given():
    """Without ``out`` too: a walk by levels leaves its lists in it."""
    logits, tok, par, n = (x.cuda() for x in (torch.zeros((B, N, 41000)), *arguments()[1:]))
    scratch = torch.full((S.srt_accept_scratch_bytes(B),), 0xAB, dtype=torch.uint8, device="cuda")
    S.srt_accept_rules(logits, None, 1.0, S.Rules(), tok, par, n, D, scratch=scratch)
    assert int((scratch != 0xAB).sum()) > 0

"""The block tables of sequences that share a prompt's pages, and how many positions they share."""
import numpy as np
import pytest
import torch

from paper_2601_09083_amd.pipeline import share_prefix

PAGE = 16


def tables(seq_prompt, prefix, ctx_len, width=20):
    before = torch.arange(len(seq_prompt) * width, dtype=torch.int32).reshape(-1, width)
    after = before.clone()
    shared = share_prefix(after, np.asarray(seq_prompt), prefix, np.asarray(ctx_len), PAGE)
    return before, after, shared


@pytest.mark.parametrize("prefix,ctx,want", [
    (100, [200, 150, 300], 96), (96, [200, 150, 300], 96), (15, [200, 150, 300], 0), (0, [200, 150, 300], 0),
    (400, [200, 191, 300], 176), (400, [200, 192, 300], 192), (2 ** 31 - 1, [40, 7, 300], 0)])
def test_what_a_prompts_sequences_share(prefix, ctx, want):
    """Whole pages of the prefix and of the shortest context, and no more than these, whatever the contexts become."""
    before, after, shared = tables([0, 0, 0], [prefix], ctx)
    assert shared.tolist() == [want] and shared.dtype == np.int32
    pages = want // PAGE
    assert (after[:, :pages] == before[0, :pages]).all() and torch.equal(after[:, pages:], before[:, pages:])


def test_prompts_apart_and_prompts_with_few_sequences():
    before, after, shared = tables([1, 0, 1, 3], [64, 64, 64, 400], [100, 100, 50, 70])
    assert shared.tolist() == [64, 48, 64, 64]
    assert torch.equal(after[[0, 1, 3]], before[[0, 1, 3]])
    assert torch.equal(after[2, :3], before[0, :3]) and torch.equal(after[2, 3:], before[2, 3:])


@pytest.mark.parametrize("prefix", [-1, -5, -16, -300])
def test_a_negative_prefix_shares_nothing(prefix):
    """As the attention takes it; no row's pages become another one's."""
    before, after, shared = tables([0, 0, 0], [prefix], [200, 150, 300])
    assert torch.equal(after, before) and shared.tolist() == [0]

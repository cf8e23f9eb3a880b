"""The planted rows of rounding_util tell separately rounded scores from fused
ones: the oracle's walk takes the other token in every one of them."""
import numpy as np
import pytest

from tests.rounding_util import GREEDY, SAMPLED, Planted


@pytest.mark.parametrize("kinds,sampled,bf16", [(GREEDY, False, False), (SAMPLED, True, False), (("noise",), True, True)])
@pytest.mark.parametrize("V", [11, 1003])
def test_planted_rows_are_decided_by_a_rounding(kinds, sampled, bf16, V):
    c = Planted(V, 48, V, kinds, sampled, bf16)
    for b in range(c.B):
        k, toks, _, _ = c.want(b)
        assert k == b % 2 and toks[-1] != c.fused[b], b
        at = np.flatnonzero((c.logits[b, k] != -60) & (c.logits[b, k] != 1000))
        assert toks[-1] in at and c.fused[b] in at  # the two of them, nothing else

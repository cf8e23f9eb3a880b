"""The walks on rows that are decided by the rounding of a score (rounding_util):
every operation is rounded by itself, as include/srt.h says."""
import numpy as np
import pytest
import torch

from paper_2601_09083_amd import srt
from paper_2601_09083_amd.pipeline import bias_lists
from tests.rounding_util import GREEDY, SAMPLED, Planted

pytestmark = pytest.mark.gpu

ROWS = [1003, 45003]  # walked by one workgroup, by a launch for every level


def dev(x, dtype=None):
    return None if x is None else torch.as_tensor(np.asarray(x), device="cuda", dtype=dtype)


@pytest.mark.parametrize("V", ROWS)
@pytest.mark.parametrize("sampled", [False, True])
def test_walk_under_rules(V, sampled):
    c = Planted(V + sampled, 48, V, SAMPLED if sampled else GREEDY, sampled)
    rules = srt.Rules(seen=dev(c.words.view(np.int16)), repetition=dev(c.r), frequency=dev(c.f), presence=dev(c.q),
                      **bias_lists([dict(x) for x in c.bias]))
    c.check(srt.srt_accept_rules(dev(c.logits), dev(c.gumbel), float(c.invT), rules, dev(c.tok), dev(c.par),
                                 dev(c.n, torch.int32), c.dmax))


@pytest.mark.parametrize("V", ROWS)
def test_plain_walk(V):
    c = Planted(V + 2, 48, V, ("noise",), True)
    c.check(srt.srt_accept(dev(c.logits), dev(c.gumbel), float(c.invT), dev(c.tok), dev(c.par), dev(c.n, torch.int32),
                           c.dmax))

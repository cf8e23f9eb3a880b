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


@pytest.mark.parametrize("B", [48, 160])
@pytest.mark.parametrize("V", [1003, 70003])
def test_walk_with_the_head(V, B):
    """One hidden value that is not zero: a node's logits are a column of the head, exactly."""
    c = Planted(V + B, B, V, ("noise",), True, bf16=True)
    hidden = torch.eye(2 * B, device="cuda").to(torch.bfloat16).view(B, 2, 2 * B)
    head = dev(c.logits.reshape(2 * B, V)).t().to(torch.bfloat16)
    d = (2 * B + 63) // 64 * 64
    pad = lambda x: torch.nn.functional.pad(x, (0, d - 2 * B)).contiguous()
    c.check(srt.srt_accept_lmhead(pad(hidden), pad(head), dev(c.gumbel), float(c.invT), dev(c.tok), dev(c.par),
                                  dev(c.n, torch.int32), c.dmax))

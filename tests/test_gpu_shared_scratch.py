"""Shared-prefix attention reads nothing of its scratch that the call has not written:
every live row of every sequence is the same whatever the scratch held."""
import pytest
import torch

from paper_2601_09083_amd import srt
from tests.test_gpu_shared import Case, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,prefix,own,N,hq,hkv,d", [
    ([6, 5], [1500, 2300], (0, 900), 7, 12, 2, 128),                       # trees, split prefixes
    ([9, 1, 4], [3000, 40, 17], (0, 90), 3, 4, 2, 64),                     # a group that shares nothing, one of a page
    ([40, 30], [700, 1100], (0, 300), 1, 28, 4, 128),                      # single tokens
])
def test_a_scratch_of_any_contents(groups, prefix, own, N, hq, hkv, d):
    c = Case(31 + N, groups, prefix, own, N, hq, hkv, d, alone=2)
    need = srt.srt_tree_attn_shared_scratch_bytes(c.B, N, hq, hkv, d, 16, c.bt.shape[1], len(groups))
    live = torch.arange(N, device="cuda") < i32(c.n)[:, None]
    want = c.run()[live]
    for fill in (0, 255, 127):
        scratch = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        out = c.run(scratch=scratch)
        assert torch.equal(out[live], want), fill
        assert torch.equal(c.run(scratch=scratch)[live], want), fill  # (and what the call before has left there)
    c.check(out)

"""Walks that end without a token (every token forbidden): what they leave to the
steps that follow."""
import numpy as np
import pytest
import torch

from oracle import commit as CO
from oracle import kv_quant as KQ
from oracle import rules as RU
from paper_2601_09083_amd import srt
from paper_2601_09083_amd import workload as W
from paper_2601_09083_amd.pipeline import VerifyState
from tests.gpu_util import tree_to_np
from tests.quant_util import new_cache
from tests.test_gpu_quant_step import history

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


@pytest.mark.parametrize("kv", ["bf16", "e4m3"])
def test_sequences_that_end_stay_as_they_are(kv):
    """Sequence 1 finds its root's row forbidden in the first step, sequence 2 every
    other row, in the step in which it first leaves the root; 0 and 3 go on."""
    cfg = W.CONFIGS["tiny"]
    plain = VerifyState.build(cfg, kv_headroom=64)
    hist = [history(plain, b) for b in range(4)]
    st = plain if kv == "bf16" else VerifyState.build(cfg, kv=kv, kv_headroom=64)
    B, V, N = st.tokens.batch, cfg.vocab, cfg.n_nodes
    mask_np = np.full((B, N, V // 32), 0xFFFFFFFF, dtype=np.uint32)
    mask_np[1, 0] = 0
    mask_np[2, 1:] = 0
    st.use_rules([1.1] * B, [0.4] * B, [0.2] * B, mask=torch.as_tensor(mask_np.view(np.int32), device="cuda"))
    words = [RU.seen_add(np.zeros(V, np.uint16), list(st.tokens.seqs[b]), False, True) for b in range(B)]
    tails, t_len, ctx = st.ctx_tail.cpu().numpy(), st.draft_len.tolist(), st.attn_len.tolist()
    said = [list(y) for y in st.tokens.seqs]
    ended = [False] * B
    new = [x.float().cpu().numpy() for x in (st.k_new, st.v_new)] if kv != "bf16" else None
    for step in range(24):  # (pages of ended sequences would become full)
        tree = tree_to_np(st.draft())
        st.attention()
        st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda",
                                  boost="top", seed=300 + step)
        st.gumbel = None
        acc = {k: x.cpu().numpy() for k, x in st.accept().items()}
        st.insert()
        st.commit()
        lg = st.logits.cpu().numpy()
        for b in range(B):
            if ended[b]:
                assert (int(acc["n_accepted"][b]), int(acc["n_emitted"][b])) == (0, 0)
                assert (acc["out_tokens"][b] == -1).all() and (acc["out_nodes"][b] == -1).all()
                continue
            k, toks, nodes, e = RU.walk(lambda u: lg[b, u], None, 1.0, tree["tree_tokens"][b], tree["tree_parent"][b],
                                        int(tree["n_nodes"][b]), cfg.max_depth, words[b], 1.1, 0.4, 0.2, (),
                                        lambda u: mask_np[b, u])
            assert acc["out_tokens"][b, :len(toks)].tolist() == toks and int(acc["n_emitted"][b]) == e
            words[b] = RU.seen_add(words[b], toks[:e], False, False)
            tails[b], t_len[b] = CO.commit_tail(tails[b], t_len[b], toks[:e])
            ctx[b] += k + 1
            said[b] += toks[:e]
            ended[b] = e == k
            if new is not None:
                hist[b] = [np.concatenate([hist[b][i], new[i][b, [0] + nodes]]) for i in range(2)]
        assert st.ended.tolist() == ended
        assert np.array_equal(st.ctx_tail.cpu().numpy(), tails) and st.draft_len.tolist() == t_len
        assert st.attn_len.tolist() == ctx
        assert np.array_equal(st.seen.cpu().numpy().view(np.uint16), np.array(words))
        if ctx[0] + N + cfg.max_depth >= st.block_table.shape[1] * cfg.page:
            break
    assert ended == [False, True, True, False] and step >= 4
    assert all(len(y) == n for y, n in zip(said, t_len))
    if kv != "bf16":
        for b in range(B):
            got = srt.srt_kv_read(st.kv, i32([0] * B), max(ctx))
            for i in range(2):
                want, _, _ = KQ.context(hist[b][i], kv, cfg.page)
                want = torch.from_numpy(want.astype(np.float32)).to(torch.bfloat16)
                assert torch.equal(got[i][b, :ctx[b]].cpu(), want), (b, i)

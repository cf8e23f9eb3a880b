"""The verification step over an 8-bit KV cache and under sampling rules, its
calls strung together as a decode loop makes them, against the oracles: draft
trees, walks, count rows, cache contents and draft inputs exactly, attention
within the tolerance of quant_util.  Three steps, each from what the one before
left."""
import numpy as np
import pytest
import torch

from oracle import attention as AT
from oracle import commit as CO
from oracle import kv_quant as KQ
from oracle import rules as RU
from paper_2601_09083_amd import workload as W
from paper_2601_09083_amd.pipeline import VerifyState
from tests.gpu_util import oracle_draft_rows, oracle_trie, say, tree_to_np

pytestmark = pytest.mark.gpu


def history(st, b):
    """K and V [L, Hkv, d] float32 of a bf16 state's sequence b."""
    c, L = st.cfg, int(st.tokens.ctx_len[b])
    pages = st.block_table[b].long().clamp(min=0)
    out = []
    for cache in (st.k_cache, st.v_cache):
        x = cache[pages].float().cpu().numpy().transpose(0, 2, 1, 3).reshape(-1, c.hkv, c.head_dim)
        out.append(x[:L])
    return out


def attention_tolerance(q, K, V, parent, n, L, scale):
    """fp64 output and the tolerance of quant_util.AttnCase.reference."""
    as_cache = lambda x: x.transpose(1, 0, 2)[None]
    one = lambda v: AT.tree_attention_seq(q, as_cache(K), as_cache(v), np.zeros(1, int), L, parent, n, scale, len(K))
    ref, amp = one(V), one(np.abs(V))
    G = q.shape[1] // K.shape[1]
    s = np.stack([np.abs(q[:n, h]) @ np.abs(K[:, h // G]).T for h in range(q.shape[1])], 1).max(-1) * scale
    e = 2 * (q.shape[2] + 16) * 2.0 ** -24 * s[..., None]
    tol = 2.0 ** -8 * (amp + 2 * np.abs(ref)) + (2 * e + len(K) * 2.0 ** -24) * amp + len(K) * 448 * 2.0 ** -126
    return ref, 1.02 * tol


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_three_steps_under_rules(kv):
    cfg = W.CONFIGS["tiny"]
    plain = VerifyState.build(cfg, kv_headroom=64)  # the same vectors, in bf16
    B, V, N = plain.tokens.batch, cfg.vocab, cfg.n_nodes
    hist = [history(plain, b) for b in range(B)]
    st = VerifyState.build(cfg, kv=kv, kv_headroom=64)
    new = [x.float().cpu().numpy() for x in (st.k_new, st.v_new)]
    rng = np.random.default_rng(1)
    rep, fre, pre = [1.1, 1.0, 1.3, 0.9], [0.4, 0.0, 1.0, 0.1], [0.2, 1.0, 0.0, 0.0]
    biases = [{int(t): float(np.float32(rng.normal(0, 2))) for t in rng.choice(V, 20, replace=False)} for _ in range(B)]
    mask_np = rng.integers(0, 1 << 32, (B, N, V // 32)).astype(np.uint32)
    mask_np[rng.random((B, N)) < 0.5] = 0xFFFFFFFF
    mask = torch.as_tensor(mask_np.view(np.int32), device="cuda")
    st.use_rules(rep, fre, pre, biases, mask)
    words = [RU.seen_add(np.zeros(V, np.uint16), list(st.tokens.seqs[b]), False, True) for b in range(B)]
    assert np.array_equal(st.seen.cpu().numpy().view(np.uint16), np.array(words))
    streams = [list(st.tokens.prior[p]) for p in range(cfg.n_prompts)]
    seqs = [np.array(y) for y in st.tokens.seqs]
    tails = st.ctx_tail.cpu().numpy()
    t_len = st.draft_len.tolist()
    q = st.q.float().cpu().numpy().astype(np.float64)
    for step in range(3):
        say(f"quant step: {kv} step {step}")
        tree = tree_to_np(st.draft())
        if step == 0:
            tries = [oracle_trie(streams[p] + [seqs[b] for b in range(B) if st.tokens.seq_prompt[b] == p], cfg.trie_depth)
                     for p in range(cfg.n_prompts)]
            rows = oracle_draft_rows(st, tries, range(B))
            for b in range(B):
                assert tree["tree_tokens"][b, :rows[b][3]].tolist() == list(rows[b][0])
        out = st.attention().float().cpu().numpy()
        st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda",
                                  boost="top", seed=100 + step)
        st.gumbel = W.make_gumbel(cfg, B, device="cuda", seed=200 + step)
        acc = {k: x.cpu().numpy() for k, x in st.accept(0.9).items()}
        st.insert()
        st.commit()
        lg, gu = st.logits.cpu().numpy(), st.gumbel.cpu().numpy()
        for b in range(B):
            n, L = int(tree["n_nodes"][b]), len(hist[b][0])
            K, Vv = (np.concatenate([KQ.context(hist[b][i], kv, cfg.page)[0], new[i][b, :n].astype(np.float64)])
                     for i in range(2))
            ref, tol = attention_tolerance(q[b], K, Vv, tree["tree_parent"][b], n, L, st.scale)
            assert (np.abs(out[b, :n] - ref) <= tol).all(), (step, b)
            k, toks, nodes, e = RU.walk(lambda u: lg[b, u], lambda j: gu[b, j], 0.9, tree["tree_tokens"][b],
                                        tree["tree_parent"][b], n, cfg.max_depth, words[b], rep[b], fre[b], pre[b],
                                        sorted(biases[b].items()), lambda u: mask_np[b, u])
            assert (int(acc["n_accepted"][b]), int(acc["n_emitted"][b])) == (k, e)
            assert acc["out_tokens"][b, :len(toks)].tolist() == toks and acc["out_nodes"][b, :k].tolist() == nodes
            words[b] = RU.seen_add(words[b], toks[:e], False, False)
            hist[b] = [np.concatenate([hist[b][i], new[i][b, [0] + nodes]]) for i in range(2)]
            tails[b], t_len[b] = CO.commit_tail(tails[b], t_len[b], toks)
            assert int(st.kv.ctx_len[b]) == L + k + 1
            _, codes, scales = KQ.context(hist[b][0], kv, cfg.page)
            pg = st.block_table[b, :len(codes)].long()
            assert np.array_equal(st.kv.k_pages.view(torch.uint8)[pg].cpu().numpy(), codes.view(np.uint8))
        assert np.array_equal(st.seen.cpu().numpy().view(np.uint16), np.array(words))
        assert np.array_equal(st.ctx_tail.cpu().numpy(), tails) and st.draft_len.tolist() == t_len
    assert st.caches.status()["flags"] == 0



def test_a_step_replayed_from_a_graph_equals_the_eager_steps():
    """Attention, walk under rules, counts and commit of one captured step, replayed
    four times with eager work between: the state goes on as the eager state's does."""
    cfg = W.CONFIGS["tiny"]
    states = [VerifyState.build(cfg, kv="e4m3", kv_headroom=64) for _ in range(2)]
    for st in states:
        st.use_rules([1.1] * 4, [0.4] * 4, [0.2] * 4)
        tree = tree_to_np(st.draft())
        st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda",
                                  boost="top", seed=7)
        st.gumbel = W.make_gumbel(cfg, 4, device="cuda", seed=8)
        st.accept()  # (allocates its outputs and scratch before the capture)
        st.attn_out.zero_()  # (rows behind a tree's last node are not written)

    def step(st):
        st.attention()
        st.accept()
        st.insert()
        st.commit()

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(states[0])
    for _ in range(4):
        g.replay()
        step(states[1])
        torch.randn(1 << 18, device="cuda").sum().item()
        a, b = states
        for x, y in ((a.attn_out, b.attn_out), (a.acc["out_tokens"], b.acc["out_tokens"]), (a.seen, b.seen),
                     (a.kv.ctx_len, b.kv.ctx_len), (a.kv.k_tail, b.kv.k_tail), (a.ctx_tail, b.ctx_tail),
                     (a.kv.k_pages.view(torch.uint8), b.kv.k_pages.view(torch.uint8)), (a.kv.v_scale, b.kv.v_scale)):
            assert torch.equal(x, y)

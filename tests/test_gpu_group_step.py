"""A decode loop of groups of rollouts as its calls are used together: drafted trees,
their vectors turned and written to the cache, attention over the prompts' shared
pages, the walk of a policy that samples with top-k, top-p and min-p (under rules as
well), insertion and commit -- each stage against its oracle, three steps, each from
what the one before left."""
import numpy as np
import pytest
import torch

from oracle import commit as CO
from oracle import rope as RO
from oracle import rules as RU
from oracle import sampling as SA
from paper_2601_09083_amd import workload as W
from paper_2601_09083_amd.pipeline import VerifyState
from tests.gpu_util import say, tree_to_np
from tests.test_gpu_quant_step import attention_tolerance

pytestmark = pytest.mark.gpu
INV = (1e4 ** (-np.arange(0, 64, 2) / 64)).astype(np.float32)


def config(n_prompts, each):
    return W.CONFIGS["tiny"].scaled(n_prompts=n_prompts, seqs_per_prompt=each, ctx_len=W.Dist("uniform", 200, 500))


def projection(cfg, B, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn((B, cfg.n_nodes, cfg.hq + 2 * cfg.hkv, cfg.head_dim), generator=g, device="cuda").to(torch.bfloat16)
    return x[:, :, :cfg.hq], x[:, :, cfg.hq:cfg.hq + cfg.hkv], x[:, :, cfg.hq + cfg.hkv:]


def positions_of(st, b, upto):
    """K and V of positions 0 .. upto - 1, float64 [upto, Hkv, d]."""
    c, p = st.cfg, np.arange(upto)
    pg = st.block_table[b].long()[torch.as_tensor(p // c.page, device="cuda")]
    return [x[pg, :, torch.as_tensor(p % c.page, device="cuda")].double().cpu().numpy() for x in (st.k_cache, st.v_cache)]


def turned(x, tol_of, pos):
    """(values, tolerance) of turned rows: the tolerance that test_gpu_rope derives."""
    y = RO.turn(x, pos, INV, False, 1.0)
    both = np.abs(x[..., :32]) + np.abs(x[..., 32:])
    return y, 2.0 ** -8 * np.abs(y) + np.concatenate([both, both], -1) * tol_of


@pytest.mark.parametrize("n_prompts,each,ruled", [(3, 2, True), (20, 16, False)])
def test_three_steps_of_a_group(n_prompts, each, ruled):
    """Few sequences (attention by the plain way) with all of them checked; 320, whose
    attention shares the prompts' pages."""
    cfg = config(n_prompts, each)
    prefix = [190 - 7 * (p % 5) for p in range(n_prompts)]
    st = VerifyState.build(cfg, kv_headroom=64, prefix=prefix)
    B, V, N = st.tokens.batch, cfg.vocab, cfg.n_nodes
    ids = st.tokens.seq_prompt
    for p in range(n_prompts):
        own, w = np.flatnonzero(ids == p), prefix[p] // cfg.page
        assert (st.block_table[own, :w] == st.block_table[own[0], :w]).all() and w >= 10
    seqs = list(range(B)) if B < 20 else [0, 15, 16, 100, 319]
    st.use_rope(torch.as_tensor(INV, device="cuda"), projection(cfg, B, 1))
    cuts = [(1.0, 0, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.2, 0, 1.0, 0.05), (1.0, 5, 0.8, 0.01), (1.0, 0, 1.0, 0.0)]
    inv, top_k, top_p, min_p = (np.array([cuts[b % 5][i] for b in range(B)]) for i in range(4))
    st.use_sampling(1 / inv, top_k, top_p, min_p)
    inv, top_p, min_p = (1 / inv).astype(np.float32), top_p.astype(np.float32), min_p.astype(np.float32)
    words = None
    if ruled:
        st.use_rules([1.2] * B, [0.3] * B, [0.1] * B)
        words = [RU.seen_add(np.zeros(V, np.uint16), list(st.tokens.seqs[b]), False, True) for b in range(B)]
    qkv = [x.double().cpu().numpy() for x in st.projected]
    tails, t_len = st.ctx_tail.cpu().numpy(), st.draft_len.tolist()
    for step in range(3):
        say(f"group step {step}: {B} sequences")
        tree = tree_to_np(st.draft())
        L = st.attn_len.tolist()
        before = {b: positions_of(st, b, L[b]) for b in seqs}
        st.write_tree()
        out = st.attention().double().cpu().numpy()
        q = st.q.double().cpu().numpy()
        after = {b: positions_of(st, b, L[b] + int(tree["n_nodes"][b])) for b in seqs}
        st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda", boost="top",
                                  seed=100 + step)
        st.gumbel = W.make_gumbel(cfg, B, device="cuda", seed=200 + step)
        acc = {k: x.cpu().numpy() for k, x in st.accept().items()}
        st.insert()
        st.commit()
        lg, gu = st.logits.cpu().numpy(), st.gumbel.cpu().numpy()
        for b in seqs:
            n, par = int(tree["n_nodes"][b]), tree["tree_parent"][b]
            pos = L[b] + tree["tree_depth"][b, :n]
            for got, x in ((q[b, :n], qkv[0][b, :n]), (after[b][0][L[b]:], qkv[1][b, :n])):
                y, tol = turned(x, 2.0 ** -20, pos)
                assert (np.abs(got - y) <= tol).all(), (step, b)
            assert np.array_equal(after[b][1][L[b]:], qkv[2][b, :n])
            assert all(np.array_equal(x[:L[b]], y) for x, y in zip(after[b], before[b]))
            ref, tol = attention_tolerance(q[b], *after[b], par, n, L[b], st.scale)
            assert (np.abs(out[b, :n] - ref) <= tol).all(), (step, b)
            rest = dict(word=words[b], r=np.float32(1.2), f=np.float32(0.3), q=np.float32(0.1)) if ruled else {}
            k, toks, nodes, e = SA.walk(lambda u: lg[b, u], lambda s: gu[b, s], inv[b], int(top_k[b]), top_p[b], min_p[b],
                                        tree["tree_tokens"][b], par, n, cfg.max_depth, **rest)
            assert (int(acc["n_accepted"][b]), int(acc["n_emitted"][b])) == (k, e)
            assert acc["out_tokens"][b, :len(toks)].tolist() == toks and acc["out_nodes"][b, :k].tolist() == nodes
            if ruled:
                words[b] = RU.seen_add(words[b], toks[:e], False, False)
            assert int(st.attn_len[b]) == L[b] + k + 1
            now = positions_of(st, b, L[b] + k + 1)
            want = [np.concatenate([x[:L[b]], x[L[b]:][[0] + nodes]]) for x in after[b]]
            assert all(np.array_equal(x, y) for x, y in zip(now, want)), (step, b)
            tails[b], t_len[b] = CO.commit_tail(tails[b], t_len[b], toks)
            assert np.array_equal(st.ctx_tail[b].cpu().numpy(), tails[b])
    assert st.caches.status()["flags"] == 0


def test_a_step_of_the_8_bit_cache():
    """Turned rows, attention and commit over the 8-bit cache: the rows it commits are the turned ones."""
    cfg = config(3, 2)
    st = VerifyState.build(cfg, kv="int8", kv_headroom=64)
    st.use_rope(torch.as_tensor(INV, device="cuda"), projection(cfg, 6, 2))
    st.use_sampling(top_p=[0.9] * 6)
    tree = tree_to_np(st.draft())
    L = st.kv.ctx_len.tolist()
    st.write_tree()
    pos = np.array(L)[:, None] + tree["tree_depth"]
    live = np.arange(cfg.n_nodes)[None] < tree["n_nodes"][:, None]
    for got, x in ((st.q, st.projected[0]), (st.k_new, st.projected[1])):
        y, tol = turned(x.double().cpu().numpy(), 2.0 ** -20, np.where(live, pos, 0))
        assert (np.abs(got.double().cpu().numpy() - y) <= tol)[live].all()
    st.attention()
    st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda", boost="top", seed=1)
    st.gumbel = W.make_gumbel(cfg, 6, device="cuda", seed=2)
    acc = {k: x.cpu().numpy() for k, x in st.accept().items()}
    st.commit()
    for b in range(6):
        k = int(acc["n_accepted"][b])
        assert int(st.kv.ctx_len[b]) == L[b] + k + 1
        rows = [0] + acc["out_nodes"][b, :k].tolist()
        for j, r in enumerate(rows):
            p = L[b] + j
            if p >= int(st.kv.ctx_len[b]) // cfg.page * cfg.page:  # still in the tail
                assert torch.equal(st.kv.k_tail[b, :, p % cfg.page], st.k_new[b, r])


def test_steps_replayed_from_graphs_equal_the_eager_steps():
    """Turning, attention, walk, insertion and commit of one captured step, replayed four
    times with eager work between, for two batches whose attention shares one scratch."""
    pairs = []
    shared = None
    for n_prompts, each in ((20, 16), (2, 3)):
        cfg = config(n_prompts, each)
        states = [VerifyState.build(cfg, kv_headroom=64, prefix=[190] * n_prompts) for _ in range(2)]
        B = n_prompts * each
        if shared is None:
            shared = states[0].scratch  # (the larger one)
        states[0].scratch = shared
        for st in states:
            st.use_rope(torch.as_tensor(INV, device="cuda"), projection(cfg, B, 3))
            st.use_sampling([0.8] * B, [30] * B, [0.9] * B, [0.01] * B)
            tree = tree_to_np(st.draft())
            st.logits = W.make_logits(cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda", boost="top",
                                      seed=7)
            st.gumbel = W.make_gumbel(cfg, B, device="cuda", seed=8)
            st.accept()  # (allocates its outputs before the capture)
            st.attn_out.zero_()
        pairs.append(states)

    def step(st):
        st.write_tree()
        st.attention()
        st.accept()
        st.insert()
        st.commit()

    graphs = []
    torch.cuda.synchronize()
    for states in pairs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(states[0])
        graphs.append(g)
    for _ in range(4):
        for g, (a, b) in zip(graphs, pairs):
            g.replay()
            step(b)
            torch.randn(1 << 18, device="cuda").sum().item()
            for x, y in ((a.attn_out, b.attn_out), (a.acc["out_tokens"], b.acc["out_tokens"]), (a.attn_len, b.attn_len),
                         (a.k_cache, b.k_cache), (a.v_cache, b.v_cache), (a.ctx_tail, b.ctx_tail), (a.q, b.q)):
                assert torch.equal(x, y)

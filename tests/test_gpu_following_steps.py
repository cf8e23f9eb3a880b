"""Steps that follow one another: what changes between them reaches the next one, and
what does not stays."""
import numpy as np
import pytest
import torch

from oracle import commit as CO
from oracle import kv_quant as KQ
from oracle import sampling as SA
from paper_2601_09083_amd import srt
from paper_2601_09083_amd import workload as W
from paper_2601_09083_amd.pipeline import VerifyState
from tests.gpu_util import say, tree_to_np
from tests.test_gpu_group_step import INV, config, positions_of
from tests.test_gpu_quant_step import attention_tolerance, history

pytestmark = pytest.mark.gpu


def make_policy(st, step, sampled=True):
    tree = tree_to_np(st.tree)
    st.logits = W.make_logits(st.cfg, tree["tree_tokens"], tree["tree_parent"], tree["n_nodes"], device="cuda", boost="top",
                              seed=300 + step)
    st.gumbel = W.make_gumbel(st.cfg, st.tokens.batch, device="cuda", seed=400 + step) if sampled else None
    return tree


# --------------------------------------------------------------------------- a projection rewritten in place

class Projection:
    """Queries, keys and values of a step in buffers that every step rewrites: parts of one
    projection, packed, or (values only) heads that do not lie side by side."""

    def __init__(self, cfg, B, layout):
        N, hq, hkv, d = cfg.n_nodes, cfg.hq, cfg.hkv, cfg.head_dim
        new = lambda *s: torch.empty(s, dtype=torch.bfloat16, device="cuda")
        if layout == "fused":
            x = new(B, N, hq + 2 * hkv, d)
            self.parts = x[:, :, :hq], x[:, :, hq:hq + hkv], x[:, :, hq + hkv:]
        else:
            v = new(B, N, hkv, d) if layout == "packed" else new(B, hkv, N, d).transpose(1, 2)
            self.parts = new(B, N, hq, d), new(B, N, hkv, d), v

    def rewrite(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        for x in self.parts:
            x.copy_(torch.randn(x.shape, generator=g, device="cuda"))


@pytest.mark.parametrize("layout", ["fused", "packed", "scattered"])
@pytest.mark.parametrize("kv", ["int8", "e4m3"])
def test_values_of_each_step_over_the_8_bit_cache(kv, layout):
    """Attention and the committed keys and values of three steps, whose projection is rewritten in between."""
    cfg = config(3, 2).scaled(hkv=2)
    plain = VerifyState.build(cfg, kv_headroom=64)
    hist = [history(plain, b) for b in range(6)]
    st = VerifyState.build(cfg, kv=kv, kv_headroom=64)
    proj = Projection(cfg, 6, layout)
    proj.rewrite(1)
    st.use_rope(torch.as_tensor(INV, device="cuda"), proj.parts)
    for step in range(3):
        say(f"following steps: {kv} {layout} step {step}")
        proj.rewrite(10 + step)
        tree = tree_to_np(st.draft())
        st.write_tree()
        out, q = (x.double().cpu().numpy() for x in (st.attention(), st.q))
        make_policy(st, step)
        new = [x.float().cpu().numpy() for x in (st.k_new, proj.parts[2])]
        acc = {k: x.cpu().numpy() for k, x in st.accept().items()}
        st.commit()
        for b in range(6):
            n, L = int(tree["n_nodes"][b]), len(hist[b][0])
            K, V = (np.concatenate([KQ.context(hist[b][i], kv, cfg.page)[0], new[i][b, :n].astype(np.float64)]) for i in range(2))
            ref, tol = attention_tolerance(q[b], K, V, tree["tree_parent"][b], n, L, st.scale)
            assert (np.abs(out[b, :n] - ref) <= tol).all(), (step, b)
            rows = [0] + acc["out_nodes"][b, :int(acc["n_accepted"][b])].tolist()
            hist[b] = [np.concatenate([hist[b][i], new[i][b, rows]]) for i in range(2)]
        upto = max(len(x[0]) for x in hist)
        got = srt.srt_kv_read(st.kv, torch.zeros(6, dtype=torch.int32, device="cuda"), upto)
        for b in range(6):
            for i in range(2):
                want = torch.from_numpy(KQ.context(hist[b][i], kv, cfg.page)[0].astype(np.float32)).to(torch.bfloat16)
                assert torch.equal(got[i][b, :len(want)].cpu(), want), (step, b, "kv"[i])


@pytest.mark.parametrize("layout", ["fused", "scattered"])
def test_a_replayed_step_reads_the_projection_as_it_is(layout):
    cfg = config(3, 2).scaled(hkv=2)
    states, projs = [], []
    for _ in range(2):
        st, proj = VerifyState.build(cfg, kv="int8", kv_headroom=64), Projection(cfg, 6, layout)
        proj.rewrite(1)
        st.use_rope(torch.as_tensor(INV, device="cuda"), proj.parts)
        st.draft()
        make_policy(st, 0)
        st.accept()  # (allocates its outputs before the capture)
        st.attn_out.zero_()
        states.append(st)
        projs.append(proj)

    def step(st):
        st.write_tree()
        st.attention()
        st.accept()
        st.commit()

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(states[0])
    a, b = states
    before = None
    for i in range(4):
        for proj in projs:
            proj.rewrite(20 + i)
        g.replay()
        step(b)
        torch.randn(1 << 18, device="cuda").sum().item()
        assert torch.equal(b.v_new, projs[1].parts[2]) and (before is None or not torch.equal(b.v_new, before))
        before = b.v_new.clone()
        for x, y in ((a.attn_out, b.attn_out), (a.kv.ctx_len, b.kv.ctx_len), (a.kv.k_tail, b.kv.k_tail), (a.kv.v_tail, b.kv.v_tail),
                     (a.kv.k_pages, b.kv.k_pages), (a.kv.v_pages, b.kv.v_pages), (a.kv.v_scale, b.kv.v_scale)):
            assert torch.equal(x, y), i


# --------------------------------------------------------------------------- contexts that grow past the shared pages

def test_contexts_grow_past_the_pages_that_a_prompt_shares():
    """Prefixes beyond the shortest contexts share what those have whole pages of, then and later:
    steps until a group's shortest context has another whole page, then attention of its members."""
    cfg = config(20, 16)
    st = VerifyState.build(cfg, kv_headroom=160, prefix=[400] * 20)
    ids, page = st.tokens.seq_prompt, cfg.page
    of = lambda p: np.flatnonzero(ids == p)
    shared = [min(400, int(st.tokens.ctx_len[of(p)].min())) // page for p in range(20)]
    assert min(shared) < 400 // page
    for p in range(20):
        assert (st.block_table[of(p), :shared[p]] == st.block_table[of(p)[0], :shared[p]]).all()
        assert (st.block_table[of(p)[1:], shared[p]] != st.block_table[of(p)[0], shared[p]]).all()
    checked = set()
    for step in range(3 * page):
        st.draft()
        now = st.attn_len.cpu().numpy()
        grown = [p for p in range(20) if min(400, int(now[of(p)].min())) // page > shared[p] and p not in checked]
        if grown:
            tree, out, q = tree_to_np(st.tree), st.attention().double().cpu().numpy(), st.q.double().cpu().numpy()
            p = grown[0]
            checked.add(p)
            say(f"following steps: prompt {p} after {step} steps: {shared[p]} pages shared, contexts {now[of(p)].tolist()}")
            for b in of(p):
                n, L = int(tree["n_nodes"][b]), int(now[b])
                ref, tol = attention_tolerance(q[b], *positions_of(st, b, L + n), tree["tree_parent"][b], n, L, st.scale)
                assert (np.abs(out[b, :n] - ref) <= tol).all(), (step, b)
        if len(checked) == 2:
            break
        make_policy(st, step)
        st.accept()
        st.insert()
        st.commit()
    assert len(checked) == 2


# --------------------------------------------------------------------------- walks that end without a token

@pytest.mark.parametrize("kv", ["bf16", "int8"])
def test_sequences_that_end_without_rules_stay_as_they_are(kv):
    """Sequence 1 finds nothing to choose at its root in step 1 (a constraint that the caller has put
    into the logits), sequence 2 NaN at its root in step 2; they emit and commit no more, 0 and 3 go on."""
    cfg = W.CONFIGS["tiny"]
    st = VerifyState.build(cfg, kv=kv, kv_headroom=128)
    B, cuts = 4, (np.float32(1.0), 50, np.float32(0.9), np.float32(0.0))
    st.use_sampling(top_k=[50] * B, top_p=[0.9] * B)
    tails, t_len, ctx = st.ctx_tail.cpu().numpy(), st.draft_len.tolist(), st.attn_len.tolist()
    ended = [False] * B
    for step in range(6):
        st.draft()
        st.attention()
        tree = make_policy(st, step)
        if step >= 1:
            st.logits[1, 0] = -float("inf") if step == 1 else 0.5  # (what it would choose afterwards does not matter)
        if step == 2:
            st.logits[2, 0] = float("nan")
        acc = {k: x.cpu().numpy() for k, x in st.accept().items()}
        st.insert()
        st.commit()
        lg, gu = st.logits.cpu().numpy(), st.gumbel.cpu().numpy()
        for b in range(B):
            if ended[b]:
                assert (int(acc["n_accepted"][b]), int(acc["n_emitted"][b])) == (0, 0)
                assert (acc["out_tokens"][b] == -1).all() and (acc["out_nodes"][b] == -1).all()
                continue
            k, toks, nodes, e = SA.walk(lambda u: lg[b, u], lambda s: gu[b, s], *cuts, tree["tree_tokens"][b], tree["tree_parent"][b],
                                        int(tree["n_nodes"][b]), cfg.max_depth)
            assert acc["out_tokens"][b, :len(toks)].tolist() == toks and int(acc["n_emitted"][b]) == e
            tails[b], t_len[b] = CO.commit_tail(tails[b], t_len[b], toks[:e])
            ctx[b] += k + 1
            ended[b] = e == k
        assert st.ended.tolist() == ended
        assert st.attn_len.tolist() == ctx, step
        assert np.array_equal(st.ctx_tail.cpu().numpy(), tails) and st.draft_len.tolist() == t_len
    assert ended == [False, True, True, False]


def test_sampling_given_anew_leaves_ended_sequences_ended():
    st = VerifyState.build(W.CONFIGS["tiny"], kv_headroom=64)
    st.use_sampling(top_p=[0.9] * 4)
    st.draft()
    make_policy(st, 0)
    st.logits[3] = -float("inf")
    st.accept()
    st.commit()
    st.use_sampling(top_p=[0.5] * 4)
    assert st.ended.tolist() == [False, False, False, True]


# --------------------------------------------------------------------------- the step's temperature

@pytest.mark.parametrize("ruled", [False, True])
def test_the_steps_temperature_where_sampling_has_none(ruled):
    """It is every sequence's; temperatures of the sequences' own take its place."""
    cfg = W.CONFIGS["tiny"]
    st = VerifyState.build(cfg, kv_headroom=64)
    if ruled:
        st.use_rules([1.2] * 4, [0.3] * 4, [0.1] * 4)
    st.draft()
    tree = make_policy(st, 0)
    lg, gu = st.logits.cpu().numpy(), st.gumbel.cpu().numpy()
    rest = lambda b: dict(word=st.seen[b].cpu().numpy().view(np.uint16), r=np.float32(1.2), f=np.float32(0.3),
                          q=np.float32(0.1)) if ruled else {}
    results = []
    for own, given in ((None, 1.0), (None, 0.3), (None, 4), ([0.3, 0.5, 4.0, 1.0], 2.0), ([0.3] * 4, 1.0)):
        st.use_sampling(own, top_k=[200] * 4, min_p=[1e-4] * 4)
        acc = {k: x.cpu().numpy() for k, x in (st.accept(given) if given != 1.0 else st.accept()).items()}
        for b in range(4):
            t = np.float32(given if own is None else own[b])
            k, toks, nodes, e = SA.walk(lambda u: lg[b, u], lambda s: gu[b, s], t, 200, np.float32(1), np.float32(1e-4),
                                        tree["tree_tokens"][b], tree["tree_parent"][b], int(tree["n_nodes"][b]), cfg.max_depth, **rest(b))
            assert acc["out_tokens"][b, :len(toks)].tolist() == toks and int(acc["n_accepted"][b]) == k, (own, given, b)
        results.append(acc["out_tokens"].copy())
    assert not np.array_equal(results[0], results[1]) and np.array_equal(results[1], results[4])


def test_the_steps_temperature_in_a_graph():
    """A captured step keeps its temperature, whatever eager steps are given in between."""
    st = VerifyState.build(W.CONFIGS["tiny"], kv_headroom=64)
    st.use_sampling(top_k=[500] * 4)
    st.draft()
    make_policy(st, 0)
    want = {t: st.accept(t)["out_tokens"].clone() for t in (1.0, 0.2, 5.0)}
    assert not torch.equal(want[0.2], want[5.0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        st.accept(0.2)
    for t in (5.0, 1.0, 5.0):
        assert torch.equal(st.accept(t)["out_tokens"], want[t])
        g.replay()
        torch.randn(1 << 18, device="cuda").sum().item()
        assert torch.equal(st.acc["out_tokens"], want[0.2])


def test_a_temperature_that_is_not_a_number_is_refused():
    st = VerifyState.build(W.CONFIGS["tiny"])
    st.use_sampling(top_k=[5] * 4)
    st.draft()
    make_policy(st, 0)
    with pytest.raises(ValueError):
        st.accept(float("nan"))

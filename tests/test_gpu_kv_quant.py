"""The 8-bit KV cache on the GPU against its oracle: codes, scales, tails and
read-back bit for bit; attention within the tolerance that quant_util derives."""
import numpy as np
import pytest
import torch

from oracle import commit as CO
from oracle import kv_quant as KQ
from paper_2601_09083_amd import srt
from tests.quant_util import DTYPE, AttnCase, bf16, new_cache

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


# --------------------------------------------------------------------------- append, read

def vectors(rng, *shape):
    """bf16 values with outlier channels, as float32."""
    return bf16(rng.normal(0, 1, shape) * np.exp(rng.normal(0, 1, shape[-1]))).float().numpy()


def check_cache(c, kv, hist, b):
    """Cache of sequence b against the oracle's for its history (K, V) [L, Hkv, d]."""
    page, L = c.page, int(c.ctx_len[b])
    assert L == len(hist[0])
    pg = c.block_table[b, : L // page].long()
    for i, (pages, scale, tail) in enumerate(((c.k_pages, c.k_scale, c.k_tail), (c.v_pages, c.v_scale, c.v_tail))):
        vals, codes, scales = KQ.context(hist[i], kv, page)
        got = pages.view(torch.uint8)[pg].cpu().numpy()
        assert np.array_equal(got, codes.view(np.uint8)), f"codes of sequence {b}, tensor {i}"
        assert np.array_equal(scale[pg].cpu().numpy(), scales)
        rest = tail[b, :, : L % page].float().cpu().numpy().transpose(1, 0, 2)
        assert np.array_equal(rest, hist[i][L // page * page:])


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("d,hkv,page", [(64, 1, 16), (128, 2, 16), (128, 5, 32), (64, 3, 64), (128, 1, 128), (64, 2, 256)])
def test_append_in_many_pieces(kv, d, hkv, page):
    """Prompts, single tokens, short and long pieces: the cache is the oracle's
    after each, whatever the pieces were."""
    rng = np.random.default_rng(page + d)
    B, mp = 5, 6 * 64 // page + 3
    c = new_cache(B, hkv, page, d, kv, mp, "cuda", seed=page)
    hist = [[np.zeros((0, hkv, d), np.float32)] * 2 for _ in range(B)]
    for T, counts in ((100, [100, 0, 7, 64, 33]), (1, [1, 1, 0, 1, 1]), (64, [64, 3, 64, 0, 15]), (65, [1, 65, 40, 65, 2]),
                      (7, [-3, 9, 7, 2, 5]), (1, [1] * B), (1, [1] * B)):
        k, v = vectors(rng, B, T, hkv, d), vectors(rng, B, T, hkv, d)
        srt.srt_kv_append(c, bf16(k).cuda(), bf16(v).cuda(), i32(counts))
        for b in range(B):
            m = min(max(counts[b], 0), T)
            hist[b] = [np.concatenate([h, x[b, :m]]) for h, x in zip(hist[b], (k, v))]
            check_cache(c, kv, hist[b], b)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_rounding_ties_zeros_and_tiny_values(kv):
    """Values on the borders between codes, zero pages, pages below the least amplitude."""
    d, page = 64, 16
    c = new_cache(1, 1, page, d, kv, 4, "cuda")
    pos = KQ.e4m3_values()[:127]
    borders = np.concatenate([pos, (pos[1:] + pos[:-1]) / 2, -pos, np.arange(-127, 128) + 0.5, np.arange(-127, 128)])
    x = np.zeros((4 * page, 1, d), np.float32)
    x[:page].reshape(-1)[:] = np.resize(borders, page * d)
    x[:page].reshape(-1)[0] = KQ.TOP[kv]
    x[2 * page:3 * page] = np.float32(2.0 ** -70)
    x[3 * page:, :, ::3] = np.float32(2.0 ** 120)
    x = bf16(x).float().numpy()
    srt.srt_kv_append(c, bf16(x[None]).cuda(), bf16(-x[None]).cuda(), i32([4 * page]))
    check_cache(c, kv, [x, -x], 0)  # (-0 keeps its sign)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32)])
def test_read(kv, d, page):
    """bf16 of code * scale and of the tail; rows outside the context are left alone."""
    rng = np.random.default_rng(5)
    B, hkv, T = 4, 3, 70
    c = new_cache(B, hkv, page, d, kv, 8, "cuda")
    k, v = vectors(rng, B, 100, hkv, d), vectors(rng, B, 100, hkv, d)
    counts = [100, 37, 0, 64]
    srt.srt_kv_append(c, bf16(k).cuda(), bf16(v).cuda(), i32(counts))
    start = [30, 0, 0, -5]
    out = [torch.full((B, T, hkv, d), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    srt.srt_kv_read(c, i32(start), T, out=out)
    for b in range(B):
        for i, x in enumerate((k, v)):
            _, codes, scales = KQ.context(x[b, :counts[b]], kv, page)
            got = out[i][b].float().cpu().numpy()
            for t in range(T):
                p = start[b] + t
                if p < 0 or p >= counts[b]:
                    want = np.full((hkv, d), 7.0)
                elif p >= counts[b] // page * page:
                    want = x[b, p]
                else:
                    val = KQ.values(codes[p // page, :, p % page], kv).astype(np.float32)
                    want = bf16(val * scales[p // page][:, None]).float().numpy()
                assert np.array_equal(got[t], want), (b, i, t)
    zero = srt.srt_kv_read(c, i32(start), T)
    assert torch.equal(zero[0][2], torch.zeros_like(zero[0][2]))


@pytest.mark.parametrize("T", [40, 300])
def test_append_stops_at_capacity_and_skips_bad_pages(T):
    """Tokens past the table's room are dropped, pages outside the pool not written."""
    rng = np.random.default_rng(6)
    B, hkv, d, page, mp = 3, 2, 64, 16, 2
    c = new_cache(B, hkv, page, d, "int8", mp, "cuda")
    c.block_table[1, 0] = -1
    c.block_table[1, 1] = 10 ** 6
    before = [x.clone() for x in (c.k_pages, c.v_pages, c.k_scale)]
    c.ctx_len.copy_(i32([0, 0, 10 ** 9]))
    k = vectors(rng, B, T, hkv, d)
    srt.srt_kv_append(c, bf16(k).cuda(), bf16(k).cuda(), i32([T] * B))
    cap = (mp + 1) * page - 1
    assert c.ctx_len.tolist() == [min(T, cap)] * 2 + [cap]
    check_cache(c, "int8", [k[0][:min(T, cap)]] * 2, 0)
    mine = set(c.block_table[0].tolist())
    for x, y in zip(before, (c.k_pages, c.v_pages, c.k_scale)):
        keep = [i for i in range(len(x)) if i not in mine]
        assert torch.equal(x[keep], y[keep])


def test_append_reads_a_fused_projection_in_place():
    rng = np.random.default_rng(7)
    B, T, hq, hkv, d = 3, 40, 4, 2, 128
    for T in (40, 90):
        c = new_cache(B, hkv, 16, d, "e4m3", 8, "cuda")
        qkv = vectors(rng, B, T, hq + 2 * hkv, d)
        x = bf16(qkv).cuda()
        srt.srt_kv_append(c, x[:, :, hq:hq + hkv], x[:, :, hq + hkv:], i32([T, 5, 20]))
        for b, m in enumerate([T, 5, 20]):
            check_cache(c, "e4m3", [qkv[b, :m, hq:hq + hkv], qkv[b, :m, hq + hkv:]], b)


# --------------------------------------------------------------------------- commit

@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("d,hkv,page,N,dmax", [(64, 1, 16, 8, 4), (128, 4, 16, 64, 12), (128, 5, 32, 256, 63), (64, 2, 64, 1, 3)])
def test_commit_appends_the_accepted_path(kv, d, hkv, page, N, dmax):
    rng = np.random.default_rng(N)
    B, qmax = 6, 8
    c = new_cache(B, hkv, page, d, kv, 400 // page + 1, "cuda")
    k, v = vectors(rng, B, 60, hkv, d), vectors(rng, B, 60, hkv, d)
    start = [0, 1, 15, 16, 31, 60]
    srt.srt_kv_append(c, bf16(k).cuda(), bf16(v).cuda(), i32(start))
    hist = [[x[b, :start[b]] for x in (k, v)] for b in range(B)]
    tails = np.full((B, qmax), -1, np.int32)
    for b in range(B):
        h = min(start[b], qmax)
        tails[b, qmax - h:] = rng.integers(0, 1000, h)
    t_dev, len_dev = i32(tails), i32(start)
    for step in range(4):
        kn, vn = vectors(rng, B, N, hkv, d), vectors(rng, B, N, hkv, d)
        acc = rng.integers(0, min(dmax, N - 1) + 1, B)
        acc[step % B] = min(dmax, N - 1)
        nodes = np.full((B, dmax + 1), -1, np.int32)
        toks = np.full((B, dmax + 1), -1, np.int32)
        for b in range(B):
            nodes[b, :acc[b]] = np.sort(rng.choice(np.arange(1, N), acc[b], replace=False)) if acc[b] else []
            toks[b, :acc[b] + 1] = rng.integers(0, 1000, acc[b] + 1)
        srt.srt_commit_quant(c, bf16(kn).cuda(), bf16(vn).cuda(), i32(acc), i32(toks), i32(nodes), ctx_tail=t_dev,
                             draft_len=len_dev)
        for b in range(B):
            rows = [0] + nodes[b, :acc[b]].tolist()
            hist[b] = [np.concatenate([h, x[b, rows]]) for h, x in zip(hist[b], (kn, vn))]
            check_cache(c, kv, hist[b], b)
            tails[b], start[b] = CO.commit_tail(tails[b], start[b], toks[b, :acc[b] + 1])
        assert np.array_equal(t_dev.cpu().numpy(), tails) and len_dev.tolist() == start


def test_commit_clamps_what_the_walk_cannot_return():
    """Counts and node indices out of range stay in bounds; without draft inputs too."""
    c = new_cache(3, 1, 16, 64, "e4m3", 4, "cuda")
    x = bf16(np.random.default_rng(8).normal(0, 1, (3, 4, 1, 64))).cuda()
    nodes = i32([[99, -7, 2, 3], [1, 2, 3, 3], [-1] * 4])
    srt.srt_commit_quant(c, x, x, i32([2, 50, -9]), i32(np.zeros((3, 4))), nodes)
    assert c.ctx_len.tolist() == [3, 4, 1]
    assert torch.equal(c.k_tail[0, 0, :3], x[0, [0, 3, 0], 0]) and torch.equal(c.k_tail[1, 0, :4], x[1, [0, 1, 2, 3], 0])


# --------------------------------------------------------------------------- attention

@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("d,hq,hkv,page", [(128, 28, 4, 16), (64, 4, 1, 16), (128, 8, 8, 32), (64, 14, 2, 64), (128, 5, 1, 256)])
def test_attention_ragged(kv, d, hq, hkv, page):
    ctx = [0, 1, 15, 16, 17, 63, 64, 65, 200, 1000, 3001]
    c = AttnCase(1, len(ctx), 32, hq, hkv, d, ctx, kv, page)
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
def test_attention_rows_of_every_arrangement(kv, d):
    """1 to 448 query rows per KV head: each arrangement of the waves, on both sides of its border, with splits."""
    n = [1, 4, 5, 9, 10, 18, 19, 36, 37, 64, 2, 41]  # x 7 heads: 7, 28, 35, 63, 70, 126, 133, 252, 259, 448
    ctx = [2999, 16, 1030, 2048, 130, 511, 700, 33, 2500, 1, 1024, 3000]
    c = AttnCase(2, len(n), 64, 7, 1, d, ctx, kv, n_nodes=n)
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_attention_single_tokens_of_a_large_batch(kv):
    rng = np.random.default_rng(3)
    ctx = rng.integers(0, 2500, 150)
    c = AttnCase(3, 150, 1, 12, 2, 128, ctx, kv)
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


def test_attention_wide_trees_and_long_contexts():
    c = AttnCase(4, 3, 256, 28, 4, 128, [9000, 5, 20011], "e4m3", n_nodes=[256, 200, 129])
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_attention_splits_that_end_inside_a_tree(kv):
    """Rows that see nothing of the last split: 256-, 1024- and 2048-key splits
    that end among the tree's keys, in its tail, or just before either."""
    for B, ctx in ((3, [1014, 1023, 1008]), (2, [250, 1270]), (24, [2040 - i for i in range(24)])):
        c = AttnCase(14 + B, B, 64, 14, 2, 64, ctx, kv, n_nodes=[64] * B, max_pages=max(ctx) // 16 + 4)
        c.check(c.run(), what=f"{B} sequences")


def test_attention_takes_a_smaller_scratch():
    """A scratch for larger splits only serves; one that is too small is replaced."""
    c = AttnCase(15, 2, 4, 7, 1, 128, [900, 300])
    need = srt.srt_tree_attn_quant_scratch_bytes(c.cache, c.N, c.hq)
    for size in (need, need - 256, need // 2, 256):
        c.check(c.run(scratch=torch.empty(size, dtype=torch.uint8, device="cuda")), what=f"scratch of {size}")


def test_attention_large_splits():
    # 8192-key splits: 256 sequence-head pairs with 16k of room
    base = [8192 - 64 - 7, 8192, 9000, 12345, 16354, 100, 5000, 8193]
    c = AttnCase(5, 32, 4, 8, 8, 128, [base[i % 8] for i in range(32)], "int8")
    print(f"tolerance used: {c.check(c.run(), seqs=range(0, 32, 3)):.3f}", flush=True)


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("B,N,hq,hkv,d,page,longest", [
    (70, 4, 28, 4, 128, 16, 300),   # 28 rows, short table
    (40, 32, 8, 8, 64, 32, 700),    # 32 rows, as many nodes
    (261, 1, 32, 1, 64, 128, 900),  # 32 heads of one node
    (300, 2, 10, 2, 128, 16, 2400),  # a longer table
    (290, 3, 8, 8, 64, 64, 40),     # 2320 (sequence, KV head) pairs, few keys
])
def test_attention_large_batches_of_narrow_trees(kv, B, N, hq, hkv, d, page, longest):
    """Up to 32 query rows per KV head in more items than the GPU has CUs."""
    rng = np.random.default_rng(16)
    ctx = np.where(np.arange(B) % 7 == 0, np.arange(B) % 40, rng.integers(0, longest, B))
    c = AttnCase(16, B, N, hq, hkv, d, ctx, kv, page)
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


def test_attention_of_narrow_trees_takes_a_smaller_scratch():
    """8192-key splits where the scratch has no room for the partial results of 4096-key ones."""
    base = [8192 - 64 - 7, 8192, 9000, 12345, 16354, 100, 5000, 8193, 4096, 0]
    c = AttnCase(17, 40, 4, 8, 8, 128, [base[i % 10] for i in range(40)])
    need = srt.srt_tree_attn_quant_scratch_bytes(c.cache, c.N, c.hq)
    for size in (need, need * 6 // 10):
        out = c.run(scratch=torch.empty(size, dtype=torch.uint8, device="cuda"))
        c.check(out, seqs=range(0, 40, 3), what=f"scratch of {size}")


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
@pytest.mark.parametrize("B,N,hq,hkv,d,page,longest", [
    (260, 16, 28, 4, 128, 16, 300),   # up to 112 rows, short table
    (132, 128, 8, 8, 64, 32, 200),    # up to 128, as many nodes
    (520, 9, 10, 2, 128, 64, 2000),   # up to 45, a longer table
    (130, 8, 64, 8, 64, 16, 4500),    # up to 64, two splits
])
def test_attention_many_pairs_of_medium_trees(kv, B, N, hq, hkv, d, page, longest):
    """33 to 128 query rows per KV head, 1024 (sequence, KV head) pairs and more."""
    rng = np.random.default_rng(18)
    ctx = np.where(np.arange(B) % 7 == 0, np.arange(B) % 40, rng.integers(0, longest, B))
    c = AttnCase(18, B, N, hq, hkv, d, ctx, kv, page)
    print(f"tolerance used: {c.check(c.run(), seqs=range(0, B, 5)):.3f}", flush=True)
    need = srt.srt_tree_attn_quant_scratch_bytes(c.cache, c.N, c.hq)
    out = c.run(scratch=torch.empty(need * 6 // 10, dtype=torch.uint8, device="cuda"))  # larger splits, where it serves
    c.check(out, seqs=range(0, B, 11), what="smaller scratch")


@pytest.mark.parametrize("kv", ["e4m3", "int8"])
def test_attention_peaked(kv):
    """Scores of large magnitude: the reference is raised again and again."""
    c = AttnCase(6, 4, 16, 7, 1, 128, [300, 1500, 40, 2100], kv, qk=3.0)
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


def test_attention_scales_far_apart():
    """Pages whose V scales differ by 2^80 and all-zero pages: the sum of the probabilities keeps them all."""
    c = AttnCase(7, 2, 4, 7, 1, 64, [1600, 333], "e4m3")
    h = c.host
    for b in range(2):
        for j in range(c.ctx[b] // 16):
            s = (2.0 ** -60 / 448, 1.0, 2.0 ** 12)[j % 3]
            h["scales"][1][h["bt"][b, j]] = s
            if j % 3 == 0:
                h["codes"][1][h["bt"][b, j]] = 0
    c.cache.v_scale.copy_(h["scales"][1])
    c.cache.v_pages.view(torch.uint8).copy_(h["codes"][1])
    print(f"tolerance used: {c.check(c.run()):.3f}", flush=True)


def test_attention_leaves_other_rows_alone_and_clamps():
    """Rows behind a tree's last node keep their contents; counts and lengths out
    of range and pages outside the pool are clamped or read as zero."""
    c = AttnCase(8, 3, 8, 4, 2, 64, [100, 40, 0], "e4m3", n_nodes=[3, 8, 1])
    out = torch.full_like(c.q, 5.0)
    c.run(out=out)
    c.check(out)
    for b in range(3):
        assert (out[b, int(c.n_nodes[b]):] == 5.0).all()
    # a page outside the pool reads as zero keys and values
    pages = c.cache.block_table[0, 2].clone()
    c.cache.block_table[0, 2] = 10 ** 8
    h = c.host
    bad = c.run()
    for i in range(2):
        h["codes"][i][int(pages)] = 0
        h["scales"][i][int(pages)] = 1.0
    c.check(bad, seqs=[0])
    c.cache.block_table[0, 2] = pages
    # n_nodes and ctx_len out of range
    c.n_dev.copy_(i32([0, 99, 1]))
    c.cache.ctx_len.copy_(i32([-4, 40, 0]))
    o = c.run()
    c.ctx[0], c.n_nodes[0] = 0, 1
    c.check(o, seqs=[0, 1])
    c.cache.ctx_len.copy_(i32([100, 10 ** 9, 0]))
    c.cache.k_tail.zero_(), c.cache.v_tail.zero_()
    c.run()
    torch.cuda.synchronize()


def test_attention_reads_a_fused_projection_in_place():
    c = AttnCase(9, 3, 16, 8, 2, 128, [100, 40, 500])
    qkv = torch.cat([c.q, c.new[0], c.new[1]], 2)
    got = srt.srt_tree_attn_quant(c.q, c.cache, qkv[:, :, 8:10], qkv[:, :, 10:], c.par_dev, c.n_dev, c.scale)
    for b in range(3):
        n = int(c.n_nodes[b])
        assert torch.equal(got[b, :n], c.run()[b, :n])
    c.check(got)


def test_attention_on_a_side_stream_and_from_a_graph():
    """Two captured graphs with workspaces of their own, replayed in turn with
    eager work between: every replay equals the eager result."""
    cases = [AttnCase(10, 6, 8, 7, 1, 128, [900, 100, 33, 2000, 0, 64]), AttnCase(11, 40, 2, 8, 8, 64, list(range(7, 2007, 50)), "int8")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    eager = [c.run() for c in cases]
    torch.cuda.synchronize()
    live = lambda c, x: torch.cat([x[b, :int(c.n_nodes[b])].flatten() for b in range(c.B)])
    for c, e in zip(cases, eager):
        got = c.run(stream=side)
        side.synchronize()
        assert torch.equal(live(c, got), live(c, e))
    graphs, outs = [], []
    for c in cases:
        out = torch.zeros_like(c.q)
        scratch = torch.empty(srt.srt_tree_attn_quant_scratch_bytes(c.cache, c.N, c.hq), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run(out=out, scratch=scratch)
        graphs.append((g, scratch))
        outs.append(out)
    for _ in range(3):
        for (g, _s), c, out, e in zip(graphs, cases, outs, eager):
            out.zero_()
            g.replay()
            other = torch.randn(1 << 20, device="cuda").sum()
            torch.cuda.synchronize()
            assert torch.equal(live(c, out), live(c, e)) and torch.isfinite(other)


def test_a_growing_sequence_equals_the_cache_built_at_once():
    """Decode loop in miniature: attention, commit, attention .. against a cache
    into which the same tokens were appended in one piece: the same bits."""
    rng = np.random.default_rng(12)
    B, N, hq, hkv, d, page = 3, 6, 4, 2, 64, 16
    for kv in ("e4m3", "int8"):
        c = new_cache(B, hkv, page, d, kv, 12, "cuda")
        k, v = vectors(rng, B, 50, hkv, d), vectors(rng, B, 50, hkv, d)
        m = [50, 13, 0]
        srt.srt_kv_append(c, bf16(k).cuda(), bf16(v).cuda(), i32(m))
        hist = [[x[b, :m[b]] for x in (k, v)] for b in range(B)]
        par = i32([[-1, 0, 1, 2, 0, 4]] * B)
        for step in range(8):
            kn, vn, q = vectors(rng, B, N, hkv, d), vectors(rng, B, N, hkv, d), bf16(rng.normal(0, 1, (B, N, hq, d))).cuda()
            got = srt.srt_tree_attn_quant(q, c, bf16(kn).cuda(), bf16(vn).cuda(), par, i32([N] * B), d ** -0.5)
            once = new_cache(B, hkv, page, d, kv, 12, "cuda", seed=99)
            L = max(len(h[0]) for h in hist)
            full = [np.zeros((B, max(L, 1), hkv, d), np.float32) for _ in range(2)]
            for b in range(B):
                for i in range(2):
                    full[i][b, :len(hist[b][i])] = hist[b][i]
            srt.srt_kv_append(once, bf16(full[0]).cuda(), bf16(full[1]).cuda(), i32([len(h[0]) for h in hist]))
            want = srt.srt_tree_attn_quant(q, once, bf16(kn).cuda(), bf16(vn).cuda(), par, i32([N] * B), d ** -0.5)
            assert torch.equal(got, want)
            acc = rng.integers(0, 4, B)
            nodes = np.tile(np.array([1, 2, 3, -1], np.int32), (B, 1))
            srt.srt_commit_quant(c, bf16(kn).cuda(), bf16(vn).cuda(), i32(acc), i32(np.zeros((B, 4))), i32(nodes))
            for b in range(B):
                rows = [0, 1, 2, 3][:acc[b] + 1]
                hist[b] = [np.concatenate([h, x[b, rows]]) for h, x in zip(hist[b], (kn, vn))]


def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB whose far pages are used."""
    hkv, page, d = 8, 256, 128
    P = (5 << 30) // (hkv * page * d)
    pages = [torch.zeros((P, hkv, page, d), dtype=torch.int8, device="cuda") for _ in range(2)]
    scale = [torch.zeros((P, hkv), device="cuda") for _ in range(2)]
    tail = [torch.zeros((1, hkv, page, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    bt = i32([[P - 1, P - 2, 3]])
    c = srt.KvQuant(*pages, *scale, *tail, bt, i32([0]))
    rng = np.random.default_rng(13)
    k, v = vectors(rng, 1, 700, hkv, d), vectors(rng, 1, 700, hkv, d)
    srt.srt_kv_append(c, bf16(k).cuda(), bf16(v).cuda(), i32([700]))
    check_cache(c, "int8", [k[0], v[0]], 0)
    got = srt.srt_kv_read(c, i32([0]), 700)
    want, _, _ = KQ.context(k[0], "int8", page)
    assert np.abs(got[0][0].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max()
    q = bf16(rng.normal(0, 1, (1, 1, 8, d))).cuda()
    kn = bf16(vectors(rng, 1, 1, hkv, d)).cuda()
    a = srt.srt_tree_attn_quant(q, c, kn, kn, i32([[-1]]), i32([1]), d ** -0.5)
    near = new_cache(1, hkv, page, d, "int8", 3, "cuda")
    srt.srt_kv_append(near, bf16(k).cuda(), bf16(v).cuda(), i32([700]))
    assert torch.equal(a, srt.srt_tree_attn_quant(q, near, kn, kn, i32([[-1]]), i32([1]), d ** -0.5))


@pytest.mark.parametrize("kv,d,page", [("e4m3", 128, 16), ("int8", 128, 32), ("e4m3", 64, 64), ("int8", 64, 128)])
def test_calls_that_stream_equal_small_ones(kv, d, page):
    """128 MiB of rows and more are written and read non-temporally: the same bits
    as in pieces, and a sample of them as the oracle's."""
    B, T, hkv = 4, 8192 + 40, 1024 // d
    g = torch.Generator(device="cuda").manual_seed(d + page)
    k, v = (torch.randn((B, T, hkv, d), generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    counts = [T, T - 7, 0, 5000]
    big, small = (new_cache(B, hkv, page, d, kv, T // page + 1, "cuda", seed=3) for _ in range(2))
    srt.srt_kv_append(big, k, v, i32(counts))
    for t0 in range(0, T, 2000):
        part = [x[:, t0:t0 + 2000].contiguous() for x in (k, v)]
        srt.srt_kv_append(small, *part, i32(np.clip(np.array(counts) - t0, 0, part[0].shape[1])))
    for x, y in zip(big.tensors[:4] + (big.ctx_len,), small.tensors[:4] + (small.ctx_len,)):
        same = (lambda z: z.view(torch.uint8)) if x.element_size() == 1 else (lambda z: z)
        assert torch.equal(same(x), same(y))
    zero = i32([0] * B)
    whole = srt.srt_kv_read(big, zero, T)  # (tails among them; their rows behind the context hold anything)
    for x, y in zip(whole, srt.srt_kv_read(small, zero, T)):
        assert torch.equal(x, y)
    for t0 in range(0, T, 2000):
        part = srt.srt_kv_read(big, i32([t0] * B), min(2000, T - t0))
        for x, y in zip(whole, part):
            assert torch.equal(x[:, t0:t0 + 2000], y)
    want, _, _ = KQ.context(k[1, :3 * page + 1].float().cpu().numpy(), kv, page)
    assert torch.equal(whole[0][1, :3 * page].cpu(), bf16(want[:3 * page]))

"""Attention of groups of sequences that share a prefix's pages, against the fp64
oracle, and against srt_tree_attn on the same cache.

Tolerance, as for any attention on bf16 probabilities: probabilities are rounded
half a step (2^-8) each, the same ones in numerator and sum, so the output moves by
at most 2^-8 (A + |out|) with A = sum p |v| / sum p; its own rounding 2^-8 |out|;
a score is off by e = (d + 16) 2^-24 sum |q k| scale (fp32 sums; the other
operations count as 16), which moves the output by at most 2 e A on either side of
the maximum it is taken from; fp32 sums over keys and the join of the parts,
(keys + 64) 2^-24 A."""
import numpy as np
import pytest
import torch

from oracle import attention as AT
from paper_2601_09083_amd import srt

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x), dtype=torch.int32, device="cuda")


def room(pairs):
    """Positions of a block table at which srt_tree_attn would not give each of the
    batch's items (1024 keys of a (sequence, KV head) pair) a CU of its own, so that the
    call takes its own way whatever the number of pairs."""
    return 0 if pairs > 256 else 1024 * (300 // pairs + 1)


class Case:
    """Groups of given sizes and prefixes; own[b] keys behind the prefix.  Pages
    that no call may read hold NaN."""

    def __init__(self, seed, groups, prefix, own, N, hq, hkv, d, page=16, n=None, shuffle=True, alone=0, amp=1.0, spare=0):
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda").manual_seed(seed)
        ids = np.repeat(np.arange(len(groups)), groups)
        ids = np.concatenate([ids, [-1, len(groups)][: min(alone, 2)] * ((alone + 1) // 2)])[: sum(groups) + alone].astype(np.int64)
        if shuffle:
            ids = rng.permutation(ids)
        B = len(ids)
        self.N, self.hq, self.hkv, self.d, self.page, self.B = N, hq, hkv, d, page, B
        self.ids, self.prefix = ids, np.asarray(prefix, dtype=np.int64)
        in_group = (ids >= 0) & (ids < len(groups))
        P = np.where(in_group, self.prefix[np.clip(ids, 0, len(groups) - 1)], 0)
        own = rng.integers(own[0], own[1] + 1, B) if isinstance(own, tuple) else np.asarray(own)
        self.L = P + own
        self.n = rng.integers(1, N + 1, B) if n is None else np.broadcast_to(np.asarray(n), (B,)).copy()
        whole, need = P // page, (self.L + self.n + page - 1) // page
        total = int((self.prefix // page).sum() + (need - whole).sum()) + 3
        order, at, heads = rng.permutation(total), 0, []
        for p in self.prefix // page:
            heads.append(order[at:at + p])
            at += p
        self.bt = np.full((B, max(int(need.max()) + spare, room(B * hkv) // page)), -1, dtype=np.int32)
        for b in range(B):
            w, m = int(whole[b]), int(need[b])
            if w:
                self.bt[b, :w] = heads[ids[b]]
            self.bt[b, w:m] = order[at:at + m - w]
            at += m - w
        self.used = order[:at]
        self.par = np.full((B, N), -1)
        for b in range(B):
            for i in range(1, self.n[b]):
                self.par[b, i] = rng.integers(max(0, i - 6), i) if rng.random() < 0.8 else rng.integers(0, i)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.q = (r(B, N, hq, d) * amp).to(torch.bfloat16)
        self.cache = [(r(total, hkv, page, d) * a).to(torch.bfloat16) for a in (amp, 1.0)]
        free = torch.as_tensor(np.setdiff1d(np.arange(total), self.used), device="cuda")
        for x in self.cache:
            x[free] = float("nan")
        self.scale = d ** -0.5

    def args(self):
        return (self.q, *self.cache, i32(self.bt), i32(self.L), i32(self.par), i32(self.n))

    def run(self, **kw):
        return srt.srt_tree_attn_shared(*self.args(), i32(self.ids), i32(self.prefix), self.scale, **kw)

    def plain(self):
        return srt.srt_tree_attn(*self.args(), self.scale)

    def check(self, out, seqs=None):
        o = out.double().cpu().numpy()
        q = self.q.double().cpu().numpy()
        k, v = (x.double().cpu().numpy() for x in self.cache)
        G = self.hq // self.hkv
        for b in range(self.B) if seqs is None else seqs:
            n, L = int(self.n[b]), int(self.L[b])
            one = lambda vv: AT.tree_attention_seq(q[b], k, vv, self.bt[b], L, self.par[b], n, self.scale, self.page)
            ref, amp = one(v), one(np.abs(v))
            K = np.abs(AT.gather_positions(k, self.bt[b], L + n, self.page))
            s_abs = np.stack([(np.abs(q[b, :n, h]) @ K[:, h // G].T).max(-1) for h in range(self.hq)], 1) * self.scale
            e = 2 * (self.d + 16) * 2.0 ** -24 * s_abs[..., None]
            tol = 2.0 ** -8 * (amp + 2 * np.abs(ref)) + (2 * e + (L + n + 64) * 2.0 ** -24) * amp
            err = np.abs(o[b, :n] - ref)
            assert np.isfinite(o[b, :n]).all() and (err <= 1.02 * tol).all(), \
                (b, L, n, float(np.nanmax(err / tol)), np.argwhere(~(err <= 1.02 * tol))[:4].tolist())


HEADS = [(4, 1, 64), (28, 4, 128), (12, 2, 128), (8, 8, 64), (5, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("N", [1, 8, 40])
def test_groups_of_many_sizes(hq, hkv, d, N):
    """Groups of one to nine members, prefixes from none to several splits, none of them a whole page, and sequences of no group."""
    c = Case(N + hq, [1, 2, 5, 9, 3, 2], [100, 0, 77, 513, 2085, 15], (0, 130), N, hq, hkv, d, page=32 if N == 8 else 16, alone=3)
    c.check(c.run())


@pytest.mark.parametrize("P", [15, 16, 63, 64, 65, 255, 256, 257, 272, 511, 1023, 1024, 1025, 1040, 5000])
def test_prefixes_around_tiles_and_splits(P):
    """Nothing behind the prefix but the tree (own 0), or a few keys; splits of 256 keys
    and more (336 pairs of a sequence and a KV head)."""
    c = Case(P, [3, 4] * 6, [P, 2 * P + 1] * 6, [0, 0, 0, 1, 15, 16, 64] * 6, 5, 16, 8, 64, shuffle=False)
    c.check(c.run(), seqs=[*range(7), 20, 41])


def test_small_batches_take_the_plain_way():
    """Every item has a CU of its own: the result is srt_tree_attn's."""
    c = Case(21, [2, 3], [400, 500], (0, 100), 5, 4, 1, 64)
    c.bt = np.ascontiguousarray(c.bt[:, :40])
    live = torch.arange(5, device="cuda") < i32(c.n)[:, None]
    assert torch.equal(c.run()[live], c.plain()[live])
    c.check(c.run())


@pytest.mark.parametrize("N,n", [(256, None), (256, 256), (64, 1)])
def test_wide_trees(N, n):
    c = Case(N, [3, 2], [700, 1100], (0, 1500), N, 14, 2, 128, n=n)
    c.check(c.run())


def test_many_members_and_row_blocks():
    """70 members of a group: node lists of several row blocks, whose last one ends inside a wave."""
    c = Case(5, [70, 3], [3000, 40], (0, 300), 9, 7, 1, 128)
    c.check(c.run(), seqs=range(0, 73, 3))


def test_many_groups_and_more_than_1024_sequences():
    rng = np.random.default_rng(6)
    c = Case(6, rng.integers(1, 4, 700).tolist(), rng.integers(0, 200, 700), (0, 40), 2, 4, 2, 64)
    assert c.B > 1024
    got, want = c.run(), c.plain()
    c.check(got, seqs=range(0, c.B, 37))
    live = torch.arange(2, device="cuda") < i32(c.n)[:, None]
    assert (got - want)[live].abs().max() < 0.05


def test_pages_larger_than_the_prefix_and_large_pages():
    c = Case(7, [4, 3], [200, 700], (0, 600), 6, 4, 2, 128, page=256)
    c.check(c.run())
    c = Case(8, [40], [100], (0, 600), 6, 16, 8, 128, page=1024)  # no whole page: nothing is shared
    c.check(c.run())


def test_peaked_scores():
    """Queries and keys of deviation 3: the parts' maxima differ widely."""
    c = Case(9, [5, 4], [900, 2500], (0, 900), 7, 12, 2, 128, amp=3.0)
    c.check(c.run())


def test_no_groups_is_the_plain_attention():
    c = Case(10, [3, 3], [600, 900], (0, 3000), 6, 4, 2, 128)
    z = i32(np.zeros(0))
    got = srt.srt_tree_attn_shared(*c.args(), i32(c.ids), z, c.scale)
    c.check(got)
    c.ids[:] = 99
    c.check(c.run())
    c.ids[:] = -2 ** 31
    c.check(c.run())


def test_prefix_lengths_are_clipped_to_the_contexts():
    """A stated prefix beyond a member's context shares that member's whole pages; a negative one nothing."""
    c = Case(11, [4, 3], [500, 300], (0, 200), 5, 4, 2, 64)
    p = c.prefix.copy()
    short = int(c.L[c.ids == 0].min())
    c.L[np.flatnonzero(c.ids == 0)[1]] = 37  # one member has rolled back into the prompt
    c.prefix = np.array([2 ** 31 - 1 if short < 500 + 16 else 500, -5])
    c.check(c.run())
    c.prefix = np.minimum(p, 500)
    c.check(c.run())


def test_rows_behind_the_trees_are_left():
    c = Case(12, [4, 3], [500, 300], (0, 200), 9, 4, 2, 128)
    out = torch.full_like(c.q, 7.0)
    c.run(out=out)
    c.check(out)
    dead = torch.arange(9, device="cuda") >= i32(c.n)[:, None]
    assert (out[dead] == 7.0).all()


def test_sizes_out_of_range_on_the_device_are_clamped():
    """Node counts, lengths and pages outside their ranges: no access outside, other sequences unharmed."""
    c = Case(13, [3, 3], [200, 300], (20, 90), 5, 4, 2, 64, shuffle=False, spare=2)
    for x in c.cache:  # (pages that nobody has are read by the bad sequences)
        x.nan_to_num_(0.0)
    c.n[1], c.L[2] = 900, -7
    c.bt[1, 30:], c.bt[5, 15] = 1 << 30, -77
    c.prefix[0] = 0  # (sequence 2's context is empty)
    c.run(scratch=torch.full((srt.srt_tree_attn_shared_scratch_bytes(6, 5, 4, 2, 64, 16, c.bt.shape[1], 2),), 255,
                             dtype=torch.uint8, device="cuda"))
    c.check(c.run(), seqs=[0, 3, 4])


def test_the_same_twice_and_a_scratch_of_any_contents():
    c = Case(14, [6, 5], [1500, 2300], (0, 900), 7, 12, 2, 128)
    need = srt.srt_tree_attn_shared_scratch_bytes(c.B, 7, 12, 2, 128, 16, c.bt.shape[1], 2)
    a = c.run()
    for fill in (0, 255, 127):
        assert torch.equal(c.run(scratch=torch.full((need,), fill, dtype=torch.uint8, device="cuda"))[0, 0], a[0, 0])
    b = c.run(scratch=torch.empty(16, dtype=torch.uint8, device="cuda"))  # (too small: another one is taken)
    live = torch.arange(7, device="cuda") < i32(c.n)[:, None]
    assert torch.equal(a[live], b[live])


def test_on_a_side_stream_and_replayed_from_graphs_with_one_scratch():
    cases = [Case(15, [4, 3], [900, 40], (0, 300), 6, 4, 2, 128), Case(16, [9], [3000], (0, 90), 3, 12, 2, 64)]
    need = max(srt.srt_tree_attn_shared_scratch_bytes(c.B, c.N, c.hq, c.hkv, c.d, 16, c.bt.shape[1], len(c.prefix)) for c in cases)
    scratch = torch.empty(need, dtype=torch.uint8, device="cuda")  # shared by both graphs, replayed in order
    side, held = torch.cuda.Stream(), []
    for c in cases:
        live = torch.arange(c.N, device="cuda") < i32(c.n)[:, None]
        want = c.run()
        side.wait_stream(torch.cuda.current_stream())
        got = c.run(stream=side)
        side.synchronize()
        assert torch.equal(got[live], want[live])
        args, ids, prefix, out = c.args(), i32(c.ids), i32(c.prefix), torch.zeros_like(want)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            srt.srt_tree_attn_shared(*args, ids, prefix, c.scale, out=out, scratch=scratch)
        held.append((g, out, want, live, args, ids, prefix))
    for _ in range(3):
        for g, out, want, live, *_ in held:
            out.fill_(9)
            g.replay()
            torch.randn(1 << 20, device="cuda").sum().item()
            assert torch.equal(out[live], want[live]) and (out[~live] == 9).all()


def test_wrong_shapes_are_refused():
    c = Case(17, [2, 2], [64, 64], (0, 20), 3, 4, 2, 64)
    a = dict(zip(("q", "k_cache", "v_cache", "block_table", "ctx_len", "tree_parent", "n_nodes"), c.args()))
    a.update(group_ids=i32(c.ids), prefix_len=i32(c.prefix), scale=c.scale)
    for kw in (dict(q=c.q.float()), dict(q=c.q[:, :, :, :32]), dict(k_cache=c.cache[0][:, :1]), dict(v_cache=c.cache[1].cpu()),
               dict(block_table=a["block_table"][:2]), dict(block_table=a["block_table"][:, ::2]), dict(ctx_len=a["ctx_len"][:3]),
               dict(tree_parent=a["tree_parent"][:, :2]), dict(n_nodes=a["n_nodes"].long()), dict(group_ids=a["group_ids"][:3]),
               dict(prefix_len=a["prefix_len"].long()), dict(prefix_len=a["prefix_len"][None]), dict(out=torch.empty_like(c.q)[:1])):
        with pytest.raises(ValueError):
            srt.srt_tree_attn_shared(**{**a, **kw})
    with pytest.raises(srt.SrtError):
        srt.srt_tree_attn_shared(**{**a, "scale": float("nan")})

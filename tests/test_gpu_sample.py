"""The acceptance walk of a policy that samples with top-k, top-p and min-p on the
GPU: tokens, nodes and counts bit for bit against the fp64 oracle.  (The place of a
top-p cut is a comparison of sums; it is decided alike unless the token at the cut is
the chosen one and the sums differ by less than 1e-7 of the mass there.)"""
import numpy as np
import pytest
import torch

from oracle import rules as RU
from oracle import sampling as SA
from paper_2601_09083_amd import srt

pytestmark = pytest.mark.gpu
CUTS = [(0, 1.0, 0.0), (1, 1.0, 0.0), (5, 1.0, 0.0), (0, 0.9, 0.0), (0, 0.5, 0.0), (0, 1.0, 0.1), (20, 0.8, 0.0), (300, 0.95, 0.02),
        (0, 0.99, 0.001), (0, 0.0, 0.0), (0, 1.0, 1.0), (0, 1.0, 7.0), (-3, 2.0, -1.0), (50, 1.0, 0.05), (10 ** 9, 0.7, 0.0)]


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x).astype(np.int32), device="cuda")


def f32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.float32), device="cuda")


class Case:
    """Rows whose probability falls with the rank as rank ** -a; planted paths."""

    def __init__(self, seed, B, N, V, dmax, a=1.5, cuts=None, invT=(1.0, 0.7, 1.4), ruled=False, bias=6):
        rng = np.random.default_rng(seed)
        self.B, self.N, self.V, self.dmax = B, N, V, dmax
        self.logits = (rng.exponential(a, (B, N, V)) if np.isscalar(a) else rng.exponential(1.0, (B, N, V)) *
                       np.asarray(a)[np.arange(B) % len(a), None, None]).astype(np.float32)
        self.gumbel = rng.gumbel(size=(B, dmax + 1, V)).astype(np.float32)
        self.n = rng.integers(max(1, N // 2), N + 1, B)
        self.tok = rng.integers(0, V, (B, N))
        self.par = np.full((B, N), -1)
        for b in range(B):
            for i in range(1, int(self.n[b])):
                self.par[b, i] = rng.integers(max(0, i - 3), i)
                self.logits[b, self.par[b, i], self.tok[b, i]] = np.float32(6 + self.logits[b].max() * 0.9 + rng.random())
        cuts = CUTS if cuts is None else cuts
        pick = [cuts[i % len(cuts)] for i in rng.permutation(max(B, len(cuts)))[:B]] if B < len(cuts) else \
            [cuts[i % len(cuts)] for i in range(B)]
        self.k, self.p, self.m = (np.array(x) for x in zip(*pick))
        self.k = self.k.astype(np.int64)
        self.p, self.m = self.p.astype(np.float32), self.m.astype(np.float32)
        self.invT = np.array([invT[i % len(invT)] for i in range(B)], dtype=np.float32)
        self.words = self.mask = self.bias = None
        self.r = self.f = self.q = None
        if ruled:
            w = np.where(rng.random((B, V)) < 0.2, rng.integers(1, 9, (B, V)), 0)
            self.words = (w | np.where(rng.random((B, V)) < 0.1, 0x8000, 0)).astype(np.uint16)
            self.r, self.f, self.q = (rng.choice(x, B).astype(np.float32) for x in ((1.0, 1.3, 0.8), (0.0, 0.2, -0.1), (0.0, 0.5)))
            self.bias = [sorted((int(rng.integers(-2, V + 3)), float(np.float32(rng.normal(0, 3)))) for _ in range(rng.integers(0, bias + 1)))
                         for _ in range(B)]
            self.mask = np.where(rng.random((B, N, 1)) < 0.3, 0xFFFFFFFF, rng.integers(0, 1 << 32, (B, N, (V + 31) // 32))).astype(np.uint32)
            for b in range(B):
                for i in range(1, int(self.n[b])):
                    t = self.tok[b, i]
                    self.mask[b, self.par[b, i], t // 32] |= np.uint32(1 << int(t % 32))
            bits = (self.mask[:, :, np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
            self.logits = np.where(bits == 0, rng.choice([np.nan, np.inf, -np.inf, 3e38, 0.0], (B, N, V)), self.logits).astype(np.float32)

    def rules(self):
        if self.words is None and self.mask is None and self.bias is None:
            return None
        c = lambda x: None if x is None else torch.as_tensor(x, device="cuda")
        off = tok = val = None
        if self.bias is not None:
            off = i32(np.cumsum([0] + [len(x) for x in self.bias]))
            tok = i32(np.array([t for x in self.bias for t, _ in x]))
            val = f32([v for x in self.bias for _, v in x])
        return srt.Rules(seen=c(None if self.words is None else self.words.view(np.int16)), repetition=c(self.r), frequency=c(self.f),
                         presence=c(self.q), bias_offsets=off, bias_tokens=tok, bias_values=val,
                         mask=c(None if self.mask is None else self.mask.view(np.int32)))

    def sampling(self):
        return srt.Sampling(inv_temperature=f32(self.invT), top_k=i32(self.k), top_p=f32(self.p), min_p=f32(self.m))

    def args(self):
        return (f32(self.logits), None if self.gumbel is None else f32(self.gumbel), self.sampling(), i32(self.tok), i32(self.par),
                i32(self.n), self.dmax)

    def run(self, **kw):
        return srt.srt_accept_sample(*self.args(), rules=self.rules(), **kw)

    def want(self, b):
        at = lambda x, z: z if x is None else x[b]
        return SA.walk(lambda u: self.logits[b, u], None if self.gumbel is None else lambda s: self.gumbel[b, s], self.invT[b],
                       int(self.k[b]), self.p[b], self.m[b], self.tok[b], self.par[b], int(self.n[b]), self.dmax,
                       at(self.words, None), at(self.r, 1.0), at(self.f, 0.0), at(self.q, 0.0), at(self.bias, ()),
                       None if self.mask is None else lambda u: self.mask[b, u])

    def check(self, got):
        got, depth = {k: v.cpu().numpy() for k, v in got.items()}, 0
        for b in range(self.B):
            k, toks, nodes, e = self.want(b)
            pad = lambda x: x + [-1] * (self.dmax + 1 - len(x))
            say = (b, int(self.k[b]), float(self.p[b]), float(self.m[b]), got["out_tokens"][b].tolist(), toks)
            assert got["out_tokens"][b].tolist() == pad(toks) and got["out_nodes"][b].tolist() == pad(nodes), say
            assert int(got["n_accepted"][b]) == k and int(got["n_emitted"][b]) == e, say
            depth = max(depth, k)
        return depth


@pytest.mark.parametrize("ruled", [False, True])
@pytest.mark.parametrize("V", [1, 2, 3, 31, 33, 1000, 5119, 8192, 8193, 20483, 50001])
def test_every_cut(V, ruled):
    """Odd rows, both numbers of threads, sure and flat rows."""
    c = Case(V, 30, 6, V, 4, a=(0.5, 1.0, 1.5, 2.5), ruled=ruled)
    depth = c.check(c.run())
    assert depth >= 1 or V < 50


@pytest.mark.parametrize("V", [152064, 262143, 400001])
def test_long_rows(V):
    """Segments of one batch and of several."""
    c = Case(V, 5, 2, V, 1, a=(0.4, 1.5, 2.0), cuts=[(0, 0.9, 0.0), (40, 0.9, 0.01), (0, 1.0, 1e-4), (6000, 1.0, 0.0), (0, 0.5, 0.0)])
    c.check(c.run())


@pytest.mark.parametrize("V", [9000, 60001])
@pytest.mark.parametrize("cut", [(5000, 1.0, 0.0), (8000, 0.7, 0.0), (0, 0.9999, 0.0), (0, 0.99999994, 0.0), (0, 0.3, 0.0), (0, 1.0, 1e-3),
                                 (4096, 1.0, 0.0), (4097, 0.99, 1e-6), (8999, 1.0, 0.0)])
def test_more_kept_tokens_than_the_list_holds(V, cut):
    c = Case(V, 6, 3, V, 2, a=0.3, cuts=[cut])
    c.check(c.run())


def test_rows_of_ties():
    """Equal scores: the order goes by the token, whatever path finds the cut."""
    for V, levels in ((50, 2), (700, 3), (30000, 1), (30000, 2), (30000, 40), (70000, 1)):
        cuts = [(7, 1.0, 0.0), (V // 3, 1.0, 0.0), (0, 0.5, 0.0), (0, 0.3, 0.0), (V // 2, 0.5, 0.0), (0, 1.0, 0.5), (0, 0.9, 0.1)]
        c = Case(V, 14, 1, V, 0, cuts=cuts, invT=(1.0,))
        c.logits[:] = np.random.default_rng(V).integers(0, levels, c.logits.shape) * 0.5
        c.check(c.run())


def test_scores_close_together_and_far_apart():
    """Ranges of scores from a few units in the last place to nearly all of fp32."""
    V, rng = 40000, np.random.default_rng(1)
    cuts = [(9000, 1.0, 0.0), (0, 0.4, 0.0), (20000, 0.5, 0.0), (100, 0.5, 0.0)]
    for values in (1000 + rng.integers(0, 30, (8, 1, V)) * 2.0 ** -13, 1 + rng.random((8, 1, V)) * 1e-5,
                   rng.choice([-1e9, -1e30, -3e38, 3e38], (8, 1, V)), rng.normal(0, 1e37, (8, 1, V)), rng.normal(0, 1e-41, (8, 1, V)),
                   rng.choice([-3.4028235e38, 0.0], (8, 1, V), p=[0.9997, 0.0003])):
        c = Case(2, 8, 1, V, 0, cuts=cuts, invT=(1.0,))
        c.logits[:] = values
        c.check(c.run())


def test_values_that_take_no_part():
    for V in (60, 30000):
        c = Case(3, 12, 1, V, 2, cuts=[(10, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.1), (0, 1.0, 0.0)])
        rng = np.random.default_rng(V)
        odd = rng.choice([np.nan, -np.inf], c.logits.shape)
        c.logits = np.where(rng.random(c.logits.shape) < 0.9, odd, c.logits).astype(np.float32)
        c.logits[4] = -np.inf
        c.logits[5] = np.nan
        c.logits[6:10, 0, [V // 2, V - 1]] = np.inf
        c.logits[10, 0] = -np.inf
        c.logits[10, 0, V - 1] = -5.0  # one token left: the row's last
        got = c.run()
        c.check(got)
        assert got["n_emitted"].tolist()[4:6] == [0, 0] and got["out_tokens"][10, 0].item() == V - 1
        assert got["out_tokens"][6:10, 0].tolist() == [V // 2] * 4


def test_parameters_that_are_not_numbers():
    """A NaN in top_p or min_p keeps the first token alone."""
    for V in (100, 20000):
        c = Case(4, 4, 1, V, 0, cuts=[(0, float("nan"), 0.0), (0, 1.0, float("nan")), (0, 0.9, float("nan")), (3, float("nan"), 0.5)])
        c.check(c.run())


def test_parameters_left_out():
    c = Case(5, 9, 6, 12000, 4, cuts=[(0, 0.9, 0.0), (30, 1.0, 0.0), (0, 1.0, 0.05)])
    a = c.args()
    one = lambda **kw: srt.srt_accept_sample(a[0], a[1], srt.Sampling(**kw), *a[3:])
    keep = c.invT, c.k, c.p, c.m
    for name, on in (("inv_temperature", 0), ("top_k", 1), ("top_p", 2), ("min_p", 3)):
        c.invT, c.k, c.p, c.m = (x if i == on else np.full_like(x, z) for i, (x, z) in enumerate(zip(keep, (1, 0, 1, 0))))
        c.check(one(**{name: (i32 if on == 1 else f32)(keep[on])}))


def test_without_cuts_it_is_the_plain_walk():
    """Bit for bit srt_accept's and srt_accept_rules' results, sampled and greedy."""
    for ruled in (False, True):
        for V in (900, 30001):
            c = Case(6, 10, 8, V, 5, cuts=[(0, 1.0, 0.0)], invT=(0.8,), ruled=ruled)
            a = c.args()
            for noise in (a[1], None):
                got = srt.srt_accept_sample(a[0], noise, a[2], *a[3:], rules=c.rules())
                tree = (a[3], a[4], a[5], c.dmax)
                want = srt.srt_accept_rules(a[0], noise, 0.8, c.rules(), *tree) if ruled else srt.srt_accept(a[0], noise, 0.8, *tree)
                assert all(torch.equal(got[k], want[k]) for k in want)


def test_greedy_ignores_the_parameters():
    c = Case(7, 15, 6, 3000, 4)
    c.gumbel = None
    c.check(c.run())


def test_long_bias_lists_and_tokens_listed_again():
    for V in (900, 20000):
        c = Case(8, 6, 8, V, 4, ruled=True, bias=600, cuts=[(10, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.1)])
        for x in c.bias:
            x.extend([(11, 1.25), (11, -0.5), (11, 2.0)])
            x.sort(key=lambda e: e[0])
        c.check(c.run())


def test_bias_lists_beyond_their_room():
    """Longer than what is staged, and than what is scored apart together with the counted tokens."""
    for V, n in ((9001, 513), (20000, 5000), (20000, 12000)):
        c = Case(17, 4, 6, V, 3, ruled=True, bias=0, cuts=[(10, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.1), (0, 1.0, 0.0)])
        rng = np.random.default_rng(18)
        for b in (0, 1, 2):
            c.bias[b] = sorted((int(t), float(np.float32(x))) for t, x in zip(rng.integers(-2, V + 3, n), rng.normal(0, 2, n)))
        c.check(c.run())


@pytest.mark.parametrize("V,ruled", [(1 << 21, False), (1 << 18, True)])
def test_the_largest_vocabularies(V, ruled):
    c = Case(19, 2, 2, V, 1, a=(0.5, 1.5), cuts=[(0, 0.9, 0.0), (50, 0.9, 0.0)], ruled=ruled)
    c.check(c.run())


@pytest.mark.parametrize("ruled", [False, True])
def test_the_deepest_walks_of_the_widest_trees(ruled):
    c = Case(20, 4, 256, 200, 63, cuts=[(1, 1.0, 0.0), (0, 1e-6, 0.0), (2, 1.0, 0.99), (0, 1.0, 0.0)])
    for b in range(c.B):
        c.n[b] = 256
        for i in range(1, 256):  # a chain of 64 levels, and side branches of other tokens
            c.par[b, i] = i - 1 if i < 64 else i % 64
            c.tok[b, i] = (3 * i) % 100 if i < 64 else 100 + i % 100
        top = c.logits[b].max() + 60  # (above the tokens that Case has planted)
        for i in range(63):
            c.logits[b, i, c.tok[b, i + 1]] = top
    if ruled:
        c.words = np.zeros((c.B, c.V), dtype=np.uint16)
        c.f = np.full(c.B, 0.25, dtype=np.float32)
        c.r = c.q = None
    assert c.check(c.run()) == 63


@pytest.mark.parametrize("V", [700, 30000])
def test_inverse_temperatures_that_turn_or_flatten_the_order(V):
    """Of 0 all scores are equal, of a negative one the least logit is the first."""
    c = Case(21, 12, 3, V, 2, invT=(0.0, -1.0, 1e-30, 1e30), cuts=[(7, 1.0, 0.0), (0, 0.5, 0.0), (V // 2, 0.5, 0.0)])
    c.check(c.run())


@pytest.mark.parametrize("V", [700, 30000])
def test_noise_of_tokens_that_are_not_kept(V):
    """None of these cuts keeps a token of a row's lower half."""
    c = Case(24, 16, 1, V, 0, a=(0.3, 1.5), cuts=[(20, 1.0, 0.0), (0, 0.5, 0.0), (0, 1.0, 0.9), (V // 3, 0.9, 0.0)])
    rng = np.random.default_rng(25)
    low = c.logits < np.median(c.logits, axis=2, keepdims=True)
    c.gumbel = np.where(low, rng.choice([np.nan, np.inf, -np.inf, 3e38], c.gumbel.shape), c.gumbel).astype(np.float32)
    c.check(c.run())


def test_two_walks_at_once():
    cs = [Case(22, 32, 8, 20483, 4), Case(23, 16, 8, 9000, 4, ruled=True)]
    want = [c.run() for c in cs]
    args = [(c.args(), c.rules()) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for (a, rules), s in zip(args, streams):
            with torch.cuda.stream(s):
                got.append(srt.srt_accept_sample(*a, rules=rules))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(g[k], want[i % 2][k]) for k in g)


def test_masks_that_leave_little_or_nothing():
    for V in (40, 30000):
        c = Case(9, 8, 6, V, 3, ruled=True, bias=0, cuts=[(5, 0.9, 0.0), (0, 0.8, 0.0)])
        c.mask[0] = 0
        c.mask[1, 1:] = 0
        c.mask[2] = 0
        c.mask[2, :, -1] = np.uint32(1 << ((V - 1) % 32))
        c.logits[2, :, V - 1] = 0.0
        got = c.run()
        c.check(got)
        assert got["n_emitted"][0].item() == 0 and got["out_tokens"][2, 0].item() == V - 1


@pytest.mark.parametrize("shift", [0.0, -1.0, -60.0, 1e5])
def test_the_mass_of_the_first_of_many(shift):
    """More than a list's tokens under a top-k and a top-p: the k-th place is searched for."""
    c = Case(14, 6, 3, 60001, 2, a=(0.4, 1.0), cuts=[(6000, 0.9, 0.0), (20000, 0.5, 0.0), (59000, 0.99, 0.3), (30000, 0.999, 0.9)])
    c.logits += np.float32(shift)
    c.check(c.run())


def test_fewer_tokens_than_the_first_k():
    c = Case(15, 6, 3, 60001, 2, a=(0.4, 1.0), cuts=[(50000, 0.9, 0.0), (60000, 0.5, 0.0), (59000, 0.99, 0.3)])
    rng = np.random.default_rng(16)
    gone = rng.random(c.logits.shape) < np.array([0.5, 0.9, 0.3])[None, :, None]
    for b in range(c.B):
        for i in range(1, int(c.n[b])):
            gone[b, c.par[b, i], c.tok[b, i]] = False
    c.logits[gone] = -np.inf
    c.check(c.run())


def test_the_same_again_and_many_sequences():
    """Sums and lists do not depend on the order of atomics."""
    c = Case(10, 300, 4, 6000, 3, a=(0.4, 1.4))
    first = c.run()
    c.check(first)
    for _ in range(3):
        again = c.run()
        assert all(torch.equal(first[k], again[k]) for k in first)


def test_on_a_side_stream_and_replayed_from_graphs():
    held, side = [], torch.cuda.Stream()
    for c in (Case(11, 16, 8, 3000, 4), Case(12, 4, 8, 60000, 4, a=0.5, ruled=True)):
        want = c.run()
        c.check(want)
        side.wait_stream(torch.cuda.current_stream())
        got = c.run(stream=side)
        side.synchronize()
        assert all(torch.equal(got[k], want[k]) for k in want)
        a, rules, out = c.args(), c.rules(), {k: torch.zeros_like(v) for k, v in want.items()}
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            srt.srt_accept_sample(*a, rules=rules, out=out)
        held.append((g, out, want, a, rules))
    for _ in range(3):
        for g, out, want, *_ in held:
            for x in out.values():
                x.fill_(9)
            g.replay()
            torch.randn(1 << 20, device="cuda").sum().item()
            assert all(torch.equal(out[k], want[k]) for k in want)


def test_a_decode_loop_under_penalties():
    """Walk, count, walk: the count rows follow the emitted tokens."""
    c = Case(13, 8, 8, 900, 4, ruled=True, bias=0)
    c.mask = c.bias = None
    c.logits = np.nan_to_num(c.logits, nan=0.0, posinf=1.0, neginf=-1.0).clip(-50, 50)
    seen = torch.as_tensor(c.words.view(np.int16).copy(), device="cuda")
    rules = srt.Rules(seen=seen, repetition=f32(c.r), frequency=f32(c.f), presence=f32(c.q))
    for _ in range(4):
        got = srt.srt_accept_sample(*c.args(), rules=rules)
        c.check(got)
        srt.srt_seen_add(seen, got["out_tokens"], got["n_emitted"])
        for b in range(c.B):
            _, toks, _, e = c.want(b)
            c.words[b] = RU.seen_add(c.words[b], toks[:e], False, False)


def test_wrong_shapes_are_refused():
    c = Case(14, 4, 3, 50, 2)
    a = dict(zip(("logits", "gumbel", "sampling", "tree_tokens", "tree_parent", "n_nodes", "max_depth"), c.args()))
    out = srt.srt_accept_sample(**a)
    for kw in (dict(logits=a["logits"].double()), dict(logits=a["logits"][0]), dict(logits=a["logits"].cpu()),
               dict(gumbel=a["gumbel"][:, 1:]), dict(tree_tokens=a["tree_tokens"][:, :2]), dict(n_nodes=a["n_nodes"][:3]),
               dict(n_nodes=a["n_nodes"].long()), dict(sampling=srt.Sampling(top_k=i32([1, 2]))),
               dict(sampling=srt.Sampling(top_p=torch.ones(4))), dict(out={**out, "out_nodes": out["out_nodes"][:, :2]}),
               dict(rules=srt.Rules(presence=f32([0.0])))):
        with pytest.raises(ValueError):
            srt.srt_accept_sample(**{**a, **kw})

"""The acceptance walk under sampling rules and the token counts on the GPU:
bit for bit against their oracle."""
import numpy as np
import pytest
import torch

from oracle import rules as RU
from paper_2601_09083_amd import srt

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.as_tensor(np.ascontiguousarray(x).astype(np.int32), device="cuda")


class Case:
    """A batch with every rule, near ties and planted paths."""

    def __init__(self, seed, B, N, V, dmax, sampled=True, seen=True, penalties=True, bias=8, mask=True, integer=False):
        rng = np.random.default_rng(seed)
        self.B, self.N, self.V, self.dmax = B, N, V, dmax
        self.n = rng.integers(1, N + 1, B)
        self.tok = rng.integers(0, V, (B, N))
        self.par = np.full((B, N), -1)
        logits = rng.normal(0, 2, (B, N, V))
        if integer:
            logits = np.round(logits)
        self.words = None
        if seen:
            w = np.where(rng.random((B, V)) < 0.2, rng.integers(1, 12, (B, V)), 0)
            self.words = (w | np.where(rng.random((B, V)) < 0.1, 0x8000, 0)).astype(np.uint16)
        self.r = rng.choice([1.0, 1.1, 0.8, 1.5], B).astype(np.float32) if penalties else None
        self.f = rng.choice([0.0, 0.3, -0.2, 2.0], B).astype(np.float32) if penalties else None
        self.q = rng.choice([0.0, 0.5, -1.0], B).astype(np.float32) if penalties else None
        self.bias = [sorted((int(rng.integers(-2, V + 3)), float(np.float32(rng.normal(0, 2)))) for _ in range(rng.integers(0, bias + 1)))
                     for _ in range(B)] if bias else None
        W = (V + 31) // 32
        self.mask = None
        if mask:
            keep = rng.random((B, N, 1)) < 0.4
            self.mask = np.where(keep, 0xFFFFFFFF, rng.integers(0, 1 << 32, (B, N, W))).astype(np.uint32)
        for b in range(B):
            n = int(self.n[b])
            for i in range(1, n):
                self.par[b, i] = rng.integers(max(0, i - 3), i)
                if rng.random() < 0.3:  # paths that say a token again
                    self.tok[b, i] = self.tok[b, self.par[b, i]]
            for i in range(1, n):  # the last planted child of a node is its choice, mostly
                logits[b, self.par[b, i], self.tok[b, i]] = 14 + 3 * rng.random()
                if mask:
                    t = self.tok[b, i]
                    self.mask[b, self.par[b, i], t // 32] |= np.uint32(1 << int(t % 32))
            self.tok[b, n:] = -1
        if mask:  # what is forbidden may hold anything
            bits = (self.mask[:, :, np.arange(V) // 32] >> (np.arange(V) % 32).astype(np.uint32)) & 1
            odd = rng.choice([np.nan, np.inf, -np.inf, 3e38, 0.0], (B, N, V))
            logits = np.where(bits == 0, odd, logits)
        self.logits = logits.astype(np.float32)
        self.gumbel = rng.gumbel(size=(B, dmax + 1, V)).astype(np.float32) if sampled else None
        self.invT = 0.8

    def run(self, **kw):
        c = lambda x: None if x is None else torch.as_tensor(x, device="cuda")
        off = tok = val = None
        if self.bias is not None:
            off = i32(np.cumsum([0] + [len(x) for x in self.bias]))
            tok = i32(np.array([t for x in self.bias for t, _ in x]))
            val = torch.tensor([v for x in self.bias for _, v in x], dtype=torch.float32, device="cuda")
        rules = srt.Rules(seen=c(None if self.words is None else self.words.view(np.int16)), repetition=c(self.r),
                          frequency=c(self.f), presence=c(self.q), bias_offsets=off, bias_tokens=tok, bias_values=val,
                          mask=c(None if self.mask is None else self.mask.view(np.int32)))
        return srt.srt_accept_rules(c(self.logits), c(self.gumbel), self.invT, rules, i32(self.tok), i32(self.par),
                                    i32(self.n), self.dmax, **kw)

    def want(self, b):
        at = lambda x, z: z if x is None else x[b]
        return RU.walk(lambda u: self.logits[b, u], None if self.gumbel is None else lambda k: self.gumbel[b, k], self.invT,
                       self.tok[b], self.par[b], int(self.n[b]), self.dmax, at(self.words, None), at(self.r, 1.0),
                       at(self.f, 0.0), at(self.q, 0.0), at(self.bias, ()),
                       None if self.mask is None else lambda u: self.mask[b, u])

    def check(self, got):
        got = {k: v.cpu().numpy() for k, v in got.items()}
        depth = 0
        for b in range(self.B):
            k, toks, nodes, e = self.want(b)
            pad = lambda x: x + [-1] * (self.dmax + 1 - len(x))
            assert int(got["n_accepted"][b]) == k and int(got["n_emitted"][b]) == e, b
            assert got["out_tokens"][b].tolist() == pad(toks) and got["out_nodes"][b].tolist() == pad(nodes), b
            depth = max(depth, k)
        return depth


@pytest.mark.parametrize("sampled", [True, False])
@pytest.mark.parametrize("V", [1, 31, 33, 1000, 2047, 20480, 20483, 40961, 50001])
def test_walk_with_every_rule(V, sampled):
    """Both routes of the walk, on both sides of their border; odd rows."""
    small = V <= 2047
    c = Case(V, 24 if small else 6, 12, V, 5, sampled)
    depth = c.check(c.run())
    assert depth >= 1 or V < 100  # (the oracle's walks leave the root)


@pytest.mark.parametrize("only", ["seen", "penalties", "bias", "mask", "none"])
def test_each_rule_alone(only):
    for V, sampled in ((700, False), (41001, True)):
        on = lambda x: only == x
        c = Case(5, 8, 10, V, 4, sampled, seen=on("seen") or on("penalties"), penalties=on("penalties"),
                 bias=8 if on("bias") else 0, mask=on("mask"))
        c.check(c.run())
        if only == "none":  # the plain walk
            t = lambda x: torch.as_tensor(x, device="cuda")
            want = srt.srt_accept(t(c.logits), None if c.gumbel is None else t(c.gumbel), c.invT, i32(c.tok), i32(c.par),
                                  i32(c.n), c.dmax)
            got = c.run()
            assert all(torch.equal(got[k], want[k]) for k in want)


def test_ties_go_to_the_lowest_token():
    for V in (300, 42000):
        c = Case(6, 12, 8, V, 4, sampled=False, integer=True, penalties=False)
        c.check(c.run())


def test_long_bias_lists_and_tokens_listed_again():
    for V in (900, 45000):
        c = Case(7, 5, 8, V, 4, bias=700)
        for x in c.bias:
            x.extend([(11, 1.25), (11, -0.5), (11, 2.0)])
            x.sort(key=lambda e: e[0])
        c.check(c.run())


def test_rows_with_nothing_left():
    """Every token forbidden at the root, or deeper, or all -inf or NaN: the walk ends without a token."""
    for V in (40, 44000):
        c = Case(8, 6, 6, V, 3, sampled=False, bias=0, penalties=False, seen=False)
        c.n[:] = 6
        c.par[:] = [-1, 0, 1, 2, 3, 4]
        c.mask[:] = 0xFFFFFFFF
        c.logits[:] = np.random.default_rng(1).normal(0, 1, c.logits.shape)
        c.tok[:] = np.arange(6) + 3
        for i in range(1, 6):
            c.logits[:, i - 1, i + 3] = 50.0
        c.mask[0, 0] = 0
        c.mask[1, 2] = 0
        c.logits[2, 1] = -np.inf
        c.logits[3, 0] = np.nan
        c.mask[4, 0] = 0
        c.mask[4, 0, -1] = np.uint32(1 << ((V - 1) % 32))  # the last token alone
        got = c.run()
        c.check(got)
        assert got["n_emitted"].tolist()[:5] == [0, 2, 1, 0, 1] and got["out_tokens"][4, 0].item() == V - 1


def test_infinite_scores():
    """+inf is the largest score (lowest index on ties); a bias may forbid."""
    V = 500
    c = Case(9, 4, 3, V, 2, sampled=False, bias=0, penalties=False, seen=False, mask=False)
    c.logits[0, 0, [77, 400]] = np.inf
    c.bias = [[], [(int(np.argmax(c.logits[1, 0])), float("-inf"))], [(3, float("inf"))], []]
    c.check(c.run())


def test_walk_on_a_side_stream_and_replayed_from_graphs():
    cases = [Case(10, 16, 10, 3000, 4), Case(11, 4, 10, 60000, 4)]
    eager = [c.run() for c in cases]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = [c.run() for c in cases]
    side.synchronize()
    for c, e, x in zip(cases, eager, got):
        c.check(x)
        assert all(torch.equal(e[k], x[k]) for k in e)
    t = lambda x: torch.as_tensor(x, device="cuda")
    held = []
    for c in cases:
        a = dict(logits=t(c.logits), gumbel=t(c.gumbel), tok=i32(c.tok), par=i32(c.par), n=i32(c.n))
        rules = srt.Rules(seen=t(c.words.view(np.int16)), repetition=t(c.r), frequency=t(c.f), presence=t(c.q),
                          mask=t(c.mask.view(np.int32)))
        c.bias = None
        call = lambda out, scratch, a=a, rules=rules, c=c: srt.srt_accept_rules(
            a["logits"], a["gumbel"], c.invT, rules, a["tok"], a["par"], a["n"], c.dmax, out=out, scratch=scratch)
        want = call(None, None)
        out = {k: torch.zeros_like(v) for k, v in want.items()}
        scratch = torch.empty(srt.srt_accept_scratch_bytes(c.B), dtype=torch.uint8, device="cuda")
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call(out, scratch)
        held.append((g, out, want, scratch, a, rules))
    for _ in range(3):
        for g, out, want, *_ in held:
            for x in out.values():
                x.fill_(9)
            g.replay()
            torch.randn(1 << 20, device="cuda").sum().item()
            assert all(torch.equal(out[k], want[k]) for k in want)


# --------------------------------------------------------------------------- counts

@pytest.mark.parametrize("V", [1, 7, 1001, 16384, 16385, 32767, 32769, 70000])
@pytest.mark.parametrize("T", [1, 13, 64, 65, 3000, 66000])
def test_seen_add(V, T):
    rng = np.random.default_rng(V + T)
    B = 5
    words = (rng.integers(0, 0x8000, (B, V)) | np.where(rng.random((B, V)) < 0.3, 0x8000, 0)).astype(np.uint16)
    words[0] = 0x7FFE
    tok = rng.integers(-2, V + 2, (B, T))
    tok[1] = rng.integers(0, min(V, 5), T)
    lens = np.array([T, T, 0, T // 2, -3])
    lens[3] = min(T + 5, 2 * T)  # clamped
    for prompt in (False, True):
        for reset in (False, True):
            seen = torch.as_tensor(words.view(np.int16).copy(), device="cuda")
            srt.srt_seen_add(seen, i32(tok), i32(lens), prompt=prompt, reset=reset)
            got = seen.cpu().numpy().view(np.uint16)
            for b in range(B):
                want = RU.seen_add(words[b], tok[b, :min(max(lens[b], 0), T)].tolist(), prompt, reset)
                assert np.array_equal(got[b], want), (b, prompt, reset)


def test_a_decode_loop_under_penalties():
    """Walk, count, walk: the count rows follow the emitted tokens as they come."""
    c = Case(12, 8, 10, 900, 4, bias=0, mask=False)
    seen = torch.as_tensor(c.words.view(np.int16).copy(), device="cuda")
    t = lambda x: torch.as_tensor(x, device="cuda")
    rules = srt.Rules(seen=seen, repetition=t(c.r), frequency=t(c.f), presence=t(c.q))
    for _ in range(5):
        got = srt.srt_accept_rules(t(c.logits), t(c.gumbel), c.invT, rules, i32(c.tok), i32(c.par), i32(c.n), c.dmax)
        c.check(got)
        srt.srt_seen_add(seen, got["out_tokens"], got["n_emitted"])
        for b in range(c.B):
            k, toks, _, e = c.want(b)
            c.words[b] = RU.seen_add(c.words[b], toks[:e], False, False)
        assert np.array_equal(seen.cpu().numpy().view(np.uint16), c.words)

"""The operators of a decode step of a group of rollouts, as measurable cases.

Each case is one operator as a decode loop uses it, in a plain form of
elementary torch operations and, where ``own`` is true, through the public
binding ``paper_2601_09083_amd.srt``:

* ``rope``    srt_rope_append: the rotary position encoding of a step's queries
  and keys, the rotated keys and the values written to their places in the paged
  cache; or srt_rope_rows: the rotated keys as rows, which the calls of the 8-bit
  cache read;
* ``shared``  srt_tree_attn_shared: every tree node against a paged cache in which
  groups of sequences share the pages of a long prefix, read once for all of them;
* ``sample``  srt_accept_sample: the acceptance walk where the policy samples with a
  temperature, top-k, top-p and min-p of each sequence's own, from given noise.

Lengths, tree sizes, accepted lengths and sampling parameters are the quantiles
of their distributions in an order drawn from the seed, so that the work of a
case does not depend on the seed.
"""
import math
import statistics

import numpy as np
import torch

own = False

DEV = "cuda"
PROMPT = 0x8000  # bit of a seen word: the token is in the prompt


def listed():
    return [
        # Four small sequences' draft trees: the smallest step, where the launch counts.
        dict(name="rope_small", kind="rope", to="cache", B=4, T=8, hq=4, hkv=1, d=64, rot=64, pairs="halves", page=16,
             lo=128, hi=512, rows="trees"),
        # The draft trees of a batch of 256, as the decode loop drafts them.
        dict(name="rope_trees", kind="rope", to="cache", B=256, T=64, hq=28, hkv=4, d=128, rot=128, pairs="halves", page=16,
             lo=1000, hi=16384, rows="trees"),
        # Prompts of up to 4k tokens enter the cache; half of each head turns, neighbouring dims together.
        dict(name="rope_prompts", kind="rope", to="cache", B=16, T=4096, hq=32, hkv=8, d=128, rot=64, pairs="neighbours",
             page=32, lo=0, hi=64, rows="prompts"),
        # Trees at far positions, for the 8-bit cache.
        dict(name="rope_rows", kind="rope", to="rows", B=61, T=16, hq=12, hkv=2, d=128, rot=128, pairs="halves", page=16,
             lo=100000, hi=1000000, rows="trees"),
        # Two prompts with two answers each, one small layer.
        dict(name="shared_small", kind="shared", groups=2, each=2, N=8, hq=4, hkv=1, d=64, page=16, plo=64, phi=256, olo=1,
             ohi=128, trees="mixed", order="runs"),
        # Plain decoding of 32 prompts with eight answers each, slots taken as they came free.
        dict(name="shared_decode", kind="shared", groups=32, each=8, N=1, hq=28, hkv=4, d=128, page=16, plo=2048, phi=8192,
             olo=1000, ohi=8192, trees="full", order="any"),
        # Verification of 16 prompts with eight answers each, trees as the decode loop drafts them.
        dict(name="shared_tree", kind="shared", groups=16, each=8, N=64, hq=12, hkv=2, d=128, page=16, plo=2048, phi=4096,
             olo=500, ohi=4096, trees="mixed", order="runs"),
        # Many answers to one very long prompt, small trees.
        dict(name="shared_long", kind="shared", groups=1, each=64, N=8, hq=28, hkv=4, d=128, page=32, plo=32768, phi=32768,
             olo=100, ohi=4001, trees="mixed", order="runs"),
        # A small vocabulary, a handful of sequences.
        dict(name="sample_small", kind="sample", B=4, N=8, V=1024, dmax=4, rows="sharp", ruled=False),
        # The walk of the 256-sequence batch: most rows are sure of a few tokens, some are not.
        dict(name="sample_batch", kind="sample", B=256, N=64, V=152064, dmax=12, rows="mixed", ruled=False),
        # The same with penalties, biases and masks.
        dict(name="sample_rules", kind="sample", B=64, N=32, V=151936, dmax=8, rows="mixed", ruled=True),
        # An untrained policy, whose rows are all flat: what is kept is a large part of the vocabulary.
        dict(name="sample_flat", kind="sample", B=64, N=16, V=50001, dmax=6, rows="flat", ruled=False),
    ]


HEADS = ((4, 1, 64), (8, 8, 64), (12, 2, 128), (28, 4, 128), (32, 8, 128), (5, 1, 128), (24, 8, 64))


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("rope", "shared", "sample"))
    hq, hkv, d = rng.choice(HEADS)
    page = rng.choice((16, 16, 32, 64, 128))
    for _ in range(1000):
        if kind == "rope":
            rows = rng.choice(("trees", "trees", "prompts"))
            lo = _log(rng, 1, 500000)
            c = dict(kind=kind, to=rng.choice(("cache", "cache", "rows")), B=_log(rng, 1, 512),
                     T=_log(rng, 1, 256 if rows == "trees" else 4096), hq=hq, hkv=hkv, d=d,
                     rot=rng.choice((d, d, d // 2, d // 4)), pairs=rng.choice(("halves", "neighbours")), page=page, lo=lo,
                     hi=lo + _log(rng, 1, 500000), rows=rows)
            if c["B"] * c["T"] * (hq + 2 * hkv) * d <= 3.5e8 and c["B"] * (c["hi"] + c["T"]) / page <= 1e7:
                return c
        elif kind == "shared":
            plo, olo = _log(rng, 1, 32768), _log(rng, 1, 4096)
            c = dict(kind=kind, groups=_log(rng, 1, 64), each=_log(rng, 1, 64), N=_log(rng, 1, 128), hq=hq, hkv=hkv, d=d,
                     page=page, plo=plo, phi=min(32768, _log(rng, plo, 4 * plo)), olo=olo, ohi=_log(rng, olo + 1, 8 * olo + 8),
                     trees=rng.choice(("mixed", "mixed", "full")), order=rng.choice(("runs", "any")))
            B, T = c["groups"] * c["each"], c["phi"] + c["ohi"] + c["N"]
            w = work(c)
            if w["flops"] <= 3e11 and w["bytes"] <= 1.2e9 and B * T * hkv * d <= 2.2e9 and B * c["N"] * hq * T <= 1.2e9:
                return c
        else:
            c = dict(kind=kind, B=_log(rng, 1, 256), N=_log(rng, 1, 64), V=_log(rng, 1000, 152064), dmax=rng.randint(1, 12),
                     rows=rng.choice(("sharp", "mixed", "mixed", "flat")), ruled=rng.random() < 0.4)
            if c["B"] * (c["N"] + c["dmax"] + 1) * c["V"] <= 2.9e9:
                return c
    raise RuntimeError("no case drawn")


# --------------------------------------------------------------------------- sizes of a case

def _spread(lo, hi, n, shape="uniform"):
    """n lengths of [lo, hi]: the quantiles of the distribution (lognormal: median lo, cut at hi)."""
    q = [(i + 0.5) / n for i in range(n)]
    if shape == "uniform" or hi <= lo:
        return np.array([round(lo + x * (hi - lo)) for x in q], dtype=np.int64)
    sigma = math.log(hi / lo) / 3.0
    nd = statistics.NormalDist()
    v = [round(lo * math.exp(sigma * nd.inv_cdf(x))) for x in q]
    return np.clip(np.array(v, dtype=np.int64), 1, hi)


def _tree_sizes(trees, B, N):
    """Nodes of each tree.  "mixed": as the decode loop drafts them, 37% find
    nothing in their cache (the root alone), 22% fill the tree, the rest lie between."""
    q = (np.arange(B) + 0.5) / B
    if trees == "full":
        return np.full(B, N, dtype=np.int64)
    n = np.where(q < 0.37, 1, np.where(q > 0.78, N, 2 + (q - 0.37) / 0.41 * (N - 2)))
    return np.clip(np.round(n).astype(np.int64), 1, N)


def _row_counts(c):
    if c["rows"] == "trees":
        return _tree_sizes("mixed", c["B"], c["T"])
    return np.clip(_spread(c["T"] / 4, 1.05 * c["T"], c["B"]), 1, c["T"])


def _accepted(c):
    """Accepted tokens of each sequence: 55% stop at the root, each further
    level keeps 84% of the walks, at most dmax."""
    q = (np.arange(c["B"]) + 0.5) / c["B"]
    a = np.where(q < 0.55, 0, 1 + np.floor(np.log((1 - q) / 0.45) / math.log(0.84)))
    a = np.minimum(a, c["dmax"]).astype(np.int64)
    return np.minimum(a, _tree_sizes("mixed", c["B"], c["N"]) - 1)


# What requests ask for: (temperature, top-k, top-p, min-p); the last one, none of them.
ASKED = ((1.0, 0, 0.95, 0.0), (0.7, 50, 0.9, 0.0), (0.9, 0, 0.8, 0.0), (1.0, 20, 1.0, 0.0), (1.2, 0, 1.0, 0.05),
         (0.6, 200, 0.95, 0.01), (1.0, 1, 1.0, 0.0), (1.0, 0, 1.0, 0.0))


def work(case):
    c = case
    if c["kind"] == "rope":
        m = float(_row_counts(c).sum())
        heads = c["hq"] + (2 if c["to"] == "cache" else 1) * c["hkv"]
        return {"bytes": m * heads * c["d"] * 4, "flops": m * (c["hq"] + c["hkv"]) * c["rot"] * 3}
    if c["kind"] == "shared":
        B = c["groups"] * c["each"]
        P, o = _spread(c["plo"], c["phi"], c["groups"], "lognormal"), _spread(c["olo"], c["ohi"], B, "lognormal")
        n = _tree_sizes(c["trees"], B, c["N"])
        kv = float(P.sum() + o.sum() + n.sum()) * c["hkv"] * c["d"] * 4
        qo = float(n.sum()) * c["hq"] * c["d"] * 4
        return {"bytes": kv + qo, "flops": 4.0 * c["d"] * c["hq"] * float(n.sum()) * float(P.mean() + o.mean() + 4)}
    rows = float((_accepted(c) + 1).sum())
    # the row's logits; where nothing is asked for, its noise too; under rules its count words and mask bits
    per = 4 + 4 / len(ASKED) + (2 + 0.125 if c["ruled"] else 0)
    return {"bytes": rows * c["V"] * per, "flops": rows * c["V"] * 4}


# --------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).to(DEV)


def _vectors(shape, g, spread):
    """Queries, keys or values as a layer makes them: normal, each head dim with an amplitude of its own."""
    amp = torch.exp(torch.randn(shape[-1], generator=g, device=DEV) * spread)
    return (torch.randn(shape, generator=g, device=DEV) * amp).to(torch.bfloat16)


def _trees(n, N, rng):
    """Parents [B, N] and depths of random trees of n nodes each (-1 and 0 behind them)."""
    B, i = len(n), np.arange(N)
    par = np.maximum(i - rng.integers(1, 6, size=(B, N)), 0)
    par[:, 0] = -1
    par[i[None, :] >= n[:, None]] = -1
    depth = np.zeros((B, N), dtype=np.int64)
    for j in range(1, N):
        depth[:, j] = np.where(par[:, j] >= 0, depth[np.arange(B), np.maximum(par[:, j], 0)] + 1, 0)
    return par, depth


def _prepare_rope(c, s, rng, g):
    B, T, d, page = c["B"], c["T"], c["d"], c["page"]
    L, n = rng.permutation(_spread(c["lo"], c["hi"], B)), rng.permutation(_row_counts(c))
    # one projection gives queries, keys and values: a token's heads side by side
    qkv = _vectors((B, T, c["hq"] + 2 * c["hkv"], d), g, 0.3)
    s["q"], s["k"], s["v"] = qkv[:, :, :c["hq"]], qkv[:, :, c["hq"]:c["hq"] + c["hkv"]], qkv[:, :, c["hq"] + c["hkv"]:]
    s["counts"], s["ctx_len"] = _i32(n), _i32(L)
    s["depth"] = _i32(_trees(n, T, rng)[1]) if c["rows"] == "trees" else None
    # bases of short and of long contexts, the latter with the attention's temperature of a stretched context
    base, s["factor"] = (1e6, 1.0) if c["lo"] < 50000 else (5e6, 1.0625)
    s["inv_freq"] = torch.as_tensor(base ** (-np.arange(0, c["rot"], 2) / c["rot"]), dtype=torch.float32).to(DEV)
    s["q_out"] = torch.zeros((B, T, c["hq"], d), dtype=torch.bfloat16, device=DEV)
    if c["to"] == "rows":
        s["k_out"] = torch.zeros((B, T, c["hkv"], d), dtype=torch.bfloat16, device=DEV)
        return
    # the pool holds the pages that the step touches and one more, which belongs to nobody
    first, last = L // page, (L + T - 1) // page
    P = int((last - first + 1).sum())
    order, bt, at = rng.permutation(P), np.full((B, int(last.max()) + 1), -1, dtype=np.int32), 0
    for b in range(B):
        k = int(last[b] - first[b] + 1)
        bt[b, first[b]:last[b] + 1] = order[at:at + k]
        at += k
    s["bt"] = _i32(bt)
    s["pool"] = [_vectors((P + 1, c["hkv"], page, d), g, x) for x in (0.3, 0.0)]


def _prepare_shared(c, s, rng, g):
    G, N, page, hkv, d = c["groups"], c["N"], c["page"], c["hkv"], c["d"]
    B = G * c["each"]
    P = rng.permutation(_spread(c["plo"], c["phi"], G, "lognormal"))
    ids = np.repeat(np.arange(G), c["each"])
    if c["order"] == "any":
        ids = rng.permutation(ids)
    L = P[ids] + rng.permutation(_spread(c["olo"], c["ohi"], B, "lognormal"))
    n = rng.permutation(_tree_sizes(c["trees"], B, N))
    # whole pages of the prefix are the group's, the rest is each sequence's own
    whole, need = P // page, (L + N + page - 1) // page
    total = int(whole.sum() + (need - whole[ids]).sum())
    order, at = rng.permutation(total), 0
    heads = []
    for w in whole:
        heads.append(order[at:at + w])
        at += w
    bt = np.full((B, int(need.max())), -1, dtype=np.int32)
    for b in range(B):
        w, m = int(whole[ids[b]]), int(need[b])
        bt[b, :w] = heads[ids[b]]
        bt[b, w:m] = order[at:at + m - w]
        at += m - w
    s.update(bt=_i32(bt), ctx_len=_i32(L), n=_i32(n), parent=_i32(_trees(n, N, rng)[0]), ids=_i32(ids), prefix=_i32(P),
             scale=d ** -0.5, top=int(L.max()))
    s["pool"] = [_vectors((total, hkv, page, d), g, x) for x in (0.5, 0.0)]
    s["q"] = _vectors((B, N, c["hq"], d), g, 0.0)
    s["out"] = torch.zeros_like(s["q"])


def _paths(c, rng):
    """Trees with one path each that the walk follows: tokens, parents, sizes,
    nodes on the path [B, dmax + 1], their counts."""
    B, N, dmax = c["B"], c["N"], c["dmax"]
    n, acc = _tree_sizes("mixed", B, N), _accepted(c)
    order = rng.permutation(B)
    n, acc = n[order], acc[order]
    tok = rng.integers(0, c["V"], size=(B, N)).astype(np.int32)
    par = np.full((B, N), -1, dtype=np.int32)
    nodes = np.full((B, dmax + 1), -1, dtype=np.int32)
    back = rng.integers(1, 6, size=(B, N))
    for b in range(B):
        path = np.sort(rng.choice(np.arange(1, n[b]), size=acc[b], replace=False)) if acc[b] else np.zeros(0, np.int64)
        nodes[b, :acc[b]] = path
        depth, last, on = [0] * N, 0, set(int(x) for x in path)
        for i in range(1, int(n[b])):
            p = max(0, i - int(back[b, i]))
            if i in on:
                p, last = last, i
            elif depth[p] >= dmax:
                p = 0
            par[b, i] = p
            depth[i] = depth[p] + 1
        tok[b, n[b]:] = -1
    return tok, par, n, nodes, acc


def _as_words(w):
    """int32 0..65535 as the int16 with those bits."""
    return torch.where(w >= PROMPT, w - 2 * PROMPT, w).to(torch.int16)


def _prepare_sample(c, s, rng, g):
    B, N, V, dmax = c["B"], c["N"], c["V"], c["dmax"]
    tok, par, n, nodes, acc = _paths(c, rng)
    z = lambda *x: torch.zeros(x, dtype=torch.int32, device=DEV)
    s.update(tok=_i32(tok), par=_i32(par), n=_i32(n),
             out=dict(n_accepted=z(B), out_tokens=z(B, dmax + 1), out_nodes=z(B, dmax + 1), n_emitted=z(B)))
    s["gumbel"] = torch.empty((B, dmax + 1, V), device=DEV).exponential_(generator=g).log_().neg_()
    # probability falls with the rank of a token as rank ** -a: sure rows of a few tokens (a = 1.3 .. 3), flat ones
    # (0.3 .. 0.9), whose nucleus is a large part of the vocabulary; "mixed": one sequence in ten is flat
    q = (np.arange(B) + 0.5) / B
    a = 1.3 + 1.7 * q if c["rows"] == "sharp" else 0.3 + 0.6 * q if c["rows"] == "flat" else np.where(
        q < 0.1, 0.3 + 6 * q, 1.3 + 1.7 * q)
    a = rng.permutation(a)
    s["logits"] = torch.empty((B, N, V), device=DEV).exponential_(generator=g)
    s["logits"] *= torch.as_tensor(a, dtype=torch.float32, device=DEV)[:, None, None]
    # the policy follows the path, nearly always
    fb = np.repeat(np.arange(B), acc)
    fu = np.concatenate([np.concatenate([[0], nodes[b, :acc[b] - 1]]) if acc[b] else np.zeros(0) for b in range(B)])
    ft = np.concatenate([tok[b, nodes[b, :acc[b]]] for b in range(B)])
    sure = torch.as_tensor(a[fb] * math.log(V) + np.where(a[fb] < 1, 16, 8), dtype=torch.float32, device=DEV)
    fb, fu, ft = (torch.as_tensor(np.asarray(x, dtype=np.int64), device=DEV) for x in (fb, fu, ft))
    s["logits"][fb, fu, ft] = sure
    asked = np.array([ASKED[i % len(ASKED)] for i in range(B)])[rng.permutation(B)]
    f = lambda x: torch.as_tensor(x.astype(np.float32), device=DEV)
    s["inv_temperature"], s["top_p"], s["min_p"] = f(1 / asked[:, 0]), f(asked[:, 2]), f(asked[:, 3])
    s["top_k"] = _i32(asked[:, 1])
    if not c["ruled"]:
        return
    # a prompt of 1/64 of the vocabulary, outputs that repeat 1/256 of it one to nine times; 16 biases a sequence; half
    # of the sequences unconstrained, the others with about half of the tokens allowed
    u = torch.rand((B, V), generator=g, device=DEV)
    m = torch.randint(1, 10, (B, V), generator=g, device=DEV, dtype=torch.int32)
    s["seen"] = _as_words(torch.where(u < 1 / 256, m, 0) + torch.where((u > 1 / 512) & (u < 1 / 512 + 1 / 64), PROMPT, 0))
    pick = lambda *x: f(rng.choice(x, B))
    s["repetition"], s["frequency"], s["presence"] = pick(1.0, 1.05, 1.2), pick(0.0, 0.1, 0.3), pick(0.0, 0.2, 0.5)
    bt = np.sort(np.argsort(rng.random((B, 64)), axis=1)[:, :16], axis=1) * (V // 64)
    s["bias_at"], s["bias_tok"] = _i32(np.arange(B + 1) * 16), _i32(bt.reshape(-1))
    s["bias_val"] = f(rng.normal(0, 3, bt.size))
    W = (V + 31) // 32
    m = torch.randint(-2 ** 31, 2 ** 31, (B, N, W), generator=g, device=DEV).to(torch.int32)
    m[torch.as_tensor(rng.permutation(B)[: B // 2], device=DEV)] = -1
    m[fb, fu, ft // 32] = -1
    m[torch.as_tensor(rng.permutation(B)[: B // 32], device=DEV), -1] = 0  # a dead end
    # what the constraint forbids may hold anything
    s["logits"][:, :, V - 1] = float("nan")
    m[:, :, W - 1] &= (1 << ((V - 1) % 32)) - 1
    s["mask"] = m


def prepare(case, seed):
    s = {"case": case}
    make = {"rope": _prepare_rope, "shared": _prepare_shared, "sample": _prepare_sample}[case["kind"]]
    make(case, s, np.random.default_rng(seed), _gen(seed))
    return s


# --------------------------------------------------------------------------- the plain forms

def _split(x, c):
    """The first and second of each pair that turns together, and the dims that stay."""
    if c["pairs"] == "halves":
        return x[..., :c["rot"] // 2], x[..., c["rot"] // 2:c["rot"]], x[..., c["rot"]:]
    return x[..., 0:c["rot"]:2], x[..., 1:c["rot"]:2], x[..., c["rot"]:]


def _turned(x, c, cos, sin):
    """x [B, T, heads, d], cos and sin [B, T, 1, rot / 2]."""
    a, b, rest = _split(x, c)
    a, b = a * cos - b * sin, b * cos + a * sin
    both = torch.cat([a, b], -1) if c["pairs"] == "halves" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([both, rest], -1)


def _angles(s):
    c = s["case"]
    after = s["depth"] if s["depth"] is not None else torch.arange(c["T"], device=DEV)
    return ((s["ctx_len"][:, None] + after).double()[..., None] * s["inv_freq"].double())[:, :, None]


def _places(s):
    """Page and slot of every row; rows that are not written go to the page that belongs to nobody."""
    c = s["case"]
    p = s["ctx_len"][:, None] + torch.arange(c["T"], device=DEV)
    live = torch.arange(c["T"], device=DEV) < s["counts"][:, None]
    pg = s["bt"].gather(1, (p // c["page"]).long())
    return torch.where(live, pg, s["pool"][0].shape[0] - 1).long(), p % c["page"], live


def _plain_rope(s):
    c, ang = s["case"], _angles(s)
    cos, sin = ang.cos().float() * s["factor"], ang.sin().float() * s["factor"]
    live = (torch.arange(c["T"], device=DEV) < s["counts"][:, None])[..., None, None]
    q, k = (_turned(s[x].float(), c, cos, sin).to(torch.bfloat16) for x in "qk")
    s["q_out"].copy_(torch.where(live, q, s["q_out"]))
    if c["to"] == "rows":
        s["k_out"].copy_(torch.where(live, k, s["k_out"]))
        return
    pg, slot, _ = _places(s)
    for pool, x in zip(s["pool"], (k, s["v"])):
        pool[pg, :, slot] = x


def _plain_shared(s):
    c = s["case"]
    N, hq, hkv, d, page = c["N"], c["hq"], c["hkv"], c["d"], c["page"]
    B, T, G = c["groups"] * c["each"], s["top"], hq // hkv
    at = s["ctx_len"][:, None] + torch.arange(N, device=DEV)
    pg = s["bt"].gather(1, (at // page).long()).long()
    k, v = (torch.cat([x[s["bt"].clamp(min=0).long()].float().transpose(2, 3).reshape(B, -1, hkv, d)[:, :T],
                       x[pg, :, at % page].float()], 1).transpose(1, 2).contiguous() for x in s["pool"])
    q = s["q"].float().reshape(B, N, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, hkv, N, G, T + N)
    # a node sees the context and its ancestors: the closure of the parent relation by squaring
    see = (torch.eye(N, dtype=torch.bool, device=DEV) | (s["parent"][:, :, None] == torch.arange(N, device=DEV))).float()
    for _ in range(max(1, (N - 1).bit_length())):
        see = torch.matmul(see, see).clamp_(max=1)
    past = (torch.arange(T, device=DEV) < s["ctx_len"][:, None])[:, None].expand(B, N, T)
    hide = ~torch.cat([past, see > 0], 2)
    x = x.masked_fill_(hide[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    den = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hkv, -1, T + N), v) / den.view(B, hkv, -1, 1)
    o = o.view(B, hkv, N, G, d).permute(0, 2, 1, 3, 4).reshape(B, N, hq, d)
    live = torch.arange(N, device=DEV) < s["n"][:, None]
    return torch.where(live[..., None, None], o, 0).to(torch.bfloat16)


def _ruled(s, x, rows, u, count):
    """Logits x [B, V] of nodes u under the rules, forbidden ones as NaN."""
    c, col = s["case"], lambda k: s[k][:, None]
    said = s["seen"].int() & PROMPT != 0
    x = torch.where(said | (count > 0), torch.where(x > 0, x / col("repetition"), x * col("repetition")), x)
    x = x - col("frequency") * count
    x = torch.where(count > 0, x - col("presence"), x)
    x[torch.repeat_interleave(rows, 16), s["bias_tok"].long()] += s["bias_val"]
    at = torch.arange(c["V"], device=DEV)
    return torch.where((s["mask"][rows, u][:, at // 32] >> (at % 32)) & 1 == 1, x, math.nan)


def _plain_sample(s):
    c = s["case"]
    B, N, V, dmax = c["B"], c["N"], c["V"], c["dmax"]
    rows, node, rank = (torch.arange(n, device=DEV) for n in (B, N, V))
    u, live = torch.zeros(B, dtype=torch.long, device=DEV), torch.ones(B, dtype=torch.bool, device=DEV)
    out = {"n_accepted": torch.zeros(B, dtype=torch.int32, device=DEV),
           "n_emitted": torch.zeros(B, dtype=torch.int32, device=DEV),
           "out_tokens": torch.full((B, dmax + 1), -1, dtype=torch.int32, device=DEV),
           "out_nodes": torch.full((B, dmax + 1), -1, dtype=torch.int32, device=DEV)}
    count = (s["seen"].int() & (PROMPT - 1)) if c["ruled"] else None
    first = rank == 0
    top_k = torch.where(s["top_k"] > 0, s["top_k"], V)[:, None]
    top_p, min_p = s["top_p"].double()[:, None], s["min_p"].double()[:, None]
    for k in range(dmax + 1):  # (a level needs the token of the one before)
        x = s["logits"][rows, u]
        if c["ruled"]:
            x = _ruled(s, x, rows, u, count)
        z = x * s["inv_temperature"][:, None]
        z, idx = torch.sort(z.masked_fill_(z.isnan(), -math.inf), dim=1, descending=True, stable=True)
        less = z.double() - z[:, :1].double()  # NaN where every score is -inf
        keep = rank < top_k
        w = torch.where(keep, less.exp(), 0)
        mass = w.cumsum(1)
        before = torch.cat([torch.zeros_like(mass[:, :1]), mass[:, :-1]], 1)
        keep &= first | (top_p >= 1) | (before < top_p * mass[:, -1:])
        keep &= first | (min_p <= 0) | (less >= min_p.log())
        keep &= z > -math.inf
        score = torch.where(keep, z + s["gumbel"][:, k].gather(1, idx), -math.inf)
        top = score.amax(1, keepdim=True)
        none = top[:, 0] == -math.inf
        tok = torch.where(score == top, idx, V).amin(1)
        kid = (s["par"] == u[:, None]) & (s["tok"] == tok[:, None]) & (node < s["n"][:, None]) & (node > u[:, None])
        child = torch.where(kid, node, N).amin(1)
        go = live & ~none & (child < N) & (k < dmax)
        stop = live & ~go
        out["out_tokens"][:, k] = torch.where(live & ~none, tok, out["out_tokens"][:, k]).int()
        out["out_nodes"][:, k] = torch.where(go, child, out["out_nodes"][:, k]).int()
        out["n_accepted"] = torch.where(stop, k, out["n_accepted"])
        out["n_emitted"] = torch.where(stop, k + (~none).int(), out["n_emitted"])
        if c["ruled"]:
            count = count.scatter_add(1, tok[:, None], go[:, None].int())
        u, live = torch.where(go, child, u), go
    return out


# --------------------------------------------------------------------------- one pass

def _kept(s, key, make):
    """What a user's program makes once and keeps: a handle, a workspace, the walk's rules."""
    if key not in s:
        s[key] = make()
    return s[key]


def _own_rope(s):
    from paper_2601_09083_amd import srt
    c = s["case"]
    rope = _kept(s, "rope", lambda: srt.Rope(s["inv_freq"], interleaved=c["pairs"] == "neighbours", factor=s["factor"]))
    if c["to"] == "rows":
        srt.srt_rope_rows(rope, s["q"], s["k"], s["counts"], s["ctx_len"], depth=s["depth"], q_out=s["q_out"],
                          k_out=s["k_out"])
    else:
        srt.srt_rope_append(rope, s["q"], s["k"], s["v"], s["counts"], s["pool"][0], s["pool"][1], s["bt"], s["ctx_len"],
                            depth=s["depth"], q_out=s["q_out"])


def _own_shared(s):
    from paper_2601_09083_amd import srt
    c = s["case"]
    k, v = s["pool"]
    need = lambda: torch.empty(srt.srt_tree_attn_shared_scratch_bytes(
        c["groups"] * c["each"], c["N"], c["hq"], c["hkv"], c["d"], c["page"], s["bt"].shape[1], c["groups"]),
        dtype=torch.uint8, device=DEV)
    return srt.srt_tree_attn_shared(s["q"], k, v, s["bt"], s["ctx_len"], s["parent"], s["n"], s["ids"], s["prefix"],
                                    s["scale"], out=s["out"], scratch=_kept(s, "scratch", need))


def _own_sample(s):
    from paper_2601_09083_amd import srt
    c = s["case"]
    asked = _kept(s, "asked", lambda: srt.Sampling(inv_temperature=s["inv_temperature"], top_k=s["top_k"],
                                                   top_p=s["top_p"], min_p=s["min_p"]))
    rules = _kept(s, "rules", lambda: srt.Rules(
        seen=s["seen"], repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
        bias_offsets=s["bias_at"], bias_tokens=s["bias_tok"], bias_values=s["bias_val"], mask=s["mask"])
        if c["ruled"] else None)
    return srt.srt_accept_sample(s["logits"], s["gumbel"], asked, s["tok"], s["par"], s["n"], c["dmax"], rules=rules,
                                 out=s["out"])


def run(s):
    kind = s["case"]["kind"]
    if kind == "shared":
        return _own_shared(s) if own else _plain_shared(s)
    if kind == "sample":
        return _own_sample(s) if own else _plain_sample(s)
    if own:
        _own_rope(s)
    else:
        _plain_rope(s)
    if s["case"]["to"] == "rows":
        return dict(q=s["q_out"], k=s["k_out"])
    return dict(q=s["q_out"], k_cache=s["pool"][0][:-1], v_cache=s["pool"][1][:-1])


# --------------------------------------------------------------------------- the same in 64 bits

def _exact_rope(s):
    c = s["case"]
    B, T, rot = c["B"], c["T"], c["rot"]
    after = s["depth"].double() if s["depth"] is not None else torch.arange(T, device=DEV, dtype=torch.float64).expand(B, T)
    ang = (s["ctx_len"].double()[:, None] + after)[:, :, None, None] * s["inv_freq"].double()
    i = torch.arange(rot // 2, device=DEV)
    lo, hi = (i, i + rot // 2) if c["pairs"] == "halves" else (2 * i, 2 * i + 1)
    live = torch.arange(T, device=DEV) < s["counts"][:, None]
    turn = torch.polar(torch.full_like(ang, s["factor"]), ang)
    got = []
    for x in (s["q"], s["k"]):
        y = x.double()
        z = torch.complex(y[..., lo], y[..., hi]) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        got.append(y.masked_fill_(~live[..., None, None], 0))
    if c["to"] == "rows":
        return dict(q=got[0], k=got[1])
    pools = [x.double() for x in s["pool"]]
    pg, slot, _ = _places(s)
    pools[0][pg, :, slot] = got[1]
    pools[1][pg, :, slot] = s["v"].double()
    return dict(q=got[0], k_cache=pools[0][:-1], v_cache=pools[1][:-1])


def _exact_shared(s):
    c = s["case"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    G, d, hkv, page = c["hq"] // c["hkv"], c["d"], c["hkv"], c["page"]
    L, n, par = s["ctx_len"].tolist(), s["n"].tolist(), s["parent"].cpu().numpy()
    for b in range(len(L)):
        m, total = n[b], L[b] + n[b]
        ids = s["bt"][b, :(total + page - 1) // page].long()
        k, v = (x[ids].double().transpose(0, 1).reshape(hkv, -1, d)[:, :total] for x in s["pool"])
        see = np.zeros((m, m), dtype=bool)
        for i in range(m):
            see[i] = see[par[b, i]] if i else False
            see[i, i] = True
        q = s["q"][b, :m].double().reshape(m, hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, m * G, d)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).mul_(s["scale"])
        x[:, :, L[b]:].masked_fill_(torch.as_tensor(~see, device=DEV).repeat_interleave(G, 0)[None], -math.inf)
        o = torch.matmul(torch.softmax(x, -1), v)
        out[b, :m] = o.reshape(hkv, m, G, d).permute(1, 0, 2, 3).reshape(m, c["hq"], d)
    return out


def exact(case, seed):
    if case["kind"] == "rope":
        return _exact_rope(prepare(case, seed))
    if case["kind"] == "shared":
        return _exact_shared(prepare(case, seed))
    return None  # tokens: whole numbers

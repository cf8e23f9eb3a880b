"""The operators of the 8-bit KV cache and of the sampling rules, as measurable cases.

Each case is one operator as a decode loop uses it, in a plain form of
elementary torch operations and, where ``own`` is true, through the public
binding ``paper_2601_09083_amd.srt``:

* ``attn``    srt_tree_attn_quant: every tree node against a paged cache held in
  8 bits (a scale for each page and KV head) and the tree's own K/V;
* ``append``  srt_kv_append: new tokens into that cache (a page is quantised
  when it is full, the rest waits in bf16), then srt_kv_read: the positions
  just written, back as bf16;
* ``commit``  srt_commit_quant: the accepted path into the cache, the draft inputs
  advanced, then the touched positions read back;
* ``rules``   srt_accept_rules: the acceptance walk with penalties for repeated
  tokens, biases and grammar masks on the rows it visits;
* ``seen``    srt_seen_add: the token counts that the penalties read.

Lengths, tree sizes and accepted lengths are the quantiles of their
distributions in an order drawn from the seed, so that the work of a case does
not depend on the seed.
"""
import math
import statistics

import numpy as np
import torch

own = False

DEV = "cuda"
LARGEST = {"e4m3": 448.0, "int8": 127.0}  # what a page's largest value is scaled to
LEAST = 2.0 ** -60                        # amplitude below which a page's scale does not go
PROMPT = 0x8000                           # bit of a seen word: the token is in the prompt


def listed():
    return [
        # Four short sequences, one small layer: the smallest step, where launches count.
        dict(name="attn_small", kind="attn", kv="e4m3", B=4, N=8, hq=4, hkv=1, d=64, page=16,
             ctx="uniform", lo=128, hi=512, trees="mixed"),
        # Plain decoding of one token for each of 256 sequences, long-tailed contexts: the cache is read at full rate.
        dict(name="attn_decode", kind="attn", kv="e4m3", B=256, N=1, hq=28, hkv=4, d=128, page=16,
             ctx="lognormal", lo=4096, hi=16384, trees="full"),
        # Verification of a rollout batch with trees as the decode loop drafts them.
        dict(name="attn_tree", kind="attn", kv="e4m3", B=64, N=64, hq=28, hkv=4, d=128, page=16,
             ctx="lognormal", lo=4096, hi=16384, trees="mixed"),
        # Long-tail run-ahead: few sequences, long contexts, very wide trees, codes of int8.
        dict(name="attn_longtail", kind="attn", kv="int8", B=8, N=256, hq=28, hkv=4, d=128, page=16,
             ctx="uniform", lo=16384, hi=32768, trees="wide"),
        # Prompts of up to 4k tokens enter the cache.
        dict(name="append_prompts", kind="append", kv="e4m3", B=32, T=4096, hkv=4, d=128, page=16, lo=0, hi=64),
        # A few tokens each (a decode without drafts, a tool's short answer), odd numbers of them.
        dict(name="append_short", kind="append", kv="int8", B=37, T=7, hkv=2, d=128, page=32, lo=1, hi=999),
        # The accepted paths of the 256-sequence batch.
        dict(name="commit_batch", kind="commit", kv="e4m3", B=256, N=64, hkv=4, d=128, page=16, dmax=12, qmax=8,
             lo=1, hi=777),
        # The same for a handful of small sequences.
        dict(name="commit_small", kind="commit", kv="int8", B=4, N=8, hkv=1, d=64, page=16, dmax=4, qmax=8,
             lo=1, hi=99),
        # Sampled walk of the 256-sequence batch under penalties, biases and grammar masks.
        dict(name="rules_batch", kind="rules", B=256, N=64, V=152064, dmax=12, sampled=True, bias=64, masked=True),
        # Greedy walk of a small vocabulary, penalties only.
        dict(name="rules_small", kind="rules", B=4, N=8, V=1024, dmax=4, sampled=False, bias=0, masked=False),
        # Prompts of new sequences entered into their count rows.
        dict(name="seen_prompts", kind="seen", B=256, T=4096, V=152064, prompt=True, reset=True),
        # The emitted tokens of one step.
        dict(name="seen_step", kind="seen", B=256, T=13, V=152064, prompt=False, reset=False),
    ]


HEADS = ((4, 1, 64), (8, 8, 64), (12, 2, 128), (28, 4, 128), (32, 8, 128), (5, 1, 128), (24, 8, 64))


def _log(rng, lo, hi):
    """A whole number of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("attn", "append", "commit", "rules", "seen"), (8, 3, 3, 4, 2))[0]
    kv = rng.choice(("e4m3", "int8"))
    hq, hkv, d = rng.choice(HEADS)
    page = rng.choice((16, 16, 32, 64, 128))
    for _ in range(1000):
        if kind == "attn":
            lo = _log(rng, 1, 16384)
            c = dict(kind=kind, kv=kv, B=_log(rng, 1, 512), N=_log(rng, 1, 256), hq=hq, hkv=hkv, d=d, page=page,
                     ctx=rng.choice(("uniform", "lognormal")), lo=lo, hi=min(32768, _log(rng, lo + 1, 8 * lo + 8)),
                     trees=rng.choice(("mixed", "mixed", "full", "wide")))
            w = work(c)
            T = c["hi"] + c["N"]
            if (w["flops"] <= 5e11 and w["bytes"] <= 1.6e9 and c["B"] * T * hkv * d <= 2.2e9
                    and c["B"] * c["N"] * hq * T <= 1.9e9):
                return c
        elif kind == "append":
            lo = rng.choice((0, _log(rng, 1, 1000)))
            c = dict(kind=kind, kv=kv, B=_log(rng, 1, 512), T=_log(rng, 1, 8192), hkv=hkv, d=d, page=page, lo=lo,
                     hi=lo + _log(rng, 1, 1000))
            if c["B"] * (c["T"] + c["hi"]) * hkv * d <= 6.8e7:
                return c
        elif kind == "commit":
            lo = _log(rng, 1, 1000)
            c = dict(kind=kind, kv=kv, B=_log(rng, 1, 256), N=_log(rng, 1, 256), hkv=hkv, d=d, page=page,
                     dmax=rng.randint(1, 16), qmax=rng.choice((4, 8, 16)), lo=lo, hi=lo + _log(rng, 1, 1000))
            if c["B"] * (c["N"] + c["hi"]) * hkv * d <= 1.2e8:
                return c
        elif kind == "rules":
            c = dict(kind=kind, B=_log(rng, 1, 256), N=_log(rng, 1, 64), V=_log(rng, 1000, 152064),
                     dmax=rng.randint(1, 12), sampled=rng.random() < 0.6, bias=rng.choice((0, 0, 1, 17, 300)),
                     masked=rng.random() < 0.6)
            if c["B"] * (c["N"] + c["dmax"] + 1) * c["V"] <= 2.9e9:
                return c
        else:
            return dict(kind=kind, B=_log(rng, 1, 256), T=_log(rng, 1, 4096), V=_log(rng, 1000, 152064),
                        prompt=rng.random() < 0.5, reset=rng.random() < 0.5)
    raise RuntimeError("no case drawn")


# --------------------------------------------------------------------------- sizes of a case

def _lens(c, n):
    """n context lengths: the quantiles of the case's distribution."""
    q = [(i + 0.5) / n for i in range(n)]
    if c.get("ctx", "uniform") == "uniform":
        return np.array([round(c["lo"] + x * (c["hi"] - c["lo"])) for x in q], dtype=np.int64)
    sigma = math.log(c["hi"] / c["lo"]) / 3.0  # log-normal with median lo, cut at hi
    nd = statistics.NormalDist()
    v = [round(c["lo"] * math.exp(sigma * nd.inv_cdf(x))) for x in q]
    return np.clip(np.array(v, dtype=np.int64), 1, c["hi"])


def _tree_sizes(trees, B, N):
    """Nodes of each tree.  "mixed": as the decode loop drafts them, 37% find
    nothing in their cache (the root alone), 22% fill the tree, the rest lie
    between; "wide": N/4 .. N nodes."""
    q = (np.arange(B) + 0.5) / B
    if trees == "full":
        n = np.full(B, N)
    elif trees == "wide":
        n = N / 4 + q * (3 * N / 4)
    else:
        n = np.where(q < 0.37, 1, np.where(q > 0.78, N, 2 + (q - 0.37) / 0.41 * (N - 2)))
    return np.clip(np.round(n).astype(np.int64), 1, N)


def _accepted(c):
    """Accepted tokens of each sequence: 55% stop at the root, each further
    level keeps 84% of the walks, at most dmax."""
    q = (np.arange(c["B"]) + 0.5) / c["B"]
    a = np.where(q < 0.55, 0, 1 + np.floor(np.log((1 - q) / 0.45) / math.log(0.84)))
    a = np.minimum(a, c["dmax"]).astype(np.int64)
    return np.minimum(a, _tree_sizes("mixed", c["B"], c["N"]) - 1)


def _counts(c):
    """New tokens of each sequence: T/4 .. T (0 or 1 where T is small)."""
    q = (np.arange(c["B"]) + 0.5) / c["B"]
    return np.minimum(np.round(c["T"] * (0.25 + 0.8 * q)).astype(np.int64), c["T"])


def work(case):
    c = case
    if c["kind"] == "attn":
        L, n = _lens(c, c["B"]), _tree_sizes(c["trees"], c["B"], c["N"])
        full = float((L // c["page"] * c["page"]).sum())
        kv = full * c["hkv"] * (2 * c["d"] + 8 / c["page"])
        kv += (float(L.sum()) - full + float(n.sum())) * c["hkv"] * c["d"] * 4
        qo = float(n.sum()) * c["hq"] * c["d"] * 4
        return {"bytes": kv + qo, "flops": 4.0 * c["d"] * c["hq"] * float(n.sum()) * float(L.mean() + 4)}
    if c["kind"] in ("append", "commit"):
        m = float(_counts(c).sum()) if c["kind"] == "append" else float((_accepted(c) + 1).sum())
        # the rows read in bf16 and written in 8 bits, then read so and given in bf16
        return {"bytes": m * c["hkv"] * c["d"] * 2 * (3 + 3), "flops": m * c["hkv"] * c["d"] * 2 * 4}
    if c["kind"] == "rules":
        rows = float((_accepted(c) + 1).sum())
        per = 4 + 2 + (4 if c["sampled"] else 0) + (0.125 if c["masked"] else 0)
        return {"bytes": rows * c["V"] * per, "flops": rows * c["V"] * 4}
    m = float(_counts(c).sum())
    return {"bytes": m * 4 + (c["B"] * c["V"] * 2.0 if c["reset"] else m * 4), "flops": m}


# --------------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32).to(DEV)


def _vectors(shape, g, spread):
    """Keys or values as a layer makes them: normal, each head dim with an amplitude of its own."""
    amp = torch.exp(torch.randn(shape[-1], generator=g, device=DEV) * spread)
    return (torch.randn(shape, generator=g, device=DEV) * amp).to(torch.bfloat16)


def _pages(P, hkv, page, d, kv, g, spread):
    """A pool of quantised pages and their scales (the last page belongs to nobody)."""
    x = _vectors((P, hkv, page, d), g, spread).float()
    return _quantised(x, kv)


def _cache(c, L, room, g, rng):
    """The cache of sequences of lengths L with table room for `room` more
    tokens each, pages in random order."""
    B, page, hkv, d = len(L), c["page"], c["hkv"], c["d"]
    per = (L + room) // page
    P, mp = int(per.sum()), max(1, int(per.max()))
    order = rng.permutation(P).astype(np.int32)
    bt = np.full((B, mp), -1, dtype=np.int32)
    ends = np.cumsum(per)
    bt[np.arange(mp)[None, :] < per[:, None]] = order
    assert int(ends[-1]) == P
    k, ks = _pages(P + 1, hkv, page, d, c["kv"], g, 0.5)
    v, vs = _pages(P + 1, hkv, page, d, c["kv"], g, 0.0)
    tail = torch.stack([_vectors((B, hkv, page, d), g, s) for s in (0.5, 0.0)])
    return dict(k=k, v=v, ks=ks, vs=vs, bt=_i32(bt), tail=tail)


def _paths(c, rng):
    """Trees with one path each that the walk follows: tokens, parents, sizes,
    accepted nodes [B, dmax + 1], accepted counts."""
    B, N, dmax = c["B"], c["N"], c["dmax"]
    n, acc = _tree_sizes("mixed", B, N), _accepted(c)
    order = rng.permutation(B)
    n, acc = n[order], acc[order]
    tok = rng.integers(0, c.get("V", 1 << 15), size=(B, N)).astype(np.int32)
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


def _walk_outputs(B, dmax):
    z = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    return dict(n_accepted=z(B), out_tokens=z(B, dmax + 1), out_nodes=z(B, dmax + 1), n_emitted=z(B))


def _seen_rows(B, V, g):
    """Count rows of running sequences: a prompt of 1/64 of the vocabulary,
    outputs that repeat 1/128 of it one to nine times."""
    u = torch.rand((B, V), generator=g, device=DEV)
    n = torch.randint(1, 10, (B, V), generator=g, device=DEV, dtype=torch.int32)
    w = torch.where(u < 1 / 128, n, 0) + torch.where((u > 1 / 256) & (u < 1 / 256 + 1 / 64), PROMPT, 0)
    return _as_words(w)


def _as_words(w):
    """int32 0..65535 as the int16 with those bits."""
    return torch.where(w >= PROMPT, w - 2 * PROMPT, w).to(torch.int16)


def prepare(case, seed):
    c, s = case, {"case": case}
    rng, g = np.random.default_rng(seed), _gen(seed)
    B = c["B"]
    if c["kind"] == "attn":
        N, hkv, d = c["N"], c["hkv"], c["d"]
        L, n = rng.permutation(_lens(c, B)), rng.permutation(_tree_sizes(c["trees"], B, N))
        i = np.arange(N)
        par = np.maximum(i - rng.integers(1, 6, size=(B, N)), 0)
        par[:, 0] = -1
        par[i[None, :] >= n[:, None]] = -1
        s.update(_cache(c, L, 0, g, rng), ctx_len=_i32(L), parent=_i32(par), n=_i32(n), scale=d ** -0.5)
        # queries, keys and values of the tree as one projection gives them: a token's heads side by side
        qkv = _vectors((B, N, (c["hq"] + 2 * hkv), d), g, 0.0)
        s["q"] = qkv[:, :, :c["hq"]].contiguous()
        s["k_new"], s["v_new"] = qkv[:, :, c["hq"]:c["hq"] + hkv], qkv[:, :, c["hq"] + hkv:]
        s["out"] = torch.zeros_like(s["q"])
    elif c["kind"] in ("append", "commit"):
        L = rng.permutation(_lens(c, B))
        T = c["T"] if c["kind"] == "append" else c["N"]
        s.update(_cache(c, L, T if c["kind"] == "append" else c["dmax"] + 1, g, rng))
        s["k_new"], s["v_new"] = (_vectors((B, T, c["hkv"], c["d"]), g, x) for x in (0.5, 0.0))
        s["tail0"] = s["tail"].clone()  # (each pass writes the same tokens again)
        W = c["page"] + (T if c["kind"] == "append" else c["dmax"] + 1)
        s["out"] = [torch.zeros((B, W, c["hkv"], c["d"]), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        s["start"] = _i32(L // c["page"] * c["page"])
        if c["kind"] == "append":
            s["counts"] = _i32(rng.permutation(_counts(c)))
            s["state0"] = _i32(L)
            s["state"] = s["state0"].clone()
            s["ctx_len"] = s["state"]
        else:
            tok, par, n, nodes, acc = _paths(c, rng)
            emitted = np.where(np.arange(c["dmax"] + 1)[None] <= acc[:, None],
                               rng.integers(0, 1 << 15, (B, c["dmax"] + 1)), -1)
            s.update(nodes=_i32(nodes), acc=_i32(acc), emitted=_i32(emitted))
            old = rng.integers(0, 1 << 15, (B, c["qmax"]))
            old[np.arange(c["qmax"])[None] < c["qmax"] - L[:, None]] = -1
            s["state0"] = _i32(np.concatenate([L, L, old.reshape(-1)]))
            s["state"] = s["state0"].clone()
            s["ctx_len"], s["draft_len"] = s["state"][:B], s["state"][B:2 * B]
            s["ctx_tail"] = s["state"][2 * B:].view(B, c["qmax"])
    elif c["kind"] == "rules":
        N, V = c["N"], c["V"]
        tok, par, n, nodes, acc = _paths(c, rng)
        s.update(tok=_i32(tok), par=_i32(par), n=_i32(n), out=_walk_outputs(B, c["dmax"]))
        s["gumbel"] = (torch.empty((B, c["dmax"] + 1, V), device=DEV).exponential_(generator=g).log_().neg_()
                       if c["sampled"] else None)
        s["logits"] = torch.randn((B, N, V), generator=g, device=DEV).mul_(2.0)
        s["seen"] = _seen_rows(B, V, g)
        # the policy follows the path; at every node a token said before would win by a little without its penalty
        fb = np.repeat(np.arange(B), acc)
        fu = np.concatenate([np.concatenate([[0], nodes[b, :acc[b] - 1]]) if acc[b] else np.zeros(0) for b in range(B)])
        ft = np.concatenate([tok[b, nodes[b, :acc[b]]] for b in range(B)])
        rival = rng.integers(0, V, B)
        s["seen"][torch.arange(B, device=DEV), torch.as_tensor(rival, device=DEV)] = 3
        s["logits"][torch.arange(B, device=DEV), :, torch.as_tensor(rival, device=DEV)] = 62.0
        fb, fu, ft = (torch.as_tensor(np.asarray(x, dtype=np.int64), device=DEV) for x in (fb, fu, ft))
        s["logits"][fb, fu, ft] = 66.0
        s["repetition"] = torch.as_tensor(rng.choice([1.0, 1.05, 1.2], B).astype(np.float32), device=DEV)
        s["frequency"] = torch.as_tensor(rng.choice([0.0, 0.3, 1.5], B).astype(np.float32), device=DEV)
        s["presence"] = torch.as_tensor(rng.choice([0.0, 0.5, 4.0], B).astype(np.float32), device=DEV)
        s["bias_at"] = s["bias_tok"] = s["bias_val"] = s["mask"] = None
        if c["bias"]:
            bt = np.sort(np.argsort(rng.random((B, min(V, 4 * c["bias"]))), axis=1)[:, :c["bias"]], axis=1)
            bt = np.minimum(bt * max(1, V // (4 * c["bias"])), V - 1)
            s["bias_at"] = _i32(np.arange(B + 1) * c["bias"])
            s["bias_tok"] = _i32(bt.reshape(-1))
            s["bias_val"] = torch.as_tensor(rng.normal(0, 3, bt.size).astype(np.float32), device=DEV)
        if c["masked"]:
            # half of the sequences unconstrained, the others with about half of the tokens allowed
            W = (V + 31) // 32
            m = torch.randint(-2 ** 31, 2 ** 31, (B, N, W), generator=g, device=DEV).to(torch.int32)
            m[torch.as_tensor(rng.permutation(B)[: B // 2], device=DEV)] = -1
            m[fb, fu, ft // 32] = -1
            m[torch.as_tensor(rng.permutation(B)[: B // 32], device=DEV), -1] = 0  # a dead end
            s["mask"] = m
            # what the constraint forbids may hold anything
            s["logits"][:, :, V - 1] = float("nan")
            if V % 32:
                m[:, :, W - 1] &= (1 << (V % 32 - 1)) - 1
            else:
                m[:, :, W - 1] &= 0x7FFFFFFF
    else:
        words = torch.randint(0, c["V"], (B, c["T"]), generator=g, device=DEV, dtype=torch.int32)
        common = torch.randint(0, min(64, c["V"]), (B, c["T"]), generator=g, device=DEV, dtype=torch.int32)
        pick = torch.rand((B, c["T"]), generator=g, device=DEV) < 0.4
        s["tokens"] = torch.where(pick, common, words)
        s["lengths"] = _i32(rng.permutation(_counts(c)))
        s["seen"] = _seen_rows(B, c["V"], g)
    return s


# --------------------------------------------------------------------------- the plain forms

def _quantised(x, kv):
    """x [..., page, d] fp32 in 8 bits with a scale for each [...]."""
    top = LARGEST[kv]
    amp = x.abs().amax((-2, -1)).clamp_(min=LEAST)
    top_t = torch.full_like(amp, top)
    y = (x * (top_t / amp)[..., None, None]).clamp_(-top, top)
    q = y.to(torch.float8_e4m3fn) if kv == "e4m3" else y.round_().to(torch.int8)
    return q, amp / top_t


def _context(s, which, rows):
    """The first `rows` context positions of every sequence, [B, rows, Hkv, d] fp32
    (rows past a sequence's length hold anything finite)."""
    c, i = s["case"], 0 if which == "k" else 1
    bt = s["bt"].clamp(min=0).long()
    x = s[which][bt].float() * s[which + "s"][bt][..., None, None]       # [B, pages, Hkv, page, d]
    x = x.transpose(2, 3).reshape(c["B"], -1, c["hkv"], c["d"])
    x = torch.cat([x, x.new_zeros(c["B"], max(0, rows - x.shape[1]), c["hkv"], c["d"])], 1)[:, :rows]
    at = torch.arange(rows, device=DEV)
    open_ = (at >= (s["ctx_len"] // c["page"] * c["page"])[:, None])[..., None, None]
    tail = s["tail"][i].transpose(1, 2)[:, at % c["page"]].float()
    return torch.where(open_, tail, x)


def _plain_attn(s):
    c = s["case"]
    B, N, hq, hkv, d = c["B"], c["N"], c["hq"], c["hkv"], c["d"]
    T = max(1, c["hi"])
    k, v = (torch.cat([_context(s, x, T), s[x + "_new"].float()], 1).transpose(1, 2).contiguous() for x in "kv")
    q = s["q"].float().reshape(B, N, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    x = torch.matmul(q, k.transpose(2, 3)).mul_(s["scale"]).view(B, hkv, N, hq // hkv, T + N)
    # a node sees the context and its ancestors: the closure of the parent relation by squaring
    eye = torch.eye(N, dtype=torch.bool, device=DEV)
    see = (eye | (s["parent"][:, :, None] == torch.arange(N, device=DEV))).float()
    for _ in range(max(1, (N - 1).bit_length())):
        see = torch.matmul(see, see).clamp_(max=1)
    past = (torch.arange(T, device=DEV) < s["ctx_len"][:, None])[:, None].expand(B, N, T)
    hide = ~torch.cat([past, see > 0], 2)
    x = x.masked_fill_(hide[:, None, :, None], -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True)).exp_()
    den = x.sum(-1, keepdim=True)
    o = torch.matmul(x.view(B, hkv, -1, T + N), v) / den.view(B, hkv, -1, 1)
    o = o.view(B, hkv, N, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, N, hq, d)
    live = torch.arange(N, device=DEV) < s["n"][:, None]
    return torch.where(live[..., None, None], o, 0).to(torch.bfloat16)


def _plain_write(s, rows, count):
    """count[b] of the new rows rows[b, :] follow the context; full pages are quantised."""
    c = s["case"]
    B, page, hkv, d = c["B"], c["page"], c["hkv"], c["d"]
    first, have = s["ctx_len"] // page, s["ctx_len"] % page
    m = rows.shape[1]
    W = (page - 1 + m + page - 1) // page * page
    at = torch.arange(W, device=DEV)
    src = (at - have[:, None]).clamp(0, m - 1)
    src = rows.gather(1, src)
    full = (torch.arange(W // page, device=DEV) + 1) * page <= (have + count)[:, None]
    slot = first[:, None] + torch.arange(W // page, device=DEV)
    last = s["bt"].shape[1] - 1
    to = torch.where(full, s["bt"].gather(1, slot.clamp(max=last).long()), s["k"].shape[0] - 1).reshape(-1).long()
    rest = (have + count) // page * page  # first row of the page that stays open
    for i, which in enumerate("kv"):
        new = s[which + "_new"].gather(1, src[..., None, None].expand(-1, -1, hkv, d))
        old = s["tail"][i].transpose(1, 2)[:, at % page]
        x = torch.where((at < have[:, None])[..., None, None], old, new)
        q, scale = _quantised(x.view(B, W // page, page, hkv, d).transpose(2, 3).float(), c["kv"])
        # (a page that is not full goes to the spare one, which belongs to nobody)
        s[which].view(torch.uint8)[to] = q.reshape(-1, hkv, page, d).view(torch.uint8)
        s[which + "s"][to] = scale.reshape(-1, hkv)
        left = (rest[:, None] + torch.arange(page, device=DEV)).clamp(max=W - 1).long()
        s["tail"][i].copy_(x.gather(1, left[..., None, None].expand(-1, -1, hkv, d)).transpose(1, 2))
    s["ctx_len"] += count


def _plain_read(s, which, out):
    """Positions start + t < ctx_len as bf16."""
    c, W = s["case"], out.shape[1]
    p = s["start"][:, None] + torch.arange(W, device=DEV)
    slot = (p // c["page"]).clamp(max=s["bt"].shape[1] - 1).long()
    pg = s["bt"].gather(1, slot).clamp(min=0).long()
    x = s[which][pg, :, p % c["page"]].float() * s[which + "s"][pg][..., None]
    tail = s["tail"]["kv".index(which)]
    t = tail[torch.arange(c["B"], device=DEV)[:, None], :, p % c["page"]].float()
    x = torch.where((p >= (s["ctx_len"] // c["page"] * c["page"])[:, None])[..., None, None], t, x)
    return torch.where((p < s["ctx_len"][:, None])[..., None, None], x, 0).to(torch.bfloat16)


def _plain_rules(s):
    c = s["case"]
    B, N, V, dmax = c["B"], c["N"], c["V"], c["dmax"]
    rows = torch.arange(B, device=DEV)
    word = s["seen"].int() & 0xFFFF
    said, count = word >= PROMPT, word & (PROMPT - 1)
    rep, fre, pre = (s[k][:, None] for k in ("repetition", "frequency", "presence"))
    node, at = torch.arange(N, device=DEV), torch.arange(V, device=DEV)
    u, live = torch.zeros(B, dtype=torch.long, device=DEV), torch.ones(B, dtype=torch.bool, device=DEV)
    out = {"n_accepted": torch.zeros(B, dtype=torch.int32, device=DEV),
           "n_emitted": torch.zeros(B, dtype=torch.int32, device=DEV),
           "out_tokens": torch.full((B, dmax + 1), -1, dtype=torch.int32, device=DEV),
           "out_nodes": torch.full((B, dmax + 1), -1, dtype=torch.int32, device=DEV)}
    bias_row = None
    if s["bias_at"] is not None:
        bias_row = torch.repeat_interleave(rows, c["bias"])
    for k in range(dmax + 1):  # (a level needs the token of the one before)
        x = s["logits"][rows, u]
        x = torch.where(said | (count > 0), torch.where(x > 0, x / rep, x * rep), x)
        x = x - fre * count
        x = torch.where(count > 0, x - pre, x)
        if bias_row is not None:
            x[bias_row, s["bias_tok"].long()] += s["bias_val"]
        if s["gumbel"] is not None:
            x = x * 0.9 + s["gumbel"][:, k]
        bad = x.isnan()
        if s["mask"] is not None:
            bad |= (s["mask"][rows, u][:, at // 32] >> (at % 32)) & 1 == 0
        x = x.masked_fill(bad, -math.inf)
        top = x.amax(-1, keepdim=True)
        tok = torch.where(x == top, at, V).amin(-1)
        none = top[:, 0] == -math.inf
        kid = (s["par"] == u[:, None]) & (s["tok"] == tok[:, None]) & (node < s["n"][:, None]) & (node > u[:, None])
        child = torch.where(kid, node, N).amin(-1)
        go = live & ~none & (child < N) & (k < dmax)
        stop = live & ~go
        out["out_tokens"][:, k] = torch.where(live & ~none, tok, out["out_tokens"][:, k]).int()
        out["out_nodes"][:, k] = torch.where(go, child, out["out_nodes"][:, k]).int()
        out["n_accepted"] = torch.where(stop, k, out["n_accepted"])
        out["n_emitted"] = torch.where(stop, k + (~none).int(), out["n_emitted"])
        count = count.scatter_add(1, tok[:, None], go[:, None].int())
        u, live = torch.where(go, child, u), go
    return out


def _plain_seen(s):
    c = s["case"]
    ok = (torch.arange(c["T"], device=DEV) < s["lengths"][:, None]).int()
    n = torch.zeros((c["B"], c["V"]), dtype=torch.int32, device=DEV).scatter_add_(1, s["tokens"].long(), ok)
    old = torch.zeros_like(n) if c["reset"] else s["seen"].int() & 0xFFFF
    if c["prompt"]:
        w = torch.where(n > 0, old | PROMPT, old)
    else:
        w = (old & PROMPT) | ((old & (PROMPT - 1)) + n).clamp(max=PROMPT - 1)
    s["seen"].copy_(_as_words(w))
    return s["seen"]


# --------------------------------------------------------------------------- one pass

def _kept(s, key, make):
    """What a user's program makes once and keeps: a handle, a workspace, the walk's rules."""
    if key not in s:
        s[key] = make()
    return s[key]


def _handle(s):
    from paper_2601_09083_amd import srt
    return _kept(s, "handle", lambda: srt.KvQuant(s["k"], s["v"], s["ks"], s["vs"], s["tail"][0], s["tail"][1], s["bt"],
                                               s["ctx_len"]))


def _own_run(s):
    from paper_2601_09083_amd import srt
    c = s["case"]
    if c["kind"] == "attn":
        kv = _handle(s)
        scratch = _kept(s, "scratch", lambda: torch.empty(srt.srt_tree_attn_quant_scratch_bytes(kv, c["N"], c["hq"]),
                                                          dtype=torch.uint8, device=DEV))
        return srt.srt_tree_attn_quant(s["q"], kv, s["k_new"], s["v_new"], s["parent"], s["n"], s["scale"], out=s["out"],
                                    scratch=scratch)
    if c["kind"] == "append":
        srt.srt_kv_append(_handle(s), s["k_new"], s["v_new"], s["counts"])
    if c["kind"] == "commit":
        srt.srt_commit_quant(_handle(s), s["k_new"], s["v_new"], s["acc"], s["emitted"], s["nodes"],
                          ctx_tail=s["ctx_tail"], draft_len=s["draft_len"])
    if c["kind"] in ("append", "commit"):
        return srt.srt_kv_read(_handle(s), s["start"], s["out"][0].shape[1], out=s["out"])
    if c["kind"] == "rules":
        rules = _kept(s, "rules", lambda: srt.Rules(
            seen=s["seen"], repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
            bias_offsets=s["bias_at"], bias_tokens=s["bias_tok"], bias_values=s["bias_val"], mask=s["mask"]))
        scratch = _kept(s, "scratch", lambda: torch.empty(srt.srt_accept_scratch_bytes(c["B"]), dtype=torch.uint8,
                                                          device=DEV))
        return srt.srt_accept_rules(s["logits"], s["gumbel"], 0.9, rules, s["tok"], s["par"], s["n"], c["dmax"],
                                    out=s["out"], scratch=scratch)
    srt.srt_seen_add(s["seen"], s["tokens"], s["lengths"], prompt=c["prompt"], reset=c["reset"])
    return s["seen"]


def _plain_run(s):
    c = s["case"]
    if c["kind"] == "attn":
        return _plain_attn(s)
    if c["kind"] == "append":
        m = torch.arange(c["T"], device=DEV).expand(c["B"], -1)
        _plain_write(s, m, s["counts"])
    if c["kind"] == "commit":
        e, qmax = s["acc"] + 1, c["qmax"]
        m = torch.cat([torch.zeros_like(s["nodes"][:, :1]), s["nodes"][:, :-1].clamp(min=0)], 1).long()
        _plain_write(s, m, e)
        both = torch.cat([s["ctx_tail"], s["emitted"]], 1)
        s["ctx_tail"].copy_(both.gather(1, (torch.arange(qmax, device=DEV) + e[:, None]).long()))
        s["draft_len"] += e
    if c["kind"] in ("append", "commit"):
        return [_plain_read(s, x, o) for x, o in zip("kv", s["out"])]
    if c["kind"] == "rules":
        return _plain_rules(s)
    return _plain_seen(s)


def run(s):
    c = s["case"]
    if c["kind"] in ("append", "commit"):  # every pass writes from where the batch stood
        s["state"].copy_(s["state0"])
        s["tail"].copy_(s["tail0"])
    got = _own_run(s) if own else _plain_run(s)
    if c["kind"] == "append":
        return dict(kv=got, ctx_len=s["ctx_len"])
    if c["kind"] == "commit":
        return dict(kv=got, ctx_len=s["ctx_len"], draft_len=s["draft_len"], ctx_tail=s["ctx_tail"])
    return got


# --------------------------------------------------------------------------- the same in 64 bits

def _exact_attn(s):
    c, out = s["case"], torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    L, n, par = s["ctx_len"].tolist(), s["n"].tolist(), s["parent"].cpu().numpy()
    G, d, hkv, page = c["hq"] // c["hkv"], c["d"], c["hkv"], c["page"]
    for b in range(c["B"]):
        full = L[b] // page
        ids = s["bt"][b, :full].long()
        kv = []
        for i, (x, xs) in enumerate((("k", "ks"), ("v", "vs"))):
            y = s[x][ids].double() * s[xs][ids].double()[:, :, None, None]
            y = y.transpose(0, 1).reshape(hkv, full * page, d)
            rest, new = s["tail"][i][b, :, : L[b] - full * page], s[x + "_new"][b, : n[b]].transpose(0, 1)
            kv.append(torch.cat([y, rest.double(), new.double()], 1))
        see = np.zeros((n[b], n[b]), dtype=bool)
        for i in range(n[b]):
            see[i] = see[par[b, i]] if i else False
            see[i, i] = True
        q = s["q"][b, : n[b]].double().reshape(n[b], hkv, G, d).permute(1, 0, 2, 3).reshape(hkv, n[b] * G, d)
        x = torch.matmul(q, kv[0].transpose(1, 2).contiguous()).mul_(s["scale"])
        hide = torch.as_tensor(~see, device=DEV).repeat_interleave(G, 0)
        x[:, :, L[b]:].masked_fill_(hide[None], -math.inf)
        o = torch.matmul(torch.softmax(x, -1), kv[1])
        out[b, : n[b]] = o.reshape(hkv, n[b], G, d).permute(1, 0, 2, 3).reshape(n[b], c["hq"], d)
    return out


def _nearest(x, kv):
    """float64 x at its nearest codes (ties to even)."""
    if kv == "int8":
        return x.round()
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))).clamp_(-6, 8)
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _exact_write(s):
    """The positions that the pass reads back, from the definition."""
    c = s["case"]
    B, page, top = c["B"], c["page"], LARGEST[c["kv"]]
    L, start = s["ctx_len"].tolist(), s["start"].tolist()
    if c["kind"] == "append":
        rows = [list(range(m)) for m in s["counts"].tolist()]
    else:
        rows = [[0] + r[:a] for r, a in zip(s["nodes"].tolist(), s["acc"].tolist())]
    got = []
    for i, x in enumerate("kv"):
        out = torch.zeros(s["out"][0].shape, dtype=torch.float64, device=DEV)
        for b in range(B):
            new = s[x + "_new"][b, torch.as_tensor(rows[b], dtype=torch.long, device=DEV)].double()
            y = torch.cat([s["tail"][i][b].transpose(0, 1)[: L[b] - start[b]].double(), new])
            full = len(y) // page * page
            z = y[:full].reshape(-1, page, c["hkv"], c["d"])
            amp = z.abs().amax((1, 3), keepdim=True).clamp_(min=LEAST)
            out[b, :full] = (_nearest(z * (top / amp), c["kv"]) * (amp / top)).reshape(full, c["hkv"], c["d"])
            out[b, full:len(y)] = y[full:]
        got.append(out)
    none = {k: None for k in (("ctx_len",) if c["kind"] == "append" else ("ctx_len", "draft_len", "ctx_tail"))}
    return dict(kv=got, **none)


def exact(case, seed):
    if case["kind"] == "attn":
        return _exact_attn(prepare(case, seed))
    if case["kind"] in ("append", "commit"):
        return _exact_write(prepare(case, seed))
    return None  # tokens and counts: whole numbers

"""Helpers for the tests of the 8-bit KV cache: random caches, their values in
fp64 and the attention tolerance derived from the kernel's roundings."""
from __future__ import annotations

import numpy as np
import torch

from oracle import attention as AT
from oracle import kv_quant as KQ
from paper_2601_09083_amd import srt

DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def bf16(x: np.ndarray) -> torch.Tensor:
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def new_cache(B, hkv, page, d, kv, max_pages, device, ctx=None, seed=0, spare=3, fill=None):
    """A KvQuant whose pages are in random order; pages, scales and tails hold
    ``fill`` bytes / values (default zero)."""
    rng = np.random.default_rng(seed)
    P = B * max_pages + spare
    bt = rng.permutation(P)[: B * max_pages].reshape(B, max_pages).astype(np.int32)
    pages = [torch.zeros((P, hkv, page, d), dtype=torch.uint8) for _ in range(2)]
    if fill is not None:
        for x in pages:
            x.fill_(fill)
    scales = [torch.zeros((P, hkv)) for _ in range(2)]
    tails = [torch.zeros((B, hkv, page, d), dtype=torch.bfloat16) for _ in range(2)]
    ctx = np.zeros(B, dtype=np.int32) if ctx is None else np.asarray(ctx, dtype=np.int32)
    dev = lambda t: t.to(device)
    return srt.KvQuant(*[dev(x).view(DTYPE[kv]) for x in pages], *map(dev, scales), *map(dev, tails),
                       dev(torch.from_numpy(bt)), dev(torch.from_numpy(ctx)))


class AttnCase:
    """Random codes, scales, tails and trees with the fp64 reference."""

    def __init__(self, seed, B, N, hq, hkv, d, ctx, kv="e4m3", page=16, n_nodes=None, max_pages=None, qk=1.0,
                 device="cuda"):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.B, self.N, self.hq, self.hkv, self.d, self.kv, self.page = B, N, hq, hkv, d, kv, page
        self.ctx = np.asarray(ctx, dtype=np.int32)
        mp = max(1, int(self.ctx.max()) // page) if max_pages is None else max_pages
        c = new_cache(B, hkv, page, d, kv, mp, "cpu", self.ctx, seed) if device == "cpu" else None
        P = B * mp + 3
        # every code but e4m3's NaN; unused pages hold NaN codes and NaN scales
        codes = []
        for _ in range(2):
            x = torch.randint(0, 256, (P, hkv, page, d), generator=g, dtype=torch.int32).to(torch.uint8)
            if kv == "e4m3":  # about normal magnitudes: exponents 1 .. 9 of 15
                x = torch.where((x & 0x78) > 0x48, x & 0xC7, x)
            codes.append(x)
        used = torch.zeros(P, dtype=torch.bool)
        bt = rng.permutation(P)[: B * mp].reshape(B, mp).astype(np.int32)
        for b in range(B):
            used[torch.from_numpy(bt[b, : self.ctx[b] // page]).long()] = True
        if kv == "e4m3":
            for x in codes:
                x[~used] = 0x7F
        top = {"e4m3": 0.25, "int8": 1 / 64.0}[kv]  # values of order one
        scales = [torch.exp(torch.randn((P, hkv), generator=g) * 0.7) * top * s for s in (qk, 1.0)]
        for x in scales:
            x[~used] = float("nan")
        tails = [torch.randn((B, hkv, page, d), generator=g) * s for s in (qk, 1.0)]
        new = [torch.randn((B, N, hkv, d), generator=g) * s for s in (qk, 1.0)]
        self.n_nodes = rng.integers(1, N + 1, B).astype(np.int32) if n_nodes is None else np.asarray(n_nodes, np.int32)
        for b in range(B):  # what is not part of the call
            for x in tails:
                x[b, :, self.ctx[b] % page:] = float("nan")
            for x in new:
                x[b, self.n_nodes[b]:] = float("nan")
        par = np.full((B, N), -1, dtype=np.int32)
        for b in range(B):
            for i in range(1, self.n_nodes[b]):
                par[b, i] = rng.integers(max(0, i - 6), i) if rng.random() < 0.8 else rng.integers(0, i)
        self.parent = par
        self.scale = d ** -0.5
        self.host = dict(codes=codes, scales=scales, tails=[x.to(torch.bfloat16) for x in tails],
                         new=[x.to(torch.bfloat16) for x in new], bt=bt,
                         q=(torch.randn((B, N, hq, d), generator=g) * qk).to(torch.bfloat16))
        h = self.host
        dev = lambda t: t.to(device)
        self.cache = srt.KvQuant(*[dev(x).view(DTYPE[kv]) for x in codes], *map(dev, scales), *map(dev, h["tails"]),
                                 dev(torch.from_numpy(bt)), dev(torch.from_numpy(self.ctx.copy())))
        self.q, self.new = dev(h["q"]), [dev(x) for x in h["new"]]
        self.par_dev, self.n_dev = dev(torch.from_numpy(par)), dev(torch.from_numpy(self.n_nodes))

    def run(self, **kw):
        return srt.srt_tree_attn_quant(self.q, self.cache, *self.new, self.par_dev, self.n_dev, self.scale, **kw)

    def rows(self, b, i):
        """K (i = 0) or V of sequence b: float64 [L + n, Hkv, d]."""
        h, L, page = self.host, int(self.ctx[b]), self.page
        full = L // page
        pg = torch.from_numpy(h["bt"][b, :full]).long()
        codes = h["codes"][i][pg].numpy().view(np.uint8 if self.kv == "e4m3" else np.int8)
        x = KQ.values(codes, self.kv) * h["scales"][i][pg].double().numpy()[:, :, None, None]
        x = x.transpose(0, 2, 1, 3).reshape(full * page, self.hkv, self.d)
        t = h["tails"][i][b, :, : L % page].double().numpy().transpose(1, 0, 2)
        return np.concatenate([x, t, h["new"][i][b, : self.n_nodes[b]].double().numpy()])

    def reference(self, b):
        """(out, tolerance) [n, Hq, d] float64.

        Roundings: probabilities to bf16, half a step each (2^-8), in the
        numerator and the same ones in the sum, so |d out| <= 2^-8 (A + |out|)
        with A = sum p |v| / sum p; the output to bf16, 2^-8 |out|; fp32 sums of
        the d products of a score, d 2^-24 sum |q k| scale, and as much again
        for the score's other operations (log2 of a scale, the reference, exp2):
        an absolute error e of a score changes a probability by the factor
        1 + e, and so the output by at most 2 e A.  fp32 sums of the second
        product are 2^-24 per key, L of them at most, of A.  A probability times
        its scale that is below 2^-126 is lost: with codes up to 448 and a sum of
        probabilities of at least 1 (the row's largest is at least the reference's
        1) that is at most 2^-126 448 per key, the whole value where a row's other
        keys weigh nothing and the heaviest one's code is 0."""
        n, L = int(self.n_nodes[b]), int(self.ctx[b])
        K, V = self.rows(b, 0), self.rows(b, 1)
        q = self.host["q"][b, :n].double().numpy()
        as_cache = lambda x: x.transpose(1, 0, 2)[None]
        one = lambda k, v, qq: AT.tree_attention_seq(qq, as_cache(k), as_cache(v), np.zeros(1, int), L, self.parent[b], n,
                                                     self.scale, L + n)
        ref, amp = one(K, V, q), one(K, np.abs(V), q)
        G = self.hq // self.hkv
        s_abs = np.stack([np.abs(q[:, h]) @ np.abs(K[:, h // G]).T for h in range(self.hq)], 1).max(-1) * self.scale
        e = 2 * (self.d + 16) * 2.0 ** -24 * s_abs[..., None]
        tol = 2.0 ** -8 * (amp + np.abs(ref)) + 2.0 ** -8 * np.abs(ref) + (2 * e + (L + n) * 2.0 ** -24) * amp
        tol += (L + n) * 448 * 2.0 ** -126
        return ref, 1.02 * tol  # (second order terms)

    def check(self, out, seqs=None, what=""):
        o = out.double().cpu().numpy()
        worst = 0.0
        for b in range(self.B) if seqs is None else seqs:
            n = int(self.n_nodes[b])
            ref, tol = self.reference(b)
            err = np.abs(o[b, :n] - ref)
            assert np.isfinite(o[b, :n]).all() and (err <= tol).all(), \
                f"{what} seq {b} (ctx {self.ctx[b]}, n {n}): worst {np.nanmax(err / tol):.3f} of the tolerance"
            worst = max(worst, float((err / tol).max()))
        return worst

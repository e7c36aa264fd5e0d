"""Inputs, 64-bit references and tolerances of the tests of packed prompts' attention, of single tokens' attention over paged
caches with running scores, and of the eviction from them.  Nothing here is the framework's own arithmetic."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests.shared_cases import F32, U, assert_within, gaussian

NAN = float("nan")


def on_gpu(t):
    """The tensor on the GPU with the strides that it has (expanded axes stay so)."""
    if t is None:
        return None
    if t.is_contiguous() or 0 in t.stride():
        return t.cuda()
    return torch.empty_strided(t.size(), t.stride(), dtype=t.dtype, device="cuda").copy_(t)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def rows_of_attention(q, k, v, hidden, scale, dtype):
    """(out, tolerance, lse, tolerance) of rows q [n, d] over keys and values [m, d], in 64 bits.

    Tolerances.  A logit is a sum of d products in fp32: off by `delta` = 20 half steps of the scaled sum of the
    products' sizes (chains of up to d / 4 additions, whose roundings are a random walk, joined), which a weight is off by
    relatively, twice with the normaliser.  Sums over the keys: 4 sqrt(keys) + 16 half steps (a random walk).  bf16: weights go
    into the second product rounded to bf16, independent errors of 2^-8 at most, whose sum has a standard
    deviation of 2^-8 / sqrt(3) |(p_j v_j)|; six of them.  And the output's own half step."""
    a = (q @ k.t() * scale).masked_fill(hidden, -math.inf)
    size = (q.abs() @ k.abs().t() * scale).masked_fill(hidden, 0.0)
    p = torch.nan_to_num(torch.softmax(a, 1), nan=0.0)
    out, lse = p @ v, torch.logsumexp(a, 1)
    delta = 20 * F32 * size.amax(1)
    walk = F32 * (4 * math.sqrt(a.size(1)) + 16)
    tol = (2 * delta[:, None] + walk) * (p @ v.abs()) + U[dtype] * out.abs()
    if dtype == torch.bfloat16:
        tol += 6 * U[dtype] / math.sqrt(3) * ((p * p) @ (v * v)).sqrt()
    return out, tol, lse, 2 * delta + walk + 2 * F32 * lse.abs()


# ------------------------------------------------------------ packed prompts --
class Prompts:
    """Packed prompts on the host: `gap` rows before the first and behind the last one that belong to none, NaN in everything that
    no row may look at."""

    def __init__(self, seed, lens, *, q_heads, kv_heads, d, dtype=torch.bfloat16, layout="thd", gap=0, scale=None, hot=0.0, pad=0,
                 heads=None):
        self.lens, self.hq, self.hkv, self.d, self.dtype = lens, q_heads, kv_heads, d, dtype
        self.heads = list(range(q_heads)) if heads is None else heads  # that are compared
        self.scale = d ** -0.5 if scale is None else scale
        self.tokens = sum(lens) + 2 * gap
        self.first = [gap + sum(lens[:s]) for s in range(len(lens) + 1)]

        def rows(k, heads):
            t = gaussian(seed + k, self.tokens, heads, d + pad, dtype=dtype)[..., :d]
            return t if layout == "thd" else t.transpose(0, 1).contiguous().transpose(0, 1)
        self.q, self.k, self.v = rows(1, q_heads), rows(2, kv_heads), rows(3, kv_heads)
        if hot:
            self.k *= torch.where(torch.rand(self.k.shape[:2], generator=torch.Generator().manual_seed(seed)) < 0.02, hot, 1.0).to(dtype)[..., None]
        for t in (self.q, self.k, self.v):
            t[:self.first[0]] = NAN
            t[self.first[-1]:] = NAN

    def reference(self):
        """Of the heads that are compared."""
        out, lse = np.full((self.tokens, len(self.heads), self.d), np.nan), np.full((len(self.heads), self.tokens), np.nan)
        tol, ltol = np.zeros_like(out), np.zeros_like(lse)
        for lo, hi in zip(self.first, self.first[1:]):
            if hi == lo:
                continue
            later = torch.ones(hi - lo, hi - lo, dtype=torch.bool).triu(1)
            for i, h in enumerate(self.heads):
                kv = h * self.hkv // self.hq
                o, t, l, lt = rows_of_attention(self.q[lo:hi, h].double(), self.k[lo:hi, kv].double(), self.v[lo:hi, kv].double(),
                                                later, self.scale, self.dtype)
                out[lo:hi, i], tol[lo:hi, i], lse[i, lo:hi], ltol[i, lo:hi] = o.numpy(), t.numpy(), l.numpy(), lt.numpy()
        return out, tol, lse, ltol

    def upload(self):
        from paper_2506_03762_amd import binding as B
        d = dict(q=on_gpu(self.q), k=on_gpu(self.k), v=on_gpu(self.v), first=i32(self.first))
        d["out"] = torch.full_like(d["q"], NAN)
        d["lse"] = torch.full((self.hq, self.tokens), NAN, device="cuda")
        d["p"] = B.PromptAttention.of(d["q"], d["k"], d["v"], d["out"], d["first"], self.scale)
        d["ws"] = B.alloc_prompt_workspace(d["p"])
        d["ws"].fill_(0xA5)
        return d

    @staticmethod
    def run(d, lse=True):
        from paper_2506_03762_amd import binding as B
        B.aha_prompt_attention(d["p"], d["q"], d["k"], d["v"], d["first"], d["out"], d["lse"] if lse else None, d["ws"])

    def check(self, d=None):
        print("prompts %s, heads %d / %d, d %d, %s, scale %g" % (
            self.lens if len(self.lens) < 40 else len(self.lens), self.hq, self.hkv, self.d, self.dtype, self.scale), flush=True)
        if d is None:
            d = self.upload()
            self.run(d)
        torch.cuda.synchronize()
        out, tol, lse, ltol = self.reference()
        got_out, got_lse = d["out"].float().cpu().numpy(), d["lse"].cpu().numpy()
        none = np.ones(self.tokens, bool)
        none[self.first[0]:self.first[-1]] = False
        assert np.isnan(got_out[none]).all() and np.isnan(got_lse[:, none]).all(), "rows that belong to no prompt are written"
        assert not np.isnan(got_out[~none]).any() and not np.isnan(got_lse[:, ~none]).any(), "rows are not written, or not numbers"
        some, heads = torch.from_numpy(~none).cuda(), torch.tensor(self.heads).cuda()
        assert_within(d["out"][some][:, heads], out[~none], tol[~none], "out")
        assert_within(d["lse"][heads][:, some], lse[:, ~none], ltol[:, ~none], "lse")
        return d


# ------------------------------------------------------------- paged caches --
class Caches:
    """Paged caches on the host: `tail` tokens per sequence, pages in no order, `holes`: entries of the table that are something
    else; scores and positions of all tokens; NaN in rows that no token has."""

    def __init__(self, seed, tail, *, kv_heads, d, q_heads=0, page=16, dtype=torch.bfloat16, layout="phrd", holes=(), width=None, slots=None,
                 seen=None, scores=None, pos=None, slot_pad=0, hot=0.0):
        rng = np.random.default_rng(seed)
        self.tail, self.hkv, self.hq, self.d, self.page, self.dtype = list(tail), kv_heads, q_heads, d, page, dtype
        self.batch = len(tail)
        width = max(1, -(-max(list(tail) + [1]) // page)) if width is None else width
        self.width, self.slots = width, width * page if slots is None else slots
        pages = self.batch * width + 2
        self.table = torch.from_numpy(rng.permutation(pages)[:self.batch * width].reshape(self.batch, width).astype(np.int32))
        for at, value in dict(holes).items():
            self.table[at] = value

        def pool(k):
            t = gaussian(seed + k, pages, kv_heads, page, d, dtype=dtype)
            return t if layout == "phrd" else t.transpose(1, 2).contiguous().transpose(1, 2)
        self.k, self.v = pool(4), pool(5)
        if hot:
            self.k *= torch.where(torch.rand(self.k.shape[:3], generator=torch.Generator().manual_seed(seed)) < 0.02, hot, 1.0).to(dtype)[..., None]
        real = torch.zeros(pages, page, dtype=torch.bool)
        for b in range(self.batch):
            for _, p, r in self.places(b):
                real[p, r] = True
        for t in (self.k, self.v):
            t.masked_fill_(~real[:, None, :, None], NAN)
        shape = (self.batch, kv_heads, self.slots + slot_pad)
        self.scores = torch.from_numpy(np.exp(rng.standard_normal(shape)).astype(np.float32)) if scores is None else scores
        self.pos = torch.from_numpy(np.sort(rng.integers(0, 4 * self.slots, shape), axis=2).astype(np.int32)) if pos is None else pos
        self.scores, self.pos = self.scores[..., :self.slots], self.pos[..., :self.slots]
        self.seen = seen
        if q_heads:
            self.q = gaussian(seed + 6, self.batch, q_heads, d, dtype=dtype)

    def length(self, b):
        return max(0, min(self.tail[b], self.width * self.page, self.slots if self.slots else 1 << 40))

    def places(self, b):
        """(token, page, row) of the tokens of sequence b that are in a page."""
        n = max(0, min(self.tail[b], self.width * self.page, self.slots if self.slots else 1 << 40))
        table = self.table[b].tolist()
        return [(j, table[j // self.page], j % self.page) for j in range(n) if 0 <= table[j // self.page] < self.batch * self.width + 2]

    def seen_of(self, b):
        return self.tail[b] if self.seen is None else self.seen[b]

    def pages(self, d):
        from paper_2506_03762_amd import binding as B
        d.update(k=on_gpu(self.k), v=on_gpu(self.v), table=self.table.cuda(), tail=i32(self.tail),
                 seen=None if self.seen is None else i32(self.seen), scores=on_gpu(self.scores), pos=on_gpu(self.pos))
        d["cache"] = B.Pages.of(d["k"], d["v"], d["table"])
        return d


class Steps(Caches):
    """A generation step's attention."""

    def __init__(self, seed, tail, *, scale=None, adaptive=True, fixed=0.0, floor=-1.0, budget=64, with_scores=True, with_pos=True, **kw):
        super().__init__(seed, tail, **kw)
        self.scale = self.d ** -0.5 if scale is None else scale
        self.adaptive, self.fixed, self.floor, self.budget = adaptive, fixed, floor, budget
        self.with_scores, self.with_pos = with_scores, with_pos and with_scores

    def lam(self, b):
        if not self.adaptive:
            return self.fixed
        floor = self.d ** -0.5 if self.floor < 0 else self.floor
        return max(floor, math.sqrt(2 * max(0.0, math.log(max(1, self.seen_of(b)) / self.budget)) / self.d))

    def reference(self):
        """out, lse, scores, pos and the tolerances of the first three.

        Scores: a weight is off by `delta` (rows_of_attention), twice with the normaliser, and by the scale's own rounding, 4 half
        steps of the logits' size; sums over keys and query heads, the exponential and the addition to the score half a step each.
        (Weights below 2^-126 may be 0.)"""
        out, lse = np.zeros((self.batch, self.hq, self.d)), np.full((self.batch, self.hq), -np.inf)
        tol, ltol = np.zeros_like(out), np.zeros_like(lse)
        scores, pos = self.scores.double().numpy().copy(), self.pos.numpy().copy()
        stol, group = np.zeros_like(scores), self.hq // self.hkv
        for b in range(self.batch):
            there, n = self.places(b), self.length(b)
            if n and self.with_scores:
                scores[b, :, n - 1] = 0.0
                pos[b, :, n - 1] = self.seen_of(b) - 1
            if not there:
                continue
            at, pages, rows = ([x[i] for x in there] for i in range(3))
            for kv in range(self.hkv):
                k, v = self.k[pages, kv, rows].double(), self.v[pages, kv, rows].double()
                heads = slice(kv * group, (kv + 1) * group)
                q = self.q[b, heads].double()
                o, t, l, lt = rows_of_attention(q, k, v, torch.zeros(group, len(at), dtype=torch.bool), self.scale, self.dtype)
                out[b, heads], tol[b, heads], lse[b, heads], ltol[b, heads] = o.numpy(), t.numpy(), l.numpy(), lt.numpy()
                if not self.with_scores:
                    continue
                lam = self.lam(b)
                w = torch.softmax(q @ k.t() * lam, 1)
                size = (q.abs() @ k.abs().t() * lam).amax(1)
                off = 2 * (20 + 4) * F32 * size + F32 * (4 * math.sqrt(len(at)) + 20)
                scores[b, kv, at] += w.sum(0).numpy()
                stol[b, kv, at] = ((w * off[:, None]).sum(0) + group * F32 * w.sum(0)).numpy() + 2 * F32 * np.abs(scores[b, kv, at]) + group * 2.0 ** -120
        return out, tol, lse, ltol, scores, stol, pos

    def upload(self):
        from paper_2506_03762_amd import binding as B
        d = self.pages(dict(q=on_gpu(self.q)))
        d["out"], d["lse"] = torch.full_like(d["q"], NAN), torch.full((self.batch, self.hq), NAN, device="cuda")
        d["p"] = B.PagedAttention.of(d["q"], d["out"], d["scores"] if self.with_scores else None, d["pos"] if self.with_pos else None,
                                     n_kv_heads=self.hkv, scale=self.scale, budget=self.budget, fixed_scale=self.fixed,
                                     lambda_floor=self.floor, scale_mode=B.AHA_SCALE_ADAPTIVE if self.adaptive else B.AHA_SCALE_FIXED)
        d["ws"] = B.alloc_paged_workspace(d["p"], d["cache"])
        d["ws"].fill_(0xA5)
        return d

    def run(self, d, lse=True):
        from paper_2506_03762_amd import binding as B
        B.aha_paged_attention(d["p"], d["cache"], d["q"], d["k"], d["v"], d["table"], d["tail"], d["seen"],
                              d["scores"] if self.with_scores else None, d["pos"] if self.with_pos else None, d["out"],
                              d["lse"] if lse else None, d["ws"])

    def check(self, d=None):
        print("caches of %s tokens, heads %d / %d, d %d, page %d, %s, budget %d, seen %s" % (
            self.tail, self.hq, self.hkv, self.d, self.page, self.dtype, self.budget, self.seen), flush=True)
        if d is None:
            d = self.upload()
            self.run(d)
        torch.cuda.synchronize()
        out, tol, lse, ltol, scores, stol, pos = self.reference()
        assert_within(d["out"], out, tol, "out")
        got, none = d["lse"].cpu().numpy().astype(np.float64), np.isneginf(lse)
        assert np.array_equal(np.isneginf(got), none), "rows without a key"
        assert_within(d["lse"][torch.from_numpy(~none).cuda()], lse[~none], ltol[~none], "lse")
        if self.with_scores:
            some = stol > 0
            assert_within(d["scores"][torch.from_numpy(some).cuda()], scores[some], stol[some], "scores")
            assert np.array_equal(d["scores"].cpu().numpy()[~some], scores[~some].astype(np.float32), equal_nan=True), \
                "scores of no token are changed"
        assert np.array_equal(d["pos"].cpu().numpy(), pos if self.with_pos else self.pos.numpy()), "pos"
        assert torch.equal(d["k"].cpu().view(torch.uint8), self.k.contiguous().view(torch.uint8)) if self.k.is_contiguous() else True
        return d


class Evictions(Caches):
    """Sequences brought back to their budget."""

    def __init__(self, seed, tail, *, budget, recent=0, sink=0, in_place=True, with_pos=True, **kw):
        super().__init__(seed, tail, **kw)
        self.budget, self.recent, self.sink, self.in_place, self.with_pos = budget, recent, sink, in_place, with_pos

    def reference(self):
        """k, v, scores, pos, lengths; what no output says stays (NaN and -7 in outputs of their own)."""
        k, v = self.k.clone(), self.v.clone()
        scores = self.scores.clone() if self.in_place else torch.full_like(self.scores, NAN)
        pos = self.pos.clone() if self.in_place and self.with_pos else torch.full_like(self.pos, -7)
        lens = []
        for b in range(self.batch):
            n = self.length(b)
            there = self.places(b)
            keep = min(n, self.budget) if len(there) == n else n
            lens.append(keep)
            for h in range(self.hkv):
                at = self.pos[b, h, :n].tolist() if self.with_pos else list(range(n))
                sc = self.scores[b, h, :n].tolist()
                safe = [p >= self.seen_of(b) - self.recent or p < self.sink for p in at]
                def worth(j):
                    if safe[j]:
                        return (2, 0.0, -at[j], -j)
                    return (0, 0.0, -at[j], -j) if sc[j] != sc[j] else (1, sc[j], -at[j], -j)
                stay = sorted(sorted(range(n), key=worth)[n - keep:])
                kept = set(stay)
                free = [j for j in range(keep) if j not in kept]
                source = list(range(keep))
                for to, frm in zip(free, [j for j in stay if j >= keep]):
                    source[to] = frm
                    for new, old in ((k, self.k), (v, self.v)):
                        new[there[to][1], h, there[to][2]] = old[there[frm][1], h, there[frm][2]]
                scores[b, h, :keep] = self.scores[b, h, source]
                pos[b, h, :keep] = self.pos[b, h, source] if self.with_pos else torch.tensor(source, dtype=torch.int32)
        return k, v, scores, pos, lens

    def upload(self):
        from paper_2506_03762_amd import binding as B
        d = self.pages({})
        d["scores_out"] = d["scores"] if self.in_place else torch.full_like(d["scores"], NAN)
        d["pos_out"] = d["pos"] if self.in_place and self.with_pos else torch.full_like(d["pos"], -7)
        d["len_out"] = torch.full((self.batch,), -7, dtype=torch.int32, device="cuda")
        d["p"] = B.PagedEviction.of(d["scores"], d["pos"] if self.with_pos else None, d["scores_out"], d["pos_out"], d["cache"],
                                    budget=self.budget, recent=self.recent, sink=self.sink)
        d["ws"] = B.alloc_evict_workspace(d["p"], d["cache"])
        d["ws"].fill_(0xA5)
        return d

    def run(self, d):
        from paper_2506_03762_amd import binding as B
        B.aha_paged_evict(d["p"], d["cache"], d["scores"], d["pos"] if self.with_pos else None, d["k"], d["v"], d["table"], d["tail"],
                          d["seen"], d["scores_out"], d["pos_out"], d["len_out"], d["ws"])

    def check(self, d=None):
        print("eviction from %s tokens to %d, recent %d, sink %d, %d heads, d %d, page %d, %s, seen %s, in place %s" % (
            self.tail, self.budget, self.recent, self.sink, self.hkv, self.d, self.page, self.dtype, self.seen, self.in_place), flush=True)
        if d is None:
            d = self.upload()
            self.run(d)
        torch.cuda.synchronize()
        k, v, scores, pos, lens = self.reference()
        bits = lambda t: t.cpu().contiguous().view(torch.uint8)
        assert d["len_out"].tolist() == lens
        assert torch.equal(bits(d["pos_out"]), bits(pos)), "positions"
        assert torch.equal(bits(d["scores_out"]), bits(scores)), "scores"
        assert torch.equal(bits(d["k"]), bits(k)) and torch.equal(bits(d["v"]), bits(v)), "keys or values"
        return d

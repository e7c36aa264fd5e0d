"""Inputs, 64-bit references and tolerances of the tests of rotation, the paged cache and the attention
behind shared prefixes.  Nothing here is the framework's own arithmetic.

A rounding to type t is off by at most half a step, U[t] relative to the value: 2^-8 for bf16, 2^-24 for fp32."""
from __future__ import annotations

import math

import numpy as np
import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -24


def gaussian(seed, *shape, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype)


# ---------------------------------------------------------------- rotation --
def angles(positions, inv_freq, pair_axis):
    """[b, n, pairs] angles in extended precision (64 bits of mantissa): positions [axes, b, n]."""
    pos = positions.numpy().astype(np.longdouble)
    w = inv_freq.numpy().astype(np.longdouble)
    axis = np.zeros(len(w), np.int64) if pair_axis is None else np.clip(pair_axis.numpy(), 0, pos.shape[0] - 1)
    return np.moveaxis(pos[axis], 0, -1) * w


def rotated(x, ang, rot, neighbours, transpose):
    """(result, tolerance) of turning x [b, h, n, d] by ang [b, n, rot / 2], in 64 bits.

    Tolerance: the storage's half step, and of |x0| + |x1| what fp32 leaves open: the angle, known to 2^-26 of
    a turn and 2^-52 of its turns (two products in double); sine and cosine, 2 units each; two products
    and a sum, 3 half units."""
    dtype, x = x.dtype, x.double().numpy()
    c, s = (np.asarray(f(ang), np.float64)[:, None] for f in (np.cos, np.sin))
    s = -s if transpose else s
    half = rot // 2
    at = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if neighbours else (np.arange(half), half + np.arange(half))
    a, b = x[..., at[0]], x[..., at[1]]
    y, tol = x.copy(), np.zeros_like(x)
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    turns = np.asarray(np.abs(ang), np.float64)[:, None] / (2 * math.pi)
    off = 2 * math.pi * (2.0 ** -26 + turns * 2.0 ** -52) + (4 + 3) * F32
    for i in at:
        tol[..., i] = (np.abs(a) + np.abs(b)) * off + U[dtype] * np.abs(y[..., i])
    return y, tol


def assert_within(got, want, tol, what):
    got = got.detach().cpu().double().numpy()
    bad = ~(np.abs(got - want) <= tol)
    if bad.any():
        at = np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) - tol, -np.inf)), bad.shape)
        raise AssertionError("%s: %d of %d values off, worst at %s: %.9g, not %.9g (tolerance %.3g)" % (
            what, bad.sum(), bad.size, at, got[at], want[at], tol[at]))


# --------------------------------------------------------------- attention --
class Batch:
    """A batch behind shared prefixes, on the host: lengths, members, pages (in no order, `holes`: entries of the
    table that are -1), Gaussian rows, everything that no row may look at filled with NaN."""

    def __init__(self, seed, *, q_heads, kv_heads, d, q_len, tail, new=None, prefix=(), first=None, page=16,
                 cap=None, dtype=torch.bfloat16, layout="bhnd", holes=(), scale=None, tails=True, hot=0.0):
        self.batch, self.q_len, self.hq, self.hkv, self.d = len(tail), q_len, q_heads, kv_heads, d
        self.tail, self.new = list(tail), list(new) if new is not None else None
        self.prefix, self.first = list(prefix), list(first) if first is not None else [0] + [len(tail)] * len(prefix)
        self.dtype, self.page, self.tails = dtype, page, tails
        self.scale = d ** -0.5 if scale is None else scale
        b, width = self.batch, max(1, -(-max(list(tail) + [1]) // page))
        self.cap = max(list(prefix) + [1]) if cap is None else cap
        rng = np.random.default_rng(seed)
        pages = b * width + 2
        self.table = torch.from_numpy(rng.permutation(pages)[:b * width].reshape(b, width).astype(np.int32))
        for at, value in dict(holes).items():
            self.table[at] = value
        def rows(k, *shape):  # [x, heads, n, d] in the layout
            t = gaussian(seed + k, *shape, d, dtype=dtype)
            return t if layout == "bhnd" else t.transpose(1, 2).contiguous().transpose(1, 2)
        self.q = rows(1, b, q_heads, q_len)
        n_prefixes = max(1, len(self.prefix))
        self.kp, self.vp = rows(2, n_prefixes, kv_heads, self.cap), rows(3, n_prefixes, kv_heads, self.cap)
        self.kt, self.vt = rows(4, pages, kv_heads, page), rows(5, pages, kv_heads, page)
        if hot:  # some keys that weigh much more than the others
            for t in (self.kp, self.kt):
                t *= torch.where(torch.rand(t.shape[:3], generator=torch.Generator().manual_seed(seed)) < 0.02, hot, 1.0).to(dtype)[..., None]
        self._forget_unseen()

    def fresh(self, b):
        return self.q_len if self.new is None else min(max(self.new[b], 0), self.q_len)

    def slots(self, b):
        """(slot, page, row) of the tail tokens of sequence b that are there."""
        room = self.table.size(1) * self.page
        return [(j, int(self.table[b, j // self.page]), j % self.page) for j in range(min(self.tail[b], room))
                if 0 <= int(self.table[b, j // self.page]) < self.kt.size(0)] if self.tails else []

    def group(self, b):
        for g in range(len(self.prefix)):
            if self.first[g] <= b < self.first[g + 1]:
                return g
        return None

    def _forget_unseen(self):
        nan = float("nan")
        seen = torch.zeros(self.kt.shape[0], self.page, dtype=torch.bool)
        for b in range(self.batch):
            for _, p, r in self.slots(b):
                seen[p, r] = True
        for t in (self.kt, self.vt):
            t.masked_fill_(~seen[:, None, :, None], nan)
        for g, n in enumerate(self.prefix):
            self.kp[g, :, n:] = nan
            self.vp[g, :, n:] = nan
        for b in range(self.batch):
            self.q[b, :, self.fresh(b):] = nan

    def reference(self):
        """out, tolerance, lse, tolerance of all rows (NaN where nothing is written), in 64 bits.

        Tolerances.  A logit is a sum of d products in fp32: off by `delta` = 20 half steps of the scaled sum of
        the products' sizes (chains of up to d / 4 additions, whose roundings are a random walk, joined), which a weight is off by relatively, twice with
        the normaliser.  Sums over the keys: 4 sqrt(keys) + 16 half steps (a random walk).  bf16: weights go
        into the second product rounded to bf16, independent errors of 2^-8 at most, whose sum has a standard deviation
        of 2^-8 / sqrt(3) |(p_j v_j)|; six of them.  And the output's own half step."""
        b, n = self.batch, self.q_len
        out = np.full((b, self.hq, n, self.d), np.nan)
        tol, lse, ltol = np.zeros_like(out), np.full((b, self.hq, n), np.nan), np.zeros((b, self.hq, n))
        for i in range(b):
            fresh, there, g = self.fresh(i), self.slots(i), self.group(i)
            if fresh == 0:
                continue
            pages, rows = [x[1] for x in there], [x[2] for x in there]
            k, v = ((x[pages, :, rows] if there else x[:0, :, 0]).double() for x in (self.kt, self.vt))
            ahead = 0 if g is None else min(max(self.prefix[g], 0), self.cap)
            if ahead:
                k, v = (torch.cat([x[g, :, :ahead].double().transpose(0, 1), y]) for x, y in ((self.kp, k), (self.vp, v)))
            slot = torch.tensor([-2 ** 40] * ahead + [x[0] for x in there])
            limit = self.tail[i] - fresh + torch.arange(fresh)
            hidden = slot[None, :] > limit[:, None]
            for h in range(self.hq):
                kv = h * self.hkv // self.hq
                q = self.q[i, h, :fresh].double()
                a = (q @ k[:, kv].t() * self.scale).masked_fill(hidden, -math.inf)
                size = (q.abs() @ k[:, kv].abs().t() * self.scale).masked_fill(hidden, 0.0)
                p = torch.nan_to_num(torch.softmax(a, 1), nan=0.0) if a.size(1) else a
                lse[i, h, :fresh] = torch.logsumexp(a, 1).numpy() if a.size(1) else -math.inf
                o = p @ v[:, kv]
                out[i, h, :fresh] = o.numpy()
                keys = max(1, a.size(1))
                delta = 20 * F32 * (size.amax(1) if a.size(1) else torch.zeros(fresh))
                walk = F32 * (4 * math.sqrt(keys) + 16)
                t = (2 * delta[:, None] + walk) * (p @ v[:, kv].abs()) + U[self.dtype] * o.abs()
                if self.dtype == torch.bfloat16:
                    t += 6 * U[self.dtype] / math.sqrt(3) * ((p * p) @ (v[:, kv] * v[:, kv])).sqrt()
                tol[i, h, :fresh] = t.numpy()
                ltol[i, h, :fresh] = 2 * delta.numpy() + walk + 2 * F32 * np.abs(np.nan_to_num(lse[i, h, :fresh], neginf=0.0))
        return out, tol, lse, ltol

    # ---- the framework's side ----
    def upload(self):
        from paper_2506_03762_amd import binding as B
        dev = lambda t: (t.cuda() if 0 in t.stride() else torch.empty_strided(t.size(), t.stride(), dtype=t.dtype, device="cuda").copy_(t))
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        d = dict(q=dev(self.q), tail=i32(self.tail), new=None if self.new is None else i32(self.new))
        d["out"] = torch.full_like(d["q"], float("nan"))
        d["lse"] = torch.full(self.q.shape[:3], float("nan"), device="cuda")
        if self.prefix:
            d.update(kp=dev(self.kp), vp=dev(self.vp), prefix=i32(self.prefix), first=i32(self.first))
        if self.tails:
            d.update(kt=dev(self.kt), vt=dev(self.vt), table=self.table.cuda())
            d["cache"] = B.Pages.of(d["kt"], d["vt"], d["table"])
        d["p"] = B.SharedAttention.of(d["q"], d["out"], d.get("kp"), d.get("vp"), self.scale, n_kv_heads=self.hkv)
        d["ws"] = B.alloc_shared_workspace(d["p"], d.get("cache"))
        d["ws"].fill_(0xA5)
        return d

    @staticmethod
    def run(d, lse=True):
        from paper_2506_03762_amd import binding as B
        tails = "cache" in d
        B.aha_shared_attention(d["p"], d.get("cache"), d["q"], d.get("kp"), d.get("vp"), d.get("prefix"), d.get("first"),
                               d.get("kt"), d.get("vt"), d.get("table"), d["tail"] if tails else None, d["new"],
                               d["out"], d["lse"] if lse else None, d["ws"])

    def check(self, d=None):
        print("batch %d x %d rows, heads %d / %d, d %d, prefixes %s first %s, tails %s, new %s, page %d, %s" % (
            self.batch, self.q_len, self.hq, self.hkv, self.d, self.prefix, self.first, self.tail, self.new,
            self.page, self.dtype), flush=True)
        if d is None:
            d = self.upload()
            self.run(d)
        torch.cuda.synchronize()
        self.compare(d)
        return d

    def compare(self, d):
        out, tol, lse, ltol = self.reference()
        written = ~np.isnan(lse)
        got = d["lse"].cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isnan(got), ~written), "lse: other rows than the new ones are written"
        o = d["out"].float().cpu().numpy()
        assert np.array_equal(np.isnan(o).any(-1), ~written), "out: other rows are written, or not numbers"
        assert np.isnan(o).all(-1)[~written].all()
        none = np.isneginf(lse)
        assert np.array_equal(np.isneginf(got), none) and not np.any(o[none])
        there = written & ~none
        assert_within(d["out"][torch.from_numpy(there).cuda()], out[there], tol[there], "out")
        assert_within(d["lse"][torch.from_numpy(there).cuda()], lse[there], ltol[there], "lse")

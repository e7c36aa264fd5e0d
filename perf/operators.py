"""Work of the operators around a cache that several continuations of a prompt share, to be measured.

Three kinds of pass, as the program around a language model makes them:

  rotate  the rotation of a prompt's queries and keys by their positions, or its gradient's (transpose);
  append  one layer's new tokens: queries and keys rotated, keys and values written to the paged cache;
  attend  the attention of the new tokens over a prefix that several sequences share and over their own
          tails in the paged cache.

`own` chooses between the operators' plain form, elementary operations in 32 bits, and the framework's
entry points.  Lengths and page tables follow from the case alone, what the tensors hold from the seed.
"""
import math
import random

import torch

own = False

FREQUENCY_BASE = 10000.0   # pair f of F turns by base^(-f / F) per position
KEY_MEAN = 0.7             # of a KV head's keys along a direction that its queries lean on, too
FREE_PAGES = 3             # pages of the pool that no sequence holds


def _rotate(name, batch, n, hq, hkv, d, **more):
    case = dict(kind="rotate", batch=batch, n=n, hq=hq, hkv=hkv, d=d, rot=d, axes=1, neighbours=False,
                transpose=False, start=0, dtype="bf16", layout="bhnd")
    return _named(case, name, more)


def _append(name, batch, n, hq, hkv, d, held, page, **more):
    case = dict(kind="append", batch=batch, n=n, hq=hq, hkv=hkv, d=d, held=held, page=page, rot=d, axes=1,
                neighbours=False, transpose=False, start=0, ragged=False, dtype="bf16", layout="bhnd")
    return _named(case, name, more)


def _attend(name, batch, n, hq, hkv, d, prefixes, prefix, held, page, **more):
    case = dict(kind="attend", batch=batch, n=n, hq=hq, hkv=hkv, d=d, prefixes=prefixes, prefix=prefix,
                held=held, page=page, ragged=False, dtype="bf16", layout="bhnd")
    return _named(case, name, more)


def _named(case, name, more):
    if name:
        case["name"] = name
    case.update(more)
    return case


def listed():
    return [
        # a short prompt of a small fp32 model, where latency is everything
        _rotate("rotate_short_f32", 1, 512, 2, 2, 64, dtype="f32"),
        # one layer of a grouped-query model, a long prompt
        _rotate("rotate_prompt", 1, 32768, 32, 8, 128),
        # images and video: positions in time, height and width, sizes that divide nothing, token-major
        _rotate("rotate_three_axes", 3, 5003, 12, 4, 128, axes=3, layout="bnhd"),
        # the gradient of a batch of prompts of which half of the channels are rotated, in neighbouring pairs
        _rotate("rotate_transposed", 4, 4096, 32, 32, 128, rot=64, neighbours=True, transpose=True),
        # one generated token of each of 64 sequences, far positions
        _append("append_step", 64, 1, 32, 8, 128, 700, 64, start=100000),
        # chunks of prompts of several lengths
        _append("append_chunk", 8, 2048, 32, 8, 128, 1000, 64, ragged=True),
        # fp32, small pages, neighbouring pairs, odd lengths, token-major
        _append("append_odd_f32", 5, 333, 6, 2, 64, 77, 16, neighbours=True, ragged=True, dtype="f32",
                layout="bnhd"),
        # one compacted prompt, eight continuations that have hardly begun: latency
        _attend("shared_few", 8, 1, 32, 8, 128, 1, 2048, 100, 64),
        # generation for 64 sequences of four compacted prompts: bound by the tails' bytes
        _attend("shared_batch", 64, 1, 32, 8, 128, 4, 4096, 1000, 64),
        # a whole long prompt and 32 continuations with eight query heads per KV head: products
        _attend("shared_long", 32, 1, 64, 8, 128, 1, 32768, 256, 64),
        # chunks of 256 tokens of four sequences behind a long prefix: the most products
        _attend("shared_chunk", 4, 256, 32, 8, 128, 1, 16384, 500, 64),
        # fp32, ragged prefixes and tails, small pages of which some have been given back, token-major
        _attend("shared_odd_f32", 7, 3, 6, 2, 64, 3, 901, 333, 16, ragged=True, dtype="f32", layout="bnhd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the ranges that the listed ones stand for, odd ones among them."""
    kind = rng.choice(["rotate", "rotate", "append", "append", "attend", "attend", "attend", "attend"])
    f32 = rng.random() < 0.2
    d, hkv, group = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 7, 8])
    more = dict(dtype="f32" if f32 else "bf16", layout=rng.choice(["bhnd", "bhnd", "bnhd"]))
    if kind == "attend":
        n = rng.choice([1, 1, 1, rng.randint(2, 8), _log_int(rng, 9, 160)])
        batch, prefix = _log_int(rng, 1, 64), _log_int(rng, 1, 4096 if f32 else 32768)
        held, prefixes = _log_int(rng, 1, 1200), rng.choice([0, 1, 1, 2, 4, 7])
        most = 4e9 if f32 else 2.5e11
        while batch > 1 and 4 * d * hkv * group * batch * n * (prefix + held + n) > most:
            batch //= 2
        while n > 1 and 4 * d * hkv * group * batch * n * (prefix + held + n) > most:
            n //= 2
        while prefixes * hkv * prefix > 2 ** 18:
            prefixes //= 2
        return _attend(None, batch, n, hkv * group, hkv, d, prefixes, prefix, held,
                       rng.choice([1, 8, 16, 32, 64, 64, 128, 256]), ragged=rng.random() < 0.6, **more)
    more.update(axes=rng.choice([1, 1, 2, 3]), neighbours=rng.random() < 0.3,
                rot=rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)]), start=rng.choice([0, 0, 777, 1000003]))
    if kind == "append":
        n = rng.choice([1, rng.randint(2, 40), _log_int(rng, 41, 2500)])
        batch = _log_int(rng, 1, 64)
        while batch > 1 and batch * n * (hkv * group + 2 * hkv) * d > 8 * 2048 * 48 * 128 // 2:
            batch //= 2
        return _append(None, batch, n, hkv * group, hkv, d, rng.randint(0, 1500), rng.choice([1, 8, 16, 32, 64, 128]),
                       ragged=n > 1 and rng.random() < 0.6, **more)
    n, batch = _log_int(rng, 1, 32768), _log_int(rng, 1, 16)
    while batch * n * (hkv + hkv * group) * d > 32768 * 40 * 128 // 2:
        batch, n = max(1, batch // 2), n // 2
    return _rotate(None, batch, n, hkv * group, hkv, d, transpose=rng.random() < 0.3, **more)


# ---- what follows from the case: lengths, members, pages ----

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """new tokens and tail lengths (new ones among them) of the sequences, lengths and first sequences of the
    prefixes.  A sequence behind the last prefix's has none."""
    rng = random.Random(case["batch"] * 1009 + case["held"] * 31 + case["n"])
    new = [rng.randint(1, case["n"]) if case["ragged"] else case["n"] for _ in range(case["batch"])]
    tail = [x + rng.randint(0, case["held"]) for x in new]
    prefixes, batch = case.get("prefixes", 0), case["batch"]
    lens = [rng.randint(0, case["prefix"]) if case["ragged"] and g else case["prefix"] for g in range(prefixes)]
    with_prefix = batch - 1 if case["ragged"] and batch > 2 * prefixes else batch
    if not prefixes:
        return new, tail, [], [0]
    cuts = [rng.randint(0, with_prefix) for _ in range(prefixes - 1)] if case["ragged"] else \
        [g * batch // prefixes for g in range(1, prefixes)]
    return new, tail, lens, [0] + sorted(cuts) + [with_prefix]


def _pages(case, tail):
    """Pages per sequence of the table, pages of the pool, and the table: pages in no order, some given back
    (-1) at the start of a ragged case's longer tails."""
    width = -(-(case["n"] + case["held"]) // case["page"])
    rng = random.Random(case["page"] * 7 + case["batch"])
    held = [-(-x // case["page"]) for x in tail]
    pool = list(range(sum(held) + FREE_PAGES))
    rng.shuffle(pool)
    table = [[pool.pop() for _ in range(h)] + [-1] * (width - h) for h in held]
    if case["ragged"] and case["kind"] == "attend":
        for b in range(0, case["batch"], 3):
            table[b][:held[b] // 3] = [-1] * (held[b] // 3)
    return width, sum(held) + FREE_PAGES, table


def _axis_of_pair(case):
    """Which axis turns a pair: runs of pairs, the first axis the shortest (an eighth of them)."""
    pairs, axes = case["rot"] // 2, case["axes"]
    first = pairs if axes == 1 else pairs // 8
    return [0 if f < first else 1 + (f - first) * (axes - 1) // (pairs - first) for f in range(pairs)]


def _positions(case):
    """[axes][batch][n]: the tokens' places; of several axes the further ones walk rows and columns of a
    picture of 24 columns."""
    b, n = case["batch"], case["n"]
    t = case["start"] + torch.arange(n, device="cuda").repeat(b, 1) + 3 * torch.arange(b, device="cuda").unsqueeze(1)
    return torch.stack([t, t // 24, t % 24][:case["axes"]]).to(torch.int32)


def _heads(case, gen, heads, n=None, batch=None):
    """A Gaussian [b, heads, n, d] tensor in the layout of the case."""
    b, n, d = batch or case["batch"], n or case["n"], case["d"]
    if case["layout"] == "bnhd":
        return torch.randn((b, n, heads, d), generator=gen, device="cuda", dtype=_dtype(case)).transpose(1, 2)
    return torch.randn((b, heads, n, d), generator=gen, device="cuda", dtype=_dtype(case))


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    s = dict(kind=case["kind"], q=_heads(case, gen, hq))
    if case["kind"] != "attend":
        pairs = case["rot"] // 2
        s.update(k=_heads(case, gen, hkv), q_out=_heads(case, gen, hq), positions=_positions(case),
                 inv_freq=(FREQUENCY_BASE ** (-torch.arange(pairs, device="cuda", dtype=torch.float64) / pairs)).float(),
                 pair_axis=_int32(_axis_of_pair(case)), rot=case["rot"], neighbours=case["neighbours"],
                 transpose=case["transpose"])
        if case["kind"] == "rotate":
            s["k_out"] = _heads(case, gen, hkv)
        else:
            s["v"] = _heads(case, gen, hkv)
    if case["kind"] != "rotate":
        new, tail, lens, first = _lengths(case)
        width, pages, table = _pages(case, tail)
        pool = [_heads(case, gen, hkv, case["page"], pages) for _ in range(2)]
        s.update(k_pages=pool[0], v_pages=pool[1], page=case["page"], table=_int32(table), tail=_int32(tail),
                 new=_int32(new) if case["ragged"] else None)
    if case["kind"] == "attend":
        s.update(scale=1.0 / math.sqrt(d), prefix_len=_int32(lens), prefix_first=_int32(first),
                 out=torch.zeros_like(s["q"]), lse=torch.zeros(s["q"].shape[:3], device="cuda"))
        if case["prefixes"]:
            s.update(k_prefix=_heads(case, gen, hkv, case["prefix"], case["prefixes"]),
                     v_prefix=_heads(case, gen, hkv, case["prefix"], case["prefixes"]))
        lean = torch.randn((1, hkv, 1, d), generator=gen, device="cuda", dtype=_dtype(case))
        for name in ("k_pages", "k_prefix"):
            if name in s:
                s[name] += KEY_MEAN * lean
        s["q"] += lean.repeat_interleave(hq // hkv, dim=1)
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    """The descriptions of the calls and the workspace that a program keeps."""
    from paper_2506_03762_amd import binding as B
    if s["kind"] != "rotate":
        s["cache"] = B.Pages.of(s["k_pages"], s["v_pages"], s["table"])
    if s["kind"] == "attend":
        s["p"] = B.SharedAttention.of(s["q"], s["out"], s.get("k_prefix"), s.get("v_prefix"), s["scale"],
                                      n_kv_heads=s["k_pages"].size(1))
        s["ws"] = B.alloc_shared_workspace(s["p"], s["cache"])
    else:
        more = dict(k_out=s["k_out"]) if s["kind"] == "rotate" else dict(v=s["v"])
        s["p"] = B.Rotary.of(s["q"], s["k"], s["q_out"], rot_dim=s["rot"], n_axes=s["positions"].size(0),
                             pairing=B.AHA_PAIR_NEIGHBOURS if s["neighbours"] else B.AHA_PAIR_HALVES,
                             transpose=int(s["transpose"]), **more)


def run(state):
    s = state
    if own:
        return _run_own(s)
    if s["kind"] == "attend":
        return _plain_attend(s)
    cos, sin = _plain_turns(s)
    q, k = _plain_rotate(s["q"], cos, sin, s), _plain_rotate(s["k"], cos, sin, s)
    if s["kind"] == "rotate":
        return dict(q=q, k=k)
    return _plain_append(s, q, k)


def _run_own(s):
    from paper_2506_03762_amd import binding as B
    if s["kind"] == "rotate":
        B.aha_rotate(s["p"], s["q"], s["k"], s["inv_freq"], s["pair_axis"], s["positions"], s["q_out"], s["k_out"])
        return dict(q=s["q_out"], k=s["k_out"])
    if s["kind"] == "append":
        B.aha_append_paged(s["p"], s["cache"], s["q"], s["k"], s["v"], s["inv_freq"], s["pair_axis"], s["positions"],
                           s["table"], s["tail"], s["new"], s["q_out"], s["k_pages"], s["v_pages"])
        return dict(q=s["q_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])
    B.aha_shared_attention(s["p"], s["cache"], s["q"], s.get("k_prefix"), s.get("v_prefix"), s["prefix_len"],
                           s["prefix_first"], s["k_pages"], s["v_pages"], s["table"], s["tail"], s["new"], s["out"],
                           s["lse"], s["ws"])
    return dict(out=s["out"], lse=s["lse"])


# ---- the plain forms ----

def _plain_turns(s):
    """cos and sin [b, 1, n, pairs] of the angles, which are formed in 64 bits: positions are far."""
    turned = s["positions"][s["pair_axis"].long()].permute(1, 2, 0).double() * s["inv_freq"].double()
    turned = -turned if s["transpose"] else turned
    return turned.cos().float().unsqueeze(1), turned.sin().float().unsqueeze(1)


def _plain_rotate(x, cos, sin, s):
    half, f = s["rot"] // 2, x.float()
    if s["neighbours"]:
        a, c = f[..., 0:s["rot"]:2], f[..., 1:s["rot"]:2]
        turned = torch.stack([a * cos - c * sin, a * sin + c * cos], dim=-1).flatten(-2)
    else:
        a, c = f[..., :half], f[..., half:s["rot"]]
        turned = torch.cat([a * cos - c * sin, a * sin + c * cos], dim=-1)
    return torch.cat([turned.to(x.dtype), x[..., s["rot"]:]], dim=-1)


def _plain_new(s):
    """[b, n]: which of the rows are tokens, and their places in their sequence's tail."""
    n = s["q"].size(2)
    t = torch.arange(n, device="cuda")
    new = torch.full_like(s["tail"], n) if s["new"] is None else s["new"]
    return t < new.unsqueeze(1), s["tail"].unsqueeze(1) - new.unsqueeze(1) + t


def _plain_append(s, q, k):
    real, slot = _plain_new(s)
    page = s["table"].long().gather(1, slot.clamp(0, s["table"].size(1) * s["page"] - 1) // s["page"])[real]
    row = (slot % s["page"])[real]
    s["k_pages"][page, :, row] = k.transpose(1, 2)[real]
    s["v_pages"][page, :, row] = s["v"].transpose(1, 2)[real]
    s["q_out"].copy_(torch.where(real[:, None, :, None], q, s["q_out"]))
    return dict(q=s["q_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])


def _plain_attend(s):
    b, hq, n, d = s["q"].shape
    hkv = s["k_pages"].size(1)
    real, slot = _plain_new(s)
    held = torch.arange(s["table"].size(1) * s["page"], device="cuda")
    page = s["table"].long()[:, held // s["page"]]
    keys = s["k_pages"][page.clamp(min=0), :, held % s["page"]].transpose(1, 2).float()
    values = s["v_pages"][page.clamp(min=0), :, held % s["page"]].transpose(1, 2).float()
    seen = (held <= slot.unsqueeze(2)) & (page >= 0).unsqueeze(1)
    if "k_prefix" in s:
        group = torch.bucketize(torch.arange(b, device="cuda", dtype=torch.int32), s["prefix_first"], right=True) - 1
        length = torch.cat([s["prefix_len"], s["prefix_len"].new_zeros(1)])[group]
        group = group.clamp(max=s["k_prefix"].size(0) - 1)
        keys = torch.cat([s["k_prefix"][group].float(), keys], dim=2)
        values = torch.cat([s["v_prefix"][group].float(), values], dim=2)
        ahead = torch.arange(s["k_prefix"].size(2), device="cuda") < length.unsqueeze(1)
        seen = torch.cat([ahead.unsqueeze(1).expand(b, n, -1), seen], dim=2)
    q = s["q"].float().reshape(b, hkv, hq // hkv * n, d) * s["scale"]
    logits = torch.matmul(q, keys.transpose(2, 3).contiguous()).view(b, hq, n, -1)
    logits.masked_fill_(~seen.unsqueeze(1), -math.inf)
    top = logits.amax(dim=3, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    weights = logits.sub_(top).exp_()
    total = weights.sum(dim=3, keepdim=True)
    out = torch.matmul(weights.view(b, hkv, hq // hkv * n, -1), values).view(b, hq, n, d) / total
    out = torch.where(total > 0, out, torch.zeros_like(out)).to(s["q"].dtype)
    lse = (top + total.log()).squeeze(3)
    real = real.unsqueeze(1)
    return dict(out=torch.where(real.unsqueeze(3), out, s["out"]), lse=torch.where(real, lse, s["lse"]))


# ---- from the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(case, s)
    q, k = _exact_turned(case, s, s["q"]), _exact_turned(case, s, s["k"])
    if case["kind"] == "rotate":
        return dict(q=q, k=k)
    new, tail, _, _ = _lengths(case)
    q_out, k_pages, v_pages = (s[x].double() for x in ("q_out", "k_pages", "v_pages"))
    table = s["table"].tolist()
    for b in range(case["batch"]):
        q_out[b, :, :new[b]] = q[b, :, :new[b]]
        at = [divmod(x, case["page"]) for x in range(tail[b] - new[b], tail[b])]
        page, row = torch.tensor([table[b][p] for p, _ in at]), torch.tensor([r for _, r in at])
        k_pages[page, :, row] = k[b, :, :new[b]].transpose(0, 1)
        v_pages[page, :, row] = s["v"][b, :, :new[b]].double().transpose(0, 1)
    return dict(q=q_out, k_pages=k_pages, v_pages=v_pages)


def _exact_turned(case, s, x):
    """A pair as a complex number, times e^(i angle)."""
    x, rot = x.double().clone(), case["rot"]
    at = torch.arange(rot, device="cuda").view(-1, 2).t() if case["neighbours"] else torch.arange(rot, device="cuda").view(2, -1)
    sign = -1.0 if case["transpose"] else 1.0
    for f, axis in enumerate(_axis_of_pair(case)):
        angle = sign * s["positions"][axis].double() * float(s["inv_freq"][f])
        z = torch.complex(x[..., at[0, f]], x[..., at[1, f]]) * torch.polar(torch.ones_like(angle), angle).unsqueeze(1)
        x[..., at[0, f]], x[..., at[1, f]] = z.real, z.imag
    return x


def _exact_attend(case, s):
    new, tail, lens, first = _lengths(case)
    table, page, d = s["table"].tolist(), case["page"], case["d"]
    out, lse = s["out"].double(), s["lse"].double()
    for b in range(case["batch"]):
        slots = [j for j in range(tail[b]) if table[b][j // page] >= 0]
        own_pages, rows = torch.tensor([table[b][j // page] for j in slots]), torch.tensor([j % page for j in slots])
        k, v = (s[x][own_pages, :, rows].double() if slots else s[x][0, :, :0].double().transpose(0, 1)
                for x in ("k_pages", "v_pages"))                                          # [keys, Hkv, d]
        mine = [g for g in range(len(lens)) if first[g] <= b < first[g + 1]]
        ahead = lens[mine[0]] if mine else 0
        if ahead:
            k, v = (torch.cat([s[x][mine[0], :, :ahead].double().transpose(0, 1), y]) for x, y in (("k_prefix", k), ("v_prefix", v)))
        place = torch.tensor([-1] * ahead + slots, device="cuda")
        limit = torch.arange(tail[b] - new[b], tail[b], device="cuda")
        hidden = place.unsqueeze(0) > limit.unsqueeze(1)
        for h in range(case["hq"]):
            kv = h * case["hkv"] // case["hq"]
            a = (s["q"][b, h, :new[b]].double() @ k[:, kv].t() * s["scale"]).masked_fill(hidden, -math.inf)
            lse[b, h, :new[b]] = torch.logsumexp(a, dim=1)
            out[b, h, :new[b]] = torch.nan_to_num(torch.softmax(a, dim=1), nan=0.0) @ v[:, kv]
    return dict(out=out, lse=lse)


def work(case):
    """Every input read once and every output written once, the prefix once for all that share it; each
    product formed once."""
    d, hq, hkv, e = case["d"], case["hq"], case["hkv"], 4 if case["dtype"] == "f32" else 2
    tokens = case["batch"] * case["n"]
    if case["kind"] != "rotate":
        new, tail, lens, first = _lengths(case)
        tokens = sum(new)
    if case["kind"] != "attend":
        heads = hq + hkv + (hkv if case["kind"] == "append" else 0)
        return {"bytes": tokens * (2 * heads * d * e + 4 * case["axes"]), "flops": 3.0 * tokens * (hq + hkv) * case["rot"]}
    table, seen, read = _pages(case, tail)[2], 0, 0
    for b in range(case["batch"]):
        there = [table[b][j // case["page"]] >= 0 for j in range(tail[b])]
        ahead = sum(n for n, lo, hi in zip(lens, first, first[1:]) if lo <= b < hi)
        before = sum(there[:tail[b] - new[b]])
        read += sum(there)
        seen += sum(ahead + before + sum(there[tail[b] - new[b]:tail[b] - new[b] + t + 1]) for t in range(new[b]))
    shared = sum(n for n, lo, hi in zip(lens, first, first[1:]) if hi > lo)
    return {"bytes": 2 * (read + shared) * hkv * d * e + tokens * hq * (2 * d * e + 4), "flops": 4.0 * d * hq * seen}

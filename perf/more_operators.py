"""Work of the operators that carry a batch of prompts into generation with a bounded cache, to be measured.

Three kinds of pass, as the program around a language model makes them, one layer each:

  prompt  the causal attention of packed prompts of different lengths, output and log-sum-exp;
  attend  the attention of one new token of every sequence over its paged cache, and the weights that the tokens of
          the cache get, added to their running scores;
  evict   sequences brought back to their budget: the tokens of the smallest scores go, those behind the budget move
          into their places.

`own` chooses between the operators' plain form, elementary operations in 32 bits, and the framework's
entry points.  Lengths and page tables follow from the case alone, what the tensors hold from the seed.
"""
import math
import random

import torch

own = False

KEY_MEAN = 0.7             # of a KV head's keys along a direction that its queries lean on, too
FREE_PAGES = 3             # pages of the pool that no sequence holds
PADDING_ROWS = 5           # behind the last of ragged prompts
ROWS_BEFORE = 16           # whose weights the running scores of a cache that is attended to hold
SEEN = 4                   # tokens that a sequence has seen for each that its cache holds


def _prompt(name, sequences, n, hq, hkv, d, **more):
    case = dict(kind="prompt", sequences=sequences, n=n, hq=hq, hkv=hkv, d=d, ragged=False, dtype="bf16", layout="thd")
    return _named(case, name, more)


def _attend(name, batch, held, hq, hkv, d, budget, page, **more):
    case = dict(kind="attend", batch=batch, held=held, hq=hq, hkv=hkv, d=d, budget=budget, page=page, ragged=False,
                holes=False, adaptive=True, dtype="bf16", layout="pages, heads, rows")
    return _named(case, name, more)


def _evict(name, batch, held, hkv, d, budget, recent, page, **more):
    case = dict(kind="evict", batch=batch, held=held, hkv=hkv, d=d, budget=budget, recent=recent, sink=0, page=page,
                fresh=False, ragged=False, dtype="bf16", layout="pages, heads, rows")
    return _named(case, name, more)


def _named(case, name, more):
    if name:
        case["name"] = name
    case.update(more)
    return case


def listed():
    return [
        # a short prompt of a small fp32 model, where latency is everything
        _prompt("prompt_short_f32", 1, 512, 2, 2, 64, dtype="f32"),
        # what a server packs into one step: questions of several lengths, one layer of a grouped-query model
        _prompt("prompt_packed", 24, 1500, 32, 8, 128, ragged=True),
        # a whole long document: products
        _prompt("prompt_long", 1, 16384, 32, 8, 128),
        # sizes that divide nothing, empty prompts among them, head-major
        _prompt("prompt_odd", 9, 777, 6, 2, 64, ragged=True, layout="htd"),
        # eight sequences whose prompts were compacted: latency
        _attend("attend_few", 8, 2049, 32, 8, 128, 2048, 64),
        # a server's batch: bound by the bytes of the cache
        _attend("attend_batch", 64, 4096, 32, 8, 128, 4095, 64, ragged=True),
        # one sequence with a long cache and eight query heads per KV head
        _attend("attend_long", 1, 131072, 64, 8, 128, 131072, 64, adaptive=False),
        # fp32, ragged, small pages of which some have been given back
        _attend("attend_odd_f32", 7, 901, 6, 2, 64, 700, 16, ragged=True, holes=True, dtype="f32",
                layout="pages, rows, heads"),
        # a generation step's eviction: one token of every head goes
        _evict("evict_step", 64, 2049, 8, 128, 2048, 64, 64),
        # prompts of several lengths brought to a budget, scores as the prefill leaves them
        _evict("evict_prompt", 8, 16384, 8, 128, 2048, 64, 64, fresh=True, ragged=True),
        # a long prompt, first tokens kept
        _evict("evict_long", 1, 32768, 8, 128, 2048, 64, 64, fresh=True, sink=4),
        # fp32, ragged (some sequences below the budget), small pages, several tokens at once
        _evict("evict_odd_f32", 5, 333, 2, 64, 201, 10, 16, ragged=True, dtype="f32", layout="pages, rows, heads"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes over the ranges that the listed ones stand for, odd ones among them."""
    kind = rng.choice(["prompt", "prompt", "attend", "attend", "evict", "evict"])
    f32 = rng.random() < 0.2
    d, hkv, group = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 7, 8])
    dtype = "f32" if f32 else "bf16"
    if kind == "prompt":
        hq = hkv * group
        n, sequences = _log_int(rng, 1, 4096 if f32 else 16384), _log_int(rng, 1, 32)
        while sequences > 1 and hq * (sequences * n) ** 2 > 32 * 16384 ** 2:
            sequences = sequences // 2
        while hq * (sequences * n) ** 2 > (8 if f32 else 32) * (4096 if f32 else 16384) ** 2:
            n = n * 2 // 3
        return _prompt(None, sequences, n, hq, hkv, d, ragged=sequences > 1 and rng.random() < 0.7, dtype=dtype,
                       layout=rng.choice(["thd", "thd", "htd"]))
    batch, page = _log_int(rng, 1, 64), rng.choice([1, 8, 16, 32, 64, 64, 128, 256])
    more = dict(dtype=dtype, layout=rng.choice(["pages, heads, rows", "pages, rows, heads"]), ragged=rng.random() < 0.6)
    held = _log_int(rng, 1, 131072 if kind == "attend" else 32768)
    while batch > 1 and batch * held * hkv * d * (2 if f32 else 1) > 131072 * 8 * 128:
        batch //= 2
    while held * hkv * d * (2 if f32 else 1) > 131072 * 8 * 128:
        held //= 2
    if kind == "attend":
        return _attend(None, batch, held, hkv * group, hkv, d, rng.randint(1, held), page, holes=rng.random() < 0.3,
                       adaptive=rng.random() < 0.7, **more)
    budget = rng.choice([held - 1, rng.randint(1, held), _log_int(rng, 1, held)])
    budget = max(1, budget)
    recent = rng.randint(0, min(budget, 128))
    return _evict(None, batch, held, hkv, d, budget, recent, page, fresh=rng.random() < 0.5,
                  sink=rng.randint(0, min(4, budget - recent)), **more)


# ---- what follows from the case: lengths, pages ----

def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """Tokens of the prompts, or of the sequences' caches: the first has all, the others of a ragged case any number."""
    count = case["sequences"] if case["kind"] == "prompt" else case["batch"]
    most = case["n"] if case["kind"] == "prompt" else case["held"]
    rng = random.Random(count * 1009 + most * 31 + case["d"])
    least = 0 if case["kind"] == "prompt" else 1
    return [rng.randint(least, most) if case["ragged"] and b else most for b in range(count)]


def _pages(case, held):
    """Pages of the pool and the table [batch, width]: pages in no order, some given back (-1) at the start of every
    third sequence of a case with holes."""
    width = -(-case["held"] // case["page"])
    rng = random.Random(case["page"] * 7 + case["batch"])
    pages = [-(-x // case["page"]) for x in held]
    pool = list(range(sum(pages) + FREE_PAGES))
    rng.shuffle(pool)
    table = [[pool.pop() for _ in range(p)] + [-1] * (width - p) for p in pages]
    if case.get("holes"):
        for b in range(0, case["batch"], 3):
            table[b][:pages[b] // 3] = [-1] * (pages[b] // 3)
    return sum(pages) + FREE_PAGES, table


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(case, gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=_dtype(case))


def _pool(case, gen, pages):
    """A pool [pages, Hkv, page, d] of Gaussian rows in the layout of the case."""
    hkv, page, d = case["hkv"], case["page"], case["d"]
    if case["layout"] == "pages, rows, heads":
        return _normal(case, gen, pages, page, hkv, d).transpose(1, 2)
    return _normal(case, gen, pages, hkv, page, d)


def _rows(case, gen, tokens, heads):
    """Gaussian rows [tokens, heads, d] in the layout of the case."""
    if case["layout"] == "htd":
        return _normal(case, gen, heads, tokens, case["d"]).transpose(0, 1)
    return _normal(case, gen, tokens, heads, case["d"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"prompt": _prepare_prompt, "attend": _prepare_attend, "evict": _prepare_evict}[case["kind"]](case, gen)
    s["kind"] = case["kind"]
    if own:
        _prepare_own(s)
    return s


def _prepare_prompt(case, gen):
    lens, hq, hkv, d = _lengths(case), case["hq"], case["hkv"], case["d"]
    tokens = sum(lens) + (PADDING_ROWS if case["ragged"] else 0)
    lean = _normal(case, gen, 1, hkv, d)
    q, k, v = (_rows(case, gen, tokens, h) for h in (hq, hkv, hkv))
    k += KEY_MEAN * lean
    q += lean.repeat_interleave(hq // hkv, dim=1)
    return dict(q=q, k=k, v=v, first=_int32([sum(lens[:b]) for b in range(len(lens) + 1)]), scale=1.0 / math.sqrt(d),
                out=torch.zeros_like(q), lse=torch.zeros((hq, tokens), device="cuda"))


def _cache(case, gen):
    """A paged cache and what goes with its tokens: positions in order, the last one the newest, and running scores."""
    held = _lengths(case)
    pages, table = _pages(case, held)
    b, hkv, slots = case["batch"], case["hkv"], len(table[0]) * case["page"]
    tail = _int32(held)
    place = torch.arange(slots, device="cuda", dtype=torch.int32).expand(b, hkv, slots)
    skipped = torch.randint(0, SEEN, (b, hkv, slots), generator=gen, device="cuda", dtype=torch.int32)
    pos = SEEN * place + skipped
    newest = (place == tail.view(b, 1, 1) - 1)
    pos = torch.where(newest, SEEN * tail.view(b, 1, 1) - 1, pos)
    scores = torch.randn((b, hkv, slots), generator=gen, device="cuda").mul_(2.0).exp_()
    return dict(k_pages=_pool(case, gen, pages), v_pages=_pool(case, gen, pages), page=case["page"], table=_int32(table),
                tail=tail, seen=SEEN * tail, scores=scores, pos=pos.contiguous())


def _prepare_attend(case, gen):
    s = _cache(case, gen)
    b, hq, hkv, d = case["batch"], case["hq"], case["hkv"], case["d"]
    lean = _normal(case, gen, 1, hkv, d)
    s["k_pages"] += KEY_MEAN * lean.unsqueeze(2)
    q = _normal(case, gen, b, hq, d) + lean.repeat_interleave(hq // hkv, dim=1)
    s["scores"] *= ROWS_BEFORE * (hq // hkv) / (math.exp(2.0) * case["held"])
    s.update(q=q, out=torch.zeros_like(q), lse=torch.zeros((b, hq), device="cuda"), scale=1.0 / math.sqrt(d),
             budget=case["budget"], adaptive=case["adaptive"])
    return s


def _prepare_evict(case, gen):
    s = _cache(case, gen)
    s.update(budget=case["budget"], recent=case["recent"], sink=case["sink"], len_out=torch.zeros_like(s["tail"]),
             scores_out=s["scores"], pos_out=s["pos"])
    if case["fresh"]:  # the prompt's scores; token j is position j
        s.update(seen=None, pos=None, scores_out=torch.zeros_like(s["scores"]), pos_out=torch.full_like(s["pos_out"], -1))
    return s


def _prepare_own(s):
    """The descriptions of the calls and the workspace that a program keeps."""
    from paper_2506_03762_amd import binding as B
    if s["kind"] == "prompt":
        s["p"] = B.PromptAttention.of(s["q"], s["k"], s["v"], s["out"], s["first"], scale=s["scale"])
        s["ws"] = B.alloc_prompt_workspace(s["p"])
        return
    s["cache"] = B.Pages.of(s["k_pages"], s["v_pages"], s["table"])
    if s["kind"] == "attend":
        s["p"] = B.PagedAttention.of(s["q"], s["out"], s["scores"], s["pos"], scale=s["scale"], budget=s["budget"],
                                     scale_mode=B.AHA_SCALE_ADAPTIVE if s["adaptive"] else B.AHA_SCALE_FIXED,
                                     fixed_scale=s["scale"])
        s["ws"] = B.alloc_paged_workspace(s["p"], s["cache"])
    else:
        s["p"] = B.PagedEviction.of(s["scores"], s["pos"], s["scores_out"], s["pos_out"], s["cache"], budget=s["budget"],
                                    recent=s["recent"], sink=s["sink"])
        s["ws"] = B.alloc_evict_workspace(s["p"], s["cache"])


def run(state):
    s = state
    if own:
        return _run_own(s)
    return {"prompt": _plain_prompt, "attend": _plain_attend, "evict": _plain_evict}[s["kind"]](s)


def _run_own(s):
    from paper_2506_03762_amd import binding as B
    if s["kind"] == "prompt":
        B.aha_prompt_attention(s["p"], s["q"], s["k"], s["v"], s["first"], s["out"], s["lse"], s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    if s["kind"] == "attend":
        B.aha_paged_attention(s["p"], s["cache"], s["q"], s["k_pages"], s["v_pages"], s["table"], s["tail"], s["seen"],
                              s["scores"], s["pos"], s["out"], s["lse"], s["ws"])
        return dict(out=s["out"], lse=s["lse"], scores=s["scores"], pos=s["pos"])
    B.aha_paged_evict(s["p"], s["cache"], s["scores"], s["pos"], s["k_pages"], s["v_pages"], s["table"], s["tail"],
                      s["seen"], s["scores_out"], s["pos_out"], s["len_out"], s["ws"])
    return _evicted(s)


def _evicted(s):
    return dict(k_pages=s["k_pages"], v_pages=s["v_pages"], scores=s["scores_out"], pos=s["pos_out"], length=s["len_out"])


# ---- the plain forms ----

def _plain_prompt(s):
    """All rows against all keys, those of other prompts and later ones masked."""
    t, hq, d = s["q"].shape
    hkv = s["k"].size(1)
    place = torch.arange(t, device="cuda", dtype=torch.int32)
    mine = torch.bucketize(place, s["first"], right=True)  # 1 .. prompts; behind the last: one more
    seen = (mine.unsqueeze(1) == mine) & (place.unsqueeze(1) >= place)
    real = mine < s["first"].numel()
    q = s["q"].transpose(0, 1).float().reshape(hkv, hq // hkv * t, d) * s["scale"]
    logits = torch.matmul(q, s["k"].permute(1, 2, 0).float().contiguous()).view(hq, t, t)
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(dim=2, keepdim=True)
    weights = logits.sub_(top).exp_()
    total = weights.sum(dim=2, keepdim=True)
    values = s["v"].transpose(0, 1).float().contiguous()
    out = torch.matmul(weights.view(hkv, hq // hkv * t, t), values).view(hq, t, d) / total
    lse = (top + total.log()).squeeze(2)
    out = out.transpose(0, 1).to(s["q"].dtype)
    return dict(out=torch.where(real.view(-1, 1, 1), out, s["out"]), lse=torch.where(real, lse, s["lse"]))


def _score_scale(s, d):
    """[b] softmax scales of the accumulated weights."""
    if not s["adaptive"]:
        return torch.full(s["tail"].shape, s["scale"], device="cuda")
    gain = (s["seen"].double() / s["budget"]).log().clamp(min=0.0)
    return (2.0 * gain / d).sqrt().clamp(min=1.0 / math.sqrt(d)).float()


def _plain_attend(s):
    b, hq, d = s["q"].shape
    hkv, slots = s["k_pages"].size(1), s["scores"].size(2)
    held = torch.arange(slots, device="cuda")
    page = s["table"].long()[:, held // s["page"]]
    keys = s["k_pages"][page.clamp(min=0), :, held % s["page"]].permute(0, 2, 3, 1).float().contiguous()
    values = s["v_pages"][page.clamp(min=0), :, held % s["page"]].transpose(1, 2).float().contiguous()
    there = (held < s["tail"].unsqueeze(1)) & (page >= 0)
    dots = torch.matmul(s["q"].float().view(b, hkv, hq // hkv, d), keys).view(b, hq, slots)
    dots.masked_fill_(~there.unsqueeze(1), -math.inf)
    weights, total, lse = _softmax(dots * s["scale"])
    out = torch.matmul(weights.view(b, hkv, hq // hkv, slots), values).view(b, hq, d) / total
    s["out"].copy_(torch.where(total > 0, out, torch.zeros_like(out)))
    s["lse"].copy_(lse)
    weights, total, _ = _softmax(dots * _score_scale(s, d).view(b, 1, 1))
    added = (weights / total.clamp(min=1e-30)).view(b, hkv, hq // hkv, slots).sum(dim=2)
    newest = (held == s["tail"].unsqueeze(1) - 1).unsqueeze(1)
    kept = torch.where(newest, torch.zeros_like(s["scores"]), s["scores"])
    s["scores"].copy_(torch.where(held < s["tail"].view(b, 1, 1), kept + added, s["scores"]))
    s["pos"].copy_(torch.where(newest, s["seen"].view(b, 1, 1) - 1, s["pos"]))
    return dict(out=s["out"], lse=s["lse"], scores=s["scores"], pos=s["pos"])


def _softmax(logits):
    """Weights relative to the largest, their sum, and the log-sum-exp of the rows."""
    top = logits.amax(dim=2, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    weights = logits.sub_(top).exp_()
    total = weights.sum(dim=2, keepdim=True)
    return weights, total, (top + total.log()).squeeze(2)


def _plain_evict(s):
    """Every token's rank by protection, score and position (of equal ones the later goes first); the gaps below the
    new length take, in order, the tokens that stay and lie behind it."""
    slots, hkv = s["scores"].size(2), s["scores"].size(1)
    place = torch.arange(slots, device="cuda")
    tail = s["tail"].view(-1, 1, 1)
    new = tail.clamp(max=s["budget"])
    pos = (place.expand_as(s["scores"]) if s["pos"] is None else s["pos"]).long()
    seen = tail if s["seen"] is None else s["seen"].view(-1, 1, 1)
    held = place < tail
    safe = (pos >= seen - s["recent"]) | (pos < s["sink"])
    score = (s["scores"] + 0.0).masked_fill(~(held & ~safe), math.inf)
    by_pos = torch.argsort(pos.flip(2), dim=2, descending=True, stable=True)            # places from the last one
    order = by_pos.gather(2, torch.argsort(score.flip(2).gather(2, by_pos), dim=2, stable=True))
    order = slots - 1 - order
    order = order.gather(2, torch.argsort((safe & held).gather(2, order).int() + 2 * (~held).expand_as(safe).gather(2, order).int(),
                                          dim=2, stable=True))
    gone = torch.zeros_like(held.expand_as(safe)).scatter(2, order, (place < tail - new).expand_as(safe))
    gap, mover = gone & (place < new), held & ~gone & (place >= new)
    b, h, to = gap.nonzero(as_tuple=True)
    _, _, at = mover.nonzero(as_tuple=True)
    into, from_ = s["table"].long()[b, to // s["page"]], s["table"].long()[b, at // s["page"]]
    for pool in (s["k_pages"], s["v_pages"]):
        pool[into, h, to % s["page"]] = pool[from_, h, at % s["page"]]
    source = place.expand_as(safe).clone()
    source[b, h, to] = at
    stays = (place < new).expand_as(safe)
    s["scores_out"].copy_(torch.where(stays, s["scores"].gather(2, source), s["scores_out"]))
    s["pos_out"].copy_(torch.where(stays, pos.gather(2, source).int(), s["pos_out"]))
    s["len_out"].copy_(new.view(-1))
    return _evicted(s)


# ---- from the definitions, in 64 bits ----

def exact(case, seed):
    s = prepare(case, seed)
    return {"prompt": _exact_prompt, "attend": _exact_attend, "evict": _exact_evict}[case["kind"]](case, s)


def _exact_prompt(case, s):
    out, lse = s["out"].double(), s["lse"].double()
    first = s["first"].tolist()
    for lo, hi in zip(first, first[1:]):
        if hi == lo:
            continue
        later = torch.ones(hi - lo, hi - lo, dtype=torch.bool, device="cuda").triu(1)
        for h in range(case["hq"]):
            kv = h * case["hkv"] // case["hq"]
            a = s["q"][lo:hi, h].double() @ s["k"][lo:hi, kv].double().t() * s["scale"]
            a.masked_fill_(later, -math.inf)
            lse[h, lo:hi] = torch.logsumexp(a, dim=1)
            out[lo:hi, h] = torch.softmax(a, dim=1) @ s["v"][lo:hi, kv].double()
    return dict(out=out, lse=lse)


def _exact_attend(case, s):
    out, lse, scores, pos = s["out"].double(), s["lse"].double(), s["scores"].double(), s["pos"].clone()
    held, group, d = _lengths(case), case["hq"] // case["hkv"], case["d"]
    for b, n in enumerate(held):
        place = torch.arange(n, device="cuda")
        page = s["table"][b].long()[place // case["page"]]
        place, page = place[page >= 0], page[page >= 0]
        gain = s["scale"]
        if case["adaptive"]:
            gain = max(1.0 / math.sqrt(d), math.sqrt(2.0 * max(0.0, math.log(SEEN * n / case["budget"])) / d))
        scores[b, :, n - 1] = 0.0
        pos[b, :, n - 1] = SEEN * n - 1
        for kv in range(case["hkv"]):
            k, v = (s[x][page, kv, place % case["page"]].double() for x in ("k_pages", "v_pages"))
            rows = slice(kv * group, (kv + 1) * group)
            x = s["q"][b, rows].double() @ k.t()
            lse[b, rows] = torch.logsumexp(x * s["scale"], dim=1)
            if len(place):
                out[b, rows] = torch.softmax(x * s["scale"], dim=1) @ v
                scores[b, kv, place] += torch.softmax(x * gain, dim=1).sum(dim=0)
    return dict(out=out, lse=lse, scores=scores, pos=pos)


def _exact_evict(case, s):
    k, v = s["k_pages"].double(), s["v_pages"].double()
    scores, pos, held = s["scores_out"].double(), s["pos_out"].clone(), _lengths(case)
    given_scores = s["scores"].tolist()
    given_pos = None if s["pos"] is None else s["pos"].tolist()
    table, page = s["table"].tolist(), case["page"]
    into, source = [], []
    for b, n in enumerate(held):
        keep, seen = min(n, case["budget"]), n if case["fresh"] else SEEN * n
        for h in range(case["hkv"]):
            at = list(range(n)) if given_pos is None else given_pos[b][h][:n]
            safe = [p >= seen - case["recent"] or p < case["sink"] for p in at]
            worth = sorted(range(n), key=lambda j: (safe[j], 0.0 if safe[j] else given_scores[b][h][j], -at[j], -j))
            stays = set(worth[n - keep:])
            movers = iter(j for j in range(keep, n) if j in stays)
            into += [(b, h, j) for j in range(keep)]
            source += [(b, h, j if j in stays else next(movers)) for j in range(keep)]
    i, j = (torch.tensor(x, device="cuda").t() for x in (into, source))
    tables = torch.tensor(table, device="cuda")
    for pool in (k, v):
        pool[tables[i[0], i[2] // page], i[1], i[2] % page] = pool[tables[j[0], j[2] // page], j[1], j[2] % page]
    scores[i[0], i[1], i[2]] = s["scores"].double()[j[0], j[1], j[2]]
    pos[i[0], i[1], i[2]] = (j[2] if s["pos"] is None else s["pos"][j[0], j[1], j[2]]).int()
    return dict(k_pages=k, v_pages=v, scores=scores, pos=pos, length=_int32([min(n, case["budget"]) for n in held]))


def work(case):
    """Every input read once and every output written once; each product of a row and a key that it sees formed once."""
    d, hkv, e, held = case["d"], case["hkv"], 4 if case["dtype"] == "f32" else 2, _lengths(case)
    if case["kind"] == "prompt":
        hq, tokens = case["hq"], sum(held)
        return {"bytes": tokens * (2 * (hq + hkv) * d * e + 4 * hq), "flops": sum(2.0 * d * hq * n * (n + 1) for n in held)}
    if case["kind"] == "attend":
        table, hq = _pages(case, held)[1], case["hq"]
        there = sum(table[b][j // case["page"]] >= 0 for b, n in enumerate(held) for j in range(n))
        return {"bytes": there * hkv * (2 * d * e + 8) + case["batch"] * hq * (2 * d * e + 4), "flops": 4.0 * d * hq * there}
    # kept tokens behind the new length: the recent ones, and of the others as many as lie there
    moved = values = 0.0
    for n in held:
        keep, fixed = min(n, case["budget"]), case["recent"] + case["sink"]
        if n > keep:
            recent = min(case["recent"] if case["fresh"] else (case["recent"] + SEEN - 1) // SEEN, keep, n - keep)
            moved += recent + (keep - min(keep, fixed)) * max(0, n - keep - recent) / max(1, n - fixed) if n > keep + 1 else 1
        values += n * (1 if case["fresh"] else 2) + (2 * keep if case["fresh"] else 0)
    return {"bytes": hkv * (moved * 4 * d * e + values * 4), "flops": float(hkv * sum(held))}

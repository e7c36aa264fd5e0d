"""Packed prompts' attention, their eviction into the paged cache and generation with running scores together, as a program
uses them; calls captured into graphs, on two streams, with far strides."""
import numpy as np
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests.paged_cases import NAN, Evictions, Prompts, Steps, i32
from tests.shared_cases import assert_within, gaussian

pytestmark = pytest.mark.gpu


def on_host(case, d, **more):
    """The case with the caches, scores and lengths that the GPU holds now."""
    for name in ("k", "v", "scores", "pos", "table"):
        setattr(case, name, d[name].cpu())
    case.tail = d["tail"].tolist()
    case.seen = d["seen"].tolist()
    case.__dict__.update(more)
    return case


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_prompts_are_packed_evicted_and_continued(dtype):
    """Three prompts of different lengths: turned, attended to, appended to pages, scored from the attention's own
    normalisers, evicted to the budget; then generation: append, attend with running scores, evict.  Every call's results
    are compared, with what the GPU held before it."""
    lens, hq, hkv, d, budget, recent, window, page, width = [300, 45, 171], 8, 2, 64, 64, 16, 16, 16, 20
    batch, freq = len(lens), B.rotary_tables(d)[0]
    c = Prompts(1, lens, q_heads=hq, kv_heads=hkv, d=d, dtype=dtype)
    dev = c.upload()
    q4, k4 = (t.transpose(0, 1).unsqueeze(0) for t in (dev["q"], dev["k"]))
    at = torch.cat([torch.arange(n, dtype=torch.int32) for n in lens]).reshape(1, 1, -1).cuda()
    B.aha_rotate(B.Rotary.of(q4, k4, q4, k4), q4, k4, freq, None, at, q4, k4)
    c.run(dev)
    c.q, c.k = dev["q"].cpu(), dev["k"].cpu()
    c.check(dev)

    pools = [torch.zeros(batch * width, hkv, page, d, dtype=dtype, device="cuda") for _ in range(2)]
    table = torch.from_numpy(np.random.default_rng(2).permutation(batch * width).reshape(batch, width).astype(np.int32)).cuda()
    cache = B.Pages.of(*pools, table)
    fresh = torch.zeros(batch, hkv, width * page, device="cuda")
    longest = max(lens)
    padded = [torch.zeros(batch, hkv, longest, d, dtype=dtype, device="cuda") for _ in range(2)]
    for b, n in enumerate(lens):
        lo, hi = c.first[b], c.first[b + 1]
        for t, x in zip(padded, (dev["k"], dev["v"])):
            t[b, :, :n] = x[lo:hi].transpose(0, 1)
        q, k, v = (dev[x][lo:hi].transpose(0, 1).unsqueeze(0) for x in "qkv")
        p = B.Params(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_len=n, window=window, budget=min(budget, n), recent=recent,
                     dtype=B.AHA_BF16 if dtype == torch.bfloat16 else B.AHA_F32, scale_mode=B.AHA_SCALE_FIXED,
                     fixed_scale=d ** -0.5).with_strides(q, k, v)
        ws = B.alloc_workspace(p)
        given, own = (torch.empty(1, hkv, n, device="cuda") for _ in range(2))
        B.aha_prefill_scores_lse(p, q, k, v, dev["lse"][:, hi - window:hi].contiguous(), given, ws)
        B.aha_prefill_scores(p, q, k, v, own, ws)
        # normalisers of another kernel: 5e-6 of the exponent's argument at most in fp32 logits of tens, as the rows' own
        assert torch.allclose(given, own, rtol=1e-4)
        fresh[b, :, :n] = given[0]
    tail = i32(lens)
    rot = B.Rotary.of(None, padded[0], None, v=padded[1], rot_dim=0)
    B.aha_append_paged(rot, cache, None, *padded, None, None, None, table, tail, tail, None, *pools)

    scores, pos = torch.zeros_like(fresh), torch.full(fresh.shape, -1, dtype=torch.int32, device="cuda")
    e = Evictions(3, lens, budget=budget, recent=recent, in_place=False, with_pos=False, kv_heads=hkv, d=d, page=page, width=width, dtype=dtype)
    held = dict(k=pools[0], v=pools[1], scores=fresh, pos=pos, table=table, tail=tail, seen=i32(lens), cache=cache)
    on_host(e, held)
    held.update(scores_out=scores, pos_out=pos, len_out=i32([0] * batch))
    held["scores_out"].fill_(NAN)
    held["pos_out"].fill_(-7)
    held["p"] = B.PagedEviction.of(fresh, None, scores, pos, cache, budget=budget, recent=recent)
    held["ws"] = B.alloc_evict_workspace(held["p"], cache)
    e.run(held)
    e.check(held)

    held.update(scores=scores, tail=held["len_out"], q=torch.zeros(batch, hq, d, dtype=dtype, device="cuda"),
                lse=torch.zeros(batch, hq, device="cuda"))
    held["out"] = torch.zeros_like(held["q"])
    held["p_attend"] = B.PagedAttention.of(held["q"], held["out"], scores, pos, budget=budget)
    held["ws_attend"] = B.alloc_paged_workspace(held["p_attend"], cache)
    held["p_evict"] = B.PagedEviction.of(scores, pos, scores, pos, cache, budget=budget, recent=recent)
    held["ws_evict"] = B.alloc_evict_workspace(held["p_evict"], cache)
    for step in range(25):
        held["tail"] = held["tail"] + 1
        held["seen"] = held["seen"] + 1
        q, k, v = (gaussian(100 + 3 * step + i, batch, h, 1, d, dtype=dtype).cuda() for i, h in ((0, hq), (1, hkv), (2, hkv)))
        q_out = held["q"].unsqueeze(2)
        B.aha_append_paged(B.Rotary.of(q, k, q_out, v=v), cache, q, k, v, freq, None, (held["seen"] - 1).view(1, batch, 1), table, held["tail"],
                           None, q_out, *pools)
        s = Steps(4, held["tail"].tolist(), q_heads=hq, kv_heads=hkv, d=d, page=page, width=width, dtype=dtype, budget=budget)
        on_host(s, held, q=held["q"].cpu())
        held.update(p=held["p_attend"], ws=held["ws_attend"])
        s.run(held)
        if step % 6 == 0:
            s.check(held)
        e = Evictions(5, s.tail, budget=budget, recent=recent, kv_heads=hkv, d=d, page=page, width=width, dtype=dtype)
        on_host(e, held)
        held.update(p=held["p_evict"], ws=held["ws_evict"], scores_out=scores, pos_out=pos, len_out=i32([0] * batch))
        e.run(held)
        if step % 6 == 0:
            e.check(held)
        held["tail"] = held["len_out"]
    assert held["tail"].tolist() == [budget] * batch
    for b in range(batch):
        for h in range(hkv):
            left = pos[b, h, :budget].tolist()
            assert len(set(left)) == budget and set(range(lens[b] + 25 - recent, lens[b] + 25)) <= set(left)


def test_captured_steps_follow_the_lengths():
    """A step's append, attention and eviction captured into a graph; replayed with other lengths and rows, with eager calls and
    synchronizations between the replays: bit by bit the eager calls' results each time."""
    batch, hq, hkv, d, page, width, budget = 4, 8, 2, 128, 16, 12, 100
    pools0 = [gaussian(s, batch * width, hkv, page, d, dtype=torch.bfloat16).cuda() for s in (1, 2)]
    pools = [t.clone() for t in pools0]
    table = torch.randperm(batch * width, generator=torch.Generator().manual_seed(3)).int().view(batch, width).cuda()
    cache = B.Pages.of(*pools, table)
    scores0 = torch.rand(batch, hkv, width * page, device="cuda")
    pos0 = torch.arange(width * page, dtype=torch.int32, device="cuda").expand(batch, hkv, -1).contiguous()
    scores, pos = scores0.clone(), pos0.clone()
    q, k, v = (gaussian(s, batch, h, 1, d, dtype=torch.bfloat16).cuda() for s, h in ((4, hq), (5, hkv), (6, hkv)))
    q_out = torch.zeros_like(q)
    out, lse = torch.zeros(batch, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(batch, hq, device="cuda")
    tail, seen, len_out = i32([1] * batch), i32([1] * batch), i32([0] * batch)
    at, freq = torch.zeros(1, batch, 1, dtype=torch.int32, device="cuda"), B.rotary_tables(d)[0]
    rot = B.Rotary.of(q, k, q_out, v=v)
    pa = B.PagedAttention.of(q_out[:, :, 0], out, scores, pos, budget=budget)
    pe = B.PagedEviction.of(scores, pos, scores, pos, cache, budget=budget, recent=5)
    wa, we = B.alloc_paged_workspace(pa, cache), B.alloc_evict_workspace(pe, cache)

    def step():
        B.aha_append_paged(rot, cache, q, k, v, freq, None, at, table, tail, None, q_out, *pools)
        B.aha_paged_attention(pa, cache, q_out[:, :, 0], *pools, table, tail, seen, scores, pos, out, lse, wa)
        B.aha_paged_evict(pe, cache, scores, pos, *pools, table, tail, seen, scores, pos, len_out, we)

    def reset(i):
        g = torch.Generator().manual_seed(i)
        tail.copy_(torch.randint(1, width * page, (batch,), generator=g))
        seen.copy_(torch.randint(200, 3000, (batch,), generator=g))
        at.copy_((seen - 1).view(1, batch, 1))
        q.copy_(torch.randn(q.shape, generator=g))
        for t, t0 in zip(pools + [scores, pos], pools0 + [scores0, pos0]):
            t.copy_(t0)

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    reset(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    small = Steps(7, [20, 3], q_heads=4, kv_heads=2, d=64, page=8)
    other = small.upload()
    results = lambda: [t.clone() for t in (out, lse, scores, pos, len_out, q_out, *pools)]
    for i in range(1, 7):
        reset(i)
        graph.replay()
        torch.cuda.synchronize()
        got = results()
        small.run(other)
        reset(i)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, results())), "replay %d" % i


def test_captured_prompts_follow_their_lengths():
    c = Prompts(8, [500, 300], q_heads=4, kv_heads=2, d=128)
    d = c.upload()
    c.run(d)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            c.run(d)
    for first in ([0, 800, 800], [0, 1, 800], [3, 400, 790], [0, 500, 800]):
        c.first, c.lens = first, [first[1] - first[0], first[2] - first[1]]
        d["first"].copy_(i32(first))
        d["out"].fill_(NAN)
        d["lse"].fill_(NAN)
        graph.replay()
        c.check(d)


def test_two_streams_at_once():
    """The same kinds of call on two streams, each with its own workspace."""
    cases = [Steps(9 + i, [700, 40, 1000], q_heads=8, kv_heads=2, d=128, page=32) for i in range(2)]
    prompts = [Prompts(11 + i, [400, 90], q_heads=4, kv_heads=2, d=128) for i in range(2)]
    evictions = [Evictions(13 + i, [700, 40, 300], kv_heads=2, d=128, budget=50, page=32) for i in range(2)]
    devs = [[x.upload() for x in t] for t in zip(cases, prompts, evictions)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for i, st in enumerate(streams):
        with torch.cuda.stream(st):
            for x, d in zip((cases[i], prompts[i], evictions[i]), devs[i]):
                x.run(d)
    torch.cuda.synchronize()
    for i in range(2):
        for x, d in zip((cases[i], prompts[i], evictions[i]), devs[i]):
            x.check(d)


def test_far_strides():
    """Rows whose offsets pass 2^31 elements, in prompts and in pools."""
    step = 2 ** 31 // 150 // 8 * 8 + 1024
    n, d = 170, 64
    base = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    c = Prompts(20, [n], q_heads=1, kv_heads=1, d=d)
    dev = c.upload()
    for i, name in enumerate(("q", "k", "v", "out")):
        far = base.as_strided((n, 1, d), (step, d, 1), 128 * i)
        far.copy_(dev[name])
        dev[name] = far
    dev["p"] = B.PromptAttention.of(dev["q"], dev["k"], dev["v"], dev["out"], dev["first"], c.scale)
    c.run(dev)
    c.check(dev)

    s = Steps(21, [160, 90], q_heads=2, kv_heads=1, d=d, page=1)
    dev = s.upload()
    pages = s.k.size(0)
    far_step = 2 ** 31 // (pages - 20) // 8 * 8 + 1024
    assert pages * far_step <= base.numel()
    for i, name in enumerate(("k", "v")):
        far = base.as_strided(s.k.shape, (far_step, d, d, 1), 128 * i)
        far.copy_(dev[name])
        dev[name] = far
    dev["cache"] = B.Pages.of(dev["k"], dev["v"], dev["table"])
    s.run(dev)
    s.check(dev)

    e = Evictions(22, [160, 90], kv_heads=1, d=d, budget=40, page=1)
    ed = e.upload()
    for i, name in enumerate(("k", "v")):
        far = base.as_strided(e.k.shape, (far_step, d, d, 1), 128 * i)
        far.copy_(ed[name])
        ed[name] = far
    ed["cache"] = B.Pages.of(ed["k"], ed["v"], ed["table"])
    ed["p"] = B.PagedEviction.of(ed["scores"], ed["pos"], ed["scores"], ed["pos"], ed["cache"], budget=40)
    e.run(ed)
    e.check(ed)

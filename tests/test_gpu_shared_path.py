"""Rotation, eviction, the paged cache and the attention behind shared prefixes together, as a program uses them; calls
captured into graphs, on two streams, with far strides."""
import numpy as np
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests import shared_cases as S
from tests.shared_cases import Batch

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_prompt_is_evicted_and_continued(dtype):
    """A prompt's queries and keys are turned, its cache is evicted, and three sequences continue it for some steps, each
    with its own tokens: append, then attend over the compact cache and the tail.  What is compared in each step is the
    attention of the rows that the caches hold, against 64 bits; the caches' rows against the turned keys."""
    n, hq, hkv, d, budget, batch, page, steps = 700, 8, 2, 64, 96, 3, 4, 9
    q, k, v = (S.gaussian(s, 1, h, n, d, dtype=dtype) for s, h in ((1, hq), (2, hkv), (3, hkv)))
    freq, _ = B.rotary_tables(d)
    pos = torch.arange(n, dtype=torch.int32).reshape(1, 1, n)
    dq, dk, dv = q.cuda(), k.cuda(), v.cuda()
    p = B.Rotary.of(dq, dk, dq, dk)
    B.aha_rotate(p, dq, dk, freq, None, pos.cuda(), dq, dk)                     # in place
    ang = S.angles(pos, freq.cpu(), None)
    S.assert_within(dk, *S.rotated(k, ang, d, False, 0), "the prompt's keys")

    params = B.Params(batch=1, n_q_heads=hq, n_kv_heads=hkv, head_dim=d, seq_len=n, window=16, budget=budget, recent=16,
                      dtype=B.AHA_BF16 if dtype == torch.bfloat16 else B.AHA_F32).with_strides(dq, dk, dv)
    ws = B.alloc_workspace(params)
    scores, idx = torch.empty(1, hkv, n, device="cuda"), torch.empty(1, hkv, budget, dtype=torch.int32, device="cuda")
    c = B.CompactCache.empty(params)
    B.aha_prefill_scores(params, dq, dk, dv, scores, ws)
    B.aha_select_topk(params, scores, idx, ws)
    B.aha_compact_kv(params, dk, dv, scores, idx, c.k, c.v, c.scores, c.pos, c.free_slot)
    torch.cuda.synchronize()
    for h in range(hkv):
        at = idx[0, h].long()
        assert torch.equal(c.k[0, h, :budget], dk[0, h, at]) and torch.equal(c.v[0, h, :budget], dv[0, h, at])

    width = -(-steps // page)
    b = Batch(7, q_heads=hq, kv_heads=hkv, d=d, q_len=1, tail=[0] * batch, prefix=[budget], page=page, cap=budget + 1, dtype=dtype)
    b.kp, b.vp = c.k.cpu(), c.v.cpu()
    b.table = torch.from_numpy(np.random.default_rng(1).permutation(batch * width).reshape(batch, width).astype(np.int32))
    b.kt, b.vt = (torch.zeros(batch * width, hkv, page, d, dtype=dtype) for _ in range(2))
    dev = b.upload()
    dev["kp"], dev["vp"] = c.k, c.v
    dev["p"] = B.SharedAttention.of(dev["q"], dev["out"], c.k, c.v, b.scale)
    for step in range(steps):
        new = [S.gaussian(100 + 3 * step + i, batch, h, 1, d, dtype=dtype) for i, h in ((0, hq), (1, hkv), (2, hkv))]
        nq, nk, nv = (t.cuda() for t in new)
        at = torch.full((1, batch, 1), n + step, dtype=torch.int32)
        dev["tail"].add_(1)
        rot = B.Rotary.of(nq, nk, dev["q"], v=nv)
        B.aha_append_paged(rot, dev["cache"], nq, nk, nv, freq, None, at.cuda(), dev["table"], dev["tail"], None, dev["q"],
                           dev["kt"], dev["vt"])
        b.run(dev)
        torch.cuda.synchronize()
        ang = S.angles(at, freq.cpu(), None)
        S.assert_within(dev["q"], *S.rotated(new[0], ang, d, False, 0), "turned queries")
        want, tol = S.rotated(new[1], ang, d, False, 0)
        for i in range(batch):
            pg, r = int(b.table[i, step // page]), step % page
            S.assert_within(dev["kt"][pg, :, r], want[i, :, 0], tol[i, :, 0], "appended keys")
            assert torch.equal(dev["vt"][pg, :, r].cpu(), new[2][i, :, 0])
        b.q, b.kt, b.vt, b.tail = dev["q"].cpu(), dev["kt"].cpu(), dev["vt"].cpu(), [step + 1] * batch
        b.compare(dev)


@pytest.mark.parametrize("q_len,rows", [(1, 4), (40, 4)])
def test_captured_steps_follow_the_lengths(q_len, rows):
    """One generation step captured into a graph, append and attention; replayed with other lengths, tables and rows, with
    eager calls of other shapes in the same workspace and synchronizations between the replays: bit by bit the
    eager call's results each time.  (Small tiles, and large ones.)"""
    d, page, batch = 128, 16, 5
    tails = [[q_len + 3 + 7 * i for i in range(batch)], [q_len] * batch, [q_len + 60 - 9 * i for i in range(batch)]]
    b = Batch(31, q_heads=2 * rows, kv_heads=2, d=d, q_len=q_len, tail=tails[0], new=[q_len] * batch, prefix=[500, 300],
              first=[0, 3, 5], page=page, cap=520)
    width = -(-(q_len + 70) // page)
    b.table = torch.arange(batch * width, dtype=torch.int32).reshape(batch, width)
    b.kt, b.vt = (S.gaussian(s, batch * width, 2, page, d, dtype=b.dtype) for s in (41, 42))
    b.kp, b.vp = (S.gaussian(s, 2, 2, 520, d, dtype=b.dtype) for s in (43, 44))
    dev = b.upload()
    freq, _ = B.rotary_tables(d)
    new = [S.gaussian(51 + i, batch, h, q_len, d, dtype=b.dtype).cuda() for i, h in ((0, 2 * rows), (1, 2), (2, 2))]
    pos = torch.zeros(1, batch, q_len, dtype=torch.int32, device="cuda")
    rot = B.Rotary.of(new[0], new[1], dev["q"], v=new[2])
    def step():
        B.aha_append_paged(rot, dev["cache"], *new, freq, None, pos, dev["table"], dev["tail"], dev["new"], dev["q"], dev["kt"], dev["vt"])
        b.run(dev)
    step()
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        step()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            step()
    torch.cuda.synchronize()
    small = Batch(32, q_heads=4, kv_heads=2, d=64, q_len=1, tail=[20, 3], prefix=[77], page=8)
    other = small.upload()
    pools = dev["kt"].clone(), dev["vt"].clone()
    for i in range(7):
        dev["tail"].copy_(i32(tails[i % 3]))
        dev["new"].copy_(i32([q_len - (i * j) % (q_len + 1) for j in range(batch)]))
        dev["prefix"].copy_(i32([500 - 70 * i, 41 * i]))
        dev["first"].copy_(i32([0, i % 4, 4]))
        pos.fill_(1000 * i)
        for t in new:
            t.mul_(0.9)
        got = []
        for way in (graph.replay, step):
            dev["kt"].copy_(pools[0])
            dev["vt"].copy_(pools[1])
            for t in (dev["q"], dev["out"], dev["lse"]):
                t.fill_(7.0)
            other["out"].fill_(float("nan"))
            if other["ws"].numel() <= dev["ws"].numel():
                other["ws"] = dev["ws"][:other["ws"].numel()]
            small.run(other)
            way()
            torch.cuda.synchronize()
            got.append([dev[x].clone() for x in ("q", "kt", "vt", "out", "lse")])
        for x, y in zip(*got):
            assert torch.equal(x, y)
        assert not torch.isnan(got[0][3].float()).any()
    small.check(other)


def test_two_streams_with_a_workspace_each():
    batches = [Batch(61 + i, q_heads=8, kv_heads=2, d=128, q_len=1 + 39 * i, tail=[150, 90, 64], prefix=[900], page=16) for i in range(2)]
    devs, streams = [b.upload() for b in batches], [torch.cuda.Stream() for _ in batches]
    torch.cuda.synchronize()
    for _ in range(5):
        for b, dev, stream in zip(batches, devs, streams):
            with torch.cuda.stream(stream):
                b.run(dev)
    torch.cuda.synchronize()
    for b, dev in zip(batches, devs):
        b.compare(dev)


@pytest.mark.parametrize("q_len", [1, 70])
def test_results_do_not_change(q_len):
    b = Batch(71, q_heads=8, kv_heads=2, d=128, q_len=q_len, tail=[300, 99], prefix=[1200], page=32)
    dev = b.upload()
    b.run(dev)
    first = dev["out"].clone(), dev["lse"].clone()
    for poison in (0x00, 0xff, 0x7f):
        dev["ws"].fill_(poison)
        b.run(dev)
        torch.cuda.synchronize()
        assert torch.equal(dev["out"], first[0]) and torch.equal(dev["lse"], first[1])


def far(t, axis, stride):
    """A copy of t on the GPU whose `axis` has the given stride, and a view of it; the memory between is not touched."""
    strides = list(torch.empty(t.shape, device="meta").stride())
    strides[axis] = stride
    memory = torch.empty((t.size(axis) - 1) * stride + t.numel(), dtype=t.dtype, device="cuda")
    view = memory.as_strided(t.shape, strides)
    view.copy_(t)
    return view


@pytest.mark.parametrize("q_len", [1, 80])
@pytest.mark.parametrize("where", ["tokens", "pages", "heads"])
def test_offsets_beyond_32_bits(q_len, where):
    """Prefix tokens, pages and heads so far apart that offsets in bytes and in elements pass 2^32."""
    b = Batch(81, q_heads=4, kv_heads=2, d=64, q_len=q_len, tail=[q_len + 10, q_len + 25], prefix=[41], page=8)
    b.kt, b.vt, b.kp, b.vp = (torch.nan_to_num(t) for t in (b.kt, b.vt, b.kp, b.vp))
    dev = b.upload()
    if where == "tokens":
        dev["kp"], dev["vp"] = (far(t, 2, 1 << 27) for t in (b.kp, b.vp))
    elif where == "heads":
        dev["kp"], dev["vp"] = (far(t, 1, (1 << 32) + 64) for t in (b.kp, b.vp))
        dev["kt"], dev["vt"] = (far(t, 1, (1 << 32) + 64) for t in (b.kt, b.vt))
    else:
        dev["kt"], dev["vt"] = (far(t, 0, (1 << 32) // b.kt.size(0) // 8 * 8 + 512) for t in (b.kt, b.vt))
    dev["cache"] = B.Pages.of(dev["kt"], dev["vt"], dev["table"])
    dev["p"] = B.SharedAttention.of(dev["q"], dev["out"], dev["kp"], dev["vp"], b.scale)
    b.run(dev)
    b.check(dev)
    # what appending writes there
    nk = S.gaussian(82, 2, 2, 3, 64, dtype=b.dtype)
    nv = S.gaussian(83, 2, 2, 3, 64, dtype=b.dtype)
    before = dev["kt"].cpu(), dev["vt"].cpu()
    freq, _ = B.rotary_tables(0)
    pos = torch.zeros(1, 2, 3, dtype=torch.int32, device="cuda")
    B.aha_append_paged(B.Rotary.of(None, nk.cuda(), v=nv.cuda(), rot_dim=0), dev["cache"], None, nk.cuda(), nv.cuda(), freq, None, pos,
                       dev["table"], dev["tail"], None, None, dev["kt"], dev["vt"])
    torch.cuda.synchronize()
    for got, was, rows in zip((dev["kt"], dev["vt"]), before, (nk, nv)):
        for i in range(2):
            for t in range(3):
                s = b.tail[i] - 3 + t
                was[int(b.table[i, s // 8]), :, s % 8] = rows[i, :, t]
        assert torch.equal(got.cpu(), was)


def test_rotation_of_rows_beyond_32_bits():
    x = S.gaussian(91, 1, 2, 33, 64, dtype=torch.bfloat16)
    freq, _ = B.rotary_tables(64)
    pos = torch.arange(33, dtype=torch.int32).reshape(1, 1, 33)
    for axis, stride in ((1, (1 << 32) + 64), (2, 1 << 28)):
        view = far(x, axis, stride)
        p = B.Rotary.of(view, None, view)
        B.aha_rotate(p, view, None, freq, None, pos.cuda(), view, None)
        S.assert_within(view, *S.rotated(x, S.angles(pos, freq.cpu(), None), 64, False, 0), "turned in place")
        del view

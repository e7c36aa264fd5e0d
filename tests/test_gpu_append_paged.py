"""Appending to the paged cache with the rotation on the way (aha_append_paged): every row of the pools and of the
turned queries, those that stay as they were among them."""
import numpy as np
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests import shared_cases as S

pytestmark = pytest.mark.gpu


def check(seed, tail, new, *, tokens, hq=4, hkv=2, d=64, page=8, dtype=torch.bfloat16, rot=None, pairing=B.AHA_PAIR_HALVES,
          pool_layout="phrd", table=None, width=None, with_q=True, start=0):
    batch, rot = len(tail), d if rot is None else rot
    print("append", tail, new, tokens, hq, hkv, d, page, dtype, rot, pairing, pool_layout, flush=True)
    width = len(table[0]) if table is not None else width or max(1, -(-max(list(tail) + [1]) // page))
    pages = batch * width + 1
    if table is None:
        table = np.random.default_rng(seed).permutation(pages)[:batch * width].reshape(batch, width)
    table = torch.as_tensor(np.asarray(table), dtype=torch.int32)
    q, k, v = (S.gaussian(seed + i, batch, h, tokens, d, dtype=dtype) for i, h in ((1, hq), (2, hkv), (3, hkv)))
    shape = (pages, hkv, page, d) if pool_layout == "phrd" else (pages, page, hkv, d)
    pools = [S.gaussian(seed + i, *shape, dtype=dtype) for i in (4, 5)]
    dp = [t.cuda() for t in pools]
    if pool_layout != "phrd":
        pools, dp = ([t.transpose(1, 2) for t in x] for x in (pools, dp))
    pos = torch.from_numpy((start + np.arange(tokens)[None, None] + 3 * np.arange(batch)[None, :, None]).astype(np.int32))
    inv_freq, _ = B.rotary_tables(rot, device="cpu")
    dq, dk, dv, dt = q.cuda(), k.cuda(), v.cuda(), table.cuda()
    q_out = torch.full_like(dq, 7.0) if with_q else None
    lens = [None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda") for x in (tail, new)]
    p = B.Rotary.of(dq if with_q else None, dk, q_out, v=dv, rot_dim=rot, pairing=pairing)
    cache = B.Pages.of(dp[0], dp[1], dt)
    B.aha_append_paged(p, cache, dq if with_q else None, dk, dv, inv_freq.cuda(), None, pos.cuda(), dt, lens[0], lens[1],
                       q_out, dp[0], dp[1])
    torch.cuda.synchronize()
    ang = S.angles(pos, inv_freq, None)
    (wq, tq), (wk, tk) = (S.rotated(x, ang, rot, pairing == B.AHA_PAIR_NEIGHBOURS, 0) for x in (q, k))
    kp, kt, vp = pools[0].double().numpy().copy(), np.zeros(pools[0].shape), pools[1].double().numpy().copy()
    real = np.zeros((batch, tokens), bool)
    for b in range(batch):
        fresh = tokens if new is None else min(max(new[b], 0), tokens)
        real[b, :fresh] = True
        for t in range(fresh):
            s = tail[b] - fresh + t
            if s < 0 or s // page >= width or not 0 <= int(table[b, s // page]) < pages:
                continue
            at = (int(table[b, s // page]), slice(None), s % page)
            kp[at], kt[at], vp[at] = wk[b, :, t], tk[b, :, t], v[b, :, t].double().numpy()
    S.assert_within(dp[0], kp, kt, "keys")
    S.assert_within(dp[1], vp, np.zeros_like(vp), "values")
    if with_q:
        keep = real[:, None, :, None]
        S.assert_within(q_out, np.where(keep, wq, 7.0), np.where(keep, tq, 0.0), "queries")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pool_layout", ["phrd", "prhd"])
def test_append(dtype, pool_layout):
    check(1, [1, 9, 40], None, tokens=1, dtype=dtype, pool_layout=pool_layout)
    check(2, [13, 30, 5], [13, 7, 0], tokens=13, d=128, dtype=dtype, pool_layout=pool_layout)
    check(3, [70], None, tokens=70, hq=3, hkv=3, page=16, rot=32, pairing=B.AHA_PAIR_NEIGHBOURS, dtype=dtype,
          pool_layout=pool_layout)
    check(4, [6, 2], [2, 2], tokens=4, page=1, rot=0, dtype=dtype, pool_layout=pool_layout)
    check(5, [600, 1, 333], [300, 1, 77], tokens=300, hkv=1, page=64, d=128, start=100000, dtype=dtype, pool_layout=pool_layout)


def test_without_queries():
    check(6, [11, 12], None, tokens=3, with_q=False)


def test_places_that_are_not_there():
    """Tokens before 0, behind the table, and in holes of the table: dropped, nothing else is touched."""
    check(7, [2, 3], None, tokens=5, page=4, width=1)                               # the first ones before 0
    check(8, [9, 20], None, tokens=6, page=4, width=2)                              # the last ones behind 8 slots
    check(9, [8, 8], None, tokens=8, page=4, table=[[-1, 3], [1, 99]])              # -1 and 99: no pages
    check(10, [8, 2 ** 31 - 1], None, tokens=8, page=4, table=[[-2 ** 31, 2 ** 31 - 1], [0, 1]])
    check(11, [-5, -2 ** 31 + 8], [3, 99], tokens=8, page=4, width=2)               # new_len clamped, tails below 0

"""Attention of single tokens over paged caches with running scores (aha_paged_attention) against 64 bits."""
import numpy as np
import pytest
import torch

from tests.paged_cases import NAN, Steps

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
HEADS = pytest.mark.parametrize("d", [64, 128])


@BOTH
@HEADS
def test_lengths(dtype, d):
    Steps(1, [1], q_heads=1, kv_heads=1, d=d, dtype=dtype).check()
    Steps(2, [1, 2, 31, 32, 33, 64, 127, 128, 129, 300], q_heads=4, kv_heads=2, d=d, dtype=dtype).check()
    Steps(3, [1000, 5, 2500], q_heads=8, kv_heads=2, d=d, dtype=dtype, page=64, layout="prhd").check()


@BOTH
@pytest.mark.parametrize("page", [1, 2, 8, 32, 64, 256, 1024])
def test_pages(dtype, page):
    Steps(4, [page, 3 * page - 1, 2 * page + 1, 190], q_heads=4, kv_heads=2, d=64, page=page, dtype=dtype).check()


@BOTH
@pytest.mark.parametrize("group", [1, 2, 3, 5, 8, 16, 31, 32, 33, 40, 70])
def test_groups(dtype, group):
    Steps(5, [100, 260], q_heads=2 * group, kv_heads=2, d=64, dtype=dtype).check()


@BOTH
def test_rows_without_keys(dtype):
    """Nothing cached, lengths below 0, all pages given back."""
    d = Steps(6, [0, -5, 33, 40], q_heads=4, kv_heads=2, d=64, dtype=dtype, holes={(3, 0): -1, (3, 1): 10 ** 6, (3, 2): -9}).check()
    assert not d["out"][0].any() and torch.isneginf(d["lse"][3]).all()


@BOTH
def test_holes(dtype):
    for page in (4, 16, 32, 64):
        holes = {(0, 0): -1, (0, 2): 10 ** 6, (1, 1): -7, (2, 2): -1}  # (the newest token of the last one is dropped)
        Steps(7, [3 * page, 2 * page + 1, 3 * page - 1], q_heads=4, kv_heads=2, d=128, page=page, dtype=dtype, holes=holes).check()


@BOTH
@HEADS
def test_caches_in_parts(dtype, d):
    """Tables of many places, which are divided, for sequences of all lengths, most of whose parts have no key."""
    holes = {(4, 0): -1, (4, 9): 10 ** 6, (5, 62): -1, (6, 0): -1}  # (the newest token of the next to last one is dropped; the last one has nothing)
    Steps(30, [0, 1, 129, -3, 700, 1000, 16, 1600], q_heads=4, kv_heads=2, d=d, dtype=dtype, width=100, holes=holes).check()
    Steps(31, [1600, 513, 10 ** 9], q_heads=10, kv_heads=2, d=d, dtype=dtype, width=100, slots=1333, slot_pad=7, seen=[5000, 513, 70]).check()
    Steps(32, [1200, 77], q_heads=6, kv_heads=2, d=d, dtype=dtype, width=100, with_scores=False).check()
    Steps(33, [1200, 77], q_heads=6, kv_heads=2, d=d, dtype=dtype, width=100, with_pos=False, adaptive=False, fixed=0.2).check()
    Steps(34, [1500, 300], q_heads=70, kv_heads=2, d=d, dtype=dtype, width=100, hot=4.0).check()


@BOTH
def test_scales_of_the_scores(dtype):
    for seen in ([500, 500], [50, 10 ** 9], [1, 0], [-3, 65]):
        Steps(8, [200, 64], q_heads=4, kv_heads=2, d=64, dtype=dtype, budget=64, seen=seen).check()
    Steps(9, [200, 64], q_heads=4, kv_heads=2, d=128, dtype=dtype, budget=3, floor=0.0, seen=[3, 900]).check()
    Steps(10, [200, 64], q_heads=4, kv_heads=2, d=128, dtype=dtype, adaptive=False, fixed=0.05).check()
    Steps(11, [200, 64], q_heads=4, kv_heads=2, d=128, dtype=dtype, adaptive=False, fixed=0.0, scale=0.0).check()
    Steps(12, [700], q_heads=4, kv_heads=2, d=128, dtype=dtype, hot=6.0, budget=8).check()


@BOTH
def test_without_scores_or_positions(dtype):
    Steps(13, [300, 7], q_heads=4, kv_heads=2, d=64, dtype=dtype, with_scores=False).check()
    Steps(14, [300, 7], q_heads=4, kv_heads=2, d=64, dtype=dtype, with_pos=False).check()
    c = Steps(15, [300, 7], q_heads=4, kv_heads=2, d=64, dtype=dtype)
    d = c.upload()
    c.run(d, lse=False)
    torch.cuda.synchronize()
    assert torch.isnan(d["lse"]).all()


@BOTH
def test_lengths_beyond_what_is_there_are_clamped(dtype):
    Steps(16, [10 ** 9, 70], q_heads=4, kv_heads=2, d=64, dtype=dtype, width=5, page=16).check()
    Steps(17, [75, 2 ** 31 - 1], q_heads=4, kv_heads=2, d=64, dtype=dtype, width=5, page=16, slots=75).check()


@BOTH
def test_strides_of_scores(dtype):
    Steps(18, [80, 77], q_heads=4, kv_heads=2, d=64, dtype=dtype, slot_pad=3).check()


def test_the_newest_token_starts_from_nothing():
    c = Steps(19, [90, 33], q_heads=4, kv_heads=2, d=64)
    c.scores[0, :, 89] = NAN
    c.scores[1, :, 32] = float("inf")
    c.check()


@BOTH
@pytest.mark.parametrize("width", [None, 100])
def test_keys_and_values_that_are_not_finite(dtype, width):
    """They reach their own sequence and KV head alone."""
    c = Steps(20, [300, 200], q_heads=4, kv_heads=2, d=64, dtype=dtype, width=width)
    d = c.upload()
    c.run(d)
    torch.cuda.synchronize()
    out, scores = d["out"].clone(), d["scores"].clone()
    d["scores"].copy_(c.scores)
    d["k"][int(c.table[0, 3]), 1, 5] = NAN
    c.run(d)
    torch.cuda.synchronize()
    assert torch.equal(d["out"][1], out[1]) and torch.equal(d["out"][0, :2], out[0, :2])
    assert torch.equal(d["scores"][1], scores[1]) and torch.equal(d["scores"][0, 0], scores[0, 0])
    assert torch.isnan(d["out"][0, 2:].float()).all() and torch.isnan(d["scores"][0, 1, :300]).all()


@BOTH
@pytest.mark.parametrize("batch", [1, 3, 40, 150])
def test_batches(dtype, batch):
    """From many parts of few sequences' keys to one part of each of many."""
    rng = np.random.default_rng(batch)
    tail = rng.integers(1, 700 if batch < 100 else 200, batch).tolist()
    Steps(21, tail, q_heads=8, kv_heads=4, d=64, dtype=dtype, page=32, seen=(np.array(tail) * 3).tolist(), budget=100).check()


def test_a_long_cache():
    Steps(22, [20000], q_heads=4, kv_heads=1, d=128, page=64, budget=500).check()


@BOTH
def test_same_result_every_time(dtype):
    c = Steps(23, [3000, 100], q_heads=8, kv_heads=2, d=128, page=64, dtype=dtype)
    d = c.upload()
    c.run(d)
    first = [d[x].clone() for x in ("out", "lse", "scores")]
    for _ in range(3):
        d["scores"].copy_(c.scores)
        c.run(d)
        assert all(torch.equal(d[x], y) for x, y in zip(("out", "lse", "scores"), first))

"""Eviction from paged caches (aha_paged_evict) against a sort."""
import numpy as np
import pytest
import torch

from tests.paged_cases import NAN, Evictions

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
PLACE = pytest.mark.parametrize("in_place", [True, False])


def pos_of(batch, heads, slots, step=1):
    return (step * torch.arange(slots, dtype=torch.int32)).expand(batch, heads, slots).contiguous()


@BOTH
@PLACE
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(dtype, in_place, d):
    Evictions(1, [1, 2, 33, 64, 65, 200, 0], kv_heads=2, d=d, dtype=dtype, budget=32, in_place=in_place).check()
    Evictions(2, [500, 1300], kv_heads=3, d=d, dtype=dtype, budget=100, recent=20, sink=4, page=64, layout="prhd", in_place=in_place,
              pos=pos_of(2, 3, 21 * 64), seen=[500, 1300]).check()


@PLACE
@pytest.mark.parametrize("budget", [1, 2, 100, 998, 999, 1000, 1001, 5000])
def test_budgets(in_place, budget):
    Evictions(3, [1000, 999, 17], kv_heads=2, d=64, budget=budget, in_place=in_place).check()


@pytest.mark.parametrize("recent, sink", [(0, 0), (64, 0), (0, 64), (40, 24), (1, 1)])
def test_protected_tokens(recent, sink):
    c = Evictions(4, [400, 64, 65], kv_heads=2, d=64, budget=64, recent=recent, sink=sink, pos=pos_of(3, 2, 400), page=16)
    d = c.check()
    left = d["pos_out"][0, 0, :64].tolist()
    assert set(range(sink)) <= set(left) and set(range(400 - recent, 400)) <= set(left) and len(set(left)) == 64


@PLACE
def test_a_prompts_scores(in_place):
    """Without positions: token j has position j."""
    Evictions(5, [700, 20, 300], kv_heads=2, d=128, budget=90, recent=16, sink=2, with_pos=False, in_place=in_place, page=32).check()


@pytest.mark.parametrize("page", [1, 8, 128, 1024])
def test_pages(page):
    Evictions(6, [3 * page, 2 * page + 1, 150], kv_heads=2, d=64, budget=40, page=page).check()


def test_equal_scores():
    """The highest position goes first, of equal positions the last place."""
    for values in (1, 2, 5):
        rng = np.random.default_rng(values)
        scores = torch.from_numpy(rng.integers(0, values, (2, 2, 640)).astype(np.float32))
        pos = torch.from_numpy(rng.permuted(np.tile(np.arange(640), (2, 2, 1)), axis=2).astype(np.int32))
        Evictions(7, [640, 333], kv_heads=2, d=64, budget=100, scores=scores, pos=pos, seen=[640, 640], recent=10).check()
        few = torch.from_numpy(rng.integers(0, 3, (2, 2, 640)).astype(np.int32))
        Evictions(8, [640, 333], kv_heads=2, d=64, budget=100, scores=scores, pos=few, seen=[10 ** 6] * 2).check()
        # everything is protected: the rule among them still holds
        Evictions(9, [640, 333], kv_heads=2, d=64, budget=100, scores=scores, pos=few, recent=100, seen=[3, 3]).check()


def test_any_scores():
    """Negative ones, zeros of both signs, infinities, NaN of both signs, subnormals; positions of any size."""
    rng = np.random.default_rng(3)
    pick = np.array([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan, -np.nan, 1e-45, -1e-45, 3e38, -3e38, 1.0000001], np.float32)
    scores = torch.from_numpy(rng.choice(pick, (2, 3, 400)))
    pos = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (2, 3, 400)).astype(np.int32))
    for budget in (1, 7, 100, 250, 390):
        Evictions(10, [400, 399], kv_heads=3, d=64, budget=budget, scores=scores, pos=pos, seen=[2 ** 31 - 1, -2 ** 31], recent=1).check()


def test_sequences_with_holes_keep_their_tokens():
    holes = {(0, 1): -1, (2, 3): 10 ** 6, (3, 9): -1}  # (the last one lies behind the sequence's tokens)
    Evictions(11, [100, 100, 64, 100], kv_heads=2, d=64, budget=30, holes=holes, width=10).check()
    Evictions(12, [100, 100, 64, 100], kv_heads=2, d=64, budget=30, holes=holes, width=10, in_place=False).check()


def test_lengths_beyond_what_is_there_are_clamped():
    Evictions(13, [10 ** 9, -4, 2 ** 31 - 1], kv_heads=2, d=64, budget=30, width=6).check()
    Evictions(14, [10 ** 9, -4, 50], kv_heads=2, d=64, budget=30, width=6, slots=77, slot_pad=3).check()


def test_one_token_of_many_heads():
    """What a generation step takes away."""
    Evictions(15, [513] * 5 + [512, 511], kv_heads=4, d=128, budget=512, recent=32, page=64, pos=pos_of(7, 4, 9 * 64, 3),
              seen=[3 * 513] * 7).check()


@pytest.mark.parametrize("n", [4096, 20000, 33000, 70000])
def test_long_prompts(n):
    Evictions(16, [n, n // 2], kv_heads=1, d=64, budget=1000, recent=64, with_pos=False, in_place=False, page=64).check()
    scores = torch.from_numpy(np.random.default_rng(n).integers(0, 50, (1, 2, n)).astype(np.float32))
    Evictions(17, [n], kv_heads=2, d=64, budget=n - 700, recent=64, scores=scores, pos=pos_of(1, 2, n), page=16, slots=n).check()


def test_few_long_sequences_among_many():
    """More (sequence, KV head) pairs than the moving launch has workgroups for all their moves."""
    from paper_2506_03762_amd import binding as B
    small = Evictions(20, [640, 600, 300], kv_heads=2, d=64, budget=280)
    want, d = small.check(), small.upload()
    batch, at = 4200, [0, 2500, 4199]
    def wide(t, rest):
        return torch.full((batch, *t.shape[1:]), rest, dtype=t.dtype, device="cuda").index_copy_(0, torch.tensor(at, device="cuda"), t)
    table, scores, pos, tail = wide(d["table"], -1), wide(d["scores"], 1.0), wide(d["pos"], 5), wide(d["tail"], 0)
    lens, cache = torch.full_like(tail, -7), B.Pages.of(d["k"], d["v"], table)
    p = B.PagedEviction.of(scores, pos, scores, pos, cache, budget=280)
    B.aha_paged_evict(p, cache, scores, pos, d["k"], d["v"], table, tail, None, scores, pos, lens, B.alloc_evict_workspace(p, cache))
    assert torch.equal(lens, wide(want["len_out"], 0))
    assert torch.equal(scores, wide(want["scores_out"], 1.0)) and torch.equal(pos, wide(want["pos_out"], 5))
    for name in ("k", "v"):
        assert torch.equal(d[name].view(torch.uint8), want[name].view(torch.uint8)), name


@PLACE
def test_long_sequences_of_any_kind(in_place):
    """Ties, infinities, NaN, most tokens protected, pages that are not there, one token and nearly all that go."""
    n = 40000
    rng = np.random.default_rng(11)
    tied = torch.from_numpy(rng.choice(np.array([0.0, -0.0, 2.0, np.nan, np.inf, -1.0], np.float32), (1, 2, n)))
    pos = torch.from_numpy(rng.permuted(np.tile(np.arange(n), (1, 2, 1)), axis=2).astype(np.int32))
    for budget, recent in ((n - 1, 0), (n - 300, 20000), (5, 3), (12000, 12000)):
        Evictions(21, [n], kv_heads=2, d=64, budget=budget, recent=recent, scores=tied, pos=pos, page=64, slots=n, seen=[n + 5000], in_place=in_place).check()
    Evictions(22, [n], kv_heads=2, d=64, budget=15000, recent=15000, seen=[0], page=64, slots=n, in_place=in_place).check()
    Evictions(23, [n, 36000], kv_heads=1, d=64, budget=900, page=64, holes={(1, 300): -1}, in_place=in_place).check()


@pytest.mark.parametrize("n", [900, 3000, 9000, 40000])
def test_many_alike(n):
    """More of one score than are compared with each other; of one position too; more protected tokens than the budget."""
    rng = np.random.default_rng(n)
    shape = (1, 2, n)
    few = torch.from_numpy(rng.integers(0, 3, shape).astype(np.float32))
    some = torch.from_numpy(np.where(rng.random(shape) < 0.4, 0.5, rng.random(shape)).astype(np.float32))
    at = torch.from_numpy(rng.integers(0, n, shape).astype(np.int32))
    for scores, pos, budget in ((few, at, n // 2), (some, at, n // 3), (torch.zeros(shape), at, n - 500), (torch.zeros(shape), at // 100, 700),
                                (torch.zeros(shape), torch.zeros(shape, dtype=torch.int32), n // 2), (few, at % 2, n - 1)):
        Evictions(24, [n], kv_heads=2, d=64, budget=budget, scores=scores, pos=pos, page=64, slots=n, seen=[10 ** 6]).check()
    Evictions(25, [n], kv_heads=2, d=64, budget=n // 2, recent=n // 2, scores=some, pos=at % 5, page=64, slots=n, seen=[3]).check()


def test_shared_scores():
    """One row of scores for all heads, expanded, into outputs of their own."""
    base = torch.rand(2, 1, 160, generator=torch.Generator().manual_seed(1))
    c = Evictions(18, [150, 99], kv_heads=4, d=64, budget=40, scores=base.expand(2, 4, 160), in_place=False, with_pos=False)
    c.check()

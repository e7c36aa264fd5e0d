"""Eviction from paged caches where all unprotected tokens go and protected ones too, more of them alike than are compared with each
other (aha_paged_evict), against a sort."""
import numpy as np
import pytest
import torch

from tests.paged_cases import Evictions

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("n", [900, 3000, 9000, 40000])
def test_protected_tokens_go_behind_all_others(n, in_place):
    rng = np.random.default_rng(n)
    shape, last = (1, 2, n), 10 ** 6
    scores = torch.from_numpy(rng.random(shape).astype(np.float32))
    scores[torch.from_numpy(rng.random(shape) < 0.01)] = float("nan")
    free = rng.random(shape) < 0.1  # unprotected: positions of their own between the sink and the recent ones
    among = rng.permuted(np.tile(np.arange(100, 100 + n), (1, 2, 1)), axis=2)
    protected = (np.full(shape, last - 1),                                       # one position
                 rng.integers(last - 3, last, shape),                            # three
                 np.where(rng.random(shape) < 0.9, last - 2, rng.integers(last - 40, last, shape)),
                 np.where(rng.random(shape) < 0.5, 1, last - 1))                 # the sink's, too
    for i, at in enumerate(protected):
        pos = torch.from_numpy(np.where(free, among, at).astype(np.int32))
        for budget in (60, n // 3, n * 7 // 10):
            c = Evictions(30 + i, [n], kv_heads=2, d=64, budget=budget, recent=50, sink=3, scores=scores, pos=pos, page=64, slots=n, seen=[last],
                          in_place=in_place)
            unprotected = free.sum(2)[0]
            assert (n - budget > unprotected).all() and (unprotected > 0).all()
            c.check()

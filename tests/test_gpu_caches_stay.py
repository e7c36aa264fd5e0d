"""A generation step's attention over paged caches leaves keys and values as they were, in pages of heads and in pages of rows."""
import pytest
import torch

from tests.paged_cases import Steps

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["phrd", "prhd"])
@pytest.mark.parametrize("tail, width", [([33, 1, 0, 64], None), ([1900, 5, 777], None), ([300] * 40, 30)])
def test_keys_and_values_stay(dtype, layout, tail, width):
    c = Steps(1, tail, q_heads=8, kv_heads=2, d=128, dtype=dtype, layout=layout, width=width)
    d = c.upload()
    for _ in range(2):
        c.run(d)
    torch.cuda.synchronize()
    for name, was in (("k", c.k), ("v", c.v)):
        assert d[name].stride() == was.stride() and torch.equal(
            d[name].cpu().contiguous().view(torch.uint8), was.contiguous().view(torch.uint8)), name

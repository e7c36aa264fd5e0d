"""Scales of the attention behind shared prefixes that are refused, no GPU needed."""
import ctypes

import pytest

from paper_2506_03762_amd import binding as B
from tests.test_shared_host import BAD, attend, pages, shared


@pytest.mark.parametrize("scale,code", [(2.3e38, B.AHA_OK), (2.4e38, BAD), (3.4e38, BAD), (float("inf"), BAD), (float("nan"), BAD), (-1e-45, BAD),
                                        (0.0, B.AHA_OK), (-0.0, B.AHA_OK)])
def test_scales(scale, code):
    """Times log2(e), by which the kernels multiply, the largest fp32 numbers are infinite: every logit would be, or no number."""
    p, out = shared(scale=scale), ctypes.c_size_t()
    assert B.load().aha_shared_attention_workspace_bytes(ctypes.byref(p), None, ctypes.byref(out)) == code
    if code != B.AHA_OK:
        assert attend(p, pages()) == code

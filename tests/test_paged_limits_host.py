"""How large a problem the attention of single tokens over paged caches takes, no GPU needed: what the header says."""
import ctypes

import pytest

from paper_2506_03762_amd import binding as B
from tests.test_paged_host import attention, paged, pages, ref


def asked(p, pg):
    n = ctypes.c_size_t(0)
    return B.load().aha_paged_attention_workspace_bytes(ref(p), ref(pg), ctypes.byref(n)), n.value


@pytest.mark.parametrize("batch, kv_heads, group", [(64527, 1, 65), (21845, 3, 64), (31, 65, 1024), (2 ** 12, 1, 1024), (8191, 8, 33)])
@pytest.mark.parametrize("dtype", [B.AHA_F32, B.AHA_BF16])
def test_the_largest_problems(batch, kv_heads, group, dtype):
    """Caches of up to 2^20 places, divided into as many parts as a launch has workgroups for."""
    rc, n = asked(paged(batch=batch, n_q_heads=group * kv_heads, n_kv_heads=kv_heads, dtype=dtype, slots=0), pages(table_width=2 ** 16))
    assert rc == B.AHA_OK and n >= 40 * batch * kv_heads * group * (128 + 2 + 2) * 4


@pytest.mark.parametrize("change", [dict(n_q_heads=2 * 1025), dict(batch=2 ** 13, n_q_heads=8 * 65, n_kv_heads=1), dict(batch=32768)])
def test_what_is_larger_is_refused_by_both(change):
    assert asked(paged(**change), pages())[0] == B.AHA_ERR_UNSUPPORTED and attention(paged(**change), pages()) == B.AHA_ERR_UNSUPPORTED

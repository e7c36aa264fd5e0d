"""How large a problem the attention of packed prompts takes, no GPU needed: what the header says, and the size of the workspace says the
same as the call."""
import ctypes

import pytest

from paper_2506_03762_amd import binding as B
from tests.test_paged_host import PTR, prompt, prompt_attention, ref, two


def asked(p):
    n, rows = ctypes.c_size_t(7), ctypes.c_int32(0)
    rc = B.load().aha_prompt_attention_workspace_bytes(ref(p), ctypes.byref(n))
    assert B.load().aha_prompt_attention_tile_rows(ref(p), ctypes.byref(rows)) == rc
    return rc, n.value, rows.value


@pytest.mark.parametrize("change, rows", [
    (dict(tokens=2 ** 20, n_q_heads=512, n_kv_heads=8, head_dim=64, dtype=B.AHA_F32), (16, 32)),
    (dict(tokens=2 ** 21, sequences=65535, n_q_heads=128, n_kv_heads=8), (32, 128, 256)),
    (dict(tokens=65535, sequences=65535, n_q_heads=16384, n_kv_heads=1), (32, 128, 256)),
    (dict(tokens=65535, sequences=65535, n_q_heads=16384, n_kv_heads=16384, dtype=B.AHA_F32), (16, 32)),
    (dict(tokens=2 ** 30, sequences=1, n_q_heads=1, n_kv_heads=1, dtype=B.AHA_F32), (32,)),
    (dict(tokens=2 ** 30, sequences=1, n_q_heads=1, n_kv_heads=1), (32, 128, 256)),
    (dict(tokens=1, sequences=1, n_q_heads=2 ** 25, n_kv_heads=1), (32, 128, 256)),
    (dict(tokens=1, sequences=1, n_q_heads=2 ** 25, n_kv_heads=1, dtype=B.AHA_F32), (16, 32)),
])
def test_the_largest_problems(change, rows):
    rc, n, tile = asked(prompt(**change))
    assert rc == B.AHA_OK and n == 0 and tile in rows


@pytest.mark.parametrize("change", [
    dict(tokens=2 ** 30, n_q_heads=2, n_kv_heads=1), dict(tokens=1, n_q_heads=2 ** 25 + 1, n_kv_heads=1), dict(sequences=65536),
    dict(tokens=1, n_q_heads=65536, n_kv_heads=65536),
])
def test_what_is_larger_is_refused_by_both(change):
    p = prompt(q_stride=two(2 ** 34, 128), out_stride=two(2 ** 34, 128), **change)
    assert asked(p)[0] == B.AHA_ERR_UNSUPPORTED and prompt_attention(p, ws=PTR) == B.AHA_ERR_UNSUPPORTED

"""The tiles that the attention of packed prompts works in, asked of the library, no GPU needed."""
import ctypes

import pytest

from paper_2506_03762_amd import binding as B


def described(lens, q_heads, kv_heads, d, dtype=B.AHA_BF16, **kw):
    return B.aha_prompt(tokens=sum(lens), sequences=len(lens), n_q_heads=q_heads, n_kv_heads=kv_heads, head_dim=d, dtype=dtype, scale=0.1, **kw)


def tile_rows(lens, q_heads, kv_heads, d, dtype=B.AHA_BF16):
    rows = ctypes.c_int32(0)
    assert B.load().aha_prompt_attention_tile_rows(ctypes.byref(described(lens, q_heads, kv_heads, d, dtype)), ctypes.byref(rows)) == B.AHA_OK
    return rows.value


@pytest.mark.parametrize("lens, q_heads, kv_heads, d, dtype, rows", [
    ([512], 2, 1, 64, B.AHA_F32, 16), ([4096], 32, 8, 128, B.AHA_F32, 32), ([1], 1, 1, 64, B.AHA_F32, 16),
    ([2048], 8, 2, 128, B.AHA_BF16, 32), ([1], 1, 1, 128, B.AHA_BF16, 128), ([64] * 16, 8, 2, 128, B.AHA_BF16, 128), ([1024], 32, 8, 128, B.AHA_BF16, 128),
    ([16384], 32, 8, 128, B.AHA_BF16, 256), ([4096], 32, 8, 128, B.AHA_BF16, 256),
    # heads of 64 channels: long prompts alone do not make it 256
    ([3150], 192, 48, 64, B.AHA_BF16, 128), ([3150], 256, 64, 64, B.AHA_BF16, 256), ([9400], 62, 62, 64, B.AHA_BF16, 256),
    ([6300, 1, 3100], 62, 62, 64, B.AHA_BF16, 128),
])
def test_tiles(lens, q_heads, kv_heads, d, dtype, rows):
    assert tile_rows(lens, q_heads, kv_heads, d, dtype) == rows


def test_refusals():
    ask, rows = B.load().aha_prompt_attention_tile_rows, ctypes.c_int32(-7)
    assert ask(ctypes.byref(described([100], 4, 2, 64)), None) == B.AHA_ERR_INVALID_ARG
    assert ask(None, ctypes.byref(rows)) == B.AHA_ERR_INVALID_ARG
    for bad in (described([0], 4, 2, 64), described([100], 5, 2, 64), described([100], 4, 2, 64, reserved=1)):
        assert ask(ctypes.byref(bad), ctypes.byref(rows)) == B.AHA_ERR_INVALID_ARG
    assert ask(ctypes.byref(described([100], 4, 2, 96)), ctypes.byref(rows)) == B.AHA_ERR_UNSUPPORTED and rows.value == -7

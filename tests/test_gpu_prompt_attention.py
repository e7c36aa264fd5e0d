"""Causal attention of packed prompts (aha_prompt_attention) against 64 bits."""
import pytest
import torch

from tests.paged_cases import NAN, Prompts

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
HEADS = pytest.mark.parametrize("d", [64, 128])


@BOTH
@HEADS
def test_short_prompts(dtype, d):
    Prompts(1, [1], q_heads=1, kv_heads=1, d=d, dtype=dtype).check()
    Prompts(2, [1, 2, 31, 32, 33, 0, 64, 65], q_heads=4, kv_heads=2, d=d, dtype=dtype).check()
    Prompts(3, [127, 128, 129], q_heads=3, kv_heads=1, d=d, dtype=dtype, layout="htd").check()


@BOTH
@HEADS
@pytest.mark.parametrize("n", [255, 256, 257, 300, 511, 513, 777, 1025])
def test_lengths_around_tiles(dtype, d, n):
    Prompts(4, [n], q_heads=2, kv_heads=1, d=d, dtype=dtype).check()
    Prompts(5, [n, 3, n - 130], q_heads=2, kv_heads=2, d=d, dtype=dtype, gap=3).check()


@BOTH
def test_empty_prompts_and_rows_of_none(dtype):
    Prompts(6, [0, 0, 5, 0, 300, 0], q_heads=4, kv_heads=4, d=64, dtype=dtype, gap=70).check()
    d = Prompts(7, [0, 0], q_heads=2, kv_heads=1, d=128, dtype=dtype, gap=9).check()
    assert torch.isnan(d["out"].float()).all()


@BOTH
def test_grouped_heads(dtype):
    for q_heads, kv_heads in ((8, 1), (7, 1), (12, 4), (16, 16), (40, 8)):
        Prompts(8, [150, 40], q_heads=q_heads, kv_heads=kv_heads, d=64, dtype=dtype).check()


@pytest.mark.parametrize("count", [63, 64, 65, 255, 256, 257, 700])
def test_many_prompts(count):
    """Up to 64 prompts are taken by their length, more in their order, 256 to a look."""
    g = torch.Generator().manual_seed(count)
    lens = torch.randint(0, 40, (count,), generator=g).tolist()
    lens[count // 2] = 300
    Prompts(9, lens, q_heads=2, kv_heads=1, d=64).check()


@pytest.mark.parametrize("seed, lens, heads, kv_heads, more", [
    (50, [700, 65, 333, 1, 500, 31, 260, 449], 6, 2, dict(layout="htd", gap=3)), (51, [700, 65, 333, 1, 500, 31, 260, 449], 4, 4, dict(pad=8)),
    (52, [1300], 8, 2, dict(hot=5.0)), (53, [900, 800], 6, 2, dict(scale=1.5)), (54, [1500], 8, 4, dict(scale=0.0)), (55, [640, 641], 7, 1, {})])
def test_more_tiles_of_32_rows_than_compute_units(seed, lens, heads, kv_heads, more):
    """Their keys go by way of LDS."""
    Prompts(seed, lens, q_heads=heads, kv_heads=kv_heads, d=64, **more).check()


@pytest.mark.parametrize("d", [64, 128])
def test_fp32_problems_that_fill_the_chip(d):
    """Few rows go to tiles of 16, these to tiles of 32."""
    for seed, lens, group, more in ((40, [2049], 4, {}), (41, [1500, 1, 0, 2200], 3, dict(layout="htd", gap=5)), (42, [1900, 2100], 1, dict(hot=4.0, pad=4)),
                                    (43, [31, 33, 2500, 1800], 2, dict(scale=0.7))):
        heads = 36 // group * group
        Prompts(seed, lens, q_heads=heads, kv_heads=heads // group, d=d, dtype=torch.float32, heads=[0, group - 1, heads - 1], **more).check()


@BOTH
def test_scales_and_large_logits(dtype):
    Prompts(10, [200, 33], q_heads=2, kv_heads=1, d=128, dtype=dtype, scale=0.0).check()
    Prompts(11, [600], q_heads=2, kv_heads=1, d=128, dtype=dtype, hot=6.0).check()
    Prompts(12, [300], q_heads=2, kv_heads=2, d=64, dtype=dtype, scale=3.0).check()


@BOTH
def test_rising_logits(dtype):
    """Every key weighs more than those before it: references have to follow."""
    c = Prompts(13, [700], q_heads=2, kv_heads=1, d=64, dtype=dtype)
    c.q[:] = c.q[:1].abs()
    c.k[:] = (torch.arange(700).float() / 40)[:, None, None].to(dtype)
    c.check()


@BOTH
def test_strided_rows_without_lse(dtype):
    c = Prompts(14, [333, 20], q_heads=6, kv_heads=2, d=64, dtype=dtype, pad=64)
    d = c.upload()
    c.run(d, lse=False)
    torch.cuda.synchronize()
    assert torch.isnan(d["lse"]).all()
    c.run(d)
    c.check(d)


@BOTH
def test_keys_that_are_not_finite(dtype):
    """A key of NaN or infinity is what the rows that see it get, and nothing to those before it."""
    for bad in (NAN, float("inf")):
        c = Prompts(15, [290, 100], q_heads=2, kv_heads=1, d=64, dtype=dtype)
        d = c.upload()
        c.run(d)
        torch.cuda.synchronize()
        out, lse = d["out"].clone(), d["lse"].clone()
        d["k"][137] = bad
        c.run(d)
        torch.cuda.synchronize()
        assert torch.equal(d["out"][:137], out[:137]) and torch.equal(d["out"][290:], out[290:])
        assert torch.equal(d["lse"][:, :137], lse[:, :137]) and torch.equal(d["lse"][:, 290:], lse[:, 290:])
        if bad != bad:
            assert torch.isnan(d["out"][137:290].float()).all()


def test_prompts_that_reach_beyond_the_tokens_are_clamped():
    c = Prompts(16, [100, 57], q_heads=2, kv_heads=1, d=64)
    d = c.upload()
    d["first"].copy_(torch.tensor([-2 ** 31, 100, 2 ** 31 - 1], dtype=torch.int32))
    c.run(d)
    c.check(d)


@BOTH
def test_same_result_every_time(dtype):
    c = Prompts(17, [900, 300, 44], q_heads=4, kv_heads=2, d=128, dtype=dtype)
    d = c.upload()
    c.run(d)
    first = d["out"].clone()
    for _ in range(3):
        d["out"].fill_(NAN)
        c.run(d)
        assert torch.equal(d["out"], first)

"""Causal attention of packed prompts in tiles of 256 rows (bf16, long prompts that fill the chip several times) against 64 bits."""
import pytest
import torch

from tests.paged_cases import NAN, Prompts, i32

pytestmark = pytest.mark.gpu

HEADS = pytest.mark.parametrize("d", [64, 128])


def wide(seed, lens, d, *, group=4, kv_heads=None, **kw):
    """Prompts of more than 3100 tokens on average in more than 2400 tiles of 256 rows, of which some heads are compared."""
    average = -(-sum(lens) // len(lens))
    tiles = len(lens) * -(-(-(-average // 64) * group) // 4)
    kv_heads = kv_heads or -(-2400 // tiles)
    assert average > 3100 and tiles * kv_heads >= 2400
    q_heads = group * kv_heads
    return Prompts(seed, lens, q_heads=q_heads, kv_heads=kv_heads, d=d, heads=[0, group - 1, q_heads // 2 + 1, q_heads - 1], **kw)


@HEADS
@pytest.mark.parametrize("n", [3135, 3136, 3137, 3167, 3168, 3169, 3199, 3201, 3327, 3329])
def test_lengths_around_tiles(d, n):
    wide(1, [n], d).check()


@HEADS
def test_packed_prompts(d):
    wide(2, [6300, 33, 65, 6200], d).check()
    wide(3, [0, 6100, 3300], d, gap=70).check()
    wide(4, [5000, 3, 4400], d, layout="htd", gap=3).check()


@HEADS
@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 16])
def test_groups(d, group):
    wide(5, [6300, 1, 3100], d, group=group).check()


@HEADS
def test_scales_and_large_logits(d):
    wide(7, [3300], d, scale=0.0).check()
    wide(8, [3600], d, hot=6.0).check()
    wide(9, [3400], d, scale=3.0).check()


@HEADS
def test_rising_logits(d):
    """Every key weighs more than those before it: references have to follow."""
    c = wide(10, [3150], d)
    c.q[:] = c.q[:1].abs()
    c.k[:] = (torch.arange(3150).float() / 180)[:, None, None].to(c.dtype)
    c.check()


@HEADS
def test_strided_rows_without_lse(d):
    c = wide(11, [3333, 3200], d, pad=64)
    dev = c.upload()
    c.run(dev, lse=False)
    torch.cuda.synchronize()
    assert torch.isnan(dev["lse"]).all()
    c.run(dev)
    c.check(dev)


@HEADS
@pytest.mark.parametrize("bad", [NAN, float("inf")])
def test_keys_that_are_not_finite(d, bad):
    """A key of NaN or infinity is what the rows that see it get, and nothing to those before it or of other prompts."""
    c = wide(12, [3290, 3300], d)
    dev = c.upload()
    c.run(dev)
    torch.cuda.synchronize()
    out, lse = dev["out"].clone(), dev["lse"].clone()
    dev["k"][1137] = bad
    c.run(dev)
    torch.cuda.synchronize()
    for part in (slice(0, 1137), slice(3290, 6590)):
        assert torch.equal(dev["out"][part], out[part]) and torch.equal(dev["lse"][:, part], lse[:, part])
    if bad != bad:
        assert torch.isnan(dev["out"][1137:3290].float()).all()


@HEADS
def test_same_result_every_time(d):
    c = wide(13, [6900, 2700, 44], d)
    dev = c.upload()
    c.run(dev)
    first = dev["out"].clone()
    for _ in range(3):
        dev["out"].fill_(NAN)
        c.run(dev)
        assert torch.equal(dev["out"], first)


def test_captured_prompts_follow_their_lengths():
    c = wide(14, [3500, 3300], 128)
    d = c.upload()
    c.run(d)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            c.run(d)
    for first in ([0, 6800, 6800], [0, 1, 6800], [3, 3400, 6790], [0, 3500, 6800]):
        c.first, c.lens = first, [first[1] - first[0], first[2] - first[1]]
        d["first"].copy_(i32(first))
        d["out"].fill_(NAN)
        d["lse"].fill_(NAN)
        graph.replay()
        c.check(d)


def test_far_strides():
    """Rows whose offsets pass 2^31 elements."""
    n, d = 3150, 128
    c = wide(15, [n], d, group=1)
    step = 2 ** 31 // 3000 // 8 * 8 + 1024
    base = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    dev = c.upload()
    for i, name in enumerate(("q", "k", "v", "out")):
        far = base.as_strided((n, c.hq, d), (step, d, 1), c.hq * d * i)
        far.copy_(dev[name])
        dev[name] = far
    from paper_2506_03762_amd import binding as B
    dev["p"] = B.PromptAttention.of(dev["q"], dev["k"], dev["v"], dev["out"], dev["first"], c.scale)
    c.run(dev)
    c.check(dev)

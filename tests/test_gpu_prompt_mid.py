"""Causal attention of packed prompts in tiles of 128 rows (bf16, problems that fill a good part of the chip) against 64 bits."""
import pytest
import torch

from tests.paged_cases import NAN, Prompts, i32

pytestmark = pytest.mark.gpu

HEADS = pytest.mark.parametrize("d", [64, 128])


def mid(seed, lens, d, *, group=4, kv_heads=None, **kw):
    """A problem that fills a good part of the chip, of which some heads are compared."""
    kv_heads = kv_heads or (64 if d == 64 else 32) * 4 // group
    q_heads = group * kv_heads
    blocks = (sum(lens) + 31 * len(lens)) // 64
    assert blocks * q_heads // 4 >= (176 if d == 64 else 112), "a problem of small tiles"
    return Prompts(seed, lens, q_heads=q_heads, kv_heads=kv_heads, d=d, heads=[0, group - 1, q_heads // 2 + 1, q_heads - 1], **kw)


@HEADS
@pytest.mark.parametrize("n", [255, 256, 257, 287, 288, 319, 320, 321, 511, 513, 777, 1025])
def test_lengths_around_tiles(d, n):
    mid(1, [n], d).check()


@HEADS
def test_packed_prompts(d):
    mid(2, [1, 2, 31, 32, 33, 0, 63, 64, 65, 127, 128, 129, 300], d).check()
    mid(3, [0, 0, 500, 0, 1, 0], d, gap=70).check()
    mid(4, [400, 3, 270], d, layout="htd", gap=3).check()


@HEADS
@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 16])
def test_groups(d, group):
    mid(5, [450, 1, 200], d, group=group, kv_heads=-(-160 // group)).check()


@pytest.mark.parametrize("count", [63, 64, 65, 200])
def test_many_prompts(count):
    g = torch.Generator().manual_seed(count)
    lens = torch.randint(0, 60, (count,), generator=g).tolist()
    lens[count // 2] = 400
    mid(6, lens, 128).check()


@HEADS
def test_scales_and_large_logits(d):
    mid(7, [300, 33], d, scale=0.0).check()
    mid(8, [600], d, hot=6.0).check()
    mid(9, [400], d, scale=3.0).check()


@HEADS
def test_rising_logits(d):
    """Every key weighs more than those before it: references have to follow."""
    c = mid(10, [700], d)
    c.q[:] = c.q[:1].abs()
    c.k[:] = (torch.arange(700).float() / 40)[:, None, None].to(c.dtype)
    c.check()


@HEADS
def test_strided_rows_without_lse(d):
    c = mid(11, [333, 200], d, pad=64)
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
    c = mid(12, [290, 300], d)
    dev = c.upload()
    c.run(dev)
    torch.cuda.synchronize()
    out, lse = dev["out"].clone(), dev["lse"].clone()
    dev["k"][137] = bad
    c.run(dev)
    torch.cuda.synchronize()
    for part in (slice(0, 137), slice(290, 590)):
        assert torch.equal(dev["out"][part], out[part]) and torch.equal(dev["lse"][:, part], lse[:, part])
    if bad != bad:
        assert torch.isnan(dev["out"][137:290].float()).all()


@HEADS
def test_same_result_every_time(d):
    c = mid(13, [900, 300, 44], d)
    dev = c.upload()
    c.run(dev)
    first = dev["out"].clone()
    for _ in range(3):
        dev["out"].fill_(NAN)
        c.run(dev)
        assert torch.equal(dev["out"], first)


def test_captured_prompts_follow_their_lengths():
    c = mid(14, [500, 300], 128)
    d = c.upload()
    c.run(d)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            c.run(d)
    for first in ([0, 800, 800], [0, 1, 800], [3, 400, 790], [0, 500, 800]):
        c.first, c.lens = first, [first[1] - first[0], first[2] - first[1]]
        d["first"].copy_(i32(first))
        d["out"].fill_(NAN)
        d["lse"].fill_(NAN)
        graph.replay()
        c.check(d)


def test_far_strides():
    """Rows whose offsets pass 2^31 elements."""
    n, heads, d = 320, 96, 128
    step = 2 ** 31 // 300 // 8 * 8 + 1024
    base = torch.empty(n * step, dtype=torch.bfloat16, device="cuda")
    c = mid(15, [n], d, group=1, kv_heads=heads)
    dev = c.upload()
    for i, name in enumerate(("q", "k", "v", "out")):
        far = base.as_strided((n, heads, d), (step, d, 1), heads * d * i)
        far.copy_(dev[name])
        dev[name] = far
    from paper_2506_03762_amd import binding as B
    dev["p"] = B.PromptAttention.of(dev["q"], dev["k"], dev["v"], dev["out"], dev["first"], c.scale)
    c.run(dev)
    c.check(dev)

"""Causal attention of packed prompts in tiles of 256 rows, heads of 64 channels, against 64 bits: what makes the call take these
tiles is asked of the library, not estimated here."""
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests.paged_cases import NAN, Prompts, i32
from tests.test_prompt_tiles_host import tile_rows

pytestmark = pytest.mark.gpu


def wide(seed, lens, group, **kw):
    """Prompts that the library takes in tiles of 256 rows: of as few KV heads as that needs, some heads compared."""
    kv_heads = next(h for h in range(1, 600) if all(tile_rows(lens, group * (h + i), h + i, 64) == 256 for i in range(4)))
    q_heads = group * kv_heads
    return Prompts(seed, lens, q_heads=q_heads, kv_heads=kv_heads, d=64,
                   heads=sorted({0, group - 1, q_heads // 2 + 1, q_heads - 1}), **kw)


def check(c):
    d = c.upload()
    assert B.prompt_attention_tile_rows(d["p"]) == 256
    c.run(d)
    c.check(d)


@pytest.mark.parametrize("n", [3137, 3167, 3168, 3201])
def test_lengths_around_tiles(n):
    check(wide(1, [n], 4))


def test_packed_prompts():
    check(wide(2, [6300, 33, 65, 6200], 4))


@pytest.mark.parametrize("group, lens", [(1, [6300, 1, 6400]), (2, [4097, 4300])])
def test_small_groups(group, lens):
    check(wide(3, lens, group))


@pytest.mark.parametrize("group, n", [(1, 5000), (4, 3968)])
def test_rising_logits(group, n):
    """Every key weighs more than those before it: references have to follow."""
    c = wide(4, [n], group)
    c.q[:] = c.q[:1].abs()
    c.k[:] = (torch.arange(n).float() / 180)[:, None, None].to(c.dtype)
    check(c)


def test_same_result_every_time():
    c = wide(5, [6900, 2700, 44], 4)
    d = c.upload()
    assert B.prompt_attention_tile_rows(d["p"]) == 256
    c.run(d)
    first = d["out"].clone()
    for _ in range(3):
        d["out"].fill_(NAN)
        c.run(d)
        assert torch.equal(d["out"], first)


def test_captured_prompts_follow_their_lengths():
    c = wide(6, [4200, 4800], 2)
    d = c.upload()
    assert B.prompt_attention_tile_rows(d["p"]) == 256
    c.run(d)
    torch.cuda.synchronize()
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            c.run(d)
    for first in ([0, 9000, 9000], [0, 1, 9000], [3, 4400, 8990], [0, 4200, 9000]):
        c.first, c.lens = first, [first[1] - first[0], first[2] - first[1]]
        d["first"].copy_(i32(first))
        d["out"].fill_(NAN)
        d["lse"].fill_(NAN)
        graph.replay()
        c.check(d)

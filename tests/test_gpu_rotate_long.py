"""Long prompts, whose heads are dealt over workgroups by their number: the same bits as their parts turned alone."""
import pytest
import torch

from paper_2506_03762_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (16, 4), (37, 3)])
@pytest.mark.parametrize("token_major", [False, True])
def test_a_long_prompt_is_turned_as_its_parts(dtype, d, heads, token_major):
    """More tiles of tokens than three per CU, one that is not full among them, and a quarter of the tokens at a time."""
    n = 1030 * 8192 // (d * dtype.itemsize) + 7
    gen = torch.Generator(device="cuda").manual_seed(n)
    def rows(h):
        shape = (1, n, h, d) if token_major else (1, h, n, d)
        t = torch.randn(shape, generator=gen, device="cuda", dtype=dtype)
        return t.transpose(1, 2) if token_major else t
    q, k = rows(heads[0]), rows(heads[1])
    freq, _ = B.rotary_tables(d)
    pos = torch.arange(n, dtype=torch.int32, device="cuda").reshape(1, 1, n)
    def turn(q, k, pos, q_out, k_out):
        B.aha_rotate(B.Rotary.of(q, k, q_out, k_out), q, k, freq, None, pos, q_out, k_out)
    whole, parts = ([torch.empty_like(t).fill_(7.0) for t in (q, k)] for _ in range(2))
    turn(q, k, pos, *whole)
    step = n // 4 + 1
    for at in range(0, n, step):
        piece = slice(at, min(at + step, n))
        turn(q[:, :, piece], k[:, :, piece], pos[:, :, piece].contiguous(), *(t[:, :, piece] for t in parts))
    torch.cuda.synchronize()
    for x, y in zip(whole, parts):
        assert torch.equal(x, y)
    assert not torch.equal(whole[0], q)

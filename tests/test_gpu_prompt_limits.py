"""Attention of packed prompts in more tiles than a launch has workgroups for."""
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests.paged_cases import NAN
from tests.shared_cases import F32, gaussian

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, heads, kv_heads, rows", [(torch.float32, 129, 1, (16, 32)), (torch.float32, 130, 2, (16, 32)),
                                                          (torch.bfloat16, 516, 1, (128, 256))])
def test_more_than_2_to_the_23_tiles(dtype, heads, kv_heads, rows):
    """65535 prompts of a token: each query head's output is the token's value, its log-sum-exp the scaled product.

    Tolerances.  out: the weight 2^(x - x), its reciprocal sum and two products, 6 half steps of fp32, which rounded to bf16 is the value
    again.  lse: the product's 64 terms 20 half steps of the sum of their sizes and the scale, the conversions 4 more."""
    n, d = 65535, 64
    q = gaussian(1, 1, heads, d, dtype=dtype).cuda().expand(n, heads, d)  # (the same rows for all tokens)
    k, v = gaussian(2, n, kv_heads, d, dtype=dtype).cuda(), gaussian(3, n, kv_heads, d, dtype=dtype).cuda()
    first = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    out, lse = torch.full((n, heads, d), NAN, dtype=dtype, device="cuda"), torch.full((heads, n), NAN, device="cuda")
    p = B.PromptAttention.of(q, k, v, out, first)
    assert B.prompt_attention_tile_rows(p) in rows and n * heads // (4 if dtype == torch.bfloat16 else 1) > 2 ** 23
    print("%d prompts of a token, %d heads over %d, %s" % (n, heads, kv_heads, dtype), flush=True)
    B.aha_prompt_attention(p, q, k, v, first, out, lse, B.alloc_prompt_workspace(p))
    torch.cuda.synchronize()
    per = heads // kv_heads
    tol = 0.0 if dtype == torch.bfloat16 else 6 * F32
    for h in range(heads):
        want = v[:, h // per]
        assert bool(((out[:, h] - want).abs() <= tol * want.abs()).all()), h
        product = q[0, h].double() * k[:, h // per].double() * d ** -0.5
        off = (lse[h].double() - product.sum(1)).abs()
        assert bool((off <= 24 * F32 * product.abs().sum(1)).all()), h

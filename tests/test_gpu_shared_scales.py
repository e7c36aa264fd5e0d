"""Attention behind shared prefixes at the ends of the scale's range: 0 and scales whose products only large rows make count."""
import pytest
import torch

from tests.shared_cases import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("q_len", [1, 40, 130])
@pytest.mark.parametrize("scale", [0.0, 2.0 ** -140, 2.0 ** -126, 2.0 ** -124, 2.0 ** -100])
def test_small_scales(dtype, q_len, scale):
    """Queries of about 2^60 and keys of about 2^60 in one channel each: products up to 2^124, logits up to 1 and more.  (The
    smallest scales are subnormal: fp32 holds 2^-140 times log2(e) to 2^-10, which the tolerance has in addition.)"""
    b = Batch(91, q_heads=4, kv_heads=2, d=64, q_len=q_len, tail=[q_len + 9, q_len + 40], prefix=[150], page=16, dtype=dtype, scale=scale)
    size = min(62.0, -torch.log2(torch.tensor(max(scale, 2.0 ** -124))).item() / 2)
    for t in (b.q, b.kp, b.kt):
        t[..., 1:] = torch.where(torch.isnan(t[..., 1:]), t[..., 1:], torch.zeros_like(t[..., 1:]))
        t[..., 0] = (t[..., 0].float().clamp(-1.4, 1.4) * 2.0 ** size).to(dtype)
    d = b.upload()
    b.run(d)
    torch.cuda.synchronize()
    out, tol, lse, ltol = b.reference()
    largest = scale * 2.0 ** (2 * size + 1)
    off = largest * (2.0 ** -10 if scale < 2.0 ** -126 else 0.0) + (2.0 ** -20 if scale == 0.0 else 0.0)
    assert largest <= 2.0
    got = d["out"].double().cpu().numpy(), d["lse"].double().cpu().numpy()
    v = torch.nan_to_num(torch.cat([b.vp.flatten(), b.vt.flatten()]).double()).abs().max().item()
    assert (abs(got[0] - out) <= tol + 2 * off * v).all()
    assert (abs(got[1] - lse) <= ltol + off).all()

"""The angles of the rotation: rows of pairs (1, 0), whose turned values are the cosine and the sine themselves."""
import numpy as np
import pytest
import torch

from paper_2506_03762_amd import binding as B
from tests import shared_cases as S

pytestmark = pytest.mark.gpu


def sines_and_cosines(start, freq, transpose=0, n=4096):
    """(cosines, sines) of the kernel, and in extended precision."""
    x = torch.zeros(1, 1, n, 64)
    x[..., :32] = 1.0
    pos = (start + torch.arange(n, dtype=torch.int64)).to(torch.int32).reshape(1, 1, n)
    w = torch.full((32,), freq) * torch.linspace(0.5, 1.0, 32)
    got = torch.empty_like(x, device="cuda")
    p = B.Rotary.of(x, None, got, transpose=transpose)
    B.aha_rotate(p, x.cuda(), None, w.cuda(), None, pos.cuda(), got, None)
    ang = S.angles(pos, w, None)[0]
    got = got.cpu().double().numpy()[0, 0]
    c, s = (np.asarray(f(ang), np.float64) for f in (np.cos, np.sin))
    return (got[:, :32], got[:, 32:]), (c, -s if transpose else s)


FAR = pytest.mark.parametrize("start", [0, 1000003, 2 ** 31 - 4096, -2 ** 31])


@FAR
@pytest.mark.parametrize("freq", [1.0, 0.866, 0.01])
def test_far_positions_lose_nothing(start, freq):
    """The angle is off by at most 2^-26 of a turn wherever the position lies.  Sine and cosine of it: 4 units (2^-23) of
    the value; what is turned is 1 and 0, whose products and sum are exact."""
    got, want = sines_and_cosines(start, freq)
    for g, v, slope in zip(got, want, reversed(want)):
        tol = 1.001 * 2 * np.pi * 2.0 ** -26 * (np.abs(slope) + 2.0 ** -24) + 4 * 2.0 ** -23 * np.abs(v)
        S.assert_within(torch.from_numpy(g), v, tol, "start %d, frequency %g" % (start, freq))


@FAR
@pytest.mark.parametrize("transpose", [0, 1])
def test_the_angle_is_not_rounded_to_fp32(start, transpose):
    """Sine and cosine are as near as fp32 holds them, those near 0 too: 4 units (2^-23) of the value, and what double
    leaves open of the angle (2^-49 of a turn and less, 2^-40 allowed)."""
    for freq in (1.0, 0.3):
        got, want = sines_and_cosines(start, freq, transpose)
        for g, v in zip(got, want):
            S.assert_within(torch.from_numpy(g), v, 4 * 2.0 ** -23 * np.abs(v) + 2.0 ** -40, "start %d, frequency %g" % (start, freq))

"""Calls with tensors that are laid out otherwise than described: refused before anything is launched, no GPU needed."""
import pytest
import torch

from paper_2506_03762_amd import binding as B

BF = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """The names of the entry points that are reached, in place of the library."""
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)   # (tensors of the CPU count as the device's)
    called = []
    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0
    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "_stream", lambda: None)
    return called


def rows(*shape):
    return torch.zeros(shape, dtype=BF)


def token_major(*shape):
    """The same shape, [., n, heads, d] in memory."""
    b, h, n, d = shape
    return rows(b, n, h, d).transpose(1, 2)


def wide(*shape):
    """The same shape, rows three times as far apart."""
    return rows(*shape[:3], 3 * shape[3])[..., shape[3]:2 * shape[3]]


def first_heads(*shape):
    """The same shape, the first heads of four times as many."""
    return rows(shape[0], 4 * shape[1], *shape[2:])[:, :shape[1]]


MAKERS = (rows, token_major, wide, first_heads)
PAIRS = [(a, b) for a in MAKERS for b in MAKERS if a is not b]


@pytest.mark.parametrize("described,given", PAIRS)
def test_rotated_and_appended_rows(calls, described, given):
    freq, pos = torch.zeros(32), torch.zeros(1, 2, 3, dtype=torch.int32)
    q, k = (2, 8, 3, 64), (2, 2, 3, 64)
    mine = [described(*s) for s in (q, k, q, k, k)]                                  # q, k, q_out, k_out, v
    p = B.Rotary.of(*mine)
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pools = [described(9, 2, 16, 64) for _ in range(2)]
    cache = B.Pages.of(*pools, table)
    def rotate(x):
        B.aha_rotate(p, x[0], x[1], freq, None, pos, x[2], x[3])
    def append(x, y):
        B.aha_append_paged(p, cache, x[0], x[1], x[4], freq, None, pos, table, lens, None, x[2], *y)
    rotate(mine)
    append(mine, pools)
    assert calls == ["aha_rotate", "aha_append_paged"]
    for i, shape in enumerate((q, k, q, k, k)):
        other = mine[:i] + [given(*shape)] + mine[i + 1:]
        if i != 4:
            with pytest.raises(ValueError):
                rotate(other)
        if i != 3:
            with pytest.raises(ValueError):
                append(other, pools)
    for i in range(2):
        with pytest.raises(ValueError):
            append(mine, pools[:i] + [given(9, 2, 16, 64)] + pools[i + 1:])
    assert len(calls) == 2


@pytest.mark.parametrize("described,given", PAIRS)
def test_attention(calls, described, given):
    shapes = [(3, 8, 5, 64), (2, 2, 100, 64), (2, 2, 100, 64), (9, 2, 16, 64), (9, 2, 16, 64), (3, 8, 5, 64)]
    mine = [described(*s) for s in shapes]                                           # q, prefixes, pools, out
    table, lens = torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    p, cache = B.SharedAttention.of(mine[0], mine[5], mine[1], mine[2]), B.Pages.of(mine[3], mine[4], table)
    def attend(x):
        B.aha_shared_attention(p, cache, x[0], x[1], x[2], lens[:2], torch.zeros(3, dtype=torch.int32), x[3], x[4], table, lens,
                               None, x[5], None, None)
    attend(mine)
    for i, shape in enumerate(shapes):
        with pytest.raises(ValueError):
            attend(mine[:i] + [given(*shape)] + mine[i + 1:])
    assert calls == ["aha_shared_attention"]


def test_what_lies_at_the_same_places_is_taken(calls):
    """Axes of one element have no stride that counts, and may be left out."""
    freq, pos = torch.zeros(32), torch.zeros(1, 4, 1, dtype=torch.int32)
    p = B.Rotary.of(rows(4, 8, 1, 64), None, rows(4, 8, 1, 64))
    out = rows(4, 8, 1, 64)
    for q in (token_major(4, 8, 1, 64), rows(4, 8, 64), rows(4, 1, 8, 64).transpose(1, 2)):
        B.aha_rotate(p, q, None, freq, None, pos, out, None)
    assert len(calls) == 3
    for q in (rows(4 * 8, 64), rows(8, 4, 1, 64), rows(1, 1, 1, 64).expand(4, 8, 1, 64)):
        with pytest.raises(ValueError):
            B.aha_rotate(p, q, None, freq, None, pos, out, None)
    assert len(calls) == 3


def test_as_many_elements_at_the_same_strides(calls):
    """[2, 8, ...] and [8, 2, ...] at the same strides: the memory that the one has is not the other's."""
    freq = torch.zeros(32)
    q, out = first_heads(8, 2, 3, 64), first_heads(8, 2, 3, 64)                      # 1536 elements from batch to batch
    other = rows(2, 8, 3, 64)
    assert other.stride() == q.stride() and other.numel() == q.numel()
    p = B.Rotary.of(q, None, out)
    with pytest.raises(ValueError):
        B.aha_rotate(p, other, None, freq, None, torch.zeros(1, 8, 3, dtype=torch.int32), out, None)
    assert calls == []


def test_what_is_not_described_is_refused(calls):
    freq, pos = torch.zeros(32), torch.zeros(1, 2, 3, dtype=torch.int32)
    k = rows(2, 2, 3, 64)
    p = B.Rotary.of(None, k, None, k)
    B.aha_rotate(p, None, k, freq, None, pos, None, k)
    with pytest.raises(ValueError):
        B.aha_rotate(p, k, k, freq, None, pos, k, k)
    table, lens = torch.zeros(2, 4, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    pool = rows(9, 2, 16, 64)
    with pytest.raises(ValueError):
        B.aha_append_paged(p, B.Pages.of(pool, pool, table), None, k, k, freq, None, pos, table, lens, None, None, pool, pool)
    s = B.SharedAttention.of(k, k, n_kv_heads=2)
    with pytest.raises(ValueError):
        B.aha_shared_attention(s, None, k, pool, pool, None, None, None, None, None, None, None, k, None, None)
    assert calls == ["aha_rotate"]


def test_workspace(calls):
    """One of another device, or whose elements share their memory, would be written outside its memory."""
    q = rows(2, 2, 3, 64)
    s = B.SharedAttention.of(q, q, n_kv_heads=2)
    def attend(workspace):
        B.aha_shared_attention(s, None, q, None, None, None, None, None, None, None, None, None, q, None, workspace)
    class OfAnotherDevice(torch.Tensor):
        def get_device(self):
            return 0
    attend(torch.zeros(256, dtype=torch.uint8))
    attend(None)
    for workspace in (torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(256, dtype=torch.uint8).as_subclass(OfAnotherDevice)):
        with pytest.raises(ValueError):
            attend(workspace)
    assert calls == ["aha_shared_attention"] * 2


def test_one_half_of_a_prefix():
    q, prefix = rows(2, 2, 3, 64), rows(1, 2, 50, 64)
    for k, v in ((prefix, None), (None, prefix)):
        with pytest.raises(ValueError):
            B.SharedAttention.of(q, q, k, v, n_kv_heads=2)

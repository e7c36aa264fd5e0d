"""Attention behind shared prefixes (aha_shared_attention) against 64 bits."""
import numpy as np
import pytest
import torch

from tests.shared_cases import Batch

pytestmark = pytest.mark.gpu

BOTH = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])


@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_single_tokens(dtype, d):
    Batch(1, q_heads=4, kv_heads=2, d=d, q_len=1, tail=[1, 7, 40, 16], prefix=[100], dtype=dtype).check()
    Batch(2, q_heads=3, kv_heads=3, d=d, q_len=1, tail=[5], prefix=[1], page=1, dtype=dtype).check()
    Batch(3, q_heads=8, kv_heads=1, d=d, q_len=1, tail=[33, 1, 130, 64, 65, 2, 31], prefix=[31, 257], first=[0, 3, 7],
          page=32, dtype=dtype, layout="bnhd").check()
    Batch(4, q_heads=14, kv_heads=2, d=d, q_len=1, tail=[100] * 11, prefix=[1000], page=64, dtype=dtype, hot=4.0).check()


@BOTH
@pytest.mark.parametrize("d", [64, 128])
def test_chunks(dtype, d):
    Batch(5, q_heads=4, kv_heads=2, d=d, q_len=3, tail=[3, 10, 17], prefix=[65], dtype=dtype).check()
    Batch(6, q_heads=4, kv_heads=2, d=d, q_len=33, tail=[40, 33, 200], new=[33, 20, 1], prefix=[300, 7], first=[0, 1, 3],
          page=8, dtype=dtype, layout="bnhd").check()
    Batch(7, q_heads=2, kv_heads=1, d=d, q_len=150, tail=[150, 700], new=[150, 149], prefix=[513], page=128, dtype=dtype).check()


@BOTH
def test_rows_without_keys_and_padding(dtype):
    # no prefix for sequences 0 and 4, an empty prefix, tails without tokens, sequences without new rows
    d = Batch(8, q_heads=4, kv_heads=2, d=64, q_len=2, tail=[0, 0, 9, 2, 0, 5], new=[2, 1, 2, 0, 2, 2], prefix=[0, 40],
              first=[1, 2, 4], dtype=dtype).check()
    assert torch.isneginf(d["lse"][0]).all()
    # tails shorter than their new rows: the first rows come before token 0
    Batch(9, q_heads=2, kv_heads=2, d=128, q_len=6, tail=[3, 0, 6], dtype=dtype).check()
    Batch(10, q_heads=2, kv_heads=2, d=128, q_len=40, tail=[35, -4, 2], new=[40, 3, 40], prefix=[3], first=[2, 3], dtype=dtype).check()


@BOTH
def test_holes(dtype):
    holes = {(0, 0): -1, (0, 2): 10 ** 6, (1, 1): -7, (2, 0): -1, (2, 1): -1, (2, 2): -1}
    for page in (4, 16, 32, 64):
        Batch(11, q_heads=4, kv_heads=2, d=128, q_len=2, tail=[3 * page, 2 * page + 1, 3 * page - 1], page=page, holes=holes,
              prefix=[20], first=[0, 2], dtype=dtype).check()


@BOTH
def test_prefix_alone(dtype):
    """Without tails: the attention of rows over an encoder's states, say."""
    Batch(12, q_heads=4, kv_heads=4, d=64, q_len=19, tail=[0, 0], prefix=[77, 300], first=[0, 1, 2], dtype=dtype, tails=False).check()


@BOTH
def test_tails_alone(dtype):
    Batch(13, q_heads=4, kv_heads=1, d=128, q_len=1, tail=[1, 300, 64, 999], page=16, dtype=dtype).check()


def test_lengths_beyond_what_is_there_are_clamped():
    b = Batch(14, q_heads=4, kv_heads=2, d=64, q_len=2, tail=[32, 10], new=[2, 2], prefix=[50], cap=50, page=16)
    d = b.upload()
    d["prefix"].fill_(2 ** 31 - 1)
    d["new"].fill_(99)
    d["first"].copy_(torch.tensor([0, 2 ** 31 - 1], dtype=torch.int32))
    b.run(d)
    b.check(d)
    d["first"].copy_(torch.tensor([-2 ** 31, 2], dtype=torch.int32))
    d["out"].fill_(float("nan"))
    b.run(d)
    b.check(d)


def test_members_in_many_groups():
    rng = np.random.default_rng(3)
    batch = 37
    first = np.sort(rng.integers(0, batch + 1, size=9)).tolist()
    Batch(15, q_heads=6, kv_heads=2, d=64, q_len=1, tail=rng.integers(1, 90, batch).tolist(), prefix=rng.integers(0, 400, 8).tolist(),
          first=first, page=16).check()


def test_more_prefixes_than_lanes():
    rng = np.random.default_rng(4)
    batch, n = 190, 150
    first = np.sort(rng.integers(0, batch + 1, size=n + 1)).tolist()
    Batch(19, q_heads=2, kv_heads=1, d=64, q_len=1, tail=rng.integers(1, 20, batch).tolist(), prefix=rng.integers(0, 60, n).tolist(),
          first=first, page=16).check()


@BOTH
def test_nothing_to_attend_to(dtype):
    """Neither prefixes nor tails: zeros, and -inf."""
    Batch(20, q_heads=4, kv_heads=2, d=64, q_len=3, tail=[0, 0], new=[3, 1], dtype=dtype, tails=False).check()


def test_more_pages_than_a_large_tile_keeps():
    """256 (sequence, KV head) problems, so that one item has a tail's 2500 pages of a token each; some are holes."""
    Batch(21, q_heads=128, kv_heads=128, d=64, q_len=70, tail=[2500, 2300], page=1, holes={(0, 5): -1, (0, 2200): -1, (1, 2299): -1}).check()


@BOTH
@pytest.mark.parametrize("q_len", [3, 90])
def test_what_is_not_finite_stays_with_the_rows_that_see_it(dtype, q_len):
    """Keys of one sequence's newest token, and values and keys of another one's old ones, that are NaN or infinite: the rows
    that do not see them get the same bits as without them, the others no numbers."""
    b = Batch(22, q_heads=4, kv_heads=2, d=64, q_len=q_len, tail=[q_len + 5, q_len + 30, q_len + 70], prefix=[200], page=16, dtype=dtype)
    d = b.upload()
    b.run(d)
    b.check(d)
    clean = d["out"].clone(), d["lse"].clone()
    for fill in (float("nan"), float("inf"), -float("inf")):
        kt, vt = b.kt.clone(), b.vt.clone()
        _, page, row = b.slots(0)[-1]
        kt[page, :, row] = fill                     # the newest token of sequence 0: seen by its last row alone
        _, page, row = b.slots(2)[3]
        vt[page, :, row] = fill                     # an old one of sequence 2: seen by all its rows
        d["kt"].copy_(kt)
        d["vt"].copy_(vt)
        b.run(d)
        torch.cuda.synchronize()
        for got, was in zip((d["out"], d["lse"]), clean):
            assert torch.equal(got[1], was[1]) and torch.equal(got[0, :, :-1], was[0, :, :-1])
        assert torch.equal(d["lse"][2], clean[1][2])
        assert not torch.isfinite(d["out"][2].float()).any()
        assert not torch.equal(d["lse"][0, :, -1], clean[1][0, :, -1])


def test_heads_that_share_a_prefix():
    """A prefix whose KV heads are one (a stride of 0), and queries that all heads share."""
    b = Batch(23, q_heads=4, kv_heads=2, d=128, q_len=2, tail=[9, 30], prefix=[300], page=16)
    b.q = b.q[:, :1].expand(-1, 4, -1, -1)
    b.kp, b.vp = (t[:, :1].expand(-1, 2, -1, -1) for t in (b.kp, b.vp))
    d = b.upload()
    for x, t in (("q", b.q), ("kp", b.kp), ("vp", b.vp)):
        d[x] = t[:, :1].contiguous().cuda().expand_as(t)
    from paper_2506_03762_amd import binding as B
    d["p"] = B.SharedAttention.of(d["q"], d["out"], d["kp"], d["vp"], b.scale)
    b.run(d)
    b.check(d)


def random_batch(seed):
    rng = np.random.default_rng(seed)
    log = lambda lo, hi: int(round(np.exp(rng.uniform(np.log(lo), np.log(hi)))))
    f32 = rng.random() < 0.25
    batch, hkv, group = log(1, 24), int(rng.choice([1, 2, 3])), int(rng.choice([1, 2, 3, 4, 7, 8]))
    q_len = int(rng.choice([1, 1, log(2, 8), log(9, 140)]))
    prefixes = int(rng.choice([0, 1, 1, 2, 5]))
    prefix = [int(rng.choice([0, log(1, 60), log(60, 3000)])) for _ in range(prefixes)]
    new = rng.integers(0, q_len + 1, batch) if rng.random() < 0.5 else np.full(batch, q_len)
    tail = new + [log(1, 500) - 1 for _ in range(batch)]
    page = int(rng.choice([1, 4, 16, 32, 64, 256]))
    width = -(-int(max(tail.max(), 1)) // page)
    holes = {(int(rng.integers(batch)), int(rng.integers(width))): int(rng.choice([-1, 10 ** 6])) for _ in range(rng.integers(0, 6))}
    first = np.sort(rng.integers(0, batch + 1, prefixes + 1)).tolist() if prefixes else None
    return Batch(seed, q_heads=hkv * group, kv_heads=hkv, d=int(rng.choice([64, 128])), q_len=q_len, tail=tail.tolist(),
                 new=new.tolist() if rng.random() < 0.8 or (new < q_len).any() else None, prefix=prefix, first=first, page=page, holes=holes,
                 cap=max(prefix + [1]) + int(rng.integers(0, 50)), dtype=torch.float32 if f32 else torch.bfloat16,
                 layout=str(rng.choice(["bhnd", "bnhd"])), scale=None if rng.random() < 0.8 else float(rng.choice([0.0, 0.3])),
                 hot=float(rng.choice([0.0, 3.0])))


@pytest.mark.parametrize("block", range(6))
def test_random_batches(block):
    for seed in range(100 + 10 * block, 110 + 10 * block):
        print("seed", seed, end=" ", flush=True)
        random_batch(seed).check()


@BOTH
def test_logits_that_keep_rising(dtype):
    """Keys that grow along the queries' direction: the running maximum moves in every step, in small
    and in large ones."""
    for slope in (0.02, 0.3):
        b = Batch(16, q_heads=8, kv_heads=2, d=64, q_len=2, tail=[300, 200], prefix=[1500], page=16, dtype=dtype)
        u = torch.randn(64, generator=torch.Generator().manual_seed(1)).to(dtype)
        b.q += u
        for t in (b.kp, b.kt):
            t += (torch.arange(t.size(2))[None, None, :, None] * slope * u / 8).to(dtype)
        b.check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("q_len", [25, 60])
def test_logits_that_keep_rising_in_large_tiles(d, q_len):
    """The same with 100 and 240 rows of a prefix and of a tail: references that stay (rises of less than 2^20), that move
    in some blocks and in all, and weights that would not be numbers without the move."""
    for slope in (0.003, 0.05, 0.5, 8.0):
        b = Batch(18, q_heads=4, kv_heads=1, d=d, q_len=q_len, tail=[400], prefix=[1300], page=32)
        u = torch.randn(d, generator=torch.Generator().manual_seed(1)).to(b.dtype)
        b.q += u
        for t in (b.kp, b.kt):
            t += (torch.arange(t.size(2))[None, None, :, None] * slope * u / 8).to(b.dtype)
        b.check()


@pytest.mark.parametrize("rows,prefix", [(65, 1000), (100, 64), (128, 4097), (129, 500), (200, 4000), (256, 1), (257, 777), (600, 2500)])
def test_large_tiles(rows, prefix):
    """Rows around the tiles' sizes, of one prefix and of several, single tokens and chunks."""
    for d in (64, 128):
        Batch(rows, q_heads=1, kv_heads=1, d=d, q_len=1, tail=[1 + i % 40 for i in range(rows)], prefix=[prefix], page=8).check()
        Batch(rows + 1, q_heads=2, kv_heads=2, d=d, q_len=rows, tail=[rows + 100], prefix=[prefix], page=16, holes={(0, 3): -1},
              layout="bnhd").check()
    Batch(rows + 2, q_heads=5, kv_heads=1, d=128, q_len=(rows + 9) // 10, tail=[(rows + 9) // 10 + 3] * 6, prefix=[prefix, 300, 0],
          first=[0, 2, 5, 6], page=1).check()


def test_without_lse_and_in_strided_outputs():
    b = Batch(17, q_heads=4, kv_heads=2, d=128, q_len=5, tail=[20, 9], prefix=[200])
    d = b.upload()
    b.run(d)
    wide = torch.full((2, 4, 5, 3 * 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    dense = d["out"].clone()
    from paper_2506_03762_amd import binding as B
    d["out"] = wide[..., 128:256]
    d["p"] = B.SharedAttention.of(d["q"], d["out"], d["kp"], d["vp"], b.scale)
    d["ws"].fill_(0x5A)
    b.run(d, lse=False)
    torch.cuda.synchronize()
    assert torch.equal(d["out"], dense)
    assert torch.isnan(wide[..., :128].float()).all() and torch.isnan(wide[..., 256:].float()).all()

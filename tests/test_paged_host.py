"""Host side of packed prompts' attention, single tokens' attention over paged caches and eviction from them, no GPU needed:
struct layouts, refusals before anything is launched, workspace sizes, the binding's descriptions."""
import ctypes

import pytest
import torch

from paper_2506_03762_amd import binding as B

PTR, ODD, OTHER = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x1004), ctypes.c_void_p(0x2000)


def two(*x):
    return (ctypes.c_int64 * 2)(*x)


def three(*x):
    return (ctypes.c_int64 * 3)(*x)


def test_struct_layouts():
    assert ctypes.sizeof(B.aha_prompt) == 8 * 4 + 4 * 16 and B.aha_prompt.q_stride.offset == 32
    assert ctypes.sizeof(B.aha_paged) == 14 * 4 + 6 * 16 and B.aha_paged.scale.offset == 40 and B.aha_paged.q_stride.offset == 56


def prompt(**kw):
    base = dict(tokens=100, sequences=3, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=B.AHA_BF16, scale=0.1,
                q_stride=two(1024, 128), k_stride=two(256, 128), v_stride=two(256, 128), out_stride=two(1024, 128))
    base.update(kw)
    return B.aha_prompt(**base)


def pages(**kw):
    base = dict(n_pages=50, page_size=16, table_width=20, k_stride=three(4096, 2048, 128), v_stride=three(4096, 2048, 128))
    base.update(kw)
    return B.aha_pages(**base)


def paged(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=B.AHA_BF16, slots=320, budget=64, recent=8, sink=4,
                scale_mode=B.AHA_SCALE_ADAPTIVE, scale=0.1, fixed_scale=0.0, lambda_floor=-1.0, q_stride=two(1024, 128),
                out_stride=two(1024, 128), scores_stride=two(640, 320), pos_stride=two(640, 320),
                scores_out_stride=two(640, 320), pos_out_stride=two(640, 320))
    base.update(kw)
    return B.aha_paged(**base)


def ref(p):
    return None if p is None else ctypes.byref(p)


def prompt_attention(p, ws=PTR, nbytes=1 << 40, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, first=PTR, out=PTR, lse=PTR)
    a.update(kw)
    return B.load().aha_prompt_attention(ref(p), *a.values(), ws, nbytes, None)


def attention(p, pg, ws=PTR, nbytes=1 << 40, **kw):
    a = dict(q=PTR, k_pages=PTR, v_pages=PTR, page_table=PTR, tail_len=PTR, seen=PTR, scores=PTR, pos=PTR, out=PTR, lse=PTR)
    a.update(kw)
    return B.load().aha_paged_attention(ref(p), ref(pg), *a.values(), ws, nbytes, None)


def evict(p, pg, ws=PTR, nbytes=1 << 40, **kw):
    a = dict(scores=PTR, pos=PTR, k_pages=PTR, v_pages=PTR, page_table=PTR, tail_len=PTR, seen=PTR, scores_out=PTR, pos_out=PTR,
             len_out=OTHER)
    a.update(kw)
    return B.load().aha_paged_evict(ref(p), ref(pg), *a.values(), ws, nbytes, None)


INVALID, UNSUPPORTED = B.AHA_ERR_INVALID_ARG, B.AHA_ERR_UNSUPPORTED


@pytest.mark.parametrize("change, code", [
    (dict(tokens=0), INVALID), (dict(sequences=0), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_heads=0), INVALID),
    (dict(n_q_heads=7), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(sequences=65536), UNSUPPORTED),
    (dict(tokens=2 ** 28), UNSUPPORTED), (dict(scale=-0.1), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(scale=3e38), INVALID), (dict(reserved=1), INVALID),
    (dict(q_stride=two(1024, 127)), INVALID), (dict(k_stride=two(-256, 128)), INVALID), (dict(v_stride=two(4, 128)), INVALID),
    (dict(out_stride=two(0, 128)), INVALID), (dict(out_stride=two(1024, 64)), INVALID),
])
def test_prompts_that_are_refused(change, code):
    assert prompt_attention(prompt(**change)) == code
    assert B.load().aha_last_error()


def test_prompt_pointers():
    for name in ("q", "k", "v", "first", "out"):
        assert prompt_attention(prompt(), **{name: None}) == INVALID
    for name in ("q", "k", "v", "out"):
        assert prompt_attention(prompt(), **{name: ODD}) == INVALID
    assert prompt_attention(None) == INVALID
    n = ctypes.c_size_t(0)
    assert B.load().aha_prompt_attention_workspace_bytes(ref(prompt()), None) == INVALID
    assert B.load().aha_prompt_attention_workspace_bytes(ref(prompt(tokens=0)), ctypes.byref(n)) == INVALID


BOTH_REFUSE = [
    (dict(batch=0), INVALID), (dict(n_kv_heads=0), INVALID), (dict(head_dim=32), UNSUPPORTED), (dict(dtype=-1), INVALID),
    (dict(batch=40000), UNSUPPORTED), (dict(slots=-1), INVALID), (dict(slots=2 ** 30 + 1), UNSUPPORTED), (dict(budget=0), INVALID),
    (dict(reserved=3), INVALID), (dict(scores_stride=two(-1, 320)), INVALID),
]
BAD_PAGES = [
    (dict(n_pages=0), INVALID), (dict(page_size=12), UNSUPPORTED), (dict(page_size=2048), UNSUPPORTED), (dict(table_width=0), INVALID),
    (dict(reserved=1), INVALID), (dict(k_stride=three(4096, 2048, 64)), INVALID), (dict(v_stride=three(64, 2048, 128)), INVALID),
]


@pytest.mark.parametrize("change, code", BOTH_REFUSE + [
    (dict(n_q_heads=9), INVALID), (dict(n_q_heads=4096), UNSUPPORTED), (dict(scale_mode=2), INVALID), (dict(scale=-1.0), INVALID),
    (dict(fixed_scale=float("nan")), INVALID), (dict(lambda_floor=float("inf")), INVALID), (dict(q_stride=two(1024, 4)), INVALID),
    (dict(out_stride=two(1024, 8)), INVALID), (dict(scores_stride=two(640, 100)), INVALID), (dict(pos_stride=two(0, 320)), INVALID),
    (dict(slots=0), INVALID),  # with scores
])
def test_attention_that_is_refused(change, code):
    assert attention(paged(**change), pages()) == code


@pytest.mark.parametrize("change, code", BOTH_REFUSE + [
    (dict(slots=0), INVALID), (dict(recent=-1), INVALID), (dict(sink=-1), INVALID), (dict(recent=61), INVALID),
    (dict(recent=2 ** 31 - 1, sink=2 ** 31 - 1), INVALID), (dict(scores_out_stride=two(640, 319)), INVALID),
    (dict(pos_out_stride=two(0, 320)), INVALID), (dict(scores_stride=two(1280, 320)), INVALID),  # in place
    (dict(pos_out_stride=two(640, 330)), INVALID),
])
def test_evictions_that_are_refused(change, code):
    assert evict(paged(**change), pages()) == code


@pytest.mark.parametrize("change, code", BAD_PAGES)
def test_pages_that_are_refused(change, code):
    assert attention(paged(), pages(**change)) == code and evict(paged(), pages(**change)) == code


def test_pointers_and_workspaces():
    assert attention(None, pages()) == INVALID and attention(paged(), None) == INVALID
    assert evict(None, pages()) == INVALID and evict(paged(), None) == INVALID
    for name in ("q", "k_pages", "v_pages", "page_table", "tail_len", "scores", "out"):
        assert attention(paged(), pages(), **{name: None}) == INVALID
    for name in ("scores", "k_pages", "v_pages", "page_table", "tail_len", "scores_out", "pos_out", "len_out"):
        assert evict(paged(), pages(), **{name: None}) == INVALID
    assert evict(paged(), pages(), len_out=PTR) == INVALID  # tail_len
    assert evict(paged(), pages(), len_out=PTR, tail_len=OTHER) == INVALID  # seen
    n = ctypes.c_size_t(0)
    for call, size in ((attention, B.load().aha_paged_attention_workspace_bytes), (evict, B.load().aha_paged_evict_workspace_bytes)):
        assert size(ref(paged()), ref(pages()), ctypes.byref(n)) == B.AHA_OK and n.value % 256 == 0 and n.value > 0
        assert call(paged(), pages(), nbytes=n.value - 1) == B.AHA_ERR_WORKSPACE
        assert call(paged(), pages(), ws=None) == B.AHA_ERR_WORKSPACE
        assert call(paged(), pages(), ws=ODD) == B.AHA_ERR_WORKSPACE
        assert size(ref(paged()), ref(pages()), None) == INVALID and size(ref(paged()), None, ctypes.byref(n)) == INVALID


def test_workspaces_of_the_largest_problems_fit_their_type():
    n = ctypes.c_size_t(0)
    big = paged(batch=8191, n_q_heads=512, n_kv_heads=8, slots=2 ** 30)
    assert B.load().aha_paged_attention_workspace_bytes(ref(big), ref(pages(table_width=2 ** 20, page_size=1024)), ctypes.byref(n)) == B.AHA_OK
    assert n.value >= 8191 * 512 * 2 ** 30 * 4
    assert B.load().aha_paged_evict_workspace_bytes(ref(paged(batch=8191, n_kv_heads=8, slots=2 ** 30, budget=2 ** 29)),
                                                    ref(pages(table_width=2 ** 20, page_size=1024)), ctypes.byref(n)) == B.AHA_OK
    assert n.value >= 8191 * 8 * 2 ** 29 * 8


def test_descriptions_refuse_other_layouts():
    bf = torch.bfloat16
    q, k, out = torch.zeros(10, 4, 64, dtype=bf), torch.zeros(10, 2, 64, dtype=bf), torch.zeros(10, 4, 64, dtype=bf)
    first = torch.zeros(3, dtype=torch.int32)
    p = B.PromptAttention.of(q, k, k, out, first)
    assert (p.struct.tokens, p.struct.sequences, p.struct.n_q_heads, p.struct.n_kv_heads) == (10, 2, 4, 2)
    for bad in ((q, k, k, out[:9], first), (q, k[:9], k[:9], out, first), (q, k.float(), k, out, first), (q, k, k[:, :1], out, first),
                (q.transpose(1, 2), k, k, out, first), (q[0], k, k, out, first)):
        with pytest.raises((ValueError, IndexError)):
            B.PromptAttention.of(*bad)
    scores, pos = torch.zeros(2, 2, 320), torch.zeros(2, 2, 320, dtype=torch.int32)
    q, out = torch.zeros(2, 4, 64, dtype=bf), torch.zeros(2, 4, 64, dtype=bf)
    pool, table = torch.zeros(50, 2, 16, 64, dtype=bf), torch.zeros(2, 20, dtype=torch.int32)
    cache = B.Pages.of(pool, pool, table)
    B.PagedAttention.of(q, out, scores, pos, budget=64)
    B.PagedAttention.of(q, out, n_kv_heads=2)
    for bad in (dict(scores=scores.double()), dict(scores=scores, pos=pos.long()), dict(scores=scores, pos=pos[..., :300]),
                dict(scores=scores[:1]), dict(scores=None), dict(scores=None, pos=pos, n_kv_heads=2), dict(scores=scores.transpose(1, 2))):
        with pytest.raises(ValueError):
            B.PagedAttention.of(q, out, **bad)
    B.PagedEviction.of(scores, None, scores, pos, cache, budget=64)
    for bad in ((scores[:1], None, scores, pos), (scores, None, scores[..., :9], pos), (scores, pos, scores, pos[:, :1]), (scores, None, pos, pos)):
        with pytest.raises(ValueError):
            B.PagedEviction.of(*bad, cache, budget=64)


def test_tensors_in_one_look():
    """The compiled checks of a call's tensors say the same as those that name what is wrong."""
    from paper_2506_03762_amd import _tensors
    rows, few = torch.zeros(4, 6, 8, dtype=torch.bfloat16)[:, ::2], torch.zeros(5, dtype=torch.int32)
    what = (("q", torch.bfloat16, None, rows.shape, rows.stride()), ("seen", torch.int32, 5, None, None), ("pos", torch.int32, None, (), ()))
    assert _tensors.pointers(what, (rows, few, None), -1) == [rows.data_ptr(), few.data_ptr(), None]
    assert B._fast_pointers is _tensors.pointers
    for given, device in (((rows, few, None), 0), ((rows.float(), few, None), -1), ((rows.contiguous(), few, None), -1), ((rows[:3], few, None), -1),
                          ((rows, few[:4], None), -1), ((rows, torch.zeros(10, dtype=torch.int32)[::2], None), -1), ((rows, few.long(), None), -1),
                          ((rows, few, few), -1), ((rows, few), -1), ((rows, 5, None), -1), ((rows, few.to_sparse(), None), -1),
                          ((rows, few.numpy(), None), -1)):
        assert _tensors.pointers(what, given, device) is None, given
    assert _tensors.pointers((("x",),), (few,), -1) is None and _tensors.pointers(what, (rows, few, None)) is None

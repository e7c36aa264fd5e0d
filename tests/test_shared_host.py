"""Host side of rotation, the paged cache and the attention behind shared prefixes, no GPU needed: struct layouts,
refusals before anything is launched, the binding's descriptions."""
import ctypes

import pytest
import torch

from paper_2506_03762_amd import binding as B

PTR = ctypes.c_void_p(0x1000)
ODD = ctypes.c_void_p(0x1004)


def test_struct_layouts():
    assert ctypes.sizeof(B.aha_rotary) == 10 * 4 + 5 * 24 and B.aha_rotary.q_stride.offset == 40
    assert ctypes.sizeof(B.aha_pages) == 4 * 4 + 2 * 24 and B.aha_pages.k_stride.offset == 16
    assert ctypes.sizeof(B.aha_shared) == 10 * 4 + 4 * 24 and B.aha_shared.scale.offset == 32


def three(*x):
    return (ctypes.c_int64 * 3)(*x)


def rotary(**kw):
    base = dict(batch=2, tokens=100, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=B.AHA_BF16, rot_dim=128, pairing=0,
                n_axes=1, transpose=0, q_stride=three(102400, 12800, 128), k_stride=three(25600, 12800, 128),
                v_stride=three(25600, 12800, 128), q_out_stride=three(102400, 12800, 128), k_out_stride=three(25600, 12800, 128))
    base.update(kw)
    return B.aha_rotary(**base)


def pages(**kw):
    base = dict(n_pages=50, page_size=16, table_width=20, k_stride=three(4096, 2048, 128), v_stride=three(4096, 2048, 128))
    base.update(kw)
    return B.aha_pages(**base)


def shared(**kw):
    base = dict(batch=2, q_len=1, n_q_heads=8, n_kv_heads=2, head_dim=128, dtype=B.AHA_BF16, n_prefixes=1, prefix_cap=300,
                scale=0.1, q_stride=three(1024, 128, 128), out_stride=three(1024, 128, 128),
                k_stride=three(76800, 38400, 128), v_stride=three(76800, 38400, 128))
    base.update(kw)
    return B.aha_shared(**base)


def rotate(p, **kw):
    a = dict(q=PTR, k=PTR, inv_freq=PTR, pair_axis=None, positions=PTR, q_out=PTR, k_out=PTR)
    a.update(kw)
    return B.load().aha_rotate(None if p is None else ctypes.byref(p), *a.values(), None)


def append(p, pg, **kw):
    a = dict(q=PTR, k=PTR, v=PTR, inv_freq=PTR, pair_axis=None, positions=PTR, page_table=PTR, tail_len=PTR, new_len=None,
             q_out=PTR, k_pages=PTR, v_pages=PTR)
    a.update(kw)
    return B.load().aha_append_paged(ctypes.byref(p), None if pg is None else ctypes.byref(pg), *a.values(), None)


def attend(p, pg, ws=PTR, nbytes=1 << 40, **kw):
    a = dict(q=PTR, k_prefix=PTR, v_prefix=PTR, prefix_len=PTR, prefix_first=PTR, k_pages=PTR, v_pages=PTR, page_table=PTR,
             tail_len=PTR, new_len=None, out=PTR, lse=None)
    a.update(kw)
    return B.load().aha_shared_attention(ctypes.byref(p), None if pg is None else ctypes.byref(pg), *a.values(), ws, nbytes, None)


BAD, NOT_BUILT, WS = B.AHA_ERR_INVALID_ARG, B.AHA_ERR_UNSUPPORTED, B.AHA_ERR_WORKSPACE


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), BAD), (dict(tokens=0), BAD), (dict(n_q_heads=0), BAD), (dict(n_kv_heads=-1), BAD),
    (dict(head_dim=96), NOT_BUILT), (dict(dtype=2), BAD), (dict(rot_dim=136), BAD), (dict(rot_dim=24), BAD),
    (dict(rot_dim=-16), BAD), (dict(pairing=2), BAD), (dict(n_axes=0), BAD), (dict(n_axes=5), BAD), (dict(transpose=2), BAD),
    (dict(batch=1 << 20, tokens=1 << 11), NOT_BUILT), (dict(n_q_heads=65535), NOT_BUILT),
    (dict(batch=1, tokens=(1 << 27) + 1), NOT_BUILT),                    # more threads than a launch may have
    (dict(q_stride=three(102400, 12800, 64)), BAD), (dict(q_stride=three(102400, 12801, 128)), BAD),
    (dict(q_stride=three(-8, 12800, 128)), BAD), (dict(q_out_stride=three(0, 12800, 128)), BAD),
    (dict(q_out_stride=three(102400, 0, 128)), BAD),
])
def test_rotary_descriptions_are_refused(kw, code):
    assert rotate(rotary(**kw)) == code and len(B.load().aha_last_error()) > 0
    assert append(rotary(**kw), pages()) == code


def test_rotate_arguments_are_refused():
    assert rotate(None) == BAD
    assert rotate(rotary(k_out_stride=three(25600, 64, 128))) == BAD
    assert rotate(rotary(k_stride=three(25600, 12800, 120))) == BAD
    for kw in (dict(q=None), dict(q_out=None), dict(k=None), dict(k_out=None), dict(q=ODD), dict(k_out=ODD), dict(inv_freq=None),
               dict(positions=None), dict(positions=ctypes.c_void_p(0x1002)), dict(pair_axis=ctypes.c_void_p(0x1001)),
               dict(q=None, q_out=None, k=None, k_out=None)):
        assert rotate(rotary(), **kw) == BAD, kw


@pytest.mark.parametrize("kw,code", [
    (dict(n_pages=0), BAD), (dict(table_width=0), BAD), (dict(page_size=0), NOT_BUILT), (dict(page_size=48), NOT_BUILT),
    (dict(page_size=2048), NOT_BUILT), (dict(table_width=1 << 27), NOT_BUILT), (dict(reserved=1), BAD),
    (dict(k_stride=three(0, 2048, 128)), BAD), (dict(v_stride=three(4096, 0, 128)), BAD), (dict(v_stride=three(4096, 2048, 100)), BAD),
])
def test_pages_are_refused(kw, code):
    assert append(rotary(), pages(**kw)) == code
    assert attend(shared(), pages(**kw)) == code


def test_append_arguments_are_refused():
    assert append(rotary(), None) == BAD
    for kw in (dict(k=None), dict(v=None), dict(v=ODD), dict(q_out=None), dict(page_table=None), dict(tail_len=None), dict(k_pages=None),
               dict(v_pages=ODD), dict(new_len=ctypes.c_void_p(0x1002)), dict(inv_freq=None)):
        assert append(rotary(), pages(), **kw) == BAD, kw


@pytest.mark.parametrize("kw,code", [
    (dict(batch=0), BAD), (dict(q_len=0), BAD), (dict(n_q_heads=7), BAD), (dict(head_dim=256), NOT_BUILT), (dict(dtype=-1), BAD),
    (dict(n_prefixes=-1), BAD), (dict(prefix_cap=0), BAD), (dict(prefix_cap=(1 << 30) + 1), NOT_BUILT), (dict(n_prefixes=70000), NOT_BUILT),
    (dict(scale=-0.1), BAD), (dict(scale=float("nan")), BAD), (dict(scale=float("inf")), BAD), (dict(reserved=3), BAD),
    (dict(q_len=1 << 19, batch=1, n_q_heads=65535 * 8, n_kv_heads=65535), NOT_BUILT),     # likewise
    (dict(batch=40000), NOT_BUILT), (dict(q_len=1 << 23), NOT_BUILT), (dict(q_len=1 << 30, n_q_heads=1 << 20), NOT_BUILT),
])
def test_shared_descriptions_are_refused(kw, code):
    assert attend(shared(**kw), pages()) == code and len(B.load().aha_last_error()) > 0
    p, out = shared(**kw), ctypes.c_size_t()
    assert B.load().aha_shared_attention_workspace_bytes(ctypes.byref(p), None, ctypes.byref(out)) == code


def test_shared_arguments_are_refused():
    for kw in (dict(q=None), dict(out=None), dict(out=ODD), dict(k_prefix=None), dict(v_prefix=ODD), dict(prefix_len=None),
               dict(prefix_first=None), dict(k_pages=None), dict(v_pages=None), dict(page_table=None), dict(tail_len=None),
               dict(lse=ctypes.c_void_p(0x1002)), dict(new_len=ctypes.c_void_p(0x1002))):
        assert attend(shared(), pages(), **kw) == BAD, kw
    assert attend(shared(), None) == BAD                                  # tails without their description
    for kw in (dict(q_stride=three(1024, 128, 64)), dict(out_stride=three(0, 128, 128)), dict(out_stride=three(1024, 0, 128)),
               dict(k_stride=three(1, 2, 128)), dict(v_stride=three(76800, 38400, 8))):
        assert attend(shared(**kw), pages()) == BAD, kw


def test_workspace():
    p, pg, out = shared(), pages(), ctypes.c_size_t()
    lib = B.load()
    assert lib.aha_shared_attention_workspace_bytes(ctypes.byref(p), ctypes.byref(pg), None) == BAD
    assert lib.aha_shared_attention_workspace_bytes(None, None, ctypes.byref(out)) == BAD
    assert lib.aha_shared_attention_workspace_bytes(ctypes.byref(p), ctypes.byref(pg), ctypes.byref(out)) == B.AHA_OK
    need = out.value
    assert need % 256 == 0
    if need:
        assert attend(p, pg, ws=None) == WS and attend(p, pg, ws=ODD) == WS and attend(p, pg, nbytes=need - 1) == WS


def test_descriptions_of_tensors():
    q = torch.zeros(2, 8, 3, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16).transpose(1, 2)
    p = B.Rotary.of(q, k, q, k, rot_dim=32, n_axes=2)
    c = p.struct
    assert (c.batch, c.tokens, c.n_q_heads, c.n_kv_heads, c.head_dim, c.rot_dim, c.n_axes) == (2, 3, 8, 2, 64, 32, 2)
    assert list(c.k_stride) == [384, 64, 128] and list(c.q_out_stride) == [1536, 192, 64]
    pool, table = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 4, dtype=torch.int32)
    g = B.Pages.of(pool, pool, table).struct
    assert (g.n_pages, g.page_size, g.table_width) == (9, 16, 4) and list(g.v_stride) == [2048, 1024, 64]
    s = B.SharedAttention.of(q, q, pool, pool).struct
    assert (s.n_prefixes, s.prefix_cap, s.n_kv_heads, s.q_len) == (9, 16, 2, 3) and abs(s.scale - 0.125) < 1e-7
    with pytest.raises(ValueError):
        B.SharedAttention.of(q, q)
    with pytest.raises(ValueError):
        B.SharedAttention.of(q, q, pool, pool.float())
    with pytest.raises(ValueError):
        B.Rotary.of(None, None)
    with pytest.raises(ValueError):
        B.Rotary.of(q, k[:1], q)
    with pytest.raises(ValueError):
        B.Rotary.of(q, k, q.reshape(2, 3, 8, 64))
    with pytest.raises(ValueError):
        B.Rotary.of(None, k, q)
    with pytest.raises(ValueError):
        B.Rotary.of(q.transpose(2, 3), None, q)
    with pytest.raises(ValueError):
        B.Pages.of(pool, pool[:3], table)
    with pytest.raises(ValueError):
        B.rotary_tables(64, sections=[3, 4])


def test_tensors_that_are_not_the_described_ones_are_refused(monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)   # (tensors of the CPU count as the device's)
    q = torch.zeros(2, 8, 3, 64, dtype=torch.bfloat16)
    k = torch.zeros(2, 2, 3, 64, dtype=torch.bfloat16)
    pool, table = torch.zeros(9, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(2, 4, dtype=torch.int32)
    lens, pos = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 2, 3, dtype=torch.int32)
    freq = torch.zeros(32)
    p, g, s = B.Rotary.of(q, k, q, k, v=k), B.Pages.of(pool, pool, table), B.SharedAttention.of(q, q, n_kv_heads=2)
    called = []
    class Lib:
        def __getattr__(self, name):
            return lambda *a: called.append(name) or 0
    monkeypatch.setattr(B, "_lib", Lib())
    monkeypatch.setattr(B, "_stream", lambda: None)
    good_r = (q, k, freq, None, pos, q, k)
    good_a = (q, k, k, freq, None, pos, table, lens, None, q, pool, pool)
    good_s = (q, None, None, None, None, pool, pool, table, lens, lens, q, None, None)
    B.aha_rotate(p, *good_r)
    B.aha_append_paged(p, g, *good_a)
    B.aha_shared_attention(s, g, *good_s)
    assert called == ["aha_rotate", "aha_append_paged", "aha_shared_attention"]
    def refused(call, description, good, at, value):
        with pytest.raises(ValueError):
            call(*description, *good[:at], value, *good[at + 1:])
    refused(B.aha_rotate, (p,), good_r, 0, q.float())
    refused(B.aha_rotate, (p,), good_r, 4, pos.long())
    refused(B.aha_rotate, (p,), good_r, 2, freq[:16])
    refused(B.aha_append_paged, (p, g), good_a, 7, lens.long())
    refused(B.aha_append_paged, (p, g), good_a, 6, table[:1])
    refused(B.aha_append_paged, (p, g), good_a, 6, torch.zeros(2, 8, dtype=torch.int32)[:, ::2])   # a view with gaps
    refused(B.aha_append_paged, (p, g), good_a, 11, pool[:4])
    refused(B.aha_shared_attention, (s, g), good_s, 8, lens.long())
    refused(B.aha_shared_attention, (s, g), good_s, 9, lens[:1])
    refused(B.aha_shared_attention, (s, g), good_s, 11, torch.zeros(4))
    with pytest.raises(ValueError):
        B.aha_append_paged(p, B.Pages.of(pool.float(), pool.float(), table), *good_a[:10], pool.float(), pool.float())
    assert len(called) == 3

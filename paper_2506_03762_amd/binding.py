"""Thin ctypes binding of libaha.so: argument marshalling.

Every step of the eviction path runs in the HIP kernels behind the C ABI of
``include/aha.h``; the functions here take torch tensors (device memory owned
by the caller), pass their pointers and the current HIP stream, and raise
``AhaError`` on a non-zero status.  There is no fallback: if the library has
not been built, loading fails loudly.
"""
from __future__ import annotations

import ctypes
import math
import os
from dataclasses import dataclass
from typing import Optional

import torch  # must be imported before libaha.so so that both share one HIP runtime

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaha.so")

AHA_OK = 0
AHA_ERR_INVALID_ARG = -1
AHA_ERR_UNSUPPORTED = -2
AHA_ERR_WORKSPACE = -3
AHA_ERR_HIP = -4
AHA_F32, AHA_BF16 = 0, 1
AHA_SCALE_FIXED, AHA_SCALE_ADAPTIVE = 0, 1
AHA_PAIR_HALVES, AHA_PAIR_NEIGHBOURS = 0, 1

# entry points returning an int32 status first, then the two that return strings
EXPORTS = ("aha_workspace_bytes", "aha_prefill_scores", "aha_prefill_scores_lse",
           "aha_prefill_scores_rows",
           "aha_prefill_row_stats", "aha_window_attention_workspace_bytes",
           "aha_prefill_window_attention", "aha_select_topk",
           "aha_compact_kv", "aha_decode_step", "aha_decode_step_static", "aha_profile_events",
           "aha_exchange_looks", "aha_rotate", "aha_append_paged",
           "aha_shared_attention_workspace_bytes", "aha_shared_attention", "aha_last_error",
           "aha_version")


class AhaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("aha error %d: %s" % (code, msg))
        self.code = code


class aha_params(ctypes.Structure):
    _fields_ = [
        ("batch", ctypes.c_int32), ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32), ("seq_len", ctypes.c_int32), ("window", ctypes.c_int32),
        ("budget", ctypes.c_int32), ("recent", ctypes.c_int32), ("dtype", ctypes.c_int32),
        ("scale_mode", ctypes.c_int32), ("fixed_scale", ctypes.c_float),
        ("lambda_floor", ctypes.c_float), ("value_prior", ctypes.c_int32),
        ("pool_kernel", ctypes.c_int32),
        ("q_stride", ctypes.c_int64 * 3), ("k_stride", ctypes.c_int64 * 3),
        ("v_stride", ctypes.c_int64 * 3),
        ("score_pool", ctypes.c_int32), ("sink", ctypes.c_int32),
        ("decode_value_prior", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class aha_rotary(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "tokens", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "rot_dim", "pairing", "n_axes",
        "transpose")] + [(n, ctypes.c_int64 * 3) for n in (
            "q_stride", "k_stride", "v_stride", "q_out_stride", "k_out_stride")]


class aha_pages(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "table_width", "reserved")] + [
        (n, ctypes.c_int64 * 3) for n in ("k_stride", "v_stride")]


class aha_shared(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "batch", "q_len", "n_q_heads", "n_kv_heads", "head_dim", "dtype", "n_prefixes", "prefix_cap")] + [
        ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + [(n, ctypes.c_int64 * 3) for n in (
            "q_stride", "out_stride", "k_stride", "v_stride")]


_lib = None


def load() -> ctypes.CDLL:
    """Load libaha.so (built in-tree by ``build.py``); raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(
            "libaha.so is not built: run `python -m paper_2506_03762_amd.build` "
            "(or __graft_entry__.build()); there is no fallback path")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
    pp = ctypes.POINTER(aha_params)
    lib.aha_workspace_bytes.argtypes = [pp, ctypes.POINTER(sz)]
    lib.aha_prefill_scores.argtypes = [pp, vp, vp, vp, vp, vp, sz, vp]
    lib.aha_prefill_scores_lse.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.aha_prefill_scores_rows.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.aha_prefill_row_stats.argtypes = [pp, vp, vp, vp, vp, vp, sz, vp]
    lib.aha_window_attention_workspace_bytes.argtypes = [pp, ctypes.POINTER(sz)]
    lib.aha_prefill_window_attention.argtypes = [pp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.aha_select_topk.argtypes = [pp, vp, vp, vp, sz, vp]
    lib.aha_compact_kv.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp]
    lib.aha_decode_step.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, sz, vp]
    lib.aha_decode_step_static.argtypes = [pp, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    lib.aha_profile_events.argtypes = [ctypes.POINTER(vp), i32]
    lib.aha_exchange_looks.argtypes = [i32]
    rp, gp, sp = (ctypes.POINTER(t) for t in (aha_rotary, aha_pages, aha_shared))
    lib.aha_rotate.argtypes = [rp] + [vp] * 8
    lib.aha_append_paged.argtypes = [rp, gp] + [vp] * 13
    lib.aha_shared_attention_workspace_bytes.argtypes = [sp, gp, ctypes.POINTER(sz)]
    lib.aha_shared_attention.argtypes = [sp, gp] + [vp] * 13 + [sz, vp]
    for name in EXPORTS[:-2]:
        getattr(lib, name).restype = i32
    lib.aha_last_error.restype = ctypes.c_char_p
    lib.aha_version.restype = ctypes.c_char_p
    _lib = lib
    return lib


def _check(rc: int):
    if rc != AHA_OK:
        raise AhaError(rc, load().aha_last_error().decode())


def version() -> str:
    return load().aha_version().decode()


class _Built:
    """Where a Params keeps the C struct of its values: beside its fields, not among them."""
    __slots__ = ("_built",)


@dataclass
class Params(_Built):
    """Python mirror of ``aha_params`` (see include/aha.h for the meaning)."""
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    seq_len: int
    window: int
    budget: int
    recent: int
    dtype: int = AHA_BF16
    scale_mode: int = AHA_SCALE_ADAPTIVE
    fixed_scale: float = 0.0
    lambda_floor: float = -1.0
    value_prior: int = 1
    pool_kernel: int = 7
    q_stride: tuple = (0, 0, 0)
    k_stride: tuple = (0, 0, 0)
    v_stride: tuple = (0, 0, 0)
    score_pool: int = 0
    sink: int = 0
    decode_value_prior: int = 0

    def __getstate__(self):  # copies and pickles hold the fields and build their own struct
        return dict(self.__dict__)

    def c(self) -> aha_params:
        """The C struct of these values (a copy: callers may edit theirs)."""
        return aha_params.from_buffer_copy(self._struct()[0])

    def _struct(self):
        """(C struct, pointer to it) of the present values: kept beside a copy of the fields and built
        again when they differ (0.3 us to compare, 5 to build).  Strides that can change in place
        are not kept."""
        try:
            fields, built = self._built
            if fields == self.__dict__:
                return built
        except AttributeError:
            pass
        p = aha_params()
        for f in ("batch", "n_q_heads", "n_kv_heads", "head_dim", "seq_len", "window", "budget",
                  "recent", "dtype", "scale_mode", "value_prior", "pool_kernel", "score_pool",
                  "sink", "decode_value_prior"):
            setattr(p, f, int(getattr(self, f)))
        p.fixed_scale = float(self.fixed_scale)
        p.lambda_floor = float(self.lambda_floor)
        p.q_stride = (ctypes.c_int64 * 3)(*self.q_stride)
        p.k_stride = (ctypes.c_int64 * 3)(*self.k_stride)
        p.v_stride = (ctypes.c_int64 * 3)(*self.v_stride)
        built = (p, ctypes.byref(p))
        if all(isinstance(t, tuple) for t in (self.q_stride, self.k_stride, self.v_stride)):
            self._built = (dict(self.__dict__), built)
        return built

    def with_strides(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor) -> "Params":
        """Strides (batch, head, token) of [b, h, n, d] views; the d axis must be contiguous."""
        for t in (q, k, v):
            assert t.dim() == 4 and t.stride(3) == 1
        from dataclasses import replace
        return replace(self, q_stride=tuple(q.stride()[:3]), k_stride=tuple(k.stride()[:3]),
                       v_stride=tuple(v.stride()[:3]))


# Addresses go to ctypes as plain integers (the argument types convert them): with a c_void_p
# object per tensor, a torch.cuda.Stream and a copy of the parameter struct per call, a generation
# step took 8.5 us of host time to enqueue, 5.1 us without them, a prefill step's calls 25 and 15.
def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


def _stream():
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _ws(t: Optional[torch.Tensor]):
    return (None, 0) if t is None else (t.data_ptr(), t.numel())


def torch_dtype(dtype: int):
    return torch.bfloat16 if dtype == AHA_BF16 else torch.float32


def workspace_bytes(p: Params) -> int:
    out = ctypes.c_size_t(0)
    _check(load().aha_workspace_bytes(p._struct()[1], ctypes.byref(out)))
    return out.value


def alloc_workspace(p: Params, device="cuda") -> torch.Tensor:
    return torch.empty(max(workspace_bytes(p), 256), dtype=torch.uint8, device=device)


def aha_prefill_scores(p: Params, q, k, v, scores, workspace):
    """scores[b, Hkv, n] (fp32) <- refined eviction scores of q, k, v ([b, h, n, d] views)."""
    _check((_lib or load()).aha_prefill_scores(
        p._struct()[1], _ptr(q), _ptr(k), _ptr(v), _ptr(scores), *_ws(workspace), _stream()))


def aha_prefill_scores_lse(p: Params, q, k, v, lse, scores, workspace):
    """As aha_prefill_scores, with the rows' natural-log softmax denominators lse[b, Hq, window]
    (fp32) given, e.g. by the attention forward pass: the row-statistics pass is skipped."""
    _check((_lib or load()).aha_prefill_scores_lse(
        p._struct()[1], _ptr(q), _ptr(k), _ptr(v), _ptr(lse), _ptr(scores), *_ws(workspace),
        _stream()))


def aha_prefill_scores_rows(p: Params, q, k, v, rows, scores, workspace):
    """As aha_prefill_scores, accumulated over the query rows at positions rows[b, Hq, window]
    (int32) instead of the most recent ones."""
    _check((_lib or load()).aha_prefill_scores_rows(
        p._struct()[1], _ptr(q), _ptr(k), _ptr(v), _ptr(rows), _ptr(scores), *_ws(workspace),
        _stream()))


def window_attention_workspace_bytes(p: Params) -> int:
    out = ctypes.c_size_t(0)
    _check(load().aha_window_attention_workspace_bytes(p._struct()[1], ctypes.byref(out)))
    return out.value


def aha_prefill_window_attention(p: Params, q, k, v, out, lse, workspace):
    """out [b, Hq, window, d] <- causal attention output (standard scale) of the observed rows;
    lse [b, Hq, window] fp32 (or None) <- their natural-log softmax denominators."""
    _check((_lib or load()).aha_prefill_window_attention(
        p._struct()[1], _ptr(q), _ptr(k), _ptr(v), _ptr(out), _ptr(lse), *_ws(workspace),
        _stream()))


def aha_prefill_row_stats(p: Params, q, k, lse, entropy, workspace):
    """lse / entropy [b, Hq, window] (fp32, either may be None) <- natural-log normaliser and
    entropy (nats) of the observed softmax rows."""
    _check((_lib or load()).aha_prefill_row_stats(
        p._struct()[1], _ptr(q), _ptr(k), _ptr(lse), _ptr(entropy), *_ws(workspace), _stream()))


def aha_select_topk(p: Params, scores, idx, workspace=None):
    """idx[b, Hkv, budget] (int32) <- ascending retained token positions."""
    _check((_lib or load()).aha_select_topk(
        p._struct()[1], _ptr(scores), _ptr(idx), *_ws(workspace), _stream()))


def aha_compact_kv(p: Params, k, v, scores, idx, k_cache, v_cache, scores_c, pos_c, free_slot):
    _check((_lib or load()).aha_compact_kv(
        p._struct()[1], _ptr(k), _ptr(v), _ptr(scores), _ptr(idx), _ptr(k_cache), _ptr(v_cache),
        _ptr(scores_c), _ptr(pos_c), _ptr(free_slot), k_cache.size(2), _stream()))


def aha_decode_step(p: Params, q_new, k_new, v_new, k_cache, v_cache, scores_c, pos_c, free_slot,
                    logical_pos: int, out, workspace=None):
    _check((_lib or load()).aha_decode_step(
        p._struct()[1], _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache),
        _ptr(scores_c), _ptr(pos_c), _ptr(free_slot), k_cache.size(2), int(logical_pos),
        _ptr(out), *_ws(workspace), _stream()))


def aha_decode_step_static(p: Params, q_new, k_new, v_new, k_cache, v_cache, scores_c, pos_c,
                           free_slot, logical_pos: int, out):
    """aha_decode_step on the library's built-in scratch buffer (allocates nothing)."""
    _check((_lib or load()).aha_decode_step_static(
        p._struct()[1], _ptr(q_new), _ptr(k_new), _ptr(v_new), _ptr(k_cache), _ptr(v_cache),
        _ptr(scores_c), _ptr(pos_c), _ptr(free_slot), k_cache.size(2), int(logical_pos),
        _ptr(out), _stream()))


def profile_events(events=None):
    """Stage events for aha_prefill_scores: four recorded torch.cuda.Event objects
    (enable_timing=True) or None to switch the hook off."""
    if events is None:
        _check(load().aha_profile_events(None, 0))
        return
    arr = (ctypes.c_void_p * 4)(*[ctypes.c_void_p(e.cuda_event) for e in events])
    _check(load().aha_profile_events(arr, 4))


@dataclass
class CompactCache:
    """Caller-owned device buffers of the compact cache of one layer."""
    k: torch.Tensor          # [b, Hkv, slots, d]
    v: torch.Tensor          # [b, Hkv, slots, d]
    scores: torch.Tensor     # [b, Hkv, slots] fp32
    pos: torch.Tensor        # [b, Hkv, slots] int32
    free_slot: torch.Tensor  # [b, Hkv] int32

    @staticmethod
    def empty(p: Params, slots: Optional[int] = None, device="cuda") -> "CompactCache":
        slots = p.budget + 1 if slots is None else slots
        dt = torch_dtype(p.dtype)
        shp = (p.batch, p.n_kv_heads, slots)
        return CompactCache(
            torch.empty(shp + (p.head_dim,), dtype=dt, device=device),
            torch.empty(shp + (p.head_dim,), dtype=dt, device=device),
            torch.empty(shp, dtype=torch.float32, device=device),
            torch.empty(shp, dtype=torch.int32, device=device),
            torch.empty(shp[:2], dtype=torch.int32, device=device))


def default_fixed_scale(head_dim: int) -> float:
    return 1.0 / math.sqrt(head_dim)


# ---- a prompt that several sequences continue: rotation, the paged cache, attention behind shared prefixes ----
# A description is made once (its C struct is built then) and serves every call with tensors of these shapes and strides.
# The kernels address rows by the described strides alone, so each call compares shapes, strides, element types and devices:
# another layout of as many elements would be read, or written, outside its memory.  (Sizes alone cost 0.2 us of host time less
# for each tensor of rows: 64 single tokens appended 8.2 us a call, so 9.4.)

_CODES = {torch.float32: AHA_F32, torch.bfloat16: AHA_BF16}
# what has no strides of its own: element types
_DENSE = dict.fromkeys(("pair_axis", "positions", "page_table", "tail_len", "new_len", "prefix_len", "prefix_first"), torch.int32)
_DENSE.update(inv_freq=torch.float32, lse=torch.float32)


def _view(name: str, t: torch.Tensor, like: Optional[torch.Tensor] = None):
    """Strides (first three axes) of a [., heads, ., d] view whose channels are contiguous."""
    if t.dim() != 4 or (t.stride(3) != 1 and t.size(3) > 1) or t.dtype not in _CODES:
        raise ValueError("%s must be a 4-dimensional fp32 or bf16 view with contiguous channels" % name)
    if like is not None and (t.dtype != like.dtype or t.size(3) != like.size(3)):
        raise ValueError("%s has another dtype or head size" % name)
    return (ctypes.c_int64 * 3)(*t.stride()[:3])


class _Described:
    """The C struct of a description, its rows' (batch, KV heads, head size, dtype), and of its tensors, in the order
    in which a call takes them: names, element types, numbers of elements (dense ones) or shapes and strides."""

    def __init__(self, struct, rows, dtype, *tensors):
        """tensors: name and number of elements, or name and the tensor that is described (None: not given)."""
        self._as_parameter_ = ctypes.byref(struct)
        self.struct, self.rows = struct, rows
        self.tensors = tuple(
            (name, _DENSE[name], t, None, None) if name in _DENSE else
            (name, dtype, None, (), ()) if t is None else (name, dtype, None, t.shape, t.stride())
            for name, t in tensors)


def _same_places(t, shape, stride):
    """Whether t's elements lie as described: axes of one element have any stride, or are left out."""
    return [x for x in zip(t.shape, t.stride()) if x[0] != 1] == [x for x in zip(shape, stride) if x[0] != 1]


def _pointers(tensors, given):
    """The given tensors' addresses, once they are what the description says."""
    device, out = torch._C._cuda_getDevice(), []
    for (name, dtype, n, shape, stride), t in zip(tensors, given):
        if t is None:
            out.append(None)
            continue
        if shape is None:
            if t.dtype is not dtype or t.numel() != n or t.get_device() != device or not t.is_contiguous():
                raise ValueError("%s: not a contiguous tensor of %d elements of %s on the current device" % (name, n, dtype))
        elif t.dtype is not dtype or t.get_device() != device or (
                (t.stride() != stride or t.shape != shape) and not (shape and _same_places(t, shape, stride))):
            raise ValueError("%s: not a tensor of %s on the current device with the described shape %s and strides %s" % (
                name, dtype, tuple(shape), stride) if shape else "%s is given, but not described" % name)
        out.append(t.data_ptr())
    return out


class Rotary(_Described):
    """Description of a rotation (aha_rotary of include/aha.h)."""

    @classmethod
    def of(cls, q, k, q_out=None, k_out=None, v=None, *, rot_dim: Optional[int] = None, n_axes: int = 1,
           pairing: int = AHA_PAIR_HALVES, transpose: int = 0) -> "Rotary":
        """For q [b, Hq, n, d] and k [b, Hkv, n, d] views (either may be None), what they are turned into and,
        to append, the values."""
        given = k if k is not None else q
        if given is None:
            raise ValueError("q and k are both None")
        p = aha_rotary(batch=given.size(0), tokens=given.size(2), head_dim=given.size(3), pairing=pairing,
                       n_q_heads=1 if q is None else q.size(1), n_kv_heads=1 if k is None else k.size(1),
                       dtype=_CODES.get(given.dtype, -1), n_axes=n_axes, transpose=transpose,
                       rot_dim=given.size(3) if rot_dim is None else rot_dim)
        for name, t in (("q", q), ("k", k), ("v", v), ("q_out", q_out), ("k_out", k_out)):
            if t is not None:
                setattr(p, name + "_stride", _view(name, t, given))
        if any(t is not None and (x is None or t.shape != x.shape) for t, x in ((q_out, q), (k_out, k), (v, k))):
            raise ValueError("q_out, or k_out or v, has another shape than q, or k")
        if q is not None and k is not None and (q.size(0), q.size(2)) != (k.size(0), k.size(2)):
            raise ValueError("q and k have other batches or tokens")
        self = cls(p, (p.batch, p.n_kv_heads, p.head_dim, given.dtype), given.dtype, ("q", q), ("k", k),
                   ("inv_freq", p.rot_dim // 2), ("pair_axis", p.rot_dim // 2),
                   ("positions", p.n_axes * p.batch * p.tokens), ("q_out", q_out), ("k_out", k_out), ("v", v))
        q, k, freq, axis, pos, q_out, k_out, v = self.tensors
        self.tensors = (q, k, freq, axis, pos, q_out, k_out)
        self.appended = (q, k, v, freq, axis, pos, q_out)
        return self


class Pages(_Described):
    """Description of a paged cache (aha_pages)."""

    @classmethod
    def of(cls, k_pages, v_pages, page_table) -> "Pages":
        """For pools [pages, Hkv, page size, d] (views by stride) and a table [b, width]."""
        p = aha_pages(n_pages=k_pages.size(0), page_size=k_pages.size(2), table_width=page_table.size(1),
                      k_stride=_view("k_pages", k_pages), v_stride=_view("v_pages", v_pages, k_pages))
        if k_pages.shape != v_pages.shape:
            raise ValueError("the pools have different shapes")
        batch = page_table.size(0)
        return cls(p, (batch, k_pages.size(1), k_pages.size(3), k_pages.dtype), k_pages.dtype,
                   ("k_pages", k_pages), ("v_pages", v_pages), ("page_table", page_table.numel()), ("tail_len", batch),
                   ("new_len", batch))


class SharedAttention(_Described):
    """Description of an attention behind shared prefixes (aha_shared)."""

    @classmethod
    def of(cls, q, out, k_prefix=None, v_prefix=None, scale: Optional[float] = None, *, n_kv_heads: Optional[int] = None
           ) -> "SharedAttention":
        """For q and out [b, Hq, n, d] and the prefixes [prefixes, Hkv, capacity, d] (None: none; the number of KV
        heads then has to be given).  scale None: 1 / sqrt(d)."""
        if k_prefix is None and n_kv_heads is None:
            raise ValueError("neither prefixes nor n_kv_heads are given")
        if (k_prefix is None) != (v_prefix is None):
            raise ValueError("k_prefix and v_prefix must both be given or both be None")
        p = aha_shared(batch=q.size(0), q_len=q.size(2), n_q_heads=q.size(1), head_dim=q.size(3),
                       n_kv_heads=n_kv_heads if k_prefix is None else k_prefix.size(1),
                       dtype=_CODES.get(q.dtype, -1), scale=default_fixed_scale(q.size(3)) if scale is None else scale,
                       q_stride=_view("q", q), out_stride=_view("out", out, q))
        if q.shape != out.shape or (k_prefix is not None and k_prefix.shape != v_prefix.shape):
            raise ValueError("q and out, or the prefixes' keys and values, have different shapes")
        if k_prefix is not None:
            p.n_prefixes, p.prefix_cap = k_prefix.size(0), k_prefix.size(2)
            p.k_stride, p.v_stride = _view("k_prefix", k_prefix, q), _view("v_prefix", v_prefix, q)
        return cls(p, (p.batch, p.n_kv_heads, p.head_dim, q.dtype), q.dtype, ("q", q),
                   ("k_prefix", k_prefix), ("v_prefix", v_prefix),
                   ("prefix_len", p.n_prefixes), ("prefix_first", p.n_prefixes + 1),
                   ("new_len", p.batch), ("out", out), ("lse", q.numel() // p.head_dim))


def rotary_tables(rot_dim: int, base: float = 10000.0, sections=None, device="cuda"):
    """(inv_freq, pair_axis) of rot_dim / 2 pairs: base^(-2 f / rot_dim) radians per position, and the axis that
    turns each pair: None, or runs of sections[a] pairs for axis a."""
    if sections is not None and sum(sections) != rot_dim // 2:
        raise ValueError("sections must add up to rot_dim / 2 pairs")
    f = torch.arange(rot_dim // 2, dtype=torch.float64)
    inv_freq = (base ** (-2.0 * f / max(1, rot_dim))).float().to(device)
    if sections is None:
        return inv_freq, None
    axis = [a for a, n in enumerate(sections) for _ in range(n)]
    return inv_freq, torch.tensor(axis, dtype=torch.int32, device=device)


def aha_rotate(p: Rotary, q, k, inv_freq, pair_axis, positions, q_out, k_out):
    """q_out, k_out <- the rows of q, k turned by positions [axes, b, n] (int32)."""
    at = _pointers(p.tensors, (q, k, inv_freq, pair_axis, positions, q_out, k_out))
    _check((_lib or load()).aha_rotate(p, *at, _stream()))


def aha_append_paged(p: Rotary, cache: Pages, q, k, v, inv_freq, pair_axis, positions, page_table, tail_len, new_len,
                     q_out, k_pages, v_pages):
    """The new tokens' keys (turned) and values into their places of the pools; q_out <- q turned."""
    _check_same(p, cache)
    at = _pointers(p.appended + cache.tensors, (q, k, v, inv_freq, pair_axis, positions, q_out, k_pages, v_pages,
                                                page_table, tail_len, new_len))
    _check((_lib or load()).aha_append_paged(p, cache, *at[:6], *at[9:], *at[6:9], _stream()))


def _check_same(p, cache: Pages):
    """The rows' batch, KV heads, head size and element type are the cache's."""
    if cache.rows != p.rows:
        raise ValueError("the cache is one of %s (batch, KV heads, head size, dtype), the rows are of %s" % (cache.rows, p.rows))


def shared_attention_workspace_bytes(p: SharedAttention, cache: Optional[Pages]) -> int:
    out = ctypes.c_size_t(0)
    _check(load().aha_shared_attention_workspace_bytes(p, cache, ctypes.byref(out)))
    return out.value


def alloc_shared_workspace(p: SharedAttention, cache: Optional[Pages], device="cuda") -> torch.Tensor:
    return torch.empty(max(shared_attention_workspace_bytes(p, cache), 256), dtype=torch.uint8, device=device)


def aha_shared_attention(p: SharedAttention, cache: Optional[Pages], q, k_prefix, v_prefix, prefix_len, prefix_first,
                         k_pages, v_pages, page_table, tail_len, new_len, out, lse, workspace):
    """out [b, Hq, n, d], lse [b, Hq, n] (fp32 or None) <- attention of the new tokens over their shared prefix
    and their own tail."""
    expected, given = p.tensors, (q, k_prefix, v_prefix, prefix_len, prefix_first, new_len, out, lse)
    if cache is not None:
        _check_same(p, cache)
        expected, given = expected + cache.tensors[:4], given + (k_pages, v_pages, page_table, tail_len)
    at = _pointers(expected, given)
    if workspace is not None and (workspace.get_device() != torch._C._cuda_getDevice() or not workspace.is_contiguous()):
        raise ValueError("workspace: not a contiguous tensor on the current device")
    tails = at[8:] if cache is not None else [_ptr(t) for t in (k_pages, v_pages, page_table, tail_len)]
    _check((_lib or load()).aha_shared_attention(p, cache, *at[:5], *tails, *at[5:8], *_ws(workspace), _stream()))

"""Python binding of the paged 8-bit K/V cache and of the rotary positions (the second half of ``include/sage.h``, which says what each
call computes).  Argument marshalling only, as in the package itself.

A serving loop::

    pages = PageTable.empty(n_pages, page_tokens=128, slots=64, width=256)
    layers = [PagedCache.empty(pages, Hkv, d, torch.bfloat16) for _ in range(n_layers)]
    sage_pages_reserve(pages, n_new, slots)                     # room for the step's tokens, lengths included
    for cache in layers:
        q = sage_rope(q, positions, plan)
        sage_paged_append(cache, k, v, q_start=q_start, slots=slots, rope=plan)
        out = sage_attn_fwd_paged(q, cache, causal=True, max_len=longest, q_start=q_start, slots=slots)
"""
from __future__ import annotations

import ctypes

import torch

import paper_2505_21136_amd as _sage

FORMATS = {"int8": 0, "e4m3": 1}
LAYOUTS = {"half": 0, "interleaved": 1}
SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "yarn": 3, "bands": 4}
BLOCK, TAIL, MAX_SLOTS = 64, 128, 4096


class _RopePlan(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_uint64 * 64), ("magnitude", ctypes.c_float), ("rot", ctypes.c_int), ("layout", ctypes.c_int)]


class _PageTable(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p), ("slots", ctypes.c_int),
                ("width", ctypes.c_int), ("n_pages", ctypes.c_int), ("page_tokens", ctypes.c_int)]


class _Cache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("k_tail", ctypes.c_void_p), ("v_tail", ctypes.c_void_p), ("k_shift", ctypes.c_void_p), ("Hkv", ctypes.c_int),
                ("d", ctypes.c_int), ("fmt", ctypes.c_int), ("dt", ctypes.c_int)]


def declare(L) -> None:
    i, f, vp, sz, db = ctypes.c_int, ctypes.c_float, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_double
    for name, result, args in (
            ("sage_rope_init", i, [vp, i, i, i, db, db, i, db, db, db]),
            ("sage_rope", i, [vp, vp, vp, vp, vp, i, i, i, i, vp, vp, vp, vp, vp, i, i, vp]),
            ("sage_paged_append", i, [vp, vp, vp, vp, vp, vp, vp, vp, i, i, vp, vp]),
            ("sage_paged_gather", i, [vp, vp, vp, vp, vp, vp, i, i, vp]),
            ("sage_paged_split_keys", i, [i, i, i, i, i]),
            ("sage_paged_workspace_bytes", sz, [i, i, i, i, i, i, i]),
            ("sage_attn_fwd_paged", i, [vp, vp, vp, vp, vp, vp, vp, vp, i, i, i, i, i, f, i, vp, vp, sz]),
            ("sage_pages_reserve", i, [vp, vp, vp, i, vp, vp]),
            ("sage_pages_fork", i, [vp, vp, vp, i, vp, vp, vp, vp]),
            ("sage_pages_free", i, [vp, vp, i, vp]),
            ("sage_pages_compact_workspace_bytes", sz, [i]),
            ("sage_pages_compact", i, [vp, vp, i, vp, vp, vp, sz]),
            ("sage_pages_copy", i, [vp, vp, vp, i, vp, i, vp])):
        fn = getattr(L, name)
        fn.restype, fn.argtypes = result, args


_TwoStrides = ctypes.c_int64 * 2


def _current() -> int:
    return _sage._current_device() if _sage._current_device is not None else torch.cuda.current_device()


def _here(t: torch.Tensor, what: str) -> None:
    """A device tensor of the current device: the launches go to the current stream of that device."""
    device = t.get_device()
    if device < 0:
        raise _sage.SageError(f"{what}: libsage needs device tensors (no CPU path exists)")
    if device != _current():
        raise _sage.SageError(f"{what} is on device {device}, the current device is {_current()}")


def _ours(pages: "PageTable") -> None:
    """The table, and with it the caches over it, lives on the device that the launches go to."""
    if pages.device_index != _current():
        raise _sage.SageError(f"the page table is on device {pages.device_index}, the current device is {_current()}")


def _room(t: torch.Tensor) -> int:
    """The bytes of a caller's workspace."""
    if not t.is_contiguous():
        raise _sage.SageError("workspace must be contiguous: its bytes are counted from its first one on")
    _here(t, "workspace")
    return t.numel() * t.element_size()


def _ints(t: torch.Tensor | None, what: str, n: int | None = None) -> int | None:
    """The address of a contiguous int32 list (of n entries)."""
    if t is None:
        return None
    if t.dtype != torch.int32 or t.dim() != 1 or not t.is_contiguous():
        raise _sage.SageError(f"{what} must be a contiguous one-dimensional int32 tensor")
    if n is not None and t.numel() != n:
        raise _sage.SageError(f"{what} must have {n} entries, not {t.numel()}")
    _here(t, what)
    return t.data_ptr()


def _rows(t: torch.Tensor, what: str):
    """[T, H, d] with contiguous channels -> the {token, head} element strides, None where contiguous."""
    st = t.stride()
    if len(st) != 3 or st[2] != 1:
        raise _sage.SageError(f"{what} must be [T, H, d] with a contiguous channel dimension")
    _here(t, what)
    if t.is_contiguous():
        return None
    T, H, _ = t.shape
    return _TwoStrides(st[0] if T > 1 else 0, st[1] if H > 1 else 0)


def rope_plan(rot: int, *, base: float = 10000.0, layout: str = "half", scaling: str = "none", factor: float = 1.0, trained_len: int = 0,
              low: float | None = None, high: float | None = None, magnitude: float = 0.0) -> _RopePlan:
    """A plan for sage_rope and sage_paged_append: `rot` channels turn, paired by ``layout`` ('half', 'interleaved'), with ``scaling`` 'none',
    'linear', 'ntk', 'yarn' (low, high: 1, 32) or 'bands' (1, 4).  Host work only: made once."""
    if layout not in LAYOUTS or scaling not in SCALINGS:
        raise _sage.SageError(f"layout is one of {sorted(LAYOUTS)}, scaling one of {sorted(SCALINGS)}")
    plan = _RopePlan()
    _sage._check(_sage.lib().sage_rope_init(
        ctypes.byref(plan), int(rot), LAYOUTS[layout], SCALINGS[scaling], float(base), float(factor), int(trained_len),
        float(1.0 if low is None else low), float((32.0 if scaling == "yarn" else 4.0) if high is None else high), float(magnitude)))
    return plan


def sage_rope(q: torch.Tensor, positions: torch.Tensor, plan: _RopePlan, *, k: torch.Tensor | None = None, transposed: bool = False,
              out: torch.Tensor | None = None, k_out: torch.Tensor | None = None):
    """Rotary positions of q [T, Hq, d] and, in the same launch, k [T, Hkv, d] (any views with contiguous channels): -> out, or (out, k_out).
    out = q and k_out = k rotate in place.  Autograd is not told: the gradient of out is turned back by a call with ``transposed``."""
    qs, (T, Hq, d), Hkv = _rows(q, "q"), q.shape, 0
    qos = ks = kos = None
    if out is None:
        out = torch.empty_like(q) if qs is None else q.new_empty((T, Hq, d))
    else:
        qos = _rows(out, "out")
        if out.shape != q.shape or out.dtype != q.dtype:
            raise _sage.SageError("out must have q's shape and dtype")
    if k is not None:
        ks, Hkv = _rows(k, "k"), k.shape[1]
        if k.shape != (T, Hkv, d) or k.dtype != q.dtype:
            raise _sage.SageError("k must be [T, Hkv, d] of q's dtype")
        if k_out is None:
            k_out = torch.empty_like(k) if ks is None else k.new_empty((T, Hkv, d))
        else:
            kos = _rows(k_out, "k_out")
            if k_out.shape != k.shape or k_out.dtype != k.dtype:
                raise _sage.SageError("k_out must have k's shape and dtype")
    elif k_out is not None:
        raise _sage.SageError("k_out without k")
    _sage._check(_sage.lib().sage_rope(
        q.data_ptr(), out.data_ptr(), None if k is None else k.data_ptr(), None if k is None else k_out.data_ptr(),
        _ints(positions, "positions", T), T, Hq, Hkv, d, qs, qos, ks, kos, ctypes.byref(plan), int(transposed), _sage._dt(q),
        _sage._stream()))
    return out if k is None else (out, k_out)


class _Handle:
    """Attributes are set once: the calls go by the addresses and sizes that the handle was made with, and its tensors keep that memory alive.  What
    the tensors hold is changed in place."""

    def __setattr__(self, name, value):
        if self.__dict__.get(name, value) is not value:
            raise _sage.SageError(f"{type(self).__name__}.{name} is set when the handle is made: change a tensor in place (copy_, sub_, [...] =), "
                                  "or make another handle")
        super().__setattr__(name, value)

    def __delattr__(self, name):
        raise _sage.SageError(f"{type(self).__name__}.{name} belongs to the handle as long as it lives")


class PageTable(_Handle):
    """Which pages belong to which slot: table int32 [slots, width] (-1: none), lens int32 [slots], refs int32 [n_pages].  The caches of all
    layers share one.  The tensors' values may be changed, in place (drafted tokens are taken back by ``pages.lens.sub_(n)``); the tensors stay."""

    def __init__(self, *, table: torch.Tensor, lens: torch.Tensor, refs: torch.Tensor, page_tokens: int):
        if table.dim() != 2 or table.dtype != torch.int32 or not table.is_contiguous():
            raise _sage.SageError("table must be a contiguous int32 [slots, width] tensor")
        self.slots, self.width = table.shape
        _here(table, "table")
        self.table, self.lens, self.refs, self.page_tokens, self.n_pages = table, lens, refs, int(page_tokens), refs.numel()
        self._c = _PageTable(table.data_ptr(), _ints(lens, "lens", self.slots), _ints(refs, "refs"), self.slots, self.width, self.n_pages,
                             self.page_tokens)
        self.ref = ctypes.byref(self._c)
        self.device_index = table.get_device()

    @classmethod
    def empty(cls, n_pages: int, *, page_tokens: int, slots: int, width: int, device="cuda") -> "PageTable":
        return cls(table=torch.full((slots, width), -1, dtype=torch.int32, device=device),
                   lens=torch.zeros(slots, dtype=torch.int32, device=device), refs=torch.zeros(n_pages, dtype=torch.int32, device=device),
                   page_tokens=page_tokens)


class PagedCache(_Handle):
    """The 8-bit K/V cache of one layer: k, v uint8 [n_pages, Hkv, page_tokens / 64, 64 * d], k_scale, v_scale float32 [n_pages, Hkv,
    page_tokens / 64], k_tail, v_tail [slots, Hkv, 128, d] in 16 bits, k_shift float32 [Hkv, d] or None; fmt 'int8' or 'e4m3'."""

    def __init__(self, pages: PageTable, *, k, v, k_scale, v_scale, k_tail, v_tail, fmt: str = "int8", k_shift: torch.Tensor | None = None):
        if fmt not in FORMATS:
            raise _sage.SageError(f"fmt is one of {sorted(FORMATS)}")
        _ours(pages)
        if k_tail.dim() != 4:
            raise _sage.SageError("k_tail must be [slots, Hkv, 128, d]")
        Hkv, d = k_tail.shape[1], k_tail.shape[3]
        per = pages.page_tokens // BLOCK
        for name, t, shape, dtype in (("k", k, (pages.n_pages, Hkv, per, BLOCK * d), torch.uint8), ("v", v, (pages.n_pages, Hkv, per, BLOCK * d), torch.uint8),
                                      ("k_scale", k_scale, (pages.n_pages, Hkv, per), torch.float32),
                                      ("v_scale", v_scale, (pages.n_pages, Hkv, per), torch.float32),
                                      ("k_tail", k_tail, (pages.slots, Hkv, TAIL, d), k_tail.dtype), ("v_tail", v_tail, (pages.slots, Hkv, TAIL, d), k_tail.dtype),
                                      ("k_shift", k_shift, (Hkv, d), torch.float32)):
            if t is None and name == "k_shift":
                continue
            if tuple(t.shape) != shape or t.dtype != dtype or not t.is_contiguous():
                raise _sage.SageError(f"{name} must be a contiguous {dtype} tensor of shape {shape}")
            _here(t, name)
        self.pages, self.k, self.v, self.k_scale, self.v_scale, self.k_tail, self.v_tail, self.k_shift = pages, k, v, k_scale, v_scale, k_tail, v_tail, k_shift
        self.Hkv, self.d, self.fmt, self.dtype = Hkv, d, fmt, k_tail.dtype
        self._c = _Cache(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), k_tail.data_ptr(), v_tail.data_ptr(),
                         None if k_shift is None else k_shift.data_ptr(), Hkv, d, FORMATS[fmt], _sage._dt(k_tail))
        self.ref = ctypes.byref(self._c)

    @classmethod
    def empty(cls, pages: PageTable, Hkv: int, d: int, dtype: torch.dtype, *, fmt: str = "int8", k_shift: torch.Tensor | None = None) -> "PagedCache":
        dev, per = pages.table.device, pages.page_tokens // BLOCK

        def codes():
            return torch.empty((pages.n_pages, Hkv, per, BLOCK * d), dtype=torch.uint8, device=dev)

        def scales():
            return torch.empty((pages.n_pages, Hkv, per), dtype=torch.float32, device=dev)

        def tail():
            return torch.empty((pages.slots, Hkv, TAIL, d), dtype=dtype, device=dev)

        return cls(pages, k=codes(), v=codes(), k_scale=scales(), v_scale=scales(), k_tail=tail(), v_tail=tail(), fmt=fmt, k_shift=k_shift)


def _batch(cache: PagedCache, q_start, slots, what: str) -> int:
    """The number of sequences of a call."""
    if q_start is not None:
        if q_start.numel() < 2:
            raise _sage.SageError(f"{what} must have an entry per sequence and one more")
        return q_start.numel() - 1
    return slots.numel() if slots is not None else cache.pages.slots


def _of_cache(t: torch.Tensor, cache: PagedCache, what: str, heads: int | None = None):
    s = _rows(t, what)
    if t.dtype != cache.dtype or t.shape[2] != cache.d or (heads is not None and t.shape[1] != heads):
        raise _sage.SageError(f"{what} must be [T, {'H' if heads is None else heads}, {cache.d}] of {cache.dtype}")
    return s


def sage_paged_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, *, q_start: torch.Tensor | None = None,
                      slots: torch.Tensor | None = None, rope: _RopePlan | None = None) -> None:
    """Append k, v [T, Hkv, d] (views with contiguous channels) as the last tokens of their sequences, whose lengths (cache.pages.lens)
    cover them already.  q_start int32 [B + 1], or None for T / B tokens each; slots int32 [B], or None for slot b."""
    ks, vs = _of_cache(k, cache, "k", cache.Hkv), _of_cache(v, cache, "v", cache.Hkv)
    if k.shape != v.shape:
        raise _sage.SageError("k and v must have one shape")
    _ours(cache.pages)
    B = _batch(cache, q_start, slots, "q_start")
    _sage._check(_sage.lib().sage_paged_append(
        cache.pages.ref, cache.ref, k.data_ptr(), v.data_ptr(), ks, vs, _ints(q_start, "q_start"), _ints(slots, "slots", B), B, k.shape[0],
        None if rope is None else ctypes.byref(rope), _sage._stream()))


def sage_paged_gather(cache: PagedCache, k_start: torch.Tensor, total: int, *, slots: torch.Tensor | None = None):
    """The tokens of sequence b as rows k_start[b] .. k_start[b + 1] - 1 of (k, v), [total, Hkv, d] in 16 bits; rows of no sequence are
    left unwritten."""
    _ours(cache.pages)
    B = _batch(cache, k_start, slots, "k_start")
    k = cache.k_tail.new_empty((total, cache.Hkv, cache.d))
    v = cache.k_tail.new_empty((total, cache.Hkv, cache.d))
    _sage._check(_sage.lib().sage_paged_gather(cache.pages.ref, cache.ref, k.data_ptr(), v.data_ptr(), _ints(k_start, "k_start"),
                                               _ints(slots, "slots", B), B, int(total), _sage._stream()))
    return k, v


def paged_split_keys(T: int, B: int, Hq: int, Hkv: int, max_len: int) -> int:
    """Tokens per range that sage_attn_fwd_paged uses for split_keys = 0."""
    return int(_sage.lib().sage_paged_split_keys(T, B, Hq, Hkv, max_len))


def paged_workspace_bytes(T: int, B: int, Hq: int, Hkv: int, d: int, max_len: int, split_keys: int = 0) -> int:
    """Workspace of sage_attn_fwd_paged (0: none)."""
    return int(_sage.lib().sage_paged_workspace_bytes(T, B, Hq, Hkv, d, max_len, split_keys))


def sage_attn_fwd_paged(q: torch.Tensor, cache: PagedCache, *, causal: bool, max_len: int, q_start: torch.Tensor | None = None,
                        slots: torch.Tensor | None = None, sm_scale: float = 0.0, split_keys: int = 0, out: torch.Tensor | None = None,
                        workspace: torch.Tensor | None = None) -> torch.Tensor:
    """Attention of q [T, Hq, d] (views with contiguous channels) over the cached tokens of each row's sequence.  q_start int32 [B + 1], or None
    for T / B rows each; slots int32 [B], or None for slot b; max_len: the longest sequence expected."""
    qs = _of_cache(q, cache, "q")
    T, Hq, d = q.shape
    os_ = None
    if out is None:
        out = torch.empty_like(q) if qs is None else q.new_empty((T, Hq, d))
    else:
        os_ = _of_cache(out, cache, "out")
        if out.shape != q.shape:
            raise _sage.SageError("out must have q's shape")
    _ours(cache.pages)
    B = _batch(cache, q_start, slots, "q_start")
    if workspace is None:
        workspace = _sage._workspace(paged_workspace_bytes(T, B, Hq, cache.Hkv, d, max_len, split_keys), q.device)
    room = _room(workspace)
    _sage._check(_sage.lib().sage_attn_fwd_paged(
        q.data_ptr(), out.data_ptr(), qs, os_, cache.pages.ref, cache.ref, _ints(q_start, "q_start"), _ints(slots, "slots", B), B, T, Hq,
        int(max_len), int(causal), float(sm_scale), int(split_keys), _sage._stream(), workspace.data_ptr(), room))
    return out


def sage_pages_reserve(pages: PageTable, n_new: torch.Tensor | None = None, slots: torch.Tensor | None = None) -> torch.Tensor:
    """n_new[i] more tokens (int32, or None: 1 each) for slots[i] (None: all slots): -> status int32, 0 or -1 (refused)."""
    _ours(pages)
    if slots is None:
        slots = torch.arange(pages.slots, dtype=torch.int32, device=pages.table.device)
    at, n = _ints(slots, "slots"), slots.numel()
    status = slots.new_empty(n)
    _sage._check(_sage.lib().sage_pages_reserve(pages.ref, at, _ints(n_new, "n_new", n), n, status.data_ptr(), _sage._stream()))
    return status


def sage_pages_fork(pages: PageTable, src: torch.Tensor, dst: torch.Tensor):
    """Slot dst[i] becomes a copy of slot src[i]: -> (status [n], page_moves [n, 2], slot_moves [n, 2]); sage_pages_copy then copies in
    each layer's cache."""
    _ours(pages)
    at, n = _ints(src, "src"), src.numel()
    status, moves = src.new_empty(n), src.new_empty((2, n, 2))
    p = moves.data_ptr()
    _sage._check(_sage.lib().sage_pages_fork(pages.ref, at, _ints(dst, "dst", n), n, status.data_ptr(), p, p + 8 * n, _sage._stream()))
    return (status, *moves.unbind())


def sage_pages_free(pages: PageTable, slots: torch.Tensor) -> None:
    """The listed slots' pages are given back; the slots are empty afterwards."""
    _ours(pages)
    _sage._check(_sage.lib().sage_pages_free(pages.ref, _ints(slots, "slots"), slots.numel(), _sage._stream()))


def sage_pages_compact(pages: PageTable, max_moves: int | None = None, *, workspace: torch.Tensor | None = None):
    """Live pages move to the front of the pool: -> (page_moves [max_moves, 2], counts [2] = {live pages, moves}); sage_pages_copy then
    copies in each layer's cache."""
    most = max(1, pages.n_pages // 2) if max_moves is None else int(max_moves)
    _ours(pages)
    moves, counts = pages.refs.new_empty((max(most, 0), 2)), pages.refs.new_empty(2)
    ws = workspace if workspace is not None else pages.refs.new_empty((pages.n_pages + 63) // 64 * 64)
    room = _room(ws)
    _sage._check(_sage.lib().sage_pages_compact(pages.ref, moves.data_ptr(), most, counts.data_ptr(), _sage._stream(), ws.data_ptr(), room))
    return moves, counts


def _moves(t: torch.Tensor | None, what: str):
    if t is None:
        return None, 0
    if t.dtype != torch.int32 or t.dim() != 2 or t.shape[1] != 2 or not t.is_contiguous():
        raise _sage.SageError(f"{what} must be a contiguous int32 [n, 2] tensor")
    _here(t, what)
    return t.data_ptr(), t.shape[0]


def sage_pages_copy(cache: PagedCache, page_moves: torch.Tensor | None, slot_moves: torch.Tensor | None = None) -> None:
    """Carry out the moves of sage_pages_fork or sage_pages_compact in one layer's cache."""
    pm, n = _moves(page_moves, "page_moves")
    sm, ns = _moves(slot_moves, "slot_moves")
    _ours(cache.pages)
    _sage._check(_sage.lib().sage_pages_copy(cache.pages.ref, cache.ref, pm, n, sm, ns, _sage._stream()))

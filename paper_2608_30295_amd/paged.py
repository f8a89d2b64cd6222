"""Python binding of include/catekv_paged.h: caches held in pages of one pool,
attention of several new tokens per sequence over them, and forking, dropping,
compacting and gathering their rows.

As in ``binding.py`` only arguments are marshalled here; every step runs in
``libcatekv.so``.  A ``PagedCache`` holds the tensors whose addresses its handle
passes on, and ``gather_kv_paged`` takes a table from ``kv_table``, whose tensors
must outlive its use.
"""
from __future__ import annotations

import ctypes
import math
import operator
from array import array
from dataclasses import dataclass, field
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from . import _lib
from ._lib import check, lib
from .binding import D, _dtype_code, workspace
from .cache import _bytes, _call, _device_of, _need, _need_table

PAGES = (16, 32, 64, 128, 256)


def _ints(x: Sequence[int]):
    """int32 values for a host argument (slot lists are long: the array is filled in C)."""
    a = array("i", x)
    return (ctypes.c_int32 * len(a)).from_buffer(a) if a else (ctypes.c_int32 * 1)()


@dataclass
class PagedCache:
    """A cache in pages: k, v [n_pages][page][128] (bfloat16 or float32), table int32
    [n_slots][hkv][max_pages], lens int64 [n_slots][hkv], refs int32 [n_pages] and
    free_bits int64 [ceil(n_pages / 64)], all on one GPU and contiguous; what they
    hold is described in include/catekv_paged.h.  ``paged_alloc`` makes an empty one.
    `book`: the tensor that the last four are parts of, if they are (saving and
    restoring it takes one copy)."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    lens: torch.Tensor
    refs: torch.Tensor
    free_bits: torch.Tensor
    book: Optional[torch.Tensor] = None
    handle: _lib.PagedCacheT = field(init=False, repr=False)

    def __post_init__(self) -> None:
        if self.k.dim() != 3 or self.k.shape[2] != D or self.v.shape != self.k.shape or self.v.dtype != self.k.dtype:
            raise ValueError(f"k and v must be [n_pages][page][{D}] of one type")
        if self.table.dim() != 3:
            raise ValueError("table must be [n_slots][hkv][max_pages]")
        self.n_pages, self.page = self.k.shape[:2]
        self.n_slots, self.hkv, self.max_pages = self.table.shape
        if self.page not in PAGES:
            raise ValueError(f"pages of {self.page} rows (16, 32, 64, 128 or 256)")
        _need(self.table, "table", torch.int32, self.table.numel())
        _need(self.lens, "lens", torch.int64, self.n_slots * self.hkv)
        _need(self.refs, "refs", torch.int32, self.n_pages)
        _need(self.free_bits, "free_bits", torch.int64, -(-self.n_pages // 64))
        dtype = _dtype_code(self.k)
        self.index = _device_of(self.k, self.v, self.table, self.lens, self.refs, self.free_bits)
        self.handle = _lib.PagedCacheT(self.k.data_ptr(), self.v.data_ptr(), self.table.data_ptr(), self.lens.data_ptr(),
                                       self.refs.data_ptr(), self.free_bits.data_ptr(), dtype, self.page, self.n_pages,
                                       self.n_slots, self.hkv, self.max_pages)
        self.ref = ctypes.byref(self.handle)

    @property
    def dtype(self) -> torch.dtype:
        return self.k.dtype

    @property
    def device(self) -> torch.device:
        return self.k.device


def paged_alloc(n_pages: int, page: int, n_slots: int, hkv: int, max_pages: int, device, *,
                dtype: torch.dtype) -> PagedCache:
    """An empty cache: n_pages pages of `page` rows, n_slots sequences of hkv views
    of at most max_pages pages each."""
    if min(n_pages, page, n_slots, hkv, max_pages) < 1:
        raise ValueError("sizes must be >= 1")
    k, v = (torch.empty((n_pages, page, D), dtype=dtype, device=device) for _ in "kv")
    sizes = [n_slots * hkv, -(-n_pages // 64), -(-n_pages // 2), -(-n_slots * hkv * max_pages // 2)]
    book = torch.empty(sum(sizes), dtype=torch.int64, device=device)
    lens, bits, refs, table = book.split(sizes)
    cache = PagedCache(k, v, table.view(torch.int32)[:n_slots * hkv * max_pages].view(n_slots, hkv, max_pages),
                       lens.view(n_slots, hkv), refs.view(torch.int32)[:n_pages], bits, book)
    _call(cache.index, lib().catekv_paged_init, cache.ref)
    return cache


@dataclass
class PagedPlan:
    plan: _lib.PagedPlanT
    ws: torch.Tensor
    n_tokens: int
    hq: int
    hkv: int

    def __post_init__(self) -> None:
        self.ref = ctypes.byref(self.plan)


def _whole(x, dtype, name: str) -> np.ndarray:
    """The whole numbers of x, flat; what the type does not hold is refused, not cut."""
    a = np.asarray(x)
    if a.dtype.kind == "O":                          # single tensors, or Python's long numbers
        a = np.array([operator.index(i) for i in a.ravel()], dtype=object)
    elif a.size and a.dtype.kind not in "iu":
        raise TypeError(f"{name} must be whole numbers, not {a.dtype}")
    try:
        b = a.astype(dtype, copy=False)
    except OverflowError:
        b = None
    if b is None or b is not a and (a != b).any():
        raise ValueError(f"{name} holds a number that {np.dtype(dtype)} does not")
    return np.ascontiguousarray(b).ravel()


def _plan_args(cache: PagedCache, slots, new, max_rows):
    s = _whole(slots, np.int32, "slots")
    m = _whole(new, np.int32, "new")
    r = _whole(max_rows, np.int64, "max_rows")
    if m.size != s.size or r.size != s.size * cache.hkv:
        raise ValueError(f"{s.size} slots, {m.size} counts of new tokens and {r.size} bounds for {cache.hkv} heads each")
    return (s.ctypes.data_as(_lib.P_i32), m.ctypes.data_as(_lib.P_i32), r.ctypes.data_as(_lib.P_i64), s.size), m, (s, r)


def paged_workspace(cache: PagedCache, slots, new, max_rows, hq: int) -> int:
    """Workspace bytes of a plan (0 for arguments it refuses)."""
    args, _, _hold = _plan_args(cache, slots, new, max_rows)
    return int(lib().catekv_paged_workspace(cache.ref, *args, int(hq)))


def paged_plan(cache: PagedCache, slots: Sequence[int], new: Sequence[int], max_rows, hq: int,
               ws: Optional[torch.Tensor] = None) -> PagedPlan:
    """Work list of a batch: sequence i lies in slots[i] and has new[i] new tokens;
    max_rows [n_seqs][hkv]: upper bounds of its views' rows with them (blocking).
    Attention looks no further: a view that outgrows its bound needs another plan, and
    nothing says so at the call.
    Serves the append and the attention of every layer and later step of a batch of
    this shape, on caches of this geometry."""
    args, m, _hold = _plan_args(cache, slots, new, max_rows)
    if ws is None:
        need = int(lib().catekv_paged_workspace(cache.ref, *args, int(hq)))
        ws = workspace(need, cache.device)      # plan refuses what has none
    plan = _lib.PagedPlanT()
    _call(_device_of(cache.table, ws), lib().catekv_paged_plan, cache.ref, *args, int(hq), ctypes.byref(plan),
          ws.data_ptr(), _bytes(ws))
    return PagedPlan(plan, ws, int(m.sum()), int(hq), cache.hkv)


def append_kv_paged(plan: PagedPlan, cache: PagedCache, k_new: torch.Tensor, v_new: torch.Tensor,
                    overflow: Optional[torch.Tensor] = None) -> None:
    """The new tokens' rows behind every view's of the plan's sequences; pages are
    taken, and a shared last page copied, as needed.  k_new, v_new [n_tokens][hkv][d]
    with d contiguous and any strides of tokens and heads that are multiples of 16
    bytes (the same for both).  overflow: int32 [1] on the GPU (set to 1 when a
    sequence was left unchanged because pages or max_pages do not suffice) or None."""
    if k_new.shape != (plan.n_tokens, cache.hkv, D) or v_new.shape != k_new.shape:
        raise ValueError(f"k_new and v_new must be [{plan.n_tokens}][{cache.hkv}][{D}], not {tuple(k_new.shape)}, "
                         f"{tuple(v_new.shape)}")
    if k_new.dtype != cache.dtype or v_new.dtype != cache.dtype:
        raise TypeError(f"k_new and v_new must be {cache.dtype}, not {k_new.dtype}, {v_new.dtype}")
    # (what a dimension of size 1 has for a stride leads nowhere)
    strides = [tuple(x if n > 1 else 0 for x, n in zip(t.stride(), t.shape)) for t in (k_new, v_new)]
    tok, head, one = strides[0]
    if one != 1 or strides[1] != strides[0]:
        raise ValueError("k_new and v_new need the same strides and contiguous rows")
    index = _device_of(cache.table, plan.ws, overflow)
    if k_new.get_device() != index or v_new.get_device() != index:
        raise ValueError(f"k_new and v_new must lie on the cache's GPU, {cache.device}")
    if overflow is not None:
        _need(overflow, "overflow", torch.int32, 1)
    _call(index, lib().catekv_paged_append, cache.ref, plan.ref, k_new.data_ptr(), v_new.data_ptr(), tok, head,
          None if overflow is None else overflow.data_ptr(), plan.ws.data_ptr(), _bytes(plan.ws))


def attn_paged(plan: PagedPlan, cache: PagedCache, q: torch.Tensor, scale: Optional[float] = None,
               out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
               want_lse: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of the plan's new tokens, whose rows are the last of their views
    (after append_kv_paged): each sees its view up to its own row.  q [n_tokens][hq][d]
    in the cache's type -> (out in q's type, of its shape; lse fp32 [n_tokens][hq] or
    None)."""
    if q.shape != (plan.n_tokens, plan.hq, D):
        raise ValueError(f"q must be [{plan.n_tokens}][{plan.hq}][{D}], not {tuple(q.shape)}")
    n = plan.n_tokens * plan.hq
    _need(q, "q", cache.dtype, n * D)
    if out is None:
        out = torch.empty_like(q)
    else:
        _need(out, "out", cache.dtype, n * D)
    if lse is not None:
        _need(lse, "lse", torch.float32, n)
    elif want_lse:
        lse = torch.empty((plan.n_tokens, plan.hq), dtype=torch.float32, device=q.device)
    _call(_device_of(q, cache.table, plan.ws, out, lse), lib().catekv_paged_attn, cache.ref, plan.ref, q.data_ptr(),
          1.0 / math.sqrt(D) if scale is None else float(scale), out.data_ptr(), None if lse is None else lse.data_ptr(),
          plan.ws.data_ptr(), _bytes(plan.ws))
    return out, lse


def fork_paged(cache: PagedCache, src: Sequence[int], dst: Sequence[int], refused: Optional[torch.Tensor] = None) -> None:
    """Slot dst[i] (empty) becomes a copy of slot src[i] that shares its pages; an
    append to either copies the page that it writes first.  refused: int32 [1] on
    the GPU (set to 1 when a view of a dst was not empty, and left) or None.  Lists of
    any length, checked as a whole before the first is forked."""
    if len(src) != len(dst):
        raise ValueError(f"{len(src)} sources for {len(dst)} destinations")
    index = _device_of(cache.table, refused)
    if refused is not None:
        _need(refused, "refused", torch.int32, 1)
    _call(index, lib().catekv_paged_fork, cache.ref, _ints(src), _ints(dst), len(src),
          None if refused is None else refused.data_ptr())


def drop_paged(cache: PagedCache, rows: torch.Tensor) -> None:
    """Takes the last rows[slot] rows (int64 [n_slots] on the GPU) off every view of
    every slot (all of them where a view has no more; <= 0: none) and releases the
    pages behind them."""
    _need(rows, "rows", torch.int64, cache.n_slots)
    _call(_device_of(cache.table, rows), lib().catekv_paged_drop, cache.ref, rows.data_ptr())


def compact_paged_workspace(cache: PagedCache, n_sel: int, b: int, cs: int, tail: int) -> int:
    """Workspace bytes of compact_kv_paged (0 for sizes it refuses)."""
    return int(lib().catekv_paged_compact_workspace(cache.ref, int(n_sel), int(b), int(cs), int(tail)))


def compact_kv_paged(cache: PagedCache, slot: int, heads: Sequence[int], idx: torch.Tensor, cs: int, tail: int,
                     overflow: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> None:
    """Cache(K, V, i_k, L_obs) on pages: the listed heads' views of a slot keep the
    rows of the chunks idx [n_sel][b] (int32, from select_critical with l_obs = tail)
    and their last `tail` rows, in pages of their own; the old pages are released.
    overflow: int32 [1] on the GPU (set to 1 when a view was left unchanged) or None."""
    if idx.dim() != 2 or idx.shape[0] != len(heads):
        raise ValueError(f"idx must have a row per head, not {tuple(idx.shape)} for {len(heads)}")
    _need(idx, "idx", torch.int32, idx.numel())
    index = _device_of(cache.table, idx, overflow, ws)
    if overflow is not None:
        _need(overflow, "overflow", torch.int32, 1)
    b = idx.shape[1]
    if ws is None:
        ws = workspace(compact_paged_workspace(cache, len(heads), b, cs, tail), cache.device)
    _call(index, lib().catekv_paged_compact, cache.ref, int(slot), _ints(heads), len(heads), idx.data_ptr(), b,
          int(cs), int(tail), None if overflow is None else overflow.data_ptr(), ws.data_ptr(), _bytes(ws))


def gather_kv_paged(cache: PagedCache, slots: Sequence[int], kv_out: torch.Tensor, max_rows: int) -> None:
    """Writes the first min(lens, max_rows) rows of every view of the listed slots to
    kv_out (from kv_table, [n * hkv] views, rows in the cache's type; address 0: left
    out)."""
    _need_table(kv_out, len(slots) * cache.hkv)
    _call(_device_of(cache.table, kv_out), lib().catekv_paged_gather, cache.ref, _ints(slots), len(slots),
          kv_out.data_ptr(), int(max_rows))

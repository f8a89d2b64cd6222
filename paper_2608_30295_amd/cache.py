"""Python binding of include/catekv_cache.h: caches held in 8 bits, attention
that adds its weights up per cached row, and eviction by those weights.

As in ``binding.py`` only arguments are marshalled here; every step runs in
``libcatekv.so``.  Tables (``kv_table``, ``q8_views``, ``acc_table``) hold device
addresses: the tensors behind them must outlive their use.
"""
from __future__ import annotations

import ctypes
import math
from dataclasses import dataclass, field
from typing import List, Optional, Sequence, Tuple

import torch

from . import _lib
from ._lib import check, lib
from .binding import D, DecodePlan, _dtype_code, _need_cuda, _stream, workspace

FORMATS = {"int8": _lib.CATEKV_I8, "e4m3": _lib.CATEKV_E4M3}
BLOCKS = (32, 64)


@dataclass
class Q8Views:
    """Device table of 8-bit views (k, v, k_scale, v_scale, k_tail, v_tail of each)
    with what they have in common; `hold`: tensors to keep alive with it."""
    table: torch.Tensor
    fmt: str
    block: int
    dtype: torch.dtype
    hold: List[torch.Tensor] = field(default_factory=list)

    def __len__(self) -> int:
        return self.table.shape[0]

    @property
    def code(self) -> int:
        return FORMATS[self.fmt]

    @property
    def dtype_code(self) -> int:
        return _lib.CATEKV_BF16 if self.dtype == torch.bfloat16 else _lib.CATEKV_F32


def q8_views(ptrs: Sequence[Sequence[int]], device, *, fmt: str, block: int, dtype: torch.dtype) -> Q8Views:
    """Table of views from tuples of device addresses (k, v, k_scale, v_scale,
    k_tail, v_tail), [B * Hkv] entries.  fmt "int8" or "e4m3"; block 32 or 64;
    dtype (bfloat16 or float32) is that of the tails and of the queries."""
    if fmt not in FORMATS:
        raise ValueError(f"format {fmt!r} ({' or '.join(FORMATS)})")
    if block not in BLOCKS:
        raise ValueError(f"block of {block} rows (32 or 64)")
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype} (bfloat16 or float32)")
    rows = [[int(p) for p in row] for row in ptrs]
    if not rows or any(len(r) != 6 for r in rows):
        raise ValueError("each view has six addresses")
    return Q8Views(torch.tensor(rows, dtype=torch.int64).to(device), fmt, int(block), dtype)


def q8_alloc(capacity: Sequence[int], device, *, fmt: str, block: int, dtype: torch.dtype) -> Q8Views:
    """Views of the given capacities (rows, one per view) in memory of their own."""
    rows, hold = [], []
    for c in capacity:
        n = int(c) // block
        k, v = (torch.zeros((n * block, D), dtype=torch.int8, device=device) for _ in "kv")
        ks, vs = (torch.zeros(n, dtype=torch.float32, device=device) for _ in "kv")
        kt, vt = (torch.zeros((block, D), dtype=dtype, device=device) for _ in "kv")
        hold += [k, v, ks, vs, kt, vt]
        rows.append([t.data_ptr() for t in hold[-6:]])
    views = q8_views(rows, device, fmt=fmt, block=block, dtype=dtype)
    views.hold = hold
    return views


def acc_table(ptrs: Sequence[int], device) -> torch.Tensor:
    """Device array of the addresses of the views' weight arrays (fp32), [B * Hkv].
    An array is zero where its view has no rows yet."""
    return torch.tensor([int(p) for p in ptrs], dtype=torch.int64).to(device)


def _same_device(*ts: Optional[torch.Tensor]) -> torch.device:
    dev = [t.device for t in ts if t is not None]
    if any(d != dev[0] for d in dev):
        raise ValueError(f"tensors on several devices: {sorted({str(d) for d in dev})}")
    return dev[0]


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, n: Optional[int] = None) -> None:
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} values, not {t.numel()}")


def _need_table(kv: torch.Tensor, n: int) -> None:
    _need(kv, "kv", torch.int64)
    if tuple(kv.shape) != (n, 2):
        raise ValueError(f"kv must be a table of {n} views, not {tuple(kv.shape)}")


# ------------------------------------------------------------- into 8 bits and back

def quantize_kv(kv: torch.Tensor, lens: torch.Tensor, q8: Q8Views, max_rows: int) -> None:
    """Brings the first lens rows of every view of kv (from kv_table, rows in
    q8.dtype) into the 8-bit views.  lens: int64 on the GPU, one per view, none
    above max_rows."""
    _need_cuda(kv, lens, q8.table)
    _need_table(kv, len(q8))
    _need(lens, "lens", torch.int64, len(q8))
    dev = _same_device(kv, lens, q8.table)
    with torch.cuda.device(dev):
        check(lib().catekv_q8_quantize(q8.code, q8.dtype_code, q8.block, kv.data_ptr(), lens.data_ptr(),
                                       q8.table.data_ptr(), len(q8), int(max_rows), D, _stream(dev)))


def dequantize_kv(q8: Q8Views, lens: torch.Tensor, kv_out: torch.Tensor, max_rows: int) -> None:
    """Writes the first lens rows of every 8-bit view to kv_out (from kv_table,
    rows in q8.dtype): code times scale, the tail as it is."""
    _need_cuda(kv_out, lens, q8.table)
    _need_table(kv_out, len(q8))
    _need(lens, "lens", torch.int64, len(q8))
    dev = _same_device(kv_out, lens, q8.table)
    with torch.cuda.device(dev):
        check(lib().catekv_q8_dequantize(q8.code, q8.dtype_code, q8.block, q8.table.data_ptr(), lens.data_ptr(),
                                         kv_out.data_ptr(), len(q8), int(max_rows), D, _stream(dev)))


def append_kv_q8(q8: Q8Views, capacity: torch.Tensor, lens: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                 overflow: Optional[torch.Tensor] = None) -> None:
    """append_kv on 8-bit views: the newest token's rows into the tails, lens
    bumped on the device, a full tail turned into a block.  k_new, v_new
    [B][Hkv][d] in q8.dtype; capacity, lens int64 on the GPU, one per view;
    overflow: int32 [1] on the GPU (set to 1 when a view is full) or None."""
    _need_cuda(q8.table, capacity, lens, k_new, v_new, *([overflow] if overflow is not None else []))
    B, hkv, d = k_new.shape
    if v_new.shape != k_new.shape:
        raise ValueError("k_new and v_new must have the same shape")
    if B * hkv != len(q8):
        raise ValueError(f"k_new holds {B * hkv} views, the table {len(q8)}")
    for t, name in ((k_new, "k_new"), (v_new, "v_new")):
        _need(t, name, q8.dtype)
    for t, name in ((capacity, "capacity"), (lens, "lens")):
        _need(t, name, torch.int64, len(q8))
    if overflow is not None:
        _need(overflow, "overflow", torch.int32, 1)
    dev = _same_device(q8.table, capacity, lens, k_new, v_new, overflow)
    with torch.cuda.device(dev):
        check(lib().catekv_q8_append(q8.code, q8.dtype_code, q8.block, q8.table.data_ptr(), capacity.data_ptr(),
                                     lens.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), B, hkv, d,
                                     overflow.data_ptr() if overflow is not None else None, _stream(dev)))


# ------------------------------------------------------------------------ attention

def weights_workspace(plan: DecodePlan) -> int:
    """Workspace bytes of a decode step of this plan that adds its weights up."""
    return int(lib().catekv_weights_workspace(ctypes.byref(plan.plan)))


def _attend(plan, q, views, n_views, lens, scale, out, lse, want_lse, acc, ws, call):
    _need_cuda(q, views, lens, plan.ws, *[t for t in (out, lse, acc, ws) if t is not None])
    B, hq, d = q.shape
    if n_views != B * plan.hkv:
        raise ValueError(f"a table of {n_views} views for {B} x {plan.hkv}")
    _need(lens, "lens", torch.int64, n_views)
    if scale is None:
        scale = 1.0 / math.sqrt(d)
    if out is None:
        out = torch.empty((B, hq, d), dtype=torch.float32, device=q.device)
    if lse is None and want_lse:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    _need(out, "out", torch.float32, B * hq * d)
    if lse is not None:
        _need(lse, "lse", torch.float32, B * hq)
    if acc is not None:
        _need(acc, "acc", torch.int64, n_views)
        if ws is None:
            ws = workspace(weights_workspace(plan), q.device)
    dev = _same_device(q, views, lens, plan.ws, out, lse, acc, ws)
    with torch.cuda.device(dev):
        check(call(ctypes.byref(plan.plan), q.data_ptr(), views.data_ptr(), lens.data_ptr(), B, hq, plan.hkv, d,
                   float(scale), out.data_ptr(), lse.data_ptr() if lse is not None else None,
                   acc.data_ptr() if acc is not None else None, plan.ws.data_ptr(), plan.ws.numel(),
                   ws.data_ptr() if ws is not None else None,
                   ws.numel() * ws.element_size() if ws is not None else 0, _stream(dev)))
    return out, lse


def decode_attn_q8(plan: DecodePlan, q: torch.Tensor, q8: Q8Views, lens: torch.Tensor,
                   scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                   lse: Optional[torch.Tensor] = None, want_lse: bool = True, acc: Optional[torch.Tensor] = None,
                   decay: float = 1.0, ws: Optional[torch.Tensor] = None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """decode_attn over 8-bit views: q [B][Hq][d] in q8.dtype, lens int64 [B][Hkv]
    on the GPU -> (out fp32 [B][Hq][d], lse fp32 [B][Hq] or None).  With acc (from
    acc_table) every row's softmax weight, averaged over the group's heads, is
    added to decay times what its view's array holds; ws: weights_workspace(plan)
    bytes, or None to allocate them."""
    _need(q, "q", q8.dtype)
    L = lib()
    return _attend(plan, q, q8.table, len(q8), lens, scale, out, lse, want_lse, acc, ws,
                   lambda p, qp, vp, lp, B, hq, hkv, d, sc, o, ls, ac, w, wb, ww, wwb, st: L.catekv_q8_decode_attn(
                       q8.code, q8.dtype_code, q8.block, p, qp, vp, lp, B, hq, hkv, d, sc, o, ls, ac, float(decay),
                       w, wb, ww, wwb, st))


def decode_attn_weights(plan: DecodePlan, q: torch.Tensor, kv: torch.Tensor, lens: torch.Tensor, acc: torch.Tensor,
                        decay: float = 1.0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                        ws: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """decode_attn over the same views (kv from kv_table, rows in q's dtype), its
    weights added up in acc as by decode_attn_q8."""
    code = _dtype_code(q)
    _need_cuda(kv)
    _need_table(kv, plan.batch * plan.hkv)
    L = lib()
    return _attend(plan, q, kv, kv.shape[0], lens, scale, out, lse, want_lse, acc, ws,
                   lambda p, qp, vp, lp, B, hq, hkv, d, sc, o, ls, ac, w, wb, ww, wwb, st: L.catekv_decode_attn_weights(
                       code, p, qp, vp, lp, B, hq, hkv, d, sc, o, ls, ac, float(decay), w, wb, ww, wwb, st))


# ------------------------------------------------------------------------- eviction

def evict_workspace(n_views: int, max_rows: int, cs: int) -> int:
    """Workspace bytes of the eviction calls (0 for sizes they refuse)."""
    return int(lib().catekv_evict_workspace(int(n_views), int(max_rows), int(cs)))


def _evict(views, n, lens, acc, budget, cs, max_rows, ws, call):
    _need_cuda(views, lens, acc, budget, *([ws] if ws is not None else []))
    _need(lens, "lens", torch.int64, n)
    _need(acc, "acc", torch.int64, n)
    _need(budget, "budget", torch.int32, n)
    if ws is None:
        ws = workspace(evict_workspace(n, max_rows, cs), views.device)
    dev = _same_device(views, lens, acc, budget, ws)
    with torch.cuda.device(dev):
        check(call(views.data_ptr(), lens.data_ptr(), acc.data_ptr(), budget.data_ptr(), n, int(max_rows), int(cs),
                   ws.data_ptr(), ws.numel() * ws.element_size(), _stream(dev)))


def evict_kv(kv: torch.Tensor, lens: torch.Tensor, acc: torch.Tensor, budget: torch.Tensor, *, cs: int, recent: int,
             max_rows: int, dtype: torch.dtype, ws: Optional[torch.Tensor] = None) -> None:
    """Drops, in place, the chunks of cs rows that gathered least weight: of every
    view's chunks before the last `recent` rows, the budget[view] with the
    largest acc stay (catekv_evict_kv).  lens is updated on the device; acc moves
    with its rows.  budget: int32 on the GPU, one per view, < 0 leaves a view
    alone.  dtype: that of the rows."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype} (bfloat16 or float32)")
    _need_cuda(kv)
    _need_table(kv, lens.numel())
    code = _lib.CATEKV_BF16 if dtype == torch.bfloat16 else _lib.CATEKV_F32
    L = lib()
    _evict(kv, kv.shape[0], lens, acc, budget, cs, max_rows, ws,
           lambda vp, lp, ap, bp, n, mr, c, w, wb, st: L.catekv_evict_kv(code, vp, lp, ap, bp, n, mr, c, int(recent), D,
                                                                        w, wb, st))


def evict_kv_q8(q8: Q8Views, lens: torch.Tensor, acc: torch.Tensor, budget: torch.Tensor, *, cs: int, recent: int,
                max_rows: int, ws: Optional[torch.Tensor] = None) -> None:
    """evict_kv on 8-bit views; cs is a multiple of their block, so that blocks
    move whole with their scales, and the tails stay."""
    L = lib()
    _evict(q8.table, len(q8), lens, acc, budget, cs, max_rows, ws,
           lambda vp, lp, ap, bp, n, mr, c, w, wb, st: L.catekv_q8_evict(q8.block, vp, lp, ap, bp, n, mr, c, int(recent),
                                                                        D, w, wb, st))

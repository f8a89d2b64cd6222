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
from .binding import D, DecodePlan, _dtype_code, _need_cuda, workspace

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

    def __post_init__(self) -> None:
        if self.fmt not in FORMATS:
            raise ValueError(f"format {self.fmt!r} ({' or '.join(FORMATS)})")
        if self.block not in BLOCKS:
            raise ValueError(f"block of {self.block} rows (32 or 64)")
        if self.dtype not in (torch.bfloat16, torch.float32):
            raise TypeError(f"unsupported dtype {self.dtype} (bfloat16 or float32)")
        if self.table.dtype != torch.int64 or self.table.dim() != 2 or self.table.shape[1] != 6:
            raise ValueError("the table has six addresses per view")
        self.code = FORMATS[self.fmt]
        self.dtype_code = _lib.CATEKV_BF16 if self.dtype == torch.bfloat16 else _lib.CATEKV_F32


def q8_views(ptrs: Sequence[Sequence[int]], device, *, fmt: str, block: int, dtype: torch.dtype) -> Q8Views:
    """Table of views from tuples of device addresses (k, v, k_scale, v_scale,
    k_tail, v_tail), [B * Hkv] entries.  fmt "int8" or "e4m3"; block 32 or 64;
    dtype (bfloat16 or float32) is that of the tails and of the queries."""
    rows = [[int(p) for p in row] for row in ptrs]
    if not rows or any(len(r) != 6 for r in rows):
        raise ValueError("each view has six addresses")
    return Q8Views(torch.tensor(rows, dtype=torch.int64).to(device), fmt, int(block), dtype)


def q8_alloc(capacity: Sequence[int], device, *, fmt: str, block: int, dtype: torch.dtype) -> Q8Views:
    """Views of the given capacities (rows, one per view) in memory of their own."""
    rows, hold = [], []
    for c in capacity:
        n = int(c) // max(int(block), 1)      # q8_views refuses a bad block
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


# The checks below run before every call of a serving loop: few attribute reads
# per tensor, no device guard where the current device is the tensors' own, and the
# raw stream handle (together 17 -> 13 us per call).

def _device_of(*ts: Optional[torch.Tensor]) -> int:
    """Index of the GPU that all given tensors lie on, contiguous."""
    index = ts[0].get_device()
    for t in ts:
        if t is not None and (t.get_device() != index or index < 0 or not t.is_contiguous()):
            _need_cuda(t)
            raise ValueError(f"tensors on several devices: {t.device} and {ts[0].device}")
    return index


def _call(index: int, fn, *args) -> None:
    """fn(*args, stream) on the current stream of that GPU."""
    if index == torch.cuda.current_device():
        status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    else:
        with torch.cuda.device(index):
            status = fn(*args, torch._C._cuda_getCurrentRawStream(index))
    if status:
        check(status)


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, n: int) -> None:
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.numel() != n:
        raise ValueError(f"{name} must have {n} values, not {t.numel()}")


def _need_table(kv: torch.Tensor, n: int) -> None:
    if kv.dtype != torch.int64:
        raise TypeError(f"kv must be torch.int64, not {kv.dtype}")
    if kv.shape != (n, 2):
        raise ValueError(f"kv must be a table of {n} views, not {tuple(kv.shape)}")


def _bytes(ws: torch.Tensor) -> int:
    return ws.numel() * ws.element_size()


# ------------------------------------------------------------- into 8 bits and back

def quantize_kv(kv: torch.Tensor, lens: torch.Tensor, q8: Q8Views, max_rows: int) -> None:
    """Brings the first lens rows of every view of kv (from kv_table, rows in
    q8.dtype) into the 8-bit views.  lens: int64 on the GPU, one per view, none
    above max_rows."""
    n = len(q8)
    index = _device_of(q8.table, kv, lens)
    _need_table(kv, n)
    _need(lens, "lens", torch.int64, n)
    _call(index, lib().catekv_q8_quantize, q8.code, q8.dtype_code, q8.block, kv.data_ptr(), lens.data_ptr(),
          q8.table.data_ptr(), n, int(max_rows), D)


def dequantize_kv(q8: Q8Views, lens: torch.Tensor, kv_out: torch.Tensor, max_rows: int) -> None:
    """Writes the first lens rows of every 8-bit view to kv_out (from kv_table,
    rows in q8.dtype): code times scale, the tail as it is."""
    n = len(q8)
    index = _device_of(q8.table, kv_out, lens)
    _need_table(kv_out, n)
    _need(lens, "lens", torch.int64, n)
    _call(index, lib().catekv_q8_dequantize, q8.code, q8.dtype_code, q8.block, q8.table.data_ptr(), lens.data_ptr(),
          kv_out.data_ptr(), n, int(max_rows), D)


def append_kv_q8(q8: Q8Views, capacity: torch.Tensor, lens: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                 overflow: Optional[torch.Tensor] = None) -> None:
    """append_kv on 8-bit views: the newest token's rows into the tails, lens
    bumped on the device, a full tail turned into a block.  k_new, v_new
    [B][Hkv][d] in q8.dtype; capacity, lens int64 on the GPU, one per view;
    overflow: int32 [1] on the GPU (set to 1 when a view is full) or None."""
    n = len(q8)
    index = _device_of(q8.table, capacity, lens, k_new, v_new, overflow)
    B, hkv, d = k_new.shape
    if v_new.shape != k_new.shape:
        raise ValueError("k_new and v_new must have the same shape")
    if B * hkv != n:
        raise ValueError(f"k_new holds {B * hkv} views, the table {n}")
    _need(k_new, "k_new", q8.dtype, n * d)
    _need(v_new, "v_new", q8.dtype, n * d)
    _need(capacity, "capacity", torch.int64, n)
    _need(lens, "lens", torch.int64, n)
    if overflow is not None:
        _need(overflow, "overflow", torch.int32, 1)
    _call(index, lib().catekv_q8_append, q8.code, q8.dtype_code, q8.block, q8.table.data_ptr(), capacity.data_ptr(),
          lens.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), B, hkv, d,
          overflow.data_ptr() if overflow is not None else None)


# ------------------------------------------------------------------------ attention

def weights_workspace(plan: DecodePlan) -> int:
    """Workspace bytes of a decode step of this plan that adds its weights up."""
    return int(lib().catekv_weights_workspace(ctypes.byref(plan.plan)))


def _attend(fn, kind, plan, q, views, lens, scale, out, lse, want_lse, acc, decay, ws):
    index = _device_of(q, views, lens, plan.ws, out, lse, acc, ws)
    B, hq, d = q.shape
    n = views.shape[0]
    if n != B * plan.hkv:
        raise ValueError(f"a table of {n} views for {B} x {plan.hkv}")
    _need(lens, "lens", torch.int64, n)
    if out is None:
        out = torch.empty((B, hq, d), dtype=torch.float32, device=q.device)
    else:
        _need(out, "out", torch.float32, B * hq * d)
    if lse is not None:
        _need(lse, "lse", torch.float32, B * hq)
    elif want_lse:
        lse = torch.empty((B, hq), dtype=torch.float32, device=q.device)
    if acc is not None:
        _need(acc, "acc", torch.int64, n)
        if ws is None:
            ws = workspace(weights_workspace(plan), q.device)
    _call(index, fn, *kind, ctypes.byref(plan.plan), q.data_ptr(), views.data_ptr(), lens.data_ptr(), B, hq, plan.hkv, d,
          1.0 / math.sqrt(d) if scale is None else float(scale), out.data_ptr(),
          None if lse is None else lse.data_ptr(), None if acc is None else acc.data_ptr(), float(decay),
          plan.ws.data_ptr(), _bytes(plan.ws), None if ws is None else ws.data_ptr(), 0 if ws is None else _bytes(ws))
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
    if q.dtype != q8.dtype:
        raise TypeError(f"q must be {q8.dtype}, not {q.dtype}")
    return _attend(lib().catekv_q8_decode_attn, (q8.code, q8.dtype_code, q8.block), plan, q, q8.table, lens, scale, out,
                   lse, want_lse, acc, decay, ws)


def decode_attn_weights(plan: DecodePlan, q: torch.Tensor, kv: torch.Tensor, lens: torch.Tensor, acc: torch.Tensor,
                        decay: float = 1.0, scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                        lse: Optional[torch.Tensor] = None, want_lse: bool = True,
                        ws: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """decode_attn over the same views (kv from kv_table, rows in q's dtype), its
    weights added up in acc as by decode_attn_q8."""
    _need_table(kv, plan.batch * plan.hkv)
    return _attend(lib().catekv_decode_attn_weights, (_dtype_code(q),), plan, q, kv, lens, scale, out, lse, want_lse,
                   acc, decay, ws)


# ------------------------------------------------------------------------- eviction

def evict_workspace(n_views: int, max_rows: int, cs: int) -> int:
    """Workspace bytes of the eviction calls (0 for sizes they refuse)."""
    return int(lib().catekv_evict_workspace(int(n_views), int(max_rows), int(cs)))


def _evict(fn, kind, views, lens, acc, budget, cs, recent, max_rows, ws):
    n = views.shape[0]
    index = _device_of(views, lens, acc, budget, ws)
    _need(lens, "lens", torch.int64, n)
    _need(acc, "acc", torch.int64, n)
    _need(budget, "budget", torch.int32, n)
    if ws is None:
        ws = workspace(evict_workspace(n, max_rows, cs), views.device)
    _call(index, fn, kind, views.data_ptr(), lens.data_ptr(), acc.data_ptr(), budget.data_ptr(), n, int(max_rows),
          int(cs), int(recent), D, ws.data_ptr(), _bytes(ws))


def evict_kv(kv: torch.Tensor, lens: torch.Tensor, acc: torch.Tensor, budget: torch.Tensor, *, cs: int, recent: int,
             max_rows: int, dtype: torch.dtype, ws: Optional[torch.Tensor] = None) -> None:
    """Drops, in place, the chunks of cs rows that gathered least weight: of every
    view's chunks before the last `recent` rows, the budget[view] with the
    largest acc stay (catekv_evict_kv).  lens is updated on the device; acc moves
    with its rows.  budget: int32 on the GPU, one per view, < 0 leaves a view
    alone.  dtype: that of the rows.

    Afterwards a view has at most budget * cs + recent + cs - 1 rows.  A plan cuts its
    shares by the lengths planned for, and one for the rows before leaves most of the
    GPU idle: make a new one (and choose max_rows) for that bound and the steps until
    the next eviction (8 int8 views from 131072 to 16512 rows: 50 us a step under the
    old plan, 17 under the new one)."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype} (bfloat16 or float32)")
    _need_table(kv, kv.shape[0])
    _evict(lib().catekv_evict_kv, _lib.CATEKV_BF16 if dtype == torch.bfloat16 else _lib.CATEKV_F32, kv, lens, acc, budget,
           cs, recent, max_rows, ws)


def evict_kv_q8(q8: Q8Views, lens: torch.Tensor, acc: torch.Tensor, budget: torch.Tensor, *, cs: int, recent: int,
                max_rows: int, ws: Optional[torch.Tensor] = None) -> None:
    """evict_kv on 8-bit views; cs is a multiple of their block, so that blocks
    move whole with their scales, and the tails stay."""
    _evict(lib().catekv_q8_evict, q8.block, q8.table, lens, acc, budget, cs, recent, max_rows, ws)

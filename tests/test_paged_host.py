"""What the calls of include/catekv_paged.h refuse, on the host: arguments are checked
before the GPU is touched.  The plain forms that the GPU tests compare with are pinned
by facts other than their own formulas."""
import ast
import ctypes
import inspect
import math
import os
import re
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck
from paper_2608_30295_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "catekv_paged.h")
needs_lib = pytest.mark.skipif(not os.path.exists(_lib.LIB_PATH), reason="libcatekv.so not built")

FAKE = 0x100000   # a non-null pointer value; never dereferenced on these paths
INVALID, UNSUPPORTED, WORKSPACE = _lib.CATEKV_ERR_INVALID_ARG, _lib.CATEKV_ERR_UNSUPPORTED, _lib.CATEKV_ERR_WORKSPACE
MAGIC = 0x6361746570616765


def cache(**kw):
    a = dict(k=FAKE, v=FAKE, table=FAKE, lens=FAKE, refs=FAKE, free_bits=FAKE, dtype=1, page=64, n_pages=1000, n_slots=4,
             hkv=2, max_pages=100)
    a.update(kw)
    return _lib.PagedCacheT(*[a[n] for n, _ in _lib.PagedCacheT._fields_])


def plan(**kw):
    p = _lib.PagedPlanT()
    a = dict(magic=MAGIC, n_seqs=1, n_tokens=3, hq=8, hkv=2, n_slots=4, page=64, dtype=1, ws_bytes=1 << 12)   # a plan's header
    for n, x in {**a, **kw}.items():
        setattr(p, n, x)
    return p


def i32(*x):
    return (ctypes.c_int32 * max(len(x), 1))(*x)


def i64(*x):
    return (ctypes.c_int64 * max(len(x), 1))(*x)


BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(table=None), INVALID), (dict(lens=None), INVALID),
    (dict(refs=None), INVALID), (dict(free_bits=None), INVALID), (dict(k=FAKE + 8), INVALID), (dict(v=FAKE + 2), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(page=8), INVALID), (dict(page=0), INVALID),
    (dict(page=48), INVALID), (dict(page=512), INVALID), (dict(page=-64), INVALID), (dict(n_pages=0), INVALID),
    (dict(n_slots=0), INVALID), (dict(hkv=0), INVALID), (dict(max_pages=0), INVALID), (dict(n_pages=-5), INVALID),
    (dict(hkv=1025), UNSUPPORTED), (dict(n_slots=1 << 19, hkv=4), UNSUPPORTED), (dict(max_pages=(1 << 20) + 1), UNSUPPORTED),
]


@needs_lib
def test_every_declared_symbol_is_exported_with_its_signature():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(catekv_paged_[a-z_0-9]+)\s*\(", text)))
    assert set(names) == set(_lib.PAGED_SIGNATURES) and len(names) == 10
    for n in names:
        args = re.search(n + r"\s*\(([^)]*)\)", text, flags=re.S).group(1)
        assert len(args.split(",")) == len(_lib.PAGED_SIGNATURES[n][1]), n
        assert hasattr(ck.lib(), n)


def test_structures_are_laid_out_as_declared():
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    for name, t in (("catekv_paged_cache", _lib.PagedCacheT), ("catekv_paged_plan_t", _lib.PagedPlanT)):
        body = re.search(r"typedef struct " + name + r" \{(.*?)\}", text, flags=re.S).group(1)
        fields = []
        for line in body.split(";"):
            m = re.match(r"\s*(\w+)(\s*\*)?\s*(.*)", line.strip(), flags=re.S)
            for f in m.group(3).split(",") if m and m.group(3) else []:
                ptr = bool(m.group(2)) or "*" in f
                fields.append((f.replace("*", "").strip(), 8 if ptr else {"int32_t": 4, "uint64_t": 8}[m.group(1)]))
        assert fields == [(n, ctypes.sizeof(x)) for n, x in t._fields_], name


@needs_lib
@pytest.mark.parametrize("change,status", BAD_CACHES)
def test_every_call_refuses_a_bad_cache(change, status):
    L, c, p = ck.lib(), ctypes.byref(cache(**change)), ctypes.byref(plan())
    assert L.catekv_paged_init(c, None) == status
    assert L.catekv_last_error()
    assert L.catekv_paged_workspace(c, i32(0), i32(1), i64(9, 9), 1, 8) == 0
    assert L.catekv_paged_plan(c, i32(0), i32(1), i64(9, 9), 1, 8, p, FAKE, 1 << 20, None) == status
    assert L.catekv_paged_append(c, p, FAKE, FAKE, 256, 128, None, FAKE, 1 << 20, None) == status
    assert L.catekv_paged_attn(c, p, FAKE, 0.1, FAKE, None, FAKE, 1 << 20, None) == status
    assert L.catekv_paged_fork(c, i32(0), i32(1), 1, None, None) == status
    assert L.catekv_paged_drop(c, FAKE, None) == status
    assert L.catekv_paged_compact_workspace(c, 1, 4, 8, 0) == 0
    assert L.catekv_paged_compact(c, 0, i32(0), 1, FAKE, 4, 8, 0, None, FAKE, 1 << 20, None) == status
    assert L.catekv_paged_gather(c, i32(0), 1, FAKE, 10, None) == status


@needs_lib
def test_every_call_refuses_a_missing_cache():
    L, p = ck.lib(), ctypes.byref(plan())
    assert L.catekv_paged_init(None, None) == INVALID
    assert L.catekv_paged_workspace(None, i32(0), i32(1), i64(9, 9), 1, 8) == 0
    assert L.catekv_paged_append(None, p, FAKE, FAKE, 256, 128, None, FAKE, 1 << 20, None) == INVALID
    assert L.catekv_paged_attn(None, p, FAKE, 0.1, FAKE, None, FAKE, 1 << 20, None) == INVALID
    assert L.catekv_paged_drop(None, FAKE, None) == INVALID


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(slots=None), INVALID), (dict(new=None), INVALID), (dict(rows=None), INVALID), (dict(n=0), INVALID), (dict(n=-1), INVALID),
    (dict(slots=i32(0, 4)), INVALID), (dict(slots=i32(-1, 0)), INVALID), (dict(slots=i32(2, 2)), INVALID),
    (dict(new=i32(1, -1)), INVALID), (dict(rows=i64(9, 9, 9, -1)), INVALID), (dict(rows=i64(9, 9, 9, (1 << 26) + 1)), UNSUPPORTED),
    (dict(new=i32(1 << 26, 1)), UNSUPPORTED), (dict(new=i32(2 ** 31 - 1, 1)), UNSUPPORTED), (dict(hq=6), UNSUPPORTED),
    (dict(hq=5), INVALID), (dict(hq=0), INVALID), (dict(plan=None), INVALID), (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 16), WORKSPACE), (dict(wsb=256), WORKSPACE),
])
def test_plans_refuse(change, status):
    a = dict(slots=i32(1, 3), new=i32(40, 1), rows=i64(100, 100, 1000, 0), n=2, hq=8, plan=ctypes.byref(plan()), ws=FAKE, wsb=1 << 30)
    a.update(change)
    L, c = ck.lib(), cache()
    got = L.catekv_paged_plan(ctypes.byref(c), a["slots"], a["new"], a["rows"], a["n"], a["hq"], a["plan"], a["ws"], a["wsb"], None)
    assert got == status, L.catekv_last_error()
    if status != WORKSPACE and a["plan"] is not None:
        assert L.catekv_paged_workspace(ctypes.byref(c), a["slots"], a["new"], a["rows"], a["n"], a["hq"]) == 0


@needs_lib
def test_plans_refuse_more_than_a_launch_takes():
    """2^25 tokens of 8 heads: 2^32 threads of 16 lanes a row."""
    c, L = cache(hkv=8), ck.lib()
    a = (ctypes.byref(c), i32(1), i32(1 << 25), i64(*[1 << 26] * 8), 1, 8)
    assert L.catekv_paged_workspace(*a) == 0
    assert L.catekv_paged_plan(*a, ctypes.byref(plan()), FAKE, 1 << 40, None) == UNSUPPORTED


@needs_lib
def test_workspaces_hold_what_the_calls_need():
    """At least the new tokens' and views' tables; a plan without tokens has one, too."""
    L, c = ck.lib(), ctypes.byref(cache())
    need = L.catekv_paged_workspace(c, i32(1, 3), i32(40, 1), i64(100, 100, 1000, 0), 2, 8)
    assert need % 256 == 0 and need >= 41 * 4 + 4 * 16
    assert L.catekv_paged_workspace(c, i32(1), i32(0), i64(0, 0), 1, 8) >= 256
    # a long view cut for many workgroups: a slot of 16 rows for each part at least twice
    assert L.catekv_paged_workspace(c, i32(1), i32(1), i64(6400, 6400), 1, 8) >= 2 * 2 * 16 * 130 * 4
    assert L.catekv_paged_compact_workspace(c, 2, 100, 8, 64) >= 2 * 100 * 4 + 2 * 14 * 4


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(plan=plan(magic=1)), INVALID), (dict(plan=plan(hkv=4)), INVALID), (dict(plan=plan(page=32)), INVALID),
    (dict(plan=plan(dtype=0)), INVALID), (dict(plan=plan(n_slots=5)), INVALID), (dict(x=None), INVALID), (dict(y=None), INVALID),
    (dict(x=FAKE + 8), INVALID), (dict(y=FAKE + 4), INVALID), (dict(ws=None), WORKSPACE), (dict(ws=FAKE + 128), WORKSPACE),
    (dict(wsb=(1 << 12) - 1), WORKSPACE),
])
def test_append_and_attention_refuse(change, status):
    a = dict(plan=plan(), x=FAKE, y=FAKE, ws=FAKE, wsb=1 << 20)
    a.update(change)
    L, c, p = ck.lib(), ctypes.byref(cache()), ctypes.byref(a["plan"])
    assert L.catekv_paged_append(c, p, a["x"], a["y"], 256, 128, None, a["ws"], a["wsb"], None) == status
    assert L.catekv_paged_attn(c, p, a["x"], 0.1, a["y"], None, a["ws"], a["wsb"], None) == status
    assert L.catekv_paged_append(c, None, FAKE, FAKE, 256, 128, None, FAKE, 1 << 20, None) == INVALID
    assert L.catekv_paged_attn(c, None, FAKE, 0.1, FAKE, None, FAKE, 1 << 20, None) == INVALID


@needs_lib
@pytest.mark.parametrize("tok,head", [(-256, 128), (256, -128), (257, 128), (256, 4), (1 << 41, 128), (256, 1 << 41)])
def test_append_refuses_strides(tok, head):
    assert ck.lib().catekv_paged_append(ctypes.byref(cache()), ctypes.byref(plan()), FAKE, FAKE, tok, head, None, FAKE, 1 << 20,
                                        None) == INVALID


@needs_lib
@pytest.mark.parametrize("scale", [0.0, -1.0, math.nan, math.inf])
def test_attention_refuses_scales(scale):
    assert ck.lib().catekv_paged_attn(ctypes.byref(cache()), ctypes.byref(plan()), FAKE, scale, FAKE, None, FAKE, 1 << 20,
                                      None) == INVALID


@needs_lib
@pytest.mark.parametrize("src,dst,n", [
    (None, i32(1), 1), (i32(0), None, 1), (i32(0), i32(1), 0), (i32(0), i32(1), -1), (i32(*[0] * 257), i32(*range(257)), 257),
    (i32(4), i32(1), 1), (i32(0), i32(4), 1), (i32(-1), i32(1), 1), (i32(0), i32(-1), 1), (i32(0), i32(0), 1),
    (i32(0, 0), i32(1, 1), 2), (i32(0, 1), i32(1, 2), 2),
])
def test_forks_refuse(src, dst, n):
    assert ck.lib().catekv_paged_fork(ctypes.byref(cache()), src, dst, n, None, None) == INVALID


@needs_lib
@pytest.mark.parametrize("change,status", [
    (dict(slot=-1), INVALID), (dict(slot=4), INVALID), (dict(heads=None), INVALID), (dict(heads=i32(0, 2)), INVALID),
    (dict(heads=i32(-1, 0)), INVALID), (dict(heads=i32(1, 1)), INVALID), (dict(n=0), INVALID), (dict(n=129), INVALID),
    (dict(idx=None), INVALID), (dict(b=0), INVALID), (dict(cs=0), INVALID), (dict(tail=-1), INVALID),
    (dict(b=(1 << 23) + 1), UNSUPPORTED), (dict(b=1 << 20, cs=1 << 6, tail=1), UNSUPPORTED), (dict(ws=None), WORKSPACE),
    (dict(ws=FAKE + 16), WORKSPACE), (dict(wsb=100), WORKSPACE),
])
def test_compaction_refuses(change, status):
    a = dict(slot=1, heads=i32(0, 1), n=2, idx=FAKE, b=10, cs=8, tail=16, ws=FAKE, wsb=1 << 20)
    a.update(change)
    assert ck.lib().catekv_paged_compact(ctypes.byref(cache()), a["slot"], a["heads"], a["n"], a["idx"], a["b"], a["cs"], a["tail"],
                                         None, a["ws"], a["wsb"], None) == status


@needs_lib
@pytest.mark.parametrize("slots,n,out,rows,status", [
    (None, 1, FAKE, 10, INVALID), (i32(0), 1, None, 10, INVALID), (i32(0), 0, FAKE, 10, INVALID), (i32(*[0] * 257), 257, FAKE, 10, INVALID),
    (i32(4), 1, FAKE, 10, INVALID), (i32(-1), 1, FAKE, 10, INVALID), (i32(0), 1, FAKE, 0, INVALID),
])
def test_gathering_refuses(slots, n, out, rows, status):
    assert ck.lib().catekv_paged_gather(ctypes.byref(cache()), slots, n, out, rows, None) == status


@needs_lib
def test_gathering_refuses_more_rows_than_a_launch_takes():
    c = cache(n_slots=16, hkv=1024, max_pages=1 << 20)                   # 2^26 rows of each of 16384 views
    assert ck.lib().catekv_paged_gather(ctypes.byref(c), i32(*range(16)), 16, FAKE, 1 << 40, None) == UNSUPPORTED
    assert ck.lib().catekv_paged_drop(ctypes.byref(c), None, None) == INVALID


def test_the_binding_refuses_what_has_no_place_on_the_gpu():
    t = torch.zeros
    ok = dict(k=t(4, 16, 128), v=t(4, 16, 128), table=t(2, 1, 3, dtype=torch.int32), lens=t(2, 1, dtype=torch.int64),
              refs=t(4, dtype=torch.int32), free_bits=t(1, dtype=torch.int64))
    for change, error in [
            (dict(), ValueError), (dict(k=t(4, 16, 64)), ValueError), (dict(v=t(4, 32, 128)), ValueError),
            (dict(v=t(4, 16, 128, dtype=torch.bfloat16)), ValueError), (dict(table=t(2, 3, dtype=torch.int32)), ValueError),
            (dict(table=t(2, 1, 3, dtype=torch.int64)), TypeError), (dict(lens=t(3, 1, dtype=torch.int64)), ValueError),
            (dict(lens=t(2, 1, dtype=torch.int32)), TypeError), (dict(refs=t(5, dtype=torch.int32)), ValueError),
            (dict(free_bits=t(2, dtype=torch.int64)), ValueError),
            (dict(k=t(4, 16, 128, dtype=torch.float16), v=t(4, 16, 128, dtype=torch.float16)), TypeError),
            (dict(k=t(4, 24, 128), v=t(4, 24, 128)), ValueError)]:
        with pytest.raises(error):
            ck.PagedCache(**{**ok, **change})                            # at last: tensors on the CPU
    with pytest.raises(ValueError):
        ck.paged_alloc(0, 16, 1, 1, 1, "cpu", dtype=torch.float32)


# ------------------------------------------------------- the plain forms, pinned

def test_attention_form_is_causal_softmax_attention():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((5, 2, 128), (23, 128), (23, 128)))
    out, lse, A, B = R.attention(q.numpy(), k.numpy(), v.numpy(), 5, 0.1)
    mask = torch.ones(5, 23, dtype=torch.bool).tril(23 - 5)
    want = torch.nn.functional.scaled_dot_product_attention(q.transpose(0, 1), k.expand(2, -1, -1), v.expand(2, -1, -1),
                                                            attn_mask=mask, scale=0.1)
    assert np.allclose(out, want.transpose(0, 1).numpy(), atol=1e-12)
    # the log-sum-exp: adding a constant to V's rows adds it to the output; scores shift with a key added to all
    o2, l2, _, _ = R.attention(q.numpy(), (k + 1.0).numpy(), v.numpy() + 3.0, 5, 0.1)
    assert np.allclose(o2, out + 3.0, atol=1e-12) and np.allclose(l2 - lse, 0.1 * q.sum(-1).numpy(), atol=1e-12)
    assert (A >= np.abs(out) - 1e-12).all() and (B > 0).all()
    o3, l3, _, _ = R.attention(q.numpy(), k[:2].numpy(), v[:2].numpy(), 5, 0.1)       # the first three tokens see nothing
    assert (o3[:3] == 0).all() and (l3[:3] == -np.inf).all() and np.allclose(o3[3], v[0].numpy())


def test_pages_form_keeps_rows_and_counts():
    """Whatever the calls, a view holds the rows that were appended to it, a page's count
    is that of the views that hold it, and free and held pages are all pages."""
    r = np.random.RandomState(4)
    s = R.Pages(60, 16, 6, 2, 12)
    rows = {(x, h): np.zeros((0, R.D), np.float32) for x in range(6) for h in range(2)}
    for _ in range(200):
        op = r.randint(4)
        if op == 0:
            slots = r.permutation(6)[:r.randint(1, 4)].tolist()
            new = r.randint(0, 25, len(slots)).tolist()
            k = r.randn(sum(new), 2, R.D).astype(np.float32)
            before = s.lens.copy()
            s.append(slots, new, k, -k)
            at = 0
            for x, m in zip(slots, new):
                grown = s.lens[x] - before[x]
                assert (grown == grown[0]).all() and grown[0] in (0, m)
                for h in range(2):
                    if grown[0]:
                        rows[x, h] = np.concatenate([rows[x, h], k[at:at + m, h]])
                at += m
        elif op == 1:
            a, b = r.permutation(6)[:2]
            s.fork([a], [b])
            for h in range(2):
                if not len(rows[b, h]):
                    rows[b, h] = rows[a, h]
        elif op == 2:
            n = r.choice([0, 0, 1, 5, 20, 1000], 6)
            s.drop(n)
            rows = {(x, h): v[:max(len(v) - n[x], 0)] for (x, h), v in rows.items()}
        else:
            x, h, tail = r.randint(6), r.randint(2), 3
            L = len(rows[x, h])
            idx = np.array([[0, 2, -1]])
            if not s.compact(x, [h], idx, 4, tail):
                keep = [t for c in (0, 2) for t in range(4 * c, min(4 * c + 4, L - tail))] + list(range(L - tail, L))
                rows[x, h] = rows[x, h][keep]
        held = np.zeros(60, np.int64)
        for (x, h), v in rows.items():
            k, w = s.rows(x, h)
            assert np.array_equal(k, v) and np.array_equal(w, -v)
            ids = s.table[x, h][s.table[x, h] >= 0]
            assert len(ids) == R.pages_of(len(v), 16) and len(set(ids.tolist())) == len(ids)
            held[ids] += 1
        assert np.array_equal(held, s.refs) and len(s.free()) == (held == 0).sum()
        assert sum(bin(int(w) & (2 ** 64 - 1)).count("1") for w in s.bits()) == len(s.free())


def test_bounds_count_the_roundings():
    """An output rounded to its type, with weights rounded to bf16, lies within them."""
    g = np.random.RandomState(2)
    q, k, v = g.randn(40, 1, R.D), g.randn(300, R.D), g.randn(300, R.D)
    out, lse, A, B = R.attention(q, k, v, 40, 1 / math.sqrt(R.D))
    bf = lambda x: torch.from_numpy(np.asarray(x)).to(torch.bfloat16).double().numpy()     # noqa: E731
    eo, _ = R.bounds(out, lse, A, B, 300, torch.bfloat16, 40)
    for j in range(40):
        s = (q[j] @ k[:261 + j].T) / math.sqrt(R.D)
        p = np.exp(s - s.max())
        o = bf(bf(p) @ v[:261 + j] / p.sum())
        assert (np.abs(o - out[j]) <= eo[j]).all() and np.abs(o - out[j]).max() > 0


@needs_lib
@pytest.mark.parametrize("slots,new,rows,error", [
    (np.array([2 ** 32, 1]), [1, 1], [[9, 9]] * 2, ValueError), ([0, 1], np.array([2 ** 32 + 1, 1]), [[9, 9]] * 2, ValueError),
    ([0, 1], torch.tensor([1, -2 ** 32 + 1]), [[9, 9]] * 2, ValueError), ([0, 1], [1, 1], np.array([[9, 9], [9, 2 ** 64 - 9]], np.uint64), ValueError),
    ([0, 1], [1.5, 1], [[9, 9]] * 2, TypeError), ([0, 1], [1, 1], torch.tensor([[9.0, 9], [9, math.nan]]), TypeError),
    ([0, 1], [1, 2 ** 70], [[9, 9]] * 2, ValueError), ([0, 1], [1, 1], [[9, 9], [9, None]], TypeError), ([[0], [1]], [1, 1], [9] * 4, None),
    (range(2), torch.tensor([1, 1]), np.full((2, 2), 9, np.uint8), None), ([torch.tensor(0), 1], [1, np.int64(1)], [[9, 9]] * 2, None), ([], [], [], None),
])
def test_the_binding_takes_whole_numbers_as_they_are(slots, new, rows, error):
    """Numbers that 32 bits do not hold, or that are none, are refused, and not cut to others."""
    c = SimpleNamespace(hkv=2, ref=ctypes.byref(cache()))
    if error:
        with pytest.raises(error):
            ck.paged_workspace(c, slots, new, rows, 8)
    else:
        want = ck.lib().catekv_paged_workspace(c.ref, i32(0, 1), i32(1, 1), i64(9, 9, 9, 9), len(slots), 8)
        assert ck.paged_workspace(c, slots, new, rows, 8) == want


@pytest.mark.skipif(not os.path.exists(os.path.join(ROOT, "README.md")), reason="a tree without its README")
def test_the_examples_of_the_readme_are_calls_that_exist():
    blocks = re.findall(r"```python\n(.*?)```", open(os.path.join(ROOT, "README.md")).read(), flags=re.S)
    calls = [x for b in blocks for x in ast.walk(ast.parse(b)) if isinstance(x, ast.Call) and isinstance(x.func, ast.Attribute)
             and getattr(x.func.value, "id", None) == "ck"]
    assert len(calls) > 15
    for x in calls:
        inspect.signature(getattr(ck, x.func.attr)).bind(*x.args, **{k.arg: k.value for k in x.keywords})

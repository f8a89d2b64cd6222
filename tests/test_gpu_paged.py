"""Caches in pages on the GPU against the plain forms of paged_ref: every call's
state bit for bit, attention within the bounds that its arithmetic allows."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


def randn(shape, seed, dtype=F32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(DEV)


def host(t):
    return t.float().cpu().numpy()


def cache_of(n_pages, page, n_slots, hkv, max_pages, dtype, seed=0):
    """An empty cache whose pages hold noise, and its mirror."""
    c = ck.paged_alloc(n_pages, page, n_slots, hkv, max_pages, DEV, dtype=dtype)
    c.k.copy_(randn(c.k.shape, seed + 1, dtype))
    c.v.copy_(randn(c.v.shape, seed + 2, dtype))
    return c, R.Pages.of(c)


def append(c, s, slots, new, hq, seed, bound=None, want_left=False):
    """The same append on the cache and its mirror; the plan."""
    bound = [[int(s.lens[x, h]) + m for h in range(c.hkv)] for x, m in zip(slots, new)] if bound is None else bound
    plan = ck.paged_plan(c, slots, new, bound, hq)
    k, v = (randn((sum(new), c.hkv, 128), seed + i, c.dtype) for i in (0, 1))
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.append_kv_paged(plan, c, k, v, over)
    left = s.append(slots, new, host(k), host(v))
    assert bool(over.item()) == left == want_left
    return plan


def check_attention(c, plan, slots, new, hq, seed, scale=None, q=None, bound=None):
    """Attention of the new tokens against the mirror's rows in 64 bits."""
    G, at = hq // c.hkv, 0
    q = randn((sum(new), hq, 128), seed, c.dtype) if q is None else q
    out, lse = ck.attn_paged(plan, c, q, scale=scale)
    assert out.dtype == c.dtype and out.shape == q.shape and lse.shape == q.shape[:2]
    got, got_lse, qh = host(out).astype(np.float64), lse.cpu().numpy().astype(np.float64), host(q)
    s, scale = R.Pages.of(c), 1 / math.sqrt(128) if scale is None else scale
    for i, (x, m) in enumerate(zip(slots, new)):
        for h in range(c.hkv):
            k, v = s.rows(x, h)
            if bound is not None:
                k, v = k[:bound[i][h]], v[:bound[i][h]]
            g = slice(h * G, (h + 1) * G)
            o, z, A, B = R.attention(qh[at:at + m, g], k, v, m, scale)
            eo, ez = R.bounds(o, z, A, B, len(k), c.dtype, m * G)
            a, b = got[at:at + m, g], got_lse[at:at + m, g]
            fin = np.isfinite(o)
            assert np.array_equal(np.isnan(o), np.isnan(a)), f"sequence {i} head {h}: NaN"
            assert np.array_equal(o[~fin & ~np.isnan(o)], a[~fin & ~np.isnan(o)]), f"sequence {i} head {h}: inf"
            err = np.where(fin, np.abs(a - np.where(fin, o, 0)), 0)
            fine = bool((err <= np.where(fin, np.nan_to_num(eo), 0)).all())
            assert fine, \
                f"sequence {i} head {h}: off by {err.max():.3g}, {np.nanmax(np.where(fin, err / eo, 0)):.3g} of the bound"
            fin = np.isfinite(z)
            assert np.array_equal(z[~fin], b[~fin], equal_nan=True), f"sequence {i} head {h}: lse {z[~fin]} {b[~fin]}"
            assert (np.abs(b[fin] - z[fin]) <= ez[fin]).all(), f"sequence {i} head {h}: lse off by {np.abs(b - z)[fin].max():.3g}"
        at += m
    return out, lse


# -------------------------------------------------------------------- the pages

@pytest.mark.parametrize("dtype,page,hkv,n_pages", [(BF16, 16, 2, 200), (F32, 64, 1, 90), (BF16, 256, 8, 70), (F32, 32, 3, 150)])
def test_append_fills_pages_in_order(dtype, page, hkv, n_pages):
    c, s = cache_of(n_pages, page, 5, hkv, 20, dtype)
    s.same(c)                                                   # init
    append(c, s, [3, 0, 4], [page + 1, 1, 0], hkv, 10)          # one sequence without new tokens
    s.same(c)
    append(c, s, [0, 1, 3], [page - 1, 2 * page, 5], hkv, 20)   # exactly to a page's end, whole pages, within one
    s.same(c)
    append(c, s, [0, 3, 2], [1, 1, 1], hkv, 30)                 # the first row of a new page
    s.same(c)


def test_append_of_more_views_than_the_taking_workgroup_has_threads():
    c, s = cache_of(3000, 16, 401, 3, 4, BF16)
    slots = list(range(400, -1, -1))
    append(c, s, slots, [1 + i % 17 for i in range(401)], 3, 1)
    s.same(c)
    append(c, s, slots, [i % 3 for i in range(401)], 3, 2)
    s.same(c)


def test_append_takes_strided_rows():
    c, s = cache_of(40, 32, 2, 4, 4, BF16)
    k, v = (randn((4, 50, 128), i, BF16) for i in (5, 6))        # [hkv][n][d], as the prompt's caches are
    plan = ck.paged_plan(c, [1], [50], [[50] * 4], 4)
    ck.append_kv_paged(plan, c, k.transpose(0, 1), v.transpose(0, 1))
    s.append([1], [50], host(k.transpose(0, 1)), host(v.transpose(0, 1)))
    s.same(c)


def test_sequences_without_pages_are_left_whole():
    c, s = cache_of(10, 16, 6, 2, 3, BF16)
    append(c, s, [0, 1], [16, 20], 2, 1)                         # 6 pages
    append(c, s, [2, 3, 1, 4, 0], [10, 30, 2, 16, 0], 2, 2, want_left=True)   # 2; then 4 of 2; 1 needs none; 4 none left
    assert s.lens[:, 0].tolist() == [16, 22, 10, 0, 0, 0]
    s.same(c)
    append(c, s, [0, 2], [40, 6], 2, 3, want_left=True)          # more than max_pages; the other goes on
    assert s.lens[:, 0].tolist() == [16, 22, 16, 0, 0, 0]
    s.same(c)
    c.lens[5, 1] = -3                                            # out of range
    s.lens[5, 1] = -3
    append(c, s, [5], [1], 2, 4, bound=[[1, 1]], want_left=True)
    s.same(c)


@pytest.mark.parametrize("dtype,page", [(BF16, 16), (F32, 64)])
def test_forks_share_until_they_write(dtype, page):
    c, s = cache_of(200, page, 8, 2, 8, dtype)
    append(c, s, [0, 1], [2 * page + 5, page], 2, 1)
    ref = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.fork_paged(c, [0, 0, 1, 7], [2, 3, 4, 5], ref)            # an empty slot's fork is empty
    assert s.fork([0, 0, 1, 7], [2, 3, 4, 5]) is False and ref.item() == 0
    s.same(c)
    append(c, s, [2, 0, 4], [1, 3, 1], 2, 5)                     # two of three holders write: copies, the third keeps
    s.same(c)
    append(c, s, [3], [1], 2, 6)                                 # the last holder writes in place
    s.same(c)
    ck.fork_paged(c, [0], [1], ref)                              # not empty: left, and said so
    assert s.fork([0], [1]) is True and ref.item() == 1
    s.same(c)
    c2, s2 = cache_of(60, page, 3, 1, 4, dtype)
    append(c2, s2, [0], [3], 1, 7)
    ck.fork_paged(c2, [0], [2])
    s2.fork([0], [2])
    append(c2, s2, [2, 0], [2, 2], 1, 8)                         # all holders write: the old page is free again
    s2.same(c2)
    assert s2.refs[0] == 0 and 0 in s2.free()


def test_drop_releases_what_no_one_holds():
    c, s = cache_of(100, 16, 5, 2, 8, BF16)
    append(c, s, [0, 1], [70, 33], 2, 1)
    ck.fork_paged(c, [0, 1], [2, 3])
    s.fork([0, 1], [2, 3])
    for rows in ([0, 1, 6, -5, 9], [70, 0, 22, 32, 0], [2 ** 62, 1, 10 ** 9, 1, 1]):
        ck.drop_paged(c, torch.tensor(rows, dtype=torch.int64, device=DEV))
        s.drop(rows)
        s.same(c)


@pytest.mark.parametrize("dtype,page,cs,tail,L", [(BF16, 16, 8, 64, 1003), (F32, 32, 1, 0, 77), (BF16, 64, 48, 5, 500),
                                                 (BF16, 256, 8, 16, 16), (F32, 16, 64, 31, 640)])
def test_compact_keeps_chunks_and_tail(dtype, page, cs, tail, L):
    hkv, need = 3, R.pages_of(L, page)
    c, s = cache_of(2 * hkv * need + 20, page, 3, hkv, need + 2, dtype)
    append(c, s, [2], [L], hkv, 1)
    ck.fork_paged(c, [2], [0])                                   # shared pages stay for the other holder
    s.fork([2], [0])
    n = max(R.pages_of(L - tail, cs), 1)
    r = np.random.RandomState(3)
    b = max(n // 3, 2)
    idx = np.full((2, b), -1, np.int32)
    if L > tail:
        idx[0, :min(b, n)] = np.sort(r.permutation(n)[:b])
        idx[1, 0] = n - 1                                        # the last chunk alone, perhaps partial
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.compact_kv_paged(c, 2, [2, 0], torch.from_numpy(idx).to(DEV), cs, tail, over)
    assert s.compact(2, [2, 0], idx, cs, tail) is False and over.item() == 0
    s.same(c)


def test_compact_takes_any_list_and_leaves_what_does_not_fit():
    c, s = cache_of(26, 16, 2, 3, 6, BF16)
    append(c, s, [1], [90], 3, 1)                                # 18 pages; 8 are left
    over = torch.zeros(1, dtype=torch.int32, device=DEV)

    def both(heads, idx, cs, tail):
        over.zero_()
        ck.compact_kv_paged(c, 1, heads, torch.tensor(idx, dtype=torch.int32, device=DEV), cs, tail, over)
        left = s.compact(1, heads, idx, cs, tail)
        assert bool(over.item()) == left
        s.same(c)
        return left
    # repeated, unordered and out-of-range chunks, gaps; the third of three does not find its pages
    assert both([0, 2, 1], [[3, 3, -1, 0, 99], [10, -1, 0, 1, 2], [0, 1, 2, 3, 4]], 8, 10)
    assert both([1], [[9, 11, 10, -1, -1]], 8, 10) is False
    assert both([0], [[-1]], 8, 91)                              # fewer rows than the tail
    assert both([0], [[0] * 20], 8, 0)                           # more rows than max_pages hold
    assert both([2], [[-1, -1]], 8, 0) is False and s.lens[1, 2] == 0


@pytest.mark.parametrize("dtype,page", [(BF16, 64), (F32, 16)])
def test_gather_writes_the_rows_and_nothing_else(dtype, page):
    c, s = cache_of(120, page, 4, 2, 10, dtype)
    append(c, s, [1, 3], [3 * page + 7, 1], 2, 1)
    ck.drop_paged(c, torch.tensor([0, 2, 0, 0], device=DEV))
    s.drop([0, 2, 0, 0])
    slots, n = [3, 1, 0, 1], 3 * page + 2                        # one slot twice, one empty, some rows too many
    outs = [[torch.full((n + 3, 128), 7.0, dtype=dtype, device=DEV) for _ in "kv"] for _ in range(8)]
    ptrs = [[t.data_ptr() for t in o] for o in outs]
    ptrs[2][1] = ptrs[5][0] = 0                                  # left out
    ck.gather_kv_paged(c, slots, ck.kv_table(ptrs, DEV), n)
    for i, x in enumerate(slots):
        for h in range(2):
            for o, rows, skip in zip(outs[2 * i + h], s.rows(x, h), (2 * i + h == 5, 2 * i + h == 2)):
                want = np.full((n + 3, 128), 7.0, np.float32)
                if not skip:
                    want[:min(len(rows), n)] = rows[:n]
                assert np.array_equal(host(o), want), (i, h)


# ------------------------------------------------------------------- attention

CASES = [
    # dtype, page, hkv, G, contexts before the append, new tokens
    (BF16, 16, 2, 4, [0], [1]),
    (BF16, 16, 1, 1, [0, 15, 16, 17], [1, 1, 1, 1]),
    (BF16, 64, 2, 4, [999], [1]),
    (BF16, 32, 2, 8, [130, 5], [2, 1]),
    (BF16, 64, 1, 8, [63, 64, 300], [3, 17, 2]),
    (BF16, 64, 2, 4, [0, 700], [257, 33]),
    (BF16, 128, 1, 2, [40, 1, 2000, 0], [130, 0, 4, 65]),
    (BF16, 256, 2, 1, [500], [300]),
    (BF16, 16, 8, 4, [63], [64]),
    (F32, 16, 2, 4, [0, 31], [1, 1]),
    (F32, 64, 1, 8, [200], [40]),
    (F32, 32, 3, 2, [100, 0], [33, 129]),
    (F32, 256, 1, 1, [1000], [5]),
]


@pytest.mark.parametrize("dtype,page,hkv,G,ctx,new", CASES)
def test_attention_of_new_tokens(dtype, page, hkv, G, ctx, new):
    need = sum(R.pages_of(a + b, page) for a, b in zip(ctx, new)) * hkv
    c, s = cache_of(need + 3, page, len(ctx) + 1, hkv, max(R.pages_of(a + b, page) for a, b in zip(ctx, new)), dtype)
    slots = list(range(len(ctx), 0, -1))
    if any(ctx):
        append(c, s, slots, ctx, hkv * G, 1)
    plan = append(c, s, slots, new, hkv * G, 3)
    s.same(c)
    c.k[s.free()] = float("nan")                                 # pages that no one holds
    c.v[s.free()] = float("inf")
    check_attention(c, plan, slots, new, hkv * G, 9)


@pytest.mark.parametrize("dtype,G,singles,long,chunk", [(BF16, 1, 60, 40, 600), (BF16, 2, 9, 900, 300), (BF16, 4, 40, 500, 150),
                                                        (BF16, 8, 3, 3000, 64), (F32, 4, 20, 300, 100)])
def test_single_tokens_beside_chunks(dtype, G, singles, long, chunk):
    """Many short and a few long sequences of 1 or 2 tokens in one batch with two chunks: workgroups
    that take more of them than they describe at a time, and chunks of views cut in several places."""
    hkv, r, page = 2, np.random.RandomState(singles), 32
    new = [chunk] + [int(x) for x in r.randint(1, 3 if 2 * G <= 16 else 2, size=singles)] + [chunk // 2 + 1]
    ctx = [1500] + [int(x) for x in r.randint(0, long, size=singles)] + [700]
    slots = [int(x) for x in r.permutation(singles + 4)[:singles + 2]]
    need = sum(hkv * R.pages_of(a + b, page) for a, b in zip(ctx, new))
    c, s = cache_of(need + 9, page, singles + 4, hkv, max(R.pages_of(a + b, page) for a, b in zip(ctx, new)) + 1, dtype)
    append(c, s, slots, ctx, hkv * G, 31)
    plan = append(c, s, slots, new, hkv * G, 33)
    check_attention(c, plan, slots, new, hkv * G, 35)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_views_cut_to_different_lengths(dtype):
    """Heads of one sequence with few rows, fewer than the new tokens, and none."""
    c, s = cache_of(200, 16, 2, 4, 30, dtype)
    append(c, s, [0], [400], 16, 1)
    plan = ck.paged_plan(c, [0], [20], [[400] * 4], 16)
    idx = np.array([[0, 3], [-1, -1], [-1, -1]], np.int32)
    ck.compact_kv_paged(c, 0, [1], torch.from_numpy(idx[:1]).to(DEV), 16, 20)
    ck.compact_kv_paged(c, 0, [2], torch.from_numpy(idx[1:2]).to(DEV), 16, 7)      # the first 13 tokens see nothing
    ck.compact_kv_paged(c, 0, [3], torch.from_numpy(idx[2:]).to(DEV), 16, 0)
    assert c.lens[0].tolist() == [400, 52, 7, 0]
    out, lse = check_attention(c, plan, [0], [20], 16, 5)
    assert (out[:, 12:] == 0).all() and (lse[:, 12:] == -math.inf).all() and (out[:13, 8:12] == 0).all()


@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 2), (BF16, 40), (F32, 3), (F32, 50)])
def test_plans_bound_the_rows(dtype, new):
    """Rows past the planned number are not looked at; fewer rows than planned are fine."""
    c, s = cache_of(100, 32, 1, 2, 20, dtype)
    append(c, s, [0], [300], 4, 1)
    bound = [[100, 301]]
    plan = ck.paged_plan(c, [0], [new], bound, 4)
    check_attention(c, plan, [0], [new], 4, 2, bound=bound)
    check_attention(c, ck.paged_plan(c, [0], [new], [[600, 299]], 4), [0], [new], 4, 3, bound=[[600, 299]])
    check_attention(c, ck.paged_plan(c, [0], [new], [[0, 640]], 4), [0], [new], 4, 3, bound=[[0, 640]])


@pytest.mark.parametrize("dtype,G,new", [(BF16, 4, 3), (BF16, 4, 70), (F32, 2, 3), (F32, 2, 70), (BF16, 8, 2)])
def test_what_a_token_does_not_see_does_not_reach_it(dtype, G, new):
    """NaN and infinities in K and V of later tokens of the chunk, and behind the view's end."""
    c, s = cache_of(40, 32, 1, 1, 12, dtype)
    append(c, s, [0], [150], G, 1)
    plan = append(c, s, [0], [new], G, 3)
    tail = R.pages_of(150 + new, 32) - 1
    r = (150 + new - 1) % 32 + 1
    c.k[s.table[0, 0, tail], r:] = float("nan")
    c.v[s.table[0, 0, tail], r:] = float("nan")
    check_attention(c, plan, [0], [new], G, 4)

    def put(row, x, k=None, v=None):
        p = s.table[0, 0, row // 32]
        if k is not None:
            c.k[p, row % 32, 5] = k
        if v is not None:
            c.v[p, row % 32, x] = v
    last = 150 + new - 1
    put(last, 3, v=float("nan"))
    put(last - 1, 9, v=float("inf"))
    put(last - 1, 100, v=float("-inf"))
    put(last, 100, v=float("inf"))
    q = randn((new, G, 128), 6, dtype)
    out, _ = check_attention(c, plan, [0], [new], G, 4, q=q)
    assert torch.isfinite(out[:new - 2].float()).all() and not torch.isfinite(out[-1, :, 3].float()).any()
    put(last, 3, v=0.5)
    put(last, 100, v=0.5)
    put(last, 0, k=float("nan"))                                  # the last token's own key
    out, _ = check_attention(c, plan, [0], [new], G, 4, q=q)
    assert torch.isnan(out[-1].float()).all() and torch.isfinite(out[:new - 2].float()).all()


@pytest.mark.parametrize("dtype,G,n,new", [(BF16, 4, 150, 1), (BF16, 2, 9000, 3), (BF16, 8, 700, 30), (BF16, 1, 9000, 300),
                                           (F32, 4, 150, 1), (F32, 1, 9000, 3), (F32, 4, 700, 30)])
def test_infinities_that_a_token_sees_are_its_result(dtype, G, n, new):
    """V of both infinities and NaN, alone and together in a dim, and K that takes rows out with a
    score of -inf, in rows that all tokens see and in the first token's own."""
    c, s = cache_of(2 * R.pages_of(n + new, 32) + 4, 32, 1, 2, R.pages_of(n + new, 32) + 1, dtype)
    append(c, s, [0], [n], 2 * G, 1)
    plan = append(c, s, [0], [new], 2 * G, 3)
    q = randn((new, 2 * G, 128), 5, dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    inf = float("inf")

    def at(row):
        return s.table[0, 0, row // 32], row % 32
    for row, dim, x in ((20, 3, inf), (40, 4, -inf), (21, 5, inf), (100, 5, -inf), (22, 6, float("nan")), (n, 7, inf)):
        p, r = at(row)
        c.v[p, r, dim] = x
    p, r = at(60)
    c.k[p, r, 0] = -inf
    out, _ = check_attention(c, plan, [0], [new], 2 * G, 5, q=q)
    o = out[:, :G].float()
    assert (o[..., 3] == inf).all() and (o[..., 4] == -inf).all() and torch.isnan(o[..., 5:7]).all() and (o[..., 7] == inf).all()
    assert torch.isfinite(o[..., 8:]).all() and torch.isfinite(out[:, G:].float()).all()


@pytest.mark.parametrize("dtype,new", [(BF16, 1), (BF16, 33), (F32, 1), (F32, 33)])
def test_scores_of_any_size(dtype, new):
    """Large and -inf scores, equal ones, a large maximum late in the view."""
    c, s = cache_of(60, 16, 1, 1, 40, dtype)
    append(c, s, [0], [400], 2, 1)
    plan = append(c, s, [0], [new], 2, 3)
    q = randn((new, 2, 128), 4, dtype)
    c.k.mul_(40)
    check_attention(c, plan, [0], [new], 2, 5, q=q)
    check_attention(c, plan, [0], [new], 2, 5, q=q, scale=1e-6)
    c.k[s.table[0, 0, 20], 3] = q[0, 0] * 100                      # one row far above the others
    check_attention(c, plan, [0], [new], 2, 5, q=q, scale=1.0)
    c.k.fill_(0)
    check_attention(c, plan, [0], [new], 2, 5, q=q)
    c.k.fill_(-3e36 if dtype == F32 else -1e36)                    # scores far below -1e30
    qp = q.abs() + 0.5
    check_attention(c, plan, [0], [new], 2, 5, q=qp.to(dtype), scale=0.01)
    c.k.fill_(float("-inf"))                                       # every row of every token
    out, lse = check_attention(c, plan, [0], [new], 2, 5, q=qp.to(dtype))
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("dtype,n,new,G", [(BF16, 100, 1, 4), (BF16, 20000, 1, 4), (BF16, 900, 60, 2), (BF16, 6000, 300, 2),
                                           (F32, 100, 2, 1), (F32, 20000, 2, 1), (F32, 900, 60, 4), (F32, 4000, 120, 4)])
def test_scores_that_are_all_nan_are_not_those_of_no_row(dtype, n, new, G):
    """A query that is NaN, in views that are one piece and in cut ones: its results are NaN,
    its neighbours' are not."""
    hkv = 2
    c, s = cache_of(2 * -(-n // 64) + 2 * -(-new // 64) + 4, 64, 1, hkv, -(-(n + new) // 64) + 1, dtype)
    append(c, s, [0], [n], hkv * G, 21)
    plan = append(c, s, [0], [new], hkv * G, 22)
    q = randn((new, hkv * G, 128), 23, dtype)
    q[new // 2, 1, 5] = float("nan")
    q[new - 1, hkv * G - 1] = float("nan")
    out, lse = check_attention(c, plan, [0], [new], hkv * G, 23, q=q)
    nan = torch.isnan(out.float()).all(-1)
    assert nan[new // 2, 1] and nan[new - 1, hkv * G - 1] and int(nan.sum()) == len({(new // 2, 1), (new - 1, hkv * G - 1)})


@pytest.mark.parametrize("dtype,n,new,G", [(BF16, 20000, 1, 4), (BF16, 9000, 4, 8), (BF16, 6000, 300, 2), (F32, 5000, 2, 1),
                                           (F32, 3001, 150, 4)])
def test_long_views_are_cut_and_joined(dtype, n, new, G):
    c, s = cache_of(R.pages_of(n + new, 64) * 2 + 1, 64, 2, 2, R.pages_of(n + new, 64), dtype)
    plan = ck.paged_plan(c, [1], [n], [[n] * 2], 2 * G)
    k, v = (randn((2, n, 128), i, dtype) for i in (1, 2))
    ck.append_kv_paged(plan, c, k.transpose(0, 1), v.transpose(0, 1))
    s = R.Pages.of(c)
    plan = append(c, s, [1], [new], 2 * G, 3)
    assert plan.plan.n_joins > 0
    check_attention(c, plan, [1], [new], 2 * G, 4)


# -------------------------------------------------------- as a program runs them

def test_a_serving_loop_under_graphs_on_another_stream():
    """Steps of append and attention captured once and replayed, between eager forks,
    drops and a second graph that shares the plan; every replay against the mirror."""
    c, s = cache_of(150, 16, 4, 2, 12, BF16)
    append(c, s, [0, 2], [37, 16], 8, 1)
    bound = [[12 * 16] * 2] * 2
    plan = ck.paged_plan(c, [2, 0], [1, 1], bound, 8)
    k, v, q = (torch.zeros((2, x, 128), dtype=BF16, device=DEV) for x in (2, 2, 8))
    out, lse = torch.zeros_like(q), torch.zeros((2, 8), device=DEV)
    side = torch.cuda.Stream()
    saved = c.book.clone()

    def step():
        ck.append_kv_paged(plan, c, k, v)
        ck.attn_paged(plan, c, q, out=out, lse=lse)
    graphs = []
    with torch.cuda.stream(side):
        step()
        side.synchronize()
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=side):
                step()
            graphs.append(g)
        c.book.copy_(saved)
        for i in range(40):
            for t, n in ((k, 0), (v, 1), (q, 2)):
                t.copy_(randn(t.shape, 100 * i + n, BF16))
            graphs[i % 2].replay()
            side.synchronize()
            s.append([2, 0], [1, 1], host(k), host(v))
            if i % 13 == 5:
                ck.fork_paged(c, [0], [1])
                s.fork([0], [1])
            if i % 13 == 9:
                rows = [4, 10 ** 6, 0, 0]
                ck.drop_paged(c, torch.tensor(rows, device=DEV))
                s.drop(rows)
            if i % 8 == 0:
                side.synchronize()
                s.same(c)
                first, first_lse = out.clone(), lse.clone()
                if i % 13 not in (9,):
                    o2, l2 = check_attention(c, plan, [2, 0], [1, 1], 8, 0, q=q)
                    assert torch.equal(o2, first) and torch.equal(l2, first_lse)
    side.synchronize()
    s.same(c)


def test_prompts_in_chunks_then_selection_then_decoding():
    """A prompt in three chunks, its rows gathered for select_critical, consistent heads
    cut back as compact_kv cuts them, and decoding on as decode_attn does."""
    n, hkv, G, cs, tail, b = 1500, 4, 4, 8, 32, 20
    hq = hkv * G
    k, v = (randn((hkv, n + 3, 128), i, BF16) for i in (1, 2))
    c, _ = cache_of(150, 64, 3, hkv, 30, BF16)
    at = 0
    for m in (700, 1, 799):
        plan = ck.paged_plan(c, [2], [m], [[at + m] * hkv], hq)
        ck.append_kv_paged(plan, c, k[:, at:at + m].transpose(0, 1), v[:, at:at + m].transpose(0, 1))
        check_attention(c, plan, [2], [m], hq, at)
        at += m
    kd, vd = (torch.zeros((hkv, n, 128), dtype=BF16, device=DEV) for _ in "kv")
    ck.gather_kv_paged(c, [2], ck.kv_table([(kd[h].data_ptr(), vd[h].data_ptr()) for h in range(hkv)], DEV), n)
    assert torch.equal(kd, k[:, :n]) and torch.equal(vd, v[:, :n])
    q_obs = randn((hq, tail, 128), 7, BF16)
    idx = ck.select_critical(q_obs, kd, [1, 3], cs, b)
    lens = torch.full((hkv,), n, dtype=torch.int64, device=DEV)
    kc, vc = ck.compact_kv(kd, vd, [1, 3], idx, cs, tail, lens)
    free = int((c.refs == 0).sum())
    ck.compact_kv_paged(c, 2, [1, 3], idx, cs, tail)
    assert torch.equal(c.lens[2], lens) and int((c.refs == 0).sum()) > free
    s = R.Pages.of(c)
    for h, i in ((1, 0), (3, 1)):
        assert np.array_equal(s.rows(2, h)[0], host(kc[i, :int(lens[h])])) and np.array_equal(s.rows(2, h)[1], host(vc[i, :int(lens[h])]))
    plan = ck.paged_plan(c, [2], [1], [[n + 3, b * cs + tail + 3] * 2], hq)
    full = [torch.cat([k[h, :n], k[h, :0]]) for h in range(hkv)]
    for t in range(3):
        ck.append_kv_paged(plan, c, k[:, n + t].unsqueeze(0), v[:, n + t].unsqueeze(0))
        check_attention(c, plan, [2], [1], hq, 50 + t)
    assert c.lens[2].tolist() == [int(x) + 3 for x in lens] and len(full) == hkv


def test_results_do_not_depend_on_the_run():
    """The same calls twice give the same bits, tables and pages among them."""
    def run():
        c, s = cache_of(400, 32, 9, 2, 40, BF16)
        append(c, s, [0, 1], [900, 333], 8, 1)
        ck.fork_paged(c, [0, 0, 1], [2, 3, 4])
        s.fork([0, 0, 1], [2, 3, 4])
        plan = append(c, s, [4, 0, 2, 3], [3, 1, 20, 1], 8, 3)
        out = ck.attn_paged(plan, c, randn((25, 8, 128), 9, BF16))
        ck.drop_paged(c, torch.tensor([5, 900, 0, 1, 400, 0, 0, 0, 0], device=DEV))
        return [c.table, c.lens, c.refs, c.free_bits, *out, c.k, c.v]
    for a, b in zip(run(), run()):
        assert torch.equal(a, b)


def test_a_handle_passes_cached_state_on_after_a_restore():
    c, s = cache_of(50, 16, 3, 2, 6, BF16)
    append(c, s, [0], [20], 4, 1)
    saved, mirror = c.book.clone(), R.Pages.of(c)
    append(c, s, [1, 0], [40, 9], 4, 2)
    c.book.copy_(saved)
    mirror.k, mirror.v = R.Pages.of(c).k, R.Pages.of(c).v        # rows stay where they were written
    append(c, mirror, [2], [17], 4, 3)
    mirror.same(c)


def test_entries_out_of_range_are_not_followed():
    """A table and lengths that no call leaves: nothing is read or written outside, and
    the other views' results stay as they are."""
    c, s = cache_of(40, 16, 4, 1, 6, BF16)
    plan = append(c, s, [0, 1, 2], [50, 50, 50], 4, 1)
    q = randn((150, 4, 128), 5, BF16)
    want, want_lse = ck.attn_paged(plan, c, q)
    c.table[0, 0, 1] = 10 ** 6
    c.table[1, 0, 0] = -7
    c.lens[1, 0] = 2 ** 40
    out, lse = ck.attn_paged(plan, c, q)
    assert torch.equal(out[100:], want[100:]) and torch.equal(lse[100:], want_lse[100:])
    assert (out[50:100] == 0).all() and (lse[50:100] == -math.inf).all()
    dense = torch.zeros((2, 96, 128), dtype=BF16, device=DEV)
    ck.gather_kv_paged(c, [2], ck.kv_table([(dense[0].data_ptr(), dense[1].data_ptr())], DEV), 96)
    assert np.array_equal(host(dense[0, :50]), s.rows(2, 0)[0])
    ck.fork_paged(c, [1], [3])
    assert c.lens[3, 0].item() == 0

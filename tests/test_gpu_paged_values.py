"""Attention over caches in pages where values are not ordinary ones: results beside
infinities of V, scores of any size, rows without weight.  Every result that is finite
has a bound that is finite, too: what a bound counts are the rows whose scores are."""
import math

import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck
from test_gpu_paged import BF16, DEV, F32, append, cache_of, host, randn

pytestmark = pytest.mark.gpu
inf = float("inf")


def reference(q, k, v, m, scale, dtype):
    """paged_ref's results and bounds, with the largest sum of |q k| taken over the rows of
    finite scores: the others have no weight and no part in a score's error."""
    out, lse, A, B = R.attention(q, k, v, m, scale)
    with np.errstate(invalid="ignore", over="ignore"):
        for j in range(m):
            n = max(len(k) - m + j + 1, 0)
            s = np.asarray(q[j], np.float64) @ np.asarray(k[:n], np.float64).T * scale
            size = np.abs(np.asarray(q[j], np.float64)) @ np.abs(np.asarray(k[:n], np.float64)).T * scale
            B[j] = np.where(np.isfinite(s), size, 0).max(axis=1, initial=0)
        eo, ez = R.bounds(out, lse, A, B, len(k), dtype, q.shape[0] * q.shape[1])
    assert np.isfinite(eo[np.isfinite(out)]).all() and np.isfinite(ez[np.isfinite(lse)]).all(), "a bound that holds nothing"
    return out, lse, eo, ez


def check(c, plan, q, new, G, scale=None):
    """Attention of slot 0's new tokens against the rows that the cache holds, in 64 bits."""
    got, lse = ck.attn_paged(plan, c, q, scale=scale)
    s, scale = R.Pages.of(c), 1 / math.sqrt(128) if scale is None else scale
    a, b, qh = host(got).astype(np.float64), lse.cpu().numpy().astype(np.float64), host(q)
    for h in range(c.hkv):
        k, v = s.rows(0, h)
        g = slice(h * G, (h + 1) * G)
        o, z, eo, ez = reference(qh[:, g], k, v, new, scale, c.dtype)
        x, y, fin = a[:, g], b[:, g], np.isfinite(o)
        wrong = ~(np.isnan(o) & np.isnan(x) | (o == x)) & ~fin
        assert not wrong.any(), f"head {h}: {[(w.tolist(), o[tuple(w)], x[tuple(w)]) for w in np.argwhere(wrong)[:4]]}"
        err = np.where(fin, np.abs(x - np.where(fin, o, 0)), 0)
        fine = err <= np.where(fin, eo, 0)
        assert fine.all(), f"head {h}: off by {err[~fine].max():.3g} {np.argwhere(~fine)[:4].tolist()}"
        fin = np.isfinite(z)
        assert np.array_equal(z[~fin], y[~fin], equal_nan=True), f"head {h}: lse"
        assert (np.abs(y[fin] - z[fin]) <= ez[fin]).all(), f"head {h}: lse off by {np.abs(y - z)[fin].max():.3g}"
    return got, lse


def view(dtype, n, new, G, hkv=1, page=32, seed=1):
    """Slot 0 with n rows and `new` more; put(row, head, k, v, dim) changes its rows' elements."""
    need = R.pages_of(n + new, page)
    c, s = cache_of(hkv * need + 3, page, 1, hkv, need, dtype)
    plan = ck.paged_plan(c, [0], [n], [[n] * hkv], hkv * G)
    rows = [randn((n, hkv, 128), seed + i, dtype) for i in (0, 1)]
    ck.append_kv_paged(plan, c, *rows)
    s = R.Pages.of(c)
    plan = append(c, s, [0], [new], hkv * G, seed + 2)
    table = s.table[0]

    def put(row, k=None, v=None, dim=slice(None), head=0):
        p, r = int(table[head, row // page]), row % page
        if k is not None:
            c.k[p, r, dim] = k
        if v is not None:
            c.v[p, r, dim] = v
    return c, plan, put


FORMS = [(BF16, 4, 60, 1), (BF16, 4, 150, 1), (BF16, 2, 9000, 3), (BF16, 8, 70000, 1), (BF16, 8, 700, 30), (BF16, 1, 9000, 300),
         (F32, 4, 60, 1), (F32, 4, 150, 1), (F32, 1, 9000, 3), (F32, 4, 40000, 1), (F32, 4, 700, 30), (F32, 2, 3000, 130)]


@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_finite_results_beside_infinities(dtype, G, n, new):
    """V of both infinities and NaN in some dims, rows that all tokens see and the last ones':
    the other dims and the log-sum-exp are what they are without."""
    c, plan, put = view(dtype, n, new, G, hkv=2)
    q = randn((new, 2 * G, 128), 5, dtype)
    for row, dim, x in ((20, 3, inf), (40, 4, -inf), (21, 5, inf), (n - 1, 5, -inf), (22, 6, math.nan), (n, 7, inf), (n + new - 1, 8, -inf)):
        put(row, v=x, dim=dim)
    out, _ = check(c, plan, q, new, G)
    assert torch.isfinite(out[:, :G, 9:].float()).all() and torch.isfinite(out[:, G:].float()).all()


@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_equal_scores_of_any_size_weigh_the_same(dtype, G, n, new):
    """All keys the same, scores of 1e-30 to -1e38: the mean of what a token sees of V, within
    what sums and the result's rounding add (weights are exactly 1)."""
    c, plan, put = view(dtype, n, new, G)
    q = (randn((new, G, 128), 5).abs() + 0.5).to(dtype)
    v = R.Pages.of(c).rows(0, 0)[1].astype(np.float64)
    mean = np.cumsum(v, axis=0)[n:] / np.arange(n + 1, n + new + 1)[:, None]
    size = np.cumsum(np.abs(v), axis=0)[n:] / np.arange(n + 1, n + new + 1)[:, None]
    half = torch.finfo(dtype).eps / 2
    bound = 2 * (n + new + 200) * 2.0 ** -24 * size + half * np.abs(mean) + 1e-30
    for x, scale in ((-1e36, 0.01), (-1e36, 0.7), (-3e9, 1.0), (1e20, 0.125), (1e-30, 0.125)):
        c.k.fill_(x)
        out, lse = ck.attn_paged(plan, c, q, scale=scale)
        err = np.abs(host(out).astype(np.float64) - mean[:, None])
        assert (err <= bound[:, None] * 1.01).all(), f"{x} {scale}: off by {err.max():.3g}"
        z = (host(q).astype(np.float64).sum(-1) * float(c.k[0, 0, 0]) * scale) + np.log(np.arange(n + 1, n + new + 1))[:, None]
        off = np.abs(lse.cpu().numpy() - z)
        assert (off <= 140 * 2.0 ** -24 * np.abs(z) + 2 * (n + new + 200) * 2.0 ** -24).all(), f"{x} {scale}: lse off by {off.max():.3g}"


def neighbours(scale):
    """Scores as far below 0 as fp32 still tells apart by 64 powers of two and more: one, and the
    next above it, whose products with the scale round to the same number."""
    c = np.float32(1.4426950408889634) * np.float32(scale)
    for i in range(1, 4096):
        x = -np.float32(2.0 ** 34) * np.float32(1 + i / 4096)
        up = np.nextafter(x, np.float32(0))
        if x * c == up * c:
            return float(x), float(up) - float(x)
    raise AssertionError("no such pair")


@pytest.mark.parametrize("at", [0.1, 0.5, 1.0])
@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_the_larger_of_two_huge_scores_wins(dtype, G, n, new, at):
    """Scores one step of fp32 apart, far from 0: the row that has the larger one is the result,
    also where it meets the others only as a part's or a wave's maximum."""
    scale = 0.125
    base, step = neighbours(scale)
    c, plan, put = view(dtype, n, new, G)
    q = torch.zeros((new, G, 128), dtype=dtype, device=DEV)
    q[..., :8] = 1
    hi = np.float32(torch.tensor(base).to(BF16).float().item())   # base in parts that bf16 holds
    lo = np.float32(base) - hi
    assert np.float32(torch.tensor(float(lo)).to(BF16).float().item()) == lo and np.float32(hi) + lo == np.float32(base)
    c.k.zero_()
    c.k[..., 0], c.k[..., 1] = float(hi), float(lo)
    win = int(at * (n - 1))
    put(win, k=step, dim=2)
    out, lse = ck.attn_paged(plan, c, q, scale=scale)
    v = host(c.v)[int(c.table[0, 0, win // 32]), win % 32].astype(np.float64)
    # the others: n + new of them at most, 2^-32 each
    err = np.abs(host(out).astype(np.float64) - v)
    assert (err <= torch.finfo(dtype).eps / 2 * np.abs(v) + (n + new) * 2.0 ** -32 * 8 + 2.0 ** -22 * np.abs(v)).all(), f"off by {err.max():.3g}"
    z = (base + step) * scale
    assert (np.abs(lse.cpu().numpy() - z) <= 2.0 ** -22 * abs(z)).all()


@pytest.mark.parametrize("at", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_infinities_in_rows_of_next_to_no_weight(dtype, G, n, new, at):
    """Infinite V in rows whose scores lie about 200 powers of two below one row's, in every part
    of the view: a weight that no fp32 number holds is still one, and its product infinite."""
    c, plan, put = view(dtype, n, new, G)
    q = randn((1, G, 128), 5, dtype).expand(new, -1, -1).contiguous()
    top = int(at * (n - G))
    for g in range(G):                                            # a row for every head of the group
        put(top + g, k=(q[0, g].float() * 12.4).to(dtype))
    rows = sorted({int(x) for x in np.linspace(0, n - 1, 120)} - set(range(top, top + G)))[:120]
    for i, row in enumerate(rows):
        put(row, v=inf if i % 2 else -inf, dim=i)
    put(rows[3], v=-inf, dim=len(rows) + 1)                       # and both in one dim
    put(rows[-3], v=inf, dim=len(rows) + 1)
    out, _ = check(c, plan, q, new, G)
    o = out.float()
    assert torch.isinf(o[..., :len(rows)]).all() and torch.isnan(o[..., len(rows) + 1]).all()
    assert torch.isfinite(o[..., len(rows) + 2:]).all()


@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_infinities_in_rows_without_weight(dtype, G, n, new):
    """A score of -inf is a weight of 0, and 0 times an infinity NaN, wherever the row lies: in
    single rows, and in a stretch of them that fills tiles and parts.  Where every score is
    -inf the result is 0."""
    c, plan, put = view(dtype, n, new, G, hkv=2)
    q = randn((new, 2 * G, 128), 5, dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    rows = sorted(({int(x) for x in np.linspace(0, n - 1, 60)} | {n, n + new - 1}) - {5})
    for i, row in enumerate(rows):
        put(row, k=-inf, dim=0)
        put(row, v=inf if i % 2 else -inf, dim=i)
    put(5, v=inf, dim=80)                                         # a row of ordinary weight
    for row in range(n // 4, n // 4 + min(n // 2, 400)):
        put(row, k=-inf, dim=0)
    put(n // 4 + 3, v=inf, dim=81)
    check(c, plan, q, new, G)
    for p in c.table[0, 0].tolist():
        c.k[p, :, 0] = -inf
    out, lse = check(c, plan, q, new, G)
    assert (out[:, :G] == 0).all() and (lse[:, :G] == -inf).all()


@pytest.mark.parametrize("dtype,G,singles,long,chunk", [(BF16, 1, 60, 40, 600), (BF16, 2, 9, 900, 300), (BF16, 4, 60, 500, 150), (BF16, 8, 300, 40, 3),
                                                        (BF16, 4, 400, 300, 2), (F32, 4, 60, 300, 100), (F32, 2, 300, 200, 3)])
def test_values_that_are_not_finite_all_over_a_batch(dtype, G, singles, long, chunk):
    """Sequences of all lengths in one batch, chunks beside few tokens, where one row in twenty has
    an infinity or NaN in V and one in forty scores of -inf, rows behind the views' ends among them."""
    hkv, r, page = 2, np.random.RandomState(singles), 32
    new = [chunk] + [int(x) for x in r.randint(1, 3 if 2 * G <= 16 else 2, size=singles)] + [chunk // 2 + 1]
    ctx = [1500] + [int(x) for x in r.randint(0, long, size=singles)] + [700]
    slots = [int(x) for x in r.permutation(singles + 4)[:singles + 2]]
    need = sum(hkv * R.pages_of(a + b, page) for a, b in zip(ctx, new))
    c, s = cache_of(need + 9, page, singles + 4, hkv, max(R.pages_of(a + b, page) for a, b in zip(ctx, new)) + 1, dtype)
    append(c, s, slots, ctx, hkv * G, 31)
    plan = append(c, s, slots, new, hkv * G, 33)
    k, v = c.k.view(-1, 128), c.v.view(-1, 128)
    rows = r.permutation(len(v))
    for i, x in enumerate((inf, -inf, math.nan, inf, inf, -inf)):
        at = torch.from_numpy(rows[i::120].copy()).to(DEV)
        v[at, torch.from_numpy(r.randint(0, 100, size=len(at))).to(DEV)] = x
    k[torch.from_numpy(rows[::40].copy()).to(DEV), 0] = -inf
    q = randn((sum(new), hkv * G, 128), 35, dtype)
    q[..., 0] = q[..., 0].abs() + 0.5
    out, lse = ck.attn_paged(plan, c, q)
    s, at = R.Pages.of(c), 0
    got, got_lse, qh = host(out).astype(np.float64), lse.cpu().numpy().astype(np.float64), host(q)
    for i, (slot, m) in enumerate(zip(slots, new)):
        for h in range(hkv):
            g = slice(h * G, (h + 1) * G)
            o, z, eo, ez = reference(qh[at:at + m, g], *s.rows(slot, h), m, 128 ** -0.5, dtype)
            x, y, fin = got[at:at + m, g], got_lse[at:at + m, g], np.isfinite(o)
            assert ((x == o) | (np.isnan(x) & np.isnan(o)))[~fin].all(), f"sequence {i} of {ctx[i]} + {m} head {h}: {np.argwhere(~fin & (x != o))[:4].tolist()}"
            assert (np.abs(x - o)[fin] <= eo[fin]).all(), f"sequence {i} of {ctx[i]} + {m} head {h}"
            fin = np.isfinite(z)
            assert np.array_equal(z[~fin], y[~fin], equal_nan=True) and (np.abs(y - z)[fin] <= ez[fin]).all(), f"sequence {i} head {h}: lse"
        at += m


@pytest.mark.parametrize("dtype,G,n,new", FORMS)
def test_a_score_of_plus_infinity_is_nan(dtype, G, n, new):
    """inf - inf in the softmax: NaN for the tokens that see the row, wherever it lies, and nothing
    for those that do not; finite scores as large as fp32 holds are none."""
    for row in (n // 2, n + new - 1):
        c, plan, put = view(dtype, n, new, G, hkv=2)
        q = randn((new, 2 * G, 128), 5, dtype)
        q[..., 0] = q[..., 0].abs() + 0.5
        put(row, k=inf, dim=0)
        put(3, k=-inf, dim=0, head=1)
        out, lse = check(c, plan, q, new, G)
        sees = torch.arange(n, n + new, device=DEV) >= row
        assert torch.isnan(out[sees, :G].float()).all() and torch.isnan(lse[sees, :G]).all()
        assert torch.isfinite(out[~sees].float()).all() and torch.isfinite(out[:, G:].float()).all()

"""Attention with weights where scores are not finite or far below zero, and views
whose lengths are out of range, on the GPU."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_30295_amd as ck
from test_gpu_cache import D, DEV, DT, Dense, Eight, accs, dense, lens_of, same

pytestmark = pytest.mark.gpu
KINDS = ["int8", "e4m3", "bf16", "f32"]
BLOCK = 64


def attend(kind, rows, q, plan_lens, hkv, table, decay, lens=None):
    """Attention with weights over views of the given (k, v), by the call of that kind:
    (out, lse, the rows as the views hold them)."""
    dtype = kind if kind in DT else "bf16"
    plan = ck.decode_plan(plan_lens, q.shape[1], hkv, DEV)
    n = [len(k) for k, _ in rows]
    lens = lens_of(*n) if lens is None else lens
    if kind in DT:
        d = Dense(np.random.default_rng(0), n, dtype)
        for i, (k, v) in enumerate(rows):
            d.k[i][:n[i]], d.v[i][:n[i]] = torch.from_numpy(k).to(DT[dtype]), torch.from_numpy(v).to(DT[dtype])
        return (*ck.decode_attn_weights(plan, q, d.table, lens, table, decay=decay), [d.host(i) for i in range(len(n))])
    q8 = Eight([m + BLOCK for m in n], kind, BLOCK, dtype)
    for i, (k, v) in enumerate(rows):
        q8.fill(i, k, v)
    return (*ck.decode_attn_q8(plan, q, q8.views, lens, acc=table, decay=decay), [q8.host(i, m) for i, m in enumerate(n)])


def stored(rng, n, dtype):
    return dense(rng, n, dtype).double().numpy()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_score_minus_infinity_gather_no_weight(kind):
    """K = -inf in a dimension where every query is positive: such rows have weight 0, and a
    view of nothing else has output 0, log-sum-exp -inf and weights decay * acc.  A block
    that holds an infinity reads as NaN, and so the 8-bit views have theirs in the tails."""
    rng = np.random.default_rng(51)
    dtype, decay, hkv, G = kind if kind in DT else "bf16", 0.5, 2, 4
    n = [1, 50, 63, 37] if kind in ("int8", "e4m3") else [1, 1000, 300, 37]
    gone = [np.ones(1, bool), np.ones(n[1], bool), rng.random(n[2]) < 0.5, np.zeros(n[3], bool)]
    rows = [(stored(rng, m, dtype), stored(rng, m, dtype)) for m in n]
    for (k, _), g in zip(rows, gone):
        k[g, 0] = -math.inf
    q = torch.from_numpy(rng.standard_normal((2, hkv * G, D)).astype(np.float32))
    q[..., 0] = q[..., 0].abs() + 0.5
    q = q.to(DT[dtype]).to(DEV)
    a, a0, table = accs(rng, n)
    out, lse, held = attend(kind, rows, q, n, hkv, table, decay)
    qd = q.double().cpu().numpy()
    for i, (k, v) in enumerate(held):
        b, h = divmod(i, hkv)
        heads = slice(h * G, (h + 1) * G)
        left = ~gone[i]
        want, wl, w, sa, pv = R.attend(qd[b, heads], k[left], v[left], 1 / math.sqrt(D))
        got, gl = out[b, heads].double().cpu().numpy(), lse[b, heads].double().cpu().numpy()
        new, old = a[i].double().cpu().numpy(), a0[i].double().cpu().numpy()
        if not left.any():
            assert not got.any() and np.isneginf(gl).all(), i
        else:
            m = int(left.sum())
            assert (np.abs(got - want) <= R.output_error(sa, m) * pv + 2.0 ** -24 * np.abs(want)).all(), i
            assert (np.abs(gl - wl) <= R.score_error(sa) + 2.0 ** -22 * (1 + np.abs(wl)) + R.weight_error(sa, m)).all(), i
            ref = decay * old[:n[i]][left] + w
            assert (np.abs(new[:n[i]][left] - ref) <= R.weight_error(sa, m) * w + 2.0 ** -23 * np.abs(ref)).all(), i
        # half of what was there, exactly
        assert np.array_equal(new[:n[i]][gone[i]], 0.5 * old[:n[i]][gone[i]]), i
        assert np.array_equal(new[n[i]:], old[n[i]:]), i


@pytest.mark.parametrize("kind", KINDS)
def test_scores_far_below_zero(kind):
    """Rows that are all alike and score about -10^34, which an fp32 holds: every one has
    weight 1 / n.

    Tolerances, u = 2^-24: a score is one product with at most 8 roundings (the product, the
    scale's two, the 8-bit factor's three, ln 2 and log2 e), the rows' scores are the same
    bits, so that P is the same number p for all.  An output sums n products p V and
    divides by n p: at most n + 8 roundings of sum |V| / n.  A weight is p / (4 n p) four
    times: 12 roundings, exp2's two units in the last place among them, and those of
    decay * acc + weight."""
    rng = np.random.default_rng(52)
    dtype, hkv, G, u = kind if kind in DT else "bf16", 2, 4, 2.0 ** -24
    # in 8 bits either all rows are codes or all lie in the tail, which scores the row's own value
    n = [1, 20, 64, 192] if kind in ("int8", "e4m3") else [1, 300, 17, 64]
    rows = []
    for m in n:
        k = np.zeros((m, D))
        k[:, 5] = -1e18
        rows.append((torch.from_numpy(k).to(DT[dtype]).double().numpy(), stored(rng, m, dtype)))
    q = torch.zeros((2, hkv * G, D))
    q[..., 5] = 1e17
    q = q.to(DT[dtype]).to(DEV)
    a, a0, table = accs(rng, n)
    out, lse, held = attend(kind, rows, q, n, hkv, table, 1.0)
    qd = q.double().cpu().numpy()
    for i, (k, v) in enumerate(held):
        b, h = divmod(i, hkv)
        heads, m = slice(h * G, (h + 1) * G), n[i]
        want, wl, w, _, pv = R.attend(qd[b, heads], k, v, 1 / math.sqrt(D))
        assert wl.max() < -1e33 and np.allclose(w, 1 / m, rtol=1e-12)
        got, gl = out[b, heads].double().cpu().numpy(), lse[b, heads].double().cpu().numpy()
        assert (np.abs(got - want) <= (m + 8) * u * pv).all(), i
        assert (np.abs(gl - wl) <= 8 * u * np.abs(wl)).all(), i
        ref = a0[i].double().cpu().numpy()
        ref[:m] += w
        assert (np.abs(a[i].double().cpu().numpy() - ref)[:m] <= 12 * u * w + 2 * u * ref[:m]).all(), i
        assert same(a[i][m:], a0[i][m:]), i


@pytest.mark.parametrize("kind", KINDS)
def test_views_of_negative_length_are_empty(kind):
    """Whatever the low 32 bits of the length say."""
    rng = np.random.default_rng(53)
    dtype = kind if kind in DT else "bf16"
    n = [500, 500, 500, 500, 3000, 3000]
    rows = [(stored(rng, m, dtype), stored(rng, m, dtype)) for m in n]
    lens = lens_of(-1, 500, -2 ** 33 + 300, -2 ** 62 + 17, -2 ** 40 + 2900, 3000)
    q = dense(rng, 24, dtype).view(3, 8, D).to(DEV)
    a, a0, table = accs(rng, n)
    out, lse, held = attend(kind, rows, q, n, 2, table, 1.0, lens)
    for i, m in enumerate(lens.tolist()):
        b, h = divmod(i, 2)
        heads = slice(4 * h, 4 * h + 4)
        if m < 0:
            assert same(a[i], a0[i]) and not out[b, heads].any() and torch.isneginf(lse[b, heads]).all(), i
        else:
            k, v = held[i]
            _, _, w, sa, _ = R.attend(q[b, heads].double().cpu().numpy(), k, v, 1 / math.sqrt(D))
            new, ref = (x[i][:m].double().cpu().numpy() for x in (a, a0))
            ref = ref + w
            assert (np.abs(new - ref) <= R.weight_error(sa, m) * w + 2.0 ** -23 * ref).all(), i

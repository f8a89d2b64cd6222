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

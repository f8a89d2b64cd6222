"""What eviction and conversion leave alone, and all that they move, on the GPU: K and V,
rows and weights behind the views, long views, large chunks and offsets beyond 32 bits."""
import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_30295_amd as ck
from test_gpu_cache import DEV, DT, D, Dense, Eight, acc_rows, lens_of, same

pytestmark = pytest.mark.gpu


def remaining(acc, budget, cs, recent):
    """R.evict for views of many chunks: the source row of every remaining row."""
    L = len(acc)
    nc = max(L - recent, 0) // cs
    if budget < 0 or nc <= budget:
        return np.arange(L)
    chunks = acc[:nc * cs].astype(np.float64).reshape(nc, cs)
    nan = np.isnan(chunks).any(axis=1)
    best = np.where(nan, 0.0, np.where(np.isnan(chunks), 0.0, chunks).max(axis=1))
    stay = np.sort(np.lexsort((np.arange(nc), -best, ~nan))[:budget])
    place = np.arange(budget)
    place[np.setdiff1d(place, stay)] = stay[stay >= budget]
    return np.concatenate([(place[:, None] * cs + np.arange(cs)).reshape(-1), np.arange(nc * cs, L)])


@pytest.mark.parametrize("kind", ["any", "special", "ties"])
def test_the_fast_form_is_the_plain_one(kind):
    rng = np.random.default_rng(60)
    for n, cs, recent, budget in ((300, 1, 0, 100), (777, 8, 50, 30), (50, 64, 0, 0), (50, 5, 60, 1), (200, 3, 7, -1), (90, 9, 0, 0)):
        acc = acc_rows(rng, n, kind)
        assert np.array_equal(remaining(acc, budget, cs, recent), R.evict(acc, budget, cs, recent)), (n, cs)


def check_dense_eviction(lens, dtype, kind, budget, cs, recent, max_rows, seed):
    """One eviction of views of these lengths, and everything around them, against the plain form."""
    rng = np.random.default_rng(seed)
    d = Dense(rng, lens, dtype, room=5)
    for x in d.k + d.v:      # content by row, so that a wrong row or buffer shows (bits, no numbers)
        x.view(torch.int16).random_(-30000, 30000)
    a = [torch.from_numpy(np.concatenate([acc_rows(rng, n, kind), np.full(6, 9.0, np.float32)])).to(DEV) for n in lens]
    k0, v0, a0 = [x.clone() for x in d.k], [x.clone() for x in d.v], [x.clone() for x in a]
    new = d.lens.clone()
    ck.evict_kv(d.table, new, ck.acc_table([x.data_ptr() for x in a], DEV),
                torch.tensor(budget, dtype=torch.int32, device=DEV), cs=cs, recent=recent, max_rows=max_rows, dtype=DT[dtype])
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        rows = remaining(a0[i][:n].cpu().numpy(), budget[i], cs, recent)
        m, at = len(rows), torch.from_numpy(rows).to(DEV)
        assert int(new[i]) == m, (i, n)
        for x, x0 in ((d.k[i], k0[i]), (d.v[i], v0[i])):
            assert same(x[:m], x0[at]) and same(x[m:], x0[m:]), (i, n)
        assert same(a[i][:m], a0[i][at]) and not a[i][m:n].any() and bool((a[i][n:] == 9).all()), (i, n)


@pytest.mark.parametrize("kind", ["any", "special", "ties"])
@pytest.mark.parametrize("dtype,n,cs,budget", [("bf16", 16385, 1, 5000), ("f32", 40000, 1, 32768), ("bf16", 70001, 1, 60000),
                                               ("f32", 70001, 3, 100), ("bf16", 300000, 8, 5000)])
def test_long_views(kind, dtype, n, cs, budget):
    # chunks counted by one workgroup and by many, a short view and one that stays beside the long ones
    check_dense_eviction([n, 100, n, n - 777], dtype, kind, [budget, 20, -1, budget // 2], cs, 50, n, 61)


@pytest.mark.parametrize("dtype,cs,recent,max_rows", [("bf16", 5000, 0, 61000), ("f32", 4097, 100, 61000),
                                                      ("bf16", 2049, 3, 61000), ("bf16", 8192, 9000, 1 << 20),
                                                      ("bf16", 70000, 0, 61000), ("bf16", 3000, 0, 16384)])
def test_large_chunks(dtype, cs, recent, max_rows):
    # from one chunk per workgroup of the keys to none at all
    lens = [n for n in (61000, 60000, 4 * cs, 4 * cs - 1, 5, 0) if n <= max_rows]
    lens = [min(n, 61000) for n in lens]
    check_dense_eviction(lens, dtype, "any", [2, 0, 3, 1, 1, 0][:len(lens)], cs, recent, max_rows, 62)


@pytest.mark.parametrize("dtype,recent,max_rows", [("bf16", 1024, 2304), ("f32", 1024, 2304), ("bf16", 8192, 40000),
                                                   ("f32", 20000, 40000)])
def test_many_rows_behind_the_chunks(dtype, recent, max_rows):
    # shifted over places that are sources, over each other, and by more than their number
    lens = [min(max_rows, recent + x) for x in (1, 9, 640, 1279, 1280, 16000)]
    check_dense_eviction(lens, dtype, "any", [0, 0, 70, 40, 1, 5], 8, recent, max_rows, 63)


@pytest.mark.parametrize("fmt,dtype,block,cs", [("int8", "bf16", 32, 4128), ("e4m3", "f32", 64, 8192)])
def test_large_chunks_of_8_bit_views(fmt, dtype, block, cs):
    rng = np.random.default_rng(64)
    lens = [33000, 32768, 2 * cs + block + 7, 90]
    q8 = Eight(lens, fmt, block, dtype)
    for p in q8.p:
        for name in ("k", "v"):
            p[name].random_(0, 120)
        for name in ("ks", "vs"):
            p[name].uniform_()
    a = [torch.from_numpy(acc_rows(rng, n, "any")).to(DEV) for n in lens]
    a0, old, new = [x.clone() for x in a], [q8.state(i) for i in range(4)], lens_of(*lens)
    budget = [1, 2, 0, 0]
    ck.evict_kv_q8(q8.views, new, ck.acc_table([x.data_ptr() for x in a], DEV),
                   torch.tensor(budget, dtype=torch.int32, device=DEV), cs=cs, recent=20, max_rows=33000)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        rows = remaining(a0[i].cpu().numpy(), budget[i], cs, 20)
        m, nb, at = len(rows), len(rows) // block, torch.from_numpy(rows).to(DEV)
        assert int(new[i]) == m and same(a[i][:m], a0[i][at]) and not a[i][m:].any(), i
        was = dict(zip(Eight.PARTS, old[i]))
        for name in ("k", "v"):
            assert same(q8.p[i][name][:nb * block], was[name][at[:nb * block]]), (i, name)
            assert same(q8.p[i][name][nb * block:], was[name][nb * block:]), (i, name)
            s = name + "s"
            assert same(q8.p[i][s][:nb], was[s][at[:nb * block:block] // block]) and same(q8.p[i][s][nb:], was[s][nb:]), (i, s)
            assert same(q8.p[i][name + "t"], was[name + "t"]), (i, name)


@pytest.mark.parametrize("fmt,dtype", [("int8", "bf16"), ("e4m3", "f32")])
def test_dequantize_leaves_views_out_of_range_alone(fmt, dtype):
    rng = np.random.default_rng(65)
    n = [40, 200, 64, 100]
    q8, out = Eight([256] * 4, fmt, 32, dtype), Dense(rng, n, dtype)
    for i, m in enumerate(n):
        q8.fill(i, *(rng.standard_normal((2, m, D))).astype(np.float32).astype(np.float64))
    before = [x.clone() for x in out.k + out.v]
    ck.dequantize_kv(q8.views, lens_of(40, 200, -5, 100), out.table, 100)
    torch.cuda.synchronize()
    for x, x0, i in zip(out.k + out.v, before, (0, 1, 2, 3) * 2):
        if i in (1, 2):
            assert same(x, x0), i
        else:
            assert not same(x[:n[i]], x0[:n[i]]) and same(x[n[i]:], x0[n[i]:]), i


def test_eviction_beyond_32_bits_moves_v_and_leaves_the_tails():
    # one view of 34 million rows of codes: its last chunks hold the weight
    n, block = 34_000_123, 64
    q8 = ck.q8_alloc([n], DEV, fmt="e4m3", block=block, dtype=torch.bfloat16)
    g = torch.Generator(device=DEV).manual_seed(66)
    for t in q8.hold[:2]:
        t.view(torch.uint8).random_(0, 120, generator=g)
    for t in q8.hold[2:]:
        t.uniform_(generator=g)
    nc = (n - 100) // block
    acc = torch.rand(n, generator=g, device=DEV)
    heavy = torch.arange(nc - 300, nc, 3, device=DEV)
    acc[heavy * block + 5] = 2.0
    was, old, lens = acc.clone(), [t.clone() for t in q8.hold], lens_of(n)
    ck.evict_kv_q8(q8, lens, ck.acc_table([acc.data_ptr()], DEV), torch.tensor([100], dtype=torch.int32, device=DEV), cs=block,
                   recent=100, max_rows=n)
    # the hundred heavy chunks take the hundred places, the rest follows
    at = torch.cat([(heavy[:, None] * block + torch.arange(block, device=DEV)).view(-1), torch.arange(nc * block, n, device=DEV)])
    m = at.numel()
    assert int(lens[0]) == m and int(heavy[0]) * block * D > 2 ** 32
    nb = m // block
    for i in (0, 1):
        assert same(q8.hold[i][:nb * block], old[i][at[:nb * block]]) and same(q8.hold[i][nb * block:], old[i][nb * block:]), i
        assert same(q8.hold[2 + i][:nb], old[2 + i][at[:nb * block:block] // block]), i
        assert same(q8.hold[2 + i][nb:], old[2 + i][nb:]) and same(q8.hold[4 + i], old[4 + i]), i
    assert same(acc[:m], was[at]) and not acc[m:].any()

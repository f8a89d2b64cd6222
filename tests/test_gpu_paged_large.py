"""Caches in pages whose pools and batches pass 32-bit offsets, calls of two caches at
once, and batches without tokens."""
import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck
from test_gpu_paged import append, cache_of

pytestmark = pytest.mark.gpu
DEV, F32, BF16 = "cuda", torch.float32, torch.bfloat16


def randn(shape, seed, dtype=F32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).to(dtype)


def near(out, lse, q, k, v, m, dtype, scale=128 ** -0.5):
    """out, lse of one view's group [m][G] against 64 bits within the bounds of csrc's arithmetic."""
    o, z, A, B = R.attention(q.float().cpu().numpy(), k.float().cpu().numpy(), v.float().cpu().numpy(), m, scale)
    eo, ez = R.bounds(o, z, A, B, len(k), dtype, m * q.shape[1])
    assert (np.abs(out.double().cpu().numpy() - o) <= eo).all()
    assert (np.abs(lse.double().cpu().numpy() - z) <= ez).all()


@pytest.mark.parametrize("dtype,page,n_pages", [(BF16, 64, 300000), (F32, 256, 40000)])
def test_pools_of_more_than_4_gib(dtype, page, n_pages):
    """Only pages behind the 4 GiB border are free (those of bf16 lie past the first 65536,
    too): rows appended, attended to, shared, copied on writing, cut back and gathered."""
    hkv, G, n, m = 2, 4, 2500, 70
    c = ck.paged_alloc(n_pages, page, 3, hkv, 64, DEV, dtype=dtype)
    first = -(-(1 << 32) // (page * 128 * c.k.element_size())) + 1
    assert first < n_pages - 300 and c.k.numel() * c.k.element_size() > 1 << 32
    c.refs[:first] = 1
    free = np.zeros(-(-n_pages // 64) * 64, np.uint64)
    free[first:n_pages] = 1
    c.free_bits.copy_(torch.from_numpy((free.reshape(-1, 64) << np.arange(64, dtype=np.uint64)).sum(axis=1, dtype=np.uint64).view(np.int64)))
    k, v = (randn((n + 2 * m, hkv, 128), i, dtype) for i in (1, 2))
    q = randn((n + 2 * m, hkv * G, 128), 3, dtype)
    over = torch.zeros(1, dtype=torch.int32, device=DEV)

    def add(slot, lo, hi, rows):
        plan = ck.paged_plan(c, [slot], [hi - lo], [[rows] * hkv], hkv * G)
        ck.append_kv_paged(plan, c, k[lo:hi], v[lo:hi], over)
        return ck.attn_paged(plan, c, q[lo:hi])

    def rows_of(slot, rows):
        out = torch.zeros((2, hkv, rows, 128), dtype=dtype, device=DEV)
        ck.gather_kv_paged(c, [slot], ck.kv_table([[out[0, h].data_ptr(), out[1, h].data_ptr()] for h in range(hkv)], DEV), rows)
        return out.transpose(1, 2)

    add(0, 0, n, n)
    ck.fork_paged(c, [0], [1])
    for slot, lo, hi in ((0, n, n + m), (1, n + m, n + 2 * m), (0, n + m, n + m + 1)):
        rows = n + m + (hi - lo == 1)
        out, lse = add(slot, lo, hi, rows)
        got = rows_of(slot, rows)
        at = torch.tensor([*range(n), *(range(n, n + m) if slot == 0 else ()), *range(lo, hi)][-rows:] if hi - lo == 1
                          else [*range(n), *range(lo, hi)], device=DEV)
        assert torch.equal(got[0], k[at]) and torch.equal(got[1], v[at])
        for h in range(hkv):
            g = slice(h * G, (h + 1) * G)
            near(out[:, g], lse[:, g], q[lo:hi, g], k[at, h], v[at, h], hi - lo, dtype)
    held = c.table[c.table >= 0]
    assert int(held.min()) >= first and int(over.item()) == 0
    idx = torch.tensor([[0, 5, 77]] * hkv, dtype=torch.int32, device=DEV)
    ck.compact_kv_paged(c, 0, list(range(hkv)), idx, 16, 9, over)
    at = [*range(16), *range(80, 96), *range(77 * 16, 78 * 16), *range(n + m + 1 - 9, n + m), n + m]
    got = rows_of(0, len(at))
    assert c.lens[0].tolist() == [len(at)] * hkv and torch.equal(got[0], k[at]) and torch.equal(got[1], v[at])
    ck.drop_paged(c, torch.tensor([10 ** 6] * 3, device=DEV))
    assert int(c.lens.sum()) == 0 and int(c.refs[first:].sum()) == 0 and bool((c.refs[:first] == 1).all())
    assert np.array_equal(c.free_bits.cpu().numpy().view(np.uint64), (free.reshape(-1, 64) << np.arange(64, dtype=np.uint64)).sum(axis=1, dtype=np.uint64))


def test_batches_of_more_than_4_gib():
    """16400 sequences of 32 new tokens: queries and results of 4.3 GB."""
    n, m, hkv, G = 16400, 32, 8, 4
    c = ck.paged_alloc(n * hkv, 32, n, hkv, 1, DEV, dtype=BF16)
    k, v = (randn((n * m, hkv, 128), i, BF16) for i in (1, 2))
    q = torch.empty((n * m, hkv * G, 128), dtype=BF16, device=DEV)
    for i in range(0, n * m, 1 << 16):
        q[i:i + (1 << 16)] = randn(q[i:i + (1 << 16)].shape, i + 3, BF16)
    assert q.numel() * 2 > 1 << 32
    plan = ck.paged_plan(c, range(n), [m] * n, [[m] * hkv] * n, hkv * G)
    ck.append_kv_paged(plan, c, k, v)
    out, lse = ck.attn_paged(plan, c, q)
    assert bool((c.lens == m).all()) and torch.equal(c.table.flatten().sort().values, torch.arange(n * hkv, device=DEV, dtype=torch.int32))
    for i in (0, 1, n // 2, n - 1):
        t = slice(i * m, (i + 1) * m)
        for h in (0, hkv - 1):
            g = slice(h * G, (h + 1) * G)
            near(out[t, g], lse[t, g], q[t, g], k[t, h], v[t, h], m, BF16)


def test_two_caches_on_two_streams_at_once():
    """Plans with workspaces of their own may run beside each other."""
    hkv, G, n = 4, 4, 3000

    def work(c, i):
        outs = []
        for new in ([n, 40], [1, 1], [300, 0], [1, 2]):
            bound = (c.lens[:2].cpu() + torch.tensor(new)[:, None]).tolist()
            plan = ck.paged_plan(c, [0, 1], new, bound, hkv * G)
            k, v = (randn((sum(new), hkv, 128), 10 * i + j, BF16) for j in (1, 2))
            ck.append_kv_paged(plan, c, k, v)
            outs.append(ck.attn_paged(plan, c, randn((sum(new), hkv * G, 128), 10 * i + 3, BF16)))
        return outs

    def alloc():
        return [ck.paged_alloc(600, 64, 2, hkv, 70, DEV, dtype=BF16) for _ in "ab"]
    want = [work(c, i) for i, c in enumerate(alloc())]
    caches, streams = alloc(), [torch.cuda.Stream() for _ in "ab"]
    torch.cuda.synchronize()
    plans, args = [], []
    for i, c in enumerate(caches):                     # everything that waits for the GPU comes before
        rows, p, a = np.zeros((2, hkv), np.int64), [], []
        for new in ([n, 40], [1, 1], [300, 0], [1, 2]):
            rows = rows + np.array(new)[:, None]
            p.append(ck.paged_plan(c, [0, 1], new, rows, hkv * G))
            a.append([randn((sum(new), hkv, 128), 10 * i + j, BF16) for j in (1, 2)] + [randn((sum(new), hkv * G, 128), 10 * i + 3, BF16)])
        plans.append(p)
        args.append(a)
    torch.cuda.synchronize()
    got = [[], []]
    for s in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                k, v, q = args[i][s]
                ck.append_kv_paged(plans[i][s], caches[i], k, v)
                got[i].append(ck.attn_paged(plans[i][s], caches[i], q))
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        for (o, z), (o2, z2) in zip(w, g):
            assert torch.equal(o, o2) and torch.equal(z, z2)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_batches_without_tokens(dtype):
    c = ck.paged_alloc(20, 16, 3, 2, 8, DEV, dtype=dtype)
    before = c.book.clone()
    plan = ck.paged_plan(c, [2, 0], [0, 0], [[0, 5], [9, 0]], 4)
    k = torch.zeros((0, 2, 128), dtype=dtype, device=DEV)
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.append_kv_paged(plan, c, k, k, over)
    out, lse = ck.attn_paged(plan, c, torch.zeros((0, 4, 128), dtype=dtype, device=DEV))
    torch.cuda.synchronize()
    assert out.shape == (0, 4, 128) and lse.shape == (0, 4) and torch.equal(c.book, before) and over.item() == 0


@pytest.mark.parametrize("dtype,b,cs", [(BF16, 512, 2), (BF16, 513, 2), (F32, 4097, 1), (BF16, 9001, 1)])
def test_compaction_of_long_lists(dtype, b, cs):
    """Lists around the border of the two ways to go over them, and of several turns of the
    longer one: unordered, with gaps, repeats, chunks without rows and a partial last one."""
    L, tail, page, hkv = 9100, 7, 64, 3
    c, s = cache_of(3 * R.pages_of(L, page) + 2 * 160, page, 2, hkv, 160, dtype)
    append(c, s, [1], [L], hkv, 5)
    r = np.random.RandomState(b)
    idx = r.randint(-2000, R.pages_of(L, cs) + 50, size=(2, b)).astype(np.int32)
    idx[0, 0], idx[1, -1] = R.pages_of(L - tail, cs) - 1, 1 << 30
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.compact_kv_paged(c, 1, [2, 0], torch.from_numpy(idx).to(DEV), cs, tail, over)
    assert not s.compact(1, [2, 0], idx.tolist(), cs, tail) and over.item() == 0
    s.same(c)
    ck.compact_kv_paged(c, 1, [0, 1], torch.zeros((2, 9000 + b), dtype=torch.int32, device=DEV), 2, tail, over)
    assert s.compact(1, [0, 1], np.zeros((2, 9000 + b), np.int32), 2, tail) and over.item() == 1   # more than max_pages
    s.same(c)

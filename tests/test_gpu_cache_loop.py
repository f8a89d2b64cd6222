"""The calls of the 8-bit and evicted caches together, as a serving loop uses them:
generation with appends, weights and evictions, captured into graphs, on another
stream, and on caches whose offsets pass 32 bits."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_30295_amd as ck
from test_gpu_cache import DT, D, DEV, Dense, Eight, accs, check_attention, dense, lens_of, same

pytestmark = pytest.mark.gpu


class Host:
    """One 8-bit view in 64 bits: rows in whole blocks (values) and the tail's rows."""

    def __init__(self, fmt, block):
        self.fmt, self.block = fmt, block
        self.coded, self.tail = [np.zeros((0, D)), np.zeros((0, D))], [np.zeros((0, D)), np.zeros((0, D))]

    def append(self, k, v):
        for i, x in enumerate((k, v)):
            self.tail[i] = np.concatenate([self.tail[i], x[None]])
            if len(self.tail[i]) == self.block:
                c, s = R.quantize(self.tail[i], self.fmt, self.block)
                self.coded[i] = np.concatenate([self.coded[i], R.values(c, s, self.fmt, self.block)])
                self.tail[i] = np.zeros((0, D))

    def rows(self):
        return [np.concatenate([c, t]) for c, t in zip(self.coded, self.tail)]

    def keep(self, rows):
        whole = rows[:len(rows) // self.block * self.block]
        self.coded = [c[whole] for c in self.coded]


@pytest.mark.parametrize("fmt,dtype,block", [("int8", "bf16", 32), ("e4m3", "f32", 64), ("e4m3", "bf16", 32)])
def test_generation_on_8_bit_caches_with_eviction(fmt, dtype, block):
    rng = np.random.default_rng(41)
    B, hkv, G, cap, steps, every = 2, 2, 4, 512, 150, 48
    start = [0, block - 1, 300, 257]
    q8 = ck.q8_alloc([cap] * 4, DEV, fmt=fmt, block=block, dtype=DT[dtype])
    src = Dense(rng, start, dtype)
    lens, capacity = lens_of(*start), lens_of(*[cap] * 4)
    ck.quantize_kv(src.table, lens, q8, max(start))
    acc = torch.zeros((4, cap), device=DEV)
    table = ck.acc_table([a.data_ptr() for a in acc], DEV)
    budget = torch.tensor([1, 2, 3, 128 // block], dtype=torch.int32, device=DEV)
    plan = ck.decode_plan([cap] * 4, hkv * G, hkv, DEV)
    host, want = [], [np.zeros(n) for n in start]
    for i, n in enumerate(start):
        host.append(Host(fmt, block))
        for k, v in zip(*[x[i][:n].double().cpu().numpy() for x in (src.k, src.v)]):
            host[i].append(k, v)
    for t in range(steps):
        k, v = (dense(rng, 4, dtype).view(B, hkv, D) for _ in "kv")
        q = dense(rng, B * hkv * G, dtype, 1.5).view(B, hkv * G, D).to(DEV)
        ck.append_kv_q8(q8, capacity, lens, k.to(DEV), v.to(DEV))
        before = acc.clone()
        out, lse = ck.decode_attn_q8(plan, q, q8, lens, acc=table)
        for i in range(4):
            host[i].append(k.view(4, D)[i].double().numpy(), v.view(4, D)[i].double().numpy())
        n = lens.tolist()
        assert n == [len(h.rows()[0]) for h in host], t
        if t % 7 == 0 or t == steps - 1:
            check_attention(q, lambda i: host[i].rows(), n, hkv, out, lse, list(acc), list(before), 1.0)
        if t % every == every - 1:
            was = acc.cpu().numpy()
            ck.evict_kv_q8(q8, lens, table, budget, cs=block, recent=20, max_rows=cap)
            for i in range(4):
                rows = R.evict(was[i, :n[i]], int(budget[i]), block, 20)
                host[i].keep(rows)
                assert int(lens[i]) == len(rows), (t, i)
                assert np.array_equal(acc[i, :len(rows)].cpu().numpy(), was[i][rows])
                assert not acc[i, len(rows):].any()
    assert max(lens.tolist()) < 300        # every view was evicted


def test_generation_on_bf16_caches_with_eviction():
    rng = np.random.default_rng(42)
    B, hkv, G, cap, cs = 1, 2, 2, 400, 4
    start = [200, 390]
    kv = [torch.zeros((2, cap, D), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    for x in kv:
        x[:] = dense(rng, 2 * cap, "bf16").view(2, cap, D).to(DEV)
    table = ck.kv_table([(kv[0][i].data_ptr(), kv[1][i].data_ptr()) for i in range(2)], DEV)
    rows = [[x[i, :start[i]].double().cpu().numpy() for x in kv] for i in range(2)]
    lens, capacity, acc = lens_of(*start), lens_of(cap, cap), torch.zeros((2, cap), device=DEV)
    accp, budget = ck.acc_table([a.data_ptr() for a in acc], DEV), torch.tensor([30, 60], dtype=torch.int32, device=DEV)
    plan = ck.decode_plan([cap, cap], hkv * G, hkv, DEV)
    for t in range(60):
        k, v = (dense(rng, 2, "bf16").view(B, hkv, D) for _ in "kv")
        ck.append_kv(table, capacity, lens, k.to(DEV), v.to(DEV))
        for i in range(2):
            if len(rows[i][0]) < cap:
                rows[i] = [np.concatenate([r, x[0, i:i + 1].double().numpy()]) for r, x in zip(rows[i], (k, v))]
        q, before = dense(rng, hkv * G, "bf16").view(B, hkv * G, D).to(DEV), acc.clone()
        out, lse = ck.decode_attn_weights(plan, q, table, lens, accp, decay=0.9)
        check_attention(q, lambda i: rows[i], lens.tolist(), hkv, out, lse, list(acc), list(before), 0.9)
        if t % 9 == 8:
            was = acc.cpu().numpy()
            ck.evict_kv(table, lens, accp, budget, cs=cs, recent=31, max_rows=cap, dtype=torch.bfloat16)
            for i in range(2):
                at = R.evict(was[i, :len(rows[i][0])], int(budget[i]), cs, 31)
                rows[i] = [r[at] for r in rows[i]]
                assert int(lens[i]) == len(at)


def state_of(q8, acc, lens):
    return [t.clone() for t in q8.hold] + [acc.clone(), lens.clone()]


def test_a_captured_step_replays_as_eager_steps_do():
    # append, attention with weights and eviction in one graph, replayed between the
    # program's own eager work, against the same steps eagerly: the same bits
    rng = np.random.default_rng(43)
    n, B, hkv, G, cap = 4, 2, 2, 4, 256

    def cache():
        g = np.random.default_rng(44)
        q8 = ck.q8_alloc([cap] * n, DEV, fmt="e4m3", block=32, dtype=torch.bfloat16)
        src = Dense(g, [120, 31, 0, 200], "bf16")
        lens = src.lens.clone()
        ck.quantize_kv(src.table, lens, q8, 200)
        return q8, lens, torch.zeros((n, cap), device=DEV)

    capacity, budget = lens_of(*[cap] * n), torch.full((n,), 3, dtype=torch.int32, device=DEV)
    plan = ck.decode_plan([cap] * n, hkv * G, hkv, DEV)
    ws, ews = ck.workspace(ck.weights_workspace(plan), DEV), ck.workspace(ck.evict_workspace(n, cap, 32), DEV)
    k, v = (torch.zeros((B, hkv, D), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    q = torch.zeros((B, hkv * G, D), dtype=torch.bfloat16, device=DEV)
    out, lse = torch.zeros((B, hkv * G, D), device=DEV), torch.zeros((B, hkv * G), device=DEV)

    def step(q8, lens, accp):
        ck.append_kv_q8(q8, capacity, lens, k, v)
        ck.decode_attn_q8(plan, q, q8, lens, out=out, lse=lse, acc=accp, ws=ws)
        ck.evict_kv_q8(q8, lens, accp, budget, cs=32, recent=8, max_rows=cap, ws=ews)

    (ga, la, aa), (ge, le, ae) = cache(), cache()
    pa, pe = (ck.acc_table([x.data_ptr() for x in a], DEV) for a in (aa, ae))
    warm = cache()
    step(warm[0], warm[1], ck.acc_table([x.data_ptr() for x in warm[2]], DEV))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(ga, la, pa)
    for t in range(70):
        for x in (k, v, q):
            x.copy_(dense(rng, x.numel() // D, "bf16").view(x.shape))
        graph.replay()
        got = out.clone(), lse.clone()
        if t % 3 == 0:
            torch.cuda.synchronize()
        step(ge, le, pe)
        assert same(got[0], out) and same(got[1], lse), t
        assert all(same(x, y) for x, y in zip(state_of(ga, aa, la), state_of(ge, ae, le))), t
    assert max(la.tolist()) < 200


def test_calls_run_on_the_current_stream():
    rng = np.random.default_rng(45)
    lens = [3000, 500, 64, 1]
    d = Dense(rng, lens, "bf16")
    q = dense(rng, 16, "bf16").view(2, 8, D).to(DEV)
    plan = ck.decode_plan(lens, 8, 2, DEV)

    def steps(late):
        q8 = ck.q8_alloc([3072] * 4, DEV, fmt="int8", block=64, dtype=torch.bfloat16)
        back = [torch.zeros((4, 3072, D), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
        acc = torch.zeros((4, 3072), device=DEV)
        n, cap = lens_of(*lens), lens_of(*[3072] * 4)
        table = ck.acc_table([a.data_ptr() for a in acc], DEV)
        out_t = ck.kv_table([(back[0][i].data_ptr(), back[1][i].data_ptr()) for i in range(4)], DEV)
        budget = torch.full((4,), 10, dtype=torch.int32, device=DEV)
        src = ck.kv_table([(0, 0)] * 4, DEV)
        torch.cuda.synchronize()
        if late:        # what the calls depend on arrives on their stream behind slow work
            x = torch.ones((4096, 4096), device=DEV)
            for _ in range(20):
                x = x @ x * 1e-4
        src.copy_(d.table)
        ck.quantize_kv(src, n, q8, 3000)
        ck.append_kv_q8(q8, cap, n, q[:, :2].contiguous(), q[:, 2:4].contiguous())
        out, lse = ck.decode_attn_q8(plan, q, q8, n, acc=table)
        ck.evict_kv_q8(q8, n, table, budget, cs=64, recent=0, max_rows=3072)
        ck.dequantize_kv(q8, n, out_t, 3072)
        return [out, lse, acc, n, *back]

    want = steps(False)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        got = steps(True)
    s.synchronize()
    assert all(same(a, b) for a, b in zip(got, want))


def test_the_same_call_gives_the_same_bits():
    rng = np.random.default_rng(46)
    lens = [9000, 9000, 290, 290, 31, 4100, 1, 0]
    q8 = Eight([n + 64 for n in lens], "int8", 64, "bf16")
    for i, n in enumerate(lens):
        q8.fill(i, dense(rng, n, "bf16").double().numpy(), dense(rng, n, "bf16").double().numpy())
    q = dense(rng, 32, "bf16").view(2, 16, D).to(DEV)
    plan = ck.decode_plan(lens, 16, 4, DEV)
    runs = []
    for _ in range(6):
        acc = torch.zeros((8, 9100), device=DEV)
        runs.append((*ck.decode_attn_q8(plan, q, q8.views, lens_of(*lens),
                                        acc=ck.acc_table([a.data_ptr() for a in acc], DEV)), acc))
    assert all(same(a, b) for r in runs[1:] for a, b in zip(runs[0], r))


def test_offsets_beyond_32_bits():
    # one view of 34 million rows: 4.35 GB of K codes, 8.7 GB of bf16 K
    n, block, cs = 34_000_123, 64, 64
    g = torch.Generator(device=DEV).manual_seed(5)
    k, v = (torch.empty((n, D), dtype=torch.bfloat16, device=DEV) for _ in "kv")
    for x in (k, v):
        for a in range(0, n, 1 << 22):
            x[a:a + (1 << 22)] = torch.randn((min(1 << 22, n - a), D), generator=g, device=DEV).bfloat16()
    q8 = ck.q8_alloc([n], DEV, fmt="int8", block=block, dtype=torch.bfloat16)
    lens = lens_of(n)
    ck.quantize_kv(ck.kv_table([(k.data_ptr(), v.data_ptr())], DEV), lens, q8, n)
    whole = n // block * block
    for b in (0, 16_777_216 // block, 33_554_432 // block + 3, whole // block - 1):
        for x, codes, scale in ((k, q8.hold[0], q8.hold[2]), (v, q8.hold[1], q8.hold[3])):
            c, s = R.quantize(x[b * block:(b + 1) * block].double().cpu().numpy(), "int8", block)
            assert np.array_equal(codes[b * block:(b + 1) * block].cpu().numpy().view(np.uint8), c), b
            assert float(scale[b]) == s[0]
    assert same(q8.hold[4][:n - whole], k[whole:]) and same(q8.hold[5][:n - whole], v[whole:])
    back = [torch.zeros_like(k), torch.zeros_like(v)]
    ck.dequantize_kv(q8, lens, ck.kv_table([(back[0].data_ptr(), back[1].data_ptr())], DEV), n)
    for b in (1, 33_554_432 // block + 3, whole // block - 1):
        at = slice(b * block, (b + 1) * block)
        for x, codes, scale in ((back[0], q8.hold[0], q8.hold[2]), (back[1], q8.hold[1], q8.hold[3])):
            assert torch.equal(x[at], (codes[at].float() * scale[b]).bfloat16()), b
    assert same(back[0][whole:], k[whole:])
    del k, v, back
    q = torch.randn((1, 2, D), generator=g, device=DEV).bfloat16()
    acc = torch.zeros(n, device=DEV)
    table = ck.acc_table([acc.data_ptr()], DEV)
    out, lse = ck.decode_attn_q8(ck.decode_plan([n], 2, 1, DEV), q, q8, lens, acc=table)
    # the same in 64 bits, a million rows at a time
    kc, vc, ks, vs, kt, vt = q8.hold
    qd = q[0].double() / math.sqrt(D)

    scores = []
    for a in range(0, whole, 1 << 20):
        e = min(whole, a + (1 << 20))
        kk = kc[a:e].double() * ks[a // block:e // block].double().repeat_interleave(block)[:, None]
        scores.append(qd @ kk.t())
    scores.append(qd @ kt[:n - whole].double().t())
    s = torch.cat(scores, dim=1)
    want_lse = torch.logsumexp(s, dim=1)
    p = torch.exp(s - want_lse[:, None])
    want, size = torch.zeros((2, D), dtype=torch.float64, device=DEV), torch.zeros((2, D), dtype=torch.float64, device=DEV)
    for a in range(0, n, 1 << 20):
        e = min(n, a + (1 << 20))
        vv = vc[a:min(e, whole)].double() * vs[a // block:min(e, whole) // block].double().repeat_interleave(block)[:, None]
        if e > whole:
            vv = torch.cat([vv, vt[:n - whole].double()])
        want += p[:, a:e] @ vv
        size += p[:, a:e] @ vv.abs()
    # sum |q||k| is at most the product of the norms, which 128 normal values keep below 16
    # each; a workgroup sums a 256th of the rows, then the partials are joined
    sa = 16.0 * 16.0 / math.sqrt(D)
    tol = R.output_error(sa, n / 256) * size
    assert (((out[0].double() - want).abs() <= tol).all()) and ((lse[0].double() - want_lse).abs() < 1e-4).all()
    w = p.mean(dim=0)
    assert ((acc.double() - w).abs() <= R.weight_error(sa, n / 256) * w).all()
    # eviction: 200 blocks stay
    was, old = acc.clone(), [kc.clone(), ks.clone()]
    budget = torch.tensor([200], dtype=torch.int32, device=DEV)
    ck.evict_kv_q8(q8, lens, table, budget, cs=cs, recent=100, max_rows=n)
    nc = (n - 100) // cs
    best = was[:nc * cs].view(nc, cs).amax(dim=1)
    stay = torch.sort(torch.sort(best, descending=True, stable=True).indices[:200]).values.cpu().numpy()
    place = np.arange(200)
    place[np.setdiff1d(np.arange(200), stay)] = stay[stay >= 200]
    rows = np.concatenate([(place[:, None] * cs + np.arange(cs)).reshape(-1), np.arange(nc * cs, n)])
    assert int(lens[0]) == len(rows) and place.max() * cs * D > 2 ** 32
    at = torch.from_numpy(rows).to(DEV)
    assert same(acc[:len(rows)], was[at]) and not acc[len(rows):].any()
    nb = len(rows) // block
    assert same(kc[:nb * block], old[0][at[:nb * block]]) and same(ks[:nb], old[1][at[:nb * block:block] // block])

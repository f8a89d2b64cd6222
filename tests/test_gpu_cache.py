"""8-bit caches, attention that adds its weights up, and eviction on the GPU,
against plain 64-bit forms (cache_ref.py)."""
import math

import numpy as np
import pytest
import torch

import cache_ref as R
import paper_2608_30295_amd as ck

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
D = 128
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
BAD = 1e30       # what lies behind the rows a call may read


def dense(rng, n, dtype, scale=1.0):
    x = torch.from_numpy(rng.standard_normal((n, D)).astype(np.float32) * scale)
    if n:
        x[rng.random(n) < 0.02] *= 3
    return x.to(DT[dtype])


class Dense:
    """Views of the given lengths with `room` rows behind each."""

    def __init__(self, rng, lens, dtype, room=3):
        self.k = [torch.cat([dense(rng, n, dtype), torch.full((room, D), BAD).to(DT[dtype])]).to(DEV) for n in lens]
        self.v = [torch.cat([dense(rng, n, dtype), torch.full((room, D), math.nan).to(DT[dtype])]).to(DEV) for n in lens]
        self.table = ck.kv_table([(a.data_ptr(), b.data_ptr()) for a, b in zip(self.k, self.v)], DEV)
        self.lens = torch.tensor(lens, dtype=torch.int64, device=DEV)

    def host(self, i):
        n = int(self.lens[i])
        return self.k[i][:n].double().cpu().numpy(), self.v[i][:n].double().cpu().numpy()


class Eight:
    """8-bit views of the given capacities with bytes behind every part that no call may change."""
    PARTS = ("k", "v", "ks", "vs", "kt", "vt")

    def __init__(self, capacity, fmt, block, dtype):
        self.fmt, self.block, self.dtype = fmt, block, dtype
        self.p = []
        for c in capacity:
            n = c // block
            self.p.append({"k": torch.full((n * block + 1, D), 77, dtype=torch.uint8, device=DEV),
                           "v": torch.full((n * block + 1, D), 78, dtype=torch.uint8, device=DEV),
                           "ks": torch.full((n + 1,), 79.0, device=DEV), "vs": torch.full((n + 1,), 80.0, device=DEV),
                           "kt": torch.full((block + 1, D), math.nan, device=DEV).to(DT[dtype]),
                           "vt": torch.full((block + 1, D), math.nan, device=DEV).to(DT[dtype])})
        self.views = ck.q8_views([[p[n].data_ptr() for n in self.PARTS] for p in self.p], DEV, fmt=fmt, block=block,
                                 dtype=DT[dtype])

    def fill(self, i, k, v):
        """Rows (fp64 of stored values) into view i, by the plain form."""
        nb = len(k) // self.block
        for name, x in (("k", k), ("v", v)):
            codes, scales = R.quantize(x, self.fmt, self.block)
            self.p[i][name][:len(codes)] = torch.from_numpy(codes).to(DEV)
            self.p[i][name + "s"][:nb] = torch.from_numpy(scales).to(DEV)
            rest = torch.from_numpy(x[nb * self.block:]).to(DT[self.dtype])
            self.p[i][name + "t"][:len(rest)] = rest.to(DEV)

    def host(self, i, n):
        """fp64 rows that view i of n rows stands for."""
        nb, p = n // self.block, self.p[i]
        got = []
        for name in "kv":
            c = p[name][:nb * self.block].cpu().numpy()
            got.append(np.concatenate([R.values(c, p[name + "s"][:nb].cpu().numpy(), self.fmt, self.block),
                                       p[name + "t"][:n - nb * self.block].double().cpu().numpy()]))
        return got

    def state(self, i):
        return [self.p[i][n].clone() for n in self.PARTS]


def same(a, b):
    """Bitwise equality of tensors."""
    u = {1: torch.uint8, 2: torch.int16, 4: torch.int32, 8: torch.int64}[a.element_size()]
    return a.shape == b.shape and torch.equal(a.contiguous().view(u), b.contiguous().view(u))


def lens_of(*n):
    return torch.tensor(n, dtype=torch.int64, device=DEV)


# ------------------------------------------------------------------- into 8 bits and back

def edge_rows(rng, block, dtype):
    """Blocks where rounding and scales can go wrong, as fp32 rows."""
    one = np.ones((block, D))
    rows = [np.zeros((block, D)), one * 1e-31, one * 2.0 ** -100, -one * 3e38]
    # quotients at and next to half steps: x = (i + 1/2) step with the maximum 127 step (int8), or
    # halves of e4m3 steps below 448
    half = (rng.integers(-127, 127, (block, D)) + 0.5)
    half[0, 0] = 127
    rows.append(half * 2.0 ** -4)
    rows.append(half * 0.3)
    grid = (R.E4M3[:-1] + R.E4M3[1:]) / 2
    mid = grid[rng.integers(0, len(grid), (block, D))] * rng.choice([-1.0, 1.0], (block, D))
    mid[0, 0] = 448
    rows.append(mid)
    mid2 = mid * 2.0 ** -20
    mid2[0, 0] = 449 * 2.0 ** -20
    rows.append(mid2)
    rows.append(rng.standard_normal((block, D)) * np.exp(rng.uniform(-30, 5, (block, D))))
    x = np.concatenate(rows).astype(np.float32)
    return torch.from_numpy(x).to(DT[dtype])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [32, 64])
def test_quantize_codes_scales_tails(fmt, dtype, block):
    rng = np.random.default_rng(11)
    lens = [0, 1, block - 1, block, block + 1, 5 * block, 9 * block + 17, 1000]
    d = Dense(rng, lens, dtype)
    e = edge_rows(rng, block, dtype).to(DEV)
    d.k[6][:9 * block] = e
    d.v[6][:9 * block] = e.flip(0)
    d.v[5][block + 3, 7] = math.inf
    d.v[5][3 * block, 0] = math.nan
    q = Eight([n + 2 * block for n in lens], fmt, block, dtype)
    before = [q.state(i) for i in range(len(lens))]
    ck.quantize_kv(d.table, d.lens, q.views, max(lens))
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        nb = n // block
        for name, x in zip("kv", d.host(i)):
            codes, scales = R.quantize(x, fmt, block)
            old = before[i][Eight.PARTS.index(name)], before[i][Eight.PARTS.index(name + "s")], \
                before[i][Eight.PARTS.index(name + "t")]
            got_c, got_s, got_t = q.p[i][name].cpu().numpy(), q.p[i][name + "s"], q.p[i][name + "t"]
            assert np.array_equal(got_s[:nb].cpu().numpy(), scales, equal_nan=True), (i, name)
            assert np.array_equal(got_c[:nb * block], codes), (i, name)
            raw = (d.k if name == "k" else d.v)[i]
            assert same(got_t[:n - nb * block], raw[nb * block:n]), (i, name)
            # nothing behind the rows was written
            assert np.array_equal(got_c[nb * block:], old[0].cpu().numpy()[nb * block:])
            assert same(got_s[nb:], old[1][nb:]) and same(got_t[n - nb * block:], old[2][n - nb * block:])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [32, 64])
def test_dequantize_is_code_times_scale(fmt, dtype, block):
    rng = np.random.default_rng(12)
    lens = [0, 1, block, 3 * block + 5, 700]
    q = Eight([n + block for n in lens], fmt, block, dtype)
    for i, n in enumerate(lens):
        q.fill(i, dense(rng, n, dtype).double().numpy(), dense(rng, n, dtype, 0.01).double().numpy())
    out = Dense(rng, [n + 2 for n in lens], dtype)
    before = [(a.clone(), b.clone()) for a, b in zip(out.k, out.v)]
    ck.dequantize_kv(q.views, lens_of(*lens), out.table, max(lens))
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        for got, want, old in zip((out.k[i], out.v[i]), q.host(i, n), before[i]):
            want = torch.from_numpy(want.astype(np.float32)).to(DT[dtype])   # the fp32 product, rounded once more
            assert torch.equal(got[:n].cpu(), want), i
            assert same(got[n:], old[n:])


def test_views_longer_than_max_rows_are_left_alone():
    rng = np.random.default_rng(13)
    d = Dense(rng, [40, 200, 64], "bf16")
    q = Eight([256] * 3, "int8", 32, "bf16")
    before = q.state(1), q.state(2)
    d.lens[2] = -5
    ck.quantize_kv(d.table, d.lens, q.views, 100)
    ck.dequantize_kv(q.views, d.lens, d.table, 100)
    assert all(same(a, b) for a, b in zip(before[0], q.state(1)))
    assert all(same(a, b) for a, b in zip(before[1], q.state(2)))
    assert q.p[0]["ks"][0] != 79.0


# ------------------------------------------------------------------------------ append

@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [32, 64])
def test_append_is_quantize_of_the_longer_rows(fmt, dtype, block):
    rng = np.random.default_rng(14)
    start, steps = [0, 1, block - 2, block - 1, 2 * block - 3, 5 * block + 9], block + 3
    B, hkv = 3, 2
    whole = Dense(rng, [n + steps for n in start], dtype)
    first, last = Eight([n + steps for n in start], fmt, block, dtype), Eight([n + steps for n in start], fmt, block, dtype)
    lens = lens_of(*start)
    ck.quantize_kv(whole.table, lens, first.views, max(start))
    cap = lens_of(*[n + steps for n in start])
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    for s in range(steps):
        new = [torch.stack([x[n + s] for x, n in zip(xs, start)]).view(B, hkv, D).contiguous() for xs in (whole.k, whole.v)]
        ck.append_kv_q8(first.views, cap, lens, new[0], new[1], over)
    ck.quantize_kv(whole.table, whole.lens, last.views, int(whole.lens.max()))
    assert torch.equal(lens, whole.lens) and int(over) == 0
    for i, n in enumerate(start):
        tail = (n + steps) % block
        for name in Eight.PARTS:
            a, b = first.p[i][name], last.p[i][name]
            if name in ("kt", "vt"):
                a, b = a[:tail], b[:tail]
            assert same(a, b), (i, name)
    # full views and bad lengths are refused on the device
    before = [first.state(i) for i in range(6)]
    lens[1] = -1
    was = lens.clone()
    ck.append_kv_q8(first.views, cap, lens, new[0], new[1], over)
    assert int(over) == 1 and torch.equal(lens, was)
    assert all(same(a, b) for i in range(6) for a, b in zip(before[i], first.state(i)))


# ---------------------------------------------------------------------------- attention

def check_attention(q, views, lens, hkv, out, lse, acc, acc0, decay, scale=1 / math.sqrt(D)):
    """Against the 64-bit form; acc, acc0: the views' weights after and before, or None.

    Over 8-bit views P enters the product as two fp16 numbers of 2^11 P, whose
    smaller one is a multiple of 2^-24: each P is off by up to 2^-25 / 2^11 = 2^-36
    however small it is, P / l too (l is at least the largest P, at least 1), and an
    output by 2^-36 sum |v|.  That shows where rows of almost all weight have V = 0."""
    B, hq, _ = q.shape
    G = hq // hkv
    q = q.double().cpu().numpy()
    for b in range(B):
        for h in range(hkv):
            i = b * hkv + h
            k, v = views(i)
            g = slice(h * G, (h + 1) * G)
            want, wl, w, sa, pv = R.attend(q[b, g], k, v, scale)
            n = len(k)
            got, gl = out[b, g].double().cpu().numpy(), lse[b, g].double().cpu().numpy()
            if n == 0:
                assert not got.any() and np.isneginf(gl).all(), i
            else:
                tol = R.output_error(sa, n) * pv + 2.0 ** -24 * np.abs(want) + 2.0 ** -36 * np.abs(v).sum(axis=0)
                assert (np.abs(got - want) <= tol).all(), (i, n, float((np.abs(got - want) / tol).max()))
                assert (np.abs(gl - wl) <= R.score_error(sa) + 2.0 ** -22 * (1 + np.abs(wl)) +
                        R.weight_error(sa, n)).all(), (i, n)
            if acc is not None:
                new, old = acc[i].double().cpu().numpy(), acc0[i].double().cpu().numpy()
                ref = decay * old[:n] + w
                assert (np.abs(new[:n] - ref) <= R.weight_error(sa, n) * w + 2.0 ** -23 * np.abs(ref) + 1e-37).all(), i
                assert np.array_equal(new[n:], old[n:]), i


def accs(rng, lens, room=5):
    a = [torch.from_numpy(rng.random(n + room).astype(np.float32)).to(DEV) for n in lens]
    return a, [x.clone() for x in a], ck.acc_table([x.data_ptr() for x in a], DEV)


LENS = {
    "short": [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65],
    "ragged": [1000, 7, 4099, 0, 2112, 333, 5000, 64, 96, 1, 127, 2048],
    "hybrid": [20011, 20011, 290, 290, 9000, 9000, 290, 290, 31, 31, 31, 31],
}


@pytest.mark.parametrize("which", list(LENS))
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("fmt,dtype,block", [("int8", "bf16", 32), ("int8", "bf16", 64), ("e4m3", "bf16", 64),
                                             ("int8", "f32", 64), ("e4m3", "f32", 32)])
@pytest.mark.parametrize("weights", [False, True])
def test_attention_over_8_bit_views(which, group, fmt, dtype, block, weights):
    rng = np.random.default_rng(21)
    lens, hkv = LENS[which], 4
    B = len(lens) // hkv
    q8 = Eight([n + 70 for n in lens], fmt, block, dtype)
    for i, n in enumerate(lens):
        q8.fill(i, dense(rng, n, dtype).double().numpy(), dense(rng, n, dtype).double().numpy())
    q = torch.from_numpy(rng.standard_normal((B, hkv * group, D)).astype(np.float32) * 2).to(DT[dtype]).to(DEV)
    plan = ck.decode_plan(np.array(lens) + rng.integers(0, 70, len(lens)), hkv * group, hkv, DEV)
    a, a0, table = accs(rng, lens)
    out, lse = ck.decode_attn_q8(plan, q, q8.views, lens_of(*lens).view(B, hkv), acc=table if weights else None,
                                 decay=0.75)
    check_attention(q, lambda i: q8.host(i, lens[i]), lens, hkv, out, lse, a if weights else None, a0, 0.75)


@pytest.mark.parametrize("which", list(LENS))
@pytest.mark.parametrize("group", [1, 2, 4, 8])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_with_weights(which, group, dtype):
    rng = np.random.default_rng(22)
    lens, hkv = LENS[which], 2
    B = len(lens) // hkv
    d = Dense(rng, lens, dtype)
    q = torch.from_numpy(rng.standard_normal((B, hkv * group, D)).astype(np.float32) * 2).to(DT[dtype]).to(DEV)
    plan = ck.decode_plan(np.array(lens) + rng.integers(0, 70, len(lens)), hkv * group, hkv, DEV)
    a, a0, table = accs(rng, lens)
    out, lse = ck.decode_attn_weights(plan, q, d.table, d.lens.view(B, hkv), table, decay=0.5)
    check_attention(q, d.host, lens, hkv, out, lse, a, a0, 0.5)
    # the same attention as without weights (its P has 16 bits and more)
    ref, ref_lse = ck.decode_attn(plan, q, d.table, d.lens.view(B, hkv))
    assert (out - ref).abs().max() <= 2e-3 and torch.equal(torch.isinf(lse), torch.isinf(ref_lse))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_lengths_beyond_the_plan_are_cut(fmt):
    # planned for fewer rows than there are: the rows behind are not attended to, the tail
    # starts where the lengths say
    rng = np.random.default_rng(23)
    lens, planned = [200, 200, 200, 200, 96, 130], [50, 192, 197, 64, 95, 129]
    q8 = Eight([256] * 6, fmt, 64, "bf16")
    for i, n in enumerate(lens):
        q8.fill(i, dense(rng, n, "bf16").double().numpy(), dense(rng, n, "bf16").double().numpy())
    q = torch.randn((3, 8, D), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    plan = ck.decode_plan(planned, 8, 2, DEV)
    a, a0, table = accs(rng, lens)
    out, lse = ck.decode_attn_q8(plan, q, q8.views, lens_of(*lens), acc=table)

    def cut(i):
        k, v = q8.host(i, lens[i])
        return k[:planned[i]], v[:planned[i]]
    check_attention(q, cut, planned, 2, out, lse, a, a0, 1.0)


@pytest.mark.parametrize("kind,group", [("int8", 4), ("e4m3", 8), ("bf16", 1), ("bf16", 4), ("bf16", 8), ("f32", 2),
                                        ("f32", 8)])
@pytest.mark.parametrize("split", [0, 640])
def test_long_shares_with_weights(kind, group, split):
    # shares of more than 1200 rows, whose scores are kept until the share's end where
    # they fit, and shares of a given length
    rng = np.random.default_rng(27)
    dtype = kind if kind in DT else "bf16"
    lens = [330_001, 70]
    q = torch.randn((1, 2 * group, D), generator=torch.Generator().manual_seed(4)).to(DT[dtype]).to(DEV)
    plan = ck.decode_plan(lens, 2 * group, 2, DEV, split_tokens=split)
    a, a0, table = accs(rng, lens)
    d = Dense(rng, lens, dtype)
    if kind in DT:
        out, lse = ck.decode_attn_weights(plan, q, d.table, d.lens, table)
        host = d.host
    else:
        q8 = Eight([n + 64 for n in lens], kind, 64, dtype)
        ck.quantize_kv(d.table, d.lens, q8.views, max(lens))
        out, lse = ck.decode_attn_q8(plan, q, q8.views, d.lens, acc=table)
        host = lambda i: q8.host(i, lens[i])
    check_attention(q, host, lens, 2, out, lse, a, a0, 1.0)


@pytest.mark.parametrize("kind", ["int8", "bf16"])
def test_decay_zero_leaves_this_step_s_weights(kind):
    rng = np.random.default_rng(28)
    lens = [300, 3000, 0, 17]
    d = Dense(rng, lens, "bf16")
    q = torch.randn((2, 8, D), generator=torch.Generator().manual_seed(6)).bfloat16().to(DEV)
    plan = ck.decode_plan(lens, 8, 2, DEV)
    a = [torch.full((n + 3,), math.nan, device=DEV) for n in lens]
    table = ck.acc_table([x.data_ptr() for x in a], DEV)
    if kind == "bf16":
        ck.decode_attn_weights(plan, q, d.table, d.lens, table, decay=0.0)
    else:
        q8 = Eight([n + 64 for n in lens], kind, 64, "bf16")
        ck.quantize_kv(d.table, d.lens, q8.views, max(lens))
        ck.decode_attn_q8(plan, q, q8.views, d.lens, acc=table, decay=0.0)
    for x, n in zip(a, lens):
        assert torch.isnan(x[n:]).all() and (n == 0 or abs(float(x[:n].double().sum()) - 1) < 1e-5)


@pytest.mark.parametrize("kind", ["int8", "e4m3", "bf16", "f32"])
def test_many_tiny_views(kind):
    # more segments per workgroup than its table holds at a time
    rng = np.random.default_rng(24)
    B, hkv, G = 700, 8, 1
    base = [int(x) for x in rng.integers(0, 40, 50)]
    lens = [base[i % 50] for i in range(B * hkv)]
    dtype = kind if kind in DT else "bf16"
    few = Dense(rng, base, dtype)
    q = torch.randn((B, hkv * G, D), generator=torch.Generator().manual_seed(2)).to(DT[dtype]).to(DEV)
    plan = ck.decode_plan(lens, hkv * G, hkv, DEV)
    assert plan.plan.variant == 1                 # not the one-workgroup-per-CU plan
    a, a0, table = accs(rng, lens, 2)
    if kind in DT:
        kv = few.table[torch.arange(B * hkv, device=DEV) % 50].contiguous()
        out, lse = ck.decode_attn_weights(plan, q, kv, lens_of(*lens), table)
        host = lambda i: few.host(i % 50)
    else:
        q8 = Eight([64] * 50, kind, 32, dtype)
        for i, n in enumerate(base):
            q8.fill(i, *few.host(i))
        views = ck.Q8Views(q8.views.table[torch.arange(B * hkv, device=DEV) % 50].contiguous(), kind, 32, DT[dtype])
        out, lse = ck.decode_attn_q8(plan, q, views, lens_of(*lens), acc=table)
        host = lambda i: q8.host(i % 50, base[i % 50])
    for b in (0, 1, 350, 699):
        sub = slice(b * hkv, (b + 1) * hkv)
        check_attention(q[b:b + 1], lambda i: host(b * hkv + i), lens[sub], hkv, out[b:b + 1], lse[b:b + 1], a[sub],
                        a0[sub], 1.0)
    # every view's weights sum to 1 (0 without rows)
    got = np.array([float((x - y).double().sum()) for x, y in zip(a, a0)])
    assert np.abs(got - (np.array(lens) > 0)).max() < 1e-4


@pytest.mark.parametrize("kind", ["int8", "e4m3", "bf16", "f32"])
def test_large_and_tiny_magnitudes(kind):
    # peaked softmax, magnitudes far from 1 and rows of zeros
    rng = np.random.default_rng(25)
    dtype = kind if kind in DT else "bf16"
    lens = [300, 300, 300, 300]
    for qs, ks, vs in ((30.0, 3.0, 1e-20), (1e-18, 1e18, 1e20), (1e10, 1e-10, 1.0)):
        rows = [(dense(rng, n, dtype, ks).double().numpy(), dense(rng, n, dtype, vs).double().numpy()) for n in lens]
        for k, v in rows:
            k[64:96] = 0
            v[96:128] = 0
        q = (torch.from_numpy(rng.standard_normal((2, 8, D)).astype(np.float32)) * qs).to(DT[dtype])
        q[0, 3] = 0
        q = q.to(DEV)
        plan = ck.decode_plan(lens, 8, 2, DEV)
        a, a0, table = accs(rng, lens)
        if kind in DT:
            d = Dense(rng, lens, dtype)
            for i, (k, v) in enumerate(rows):
                d.k[i][:300], d.v[i][:300] = torch.from_numpy(k).to(DT[dtype]), torch.from_numpy(v).to(DT[dtype])
            out, lse = ck.decode_attn_weights(plan, q, d.table, d.lens, table)
            host = d.host
        else:
            q8 = Eight([320] * 4, kind, 32, dtype)
            for i, (k, v) in enumerate(rows):
                q8.fill(i, k, v)
            out, lse = ck.decode_attn_q8(plan, q, q8.views, lens_of(*lens), acc=table)
            host = lambda i: q8.host(i, 300)
        check_attention(q, host, lens, 2, out, lse, a, a0, 1.0)


def test_values_that_are_not_finite_reach_their_own_heads_only():
    rng = np.random.default_rng(26)
    d = Dense(rng, [130, 130], "bf16")
    d.v[1][5, 3] = math.inf
    q8 = Eight([192, 192], "int8", 64, "bf16")
    ck.quantize_kv(d.table, d.lens, q8.views, 130)
    q = torch.randn((1, 8, D), generator=torch.Generator().manual_seed(3)).bfloat16().to(DEV)
    out, lse = ck.decode_attn_q8(ck.decode_plan([130, 130], 8, 2, DEV), q, q8.views, d.lens)
    assert torch.isfinite(out[0, :4]).all() and torch.isfinite(lse).all()
    assert torch.isnan(out[0, 4:]).all()          # V of its first block reads as NaN


# ------------------------------------------------------------------------------ eviction

def acc_rows(rng, n, kind):
    a = np.exp(2 * rng.standard_normal(n)).astype(np.float32)
    if kind == "ties":
        a = rng.integers(0, 3, n).astype(np.float32)
    elif kind == "equal":
        a[:] = 0.25
    elif kind == "special" and n > 8:
        a[rng.integers(0, n, 3)] = math.inf
        a[rng.integers(0, n, 2)] = math.nan
        a[rng.integers(0, n, n // 4)] = -0.0
        a[rng.integers(0, n, n // 4)] = 0.0
        a[rng.integers(0, n, 2)] = -math.inf
        a[rng.integers(0, n, 3)] = 1e-42
        a[rng.integers(0, n, 3)] = -3.0
    elif kind == "increasing":
        a = np.arange(n, dtype=np.float32)
    elif kind == "decreasing":
        a = np.arange(n, 0, -1).astype(np.float32)
    return a


EVICT = [0, 1, 2, 63, 64, 65, 200, 777, 1500, 2304, 300, 300]


def budgets(lens, cs, recent, rng):
    nc = [max(n - recent, 0) // cs for n in lens]
    b = [int(rng.integers(0, max(c, 1) + 1)) for c in nc]
    b[3], b[7], b[8], b[10], b[11] = -1, 0, max(nc[8] - 1, 0), 1, nc[11] + 5
    return b


@pytest.mark.parametrize("kind", ["any", "ties", "equal", "special", "increasing", "decreasing"])
@pytest.mark.parametrize("dtype,cs,recent", [("bf16", 1, 0), ("bf16", 8, 64), ("f32", 5, 33), ("bf16", 64, 1),
                                             ("f32", 16, 0), ("bf16", 12, 3000), ("bf16", 3, 1000)])
@pytest.mark.parametrize("max_rows", [2304, 40000])
def test_evict(kind, dtype, cs, recent, max_rows):
    rng = np.random.default_rng(31)
    lens = EVICT
    d = Dense(rng, lens, dtype)
    a = [torch.from_numpy(np.concatenate([acc_rows(rng, n, kind), np.full(4, 9.0, np.float32)])).to(DEV) for n in lens]
    b = budgets(lens, cs, recent, rng)
    k0, v0, a0 = [x.clone() for x in d.k], [x.clone() for x in d.v], [x.clone() for x in a]
    new = d.lens.clone()
    ck.evict_kv(d.table, new, ck.acc_table([x.data_ptr() for x in a], DEV), torch.tensor(b, dtype=torch.int32, device=DEV),
                cs=cs, recent=recent, max_rows=max_rows, dtype=DT[dtype])
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        rows = R.evict(a0[i][:n].cpu().numpy(), b[i], cs, recent)
        assert int(new[i]) == len(rows), (i, n)
        at = torch.from_numpy(rows).to(DEV)
        for x, x0 in ((d.k[i], k0[i]), (d.v[i], v0[i])):
            assert same(x[:len(rows)], x0[at]), (i, n, b[i])
            assert same(x[len(rows):], x0[len(rows):]), (i, n, b[i])
        assert same(a[i][:len(rows)], a0[i][at]) and not a[i][len(rows):n].any() and bool((a[i][n:] == 9).all()), i


@pytest.mark.parametrize("kind", ["any", "ties", "special"])
@pytest.mark.parametrize("fmt,dtype,block,cs,recent", [("int8", "bf16", 32, 32, 0), ("e4m3", "bf16", 64, 64, 100),
                                                       ("int8", "f32", 32, 96, 5), ("e4m3", "f32", 64, 128, 64)])
def test_evict_8_bit(kind, fmt, dtype, block, cs, recent):
    rng = np.random.default_rng(32)
    lens = EVICT
    q8 = Eight([n + block for n in lens], fmt, block, dtype)
    for i, n in enumerate(lens):
        q8.fill(i, dense(rng, n, dtype).double().numpy(), dense(rng, n, dtype).double().numpy())
    a = [torch.from_numpy(np.concatenate([acc_rows(rng, n, kind), np.full(4, 9.0, np.float32)])).to(DEV) for n in lens]
    b = budgets(lens, cs, recent, rng)
    old, rows0 = [q8.state(i) for i in range(len(lens))], [q8.host(i, n) for i, n in enumerate(lens)]
    a0, new = [x.clone() for x in a], lens_of(*lens)
    ck.evict_kv_q8(q8.views, new, ck.acc_table([x.data_ptr() for x in a], DEV),
                   torch.tensor(b, dtype=torch.int32, device=DEV), cs=cs, recent=recent, max_rows=2304)
    torch.cuda.synchronize()
    for i, n in enumerate(lens):
        rows = R.evict(a0[i][:n].cpu().numpy(), b[i], cs, recent)
        m, nb = len(rows), len(rows) // block
        assert int(new[i]) == m, (i, n)
        for x, x0 in zip(q8.host(i, m), rows0[i]):
            assert np.array_equal(x, x0[rows]), (i, n, b[i])
        for name, x0 in zip(Eight.PARTS, old[i]):
            keep = {"k": nb * block, "v": nb * block, "ks": nb, "vs": nb, "kt": 0, "vt": 0}[name]
            assert same(q8.p[i][name][keep:], x0[keep:]), (i, name)
        assert same(a[i][:m], a0[i][torch.from_numpy(rows).to(DEV)]) and not a[i][m:n].any(), i


@pytest.mark.parametrize("kind,n,cs,max_rows", [("dense", 2304, 8, 2304), ("dense", 2304, 8, 20000),
                                                ("int8", 2335, 32, 2400), ("int8", 2335, 32, 20000),
                                                ("e4m3", 3071, 64, 20000)])
def test_evict_many_views(kind, n, cs, max_rows):
    # many workgroups per view at work at once: what one of them writes, another may not have
    # read yet
    rng = np.random.default_rng(35)
    V, recent = 160, 64
    lens = [n - int(x) for x in rng.integers(0, 300, V)]
    a = torch.from_numpy(np.exp(2 * rng.standard_normal((V, n))).astype(np.float32)).to(DEV)
    a0, new = a.clone(), lens_of(*lens)
    b = [int(x) for x in rng.integers(0, n // cs, V)]
    budget, table = torch.tensor(b, dtype=torch.int32, device=DEV), ck.acc_table([x.data_ptr() for x in a], DEV)
    if kind == "dense":
        k = torch.randint(-30000, 30000, (V, n, D), dtype=torch.int16, device=DEV).view(torch.bfloat16)
        v = torch.randint(-30000, 30000, (V, n, D), dtype=torch.int16, device=DEV).view(torch.bfloat16)
        kv = ck.kv_table([(x.data_ptr(), y.data_ptr()) for x, y in zip(k, v)], DEV)
        old = k.clone(), v.clone()
        ck.evict_kv(kv, new, table, budget, cs=cs, recent=recent, max_rows=max_rows, dtype=torch.bfloat16)
    else:
        q8 = ck.q8_alloc([n] * V, DEV, fmt=kind, block=cs, dtype=torch.bfloat16)
        for i in range(V):
            for j in range(2):
                q8.hold[6 * i + j].copy_(torch.randint(-100, 100, q8.hold[6 * i + j].shape, dtype=torch.int8))
                q8.hold[6 * i + 2 + j].copy_(torch.rand(q8.hold[6 * i + 2 + j].shape))
        old = [t.clone() for t in q8.hold]
        ck.evict_kv_q8(q8, new, table, budget, cs=cs, recent=recent, max_rows=max_rows)
    torch.cuda.synchronize()
    for i, m in enumerate(lens):
        rows = R.evict(a0[i, :m].cpu().numpy(), b[i], cs, recent)
        at = torch.from_numpy(rows).to(DEV)
        assert int(new[i]) == len(rows), i
        assert same(a[i, :len(rows)], a0[i, at]) and not a[i, len(rows):m].any() and same(a[i, m:], a0[i, m:]), i
        if kind == "dense":
            assert same(k[i, :len(rows)], old[0][i, at]) and same(v[i, :len(rows)], old[1][i, at]), i
            assert same(k[i, len(rows):], old[0][i, len(rows):]), i
        else:
            nb = len(rows) // cs
            for j in range(2):
                assert same(q8.hold[6 * i + j][:nb * cs], old[6 * i + j][at[:nb * cs]]), i
                assert same(q8.hold[6 * i + 2 + j][:nb], old[6 * i + 2 + j][at[:nb * cs:cs] // cs]), i
                assert same(q8.hold[6 * i + 4 + j], old[6 * i + 4 + j]), i


@pytest.mark.parametrize("n,cs,budget", [(16384, 1, 5000), (16385, 1, 5000), (16500, 1, 16400), (70001, 1, 20000), (70001, 1, 60000), (40000, 1, 32768), (300000, 8, 5000)])
def test_evict_long_views(n, cs, budget):
    # more chunks than a workgroup keeps in LDS, beside a short view and one that stays
    rng = np.random.default_rng(33)
    lens = [n, 100, n]
    d = Dense(rng, lens, "bf16", 0)
    a = [torch.from_numpy(acc_rows(rng, m, "any")).to(DEV) for m in lens]
    a[0][5:5000] = 0.5                            # many ties
    b = [budget, 20, -1]
    k0, a0, new = [x.clone() for x in d.k], [x.clone() for x in a], d.lens.clone()
    ck.evict_kv(d.table, new, ck.acc_table([x.data_ptr() for x in a], DEV), torch.tensor(b, dtype=torch.int32, device=DEV),
                cs=cs, recent=50, max_rows=n, dtype=torch.bfloat16)
    for i, m in enumerate(lens):
        rows = R.evict(a0[i].cpu().numpy(), b[i], cs, 50)
        assert int(new[i]) == len(rows)
        at = torch.from_numpy(rows).to(DEV)
        assert same(d.k[i][:len(rows)], k0[i][at]) and same(a[i][:len(rows)], a0[i][at]) and not a[i][len(rows):].any()


def test_evict_views_out_of_range_are_left_alone():
    rng = np.random.default_rng(34)
    d = Dense(rng, [500, 500, 500], "bf16")
    a = [torch.rand(500, device=DEV) for _ in range(3)]
    d.lens[1] = -3
    k0, a0, was = [x.clone() for x in d.k], [x.clone() for x in a], d.lens.clone()
    ck.evict_kv(d.table, d.lens, ck.acc_table([x.data_ptr() for x in a], DEV),
                torch.tensor([10, 10, 10], dtype=torch.int32, device=DEV), cs=8, recent=0, max_rows=400,
                dtype=torch.bfloat16)
    assert torch.equal(d.lens, was)
    assert all(same(x, y) for x, y in zip(d.k + a, k0 + a0))

"""Calls on caches in pages at the ends of what their arguments may be."""
import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck
from test_gpu_paged import BF16, DEV, F32, append, cache_of, host, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [2 ** 63 - 1, 2 ** 63 - 5, 2 ** 62, 6 * 16 + 1, 6 * 16, 6 * 16 - 2, -1, -2 ** 63])
def test_lengths_of_any_size_are_checked(L):
    """A length that no call leaves, or that leaves no room for the new tokens (three are): the
    sequence stays as it is in every call, its neighbour's rows are appended."""
    c, s = cache_of(60, 16, 3, 2, 6, BF16)
    append(c, s, [0, 2], [50, 40], 2, 1)
    for h in range(2):
        c.lens[0, h] = L if h else 50
    before = R.Pages.of(c)
    plan = ck.paged_plan(c, [0, 2], [3, 1], [[96] * 2] * 2, 2)
    k, v = (randn((4, 2, 128), i, BF16) for i in (5, 6))
    over = torch.zeros(1, dtype=torch.int32, device=DEV)
    ck.append_kv_paged(plan, c, k, v, over)
    assert over.item() == 1
    before.append([2], [1], host(k[3:]), host(v[3:]))
    before.same(c)
    fine = 0 <= L <= 96
    out, lse = ck.attn_paged(plan, c, randn((4, 2, 128), 7, BF16))
    assert torch.isfinite(out.float()).all() and (fine or (out[:3, 1] == 0).all() and (lse[:3, 1] == -float("inf")).all())
    if not fine:
        over.zero_()
        ck.compact_kv_paged(c, 0, [1], torch.zeros((1, 700), dtype=torch.int32, device=DEV), 1, 0, over)    # a list of its own launch
        ck.compact_kv_paged(c, 0, [1], torch.zeros((1, 7), dtype=torch.int32, device=DEV), 1, 5, over)
        assert over.item() == 1
        ck.drop_paged(c, torch.tensor([0, 0, 0], device=DEV))
        before.same(c)


@pytest.mark.parametrize("new,hkv", [(1, 4), (3, 1), (1, 1), (0, 4)])
def test_strides_of_dimensions_of_size_one_do_not_matter(new, hkv):
    """One token, or one head: k by itself and v a part of a projection of all, whose strides
    differ where they lead nowhere; one that is no multiple of 16 bytes, too."""
    c, s = cache_of(40, 16, 2, hkv, 4, BF16)
    append(c, s, [1], [5], hkv, 1)
    plan = ck.paged_plan(c, [1], [new], [[20] * hkv], hkv)
    k = randn((new, hkv, 128), 3, BF16)
    if hkv > 1:                                                  # [token][3 hkv d + 8]: q, k and v side by side
        v = randn((max(new, 1), 3 * hkv * 128 + 8), 4, BF16).as_strided((new, hkv, 128), (3 * hkv * 128 + 8, 128, 1), 2 * hkv * 128)
    else:                                                        # [token][d], any stride of the one head
        v = randn((new, 128), 4, BF16).as_strided((new, 1, 128), (128, 77, 1))
    ck.append_kv_paged(plan, c, k, v)
    ck.attn_paged(plan, c, randn((new, hkv, 128), 5, BF16))
    s.append([1], [new], host(k), host(v))
    s.same(c)


def test_strides_that_differ_are_refused():
    c, _ = cache_of(40, 16, 2, 4, 4, BF16)
    plan = ck.paged_plan(c, [1], [2], [[20] * 4], 4)
    k, v = randn((2, 4, 128), 3, BF16), randn((2, 3, 4, 128), 4, BF16)[:, 2]
    with pytest.raises(ValueError):
        ck.append_kv_paged(plan, c, k, v)
    assert c.lens.sum().item() == 0


@pytest.mark.parametrize("n", [256, 257, 600])
def test_forks_of_any_number(n):
    """More pairs than one launch takes, one of them to a slot that is not empty, in the last launch;
    a list with a bad slot at its end forks none."""
    c, s = cache_of(80, 16, n + 5, 2, 4, BF16)
    append(c, s, [0, 1, n + 2], [37, 16, 3], 2, 1)
    src, dst = [i % 3 for i in range(n)], list(range(3, n + 3))       # (slot 2 is empty; n + 2 holds rows)
    ref = torch.zeros(1, dtype=torch.int32, device=DEV)
    with pytest.raises(Exception, match="slot"):
        ck.fork_paged(c, src + [0], dst + [n + 5], ref)
    s.same(c)
    ck.fork_paged(c, src, dst, ref)
    assert s.fork(src, dst) is True and ref.item() == 1
    s.same(c)


def test_decoding_over_pages_gives_what_decode_attn_gives():
    """A prompt's cache with two of four heads cut back, in pages and dense: three more tokens,
    each attended for by both, and both held to the same 64-bit results."""
    n, hkv, G, cs, tail, b = 900, 4, 4, 8, 32, 20
    hq = hkv * G
    k, v = (randn((hkv, n + 3, 128), i, BF16) for i in (1, 2))
    idx = ck.select_critical(randn((hq, tail, 128), 7, BF16), k[:, :n].contiguous(), [1, 3], cs, b)
    lens = torch.full((hkv,), n, dtype=torch.int64, device=DEV)
    kc, vc = ck.compact_kv(k[:, :n].contiguous(), v[:, :n].contiguous(), [1, 3], idx, cs, tail, lens)
    dense = [[torch.zeros((n + 3, 128), dtype=BF16, device=DEV) for _ in "kv"] for _ in range(hkv)]
    for h in range(hkv):
        for to, full, cut in zip(dense[h], (k, v), (kc, vc)):
            rows = cut[(1, 3).index(h)] if h in (1, 3) else full[h, :n]
            to[:int(lens[h])] = rows[:int(lens[h])]
    c, _ = cache_of(80, 64, 2, hkv, 16, BF16)
    plan = ck.paged_plan(c, [1], [n], [[n] * hkv], hq)
    ck.append_kv_paged(plan, c, k[:, :n].transpose(0, 1), v[:, :n].transpose(0, 1))
    ck.compact_kv_paged(c, 1, [1, 3], idx, cs, tail)
    assert torch.equal(c.lens[1], lens)
    plan, dense_plan = ck.paged_plan(c, [1], [1], [[n + 3] * hkv], hq), ck.decode_plan([n + 3] * hkv, hq, hkv, DEV)
    table = ck.kv_table([(a.data_ptr(), w.data_ptr()) for a, w in dense], DEV)
    for t in range(3):
        k1, v1 = (x[:, n + t].unsqueeze(0).contiguous() for x in (k, v))
        ck.append_kv_paged(plan, c, k1, v1)
        for h in range(hkv):
            dense[h][0][int(lens[h])], dense[h][1][int(lens[h])] = k1[0, h], v1[0, h]
        lens += 1
        q = randn((1, hq, 128), 20 + t, BF16)
        out, lse = ck.attn_paged(plan, c, q)
        want, want_lse = ck.decode_attn(dense_plan, q, table, lens.view(1, hkv))
        s = R.Pages.of(c)
        for h in range(hkv):
            g = slice(h * G, (h + 1) * G)
            kk, vv = s.rows(1, h)
            assert np.array_equal(kk, host(dense[h][0])[:len(kk)]) and np.array_equal(vv, host(dense[h][1])[:len(kk)])
            o, z, A, B = R.attention(host(q)[:, g], kk, vv, 1, 128 ** -0.5)
            for a, l, dtype in ((out, lse, BF16), (want, want_lse, F32)):        # decode_attn: fp32 weights and results
                eo, ez = R.bounds(o, z, A, B, len(kk), dtype, G)
                assert (np.abs(host(a)[:, g] - o) <= eo).all() and (np.abs(host(l)[:, g] - z) <= ez).all()

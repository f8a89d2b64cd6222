"""Random calls on small pools that often run out of pages, against the plain forms:
the state bit for bit after every call, and attention of what was appended."""
import numpy as np
import pytest
import torch

import paged_ref as R
import paper_2608_30295_amd as ck
from test_gpu_paged import BF16, DEV, F32, cache_of, check_attention, host, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(8))
def test_calls_in_any_order(seed):
    r = np.random.RandomState(seed)
    dtype = BF16 if seed % 3 else F32
    page, hkv, G, slots = int(r.choice([16, 32, 64])), int(r.randint(1, 6)), int(r.choice([1, 2, 4, 8])), int(r.randint(2, 7))
    max_pages = int(r.randint(3, 12))
    c, s = cache_of(int(r.randint(slots * hkv, slots * hkv * max_pages + 2)), page, slots, hkv, max_pages, dtype, seed)
    flag = torch.zeros(1, dtype=torch.int32, device=DEV)
    for step in range(40):
        flag.zero_()
        kind = r.choice(["append"] * 5 + ["fork", "drop", "compact", "gather"])
        if kind == "append":
            some = [int(x) for x in r.permutation(slots)[:r.randint(1, slots + 1)]]
            new = [int(r.choice([0, 1, 1, 3, page - 1, page, 2 * page + 5])) for _ in some]
            bound = [[int(s.lens[x, h]) + m for h in range(hkv)] for x, m in zip(some, new)]
            plan = ck.paged_plan(c, some, new, bound, hkv * G)
            # rows that are parts of wider ones, as a fused projection leaves them
            wide = randn((max(sum(new), 1), 2 * hkv + 1, 128), 1000 * seed + step, dtype)[:sum(new)]
            k, v = wide[:, :hkv], wide[:, hkv:2 * hkv]
            ck.append_kv_paged(plan, c, k, v, flag)
            left = s.append(some, new, host(k), host(v))
            if not left and sum(new):
                check_attention(c, plan, some, new, hkv * G, 1000 * seed + step)
        elif kind == "fork":
            src, dst = (int(x) for x in r.permutation(slots)[:2])
            ck.fork_paged(c, [src], [dst], flag)
            left = s.fork([src], [dst])
        elif kind == "drop":
            rows = [int(r.choice([0, 0, -1, 1, page, 1000])) for _ in range(slots)]
            ck.drop_paged(c, torch.tensor(rows, device=DEV))
            s.drop(rows)
            left = False
        elif kind == "compact":
            heads = [int(x) for x in r.permutation(hkv)[:r.randint(1, hkv + 1)]]
            cs, tail, slot = int(r.choice([1, 8, 24])), int(r.choice([0, 5, 40])), int(r.randint(slots))
            idx = r.randint(-1, 12, size=(len(heads), int(r.randint(1, 9)))).astype(np.int32)
            ck.compact_kv_paged(c, slot, heads, torch.from_numpy(idx).to(DEV), cs, tail, flag)
            left = s.compact(slot, heads, idx, cs, tail)
        else:
            n, slot, left = int(r.randint(1, max_pages * page + 9)), int(r.randint(slots)), False
            out = torch.full((2, hkv, n + 1, 128), 5.0, dtype=dtype, device=DEV)
            ck.gather_kv_paged(c, [slot], ck.kv_table([[out[0, h].data_ptr(), out[1, h].data_ptr()] for h in range(hkv)], DEV), n)
            for h in range(hkv):
                for got, rows in zip(host(out[:, h]), s.rows(slot, h)):
                    m = min(len(rows), n)
                    assert np.array_equal(got[:m], rows[:m]) and (got[m:] == 5).all()
        assert bool(flag.item()) == left, (step, kind)
        s.same(c)

"""Generation on caches that are evicted now and then, planned for the rows that can be
left: what README and evict_kv say of the bound, and the steps under the new plan."""
import numpy as np
import pytest
import torch

import paper_2608_30295_amd as ck
from test_gpu_cache import D, DEV, Dense, Eight, accs, check_attention, dense, lens_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,cs", [("e4m3", 64), ("int8", 128), ("bf16", 8)])
def test_steps_under_the_plan_of_the_rows_that_stay(kind, cs):
    rng = np.random.default_rng(71)
    B, hkv, G, cap, recent, every = 2, 2, 4, 4096, 128, 20
    start, chunks = [4000, 3000, 100, cs * 3 + recent - 10], [512 // cs, 1024 // cs, 2, 3]
    src = Dense(rng, start, "bf16", room=cap)
    lens, capacity = lens_of(*start), lens_of(*[cap] * 4)
    budget = torch.tensor(chunks, dtype=torch.int32, device=DEV)
    if kind == "bf16":
        append = lambda k, v: ck.append_kv(src.table, capacity, lens, k, v)
        attend = lambda plan, q, table: ck.decode_attn_weights(plan, q, src.table, lens, table)
        evict = lambda table, most: ck.evict_kv(src.table, lens, table, budget, cs=cs, recent=recent, max_rows=most,
                                                dtype=torch.bfloat16)
        rows = lambda i, n: [x[i][:n].double().cpu().numpy() for x in (src.k, src.v)]
    else:
        q8 = Eight([cap] * 4, kind, 64, "bf16")
        ck.quantize_kv(src.table, lens, q8.views, max(start))
        append = lambda k, v: ck.append_kv_q8(q8.views, capacity, lens, k, v)
        attend = lambda plan, q, table: ck.decode_attn_q8(plan, q, q8.views, lens, acc=table)
        evict = lambda table, most: ck.evict_kv_q8(q8.views, lens, table, budget, cs=cs, recent=recent, max_rows=most)
        rows = q8.host
    a, _, table = accs(rng, [cap] * 4, 0)
    for x, n in zip(a, start):
        x[n:] = 0
    most, plan = [cap] * 4, ck.decode_plan([cap] * 4, hkv * G, hkv, DEV)
    for t in range(3 * every):
        k, v = (dense(rng, 4, "bf16").view(B, hkv, D).to(DEV) for _ in "kv")
        append(k, v)
        q, before = dense(rng, B * hkv * G, "bf16").view(B, hkv * G, D).to(DEV), [x.clone() for x in a]
        out, lse = attend(plan, q, table)
        n = lens.tolist()
        assert all(m <= w for m, w in zip(n, most)), (t, n, most)
        if t % every in (0, every - 1):
            check_attention(q, lambda i: rows(i, n[i]), n, hkv, out, lse, a, before, 1.0)
        if t % every == every - 1:
            evict(table, max(most))
            assert all(m <= c * cs + recent + cs - 1 for m, c in zip(lens.tolist(), chunks))
            if t == every - 1:
                most = [min(cap, c * cs + recent + cs - 1 + every) for c in chunks]
                plan = ck.decode_plan(most, hkv * G, hkv, DEV)
    assert max(lens.tolist()) < 1300 and plan.plan.max_len_total == sum(most)

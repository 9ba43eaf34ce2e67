"""Plans that the GPU makes for batches of unlike shapes by turns, with attention between them: each is one plan as a whole."""
import pytest
import torch

from _kv16_plan import check_plan
from test_kv16_plan_cpu import BATCHES

pytestmark = pytest.mark.gpu


def test_plans_of_unlike_batches_by_turns(kvlib):
    from paper_2603_12707_gb300 import kv4, kv16
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    cases = []
    for name, (own, prefix_lens, prefix_of, hq, hkv, dim) in sorted(BATCHES.items()):
        batch, lens = len(own), own + prefix_lens
        i32 = dict(dtype=torch.int32, device="cuda")
        pool = kv16.Pool.empty(4, hkv, dim)
        width = max((n + 15) // 16 for n in lens)
        tables = kv4.Tables(torch.zeros((len(lens), width), **i32), torch.tensor(lens, **i32))      # every page is page 0
        ids = [batch + g if g >= 0 else -1 for g in prefix_of]
        q = torch.randn((batch, hq, dim), device="cuda").to(pool.dtype)
        cases.append((name, pool, tables, ids, torch.tensor(ids, **i32), q, torch.empty_like(q), kv16.kv16_workspace(pool, hq, batch)))
    error = torch.zeros(1, dtype=torch.int32, device="cuda")
    for turn in range(40):
        order = cases if turn % 2 else cases[::-1]
        for name, pool, tables, ids, prefix_ids, q, out, ws in order:
            ws.fill_(turn)
            kv16.kv16_plan(pool, tables, q.shape[1], len(q), ws, prefix_ids=prefix_ids, device_error=error)
            if turn % 4 == 3:
                kv16.kv16_attention(pool, tables, q, out, ws, device_error=error)
        if turn % 8 < 6:
            continue
        for name, pool, tables, ids, prefix_ids, q, out, ws in cases:
            check_plan(ws[:1 << 22].cpu().numpy().tobytes(), tables.lens.tolist(), list(range(len(q))), ids, q.shape[1], pool.num_kv_heads,
                       pool.head_dim, sms)
    assert int(error) == 0

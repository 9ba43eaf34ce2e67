"""What a caller sees of an attention call that gave up a wait.  (A wait that runs out cannot be brought about without a kernel that
hangs; what it writes over the plan's first word is written there instead.)"""
import pytest
import torch

from _kv16_common import assert_attention, attention, make_pool, make_tables
from _kv16_plan import GAVE_UP, MADE

pytestmark = pytest.mark.gpu

TIMEOUT, PLAN = 2, 16      # KVC_DEVERR_*


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,batch", [(4, 2, 64, 3), (8, 2, 128, 20), (8, 2, 64, 60)])
def test_no_partial_results_are_passed_off(kvlib, dtype, hq, hkv, d, batch):
    from paper_2603_12707_gb300 import kv4, kv16
    lens = [20 + 3 * i for i in range(batch)] + [700]
    table, pages = make_tables(lens, 4)
    pool = kv16.Pool(*(x.cuda() for x in make_pool(pages, hkv, d, dtype, 1, table, lens)))
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    work, err = kv16.kv16_workspace(pool, hq, batch), torch.zeros(1, dtype=torch.int32, device="cuda")
    pre = torch.full((batch,), batch, dtype=torch.int32, device="cuda")
    q = torch.randn((batch, hq, d), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    out, lse = torch.zeros_like(q), torch.zeros((batch, hq), device="cuda")

    def plan():
        kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=pre, device_error=err)

    def attend():
        kv16.kv16_attention(pool, tabs, q, out, work, lse=lse, device_error=err)
        assert_attention(out, lse, attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, dtype), dtype)

    plan()
    attend()
    assert int(work.view(torch.int32)[0]) == MADE
    work.view(torch.int32)[0] = GAVE_UP
    for _ in range(2):                           # this call and those behind it, until there is a new plan
        err.zero_()
        kv16.kv16_attention(pool, tabs, q, out, work, lse=lse, device_error=err)
        assert torch.isnan(out).all() and torch.isnan(lse).all() and int(err) == TIMEOUT
    kv16.kv16_attention(pool, tabs, q, out, work)      # no error word, no lse
    assert torch.isnan(out).all()
    err.zero_()
    out.fill_(5.0)
    kv16.kv16_attention(pool, tabs, q[:-1], out[:-1], work, device_error=err)     # not this plan's batch, given up or not
    assert (out == 5.0).all() and int(err) == PLAN
    err.zero_()
    plan()
    attend()
    assert int(err) == 0

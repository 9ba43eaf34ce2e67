"""What a row's result depends on: its query, its tokens and the plan, and nothing of the rows beside it."""
import pytest
import torch

from _kv16_common import make_pool, make_tables

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("hq,hkv,d,batch", [(2, 2, 64, 8), (2, 1, 128, 4), (14, 2, 64, 1), (4, 2, 128, 30), (8, 2, 64, 50)])
def test_other_queries_change_nothing(kvlib, dtype, hq, hkv, d, batch):
    """Prefixes of up to 8 query rows of a KV head, whose rows lie in one warp, and larger ones: each query head alone is kept as it was and
    all others are made ten times as large, so that their references move elsewhere."""
    from paper_2603_12707_gb300 import kv4, kv16
    lens = [20 + 3 * i for i in range(batch)] + [700]
    table, pages = make_tables(lens, 4)
    pool = kv16.Pool(*(x.cuda() for x in make_pool(pages, hkv, d, dtype, 1, table, lens)))
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    work = kv16.kv16_workspace(pool, hq, batch)
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=torch.full((batch,), batch, dtype=torch.int32, device="cuda"))
    q = torch.randn((batch, hq, d), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()

    def attend(q):
        out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        kv16.kv16_attention(pool, tabs, q, out, work, lse=lse)
        return out, lse

    out, lse = attend(q)
    for row in {0, batch // 2, batch - 1}:
        for head in range(hq):
            other = q * 10
            other[row, head] = q[row, head]
            o, l = attend(other)
            assert torch.equal(o[row, head].view(torch.int16), out[row, head].view(torch.int16)), (row, head)
            assert torch.equal(l[row, head], lse[row, head]), (row, head)

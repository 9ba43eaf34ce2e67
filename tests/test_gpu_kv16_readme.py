"""The usage sample of the 16-bit serving step, run as it stands: queries and keys turned by their positions behind the prefix."""
import os
import re

import pytest
import torch

from _kv16_common import P, assert_attention, assert_rows, attention, inv_freq, turned

pytestmark = pytest.mark.gpu

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


def test_the_sample_turns_rows_by_their_positions_behind_the_prefix(kvlib):
    from paper_2603_12707_gb300 import kv4, kv16
    sample, = [b for b in re.findall(r"```python\n(.*?)```", open(README).read(), flags=re.S) if "kv16_plan" in b]
    batch, hq, hkv, d, prefixes, own = 6, 28, 4, 128, [100, 33], [3, 0, 17, 16, 1, 40]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    g = torch.Generator().manual_seed(1)
    x = [torch.randn((batch, h, d), generator=g).bfloat16() for h in (hq, hkv, hkv)]
    weights = [(1 + 0.1 * torch.randn(d, generator=g)).bfloat16() for _ in range(2)]
    tables = kv4.Tables.empty(8192, 64, 2048)
    start = own + prefixes
    kv4.kv_tables_step(tables, dev(list(range(8))), dev(start), torch.empty(sum(start), dtype=torch.int64, device="cuda"))
    of = [0, 1, 0, -1, 1, 0]
    first = [prefixes[i] if i >= 0 else 0 for i in of]
    q, k, v = (t.cuda() for t in x)
    names = dict(tables=tables, seq_ids=dev(list(range(batch))), new_lens=dev([1] * batch), prefix_ids=dev([batch + i if i >= 0 else -1 for i in of]),
                 slots=torch.empty(batch, dtype=torch.int64, device="cuda"), positions=dev([0] * batch), first=dev(first), batch=batch,
                 inv_freq=inv_freq(d // 2), axes=[j % 3 for j in range(d // 2)], k_new=k, v_new=v, q=q, q_out=torch.empty_like(q),
                 out=torch.empty_like(q), k=k, k_out=torch.empty_like(k), q_weight=weights[0].cuda(), k_weight=weights[1].cuda(), kv4=kv4, torch=torch)
    exec(sample, names)
    torch.cuda.synchronize()
    positions = [[a + n for a, n in zip(first, own)]]
    freq = inv_freq(d // 2)
    pool, slots = names["pool"], names["slots"].cpu()
    want = [turned(x[i], positions, freq, None, weight=weights[i]) for i in range(2)]
    assert_rows(pool.k.cpu()[slots // P, :, slots % P], want[1], torch.bfloat16)
    # The sample's last line turns the same rows without norms.
    assert_rows(names["q_out"], turned(x[0], positions, freq, None), torch.bfloat16)
    assert_rows(names["k_out"], turned(x[1], positions, freq, None), torch.bfloat16)
    qn = torch.empty_like(q)
    kv16.kv_qk_rope(kv16.Rope(freq), dev(positions[0]), q, None, qn, None, q_weight=weights[0].cuda())
    lens = [n + 1 for n in own] + prefixes
    ref = attention(pool.k, pool.v, tables.block_table.cpu().numpy()[:8], lens, None, [batch + i if i >= 0 else -1 for i in of], qn, d ** -0.5, torch.bfloat16)
    assert_attention(names["out"], None, ref, torch.bfloat16)

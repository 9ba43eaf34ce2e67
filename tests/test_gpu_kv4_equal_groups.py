"""Groups of equal elements of any size: a step of 0, codes of 8, and the element itself as the middle."""
import numpy as np
import pytest
import torch

from _kv4_common import P, block_bytes
from test_gpu_kv4 import BF, FP, SHAPES, kv4, write_reference  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
def test_groups_of_equal_elements(kv4, d, group, dtype):
    n, h = 64, 2
    g = torch.Generator().manual_seed(d + group)
    e = torch.randint(-132, 128, (n, h, d // group), generator=g) if dtype is BF else torch.randint(-24, 16, (n, h, d // group), generator=g)
    x = (torch.rand(e.shape, generator=g, dtype=torch.float64) * 0.9 + 1) * 2.0 ** e.double() * torch.where(torch.rand(e.shape, generator=g) < 0.5, -1, 1)
    most = torch.finfo(dtype).max
    k = x.clamp(-most, most).to(dtype).repeat_interleave(group, -1)
    v = k.flip(0).contiguous()
    pool = kv4.Pool.empty(n // P, h, d, group, dtype)
    slots = np.arange(n)
    kv4.kv4_write(pool, torch.from_numpy(slots).cuda(), k.cuda(), v.cuda())
    want = np.zeros((n // P, h, block_bytes(d, group)), np.uint8)
    write_reference(want, slots, k, v, group)
    assert (want[..., :16 * d] == 0x88).all()          # codes of 8
    assert (pool.data.cpu().numpy() == want).all()
    back = [torch.empty((n, h, d), dtype=dtype, device="cuda") for _ in range(2)]
    kv4.kv4_read(pool, torch.from_numpy(slots).cuda(), *back)
    assert torch.equal(back[0].cpu(), k) and torch.equal(back[1].cpu(), v)

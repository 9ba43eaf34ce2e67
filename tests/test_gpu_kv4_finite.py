"""Groups that hold numbers at the end of the 16-bit type's range: written, read back and attended to, what is
finite stays finite and near."""
import numpy as np
import pytest
import torch

from _kv4_common import P, block_bytes, put, quantise, unpack
from test_gpu_kv4_sums import BF, FP, SHAPES

pytestmark = pytest.mark.gpu

OVER = {FP: 65520.0, BF: 2.0 ** 128 - 2.0 ** 119}       # the least that rounds to infinity
MOST = {FP: 65504.0, BF: 2.0 ** 128 - 2.0 ** 120}
UNIT = {FP: 2.0 ** -10, BF: 2.0 ** -7}                  # a unit in the last place, relative, at most


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def next_down(x):
    """The next smaller number of positive 16-bit numbers."""
    return (x.view(torch.int16) - 1).view(x.dtype)


def toward_zero(x, dtype):
    """float32 to 16 bits, toward zero."""
    y = x.to(dtype)
    return torch.where(y.double().abs() > x.double().abs(), next_down(y.abs()) * torch.sign(y), y)


def reference(x, group):
    """Codes, s and z of kvdecode4.h: quantise(), with the rule for groups that would not stay finite."""
    codes, s, z = quantise(x, group)
    lo = x.float().unflatten(-1, (-1, group)).amin(-1)
    sd, zd = s.double(), z.double()
    over = (zd + 7 * sd >= OVER[x.dtype]) | (zd - 8 * sd <= -OVER[x.dtype])
    s = torch.where(over, next_down(s), s)
    z = torch.where(over, toward_zero((lo.double() + 8 * s.double()).float(), x.dtype), z)
    y = x.double().unflatten(-1, (-1, group))
    c = (torch.round((y - z.double()[..., None]) / s.double()[..., None]) + 8).clamp(0, 15)
    codes = np.where(over[..., None].expand(c.shape).numpy(), c.numpy(), codes.reshape(c.shape)).astype(np.int64)
    return codes.reshape(x.shape), s, z, int(over.sum())


def extreme_rows(n, h, d, group, dtype, seed):
    """Groups whose largest or smallest element is the type's last number, the other end anywhere."""
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.rand(s, generator=g, dtype=torch.float64)  # noqa: E731
    shape = (n, h, d // group)
    far = torch.where(r(*shape) < 0.5, 1 - 2 * r(*shape), 1 - 2.0 ** (-10 * r(*shape)))      # the other end: anywhere, or near
    far = torch.where(r(*shape) < 0.2, -torch.ones(shape, dtype=torch.float64), far)         # or the other last number
    far = torch.where(r(*shape) < 0.1, torch.zeros(shape, dtype=torch.float64), far)
    x = far[..., None] + (1 - far)[..., None] * r(*shape, group)
    x[..., 0], x[..., 1] = 1.0, far
    x = x * torch.where(r(*shape) < 0.5, 1.0, -1.0)[..., None]
    return (x * MOST[dtype]).clamp(-MOST[dtype], MOST[dtype]).to(torch.float32 if dtype is BF else torch.float64).to(dtype).flatten(-2)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
def test_the_ends_of_the_range_stay_finite(kv4, d, group, dtype):
    n, h = 320, 3
    k, v = (extreme_rows(n, h, d, group, dtype, s) for s in (1, 2))
    assert torch.isfinite(k).all() and torch.isfinite(v).all()
    slots = torch.randperm(n, generator=torch.Generator().manual_seed(3))
    pool = kv4.Pool.empty(n // P, h, d, group, dtype)
    kv4.kv4_write(pool, slots.cuda(), k.cuda(), v.cuda())
    back = [torch.empty((n, h, d), dtype=dtype, device="cuda") for _ in range(2)]
    kv4.kv4_read(pool, slots.cuda(), *back)
    want = np.zeros((n // P, h, block_bytes(d, group)), np.uint8)
    changed = 0
    for side, (x, y) in enumerate(zip((k, v), back)):
        y = y.cpu().double()
        assert torch.isfinite(y).all(), int((~torch.isfinite(y)).sum())
        codes, s, z, over = reference(x, group)
        changed += over
        for t in range(n):
            for i in range(h):
                put(want[slots[t] // P, i], int(slots[t]) % P, side, codes[t, i], s[t, i], z[t, i], d, group)
        s, z = (w.double().repeat_interleave(group, -1) for w in (s, z))
        # half a step; 15 steps that are up to 1.5 units short; the middle a unit off; and the value's own rounding
        lim = s * (0.5 + 15 * 1.5 * UNIT[dtype]) + z.abs() * UNIT[dtype] + y.abs() * UNIT[dtype] / 2
        assert ((x.double() - y).abs() <= lim).all()
    assert changed > 20        # groups to which the rule applies are among them
    assert (pool.data.cpu().numpy() == want).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("n", [1, 40, 1000])
def test_attention_over_the_ends_of_the_range(kv4, d, group, dtype, n):
    """Rows whose V elements are the type's last numbers: weighted means are finite and near those."""
    h, b = 2, 3
    pages = (n + P - 1) // P
    g = torch.Generator().manual_seed(n)
    sign = torch.where(torch.rand((1, h, d), generator=g) < 0.5, -1.0, 1.0)
    shape = extreme_rows(1, h, d, group, FP, 5).double() / MOST[FP] if n == 1 else sign.double()
    scale = MOST[dtype] if dtype is FP else 2.0 ** 100        # (bf16: sums in 32 bits of n numbers past 2^100 are not finite)
    v = (shape * scale).to(torch.float32 if dtype is BF else torch.float64).to(dtype).expand(n, h, d).contiguous()
    k = torch.randn((n, h, d), generator=g).to(dtype)
    pool = kv4.Pool.empty(pages, h, d, group, dtype)
    kv4.kv4_write(pool, torch.arange(n, device="cuda"), k.cuda(), v.cuda())
    blocks = pool.data.cpu().numpy()
    c, s, z = unpack(blocks, d, group, dtype)[1]
    held = (s * (c - 8) + z)[0, :, 0]
    q = (torch.randn((b, h, d), generator=g) * 0.3).to(dtype)
    tabs = kv4.Tables(torch.arange(pages, dtype=torch.int32, device="cuda")[None].contiguous(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    out = torch.empty((b, h, d), dtype=dtype, device="cuda")
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, h), seq_ids=torch.zeros(b, dtype=torch.int32, device="cuda"))
    out = out.double().cpu().numpy()
    assert np.isfinite(out).all()
    # all values of an element are one: weights' roundings to 11 bits on 8 s, the sums', the output's own
    lim = 2.0 ** -11 * 8 * s[0, :, 0] + 1e-5 * (8 * s + np.abs(z))[0, :, 0] + UNIT[dtype] / 2 * np.abs(held)
    assert (np.abs(out - held) <= lim).all(), float((np.abs(out - held) - lim).max())

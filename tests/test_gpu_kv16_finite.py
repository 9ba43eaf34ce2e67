"""Scores and values far out in their range: what is finite gives finite outputs, and the right ones, in large runs of one and of two
tiles of rows, in small prefixes and over own tokens."""
import math

import pytest
import torch

from _kv16_common import P, UNIT, make_tables

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
LN2 = 0.6931472      # as a number of 32 bits its product with log2(e) is 1: scores are in log2 units

# (rows on a prefix, query heads, KV heads): records of own tokens, records of a small prefix, one tile of rows, two, three
SHAPES = [(0, 4, 2), (2, 4, 2), (20, 8, 2), (50, 8, 2), (80, 8, 2)]


def attend(kvlib, k, v, q, on_prefix, scale):
    """One token stream K, V [n, heads, d] for all rows, as a shared prefix or (on_prefix 0) as every row's own tokens."""
    from paper_2603_12707_gb300 import kv4, kv16
    n, hkv, d = k.shape
    batch, hq = q.shape[:2]
    lens = [n] if on_prefix == 0 else [0] * batch + [n]
    table, pages = make_tables(lens, n)
    row = torch.tensor(table[-1].astype("int64"))
    t = torch.arange(n)
    pools = [torch.full((pages, hkv, P, d), math.nan, dtype=k.dtype) for _ in range(2)]
    for pool, x in zip(pools, (k, v)):
        pool[row[t // P], :, t % P] = x
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    pool = kv16.Pool(*(x.cuda() for x in pools))
    tabs = kv4.Tables(dev(table.tolist()), dev(lens))
    work = kv16.kv16_workspace(pool, hq, batch)
    err = dev([0])
    ids, pre = (dev([0] * batch), None) if on_prefix == 0 else (None, dev([batch] * batch))
    kv16.kv16_plan(pool, tabs, hq, batch, work, seq_ids=ids, prefix_ids=pre, device_error=err)
    out, lse = torch.empty_like(q, device="cuda"), torch.empty((batch, hq), device="cuda")
    kv16.kv16_attention(pool, tabs, q.cuda(), out, work, lse=lse, softmax_scale=scale, device_error=err)
    assert int(err) == 0
    return out.cpu().double(), lse.cpu().double()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("on_prefix,hq,hkv", SHAPES)
@pytest.mark.parametrize("sign", [1, -1])
def test_equal_scores_of_any_size(kvlib, dtype, d, on_prefix, hq, hkv, sign):
    """Every token of a row has the same score, from 2^16 to 2^34 in log2 units: the output is the mean of V.  (Scores are one product
    each, exact in 32 bits.  A common weight and its rounding cancel but for UNIT of the mean of |V|; sums of 500 terms in 32 bits: 2^-14.)"""
    n, g = 500, torch.Generator().manual_seed(d)
    batch = on_prefix or 6
    k = torch.zeros((n, hkv, d), dtype=dtype)
    k[..., 0] = 60000.0 if dtype is FP else 65536.0 * 1.5
    v = (torch.randn((n, hkv, d), generator=g) + 1).to(dtype)
    q = torch.zeros((batch, hq, d), dtype=dtype)
    q[..., 0] = (sign * torch.exp2(16 * torch.rand((batch, hq), generator=g)) * (1 + torch.rand((batch, hq), generator=g)) / 2).to(dtype)
    out, lse = attend(kvlib, k, v, q, on_prefix, 1.0)
    vd = v.double().repeat_interleave(hq // hkv, 1)
    want, mag = vd.mean(0), vd.abs().mean(0)
    assert torch.isfinite(out).all()
    err = (out - want).abs()
    assert (err <= (UNIT[dtype] * (1 + UNIT[dtype]) * 1.001 + UNIT[dtype]) * mag + 2.0 ** -14 * vd.abs().max()).all(), float(err.max())
    score = q[..., 0].double() * float(k[0, 0, 0])
    assert ((lse - score - math.log(n)).abs() <= 2.0 ** -21 * score.abs() + 2.0 ** -14).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("on_prefix,hq,hkv", SHAPES)
@pytest.mark.parametrize("base", [2.0 ** e for e in range(18, 28)])
def test_far_scores_that_rise(kvlib, dtype, on_prefix, hq, hkv, base):
    """Scores of base and, later on, of base + 8 units in the last place or so: the reference does not move for them, or it does.  The
    scores are whole numbers below 2^24 units in the last place, so all of this is exact but for the weights' rounding."""
    step = max(8.0, base * 2.0 ** -22)           # (a multiple of the unit in the last place)
    n, d, batch = 200, 64, on_prefix or 6
    g = torch.Generator().manual_seed(3)
    k = torch.zeros((n, hkv, d), dtype=dtype)
    k[..., 0] = 2.0 ** 14
    k[n // 2:, :, 1] = 8.0                       # rises in the middle of a tile
    v = (torch.randn((n, hkv, d), generator=g) + 1).to(dtype)
    q = torch.zeros((batch, hq, d), dtype=dtype)
    q[..., 0], q[..., 1] = base / 2.0 ** 14, step / 8.0
    out, lse = attend(kvlib, k, v, q, on_prefix, LN2)
    w = torch.exp2(-step * (torch.arange(n) < n // 2).double())
    vd = v.double().repeat_interleave(hq // hkv, 1)
    want = (w[:, None, None] * vd).sum(0) / w.sum()
    mag = (w[:, None, None] * vd.abs()).sum(0) / w.sum()
    assert torch.isfinite(out).all()
    err = (out - want).abs()
    assert (err <= (UNIT[dtype] * (1 + UNIT[dtype]) * 1.001 + UNIT[dtype]) * mag + 2.0 ** -14 * vd.abs().max()).all(), float(err.max())
    top = (base + step) * math.log(2)
    assert ((lse - top - math.log(w.sum())).abs() <= 2.0 ** -21 * top + 2.0 ** -14).all()


@pytest.mark.parametrize("on_prefix,hq,hkv", SHAPES)
def test_values_at_the_end_of_the_range(kvlib, on_prefix, hq, hkv):
    """V is 65504 or its negative in all tokens of an element.  The tokens that count for most follow, in nearly all of a worker's shares, others that
    set the reference 7 lower; their weights, 2^14.0007, are rounded up by 2^-11.1.  An average of equal numbers stays among the type's numbers."""
    n, d, batch = 100000, 64, on_prefix or 6
    score = torch.full((n,), -20.0)
    score[::128], score[1000::2048] = 0.0, 7.0
    k = torch.zeros((n, hkv, d), dtype=FP)
    k[..., 0], k[1000::2048, :, 1] = score.to(FP)[:, None], 0.76
    v = torch.full((n, hkv, d), 65504.0, dtype=FP)
    v[..., 1::2] *= -1
    q = torch.zeros((batch, hq, d), dtype=FP)
    q[..., 0], q[..., 1] = 1.0, 2.0 ** -10
    out, lse = attend(kvlib, k, v, q, on_prefix, LN2)
    assert torch.isfinite(out).all()
    assert ((out - v[0].double().repeat_interleave(hq // hkv, 0)).abs() <= 65504 * 2.0 ** -10).all()
    exact = score.double() + k[:, 0, 1].double() * 2.0 ** -10
    assert ((lse - math.log(torch.exp2(exact).sum())).abs() <= 2.0 ** -14).all()


def test_infinite_values_stay_infinite(kvlib):
    n, d = 40, 64
    v = torch.zeros((n, 2, d), dtype=FP)
    v[3, 0, 5], v[7, 1, 9] = math.inf, -math.inf
    out, _ = attend(kvlib, torch.zeros((n, 2, d), dtype=FP), v, torch.ones((20, 4, d), dtype=FP), 20, 1.0)
    assert (out[:, :2, 5] == math.inf).all() and (out[:, 2:, 9] == -math.inf).all()
    out[:, :2, 5] = out[:, 2:, 9] = 0
    assert (out == 0).all()

"""The 16-bit serving step on the GPU against the plain reference of _kv16_common: rotated rows and written pages to one
rounding, attention over shared prefixes in 64 bits to the bound of its arithmetic."""
import math

import numpy as np
import pytest
import torch

from _kv16_common import (P, UNIT, assert_attention, assert_rows, attention, inv_freq, make_pool, make_tables, pages_of, turned)

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def kv16(kvlib):
    from paper_2603_12707_gb300 import kv16
    return kv16


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def err_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


# -------------------------------------------------------------------- rotation
def rows(n, heads, d, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((n, heads, d), generator=g) * scale).to(dtype)


def axes_of(kind, half):
    if kind == "one":
        return None, 1
    if kind == "turns":
        return [j % 3 for j in range(half)], 3
    return [0] * (half // 4) + [1] * (half // 4) + [2] * (half - 2 * (half // 4)), 3


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,rd", [(64, 64), (128, 128), (128, 64), (64, 16), (128, 48)])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("kind", ["one", "turns", "sections"])
@pytest.mark.parametrize("normed", [False, True])
def test_rotated_rows(kv16, dtype, d, rd, neighbours, kind, normed):
    n, hq, hkv = 37, 7, 3
    axes, num = axes_of(kind, rd // 2)
    freq = inv_freq(rd // 2, 1e6)
    pos = np.random.default_rng(d + rd).integers(-50, 1_000_000, (num, n)).astype(np.int32)
    q, k = rows(n, hq, d, dtype, 1, 3.0), rows(n, hkv, d, dtype, 2)
    qw, kw = (rows(1, 1, d, dtype, s).reshape(d) if normed else None for s in (3, 4))
    rope = kv16.Rope(freq, axes=axes, num_axes=num, neighbours=neighbours, scale=1.25)
    cu = lambda x: None if x is None else x.cuda()  # noqa: E731
    qo, ko = torch.full_like(q, float("nan")).cuda(), torch.full_like(k, float("nan")).cuda()
    kv16.kv_qk_rope(rope, torch.from_numpy(pos).cuda(), q.cuda(), k.cuda(), qo, ko, q_weight=cu(qw), k_weight=cu(kw), eps=1e-5)
    for got, x, w in ((qo, q, qw), (ko, k, kw)):
        assert_rows(got, turned(x, pos, freq, axes, neighbours, 1.25, w, 1e-5), dtype)


@pytest.mark.parametrize("n", [1, 2, 5, 31, 33, 700, 5000])
@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (14, 2, 64), (1, 1, 128), (9, 1, 64), (0, 5, 128), (6, 0, 64)])
def test_rows_of_every_number(kv16, n, hq, hkv, d):
    """Few tokens are shared among more warps; heads that do not fill a warp's turn."""
    freq = inv_freq(d // 2)
    pos = (np.arange(n) * 7 % 5001).astype(np.int32)
    rope = kv16.Rope(freq)
    q, k = (rows(n, h, d, BF, h + n) if h else None for h in (hq, hkv))
    w = rows(1, 1, d, BF, 9).reshape(d)
    out = [None if x is None else torch.full_like(x, float("nan")).cuda() for x in (q, k)]
    kv16.kv_qk_rope(rope, torch.from_numpy(pos).cuda(), None if q is None else q.cuda(), None if k is None else k.cuda(), *out,
                    q_weight=w.cuda())
    for got, x, ww in ((out[0], q, w), (out[1], k, None)):
        if x is not None:
            assert_rows(got, turned(x, pos, freq, None, weight=ww), BF)


@pytest.mark.parametrize("dtype", [BF, FP])
def test_slices_of_a_fused_projection_in_place(kv16, dtype):
    n, hq, hkv, d = 133, 6, 2, 128
    x = rows(n, hq + 2 * hkv, d, dtype, 5)
    pos = np.arange(n).astype(np.int32)
    freq = inv_freq(d // 2)
    y = x.cuda()
    q, k = y[:, :hq], y[:, hq:hq + hkv]
    kv16.kv_qk_rope(kv16.Rope(freq), torch.from_numpy(pos).cuda(), q, k, q, k)
    assert_rows(y[:, :hq + hkv], turned(x[:, :hq + hkv], pos, freq, None), dtype)
    assert torch.equal(y[:, hq + hkv:].cpu().view(torch.int16), x[:, hq + hkv:].view(torch.int16))


def test_far_positions_are_exact(kv16):
    """The angle is a whole number of 2^-64 turns: the last positions of 32 bits are as exact as the first."""
    d, n = 128, 64
    freq = inv_freq(d // 2, 5e5)
    pos = np.concatenate([2 ** 31 - 1 - np.arange(n // 2), -2 ** 31 + np.arange(n // 2)]).astype(np.int32)
    x = rows(n, 4, d, FP, 8)
    out = torch.empty_like(x).cuda()
    kv16.kv_qk_rope(kv16.Rope(freq), torch.from_numpy(pos).cuda(), x.cuda(), None, out, None)
    # position times frequency in 64 bits is off by 2^31 * 2^-53 radians: 2^-22, the reference's own
    ref, bound = turned(x, pos, freq, None)
    assert_rows(out, (ref, bound + 2.0 ** -22 * x.double().abs().amax(-1, keepdim=True)), FP)


def test_norms_alone_and_of_extreme_rows(kv16):
    d = 128
    x = rows(8, 2, d, BF, 3)
    x[0] = 0
    x[1] *= 2.0 ** 100
    x[2] = torch.finfo(BF).max
    x[3] *= 2.0 ** -90
    x[4] *= 2.0 ** 63
    x[5, 0, 3] = float("inf")
    x[6, 1, 7] = float("nan")
    w = rows(1, 1, d, BF, 4).reshape(d)
    out = torch.empty_like(x).cuda()
    kv16.kv_qk_rope(None, None, x.cuda(), None, out, None, q_weight=w.cuda())
    fine = [0, 1, 2, 3, 4, 7]
    assert_rows(out[fine], turned(x[fine], [], [], None, weight=w), BF)
    got = out.cpu()
    assert torch.isnan(got[5, 0, 3]) and (got[5, 0].nan_to_num() == 0).all()
    assert torch.isnan(got[6, 1]).all() and torch.isfinite(got[6, 0]).all() and torch.isfinite(got[5, 1]).all()


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("n,hq,hkv,d,rotated,normed", [(1, 28, 4, 128, True, False), (64, 32, 32, 128, True, True), (531, 14, 2, 64, True, False),
                                                       (33, 0, 5, 128, False, False), (77, 8, 8, 64, False, True), (3000, 4, 2, 128, True, True)])
def test_written_pages(kv16, dtype, n, hq, hkv, d, rotated, normed):
    rng = np.random.default_rng(n)
    pages = pages_of(n) + 4
    slots = rng.permutation(pages * P)[:n].astype(np.int64)
    skipped = rng.random(n) < 0.1
    slots[skipped] = -1
    freq = inv_freq(d // 2) if rotated else []
    pos = rng.integers(0, 100000, (1, n)).astype(np.int32)
    q, k, v = (rows(n, h, d, dtype, s) if h else None for h, s in ((hq, 1), (hkv, 2), (hkv, 3)))
    qw, kw = (rows(1, 1, d, dtype, s).reshape(d) if normed else None for s in (5, 6))
    pool = kv16.Pool(*(torch.full((pages, hkv, P, d), -3.0, dtype=dtype, device="cuda") for _ in range(2)))
    cu = lambda x: None if x is None else x.cuda()  # noqa: E731
    qo, err = None if q is None else torch.full_like(q, float("nan")).cuda(), err_word()
    kv16.kv16_write(pool, torch.from_numpy(slots).cuda(), k.cuda(), v.cuda(), rope=kv16.Rope(freq) if rotated else None,
                    positions=torch.from_numpy(pos).cuda() if rotated else None, q=cu(q), q_out=qo, q_weight=cu(qw), k_weight=cu(kw),
                    device_error=err)
    assert int(err) == 0
    if q is not None:
        assert_rows(qo, turned(q, pos, freq, None, weight=qw), dtype)
    flat = [x.cpu().transpose(1, 2).reshape(-1, hkv, d) for x in (pool.k, pool.v)]
    live = ~skipped
    assert_rows(flat[0][slots[live]], tuple(x[live] for x in turned(k, pos, freq, None, weight=kw)), dtype)
    assert torch.equal(flat[1][slots[live]].view(torch.int16), v[live].view(torch.int16))
    other = np.setdiff1d(np.arange(pages * P), slots)
    assert all((x[other] == -3.0).all() for x in flat)


def test_slots_outside_the_pool_are_reported(kv16):
    d, hkv, n = 64, 3, 6
    k, v = rows(n, hkv, d, BF, 1), rows(n, hkv, d, BF, 2)
    pool = kv16.Pool.empty(2, hkv, d)
    slots = torch.tensor([0, 32, -2, 2 ** 40, -1, 31], device="cuda")
    err = err_word()
    q = rows(n, 6, d, BF, 3)
    qo = torch.empty_like(q).cuda()
    kv16.kv16_write(pool, slots, k.cuda(), v.cuda(), q=q.cuda(), q_out=qo, device_error=err)
    assert int(err) == 1
    assert torch.equal(qo.cpu(), q)
    for x, y in ((pool.k, k), (pool.v, v)):
        flat = x.cpu().transpose(1, 2).reshape(-1, hkv, d)
        assert torch.equal(flat[0], y[0]) and torch.equal(flat[31], y[5]) and (flat[1:31] == 0).all()


# ------------------------------------------------------------------- attention
def run(kv16, kv4, lens, seq_ids, prefix_ids, hq, hkv, d, dtype, seed=0, scale=0.0, strided=False, with_lse=True, q_scale=1.0, v_mean=0.0,
        layers=1, check=True, poisoned=True):
    table, pages = make_tables(lens, seed)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor([int(n) for n in lens], dtype=torch.int32, device="cuda"))
    b = len(seq_ids) if seq_ids is not None else len(prefix_ids) if prefix_ids is not None else len(lens)
    ids = None if seq_ids is None else torch.tensor(seq_ids, dtype=torch.int32, device="cuda")
    pre = None if prefix_ids is None else torch.tensor(prefix_ids, dtype=torch.int32, device="cuda")
    err, work, results = err_word(), None, []
    for layer in range(layers):
        k, v = make_pool(pages, hkv, d, dtype, seed + 10 * layer + 1, table, lens, poisoned, v_mean)
        pool = kv16.Pool(k.cuda(), v.cuda())
        q = rows(b, hq, d, dtype, seed + layer, q_scale)
        if work is None:
            work = kv16.kv16_workspace(pool, hq, b)
            kv16.kv16_plan(pool, tabs, hq, b, work, seq_ids=ids, prefix_ids=pre, device_error=err)
        if strided:
            wide_q = torch.full((b, hq + 2 * hkv, d), float("nan"), dtype=dtype, device="cuda")
            wide_o = torch.full((b, hq + 1, d), -3.0, dtype=dtype, device="cuda")
            wide_q[:, :hq] = q.cuda()
            dq, out = wide_q[:, :hq], wide_o[:, :hq]
        else:
            dq, out = q.cuda(), torch.full((b, hq, d), float("nan"), dtype=dtype, device="cuda")
        lse = torch.full((b, hq), float("nan"), device="cuda") if with_lse else None
        first = None
        for _ in range(2):
            kv16.kv16_attention(pool, tabs, dq, out, work, lse=lse, softmax_scale=scale, device_error=err)
            first = out.clone() if first is None else first
        assert int(err) == 0, int(err)
        assert torch.equal(first.view(torch.int16), out.view(torch.int16)), "two calls differ"
        if strided:
            assert (wide_o[:, hq:] == -3.0).all()
        ref = attention(k, v, table, lens, seq_ids, prefix_ids, q, scale if scale > 0 else d ** -0.5, dtype)
        if check:
            assert_attention(out, lse, ref, dtype, (hq, hkv, d, layer))
        results.append((out, lse, ref))
    return results


HEADS = [(3, 3), (28, 4), (8, 1), (10, 5)]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
def test_own_tokens_only(kv16, kv4, hq, hkv, d, dtype):
    run(kv16, kv4, [0, 1, 2, 15, 16, 17, 31, 32, 33, 130, 255, 0, 700], None, None, hq, hkv, d, dtype, seed=hq + d)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("plen", [1, 16, 100, 128, 129, 1000])
def test_one_prefix_for_all(kv16, kv4, hq, hkv, d, dtype, plen):
    own = [0, 1, 17, 64, 5, 0, 300, 33, 16, 2, 90]
    run(kv16, kv4, own + [plen], list(range(11)), [11] * 11, hq, hkv, d, dtype, seed=plen)

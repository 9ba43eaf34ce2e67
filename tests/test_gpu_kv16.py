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


@pytest.mark.parametrize("of_q", [True, False])
def test_huge_rows_beside_normed_ones(kv16, of_q):
    """Only queries, or only keys, are normed; the others' squares pass the range of 32 bits and they are only turned."""
    n, d, freq = 9, 128, inv_freq(64)
    q, k = rows(n, 5, d, BF, 1), rows(n, 6, d, BF, 2)
    big = k if of_q else q
    big[::2] = (big[::2].float() * 2.0 ** 90).to(BF)
    w = rows(1, 1, d, BF, 3).reshape(d)
    out = torch.empty_like(q).cuda(), torch.empty_like(k).cuda()
    kv16.kv_qk_rope(kv16.Rope(freq), torch.arange(n, dtype=torch.int32, device="cuda"), q.cuda(), k.cuda(), *out,
                    **{"q_weight" if of_q else "k_weight": w.cuda()})
    for got, x, weight in zip(out, (q, k), (w, None) if of_q else (None, w)):
        assert_rows(got, turned(x, [list(range(n))], freq, None, weight=weight), BF, weight is None)


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
        ref = attention(pool.k, pool.v, table, lens, seq_ids, prefix_ids, dq, scale if scale > 0 else d ** -0.5, dtype)
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


# Several groups: prefixes of one row, of few rows (records), of many; one that comes again later; an empty one; rows
# without; own requests that repeat; a prefix that is a row's own request too.
def mixed(seed, plens=(300, 17, 0, 129, 1000, 64)):
    rng = np.random.default_rng(seed)
    rows = [(0, 9), (1, 1), (-1, 3), (2, 4), (3, 2), (0, 5), (4, 30), (5, 3), (-1, 1)]
    own, pre = [], []
    for g, n in rows:
        for _ in range(n):
            own.append(int(rng.choice([0, 1, 15, 16, 33, 100, 260])))
            pre.append(g)
    b = len(own)
    ids = list(range(b))
    ids[5] = ids[4]
    ids[20] = b + 1                                  # its own tokens are a prefix of others
    return own + list(plens), ids, [g if g < 0 else b + g for g in pre]


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(3, 3), (28, 4), (8, 1), (10, 5), (6, 2)])
def test_groups_of_every_size(kv16, kv4, hq, hkv, d, dtype):
    lens, ids, pre = mixed(hq)
    run(kv16, kv4, lens, ids, pre, hq, hkv, d, dtype, seed=hq + d, strided=True, layers=2, scale=0.07)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,batch", [(7, 1, 120), (2, 2, 700), (8, 1, 300), (5, 1, 52), (24, 3, 33), (1, 1, 257), (4, 1, 4096)])
def test_more_rows_than_a_tile_holds(kv16, kv4, hq, hkv, d, batch):
    """Chunks of rows, the last of them with fewer; one row more than two tiles hold."""
    own = [(7 * i) % 40 for i in range(batch)]
    run(kv16, kv4, own + [333], list(range(batch)), [batch] * batch, hq, hkv, d, BF, seed=batch, with_lse=False)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hq,hkv,d,plen,batch", [(28, 4, 128, 20011, 40), (14, 2, 64, 30000, 150), (8, 8, 128, 9999, 20), (16, 1, 64, 50001, 11)])
def test_long_prefixes(kv16, kv4, hq, hkv, d, plen, batch, dtype):
    own = [(13 * i) % 90 for i in range(batch)]
    if hq // hkv > 8:
        hkv = 2
    (out, lse, ref), = run(kv16, kv4, own + [plen], list(range(batch)), [batch] * batch, hq, hkv, d, dtype, seed=plen, poisoned=False)
    # The roundings of weights and of the output are spread evenly: together sqrt(2) of the output's own, which is UNIT / sqrt(3) at most.
    rel = float((out.double() - ref[0]).norm() / ref[0].norm())
    assert rel <= 1.25 * 2 ** 0.5 * UNIT[dtype] / 3 ** 0.5, rel


@pytest.mark.parametrize("d,hkv,batch,plen", [(128, 16, 20, 300), (64, 16, 24, 700), (128, 24, 40, 100), (128, 8, 150, 130), (64, 32, 17, 129)])
def test_many_jobs_of_few_workers(kv16, kv4, d, hkv, batch, plen):
    """Long own tokens take most of the GPU: each worker of the prefix goes through many short jobs, with one tile and more."""
    own = [1500 + 40 * i % 700 for i in range(batch)]
    run(kv16, kv4, own + [plen], list(range(batch)), [batch] * batch, hkv, hkv, d, BF, seed=plen, poisoned=False)


@pytest.mark.parametrize("d,hq,hkv,batch,plen,olen", [(128, 32, 32, 64, 701, 400), (64, 14, 2, 150, 4000, 100), (128, 28, 4, 70, 9000, 30)])
def test_every_call_gives_the_same(kv16, kv4, d, hq, hkv, batch, plen, olen):
    """Copies that end in another order, streams that run apart: 400 calls, bit for bit."""
    lens = [olen + i % 50 for i in range(batch)] + [plen]
    table, pages = make_tables(lens, 5)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    pool = kv16.Pool(*(torch.randn((pages, hkv, P, d), device="cuda", generator=torch.Generator("cuda").manual_seed(s)).to(BF) for s in (1, 2)))
    q = rows(batch, hq, d, BF, 3).cuda()
    work, err = kv16.kv16_workspace(pool, hq, batch), err_word()
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=torch.full((batch,), batch, dtype=torch.int32, device="cuda"), device_error=err)
    first = None
    for _ in range(400):
        out = torch.full((batch, hq, d), float("nan"), dtype=BF, device="cuda")
        kv16.kv16_attention(pool, tabs, q, out, work, device_error=err)
        first = out if first is None else first
        assert torch.equal(first.view(torch.int16), out.view(torch.int16))
    assert int(err) == 0


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("q_scale", [0.0, 6.0, 60.0])
@pytest.mark.parametrize("batch,d", [(30, 128), (63, 128), (99, 64)])     # 120, 252 and 396 query rows of a KV head
def test_flat_and_sharp_scores(kv16, kv4, dtype, q_scale, batch, d):
    """Weights that are all equal; references that move often; one token that takes all."""
    run(kv16, kv4, [0, 40, 7] * (batch // 3) + [1500], list(range(batch)), [batch] * batch, 8, 2, d, dtype, seed=4, q_scale=q_scale, v_mean=1.0)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,batch", [(64, 40), (128, 40), (128, 3), (64, 100), (128, 100), (128, 300)])
def test_scores_that_rise(kv16, kv4, dtype, d, batch):
    """Keys grow along the prefix, so every tile, and every half of one, moves the reference, by 2 to 40 in log2 units."""
    plen, hq, hkv = 900, 4, 2
    lens = [3] * batch + [plen]
    table, pages = make_tables(lens, 9)
    k, v = make_pool(pages, hkv, d, dtype, 1, table, lens)
    t = np.arange(plen)
    direction = torch.randn(d, generator=torch.Generator().manual_seed(0))
    at = table[batch][t // P].astype(np.int64)
    for step in (0.02, 0.3):
        k[at, :, t % P] = (direction * torch.tensor(t * step, dtype=torch.float32)[:, None])[:, None].to(dtype).expand(-1, hkv, -1)
        pool = kv16.Pool(k.cuda(), v.cuda())
        tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        q = (direction + 0.1 * torch.randn((batch, hq, d), generator=torch.Generator().manual_seed(1))).to(dtype).cuda()
        work, err, ids = kv16.kv16_workspace(pool, hq, batch), err_word(), torch.full((batch,), batch, dtype=torch.int32, device="cuda")
        out, lse = torch.empty_like(q), torch.empty((batch, hq), device="cuda")
        kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=ids, device_error=err)
        kv16.kv16_attention(pool, tabs, q, out, work, lse=lse, device_error=err)
        assert int(err) == 0
        ref = attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, dtype)
        assert_attention(out, lse, ref, dtype, step)


@pytest.mark.parametrize("d,batch", [(64, 20), (64, 110), (128, 75)])
def test_values_that_are_not_finite(kv16, kv4, d, batch):
    """A NaN or an infinity in a token's V reaches the rows that attend to it, in its element; a query that is none, its own head."""
    hq, hkv = 4, 2
    lens = [20] * batch + [200]
    table, pages = make_tables(lens, 2)
    k, v = make_pool(pages, hkv, d, BF, 1, table, lens)
    v[int(table[3][0]), 1, 5, 7] = float("nan")            # row 3's own token, KV head 1, element 7
    v[int(table[batch][2]), 0, 1, 9] = float("inf")        # the prefix, KV head 0, element 9
    q = rows(batch, hq, d, BF, 1)
    q[11, 2, 0] = float("nan")
    pool = kv16.Pool(k.cuda(), v.cuda())
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    work = kv16.kv16_workspace(pool, hq, batch)
    out = torch.empty((batch, hq, d), dtype=BF, device="cuda")
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=torch.full((batch,), batch, dtype=torch.int32, device="cuda"))
    kv16.kv16_attention(pool, tabs, q.cuda(), out, work)
    got = out.cpu()
    want = torch.ones((batch, hq, d), dtype=torch.bool)
    want[3, 2:, 7] = want[:, :2, 9] = want[11, 2] = False
    assert torch.equal(torch.isfinite(got), want)
    assert torch.isinf(got[0, 0, 9]) and torch.isnan(got[3, 2, 7]) and torch.isnan(got[11, 2]).all()


@pytest.mark.parametrize("d,batch", [(128, 30), (128, 70), (64, 140)])
def test_page_ids_outside_the_pool_are_left_out(kv16, kv4, d, batch):
    hq, hkv = 8, 4
    lens = [50 + i for i in range(batch)] + [700]
    table, pages = make_tables(lens, 3)
    table[batch][3], table[batch][20], table[batch][43], table[4][1] = -5, pages, 2 ** 31 - 1, pages + 7
    k, v = make_pool(pages, hkv, d, BF, 1)
    pool = kv16.Pool(k.cuda(), v.cuda())
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = rows(batch, hq, d, BF, 1).cuda()
    work, err = kv16.kv16_workspace(pool, hq, batch), err_word()
    out, lse = torch.empty_like(q), torch.empty((batch, hq), device="cuda")
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=torch.full((batch,), batch, dtype=torch.int32, device="cuda"), device_error=err)
    assert int(err) == 0
    kv16.kv16_attention(pool, tabs, q, out, work, lse=lse, device_error=err)
    assert int(err) == 1
    assert_attention(out, lse, attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, BF), BF)


@pytest.mark.parametrize("d,batch", [(64, 26), (128, 90)])
def test_rows_that_are_refused(kv16, kv4, d, batch):
    """An unknown request, a length past the table: zeros, the bit, and all other rows as ever."""
    hq, hkv = 6, 3
    lens = [30 + i for i in range(batch)] + [260, 999999, -4]
    good = [n if 0 <= n <= 400 else 0 for n in lens]
    table, pages = make_tables(good, 3)
    k, v = make_pool(pages, hkv, d, FP, 1, table, good)
    pool = kv16.Pool(k.cuda(), v.cuda())
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    ids, pre = list(range(batch)), [batch] * batch
    ids[2], ids[9], pre[12], pre[13], pre[17], ids[20] = -1, len(lens), len(lens) + 5, batch + 1, -2, batch + 2
    bad = [2, 9, 12, 13, 17, 20]
    q = rows(batch, hq, d, FP, 1).cuda()
    work, err = kv16.kv16_workspace(pool, hq, batch), err_word()
    out, lse = torch.full_like(q, 5.0), torch.full((batch, hq), 5.0, device="cuda")
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    kv16.kv16_plan(pool, tabs, hq, batch, work, seq_ids=dev(ids), prefix_ids=dev(pre), device_error=err)
    assert int(err) == 4
    kv16.kv16_attention(pool, tabs, q, out, work, lse=lse)
    assert (out[bad] == 0).all() and (lse[bad] == -math.inf).all()
    fine = [i for i in range(batch) if i not in bad]
    ref = attention(pool.k, pool.v, table, good, [ids[i] for i in fine], [pre[i] for i in fine], q[fine], d ** -0.5, FP)
    assert_attention(out[fine], lse[fine], ref, FP)


def test_a_workspace_without_this_plan(kv16, kv4):
    d, hq, hkv, batch = 64, 4, 2, 5
    lens = [20] * batch + [100]
    table, pages = make_tables(lens, 3)
    pool = kv16.Pool.empty(pages, hkv, d)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    work = kv16.kv16_workspace(pool, 8, batch)
    work.zero_()
    q = rows(batch, hq, d, BF, 1).cuda()

    def attend(q, tabs=tabs, pool=pool):
        out, err = torch.full_like(q, 5.0), err_word()
        kv16.kv16_attention(pool, tabs, q, out, work, device_error=err)
        return int(err), bool((out == 5.0).all())

    assert attend(q) == (16, True)                                   # no plan at all
    kv16.kv16_plan(pool, tabs, hq, batch, work)
    assert attend(q)[0] == 0
    assert attend(q[:4]) == (16, True)                               # of another batch
    assert attend(rows(batch, 2, d, BF, 1).cuda()) == (16, True)     # other heads
    wide = torch.cat([torch.from_numpy(table).cuda()] * 2, 1).contiguous()
    assert attend(q, kv4.Tables(wide, tabs.lens)) == (16, True)      # other tables
    kv16.kv16_plan(pool, tabs, 8, batch, work)
    assert attend(q) == (16, True)


def test_calls_that_the_binding_refuses(kv16, kv4):
    d, hkv = 64, 2
    pool = kv16.Pool.empty(4, hkv, d)
    tabs = kv4.Tables.empty(4, 2, 2)
    x = torch.zeros((3, 4, d), dtype=BF, device="cuda")
    k = torch.zeros((3, hkv, d), dtype=BF, device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, device="cuda")
    rope = kv16.Rope([1.0] * 32, num_axes=3)
    pos = torch.zeros((3, 3), dtype=torch.int32, device="cuda")
    bad = [lambda: kv16.kv_qk_rope(rope, pos.long(), x, k, x, k), lambda: kv16.kv_qk_rope(rope, pos[:2], x, k, x, k),
           lambda: kv16.kv_qk_rope(rope, None, x, k, x, k), lambda: kv16.kv_qk_rope(rope, pos.t()[:, :2], x, k, x, k),
           lambda: kv16.kv_qk_rope(rope, pos, x, k[:2], x, k), lambda: kv16.kv_qk_rope(rope, pos, x, k.half(), x, k),
           lambda: kv16.kv_qk_rope(rope, pos, x, k, x, None), lambda: kv16.kv_qk_rope(rope, pos, x, k, x[:, :3], k),
           lambda: kv16.kv_qk_rope(rope, pos, x, k, x, k, q_weight=torch.zeros(d, device="cuda")),
           lambda: kv16.kv_qk_rope(rope, pos, x, k, x, k, q_weight=torch.zeros(d - 1, dtype=BF, device="cuda")),
           lambda: kv16.kv_qk_rope(rope, pos, x.transpose(1, 2), k, x, k), lambda: kv16.kv_qk_rope(rope, pos, x.cpu(), k, x, k),
           lambda: kv16.kv16_write(pool, slots.int(), k, k), lambda: kv16.kv16_write(pool, slots, x, k),
           lambda: kv16.kv16_write(pool, slots[:2], k, k), lambda: kv16.kv16_write(pool, slots, k, k, q=x),
           lambda: kv16.kv16_plan(pool, tabs, 4, 2, torch.zeros(16, device="cuda")),
           lambda: kv16.kv16_plan(pool, tabs, 4, 2, kv16.kv16_workspace(pool, 4, 2), seq_ids=slots[:2].int()[:1]),
           lambda: kv16.kv16_attention(pool, tabs, x[:2], x[:1], kv16.kv16_workspace(pool, 4, 2)),
           lambda: kv16.Pool(pool.k, pool.v[:2]), lambda: kv16.Pool(pool.k, pool.v.half()), lambda: kv16.Pool(pool.k[:, :, :8], pool.v[:, :, :8])]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    small = kv16.kv16_workspace(pool, 4, 1)[:-256]
    with pytest.raises(kv16.kd.KVDecodeError, match="workspace"):
        kv16.kv16_plan(pool, tabs, 4, 1, small)
    kv16.kv_qk_rope(rope, torch.zeros(3, dtype=torch.int32, device="cuda"), x, k, x, k)    # one row of positions for all axes


# ------------------------------------------------------ graphs, streams, devices
def test_a_captured_step_follows_the_lengths(kv16, kv4):
    """Tables, rotation and write, plan and two layers of attention captured once and replayed while the requests grow."""
    d, hq, hkv, batch, plen = 128, 8, 2, 12, 333
    lens = [17 * i % 60 for i in range(batch)] + [plen]
    pages = sum(pages_of(n + 40) for n in lens)
    tabs = kv4.Tables.empty(pages, batch + 1, max(pages_of(n + 40) for n in lens))
    slots = torch.empty(sum(lens), dtype=torch.int64, device="cuda")
    kv4.kv_tables_step(tabs, None, torch.tensor(lens, dtype=torch.int32, device="cuda"), slots)
    pools = [kv16.Pool(*(torch.randn((pages, hkv, P, d), device="cuda").to(BF) for _ in range(2))) for _ in range(2)]
    rope = kv16.Rope(inv_freq(d // 2))
    side = torch.cuda.Stream()
    ids = torch.arange(batch, dtype=torch.int32, device="cuda")
    pre = torch.full((batch,), batch, dtype=torch.int32, device="cuda")
    ones = torch.ones(batch, dtype=torch.int32, device="cuda")
    new, pos = torch.empty(batch, dtype=torch.int64, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda")
    x = [torch.empty((batch, hq + 2 * hkv, d), dtype=BF, device="cuda") for _ in pools]
    qr, out = ([torch.empty((batch, hq, d), dtype=BF, device="cuda") for _ in pools] for _ in range(2))
    lse = [torch.empty((batch, hq), device="cuda") for _ in pools]
    work, err = kv16.kv16_workspace(pools[0], hq, batch), err_word()

    def step(s):
        kv4.kv_tables_step(tabs, ids, ones, new, pos, device_error=err, stream=s)
        kv16.kv16_plan(pools[0], tabs, hq, batch, work, seq_ids=ids, prefix_ids=pre, device_error=err, stream=s)
        for i, pool in enumerate(pools):
            q, k, v = x[i][:, :hq], x[i][:, hq:hq + hkv], x[i][:, hq + hkv:]
            kv16.kv16_write(pool, new, k, v, rope=rope, positions=pos, q=q, q_out=qr[i], device_error=err, stream=s)
            kv16.kv16_attention(pool, tabs, qr[i], out[i], work, lse=lse[i], device_error=err, stream=s)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        step(side)
    for it in range(6):
        with torch.cuda.stream(side):
            for i in range(2):
                x[i].copy_(rows(batch, hq + 2 * hkv, d, BF, 100 * it + i))
            g.replay()
        side.synchronize()
        lens = [n + 1 for n in lens[:-1]] + [plen]
        assert int(err) == 0 and tabs.lens.tolist() == lens
        table = tabs.block_table.cpu().numpy()
        for i, pool in enumerate(pools):
            assert_rows(qr[i], turned(x[i][:, :hq].cpu(), [[n - 1 for n in lens[:-1]]], inv_freq(d // 2), None), BF)
            ref = attention(pool.k, pool.v, table, lens, None, [batch] * batch, qr[i], d ** -0.5, BF)
            assert_attention(out[i], lse[i], ref, BF, (it, i))


def test_a_step_on_a_stream_of_its_own(kv16, kv4):
    """Beside slow work on the default stream, with a raw handle for the stream."""
    lens, ids, pre = mixed(1)
    b = len(ids)
    table, pages = make_tables(lens, 1)
    k, v = make_pool(pages, 4, 128, BF, 2, table, lens)
    q = rows(b, 8, 128, BF, 1)
    side = torch.cuda.Stream()
    dev = lambda t: torch.tensor(t, dtype=torch.int32, device="cuda")  # noqa: E731
    with torch.cuda.stream(side):
        pool, dq = kv16.Pool(k.cuda(), v.cuda()), q.cuda()
        tabs, work = kv4.Tables(torch.from_numpy(table).cuda(), dev(lens)), kv16.kv16_workspace(pool, 8, b)
        dids, dpre, out = dev(ids), dev(pre), torch.empty_like(dq)
    side.synchronize()
    torch.cuda._sleep(40_000_000)
    kv16.kv16_plan(pool, tabs, 8, b, work, seq_ids=dids, prefix_ids=dpre, stream=side.cuda_stream)
    kv16.kv16_attention(pool, tabs, dq, out, work, stream=side.cuda_stream)
    side.synchronize()
    assert_attention(out, None, attention(pool.k, pool.v, table, lens, ids, pre, dq, 128 ** -0.5, BF), BF)


def test_two_graphs_share_a_workspace(kv16, kv4):
    """Each holds its own plan call: replayed by turns they give what they gave alone."""
    graphs = []
    work = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for hq, hkv, d, batch, plen in ((8, 2, 128, 30, 700), (6, 6, 64, 9, 2000)):
        lens = [5 * i % 70 for i in range(batch)] + [plen]
        table, pages = make_tables(lens, batch)
        pool = kv16.Pool(*(x.cuda() for x in make_pool(pages, hkv, d, BF, 1, table, lens)))
        tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        q, pre = rows(batch, hq, d, BF, 1).cuda(), torch.full((batch,), batch, dtype=torch.int32, device="cuda")
        out = torch.empty_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=pre, stream=side)
            kv16.kv16_attention(pool, tabs, q, out, work, stream=side)
        ref = attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, BF)
        graphs.append((g, out, ref, (pool, tabs, q, pre)))
    for i in (0, 1, 1, 0, 0, 1):
        g, out, ref, _ = graphs[i]
        with torch.cuda.stream(side):
            out.fill_(float("nan"))
            g.replay()
        side.synchronize()
        assert_attention(out, None, ref, BF, i)


def test_two_streams_at_once(kv16, kv4):
    """Plans and attention of two batches on two streams, each with a workspace of its own, without order between them."""
    jobs = []
    for seed, (hq, hkv, d, batch, plen) in enumerate(((8, 2, 128, 50, 3000), (14, 2, 64, 60, 2000))):
        lens = [9 * i % 80 for i in range(batch)] + [plen]
        table, pages = make_tables(lens, seed)
        pool = kv16.Pool(*(x.cuda() for x in make_pool(pages, hkv, d, BF, seed, table, lens)))
        tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
        q, pre = rows(batch, hq, d, BF, seed).cuda(), torch.full((batch,), batch, dtype=torch.int32, device="cuda")
        ref = attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, BF)
        jobs.append((torch.cuda.Stream(), pool, tabs, q, pre, kv16.kv16_workspace(pool, hq, batch), [torch.empty_like(q) for _ in range(40)], ref))
    torch.cuda.synchronize()
    for i in range(40):
        for stream, pool, tabs, q, pre, work, outs, _ in jobs:
            kv16.kv16_plan(pool, tabs, q.shape[1], len(q), work, prefix_ids=pre, stream=stream)
            kv16.kv16_attention(pool, tabs, q, outs[i], work, stream=stream)
    torch.cuda.synchronize()
    for *_, outs, ref in jobs:
        assert_attention(outs[0], None, ref, BF)
        assert all(torch.equal(outs[0].view(torch.int16), o.view(torch.int16)) for o in outs[1:])


def test_offsets_past_32_bits(kv16, kv4):
    """A pool of more than 2^31 elements a side, and rows of queries that far apart."""
    d, hkv, hq, batch, plen, pages = 128, 1, 8, 33, 400, 1_200_000
    pool = kv16.Pool.empty(pages, hkv, d)
    assert pool.k.numel() > 2 ** 31
    lens = [1 + 5 * i % 50 for i in range(batch)] + [plen]
    table, used = make_tables(lens, 3)
    table[table >= 0] += pages - used                     # the pool's last pages
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    slots = torch.tensor([int(table[r][t // P]) * P + t % P for r, n in enumerate(lens) for t in range(n)], device="cuda")
    assert int(slots.max()) * d > 2 ** 31
    k, v = (rows(len(slots), hkv, d, BF, seed).cuda() for seed in (1, 2))
    far = torch.zeros(batch << 26, dtype=BF, device="cuda")
    q, out = (torch.as_strided(far, (batch, hq, d), (1 << 26, d, 1), at) for at in (0, hq * d))
    assert (batch - 1) << 26 > 2 ** 30 and far.numel() > 2 ** 31
    err = err_word()
    kv16.kv16_write(pool, slots, k, v, device_error=err)
    kv16.kv_qk_rope(kv16.Rope(inv_freq(d // 2)), torch.arange(batch, dtype=torch.int32, device="cuda"), rows(batch, hq, d, BF, 5).cuda(), None, q, None)
    assert_rows(q, turned(rows(batch, hq, d, BF, 5), [list(range(batch))], inv_freq(d // 2), None), BF)
    work = kv16.kv16_workspace(pool, hq, batch)
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=torch.full((batch,), batch, dtype=torch.int32, device="cuda"), device_error=err)
    kv16.kv16_attention(pool, tabs, q, out, work, device_error=err)
    assert int(err) == 0
    at = slots[:3]
    assert torch.equal(pool.k[at // P, 0, at % P], k[:3, 0]) and torch.equal(pool.v[at // P, 0, at % P], v[:3, 0])
    assert_attention(out, None, attention(pool.k, pool.v, table, lens, None, [batch] * batch, q, d ** -0.5, BF), BF)


def test_one_row_of_queries_for_all(kv16, kv4):
    """Stride 0: every row asks the same of its own tokens."""
    lens = [40, 1, 0, 33, 200]
    table, pages = make_tables(lens, 1)
    pool = kv16.Pool(*(x.cuda() for x in make_pool(pages, 2, 64, BF, 1, table, lens)))
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    q = rows(1, 4, 64, BF, 1).cuda().expand(5, 4, 64)
    out, work = torch.empty((5, 4, 64), dtype=BF, device="cuda"), kv16.kv16_workspace(pool, 4, 5)
    kv16.kv16_plan(pool, tabs, 4, 5, work)
    kv16.kv16_attention(pool, tabs, q, out, work)
    assert_attention(out, None, attention(pool.k, pool.v, table, lens, None, None, q, 64 ** -0.5, BF), BF)


@pytest.mark.parametrize("batch", [4, 40])
def test_the_first_call_is_captured(kvlib, batch):
    """In a process whose first use of these kernels is under capture."""
    import subprocess
    import sys
    code = f"""
import torch
from paper_2603_12707_gb300 import kv4, kv16
hq, hkv, d, batch = 28, 4, 128, {batch}
pool = kv16.Pool(*(torch.randn((batch + 9, hkv, 16, d), device="cuda").bfloat16() for _ in range(2)))
tabs = kv4.Tables(torch.arange(batch + 1, dtype=torch.int32, device="cuda")[:, None] * torch.ones(8, dtype=torch.int32, device="cuda"),
                  torch.tensor([16] * batch + [16], dtype=torch.int32, device="cuda"))
pre = torch.full((batch,), batch, dtype=torch.int32, device="cuda")
q = torch.randn((batch, hq, d), device="cuda").bfloat16()
out, again, work = torch.empty_like(q), torch.empty_like(q), kv16.kv16_workspace(pool, hq, batch)
rope, pos = kv16.Rope([1.0] * 64), torch.zeros(batch, dtype=torch.int32, device="cuda")
slots = torch.full((batch,), -1, dtype=torch.int64, device="cuda")
new = torch.zeros((batch, hkv, d), dtype=torch.bfloat16, device="cuda")
torch.cuda.synchronize()
s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
with torch.cuda.stream(s), torch.cuda.graph(g, stream=s):
    kv16.kv16_plan(pool, tabs, hq, batch, work, prefix_ids=pre, stream=s)
    kv16.kv16_write(pool, slots, new, new, rope=rope, positions=pos, q=q, q_out=q, stream=s)
    kv16.kv16_attention(pool, tabs, q, out, work, stream=s)
with torch.cuda.stream(s):
    g.replay()
s.synchronize()
kv16.kv16_attention(pool, tabs, q, again, work)
assert torch.isfinite(out).all() and torch.equal(out, again)
print("fine")
"""
    got = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert got.returncode == 0 and "fine" in got.stdout, got.stdout + got.stderr

"""The 4-bit cache on the GPU against the plain reference of _kv4_common:
pools byte for byte, gathered values to one rounding, attention in 64 bits to
the bound of its arithmetic, block tables and slot maps entry for entry."""
import numpy as np
import pytest
import torch

from _kv4_common import (P, TINY, UNIT, TablesModel, assert_attention, attention, block_bytes, poison, put, quantise,
                         random_pool, unpack, values)

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def err_word():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def make_tables(lens, seed, extra_pages=3, width=None, seqs=None):
    """Shuffled tables: (numpy table, number of pages in the pool)."""
    rng = np.random.default_rng(seed)
    n = [(int(x) + P - 1) // P for x in lens]
    pages = sum(n) + extra_pages
    order = rng.permutation(pages)
    table = np.full((len(lens), width or max(1, max(n))), -7, np.int32)
    at = 0
    for i, k in enumerate(n):
        table[i, :k] = order[at:at + k]
        at += k
    return table, pages


# --------------------------------------------------------------- attention
def run_attention(kv4, lens, hq, hkv, d, group, dtype, seed=0, scale=0.0, q_scale=1.0, kv_scale=1.0, strided=False,
                  with_lse=True, blocks=None, poisoned=True):
    table, pages = make_tables(lens, seed)
    if blocks is None:
        blocks = random_pool(pages, hkv, d, group, dtype, seed + 1, kv_scale)
    if poisoned:
        poison(blocks, table, lens, d, group)
    g = torch.Generator().manual_seed(seed)
    b = len(lens)
    q = (torch.randn((b, hq, d), generator=g) * q_scale).to(dtype)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, dtype)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    if strided:   # q and out are slices of wider rows
        wide_q = torch.full((b, hq + 2 * hkv, d), float("nan"), dtype=dtype, device="cuda")
        wide_o = torch.full((b, hq + 1, d), -3.0, dtype=dtype, device="cuda")
        wide_q[:, :hq] = q.cuda()
        dq, out = wide_q[:, :hq], wide_o[:, :hq]
    else:
        dq, out = q.cuda(), torch.full((b, hq, d), float("nan"), dtype=dtype, device="cuda")
    lse = torch.full((b, hq), float("nan"), device="cuda") if with_lse else None
    work, err = kv4.kv4_workspace(pool, hq), err_word()
    first = None
    for _ in range(2):   # the second call finds the workspace as the first left it
        kv4.kv4_decode_attention(pool, tabs, dq, out, work, lse=lse, softmax_scale=scale, device_error=err)
        if first is None:
            first = out.clone()
    assert torch.equal(first.view(torch.int16), out.view(torch.int16)), "two calls differ"
    assert int(err) == 0
    if strided:
        assert (wide_o[:, hq:] == -3.0).all()
    ref = attention(blocks, table, lens, q.double().numpy(), group, dtype, scale if scale > 0 else d ** -0.5)
    assert_attention(out, lse, ref, dtype, (lens, hq, hkv, d, group))


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("hq,hkv", [(3, 3), (28, 4), (8, 1), (10, 5)])
def test_attention_of_ragged_rows(kv4, hq, hkv, d, group, dtype):
    run_attention(kv4, [0, 1, 2, 15, 16, 17, 31, 32, 33, 130, 255, 0, 700], hq, hkv, d, group, dtype, seed=hq + d + group)


@pytest.mark.parametrize("lens", [[1], [0], [0, 0, 0], [16], [4097], [20000], [1] * 300, [0, 9000, 1, 0, 3], [48] * 77])
@pytest.mark.parametrize("hq,hkv,d,group,dtype", [(7, 1, 128, 128, BF), (4, 4, 64, 32, FP)])
def test_attention_of_few_many_and_long_rows(kv4, lens, hq, hkv, d, group, dtype):
    run_attention(kv4, lens, hq, hkv, d, group, dtype, seed=5, poisoned=sum(lens) < 6000)


def test_attention_of_more_rows_than_any_grid(kv4):
    rng = np.random.default_rng(3)
    run_attention(kv4, [int(x) for x in rng.integers(0, 40, 4096)], 2, 1, 64, 64, BF, seed=3, poisoned=False)


@pytest.mark.parametrize("group", [32, 128])
def test_attention_of_slices_of_wider_rows_without_lse(kv4, group):
    run_attention(kv4, [5, 100, 64, 33], 28, 4, 128, group, BF, strided=True, with_lse=False)
    run_attention(kv4, [1000], 6, 6, 128, group, FP, strided=True, scale=0.3)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("q_scale,kv_scale", [(30.0, 1.0), (1e-3, 1.0), (1.0, 1e-3), (1.0, 50.0), (2000.0, 1e-3)])
def test_attention_of_small_and_large_values(kv4, dtype, q_scale, kv_scale):
    """Peaked and flat softmaxes, scales far from one."""
    run_attention(kv4, [3, 70, 515], 14, 2, 128, 64, dtype, seed=9, q_scale=q_scale, kv_scale=kv_scale)
    run_attention(kv4, [3, 70, 515], 4, 4, 64, 32, dtype, seed=9, q_scale=q_scale, kv_scale=kv_scale)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
def test_scores_of_single_tokens(kv4, d, group, dtype):
    """A row of one token: its log-sum-exp is the score itself, with nothing to average.

    A score is d / 16 accumulations and a few operations on the groups' sums, of a size of
    at most a = scale * sum_d |q_d| (8 s + |z|); each rounds to 2^-24 or cuts off at 2^-23 of
    that.  Half of d / 16 + 4 steps at 2^-23 leave 2^-20 a at d = 128, and less at 64; errors of
    different signs take it to half of that."""
    b, hq, hkv = 64, 8, 2
    table, pages = make_tables([1] * b, 11)
    blocks = random_pool(pages, hkv, d, group, dtype, 12)
    q = torch.randn((b, hq, d), generator=torch.Generator().manual_seed(13)).to(dtype)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, dtype)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.ones(b, dtype=torch.int32, device="cuda"))
    out, lse = torch.empty((b, hq, d), dtype=dtype, device="cuda"), torch.empty((b, hq), device="cuda")
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, hq), lse=lse)
    k, _, (s, z), _ = values(blocks[table[:, 0]], d, group, dtype)                  # [b, hkv, 16, d]
    k, size = (np.repeat(x[:, :, 0], hq // hkv, 1) for x in (k, 8 * s + np.abs(z)))
    x = (q.double().numpy() * k).sum(-1) * d ** -0.5
    a = (np.abs(q.double().numpy()) * size).sum(-1) * d ** -0.5
    err = np.abs(lse.double().cpu().numpy() - x)
    assert (err <= 2.0 ** -21 * a).all(), float((err / a).max() * 2 ** 21)


def test_attention_of_bf16_values_that_fp16_cannot_hold(kv4):
    run_attention(kv4, [40, 300], 8, 2, 128, 32, BF, seed=2, q_scale=1e-30, kv_scale=1e25)
    run_attention(kv4, [40, 300], 8, 2, 128, 32, BF, seed=2, q_scale=1e20, kv_scale=1e-22)


def test_scales_that_grow_along_a_row(kv4):
    """V's scales span 2^-30 .. 2^30 over one row, in rising, falling and mixed order."""
    d, group, hkv, n = 64, 32, 2, 900
    for order in ("rise", "fall", "mix"):
        table, pages = make_tables([n], 1)
        blocks = random_pool(pages, hkv, d, group, BF, 4)
        rng = np.random.default_rng(0)
        for t in range(n):
            e = {"rise": -30 + 60 * t // n, "fall": 30 - 60 * t // n, "mix": int(rng.integers(-30, 31))}[order]
            p, off = table[0, t // P], 16 * d + 64 * 2 + (t % P) * 8
            meta = torch.from_numpy(rng.uniform(0.5, 1.0, (hkv, 2, 2)) * 2.0 ** e).to(BF)
            blocks[p][:, off:off + 8] = meta.view(torch.uint8).numpy().reshape(hkv, 8)
        run_attention(kv4, [n], 4, 2, d, group, BF, seed=1, blocks=blocks)


def test_a_row_of_equal_keys_is_the_mean_of_its_values(kv4):
    d, group, n = 128, 128, 1000
    table, pages = make_tables([n], 6)
    blocks = random_pool(pages, 1, d, group, BF, 6)
    zero = torch.tensor([0.0, 0.25], dtype=BF).view(torch.uint8).numpy()     # every key is 0.25 everywhere
    blocks[..., 16 * d:16 * d + 64] = np.tile(zero, 16)
    run_attention(kv4, [n], 8, 1, d, group, BF, seed=6, blocks=blocks)


def test_rows_choose_their_requests(kv4):
    """seq_ids in any order, one twice; ids out of range and broken lengths give empty rows and an error bit."""
    d, group, hq, hkv = 128, 64, 8, 2
    lens = [17, 0, 250, 48]
    table, pages = make_tables(lens, 8, width=20)
    blocks = random_pool(pages, hkv, d, group, BF, 8)
    ids = [2, 0, 3, 2, 1]
    q = torch.randn((5, hq, d), generator=torch.Generator().manual_seed(1)).to(BF)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, BF)
    dl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), dl)
    out, lse = torch.empty((5, hq, d), dtype=BF, device="cuda"), torch.empty((5, hq), device="cuda")
    work, err = kv4.kv4_workspace(pool, hq), err_word()

    def call(i):
        kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, work, seq_ids=torch.tensor(i, dtype=torch.int32, device="cuda"),
                                 lse=lse, device_error=err)

    call(ids)
    ref = attention(blocks, table[ids], [lens[i] for i in ids], q.double().numpy(), group, BF, d ** -0.5)
    assert_attention(out, lse, ref, BF)
    assert int(err) == 0
    call([2, -1, 4, 3, 1])
    ref = attention(blocks, table[[2, 0, 0, 3, 1]], [250, 0, 0, 48, 0], q.double().numpy(), group, BF, d ** -0.5)
    assert_attention(out, lse, ref, BF)
    assert int(err) == 4
    err.zero_()
    dl[0], dl[3] = 20 * 16 + 1, -5
    call(ids)
    ref = attention(blocks, table[ids], [250, 0, 0, 250, 0], q.double().numpy(), group, BF, d ** -0.5)
    assert_attention(out, lse, ref, BF)
    assert int(err) == 4


def test_pages_outside_the_pool_are_left_out(kv4):
    d, group = 64, 64
    lens = [40, 64]
    table, pages = make_tables(lens, 4)
    blocks = random_pool(pages, 1, d, group, FP, 4)
    q = torch.randn((2, 2, d), generator=torch.Generator().manual_seed(1)).to(FP)
    bad = table.copy()
    bad[0, 1], bad[1, 0] = pages, -2
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, FP)
    tabs = kv4.Tables(torch.from_numpy(bad).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    out, lse, err = torch.empty((2, 2, d), dtype=FP, device="cuda"), torch.empty((2, 2), device="cuda"), err_word()
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, 2), lse=lse, device_error=err)
    assert int(err) == 1
    # the same tokens without the lost pages: row 0 keeps tokens 0..15 and 32..39, row 1 tokens 16..63
    kept = np.array([[table[0, 0], table[0, 2], -7, -7], [table[1, 1], table[1, 2], table[1, 3], -7]])
    ref = attention(blocks, kept, [24, 48], q.double().numpy(), group, FP, d ** -0.5)
    assert_attention(out, lse, ref, FP)


def test_nan_reaches_only_its_own_outputs(kv4):
    """A NaN value group of one token: its outputs are NaN, other groups' and other heads' are not; a NaN key: its whole head."""
    d, group, n = 128, 32, 50
    table, pages = make_tables([n], 4)
    blocks = random_pool(pages, 3, d, group, BF, 4)
    nan = np.frombuffer(np.array([0x7FC0, 0x7FC0], np.uint16).tobytes(), np.uint8)
    tok = 37
    p = table[0, tok // P]
    off_k, off_v = 16 * d + (tok % P) * 16, 16 * d + 256 + (tok % P) * 16
    blocks[p, 0, off_v + 8:off_v + 12] = nan       # head 0: value group 2
    blocks[p, 1, off_k + 4:off_k + 8] = nan        # head 1: key group 1
    q = torch.randn((1, 6, d), generator=torch.Generator().manual_seed(1)).to(BF)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, BF)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    out = torch.empty((1, 6, d), dtype=BF, device="cuda")
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, 6))
    bad = torch.isnan(out[0]).cpu().numpy()
    assert bad[:2, 64:96].all() and not bad[:2, :64].any() and not bad[:2, 96:].any()
    assert bad[2:4].all() and not bad[4:].any()


def test_a_query_that_is_not_finite_gives_nan_in_its_own_row(kv4):
    d, n = 128, 77
    table, pages = make_tables([n], 4)
    blocks = random_pool(pages, 1, d, 128, BF, 4)
    q = torch.randn((1, 5, d), generator=torch.Generator().manual_seed(1)).to(BF)
    q[0, 1, 3], q[0, 3, 100], q[0, 4, 0] = float("inf"), float("nan"), float("-inf")
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, 128, BF)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    out = torch.empty((1, 5, d), dtype=BF, device="cuda")
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, 5))
    bad = torch.isnan(out[0]).all(-1).cpu().tolist()
    assert bad == [False, True, False, True, True]
    assert torch.isfinite(out[0, [0, 2]]).all()


def test_long_pools_pass_32_bit_offsets(kv4):
    """A pool of more than 2^32 bytes: rows on its last pages, written, read and attended."""
    d, group, hkv = 128, 128, 8
    bb = block_bytes(d, group)
    pages = 2 ** 32 // (bb * hkv) + 300
    data = torch.empty((pages, hkv, bb), dtype=torch.uint8, device="cuda")
    data[-8:] = 255
    pool = kv4.Pool(data, d, group, BF)
    n = 100
    table = np.arange(pages - 7, pages, dtype=np.int32)[::-1].copy()[None]
    g = torch.Generator().manual_seed(0)
    k, v = (torch.randn((n, hkv, d), generator=g).to(BF) for _ in range(2))
    slots = torch.from_numpy(table[0].astype(np.int64)[np.arange(n) // P] * P + np.arange(n) % P).cuda()
    kv4.kv4_write(pool, slots, k.cuda(), v.cuda())
    tail = data[-8:].cpu().numpy()
    local = table - (pages - 8)
    q = torch.randn((1, hkv, d), generator=g).to(BF)
    out = torch.empty((1, hkv, d), dtype=BF, device="cuda")
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor([n], dtype=torch.int32, device="cuda"))
    kv4.kv4_decode_attention(pool, tabs, q.cuda(), out, kv4.kv4_workspace(pool, hkv))
    assert_attention(out, None, attention(tail, local, [n], q.double().numpy(), group, BF, d ** -0.5), BF)
    back = [torch.empty((n, hkv, d), dtype=BF, device="cuda") for _ in range(2)]
    kv4.kv4_read(pool, slots, *back)
    for x, y in zip(back, (k, v)):
        c, s, z = quantise(y, group)
        want = s.double() * torch.from_numpy(c - 8).double() + z.double()     # one group a row
        assert (x.cpu().double() - want).abs().max() <= UNIT[BF] * want.abs().max()


# ------------------------------------------------------------ write and read
def write_reference(blocks, slots, k, v, group):
    d = k.shape[-1]
    for side, x in ((0, k), (1, v)):
        codes, s, z = quantise(x, group)
        for i, slot in enumerate(slots):
            if 0 <= slot < blocks.shape[0] * P:
                for h in range(k.shape[1]):
                    put(blocks[slot // P, h], int(slot % P), side, codes[i, h], s[i, h], z[i, h], d, group)


def rows_for(kind, n, h, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, h, d), generator=g)
    if kind == "equal":
        x = x[..., :1].expand(n, h, d).clone()
    elif kind == "zero":
        x = torch.zeros((n, h, d))
    elif kind == "ties":       # multiples of a half step: every second value lies between two codes
        x = torch.randint(0, 31, (n, h, d), generator=g).float() * 0.5
        x[..., ::16], x[..., 1::16] = 0.0, 15.0
    elif kind == "offset":
        x = x * 0.01 + 100.0
    elif kind == "tiny":
        x = x * (2.0 ** -130 if dtype is BF else 2.0 ** -22)
    elif kind == "huge":
        x = torch.sign(x) * (3.3e38 if dtype is BF else 65000.0) * torch.rand((n, h, d), generator=g)
    elif kind == "broken":
        x[0::3, :, 5], x[1::4, 0, d - 1], x[2::5, -1, 40] = float("nan"), float("inf"), float("-inf")
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("kind", ["normal", "equal", "zero", "ties", "offset", "tiny", "huge", "broken"])
def test_written_pools_are_the_reference_byte_for_byte(kv4, d, group, dtype, kind):
    n, h, pages = 37, 3, 6
    rng = np.random.default_rng(d + group)
    blocks = rng.integers(0, 256, (pages, h, block_bytes(d, group)), dtype=np.uint8)   # what the other slots hold stays
    slots = rng.permutation(pages * P)[:n].astype(np.int64)
    k, v = (rows_for(kind, n, h, d, dtype, s) for s in (1, 2))
    pool = kv4.Pool(torch.from_numpy(blocks.copy()).cuda(), d, group, dtype)
    err = err_word()
    kv4.kv4_write(pool, torch.from_numpy(slots).cuda(), k.cuda(), v.cuda(), device_error=err)
    write_reference(blocks, slots, k, v, group)
    got = pool.data.cpu().numpy()
    if kind == "broken":   # any NaN will do
        m = blocks[..., 16 * d:].copy().view(np.uint16)
        w = got[..., 16 * d:].copy().view(np.uint16)
        as_f = lambda x: torch.from_numpy(x.astype(np.int32)).to(torch.int16).view(dtype).float().numpy()  # noqa: E731
        fm, fw = as_f(m), as_f(w)
        assert (np.isnan(fm) == np.isnan(fw)).all() and np.isnan(fm).any()
        assert (m == w)[~np.isnan(fm)].all()
        assert (got[..., :16 * d] == blocks[..., :16 * d]).all()
    else:
        assert (got == blocks).all(), np.argwhere(got != blocks)[:5].tolist()
    assert int(err) == 0


@pytest.mark.parametrize("n,start", [(1, 0), (1, 15), (15, 1), (16, 0), (17, 3), (64, 0), (500, 7), (1003, 0)])
@pytest.mark.parametrize("h,d,group,dtype", [(4, 128, 128, BF), (1, 64, 32, FP), (32, 128, 32, BF)])
def test_runs_of_tokens_and_strided_rows(kv4, n, start, h, d, group, dtype):
    """Consecutive positions from inside a page on, pages in any order, K and V slices of one projection; skipped and
    bad slots between them."""
    if n * h * d > 5e5:
        h = 2
    rng = np.random.default_rng(n)
    pages = (n + start + P - 1) // P + 2
    order = rng.permutation(pages)
    pos = np.arange(n) + start
    slots = order[pos // P].astype(np.int64) * P + pos % P
    bad = 0
    if n > 20:
        slots[5], slots[11], slots[n - 2] = -1, pages * P, -2
        bad = 1
    qkv = torch.randn((n, 3 * h, d), generator=torch.Generator().manual_seed(n)).to(dtype)
    k, v = qkv[:, h:2 * h], qkv[:, 2 * h:]
    blocks = rng.integers(0, 256, (pages, h, block_bytes(d, group)), dtype=np.uint8)
    pool = kv4.Pool(torch.from_numpy(blocks.copy()).cuda(), d, group, dtype)
    dev, err = qkv.cuda(), err_word()
    ds = torch.from_numpy(slots).cuda()
    kv4.kv4_write(pool, ds, dev[:, h:2 * h], dev[:, 2 * h:], device_error=err)
    write_reference(blocks, slots, k, v, group)
    got = pool.data.cpu().numpy()
    assert (got == blocks).all(), np.argwhere(got != blocks)[:5].tolist()
    assert int(err) == bad
    # and back, into slices of wider rows
    wide = torch.full((n, 2 * h + 1, d), 7.0, dtype=dtype, device="cuda")
    err.zero_()
    kv4.kv4_read(pool, ds, wide[:, :h], wide[:, h:2 * h], device_error=err)
    ok = (slots >= 0) & (slots < pages * P)
    safe = np.where(ok, slots, 0)
    full = values(blocks, d, group, dtype)[:2]
    for x, want in zip((wide[:, :h], wide[:, h:2 * h]), full):
        want = want[safe // P, :, safe % P] * ok[:, None, None]
        lim = UNIT[dtype] * (1 + 2.0 ** -20) * np.abs(want) + TINY[dtype]
        # the sum s (c - 8) + z is rounded once in 32 bits before it is rounded to 16
        lim += 2.0 ** -23 * np.abs(want)
        assert (np.abs(x.cpu().double().numpy() - want) <= lim).all()
    assert (wide[:, 2 * h:] == 7.0).all()
    assert int(err) == bad


def test_reads_repeat_and_come_in_any_order(kv4):
    d, group, h, pages = 64, 64, 3, 5
    blocks = random_pool(pages, h, d, group, FP, 1)
    slots = np.random.default_rng(0).integers(-1, pages * P, 333)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, FP)
    k, v = (torch.full((333, h, d), float("nan"), dtype=FP, device="cuda") for _ in range(2))
    kv4.kv4_read(pool, torch.from_numpy(slots).cuda(), k, v)
    for x, want in zip((k, v), values(blocks, d, group, FP)[:2]):
        want = want[np.maximum(slots, 0) // P, :, np.maximum(slots, 0) % P] * (slots >= 0)[:, None, None]
        assert (np.abs(x.cpu().double().numpy() - want) <= (UNIT[FP] + 2.0 ** -22) * np.abs(want) + TINY[FP]).all()
        assert (x[torch.from_numpy(slots).cuda() == -1] == 0).all()


def test_rows_without_tokens_do_nothing(kv4):
    pool = kv4.Pool.empty(2, 2, 64, 32)
    none = torch.empty((0, 2, 64), dtype=BF, device="cuda")
    slots = torch.empty(0, dtype=torch.int64, device="cuda")
    kv4.kv4_write(pool, slots, none, none)
    kv4.kv4_read(pool, slots, none, none)
    assert not pool.data.any()


def test_tensors_that_are_refused(kv4):
    pool = kv4.Pool.empty(4, 2, 64, 32)
    tabs = kv4.Tables.empty(4, 3, 2)
    work = kv4.kv4_workspace(pool, 4)
    c = dict(device="cuda")
    slots = torch.zeros(3, dtype=torch.int64, **c)
    k = torch.zeros((3, 2, 64), dtype=BF, **c)
    for bad in (k.half(), k.cpu(), k[:2], k[..., :32], k.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            kv4.kv4_write(pool, slots, bad, k)
        with pytest.raises(ValueError):
            kv4.kv4_read(pool, slots, k, bad)
    with pytest.raises(ValueError):
        kv4.kv4_write(pool, slots.int(), k, k)
    q, out = torch.zeros((3, 4, 64), dtype=BF, **c), torch.zeros((3, 4, 64), dtype=BF, **c)
    for a in (dict(q=q.half()), dict(out=out[:2]), dict(lse=torch.zeros(11, **c)), dict(workspace=work.view(torch.int32)),
              dict(seq_ids=torch.zeros(2, dtype=torch.int32, **c))):
        with pytest.raises(ValueError):
            kv4.kv4_decode_attention(**{**dict(pool=pool, tables=tabs, q=q, out=out, workspace=work), **a})
    with pytest.raises(ValueError):
        kv4.Pool(torch.zeros((4, 2, 100), dtype=torch.uint8, **c), 64, 32)
    new = torch.ones(3, dtype=torch.int32, **c)
    with pytest.raises(ValueError):
        kv4.kv_tables_step(tabs, None, new, slots, positions=torch.zeros(2, dtype=torch.int32, **c))
    with pytest.raises(ValueError):
        kv4.kv_tables_step(tabs, new[:2], new, slots)


# -------------------------------------------------------------------- tables
class Pair:
    """Device tables and their model, stepped together."""

    def __init__(self, kv4, seqs, width, pages, seed, lens=None, order=None):
        rng = np.random.default_rng(seed)
        self.kv4 = kv4
        lens = np.zeros(seqs, np.int32) if lens is None else np.array(lens, np.int32)
        order = rng.permutation(pages).astype(np.int32) if order is None else np.array(order, np.int32)
        held = [(int(n) + P - 1) // P for n in lens]
        table = np.full((seqs, width), -1, np.int32)
        at = 0
        for i, n in enumerate(held):
            table[i, :n] = order[at:at + n]
            at += n
        head = int(rng.integers(0, pages))
        ring = np.full(pages, -9, np.int32)
        ring[(head + np.arange(pages - at)) % pages] = order[at:]
        self.m = TablesModel(table, lens, ring, head, pages - at)
        c = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        self.t = kv4.Tables(c(table), c(lens), c(ring), c([head, pages - at, 0, 0]))

    def step(self, ids, new, room=None, extras=True, pass_ids=True):
        room = int(np.maximum(new, 0).sum()) if room is None else room
        slots = torch.full((room,), 77, dtype=torch.int64, device="cuda")
        pos = torch.full((room,), 77, dtype=torch.int32, device="cuda") if extras else None
        cu = torch.full((len(new) + 1,), 77, dtype=torch.int32, device="cuda") if extras else None
        err = err_word()
        d = lambda x: torch.tensor(np.array(x), dtype=torch.int32, device="cuda")  # noqa: E731
        self.kv4.kv_tables_step(self.t, d(ids) if pass_ids else None, d(new), slots, pos, cu, device_error=err)
        ws, wp, wcu, we = self.m.step(ids, new, room)
        assert (slots.cpu().numpy() == ws).all()
        if extras:
            assert (pos.cpu().numpy() == wp).all() and (cu.cpu().numpy() == wcu).all()
        assert int(err) == we
        self.check()
        return ws, we

    def check(self):
        m, t = self.m, self.t
        assert (t.lens.cpu().numpy() == m.lens).all()
        assert t.free_state.cpu().tolist() == [m.head, m.count, 0, 0]
        live = (m.head + np.arange(m.count)) % len(m.ring)
        assert (t.free_ring.cpu().numpy()[live] == m.ring[live]).all()
        table = t.block_table.cpu().numpy()
        for i, n in enumerate(m.lens):
            k = (int(n) + P - 1) // P
            assert (table[i, :k] == m.table[i, :k]).all()


def test_steps_of_a_serving_loop(kv4):
    """Random growth, rejected drafts and closed requests, in place, over many steps; no page is ever lost or shared."""
    rng = np.random.default_rng(0)
    p = Pair(kv4, 40, 30, 300, 0)
    oom = 0
    for it in range(120):
        n = int(rng.integers(1, 41))
        ids = rng.permutation(40)[:n]
        new = np.where(rng.random(n) < 0.6, 1, rng.integers(0, 90, n))
        shrink = rng.random(n)
        have = p.m.lens[ids]
        new = np.where(shrink < 0.15, -np.minimum(have, rng.integers(0, 6, n)), new)
        new = np.where(shrink > 0.93, -have, new)
        _, e = p.step(ids, new, room=int(np.maximum(new, 0).sum()) + int(rng.integers(0, 9)), extras=bool(it % 3))
        oom += bool(e & 8)
        held = np.concatenate([p.m.table[i, :(int(l) + P - 1) // P] for i, l in enumerate(p.m.lens)])
        free = p.m.ring[(p.m.head + np.arange(p.m.count)) % 300]
        assert sorted(np.concatenate([held, free]).tolist()) == list(range(300))
    assert oom > 0     # the pool ran out on the way


@pytest.mark.parametrize("n", [1, 2, 31, 33, 1023, 1024, 1025, 2500, 4096])
def test_batches_of_any_size(kv4, n):
    rng = np.random.default_rng(n)
    p = Pair(kv4, n, 6, 6 * n, n, lens=rng.integers(0, 60, n))
    p.step(np.arange(n), rng.integers(0, 30, n), pass_ids=False)
    p.step(np.arange(n)[::-1].copy(), -np.minimum(rng.integers(0, 20, n), p.m.lens[::-1]))
    p.step(rng.permutation(n), np.ones(n, np.int64))


@pytest.mark.parametrize("tokens", [1, 16, 17, 5000, 300001])
def test_one_long_prompt(kv4, tokens):
    pages = (tokens + P - 1) // P
    p = Pair(kv4, 3, pages + 1, pages + 4, 1, lens=[0, 5, 0])
    p.step([1, 0, 2], [0, tokens, 0])
    p.step([0, 1], [-tokens, 3])


def test_refusals_of_single_rows(kv4):
    p = Pair(kv4, 6, 4, 12, 3, lens=[60, 10, 0, 16, 64, 0])     # 10 pages held, 2 free
    _, e = p.step([0, 1, 7, -1, 4], [5, 1, 3, 2, 1])            # past its row; fine; unknown twice; a full row
    assert e == 4
    _, e = p.step([3, 2, 1, 5], [1, 20, 1, 1])                  # takes one; needs two of one left; needs none; refused too
    assert e == 8
    _, e = p.step([0, 1], [-70, -5])                            # below zero; fine
    assert e == 4
    _, e = p.step([0, 3, 2], [2, 4, 1], room=5)                 # the second row passes the room, and so does the third
    assert e == 4
    _, e = p.step([1, 0], [-2 ** 31, 2 ** 31 - 1], room=8)
    assert e == 4


def test_pages_that_are_given_back_twice_are_refused(kv4):
    p = Pair(kv4, 2, 4, 6, 3, lens=[40, 10])
    p.t.free_state[1], p.m.count = 5, 5                         # the ring claims more than is free
    _, e = p.step([0, 1], [-40, 2])
    assert e == 1 and p.m.lens.tolist() == [40, 12]


def test_a_page_id_outside_the_pool_gives_no_slot(kv4):
    p = Pair(kv4, 2, 4, 8, 3, lens=[10, 10])
    at = p.m.head
    p.t.free_ring[at] = 8
    p.m.ring[at] = 8
    ws, e = p.step([0, 1], [10, 10])
    assert e == 1 and (ws[6:10] == -1).all() and (ws[:6] >= 0).all() and (ws[10:] >= 0).all()


def test_a_broken_free_state_hands_out_nothing(kv4):
    for state in ([-1, 2, 0, 0], [8, 2, 0, 0], [0, 9, 0, 0], [0, -1, 0, 0]):
        p = Pair(kv4, 2, 4, 8, 3, lens=[10, 10])
        p.t.free_state.copy_(torch.tensor(state, dtype=torch.int32))
        slots, err = torch.empty(12, dtype=torch.int64, device="cuda"), err_word()
        kv4.kv_tables_step(p.t, None, torch.tensor([2, 10], dtype=torch.int32, device="cuda"), slots, device_error=err)
        assert int(err) == 1 | 8
        assert (slots[:2] >= 0).all() and (slots[2:] == -1).all()
        assert p.t.lens.tolist() == [12, 10]


def test_a_step_may_leave_its_inputs_alone(kv4):
    """lens_out and free_state_out: the same step twice from the same state."""
    p = Pair(kv4, 5, 6, 30, 9, lens=[3, 0, 40, 16, 15])
    new = torch.tensor([1, 20, -8, 1, 2], dtype=torch.int32, device="cuda")
    before = p.t.lens.clone(), p.t.free_state.clone()
    got = []
    for _ in range(2):
        slots = torch.empty(24, dtype=torch.int64, device="cuda")
        lens, state = torch.empty(5, dtype=torch.int32, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
        kv4.kv_tables_step(p.t, None, new, slots, lens_out=lens, free_state_out=state)
        got.append((slots, lens, state))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    assert torch.equal(p.t.lens, before[0]) and torch.equal(p.t.free_state, before[1])
    ws, _, _, _ = p.m.step(np.arange(5), new.cpu().numpy(), 24)
    assert (got[0][0].cpu().numpy() == ws).all()
    assert got[0][1].tolist() == p.m.lens.tolist() and got[0][2].tolist() == [p.m.head, p.m.count, 0, 0]


# --------------------------------------------------------------- all together
def test_a_decode_loop_from_a_graph(kv4):
    """Tables, write and attention of a step captured once and replayed: lengths, slots and pages follow on the device."""
    d, group, hq, hkv, b = 128, 64, 8, 2, 5
    tabs = kv4.Tables.empty(40, 6, 8)
    pool = kv4.Pool.empty(40, hkv, d, group)
    work, err = kv4.kv4_workspace(pool, hq), err_word()
    i32 = dict(dtype=torch.int32, device="cuda")
    ids = torch.tensor([4, 0, 5, 2, 1], **i32)
    g = torch.Generator().manual_seed(0)
    prompts = [31, 16, 1, 40, 15]
    new = torch.tensor(prompts, **i32)
    slots = torch.empty(sum(prompts), dtype=torch.int64, device="cuda")
    kv = [torch.randn((sum(prompts), hkv, d), generator=g).to(BF) for _ in range(2)]
    kv4.kv_tables_step(tabs, ids, new, slots, device_error=err)
    kv4.kv4_write(pool, slots, kv[0].cuda(), kv[1].cuda(), device_error=err)
    cuts = np.cumsum(prompts)[:-1]
    hist = [list(x) for x in np.split(np.arange(sum(prompts)), cuts)]
    rows = [list(kv[0]), list(kv[1])]

    q, k1, v1 = (torch.zeros((b, n, d), dtype=BF, device="cuda") for n in (hq, hkv, hkv))
    out, lse = torch.empty_like(q), torch.empty((b, hq), device="cuda")
    one, step_slots = torch.ones(b, **i32), torch.empty(b, dtype=torch.int64, device="cuda")

    def step(stream):
        kv4.kv_tables_step(tabs, ids, one, step_slots, device_error=err, stream=stream)
        kv4.kv4_write(pool, step_slots, k1, v1, device_error=err, stream=stream)
        kv4.kv4_decode_attention(pool, tabs, q, out, work, seq_ids=ids, lse=lse, device_error=err, stream=stream)

    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step(side)
    for it in range(35):
        new_q, new_k, new_v = (torch.randn(t.shape, generator=g).to(BF) for t in (q, k1, v1))
        for t, x in ((q, new_q), (k1, new_k), (v1, new_v)):
            t.copy_(x)
        graph.replay()
        for i in range(b):
            hist[i].append(len(rows[0]))
            rows[0].append(new_k[i])
            rows[1].append(new_v[i])
        if it % 8 == 2:
            torch.cuda.synchronize()
            blocks, table = pool.data.cpu().numpy(), tabs.block_table.cpu().numpy()[ids.cpu().numpy()]
            lens = [len(x) for x in hist]
            assert tabs.lens.cpu().numpy()[ids.cpu().numpy()].tolist() == lens
            # the pool holds what was written, wherever it lies
            for i in range(b):
                at = np.array([table[i, t // P] for t in range(lens[i])])
                for side_, kept in zip((0, 1), rows):
                    want = torch.stack([kept[j] for j in hist[i]])
                    c = quantise(want, group)[0]
                    codes = unpack(blocks, d, group, BF)[side_][0]
                    assert (codes[at, :, np.arange(lens[i]) % P] == c).all()
            ref = attention(blocks, table, lens, new_q.double().numpy(), group, BF, d ** -0.5)
            assert_attention(out, lse, ref, BF, it)
    assert int(err) == 0


def test_calls_on_another_stream_follow_its_order(kv4):
    """Write, read and attention on a side stream behind a slow kernel that makes their inputs."""
    d, group, h, n = 128, 128, 4, 600
    side = torch.cuda.Stream()
    pool, tabs = kv4.Pool.empty(60, h, d, group), kv4.Tables.empty(60, 1, 40)
    work = kv4.kv4_workspace(pool, h)
    g = torch.Generator().manual_seed(3)
    k, v, q = (torch.randn(s, generator=g).to(BF).cuda() for s in ((n, h, d), (n, h, d), (1, h, d)))
    slots = torch.empty(n, dtype=torch.int64, device="cuda")
    new = torch.tensor([n], dtype=torch.int32, device="cuda")
    k2, v2, q2 = (torch.full_like(x, float("nan")) for x in (k, v, q))
    back, out = [torch.empty_like(k), torch.empty_like(k)], torch.empty_like(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        for a, b in ((k2, k), (v2, v), (q2, q)):
            a.copy_(b)
        kv4.kv_tables_step(tabs, None, new, slots, stream=side)
        kv4.kv4_write(pool, slots, k2, v2, stream=side)
        kv4.kv4_read(pool, slots, *back, stream=side)
        kv4.kv4_decode_attention(pool, tabs, q2, out, work, stream=side)
    side.synchronize()
    blocks, table = pool.data.cpu().numpy(), tabs.block_table.cpu().numpy()
    assert_attention(out, None, attention(blocks, table, [n], q.double().cpu().numpy(), group, BF, d ** -0.5), BF)
    want = values(blocks, d, group, BF)[0][table[0][np.arange(n) // P], :, np.arange(n) % P]
    assert (np.abs(back[0].double().cpu().numpy() - want) <= (UNIT[BF] + 2.0 ** -22) * np.abs(want) + TINY[BF]).all()

"""Long sums of the 4-bit attention: batches so large that one warp works hundreds to thousands of
pages of a row, against 64 bits and to a bound that follows the sums' own terms.

Many rows repeat a few requests and a few queries, so that the grid's warps are full and the
reference stays small: 4096 rows on some 2400 warps give every warp more than a whole row."""
import numpy as np
import pytest
import torch

from _kv4_common import P, TINY, UNIT, random_pool, values

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]
WINDOW = 32     # pages after which the tensor cores' sums are put away


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def reference(blocks, pages, n, q, group, dtype, scale, window=WINDOW):
    """64-bit attention of queries q [Q, Hq, D] over the first n tokens of `pages`; (out, lse, limit of an
    output's error, limit of the errors' mean, limit of lse's error).

    With weights w, scales s, codes c and middles z, out = sum w s (c - 8) + sum w z.
    * w s is rounded to 11 bits: at most 2^-11 of each term a = w s (c - 8), a standard deviation of
      2^-11 / sqrt(3) of sqrt(sum a^2) where the roundings differ, 2^-11 of |sum a| where they are alike; six
      deviations.  Terms below 2^-30 of the largest lose bits: 2^-31 of it each.
    * The tensor cores cut off up to 2^-24 of the largest addend, for 16 products and the running sum of
      codes 0 .. 15.  The running sum is at most that of a window; a code in bits 0-3 counts as 2^10 / 15 times
      itself until then, which is 17 * 1024 / (16 * 15) of a page's sum: (17 (window / 2 + 1) + 73) 2^-24 of sum
      15 w s, half of it on average (thousands of cuts: near their mean), the same for the sum that takes the 8 back.
    * A score is off by at most 2^-21 of a = scale sum |q| (8 s + |z|), what tokens share drops out: six
      deviations of that / sqrt(3) of sqrt(sum w^2 (v - out)^2).
    * fp32 sums over n / 8 tokens a lane, rounded to nearest: six deviations of sqrt(n / 8) 2^-24.
    * The output's own rounding.
    The mean of a head's D errors has half of the cuts, and 1 / sqrt(D) of the rest: of six deviations of 1 / sqrt(3) of it."""
    nq, hq, d = q.shape
    g = hq // blocks.shape[1]
    out, lse, lim = np.zeros((nq, hq, d)), np.full((nq, hq), -np.inf), np.full((nq, hq, d), TINY[dtype])
    mean, lse_lim = np.zeros((nq, hq)), np.zeros((nq, hq))
    if n == 0:
        return out, lse, lim, mean, lse_lim
    k, v, (sk, zk), (sv, zv) = values(blocks[np.asarray(pages)], d, group, dtype)
    k, v, sk, zk, sv, zv = (x.transpose(1, 0, 2, 3).reshape(blocks.shape[1], -1, d)[:, :n] for x in (k, v, sk, zk, sv, zv))
    for i in range(nq):
        for h in range(hq):
            x = k[h // g] @ q[i, h] * scale
            m = x.max()
            w = np.exp(x - m)
            lse[i, h] = m + np.log(w.sum())
            w = w / w.sum()
            V, s, z = v[h // g], np.abs(sv[h // g]), zv[h // g]
            o = w @ V
            a = w[:, None] * (V - z)
            rounding = 2.0 ** -11 * (np.abs(a.sum(0)) + 6 / 3 ** 0.5 * np.sqrt((a * a).sum(0)))
            rounding += n * 2.0 ** -31 * 15 * (w[:, None] * s).max(0)
            cut = (17 * (window / 2 + 1) + 73) * 2.0 ** -24 * 15 * (w @ s)
            size = ((8 * sk[h // g] + np.abs(zk[h // g])) @ np.abs(q[i, h])).max() * abs(scale)
            score = 2.0 ** -21 * size * 6 / 3 ** 0.5 * np.sqrt((w * w) @ (V - o) ** 2)
            sums = 6 * (n / 8 + 1) ** 0.5 * 2.0 ** -24 * (w @ np.abs(z) + np.abs(o))
            out[i, h] = o
            random = (1 + UNIT[dtype]) * (rounding + score + sums) + UNIT[dtype] * np.abs(o)
            lim[i, h] += random + cut
            mean[i, h] = (cut / 2).mean() + 6 * ((random ** 2).mean() / 3 / d) ** 0.5
            lse_lim[i, h] = 2.0 ** -21 * size + 2.0 ** -20 * (1 + abs(lse[i, h])) + 6 * (n / 8 + 1) ** 0.5 * 2.0 ** -24
    return out, lse, lim, mean, lse_lim


def run(kv4, blocks, table, lens, kept, q, hkv, group, dtype, rows=4096, scale=0.0, seed=0, error=0):
    """`rows` rows, each one of the requests and one of the queries in any order; kept[i]: (pages, tokens) that
    request i's result is to come from.  Returns outputs' error by request, [requests][rows of it, Hq, D]."""
    d, hq = q.shape[-1], q.shape[1]
    rng = np.random.default_rng(seed)
    ids, which = rng.integers(0, len(lens), rows), rng.integers(0, q.shape[0], rows)
    pool = kv4.Pool(torch.from_numpy(blocks).cuda(), d, group, dtype)
    tabs = kv4.Tables(torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"))
    dq = q.cuda()[torch.from_numpy(which).cuda()].contiguous()
    out, lse = torch.full_like(dq, float("nan")), torch.full((rows, hq), float("nan"), device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kv4.kv4_decode_attention(pool, tabs, dq, out, kv4.kv4_workspace(pool, hq), lse=lse, softmax_scale=scale, device_error=err,
                             seq_ids=torch.tensor(ids, dtype=torch.int32, device="cuda"))
    assert int(err) == error
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert np.isfinite(out).all()
    errors = []
    for i, (pages, n) in enumerate(kept):
        at = np.flatnonzero(ids == i)
        r_out, r_lse, lim, mean, lse_lim = reference(blocks, pages, n, q.double().numpy(), group, dtype, scale or d ** -0.5)
        e = out[at] - r_out[which[at]]
        over = np.abs(e) - lim[which[at]]
        assert (over <= 0).all(), (i, n, float(over.max()), np.argwhere(over > 0)[:4].tolist())
        if n == 0:
            assert (lse[at] == -np.inf).all() and not out[at].any()
            continue
        le = np.abs(lse[at] - r_lse[which[at]])
        assert (le <= lse_lim[which[at]]).all(), (i, n, float((le - lse_lim[which[at]]).max()))
        for j in np.unique(which[at]):
            off = e[which[at] == j].mean((0, 2))
            assert (np.abs(off) <= mean[j]).all(), (i, n, j, off, mean[j])
        errors.append(e)
    return errors


def queries(n, hq, d, dtype, seed, size):
    return (torch.randn((n, hq, d), generator=torch.Generator().manual_seed(seed)) * size).to(dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("pages", [300, 6000])
def test_rows_that_one_warp_works_alone(kv4, d, group, dtype, pages):
    """Flat softmaxes over thousands of pages: outputs are small next to the sums that they come from."""
    blocks = random_pool(pages, 1, d, group, dtype, pages + d)
    table = np.random.default_rng(1).permutation(pages).astype(np.int32)[None]
    q = queries(4, 1, d, dtype, 2, 0.3)
    run(kv4, blocks, table, [pages * P - 5], [(table[0], pages * P - 5)], q, 1, group, dtype)


@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("d,group", SHAPES)
def test_long_shares_of_ragged_rows(kv4, d, group, dtype):
    """Shares of some hundred pages that hold rows of all lengths, rows cut by shares, pages outside the pool."""
    lens = [3001, 517, 0, 40, 1250, 16, 77, 1]
    n = [(x + P - 1) // P for x in lens]
    order = np.random.default_rng(5).permutation(sum(n)).astype(np.int32)
    table, at = np.full((len(lens), max(n)), -7, np.int32), 0
    for i, k in enumerate(n):
        table[i, :k], at = order[at:at + k], at + k
    kept = [(table[i, :k], lens[i]) for i, k in enumerate(n)]
    table[0, 50], table[4, 0] = sum(n), -1              # their tokens are left out
    kept[0] = (np.delete(kept[0][0], 50), lens[0] - P)
    kept[4] = (kept[4][0][1:], lens[4] - P)
    blocks = random_pool(sum(n), 2, d, group, dtype, 3)
    run(kv4, blocks, table, lens, kept, queries(3, 6, d, dtype, 4, 1.0), 2, group, dtype, error=1)


@pytest.mark.parametrize("d,group", [(64, 32), (128, 32), (128, 128)])
@pytest.mark.parametrize("order", ["rise", "fall", "mix"])
def test_scales_that_move_along_a_long_share(kv4, d, group, order):
    """V's scales go through 2^-9 .. 2^9 over a row that one warp works, and scores rise along it."""
    pages = 700
    n = pages * P
    blocks = random_pool(pages, 1, d, group, BF, 8)
    rng = np.random.default_rng(0)
    g = d // group
    t = np.arange(n)
    e = {"rise": -9 + 18 * t // n, "fall": 9 - 18 * t // n, "mix": rng.integers(-9, 10, n)}[order].reshape(pages, 1, P, 1, 1)
    meta = torch.from_numpy(rng.uniform(0.5, 1.0, (pages, 1, P, g, 2)) * 2.0 ** e).to(BF)
    blocks[..., 16 * d + 64 * g:] = meta.view(torch.uint8).numpy().reshape(pages, 1, -1)
    table = np.arange(pages, dtype=np.int32)[None]       # in order: K's middles make later scores larger
    lift = torch.from_numpy(np.broadcast_to((t / n).reshape(pages, 1, P, 1), (pages, 1, P, g)).copy() * 4).to(BF)
    k = blocks[..., 16 * d:16 * d + 64 * g].copy().view(np.uint16).reshape(pages, 1, P, g, 2)
    k[..., 1] = lift.view(torch.int16).numpy().view(np.uint16)
    blocks[..., 16 * d:16 * d + 64 * g] = k.view(np.uint8).reshape(pages, 1, -1)
    q = queries(4, 1, d, BF, 6, 0.3) + 0.1
    run(kv4, blocks, table, [n], [(table[0], n)], q, 1, group, BF)

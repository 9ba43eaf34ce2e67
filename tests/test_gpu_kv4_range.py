"""V's scales far apart in the 4-bit attention: between the groups of a token, between the tokens of a group
(the widest of negligible weight), and between what the query heads of one KV head attend to.  Each output
against 64 bits, to a bound made of its own sum's terms (test_gpu_kv4_sums.reference)."""
import numpy as np
import pytest
import torch

from _kv4_common import P, random_pool
from test_gpu_kv4_sums import BF, FP, queries, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def words(blocks, side, d, group):
    """View of the scale words, uint16 [pages, heads, 16, groups, (s, z)], of K (0) or V (1): a copy and the place it goes back to."""
    n = 64 * (d // group)
    at = slice(16 * d + side * n, 16 * d + (side + 1) * n)
    return blocks[..., at].copy().view(np.uint16).reshape(*blocks.shape[:2], P, d // group, 2), at


def scale_words(blocks, side, d, group, factor, dtype):
    """Multiplies s and z of one side by powers of two `factor` (broadcast to [pages, heads, 16, groups])."""
    w, at = words(blocks, side, d, group)
    x = torch.from_numpy(w.view(np.int16).copy()).view(dtype).double()
    x = (x * torch.from_numpy(np.broadcast_to(factor, w.shape[:-1]).copy())[..., None]).to(dtype)
    blocks[..., at] = x.view(torch.int16).numpy().view(np.uint8).reshape(*blocks.shape[:2], -1)


def lift_keys(blocks, d, group, lift, dtype):
    """K's middles become `lift` (broadcast to [pages, heads, 16, groups]): queries of positive elements score them by it."""
    w, at = words(blocks, 0, d, group)
    z = torch.from_numpy(np.ascontiguousarray(np.broadcast_to(lift, w.shape[:-1])).astype(np.float64)).to(dtype)
    w[..., 1] = z.view(torch.int16).numpy().view(np.uint16)
    blocks[..., at] = w.view(np.uint8).reshape(*blocks.shape[:2], -1)


def table_of(pages):
    return np.arange(pages, dtype=np.int32)[None]


@pytest.mark.parametrize("rows", [8, 4096])
@pytest.mark.parametrize("d,group,exps", [(128, 32, [0, -20, -31, -40]), (128, 32, [-60, 60, 0, -100]), (128, 64, [0, -31]),
                                          (64, 32, [-40, 0]), (64, 32, [0, -26])])
def test_groups_far_apart(kv4, d, group, exps, rows):
    """Every group keeps its own precision, whatever the others' scales."""
    pages = 90
    blocks = random_pool(pages, 2, d, group, BF, 21)
    scale_words(blocks, 1, d, group, 2.0 ** np.array(exps, float), BF)
    n = pages * P - 3
    run(kv4, blocks, table_of(pages), [n], [(table_of(pages)[0], n)], queries(3, 6, d, BF, 4, 0.7), 2, group, BF, rows=rows)


@pytest.mark.parametrize("rows", [8, 4096])
@pytest.mark.parametrize("d,group,dtype", [(128, 128, BF), (128, 32, BF), (64, 64, BF), (64, 32, FP), (128, 64, FP)])
@pytest.mark.parametrize("tok", [0, 5, 700, 1400])
def test_a_wide_token_of_no_weight(kv4, d, group, dtype, tok, rows):
    """One token's scales are 2^40 of the others' (fp16: 2^23, theirs being 2^-10 of the usual) and its weight e^-90 of theirs."""
    pages = 90
    blocks = random_pool(pages, 1, d, group, dtype, 22)
    factor, lift = np.ones((pages, 1, P, 1)), np.full((pages, 1, P, 1), 0.0)
    if dtype is FP:
        factor *= 2.0 ** -10
    factor[tok // P, :, tok % P] = 2.0 ** 40 if dtype is BF else 2.0 ** 13
    lift[tok // P, :, tok % P] = -90 / (0.5 * d * d ** -0.5)
    scale_words(blocks, 1, d, group, factor, dtype)
    lift_keys(blocks, d, group, lift, dtype)
    q = (queries(4, 1, d, dtype, 4, 0.02) + 0.5).to(dtype)
    n = pages * P
    run(kv4, blocks, table_of(pages), [n], [(table_of(pages)[0], n)], q, 1, group, dtype, rows=rows)


@pytest.mark.parametrize("rows", [8, 4096])
@pytest.mark.parametrize("d,group", [(128, 128), (128, 32), (64, 64)])
def test_query_heads_that_attend_to_different_scales(kv4, d, group, rows):
    """Half of the tokens have scales 2^40 of the others'.  Queries of one sign attend to them, queries of the other
    sign to the rest: eight heads of one KV head, each with the precision of its own tokens."""
    pages = 60
    blocks = random_pool(pages, 1, d, group, BF, 23)
    wide = np.random.default_rng(0).random((pages, 1, P, 1)) < 0.5
    scale_words(blocks, 1, d, group, np.where(wide, 2.0 ** 40, 1.0), BF)
    lift_keys(blocks, d, group, np.where(wide, 1.0, -1.0) * 50 / (0.5 * d * d ** -0.5), BF)
    q = queries(3, 8, d, BF, 4, 0.02) + 0.5 * torch.tensor([1.0, -1, 1, 1, -1, -1, 1, -1], dtype=BF)[None, :, None]
    n = pages * P - 9
    run(kv4, blocks, table_of(pages), [n], [(table_of(pages)[0], n)], q.to(BF), 1, group, BF, rows=rows)


@pytest.mark.parametrize("rows", [8, 4096])
@pytest.mark.parametrize("d,group", [(128, 64), (64, 64), (128, 32)])
def test_wide_tokens_that_scores_leave_behind(kv4, d, group, rows):
    """Scales fall from 2^60 to 1 along a row while scores rise by 240: early tokens have all the weight when they
    come, and in the end none."""
    pages = 80
    blocks = random_pool(pages, 1, d, group, BF, 24)
    t = np.arange(pages * P).reshape(pages, 1, P, 1) / (pages * P)
    scale_words(blocks, 1, d, group, 2.0 ** np.maximum(np.floor(60 - 70 * t), 0), BF)
    lift_keys(blocks, d, group, (240 * t - 120) / (0.5 * d * d ** -0.5), BF)
    q = (queries(4, 1, d, BF, 4, 0.02) + 0.5).to(BF)
    n = pages * P
    run(kv4, blocks, table_of(pages), [n], [(table_of(pages)[0], n)], q, 1, group, BF, rows=rows)


@pytest.mark.parametrize("d,group", [(128, 128), (64, 32)])
def test_scales_at_the_ends_of_bf16(kv4, d, group):
    """All scales near the type's smallest normal numbers, and near 2^90."""
    pages = 40
    for e in (-118, 90):
        blocks = random_pool(pages, 1, d, group, BF, 25)
        scale_words(blocks, 1, d, group, 2.0 ** e, BF)
        run(kv4, blocks, table_of(pages), [pages * P], [(table_of(pages)[0], pages * P)], queries(2, 4, d, BF, 4, 0.7), 1, group, BF, rows=64)

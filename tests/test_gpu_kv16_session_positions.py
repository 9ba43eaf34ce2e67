"""Positions of a session whose prefixes change: requests that continue a prefix taken up again at another length answer as in a
session made with that length."""
import pytest
import torch

from _kv16_common import assert_attention, assert_rows, attention, inv_freq, turned
from paper_2603_12707_gb300 import workloads as wl

pytestmark = pytest.mark.gpu

CFG = wl.custom("shared_again", 1, 4, 2, 64, 3, lens=[10, 20, 30], seed=6)


def make(prefix_lens, lens=None, of=(0, 1, 0), **kw):
    from paper_2603_12707_gb300 import kv16
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    return SharedPrefixSession(CFG, prefix_lens, list(of), rope=kv16.Rope(inv_freq(32)), lens=lens, slack_pages=16, **kw)


def data(request, n):
    return [wl.kv_block(CFG, 0, request, n, kind, "cuda") for kind in "kv"]


def admit(sess, new, first=None):
    """Grow by new and write the new tokens, the same ones for a request of the same number and length."""
    slots, positions = sess.grow(new) if first is None else sess.grow(new, first_positions=first)
    blocks = [data(r, n) for r, n in enumerate(new) if n > 0]
    if blocks:
        sess.write(0, slots, positions, *(torch.cat(x) for x in zip(*blocks)))
    return positions.tolist()


def step(sess, seed=0):
    q, k, v = wl.step_inputs(CFG, seed, 0, "cuda")
    qr, out = torch.empty_like(q), torch.empty_like(q)
    sess.begin_step()
    sess.append(0, q, k, v, qr)
    sess.attend(0, qr, out)
    sess.check()
    return q, qr, out


def same(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("again", [33, 40, 57, 1])
@pytest.mark.parametrize("at_once", [True, False])
def test_a_prefix_taken_up_again(kvlib, again, at_once):
    sess = make([100, 40])
    admit(sess, [10, 20, 30, 100, 40])
    step(sess)
    sess.grow([0, -21, 0, 0, -40])               # a request and its prefix closed
    if at_once:
        assert admit(sess, [0, 5, 0, 0, again]) == [again + t for t in range(5)] + list(range(again))
    else:
        admit(sess, [0, 0, 0, 0, again])
        assert admit(sess, [0, 5, 0, 0, 0]) == [again + t for t in range(5)]
    new = make([100, again], lens=[11, 5, 31])
    admit(new, [10, 0, 30, 100, 0])
    new.grow([1, 0, 1, 0, 0])
    admit(new, [0, 5, 0, 0, again])
    got, want = step(sess, 1), step(new, 1)
    assert same(got[1], want[1])                 # queries, turned
    assert same(got[2][1], want[2][1])           # the answer of the request that continues it
    assert_rows(got[1], turned(got[0].cpu(), [[111, again + 5, 131]], inv_freq(32), None), torch.bfloat16)


def test_a_prefix_that_outgrows_its_length_before_its_requests_begin(kvlib):
    sess, new = make([100, 40], lens=[0, 0, 0], extra_tokens=140), make([130, 40], lens=[0, 0, 0], extra_tokens=140)
    admit(sess, [0, 0, 0, 100, 40])
    sess.grow([0, 0, 0, -100, 0])
    admit(sess, [0, 0, 0, 130, 0])
    admit(new, [0, 0, 0, 130, 40])
    got, want = step(sess), step(new)
    assert same(got[1], want[1]) and same(got[2], want[2])
    assert_rows(got[1], turned(got[0].cpu(), [[130, 40, 130]], inv_freq(32), None), torch.bfloat16)


def test_prefixes_in_parts_count_whole(kvlib):
    """Until a prefix has been shortened or outgrown it counts with the length that the session was made with."""
    sess = make([100, 40])
    assert admit(sess, [0, 20, 0, 60, 40]) == [40 + t for t in range(20)] + list(range(60)) + list(range(40))
    assert admit(sess, [10, 0, 30, 0, 0])[:10] == [100 + t for t in range(10)]
    slots, positions = sess.grow([0, 0, 0, 40, 0])
    assert positions.tolist() == list(range(60, 100))
    assert sess.first_positions == [100, 40, 100]


def test_tokens_that_were_turned_for_another_length_are_not_continued(kvlib):
    sess = make([100, 40])
    admit(sess, [10, 20, 30, 100, 40])
    before = sess.lens.copy()
    for new in ([0, 0, 0, 0, 1], [0, 0, 0, 0, -7], [0, 0, 0, 3, 0], [0, -19, 0, 0, 5]):
        with pytest.raises(ValueError, match="first_positions"):
            sess.grow(new)
    assert (sess.lens == before).all()
    assert sess.tables.lens.tolist() == before.tolist()
    step(sess)
    sess.grow([0, 0, 0, 0, -40])                 # it goes on without its prefix
    _, qr, _ = step(sess, 1)
    with pytest.raises(ValueError, match="first_positions"):
        sess.grow([0, 0, 0, 0, 33])
    sess.grow([0, 0, 0, 0, 40])                  # the length that its tokens were turned for
    assert sess.first_positions == [100, 40, 100]
    sess.check()


def test_first_positions_that_are_given_stay(kvlib):
    first = [7, 8, 9]
    sess = make([100, 40], first_positions=first)
    admit(sess, [10, 20, 30, 100, 40])
    sess.grow([0, -20, 0, 0, -40])
    assert admit(sess, [0, 5, 0, 0, 33])[:5] == [8 + t for t in range(5)]
    q, qr, _ = step(sess)
    assert_rows(qr, turned(q.cpu(), [[17, 13, 39]], inv_freq(32), None), torch.bfloat16)
    # ... until others are given.
    sess.grow([0, -6, 0, 0, -33])
    assert admit(sess, [0, 5, 0, 0, 12], first=[7, 4, 9])[:5] == [4 + t for t in range(5)]
    q, qr, out = step(sess, 1)
    assert_rows(qr, turned(q.cpu(), [[18, 9, 40]], inv_freq(32), None), torch.bfloat16)
    pool = sess.pools[0]
    ref = attention(pool.k, pool.v, sess.tables.block_table.cpu().numpy(), [12, 6, 32, 100, 12], None, [3, 4, 3], qr, 64 ** -0.5, torch.bfloat16)
    assert_attention(out, None, ref, torch.bfloat16)
    with pytest.raises(ValueError):
        sess.grow([0] * 5, first_positions=[1, 2])


def test_captured_steps_follow(kvlib):
    """A step captured before a prefix changes turns rows for the new length when it is replayed after."""
    side = torch.cuda.Stream()
    sess = make([100, 40], lens=[10, 0, 30], stream=side, extra_tokens=20)
    with torch.cuda.stream(side):
        admit(sess, [10, 0, 30, 100, 40])
        q, k, v = wl.step_inputs(CFG, 0, 0, "cuda")
        qr, out = torch.empty_like(q), torch.empty_like(q)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
        sess.begin_step()
        sess.append(0, q, k, v, qr)
        sess.attend(0, qr, out)
    for i in range(3):
        with torch.cuda.stream(side):
            g.replay()
    sess.check()
    assert_rows(qr, turned(q.cpu(), [[112, 42, 132]], inv_freq(32), None), torch.bfloat16)
    sess.grow([0, -3, 0, 0, -40])
    with torch.cuda.stream(side):
        admit(sess, [0, 2, 0, 0, 25])
        g.replay()
    sess.check()
    assert_rows(qr, turned(q.cpu(), [[113, 27, 133]], inv_freq(32), None), torch.bfloat16)

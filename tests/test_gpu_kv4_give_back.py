"""kv_tables_step where table entries of pages that are given back lie outside the pool: they are reported and left
out, what the ring hands out later are pages."""
import numpy as np
import pytest
import torch

from _kv4_common import P
from test_gpu_kv4 import Pair, err_word, kv4  # noqa: F401

pytestmark = pytest.mark.gpu


def give_back(kv4, p, new, room):
    """One step of all requests in order; returns its error bits."""
    slots, err = torch.empty(room, dtype=torch.int64, device="cuda"), err_word()
    kv4.kv_tables_step(p.t, None, torch.tensor(new, dtype=torch.int32, device="cuda"), slots, device_error=err)
    return int(err)


def free_pages(t):
    head, count, *rest = t.free_state.tolist()
    assert rest == [0, 0]
    ring = t.free_ring.cpu().numpy()
    return ring[(head + np.arange(count)) % len(ring)]


def test_bad_entries_among_pages_given_back(kv4):
    p = Pair(kv4, 3, 5, 20, 7, lens=[40, 64, 10])
    before, table = free_pages(p.t).tolist(), p.m.table
    p.t.block_table[0, 1] = -1
    p.t.block_table[1, 0] = 20
    assert give_back(kv4, p, [-40, -60, 2], 2) == 1
    # row 0 gives pages 0 and 2 (1 is lost), row 1 keeps its first page (the bad one) and gives 1 .. 3
    assert free_pages(p.t).tolist() == before + [table[0, 0], table[0, 2], table[1, 1], table[1, 2], table[1, 3]]
    assert p.t.lens.tolist() == [0, 4, 12]
    assert give_back(kv4, p, [0, -4, 0], 0) == 1              # now that one, too
    assert len(free_pages(p.t)) == len(before) + 5 and p.t.lens.tolist() == [0, 0, 12]


@pytest.mark.parametrize("seqs,seed", [(2, 0), (40, 1), (300, 2), (1500, 3)])
def test_many_pages_given_back_with_holes(kv4, seqs, seed):
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 12 * P, seqs)
    keep = np.minimum(lens, rng.integers(0, 3 * P, seqs))
    pages = int(((lens + P - 1) // P).sum()) + 9
    p = Pair(kv4, seqs, 12, pages, seed, lens=lens)
    before, table = free_pages(p.t).tolist(), p.m.table.copy()
    held = np.arange(12)[None] < ((lens + P - 1) // P)[:, None]
    bad = held & (rng.random(table.shape) < 0.05)
    bad[0, 0], lens_back = held[0, 0], (keep + P - 1) // P
    table[bad] = rng.choice([-1, -2 ** 31, pages, 2 ** 31 - 1], int(bad.sum()))
    p.t.block_table.copy_(torch.from_numpy(table))
    given = [table[i, c] for i in range(seqs) for c in range(lens_back[i], (lens[i] + P - 1) // P)]
    want = [int(x) for x in given if 0 <= x < pages]
    assert give_back(kv4, p, keep - lens, 0) == (1 if len(want) < len(given) else 0)
    free = free_pages(p.t).tolist()
    assert free == before + want
    assert p.t.lens.tolist() == keep.tolist()
    # what is handed out from now on are pages: all of them, to the last one
    grow = P if seqs <= 40 else 1
    fits = [i for i in range(seqs) if keep[i] + grow <= 12 * P][:len(free)]
    new = np.zeros(seqs, np.int64)
    new[fits] = grow
    slots, err = torch.empty(int(new.sum()), dtype=torch.int64, device="cuda"), err_word()
    kv4.kv_tables_step(p.t, None, torch.tensor(new, dtype=torch.int32, device="cuda"), slots, device_error=err)
    opened = [i for i in fits if (keep[i] + grow + P - 1) // P > (keep[i] + P - 1) // P]
    now = p.t.block_table.cpu().numpy()
    assert [int(now[i, (keep[i] + P - 1) // P]) for i in opened] == free[:len(opened)]
    assert free_pages(p.t).tolist() == free[len(opened):]

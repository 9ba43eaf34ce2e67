"""The 4-bit cache as a serving loop uses it: prefixes admitted and written,
decode steps, rejected drafts and closed requests, through harness.Kv4Session;
every step's output against 64-bit attention over the quantised K and V (to the
bound of the arithmetic) and over the original ones (to what 4 bits cost)."""
import numpy as np
import pytest
import torch

from _kv4_common import P, assert_attention, attention, quantise, unpack
from paper_2603_12707_gb300 import workloads as wl

pytestmark = pytest.mark.gpu


def held(sess, layer):
    blocks = sess.pools[layer].data.cpu().numpy()
    return blocks, sess.tables.block_table.cpu().numpy()


@pytest.mark.parametrize("cfg,group", [
    (wl.CONFIGS["tiny"], 64),
    (wl.custom("kv4_gqa", 2, 28, 4, 128, 5, lens=[0, 17, 300, 64, 1], seed=11), 32),
    (wl.custom("kv4_mha", 1, 8, 8, 128, 3, lens=[5, 1000, 16], seed=12), 128),
])
def test_decode_steps(kvlib, cfg, group):
    from paper_2603_12707_gb300.harness import Kv4Session
    sess = Kv4Session(cfg, extra_tokens=8, group=group)
    sess.fill_prefix()
    rows = {(l, b): [[wl.kv_block(cfg, l, b, int(sess.lens0[b]), kind, "cuda").cpu()] for kind in "kv"]
            for l in range(cfg.phys_layers) for b in range(cfg.batch)}
    for step in range(3):
        sess.begin_step()
        for layer in range(cfg.phys_layers):
            q, kn, vn = wl.step_inputs(cfg, step, layer, "cuda")
            out = torch.empty_like(q)
            lse = torch.empty(q.shape[:2], device="cuda")
            sess.append(layer, kn, vn)
            sess.attend(layer, q, out, lse=lse)
            for b in range(cfg.batch):
                rows[(layer, b)][0].append(kn[b:b + 1].cpu())
                rows[(layer, b)][1].append(vn[b:b + 1].cpu())
            blocks, table = held(sess, layer)
            lens = [int(n) for n in sess.lens]
            ref = attention(blocks, table, lens, q.double().cpu().numpy(), group, torch.bfloat16, cfg.head_dim ** -0.5)
            assert_attention(out, lse, ref, torch.bfloat16, (cfg.name, step, layer))
            for b in range(cfg.batch):     # and the codes are those of the tokens written, in their order
                at = table[b, np.arange(lens[b]) // P]
                for side in (0, 1):
                    codes = unpack(blocks, cfg.head_dim, group, torch.bfloat16)[side][0][at, :, np.arange(lens[b]) % P]
                    assert (codes == quantise(torch.cat(rows[(layer, b)][side]), group)[0]).all()
    sess.check()


def test_drafts_are_taken_back_and_requests_closed(kvlib):
    from paper_2603_12707_gb300.harness import Kv4Session
    cfg = wl.custom("kv4_drafts", 1, 14, 2, 64, 4, lens=[15, 16, 200, 33], seed=3)
    sess = Kv4Session(cfg, extra_tokens=20, group=32)
    sess.fill_prefix()
    free = lambda: int(sess.tables.free_state[1])  # noqa: E731
    before, pages = free(), sess.tables.free_ring.numel()
    assert before == pages - sum((n + P - 1) // P for n in (15, 16, 200, 33))
    sess.grow([5, 5, 5, 5])                       # drafts
    sess.grow([-4, -5, -2, 0])                    # all but some rejected
    assert sess.tables.lens.tolist() == [16, 16, 203, 38]
    assert free() == pages - sum((n + P - 1) // P for n in (16, 16, 203, 38))
    sess.grow([-16, 0, -203, 0])                  # two closed
    assert sess.tables.lens.tolist() == [0, 16, 0, 38]
    assert free() == pages - sum((n + P - 1) // P for n in (0, 16, 0, 38))
    q, kn, vn = wl.step_inputs(cfg, 0, 0, "cuda")
    out = torch.empty_like(q)
    sess.attend(0, q, out)
    assert (out[[0, 2]] == 0).all() and torch.isfinite(out[[1]]).all()
    sess.check()


def test_a_full_pool_is_reported(kvlib):
    from paper_2603_12707_gb300.harness import Kv4Session
    cfg = wl.custom("kv4_full", 1, 8, 8, 64, 2, lens=[16, 16], seed=3)
    sess = Kv4Session(cfg, extra_tokens=32, group=64, slack_pages=0)
    sess.fill_prefix()
    sess.grow([16, 16])
    sess.check()
    sess.grow([0, -16])
    sess.grow([0, 16])
    sess.check()
    sess.tables.free_state[1] = 0
    sess.begin_step()
    with pytest.raises(RuntimeError, match="0x8"):
        sess.check()

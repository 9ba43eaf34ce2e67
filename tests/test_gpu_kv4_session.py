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


def held_rows(blocks, pages, n, side, d, group):
    """Values and steps of a request's n tokens, and the sizes of their middles, float64 [n, H, D]."""
    c, s, z = (x[np.arange(n) // P if pages is None else pages[np.arange(n) // P], :, np.arange(n) % P]
               for x in unpack(blocks, d, group, torch.bfloat16)[side])
    return s * (c - 8) + z, s, np.abs(z)


@pytest.mark.parametrize("cfg,group", [
    (wl.custom("kv4_near_gqa", 1, 28, 4, 128, 4, lens=[17, 300, 64, 1], seed=31), 32),
    (wl.custom("kv4_near_mha", 1, 8, 8, 128, 3, lens=[5, 1000, 16], seed=32), 128),
    (wl.custom("kv4_near_d64", 1, 14, 2, 64, 3, lens=[900, 33, 2], seed=33), 64),
])
def test_what_is_held_and_attended_is_near_what_was_written(kvlib, cfg, group):
    """Against the original K and V, not their codes.  A value is off by at most half a step and the roundings of s
    and z to the type: u = 2^-8 of each, 7.5 and 1 times.  Over tokens those errors are spread evenly: a score is off by a
    standard deviation of scale sqrt(sum_d q_d^2 s^2 / 12 + sum_groups (sum_d q_d)^2 (u z)^2 / 3), an output by
    sqrt(sum_t w^2 (s'^2 / 12 + (u z')^2 / 3 + score^2 (v - o)^2)); six of them, the change of weights to first order and a
    quarter more for the rest, and what the arithmetic and the output's type add (2^-8 of the output and 1 % of a step)."""
    from paper_2603_12707_gb300.harness import Kv4Session
    sess = Kv4Session(cfg, extra_tokens=4, group=group)
    sess.fill_prefix()
    sess.begin_step()
    q, kn, vn = wl.step_inputs(cfg, 0, 0, "cuda")
    out = torch.empty_like(q)
    sess.append(0, kn, vn)
    sess.attend(0, q, out)
    sess.check()
    blocks, table = held(sess, 0)
    d, hq, hkv = cfg.head_dim, cfg.num_q_heads, cfg.num_kv_heads
    qd, got, scale, u = q.double().cpu().numpy(), out.double().cpu().numpy(), d ** -0.5, 2.0 ** -8
    for b in range(cfg.batch):
        n = int(sess.lens[b])
        rows = []
        for side, (kind, new) in enumerate((("k", kn), ("v", vn))):
            x = torch.cat([wl.kv_block(cfg, 0, b, n - 1, kind, "cuda"), new[b:b + 1]]).double().cpu().numpy()
            y, s, z = held_rows(blocks, table[b], n, side, d, group)
            assert (np.abs(x - y) <= s * (0.5 + 7.5 * u) + z * u + 1e-30).all()
            rows.append((x, s, z))
        (k, sk, zk), (v, sv, zv) = rows
        for h in range(hq):
            g = h // (hq // hkv)
            x = k[:, g] @ qd[b, h] * scale
            w = np.exp(x - x.max())
            w /= w.sum()
            o = w @ v[:, g]
            sums = qd[b, h].reshape(-1, group).sum(-1)
            score = scale * np.sqrt((qd[b, h] ** 2 * sk[:, g] ** 2).sum(-1) / 12 + (sums ** 2 * (u * zk[:, g, ::group]) ** 2).sum(-1) / 3)
            dev = np.sqrt((w ** 2) @ (sv[:, g] ** 2 / 12 + (u * zv[:, g]) ** 2 / 3 + score[:, None] ** 2 * (v[:, g] - o) ** 2))
            lim = 6 * 1.25 * dev + u * np.abs(o) + 0.01 * sv[:, g].max()
            err = np.abs(got[b, h] - o)
            assert (err <= lim).all(), (b, h, float((err - lim).max()))

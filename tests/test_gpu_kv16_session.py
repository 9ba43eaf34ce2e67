"""Requests that share prefixes as a serving loop holds them: prefixes and own tokens admitted and written, decode steps
with norms, rotation and attention, requests closed, all through harness.SharedPrefixSession; written pages against rows rotated in
64 bits, every step's output against 64-bit attention over the pages."""
import pytest
import torch

from _kv16_common import P, UNIT, assert_attention, assert_rows, attention, inv_freq, pages_of, turned
from paper_2603_12707_gb300 import workloads as wl

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16
SLOW = 40_000_000      # cycles: some 20 ms, far longer than all calls here take


def held(sess, layer, request, n):
    """K and V [n, heads, d] of a request's first n tokens."""
    pool, table = sess.pools[layer], sess.tables.block_table[request].cpu().tolist()
    pages = torch.tensor(table[:pages_of(n)], device=pool.k.device)
    return [x[pages].transpose(1, 2).reshape(-1, *x.shape[1::2])[:n] for x in (pool.k, pool.v)]


@pytest.mark.parametrize("cfg,prefix_lens,prefix_of,dtype,normed", [
    (wl.custom("shared_image", 2, 28, 4, 128, 6, lens=[3, 0, 17, 40, 1, 100], seed=31), [600], [0] * 6, BF, True),
    (wl.custom("shared_groups", 1, 14, 2, 64, 9, lens=[5, 33, 16, 0, 8, 90, 1, 2, 64], seed=32), [130, 1, 0, 333], [0, 0, 3, 2, -1, 3, 3, 1, 3], FP, False),
    (wl.custom("shared_mha", 2, 8, 8, 128, 24, lens=list(range(24)), seed=33), [500, 20], [0] * 20 + [1, 1, -1, -1], BF, False),
])
def test_decode_steps(kvlib, cfg, prefix_lens, prefix_of, dtype, normed):
    from paper_2603_12707_gb300 import kv16
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    d, freq = cfg.head_dim, inv_freq(cfg.head_dim // 2)
    weights = [(1 + 0.2 * torch.randn(d, generator=torch.Generator().manual_seed(s))).to(dtype) for s in (1, 2)] if normed else [None] * 2
    qw, kw = (None if w is None else w.cuda() for w in weights)
    first = [prefix_lens[g] // 2 + 1 if g >= 0 else 0 for g in prefix_of]      # an image of fewer positions than tokens
    sess = SharedPrefixSession(cfg, prefix_lens, prefix_of, rope=kv16.Rope(freq), q_weight=qw, k_weight=kw, first_positions=first, dtype=dtype)
    sess.fill_prefix()
    sess.check()
    for layer in range(cfg.phys_layers):
        for r, n in enumerate(int(x) for x in sess.lens0):
            if n:
                k, v = (wl.kv_block(cfg, layer, r, n, kind, "cuda").cpu().to(dtype) for kind in "kv")
                base = first[r] if r < cfg.batch else 0
                got_k, got_v = held(sess, layer, r, n)
                assert_rows(got_k, turned(k, [[base + t for t in range(n)]], freq, None, weight=weights[1]), dtype, (layer, r))
                assert torch.equal(got_v.cpu(), v)
    for step in range(3):
        sess.begin_step()
        lens = [int(n) for n in sess.lens]
        at = [[first[b] + lens[b] - 1 for b in range(cfg.batch)]]
        for layer in range(cfg.phys_layers):
            q, k, v = (x.to(dtype) for x in wl.step_inputs(cfg, step, layer, "cuda"))
            qr, out, lse = torch.empty_like(q), torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
            sess.append(layer, q, k, v, qr)
            sess.attend(layer, qr, out, lse=lse)
            sess.check()
            assert_rows(qr, turned(q.cpu(), at, freq, None, weight=weights[0]), dtype, (step, layer))
            new = [torch.stack([held(sess, layer, b, lens[b])[i][-1] for b in range(cfg.batch)]) for i in range(2)]
            assert_rows(new[0], turned(k.cpu(), at, freq, None, weight=weights[1]), dtype, (step, layer))
            assert torch.equal(new[1], v)
            pool = sess.pools[layer]
            ref = attention(pool.k, pool.v, sess.tables.block_table.cpu().numpy(), lens, None,
                            [cfg.batch + g if g >= 0 else -1 for g in prefix_of], qr, d ** -0.5, dtype)
            assert_attention(out, lse, ref, dtype, (step, layer))
    assert sess.tables.lens.tolist() == [int(n) for n in sess.lens]


def test_shared_and_own_prefixes_answer_alike(kvlib):
    """Requests that share a prefix, and the same requests with a copy of it each."""
    from paper_2603_12707_gb300 import kv16
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    batch, n, own = 5, 300, [7, 0, 64, 16, 30]
    cfg = wl.custom("shared", 1, 8, 2, 64, batch, lens=own, seed=5)
    rope = kv16.Rope(inv_freq(32))
    shared = SharedPrefixSession(cfg, [n], [0] * batch, rope=rope)
    alone = SharedPrefixSession(cfg, [], [-1] * batch, rope=rope, lens=[n + x for x in own])
    pk, pv = (wl.kv_block(cfg, 0, 99, n, kind, "cuda") for kind in "kv")
    tails = [[wl.kv_block(cfg, 0, b, x, kind, "cuda") for b, x in enumerate(own)] for kind in "kv"]
    slots, pos = shared.grow(own + [n])
    shared.write(0, slots, pos, *(torch.cat(t + [p]) for t, p in zip(tails, (pk, pv))))
    slots, pos = alone.grow([n + x for x in own])
    alone.write(0, slots, pos, *(torch.cat([y for x in t for y in (p, x)]) for t, p in zip(tails, (pk, pv))))
    for step in range(2):
        q, k, v = wl.step_inputs(cfg, step, 0, "cuda")
        outs = []
        for sess in (shared, alone):
            qr, out = torch.empty_like(q), torch.empty_like(q)
            sess.begin_step()
            sess.append(0, q, k, v, qr)
            sess.attend(0, qr, out)
            sess.check()
            outs.append((qr, out.double()))
        assert torch.equal(outs[0][0], outs[1][0])
        # Each is within UNIT |out| + 2 UNIT max|v| (weights rounded to bf16; 32-bit terms are far below) of the exact output.
        vmax = float(torch.cat([pv] + tails[1] + [v]).abs().max())
        lim = 2 * UNIT[BF] * (outs[0][1].abs().clamp(min=outs[1][1].abs()) + 2 * vmax)
        assert ((outs[0][1] - outs[1][1]).abs() <= lim).all()


def test_prefixes_are_dropped_and_taken_up_again(kvlib):
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    cfg = wl.custom("shared_drop", 1, 4, 4, 64, 3, lens=[10, 20, 30], seed=6)
    sess = SharedPrefixSession(cfg, [100, 40], [0, 1, 0], slack_pages=0)
    free = lambda: int(sess.tables.free_state[1])  # noqa: E731
    pages = sess.tables.free_ring.numel()
    sess.fill_prefix()
    assert free() == pages - sum(pages_of(n) for n in (10, 20, 30, 100, 40))
    sess.grow([0, -20, 0, 0, -40])                   # one request and its prefix closed
    assert free() == pages - sum(pages_of(n) for n in (10, 30, 100))
    slots, pos = sess.grow([0, 5, 0, 0, 33])         # others in their place
    assert pos.tolist() == [40 + t for t in range(5)] + list(range(33))
    k, v = (torch.randn((38, 4, 64), device="cuda").to(BF) for _ in range(2))
    sess.write(0, slots, pos, k, v)
    sess.begin_step()
    q, kn, vn = wl.step_inputs(cfg, 0, 0, "cuda")
    out = torch.empty_like(q)
    sess.append(0, q, kn, vn, q)
    sess.attend(0, q, out)
    sess.check()
    pool = sess.pools[0]
    ref = attention(pool.k, pool.v, sess.tables.block_table.cpu().numpy(), [11, 6, 31, 100, 33], None, [3, 4, 3], q, 64 ** -0.5, BF)
    assert_attention(out, None, ref, BF)
    sess.grow([-11, -6, -31, -100, -33])
    assert free() == pages and sess.tables.lens.tolist() == [0] * 5


@pytest.mark.parametrize("kind", ["stream", "handle", "default"])
def test_a_session_on_its_own_stream(kvlib, kind):
    """Beside slow work on torch's current stream and late work in memory that the allocator has to spare."""
    from paper_2603_12707_gb300 import kv16
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    cfg = wl.custom("shared_side", 2, 8, 2, 128, 6, lens=[40, 0, 333, 16, 1, 70], seed=21)

    def run(stream, beside):
        beside()
        sess = SharedPrefixSession(cfg, [700, 9], [0, 0, 1, 0, -1, 0], rope=kv16.Rope(inv_freq(64)), stream=stream)
        beside()
        sess.fill_prefix()
        on = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
        outs = []
        for step in range(3):
            beside()
            sess.begin_step()
            for layer in range(cfg.phys_layers):
                with torch.cuda.stream(on):
                    q, k, v = wl.step_inputs(cfg, step, layer, "cuda")
                    out = torch.empty_like(q)
                sess.append(layer, q, k, v, q)
                sess.attend(layer, q, out)
                outs.append(out)
        sess.check()
        return [o.cpu() for o in outs]

    def junk_and_wait():
        torch.cuda._sleep(SLOW)
        for n in (64, 4096, 1 << 16, 1 << 20):
            torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda")

    want = run(None, lambda: None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    if kind == "default":
        with torch.cuda.stream(side):
            got = run(None, junk_and_wait)
    else:
        got = run(side if kind == "stream" else side.cuda_stream, junk_and_wait)
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))


def test_what_a_session_refuses(kvlib):
    from paper_2603_12707_gb300.harness import SharedPrefixSession
    cfg = wl.custom("shared_bad", 1, 4, 4, 64, 3, lens=[1, 2, 3], seed=6)
    for kw in (dict(prefix_of=[0, 0]), dict(prefix_of=[0, 1, 0]), dict(prefix_of=[0, -2, 0]), dict(prefix_of=[0] * 3, first_positions=[1]),
               dict(prefix_of=[0] * 3, lens=[1, 2])):
        with pytest.raises(ValueError):
            SharedPrefixSession(cfg, [10], **kw)
    sess = SharedPrefixSession(cfg, [16], [0] * 3, extra_tokens=0, slack_pages=0)
    sess.fill_prefix()
    sess.grow([-1, 0, 0, 0])
    sess.grow([1, 14, 13, 0])
    sess.begin_step()                                # its table row is full (the documented bit: 4)
    with pytest.raises(RuntimeError, match="0x4"):
        sess.check()

"""A 4-bit session on a stream of its own, beside slow work on torch's current stream and on its own."""
import pytest
import torch

from paper_2603_12707_gb300 import workloads as wl

pytestmark = pytest.mark.gpu

SLOW = 40_000_000      # cycles: some 20 ms, far longer than all calls here take


def run(Session, cfg, stream, beside):
    """Outputs of three decode steps; `beside`: called before every step of the session's own work."""
    beside()
    sess = Session(cfg, extra_tokens=8, group=64, stream=stream)
    beside()
    sess.fill_prefix()
    outs = []
    on = stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(stream) if stream else torch.cuda.default_stream()
    for step in range(3):
        beside()
        sess.begin_step()
        for layer in range(cfg.phys_layers):
            with torch.cuda.stream(on):      # the caller's tensors are ready on the session's stream
                q, k, v = wl.step_inputs(cfg, step, layer, "cuda")
                out = torch.empty_like(q)
            sess.append(layer, k, v)
            sess.attend(layer, q, out)
            outs.append(out)
    beside()
    sess.grow([-2] * cfg.batch)
    sess.check()
    return sess, [o.cpu() for o in outs]


def junk_and_wait():
    """Late work on the current stream, in memory that the allocator has to spare."""
    torch.cuda._sleep(SLOW)
    for n in (64, 4096, 1 << 16, 1 << 20):
        torch.full((n,), 0x7F, dtype=torch.uint8, device="cuda")


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_a_session_on_its_own_stream(kvlib, kind):
    from paper_2603_12707_gb300.harness import Kv4Session
    cfg = wl.custom("kv4_side", 2, 8, 2, 128, 6, lens=[40, 0, 333, 16, 1, 700], seed=21)
    _, want = run(Kv4Session, cfg, None, lambda: None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    sess, got = run(Kv4Session, cfg, side if kind == "stream" else side.cuda_stream, junk_and_wait)
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    side.synchronize()
    assert sess.tables.lens.tolist() == [int(n) for n in sess.lens]


def test_check_waits_for_the_session(kvlib):
    """The error bit of a step behind slow work on the session's stream is seen."""
    from paper_2603_12707_gb300.harness import Kv4Session
    side = torch.cuda.Stream()
    cfg = wl.custom("kv4_side_full", 1, 8, 8, 64, 2, lens=[16, 16], seed=3)
    sess = Kv4Session(cfg, extra_tokens=32, group=64, slack_pages=0, stream=side)
    sess.fill_prefix()
    sess.check()
    with torch.cuda.stream(side):
        sess.tables.free_state[1] = 0          # no page is left
        torch.cuda._sleep(SLOW)
    sess.begin_step()
    with pytest.raises(RuntimeError, match="0x8"):
        sess.check()


def test_a_default_session_inside_another_current_stream(kvlib):
    """stream=None is the default stream for all that the session does, also where another stream is current."""
    from paper_2603_12707_gb300.harness import Kv4Session
    cfg = wl.custom("kv4_inside", 1, 8, 2, 128, 3, lens=[40, 100, 7], seed=5)
    _, want = run(Kv4Session, cfg, None, lambda: None)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        _, got = run(Kv4Session, cfg, None, junk_and_wait)
    for a, b in zip(want, got):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))

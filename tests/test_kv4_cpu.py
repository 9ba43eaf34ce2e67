"""CPU checks of the 4-bit cache's entry points: every function of kvdecode4.h
is exported and refuses what it says it refuses before anything is enqueued."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "kvdecode4.h")

INVALID, UNSUPPORTED = -1, -5


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def pool(kv4, **kw):
    f = dict(data=128, num_pages=8, num_kv_heads=4, head_dim=128, group=64, dtype=0)
    return kv4.kv4_pool(**{**f, **kw})


def tables(kv4, **kw):
    f = dict(block_table=16, lens=16, free_ring=16, free_state=16, num_pages=8, max_seqs=4, max_pages=3)
    return kv4.kv_tables(**{**f, **kw})


def test_header_and_library_agree(kv4, kvlib):
    names = re.findall(r"^KVC_API\s+(?:int|int64_t)\s+(\w+)\(", open(HEADER).read(), flags=re.M)
    assert sorted(names) == sorted(kv4._SIGS)
    for n in names:
        assert hasattr(kvlib.load(), n)


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=96), UNSUPPORTED), (dict(group=16), UNSUPPORTED), (dict(head_dim=64, group=128), UNSUPPORTED),
    (dict(dtype=2), INVALID), (dict(num_kv_heads=0), INVALID), (dict(num_kv_heads=1025), INVALID),
    (dict(num_pages=0), INVALID), (dict(num_pages=2 ** 31), INVALID),
])
def test_pools_that_are_refused(kv4, kvlib, kw, code):
    p = pool(kv4, **kw)
    fns = kv4._load()
    ref = ctypes.addressof(p)
    assert fns["kv4_pool_bytes"](ref) == code
    assert kvlib.load().kv_last_error().decode().startswith("kv4_pool: ")
    assert fns["kv4_write"](ref, 1, 16, 16, 512, 16, 512, None, None) == code
    assert fns["kv4_read"](ref, 1, 16, 16, 512, 16, 512, None, None) == code
    assert fns["kv4_workspace_bytes"](ref, 4) == code


@pytest.mark.parametrize("d,group,block", [(64, 32, 1280), (64, 64, 1152), (128, 32, 2560), (128, 64, 2304), (128, 128, 2176)])
def test_pool_bytes(kv4, d, group, block):
    p = pool(kv4, head_dim=d, group=group, num_pages=2 ** 31 - 1, num_kv_heads=5)
    assert kv4._load()["kv4_pool_bytes"](ctypes.addressof(p)) == (2 ** 31 - 1) * 5 * block
    assert kv4.Pool.block_bytes(d, group) == block


def test_rows_that_are_refused(kv4):
    p = pool(kv4)
    ref = ctypes.addressof(p)

    def call(fn="kv4_write", ref=ref, n=2, slots=16, k=16, ks=512, v=16, vs=512):
        return kv4._load()[fn](ref, n, slots, k, ks, v, vs, None, None)

    for fn in ("kv4_write", "kv4_read"):
        assert call(fn, ref=None) == INVALID
        assert call(fn, n=-1) == INVALID
        assert call(fn, slots=None) == INVALID and call(fn, k=None) == INVALID and call(fn, v=None) == INVALID
        assert call(fn, k=8) == INVALID and call(fn, v=18) == INVALID and call(fn, slots=12) == INVALID
        assert call(fn, ks=516) == INVALID and call(fn, vs=514) == INVALID
        assert call(fn, ks=-512) == INVALID
        assert call(fn, n=0, slots=None, k=None, v=None) == 0          # nothing to do
        assert call(fn, ref=ctypes.addressof(pool(kv4, data=64))) == INVALID
        assert call(fn, ref=ctypes.addressof(pool(kv4, data=None))) == INVALID
    assert call("kv4_read", ks=504) == INVALID                         # output rows that overlap


def test_attention_calls_that_are_refused(kv4):
    good_pool, good_tables = pool(kv4), tables(kv4)

    def call(p=good_pool, t=good_tables, batch=2, ids=None, hq=8, q=16, qs=1024, out=16, os=1024, scale=0.0, ws=256,
             wb=1 << 40):
        ref = lambda x: ctypes.addressof(x) if x is not None else None  # noqa: E731
        return kv4._load()["kv4_decode_attention"](ref(p), ref(t), batch, ids, hq, q, qs, out, os, None, scale, ws, wb,
                                                   None, None)

    assert call(p=None) == INVALID and call(t=None) == INVALID
    assert call(batch=0) == INVALID and call(batch=4097, ids=16) == INVALID
    assert call(batch=5) == INVALID                                    # rows without a request
    assert call(hq=6) == INVALID and call(hq=0) == INVALID
    assert call(hq=36) == UNSUPPORTED                                  # 9 query heads per KV head
    assert call(q=None) == INVALID and call(out=None) == INVALID and call(ws=None) == INVALID
    assert call(q=8) == INVALID and call(qs=1028) == INVALID and call(os=1016) == INVALID and call(qs=-1024) == INVALID
    assert call(scale=float("nan")) == INVALID and call(scale=float("inf")) == INVALID
    assert call(ws=128) == INVALID and call(wb=0) == INVALID
    for kw in (dict(block_table=None), dict(lens=None), dict(max_seqs=0), dict(max_pages=0),
               dict(max_seqs=2 ** 16, max_pages=2 ** 15), dict(max_seqs=1, max_pages=2 ** 27)):
        assert call(t=tables(kv4, **kw), batch=1) == INVALID


def test_table_steps_that_are_refused(kv4):
    good = tables(kv4)

    def call(t=good, batch=2, ids=None, new=16, room=4, slots=16):
        return kv4._load()["kv_tables_step"](ctypes.addressof(t), batch, ids, new, room, slots, None, None, None, None,
                                             None, None)

    assert call(new=None) == INVALID and call(slots=None) == INVALID and call(room=-1) == INVALID
    assert call(batch=0) == INVALID and call(batch=5) == INVALID and call(batch=4097, ids=16) == INVALID
    for kw in (dict(free_ring=None), dict(free_state=None), dict(num_pages=0), dict(num_pages=2 ** 31)):
        assert call(t=tables(kv4, **kw)) == INVALID


def test_softmax_scales_that_overflow_are_refused(kv4):
    """Scores are held in a unit of 2^-21: a scale that is no number there made every output NaN."""
    ref = ctypes.addressof
    p, t = pool(kv4), tables(kv4)

    def call(scale):
        return kv4._load()["kv4_decode_attention"](ref(p), ref(t), 2, None, 8, 16, 1024, 16, 1024, None, scale, 256, 0, None, None)

    for scale in (2.0 ** 100, 1e33, 3e38, float("inf"), float("nan")):
        assert call(scale) == INVALID and "softmax_scale" in kv4.kd.load().kv_last_error().decode()
    for scale in (2.0 ** 99, 0.0, -1.0, float("-inf")):    # refused for its workspace, after the scale
        assert call(scale) == INVALID and "workspace" in kv4.kd.load().kv_last_error().decode()

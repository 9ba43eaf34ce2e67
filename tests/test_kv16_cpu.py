"""CPU checks of the 16-bit serving step's entry points: every function of kvdecode16.h is exported and refuses what it
says it refuses before anything is enqueued."""
import ctypes
import math
import os
import re

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "kvdecode16.h")

INVALID, UNSUPPORTED = -1, -5


@pytest.fixture(scope="module")
def kv16(kvlib):
    from paper_2603_12707_gb300 import kv16
    return kv16


@pytest.fixture(scope="module")
def kv4(kvlib):
    from paper_2603_12707_gb300 import kv4
    return kv4


def pool(kv16, **kw):
    f = dict(k=16, v=16, num_pages=8, num_kv_heads=4, head_dim=128, dtype=0)
    return kv16.kv16_pool(**{**f, **kw})


def rope(kv16, **kw):
    f = dict(frequencies=8, axes=None, rotary_dim=128, num_axes=3, neighbours=0, scale=1.0)
    return kv16.kv_rope(**{**f, **kw})


def tables(kv4, **kw):
    f = dict(block_table=16, lens=16, free_ring=16, free_state=16, num_pages=8, max_seqs=4, max_pages=3)
    return kv4.kv_tables(**{**f, **kw})


def ref(x):
    return None if x is None else ctypes.addressof(x)


def test_header_and_library_agree(kv16, kvlib):
    names = re.findall(r"^KVC_API\s+(?:int|int64_t)\s+(\w+)\(", open(HEADER).read(), flags=re.M)
    assert sorted(names) == sorted(kv16._SIGS)
    for n in names:
        assert hasattr(kvlib.load(), n)


POOLS = [(dict(head_dim=96), UNSUPPORTED), (dict(dtype=2), INVALID), (dict(num_kv_heads=0), INVALID), (dict(num_kv_heads=1025), INVALID),
         (dict(num_pages=0), INVALID), (dict(num_pages=2 ** 25), INVALID), (dict(num_pages=2 ** 62), INVALID)]


def write(kv16, p, r=None, n=2, slots=16, pos=16, axis=2, hq=8, q=16, qs=1024, qo=16, qos=1024, k=16, ks=512, v=16, vs=512, qw=None,
          kw=None, eps=1e-6):
    return kv16._load()["kv16_write"](ref(p), ref(r), n, slots, pos, axis, hq, q, qs, qo, qos, k, ks, v, vs, qw, kw, eps, None, None)


def turn(kv16, r=None, dtype=0, d=128, n=2, pos=16, axis=2, hq=8, q=16, qs=1024, qo=16, qos=1024, hkv=4, k=16, ks=512, ko=16, kos=512,
         qw=None, kw=None, eps=1e-6):
    return kv16._load()["kv_qk_rope"](ref(r), dtype, d, n, pos, axis, hq, q, qs, qo, qos, hkv, k, ks, ko, kos, qw, kw, eps, None)


def plan(kv16, p, t, hq=8, batch=2, ids=None, pre=None, ws=256, wb=0):
    return kv16._load()["kv16_plan"](ref(p), ref(t), hq, batch, ids, pre, ws, wb, None, None)


def attend(kv16, p, t, batch=2, hq=8, q=16, qs=1024, out=16, os=1024, lse=None, scale=0.0, ws=256, wb=0):
    return kv16._load()["kv16_attention"](ref(p), ref(t), batch, hq, q, qs, out, os, lse, scale, ws, wb, None, None)


@pytest.mark.parametrize("kw,code", POOLS)
def test_pools_that_are_refused(kv16, kv4, kvlib, kw, code):
    p, t = pool(kv16, **kw), tables(kv4)
    for rc in (write(kv16, p), plan(kv16, p, t), attend(kv16, p, t), kv16._load()["kv16_workspace_bytes"](ref(p), 8, 2)):
        assert rc == code
        assert kvlib.load().kv_last_error().decode().startswith("kv16_pool: ")


@pytest.mark.parametrize("kw", [dict(frequencies=None), dict(frequencies=4), dict(rotary_dim=0), dict(rotary_dim=8), dict(rotary_dim=24),
                                dict(rotary_dim=144), dict(num_axes=0), dict(num_axes=9), dict(neighbours=2), dict(scale=math.inf),
                                dict(scale=math.nan)])
def test_rotations_that_are_refused(kv16, kvlib, kw):
    r = rope(kv16, **kw)
    assert turn(kv16, r) == INVALID and "kv_rope" in kvlib.load().kv_last_error().decode()
    assert write(kv16, pool(kv16), r) == INVALID


def test_rows_that_are_refused(kv16):
    r, p = rope(kv16), pool(kv16)
    for call in (lambda **kw: turn(kv16, r, **kw), lambda **kw: write(kv16, p, r, **kw)):
        assert call(n=-1) == INVALID and call(pos=None) == INVALID and call(pos=18) == INVALID and call(axis=-1) == INVALID
        assert call(hq=-1) == INVALID and call(hq=8193) == INVALID
        assert call(q=None) == INVALID and call(q=8) == INVALID and call(qs=1028) == INVALID and call(qs=-8) == INVALID
        assert call(qo=None) == INVALID and call(qo=24) == INVALID and call(qos=1016) == INVALID     # rows that overlap
        assert call(k=None) == INVALID and call(k=8) == INVALID and call(ks=516) == INVALID and call(ks=-512) == INVALID
        assert call(qw=8) == INVALID and call(kw=24) == INVALID
        for eps in (0.0, -1.0, math.nan, math.inf, 2.0 ** -101):
            assert call(qw=16, eps=eps) == INVALID
        assert call(n=0, q=None, qo=None, k=None, pos=None) == 0                                     # nothing to do
    assert turn(kv16, r, d=96) == UNSUPPORTED and turn(kv16, r, dtype=3) == INVALID
    assert turn(kv16, rope(kv16, rotary_dim=128), d=64) == INVALID
    assert turn(kv16, r, hkv=-1) == INVALID and turn(kv16, r, hkv=1025) == INVALID
    assert turn(kv16, r, ko=None) == INVALID and turn(kv16, r, kos=504) == INVALID
    assert turn(kv16, r, hq=0, hkv=0, q=None, k=None) == 0
    assert write(kv16, p, r, slots=None) == INVALID and write(kv16, p, r, slots=12) == INVALID
    assert write(kv16, p, r, v=None) == INVALID and write(kv16, p, r, vs=508) == INVALID
    for kw in (dict(k=None), dict(v=None), dict(k=8), dict(v=40)):
        assert write(kv16, pool(kv16, **kw), r) == INVALID


def test_plans_that_are_refused(kv16, kv4):
    p, t = pool(kv16), tables(kv4)
    assert plan(kv16, None, t) == INVALID and plan(kv16, p, None) == INVALID
    assert plan(kv16, p, t, batch=0) == INVALID and plan(kv16, p, t, batch=4097, ids=16) == INVALID
    assert plan(kv16, p, t, batch=5) == INVALID                                  # rows without a request
    assert plan(kv16, p, t, hq=6) == INVALID and plan(kv16, p, t, hq=0) == INVALID and plan(kv16, p, t, hq=36) == UNSUPPORTED
    assert plan(kv16, p, t, ids=18) == INVALID and plan(kv16, p, t, pre=18) == INVALID
    assert plan(kv16, p, t, ws=None) == INVALID and plan(kv16, p, t, ws=128) == INVALID
    for kw in (dict(block_table=None), dict(lens=None), dict(max_seqs=0), dict(max_pages=0), dict(max_seqs=1, max_pages=2 ** 27)):
        assert plan(kv16, p, tables(kv4, **kw), batch=1) == INVALID and attend(kv16, p, tables(kv4, **kw), batch=1) == INVALID
    fn = kv16._load()["kv16_workspace_bytes"]
    assert fn(ref(p), 8, 0) == INVALID and fn(ref(p), 8, 4097) == INVALID and fn(ref(p), 6, 1) == INVALID and fn(ref(p), 36, 1) == UNSUPPORTED


def test_attention_calls_that_are_refused(kv16, kv4, kvlib):
    p, t = pool(kv16), tables(kv4)

    def call(**kw):
        return attend(kv16, p, t, **kw)

    assert attend(kv16, None, t) == INVALID and attend(kv16, p, None) == INVALID
    assert call(batch=0) == INVALID and call(batch=4097) == INVALID and call(hq=6) == INVALID and call(hq=36) == UNSUPPORTED
    assert call(q=None) == INVALID and call(q=8) == INVALID and call(qs=1028) == INVALID and call(qs=-1024) == INVALID
    assert call(out=None) == INVALID and call(out=24) == INVALID and call(os=1016) == INVALID
    assert call(lse=18) == INVALID
    for scale in (2.0 ** 100, math.inf, math.nan):
        assert call(scale=scale) == INVALID and "softmax_scale" in kvlib.load().kv_last_error().decode()
    for scale in (2.0 ** 99, 0.0, -1.0, -math.inf):     # refused for its workspace, after the scale
        assert call(scale=scale, ws=128) == INVALID and "workspace" in kvlib.load().kv_last_error().decode()
    assert call(ws=None) == INVALID
    for kw in (dict(k=None), dict(v=None), dict(k=8), dict(v=40)):
        assert attend(kv16, pool(kv16, **kw), t) == INVALID


def test_frequencies_are_turns_to_the_last_bit(kv16):
    r = kv16.Rope([1.0, 0.5, math.pi, -1.0, 0.0], device="cpu")
    got = [int(x) % 2 ** 64 for x in r.frequencies]
    assert abs(got[0] / 2 ** 64 - 1 / (2 * math.pi)) < 2e-16 and got[0] - 2 * got[1] in (-1, 0, 1)
    assert abs(got[2] - 2 ** 63) < 2 ** 13 and got[3] == 2 ** 64 - got[0] and got[4] == 0
    assert r.rotary_dim == 10


@pytest.mark.parametrize("kw", [dict(inv_freq=[math.inf]), dict(inv_freq=[1.0] * 8, axes=[0] * 7), dict(inv_freq=[1.0] * 2, axes=[0, 1]),
                                dict(inv_freq=[1.0] * 2, axes=[0, -1], num_axes=2)])
def test_rope_descriptions_that_are_refused(kv16, kw):
    with pytest.raises(ValueError):
        kv16.Rope(device="cpu", **kw)


def test_tensors_that_are_refused(kv16):
    x = torch.zeros((2, 3, 16, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        kv16.Pool(x, x)                      # not on a GPU
    with pytest.raises(ValueError):
        kv16.Pool(x.float(), x.float())
    with pytest.raises(ValueError):
        kv16.kv_qk_rope(None, None, None, None, None, None)

"""The plan of a 16-bit serving step, by the kernel's own source on host threads: whatever warps run ahead of others between two barriers
of a CTA, all CTAs' parts belong to one plan."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from _kv16_plan import check_plan, parts

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2603_12707_gb300", "csrc")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    """plan(lens, seq_ids, prefix_ids, hq, hkv, dim, dawdle) -> the workspace's bytes, the error word."""
    d = tmp_path_factory.mktemp("plan")
    text = "".join(open(os.path.join(CSRC, f)).read().split("using namespace kvd;")[0] for f in ("kvd_kv16_plan.h", "kvd_kv16_plan.cu"))
    text = re.sub(r'^#include "[^"]*"$|^#pragma once$', "", text, flags=re.M)
    text, n = re.subn(r"extern __shared__ int64_t shared\[\];", "int64_t* const shared = shared_memory;", text)
    assert n == 1
    source, lib = str(d / "plan.inc"), str(d / "plan.so")
    open(source, "w").write(text)
    subprocess.run(["g++", "-std=c++17", "-O1", "-pthread", "-shared", "-fPIC", "-I", os.path.join(os.path.dirname(HERE), "include"),
                    f'-DPLAN_SOURCE="{source}"', os.path.join(HERE, "_plan_on_threads.cpp"), "-o", lib], check=True)
    fn = ctypes.CDLL(lib).plan
    fn.restype = ctypes.c_int64
    fn.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int] * 9 + [ctypes.c_void_p] * 3

    def call(lens, seq_ids, prefix_ids, hq, hkv, dim, dawdle, grid=152):
        batch = len(prefix_ids)
        threads = 64 if batch <= 64 else 128 if batch <= 128 else 256 if batch <= 256 else 512
        lens, seq_ids, prefix_ids, dawdle = (np.ascontiguousarray(x, np.int32) for x in (lens, seq_ids, prefix_ids, dawdle))
        args = [x.ctypes.data for x in (lens, seq_ids, prefix_ids)]
        shape = (len(lens), 1 << 20, batch, hq, hkv, dim, grid, threads, len(dawdle))
        room = fn(*args, *shape, dawdle.ctypes.data, None, None)
        workspace, err = np.zeros(room, np.uint8), np.zeros(1, np.int32)
        fn(*args, *shape, dawdle.ctypes.data, workspace.ctypes.data, err.ctypes.data)
        return workspace.tobytes(), int(err[0])

    return call


# (own lengths, prefix lengths, prefix of each row, query heads, KV heads, head_dim)
BATCHES = {
    "one_prefix_96_rows": ([1 + 3 * i for i in range(96)], [131009], [0] * 96, 28, 4, 128),
    "one_prefix_behind_others": ([7] * 90, [300, 20000], [-1] * 5 + [0] * 2 + [1] * 80 + [-1] * 3, 28, 4, 128),
    "one_prefix_few_tokens": ([0] * 300, [50], [0] * 300, 8, 8, 64),
    "two_prefixes_48_rows": ([200] * 96, [60000, 60000], [0] * 48 + [1] * 48, 28, 4, 128),
    "groups": ([(37 * i) % 700 for i in range(150)], [1, 9000, 40, 333, 4000, 16, 17, 2500, 801, 5, 6000],
               [min(i // 12, 10) for i in range(133)] + [-1] * 17, 14, 2, 64),
    "four_rows": ([0, 64, 1, 9], [1369], [0] * 4, 28, 4, 128),
    "alone": ([5, 0, 1000, 16, 1], [], [-1] * 5, 32, 32, 128),
    "more_rows_than_threads": ([i % 40 for i in range(1200)], [700, 1, 90], [0] * 500 + [1] * 2 + [2] * 600 + [-1] * 98, 8, 1, 128),
}


@pytest.mark.parametrize("dawdle", [[0, 0, 0, 0], [2, 1, 1, 1], [1, 2, 2, 2], [2, 2, 1, 0]])
@pytest.mark.parametrize("name", sorted(BATCHES))
def test_all_ctas_write_one_plan(plan, name, dawdle):
    """CTA 0 writes the header, 1 and 2 the runs and records, all of them starts and sources; in each nobody, all warps but the first
    or the first comes late from every barrier."""
    own, prefix_lens, prefix_of, hq, hkv, dim = BATCHES[name]
    batch = len(own)
    ids = [batch + g if g >= 0 else -1 for g in prefix_of]
    workspace, err = plan(own + prefix_lens, range(batch), ids, hq, hkv, dim, dawdle)
    assert err == 0
    if name == "one_prefix_96_rows":     # three chunks of four KV heads: the same number of CTAs for each
        assert int(parts(workspace, batch, hkv, 152)[0][0]["prefix_ctas"]) % 12 == 0
    check_plan(workspace, own + prefix_lens, list(range(batch)), ids, hq, hkv, dim, 152)

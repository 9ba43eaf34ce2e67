"""ctypes binding of the 16-bit serving step (declared in include/kvdecode16.h).

Argument marshalling only, as in ``kv4``: functions keep the C names, ``Pool``
and ``Rope`` hold the caller's tensors together with the C structs that describe
them, block tables are ``kv4.Tables``.  Tensors passed to a call are checked
here, since the kernels read through the raw pointers.  ``stream`` accepts a
``torch.cuda.Stream``, a raw handle or None (the legacy default stream); tensors
are on the device that is current.
"""
from __future__ import annotations

import ctypes
import math

import torch

from . import kvdecode as kd
from .kv4 import _DTYPES, PAGE_SIZE, Tables, _vector

KVC_DEVERR_PLAN = 16

_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64
_F = ctypes.c_float


class kv16_pool(ctypes.Structure):
    _fields_ = [("k", _P), ("v", _P), ("num_pages", _I64), ("num_kv_heads", _I32), ("head_dim", _I32), ("dtype", _I32)]


class kv_rope(ctypes.Structure):
    _fields_ = [("frequencies", _P), ("axes", _P), ("rotary_dim", _I32), ("num_axes", _I32), ("neighbours", _I32),
                ("scale", _F)]


_SIGS = {
    "kv_qk_rope": ([_P, _I32, _I32, _I32, _P, _I64, _I32, _P, _I64, _P, _I64, _I32, _P, _I64, _P, _I64, _P, _P, _F, _P], _I32),
    "kv16_write": ([_P, _P, _I32, _P, _P, _I64, _I32, _P, _I64, _P, _I64, _P, _I64, _P, _I64, _P, _P, _F, _P, _P], _I32),
    "kv16_workspace_bytes": ([_P, _I32, _I32], _I64),
    "kv16_plan": ([_P, _P, _I32, _I32, _P, _P, _P, _I64, _P, _P], _I32),
    "kv16_attention": ([_P, _P, _I32, _I32, _P, _I64, _P, _I64, _P, _F, _P, _I64, _P, _P], _I32),
}
_fns = None


def _load():
    """The library's functions of this part (kvdecode.load() raises if the library is missing)."""
    global _fns
    if _fns is None:
        lib = kd.load()
        fns = {}
        for name, (args, res) in _SIGS.items():
            fn = getattr(lib, name)
            fn.argtypes = args
            fn.restype = res
            fns[name] = fn
        _fns = fns
    return _fns


class Pool:
    """One layer's pool: ``k`` and ``v`` [num_pages][num_kv_heads][16][head_dim], bfloat16 or float16."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor):
        if k.dtype not in _DTYPES:
            raise ValueError("k must be of torch.bfloat16 or torch.float16")
        for name, x in (("k", k), ("v", v)):
            if x.dtype is not k.dtype or not x.is_cuda or not x.is_contiguous() or x.dim() != 4 or x.shape[2] != PAGE_SIZE:
                raise ValueError(f"{name} must be a contiguous CUDA tensor [num_pages][num_kv_heads][{PAGE_SIZE}][head_dim] of {k.dtype}")
        if k.shape != v.shape or k.device != v.device:
            raise ValueError("k and v must have the same shape and device")
        self.k, self.v, self.dtype = k, v, k.dtype
        self.num_kv_heads, self.head_dim = k.shape[1], k.shape[3]
        self.c = kv16_pool(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[1], k.shape[3], _DTYPES[k.dtype])
        self.ref = ctypes.addressof(self.c)

    @classmethod
    def empty(cls, num_pages: int, num_kv_heads: int, head_dim: int, dtype: torch.dtype = torch.bfloat16, device="cuda"):
        """A pool of its own memory, zero-filled."""
        return cls(*(torch.zeros((num_pages, num_kv_heads, PAGE_SIZE, head_dim), dtype=dtype, device=device) for _ in range(2)))


class Rope:
    """A rotation: pair j of a head's first ``2 * len(inv_freq)`` elements is turned by ``position * inv_freq[j]``
    radians, the position being that of axis ``axes[j]`` (None: 0).  Pairs are (j, j + len(inv_freq)), or neighbours
    (2 j, 2 j + 1).  Frequencies are numbers of 64 bits; ``scale`` multiplies cosines and sines."""

    def __init__(self, inv_freq, axes=None, num_axes: int = 1, neighbours: bool = False, scale: float = 1.0, device="cuda"):
        inv_freq = [float(f) for f in inv_freq]
        if not all(math.isfinite(f) for f in inv_freq):
            raise ValueError("inv_freq must be finite")
        if axes is not None and (len(axes) != len(inv_freq) or not all(0 <= int(a) < num_axes for a in axes)):
            raise ValueError("axes must name an axis below num_axes for each of inv_freq")
        # turns per position, modulo 1, in units of 2^-64
        turn, words = 2 * 314159265358979323846264338327950288419716939937510, []    # (2 pi in units of 10^-50)
        for num, den in map(float.as_integer_ratio, inv_freq):
            words.append((num * 10 ** 50 * 2 ** 65 + den * turn) // (2 * den * turn) % 2 ** 64)
        self.frequencies = torch.tensor([w - 2 ** 64 if w >= 2 ** 63 else w for w in words], dtype=torch.int64, device=device)
        self.axes = None if axes is None else torch.tensor([int(a) for a in axes], dtype=torch.uint8, device=device)
        self.num_axes, self.rotary_dim = num_axes, 2 * len(inv_freq)
        self.c = kv_rope(self.frequencies.data_ptr(), self.axes.data_ptr() if axes is not None else None, self.rotary_dim,
                         num_axes, int(bool(neighbours)), float(scale))
        self.ref = ctypes.addressof(self.c)


# (Calls of a few microseconds: what is said of a refused argument is put together only when it is refused.)
def _positions(rope, positions, n):
    """Address of the positions and the distance of their axes."""
    if rope is None:
        return None, 0
    if positions is None or positions.dtype is not torch.int32 or not positions.is_cuda:
        raise ValueError("positions must be a CUDA tensor of torch.int32")
    shape, stride = positions.shape, positions.stride()
    if len(shape) == 1:                 # one row for all axes
        shape, stride = (rope.num_axes, shape[0]), (0, stride[0])
    if shape != (rope.num_axes, n) or (stride[1] != 1 and n > 1):
        raise ValueError(f"positions must have shape [{n}] or [{rope.num_axes}][{n}], an axis's {n} in a row")
    return positions.data_ptr(), stride[0]


def _heads(x, name, dtype, n, dim, heads=None):
    """Address, heads and row stride of rows x [n][heads][dim] whose heads are dense (None: no heads)."""
    if x is None:
        if heads:
            raise ValueError(f"{name} must be given")
        return None, 0, 0
    if x.dtype is not dtype or not x.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor of {dtype}")
    shape = x.shape
    if len(shape) != 3 or shape[0] != n or shape[2] != dim or (heads is not None and shape[1] != heads):
        raise ValueError(f"{name} must have shape [{n}][{'heads' if heads is None else heads}][{dim}], not {tuple(shape)}")
    row, head, one = x.stride()
    have = shape[1]
    if one != 1 or (head != dim and have != 1):
        raise ValueError(f"the heads of {name} must be dense")
    return x.data_ptr(), have, row if n > 1 else have * dim


# ---------------------------------------------------------------- C names
def kv_qk_rope(rope, positions, q, k, q_out, k_out, q_weight=None, k_weight=None, eps: float = 1e-6, stream=None):
    """Rows q [n][num_q_heads][d] and k [n][num_kv_heads][d] (either may be None) normed over each head (where
    there is a weight [d]) and rotated by ``positions`` (int32 [num_axes][n], or [n] for all axes) into q_out and k_out,
    which may be q and k.  ``rope`` None: no rotation."""
    some = q if q is not None else k
    if some is None or some.dim() != 3 or some.dtype not in _DTYPES:
        raise ValueError("q or k must be given, [n][heads][d] of torch.bfloat16 or torch.float16")
    n, _, dim = some.shape
    dtype = some.dtype
    pos, axis = _positions(rope, positions, n)
    qp, hq, qs = _heads(q, "q", dtype, n, dim)
    kp, hkv, ks = _heads(k, "k", dtype, n, dim)
    qo, _, qos = _heads(q_out, "q_out", dtype, n, dim, hq) if hq else (None, 0, 0)
    ko, _, kos = _heads(k_out, "k_out", dtype, n, dim, hkv) if hkv else (None, 0, 0)
    rc = (_fns or _load())["kv_qk_rope"](
        None if rope is None else rope.ref, _DTYPES[dtype], dim, n, pos, axis, hq, qp, qs, qo, qos, hkv, kp, ks, ko, kos,
        _vector(q_weight, "q_weight", dtype, dim), _vector(k_weight, "k_weight", dtype, dim), eps, kd._stream(stream))
    if rc:
        kd._check(rc, "kv_qk_rope")


def kv16_write(pool: Pool, slots, k, v, rope=None, positions=None, q=None, q_out=None, q_weight=None, k_weight=None,
               eps: float = 1e-6, device_error=None, stream=None):
    """Rows k (normed and rotated as in kv_qk_rope) and v into their slots (int64 [n]); rows q, if any, into q_out."""
    n, dim, dtype = slots.numel(), pool.head_dim, pool.dtype
    heads = pool.num_kv_heads
    pos, axis = _positions(rope, positions, n)
    kp, _, ks = _heads(k, "k", dtype, n, dim, heads)
    vp, _, vs = _heads(v, "v", dtype, n, dim, heads)
    qp, hq, qs = _heads(q, "q", dtype, n, dim)
    qo, _, qos = _heads(q_out, "q_out", dtype, n, dim, hq) if hq else (None, 0, 0)
    rc = (_fns or _load())["kv16_write"](
        pool.ref, None if rope is None else rope.ref, n, _vector(slots, "slots", torch.int64, 0), pos, axis, hq, qp, qs, qo,
        qos, kp, ks, vp, vs, _vector(q_weight, "q_weight", dtype, dim), _vector(k_weight, "k_weight", dtype, dim), eps,
        _vector(device_error, "device_error", torch.int32, 1), kd._stream(stream))
    if rc:
        kd._check(rc, "kv16_write")


def kv16_workspace(pool: Pool, num_q_heads: int, max_batch: int) -> torch.Tensor:
    """A workspace of kv16_workspace_bytes()."""
    n = _load()["kv16_workspace_bytes"](pool.ref, num_q_heads, max_batch)
    kd._check(min(n, 0), "kv16_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=pool.k.device)


def kv16_plan(pool: Pool, tables: Tables, num_q_heads: int, batch: int, workspace, seq_ids=None, prefix_ids=None,
              device_error=None, stream=None):
    """The plan of a decode step of ``batch`` rows for pools of this shape, into the workspace."""
    i32 = torch.int32
    for name, x in (("seq_ids", seq_ids), ("prefix_ids", prefix_ids)):
        if x is not None and x.numel() != batch:
            raise ValueError(f"{name} must have an entry for each row")
    rc = (_fns or _load())["kv16_plan"](
        pool.ref, tables.ref, num_q_heads, batch, _vector(seq_ids, "seq_ids", i32, batch),
        _vector(prefix_ids, "prefix_ids", i32, batch), _vector(workspace, "workspace", torch.uint8, 1), workspace.numel(),
        _vector(device_error, "device_error", i32, 1), kd._stream(stream))
    if rc:
        kd._check(rc, "kv16_plan")


def kv16_attention(pool: Pool, tables: Tables, q, out, workspace, lse=None, softmax_scale: float = 0.0,
                   device_error=None, stream=None):
    """Decode attention of the planned rows q [batch][num_q_heads][head_dim] over their prefixes and their own tokens."""
    batch, dim, dtype = len(q), pool.head_dim, pool.dtype
    q, heads, q_stride = _heads(q, "q", dtype, batch, dim)
    out, _, out_stride = _heads(out, "out", dtype, batch, dim, heads)
    rc = (_fns or _load())["kv16_attention"](
        pool.ref, tables.ref, batch, heads, q, q_stride, out, out_stride,
        _vector(lse, "lse", torch.float32, batch * heads), softmax_scale,
        _vector(workspace, "workspace", torch.uint8, 1), workspace.numel(),
        _vector(device_error, "device_error", torch.int32, 1), kd._stream(stream))
    if rc:
        kd._check(rc, "kv16_attention")

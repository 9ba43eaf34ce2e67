"""ctypes binding of the 4-bit paged cache (declared in include/kvdecode4.h).

Argument marshalling only, as in ``kvdecode``: functions keep the C names.
``Pool`` and ``Tables`` hold the caller's tensors together with the C structs
that describe them, so that a call marshals little; tensors passed to a call
are checked here, since the kernels read through the raw pointers.  ``stream``
accepts a ``torch.cuda.Stream``, a raw handle or None (the legacy default
stream).
"""
from __future__ import annotations

import ctypes

import torch

from . import kvdecode as kd

KVC_DTYPE_BF16 = 0
KVC_DTYPE_F16 = 1
PAGE_SIZE = 16

_DTYPES = {torch.bfloat16: KVC_DTYPE_BF16, torch.float16: KVC_DTYPE_F16}
_P = ctypes.c_void_p
_I32 = ctypes.c_int32
_I64 = ctypes.c_int64


class kv4_pool(ctypes.Structure):
    _fields_ = [("data", _P), ("num_pages", _I64), ("num_kv_heads", _I32), ("head_dim", _I32), ("group", _I32),
                ("dtype", _I32)]


class kv_tables(ctypes.Structure):
    _fields_ = [("block_table", _P), ("lens", _P), ("free_ring", _P), ("free_state", _P), ("num_pages", _I64),
                ("max_seqs", _I32), ("max_pages", _I32)]


_SIGS = {
    "kv4_pool_bytes": ([_P], _I64),
    "kv4_workspace_bytes": ([_P, _I32], _I64),
    "kv_tables_step": ([_P, _I32, _P, _P, _I32, _P, _P, _P, _P, _P, _P, _P], _I32),
    "kv4_write": ([_P, _I32, _P, _P, _I64, _P, _I64, _P, _P], _I32),
    "kv4_read": ([_P, _I32, _P, _P, _I64, _P, _I64, _P, _P], _I32),
    "kv4_decode_attention": ([_P, _P, _I32, _P, _I32, _P, _I64, _P, _I64, _P, ctypes.c_float, _P, _I64, _P, _P], _I32),
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


# (Calls of a few microseconds: what is said of a refused argument is put together only when it is refused.)
def _vector(x, name, dtype, n):
    """Address of a dense CUDA vector with at least n entries (None: null)."""
    if x is None:
        return None
    if x.dtype is not dtype or not x.is_cuda or not x.is_contiguous() or x.numel() < n:
        raise ValueError(f"{name} must be a contiguous CUDA tensor of {dtype} with at least {n} entries")
    return x.data_ptr()


def _rows(x, name, dtype, shape):
    """Address and row stride of a CUDA tensor of the given shape [n][heads][dim] whose heads are dense."""
    if x.dtype is not dtype or not x.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor of {dtype}")
    if x.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, not {tuple(x.shape)}")
    row, head, one = x.stride()
    n, heads, dim = shape
    if one != 1 or (head != dim and heads != 1):
        raise ValueError(f"the heads of {name} must be dense")
    return x.data_ptr(), row if n > 1 else heads * dim


class Pool:
    """One layer's 4-bit pool: ``data`` uint8 [num_pages][num_kv_heads][block bytes] (see ``block_bytes``)."""

    def __init__(self, data: torch.Tensor, head_dim: int, group: int, dtype: torch.dtype = torch.bfloat16):
        if dtype not in _DTYPES:
            raise ValueError("dtype must be torch.bfloat16 or torch.float16")
        if data.dtype is not torch.uint8 or not data.is_cuda or not data.is_contiguous() or data.dim() != 3:
            raise ValueError("data must be a contiguous CUDA tensor of uint8 with three dimensions")
        self.data, self.head_dim, self.group, self.dtype = data, head_dim, group, dtype
        self.num_kv_heads = data.shape[1]
        self.c = kv4_pool(data.data_ptr(), data.shape[0], data.shape[1], head_dim, group, _DTYPES[dtype])
        self.ref = ctypes.addressof(self.c)
        n = kv4_pool_bytes(self)
        if n != data.numel():
            raise ValueError(f"data must have {n} bytes for its pages and heads, not {data.numel()}")

    @staticmethod
    def block_bytes(head_dim: int, group: int) -> int:
        """Bytes of the block of one page and KV head."""
        return PAGE_SIZE * head_dim + 8 * PAGE_SIZE * (head_dim // group)

    @classmethod
    def empty(cls, num_pages: int, num_kv_heads: int, head_dim: int, group: int, dtype: torch.dtype = torch.bfloat16,
              device="cuda"):
        """A pool of its own memory, zero-filled."""
        return cls(torch.zeros((num_pages, num_kv_heads, cls.block_bytes(head_dim, group)), dtype=torch.uint8,
                               device=device), head_dim, group, dtype)


class Tables:
    """Block tables int32 [max_seqs][max_pages], lengths int32 [max_seqs] and, where kv_tables_step works on
    them, the ring of free pages int32 [num_pages] and its state int32 [4]."""

    def __init__(self, block_table: torch.Tensor, lens: torch.Tensor, free_ring: torch.Tensor | None = None,
                 free_state: torch.Tensor | None = None):
        if block_table.dim() != 2:
            raise ValueError("block_table must have two dimensions")
        self.max_seqs, self.max_pages = block_table.shape
        self.block_table, self.lens, self.free_ring, self.free_state = block_table, lens, free_ring, free_state
        self.c = kv_tables(_vector(block_table, "block_table", torch.int32, 0),
                           _vector(lens, "lens", torch.int32, self.max_seqs),
                           _vector(free_ring, "free_ring", torch.int32, 1),
                           _vector(free_state, "free_state", torch.int32, 4),
                           free_ring.numel() if free_ring is not None else 0, self.max_seqs, self.max_pages)
        self.ref = ctypes.addressof(self.c)

    @classmethod
    def empty(cls, num_pages: int, max_seqs: int, max_pages: int, device="cuda"):
        """Tables of requests of length 0 with all pages free, page 0 first."""
        i32 = dict(dtype=torch.int32, device=device)
        return cls(torch.full((max_seqs, max_pages), -1, **i32), torch.zeros(max_seqs, **i32),
                   torch.arange(num_pages, **i32), torch.tensor([0, num_pages, 0, 0], **i32))


# ---------------------------------------------------------------- C names
def kv4_pool_bytes(pool: Pool) -> int:
    n = _load()["kv4_pool_bytes"](pool.ref)
    kd._check(min(n, 0), "kv4_pool_bytes")
    return n


def kv4_workspace(pool: Pool, num_q_heads: int) -> torch.Tensor:
    """A workspace of kv4_workspace_bytes()."""
    n = _load()["kv4_workspace_bytes"](pool.ref, num_q_heads)
    kd._check(min(n, 0), "kv4_workspace_bytes")
    return torch.empty(n, dtype=torch.uint8, device=pool.data.device)


def kv_tables_step(tables: Tables, seq_ids, new_lens, slots, positions=None, cu_seqlens=None, lens_out=None,
                   free_state_out=None, device_error=None, stream=None):
    """One step of the batch of requests ``seq_ids`` (None: request i is row i)
    that ``new_lens`` changes; ``slots`` (int64) has room for the new tokens."""
    n, room, i32 = new_lens.numel(), slots.numel(), torch.int32
    if seq_ids is not None and seq_ids.numel() != n:
        raise ValueError("seq_ids and new_lens must have the same number of entries")
    rc = (_fns or _load())["kv_tables_step"](
        tables.ref, n, _vector(seq_ids, "seq_ids", i32, n), _vector(new_lens, "new_lens", i32, n), room,
        _vector(slots, "slots", torch.int64, 0), _vector(positions, "positions", i32, room),
        _vector(cu_seqlens, "cu_seqlens", i32, n + 1), _vector(lens_out, "lens_out", i32, tables.max_seqs),
        _vector(free_state_out, "free_state_out", i32, 4), _vector(device_error, "device_error", i32, 1),
        kd._stream(stream))
    if rc:
        kd._check(rc, "kv_tables_step")


def _kv4_rows(fn, pool: Pool, slots, k, v, device_error, stream):
    n = slots.numel()
    shape = (n, pool.num_kv_heads, pool.head_dim)
    k, k_stride = _rows(k, "k", pool.dtype, shape)
    v, v_stride = _rows(v, "v", pool.dtype, shape)
    rc = (_fns or _load())[fn](pool.ref, n, _vector(slots, "slots", torch.int64, 0), k, k_stride, v, v_stride,
                               _vector(device_error, "device_error", torch.int32, 1), kd._stream(stream))
    if rc:
        kd._check(rc, fn)


def kv4_write(pool: Pool, slots, k, v, device_error=None, stream=None):
    """Quantise rows k and v ([n][num_kv_heads][head_dim]) into their slots (int64 [n])."""
    _kv4_rows("kv4_write", pool, slots, k, v, device_error, stream)


def kv4_read(pool: Pool, slots, k_out, v_out, device_error=None, stream=None):
    """The slots' values into k_out and v_out ([n][num_kv_heads][head_dim])."""
    _kv4_rows("kv4_read", pool, slots, k_out, v_out, device_error, stream)


def kv4_decode_attention(pool: Pool, tables: Tables, q, out, workspace, seq_ids=None, lse=None,
                         softmax_scale: float = 0.0, device_error=None, stream=None):
    """Decode attention of q [batch][num_q_heads][head_dim] over each row's request."""
    shape = q.shape
    if len(shape) != 3 or shape[2] != pool.head_dim:
        raise ValueError(f"q must have shape [batch][num_q_heads][{pool.head_dim}]")
    batch, heads = shape[0], shape[1]
    if seq_ids is not None and seq_ids.numel() != batch:
        raise ValueError("seq_ids must have an entry for each row of q")
    q, q_stride = _rows(q, "q", pool.dtype, shape)
    out, out_stride = _rows(out, "out", pool.dtype, shape)
    rc = (_fns or _load())["kv4_decode_attention"](
        pool.ref, tables.ref, batch, _vector(seq_ids, "seq_ids", torch.int32, batch), heads, q, q_stride, out,
        out_stride, _vector(lse, "lse", torch.float32, batch * heads), softmax_scale,
        _vector(workspace, "workspace", torch.uint8, 1), workspace.numel(),
        _vector(device_error, "device_error", torch.int32, 1), kd._stream(stream))
    if rc:
        kd._check(rc, "kv4_decode_attention")

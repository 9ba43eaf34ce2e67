"""Drive a decode session of a workload through the C ABI: over the bf16 cache
(``DecodeSession``), over the 4-bit one (``Kv4Session``) or over 16-bit pools in
which requests share prefixes (``SharedPrefixSession``).

Sets up a cache for a ``WorkloadConfig`` (pool sized for the prefix plus
``extra_tokens`` decode steps, page order and reservation order from the
workload), writes each sequence's cached prefix (vision tokens first, then
text) into every layer pool, and runs decode steps: ``kv_begin_step`` then, per
logical layer, ``kv_append`` and ``decode_attention``.  Torch is used only to
hold device buffers and streams.
"""
from __future__ import annotations

import numpy as np

from . import kv4, kv16
from . import kvdecode as kd
from . import workloads as wl


class DecodeSession:
    def __init__(self, cfg: wl.WorkloadConfig, extra_tokens: int = 8, device="cuda", stream=None,
                 lens=None, slack_pages: int = 8, split_pages: int = 0, host_only: bool = False):
        import torch
        self.torch = torch
        self.cfg = cfg
        self.device = device
        self.stream = stream
        self.lens = np.array(wl.context_lengths(cfg) if lens is None else lens, dtype=np.int64)
        self.lens0 = self.lens.copy()
        P = cfg.page_size
        self.max_pages = int((int(self.lens.max()) + extra_tokens + P - 1) // P)
        self.num_pages = int(sum((int(n) + extra_tokens + P - 1) // P for n in self.lens)) + slack_pages
        flags = kd.KVC_FLAG_HOST_ONLY if host_only else 0
        self.kcfg = kd.make_config(cfg.phys_layers, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim,
                                   self.num_pages, cfg.batch, self.max_pages, page_size=P, flags=flags)
        self.h = kd.kv_cache_create(self.kcfg, stream)
        order = wl.page_order(cfg, self.num_pages)
        if order is not None:
            kd.kv_cache_set_page_order(self.h, order)
        if split_pages:
            kd.kv_cache_set_split_pages(self.h, split_pages)
        self.seq_ids = [kd.kv_seq_create(self.h) for _ in range(cfg.batch)]
        for i, n in wl.reserve_schedule(cfg, self.lens):
            kd.kv_seq_reserve(self.h, self.seq_ids[i], n, stream)

    # ------------------------------------------------------------------ setup
    def fill_prefix(self, layers=None):
        """Write every sequence's cached prefix into the given layer pools."""
        cfg = self.cfg
        layers = range(cfg.phys_layers) if layers is None else layers
        for l in layers:
            for b, seq in enumerate(self.seq_ids):
                n = int(self.lens0[b])
                k = wl.kv_block(cfg, l, b, n, "k", self.device)
                v = wl.kv_block(cfg, l, b, n, "v", self.device)
                kd.kv_write_tokens(self.h, l, seq, 0, n, k, v, self.stream)
                del k, v

    # ------------------------------------------------------------------- step
    def begin_step(self):
        kd.kv_begin_step(self.h, self.seq_ids, self.stream)
        self.lens += 1

    def phys(self, layer: int) -> int:
        return layer % self.cfg.phys_layers

    def append(self, layer: int, k_new, v_new):
        kd.kv_append(self.h, self.phys(layer), self.cfg.batch, k_new, v_new, self.stream)

    def attend(self, layer: int, q, out, scale: float = 0.0):
        kd.decode_attention(self.h, self.phys(layer), self.cfg.batch, q, out, scale, self.stream)

    def append_attend(self, layer: int, q, k_new, v_new, out, scale: float = 0.0):
        """kv_append + decode_attention of one layer in one fused launch."""
        kd.decode_attention_append(self.h, self.phys(layer), self.cfg.batch, q, k_new, v_new, out, scale,
                                   self.stream)

    def query(self, raise_on_device_error=True):
        return kd.kv_cache_query(self.h, raise_on_device_error)

    def close(self):
        if self.h is not None:
            kd.kv_cache_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()


def _on_stream(s):
    """torch's work and memory on stream s: a block that is freed is handed out again behind what reads it."""
    from torch import cuda
    if not isinstance(s, cuda.Stream):
        s = cuda.ExternalStream(int(s)) if s else cuda.default_stream()
    return cuda.stream(s)


class Kv4Session:
    """The same session over a 4-bit cache: every step's block tables and slot
    map are built on the device from the requests' lengths, new K and V are
    quantised into their slots, and decode attention reads the 4-bit pages.

    Everything that the session makes and does is ordered on its stream (None: the
    default one), whatever stream is current in torch: tensors passed to ``append``
    and ``attend`` must be ready there, and what comes back is.  ``begin_step``, ``append`` and
    ``attend`` only enqueue; ``grow`` and ``fill_prefix`` copy host lengths to the device and
    ``check`` reads from it, which wait for the stream."""

    def __init__(self, cfg: wl.WorkloadConfig, extra_tokens: int = 8, group: int = 64, device="cuda", stream=None,
                 lens=None, slack_pages: int = 8):
        import torch
        self.cfg = cfg
        self.stream = stream
        self._torch, self._i32 = torch, dict(dtype=torch.int32, device=device)
        self.lens0 = np.array(wl.context_lengths(cfg) if lens is None else lens, dtype=np.int64)
        self.lens = np.zeros_like(self.lens0)      # held so far: fill_prefix admits the requests
        P = kv4.PAGE_SIZE
        max_pages = int((int(self.lens0.max()) + extra_tokens + P - 1) // P)
        num_pages = int(sum((int(n) + extra_tokens + P - 1) // P for n in self.lens0)) + slack_pages
        with self._on_stream():
            self.pools = [kv4.Pool.empty(num_pages, cfg.num_kv_heads, cfg.head_dim, group, device=device)
                          for _ in range(cfg.phys_layers)]
            self.tables = kv4.Tables.empty(num_pages, cfg.batch, max(1, max_pages), device=device)
            order = wl.page_order(cfg, num_pages)
            if order is not None:
                self.tables.free_ring.copy_(torch.from_numpy(order))
            self.error = torch.zeros(1, **self._i32)
            self.ones = torch.ones(cfg.batch, **self._i32)
            self.step_slots = torch.empty(cfg.batch, dtype=torch.int64, device=device)
            self.workspace = kv4.kv4_workspace(self.pools[0], cfg.num_q_heads)

    def _on_stream(self):
        return _on_stream(self.stream)

    def grow(self, new_lens):
        """Requests grow by new_lens tokens (host sequence), or give -n back; returns the new tokens' slots."""
        with self._on_stream():
            new = self._torch.tensor([int(n) for n in new_lens], **self._i32)
            slots = self._torch.empty(int(sum(max(0, int(n)) for n in new_lens)), dtype=self._torch.int64, device=new.device)
            kv4.kv_tables_step(self.tables, None, new, slots, device_error=self.error, stream=self.stream)
        self.lens += np.array(new_lens, dtype=np.int64)
        return slots

    def fill_prefix(self, layers=None):
        """Admit every request and write its cached prefix into the given layer pools."""
        cfg = self.cfg
        slots = self.grow(self.lens0)
        with self._on_stream():
            for l in range(cfg.phys_layers) if layers is None else layers:
                k, v, _ = wl.packed_prefix(cfg, [l], self.lens0, slots.device)
                kv4.kv4_write(self.pools[l], slots, k[0], v[0], device_error=self.error, stream=self.stream)
                del k, v

    def begin_step(self):
        kv4.kv_tables_step(self.tables, None, self.ones, self.step_slots, device_error=self.error, stream=self.stream)
        self.lens += 1

    def phys(self, layer: int) -> int:
        return layer % self.cfg.phys_layers

    def append(self, layer: int, k_new, v_new):
        kv4.kv4_write(self.pools[self.phys(layer)], self.step_slots, k_new, v_new, device_error=self.error,
                      stream=self.stream)

    def attend(self, layer: int, q, out, scale: float = 0.0, lse=None):
        kv4.kv4_decode_attention(self.pools[self.phys(layer)], self.tables, q, out, self.workspace, lse=lse,
                                 softmax_scale=scale, device_error=self.error, stream=self.stream)

    def check(self):
        """Wait for the session's stream and raise if a call has found something wrong."""
        with self._on_stream():
            bits = int(self.error.item())
        if bits:
            raise RuntimeError(f"device error bits {bits:#x}")


class SharedPrefixSession:
    """A decode session in which requests continue shared prefixes (an image and its prompt, a system prompt), each held
    once: request i of the workload holds its own tokens only and continues prefix ``prefix_of[i]`` (-1: none), whose
    ``prefix_lens`` tokens are a request of their own, row ``cfg.batch + prefix_of[i]`` of the block tables.

    A step: ``begin_step`` (slots, positions and the attention plan, on the device), then per layer ``append`` (queries
    and keys normed and rotated, K and V written into their slots) and ``attend``.  ``rope`` None: no rotation.  A token's position
    is its index behind the prefix; ``first_positions`` (a sequence) gives a request's first own token another than the
    length of its prefix, as where an image takes fewer positions than tokens.  Those stay until ``grow`` is given others.

    Requests that share a prefix read it once where they are neighbours in the workload: ``prefix_of`` is best ordered by prefix.

    Where a session with a ``rope`` was not given any, requests' first positions follow their prefix: one that has been shortened, or
    has outgrown ``prefix_lens``, counts with the length that it has (before that, and while it is held in part, with the length in
    ``prefix_lens``).  A request that holds tokens turned for another length is not continued: ``grow`` refuses such a change.
    (Without a ``rope`` nothing is turned, and first positions stay as they were made.)

    Ordered on its stream as ``Kv4Session`` is: ``begin_step``, ``append`` and ``attend`` only enqueue."""

    def __init__(self, cfg: wl.WorkloadConfig, prefix_lens, prefix_of, rope=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                 first_positions=None, extra_tokens: int = 8, dtype=None, device="cuda", stream=None, lens=None, slack_pages: int = 8):
        import torch
        self.cfg, self.rope, self.stream, self._torch = cfg, rope, stream, torch
        self.q_weight, self.k_weight, self.eps = q_weight, k_weight, eps
        self._i32 = dict(dtype=torch.int32, device=device)
        own = np.array(wl.context_lengths(cfg) if lens is None else lens, dtype=np.int64)
        self.lens0 = np.concatenate([own, np.array(prefix_lens, dtype=np.int64)])
        self.lens = np.zeros_like(self.lens0)      # held so far: fill_prefix admits requests and prefixes
        self.prefix_of = [int(g) for g in prefix_of]
        if len(self.prefix_of) != cfg.batch or len(own) != cfg.batch:
            raise ValueError("prefix_of and lens must have an entry for each request")
        if not all(-1 <= g < len(prefix_lens) for g in self.prefix_of):
            raise ValueError("prefix_of must name one of prefix_lens, or -1")
        self._follows = rope is not None and first_positions is None
        self._counts = {g: int(n) for g, n in enumerate(prefix_lens)}      # tokens that a prefix counts for its requests' positions
        self._moved = set()                                               # prefixes that have been shortened or have outgrown prefix_lens
        if first_positions is None:
            first_positions = [self._counts[g] if g >= 0 else 0 for g in self.prefix_of]
        self.first_positions = self._first_positions(first_positions)
        dtype = torch.bfloat16 if dtype is None else dtype
        P = kv4.PAGE_SIZE
        room = self.lens0 + np.array([extra_tokens] * cfg.batch + [0] * len(prefix_lens), dtype=np.int64)
        num_pages = int(((room + P - 1) // P).sum()) + slack_pages
        with self._on_stream():
            self.pools = [kv16.Pool.empty(num_pages, cfg.num_kv_heads, cfg.head_dim, dtype, device=device)
                          for _ in range(cfg.phys_layers)]
            self.tables = kv4.Tables.empty(num_pages, len(room), max(1, int((room.max() + P - 1) // P)), device=device)
            order = wl.page_order(cfg, num_pages)
            if order is not None:
                self.tables.free_ring.copy_(torch.from_numpy(order))
            self.error = torch.zeros(1, **self._i32)
            self.ones = torch.ones(cfg.batch, **self._i32)
            self.ids = torch.arange(cfg.batch, **self._i32)
            self.prefix_ids = torch.tensor([cfg.batch + g if g >= 0 else -1 for g in self.prefix_of], **self._i32)
            self.first = torch.tensor(self.first_positions, **self._i32)
            self.index, self.positions = torch.empty(cfg.batch, **self._i32), torch.empty(cfg.batch, **self._i32)
            self.step_slots = torch.empty(cfg.batch, dtype=torch.int64, device=device)
            self.workspace = kv16.kv16_workspace(self.pools[0], cfg.num_q_heads, cfg.batch)

    def _on_stream(self):
        return _on_stream(self.stream)

    def _first_positions(self, given):
        if len(given) != self.cfg.batch:
            raise ValueError("first_positions must have an entry for each request")
        return [int(p) for p in given]

    def _follow(self, new):
        """What prefixes count, which of them have moved, and first positions, once requests and prefixes have grown by new."""
        batch, counts, moved, first = self.cfg.batch, dict(self._counts), set(self._moved), list(self.first_positions)
        if not new[batch:].any():
            return counts, moved, first
        with self._on_stream():
            before = np.array(self.tables.lens.tolist(), dtype=np.int64)      # (of the device: steps of graphs count there)
        for g in (int(i) for i in np.flatnonzero(new[batch:])):
            n = int((before + new)[batch + g])
            if new[batch + g] < 0 or n > counts[g]:
                moved.add(g)
            if g in moved and n > 0:             # (a prefix that is gone may come again as it was)
                counts[g] = n
        for i, g in enumerate(self.prefix_of):
            if g >= 0 and first[i] != counts[g]:
                if before[i] > 0 and before[i] + new[i] > 0:
                    raise ValueError(f"request {i} holds tokens turned as behind {first[i]} of prefix {g}, which would be {counts[g]}: "
                                     "close it first, or give first_positions")
                first[i] = counts[g]
        return counts, moved, first

    def grow(self, new_lens, first_positions=None):
        """Requests, then prefixes, grow by new_lens tokens (host sequence), or give -n back; returns the new tokens' slots
        and positions.  A prefix may grow or be dropped only while no request that continues it takes a step.
        first_positions: the requests' first positions from now on."""
        new = np.array([int(n) for n in new_lens], dtype=np.int64)
        added = int(np.maximum(new, 0).sum())
        first = self.first_positions
        if first_positions is not None:
            first, self._follows = self._first_positions(first_positions), False
        elif self._follows:
            self._counts, self._moved, first = self._follow(new)
        with self._on_stream():
            if first != self.first_positions:
                self.first_positions = first
                self.first.copy_(self._torch.tensor(first, dtype=self.first.dtype))
            dev = self._torch.tensor(new, **self._i32)
            slots = self._torch.empty(added, dtype=self._torch.int64, device=dev.device)
            index = self._torch.empty(added, **self._i32)
            kv4.kv_tables_step(self.tables, None, dev, slots, index, device_error=self.error, stream=self.stream)
            first = np.repeat(np.array(self.first_positions + [0] * (len(new) - self.cfg.batch)), np.maximum(new, 0))
            index += self._torch.from_numpy(first.astype(np.int32)).to(dev.device)
        self.lens += new
        return slots, index

    def write(self, layer: int, slots, positions, k, v):
        """Prompt tokens' K, normed and rotated, and V into their slots."""
        kv16.kv16_write(self.pools[self.phys(layer)], slots, k, v, rope=self.rope, positions=positions if self.rope else None,
                        k_weight=self.k_weight, eps=self.eps, device_error=self.error, stream=self.stream)

    def fill_prefix(self, layers=None):
        """Admit every request and prefix and write their cached tokens into the given layer pools."""
        cfg = self.cfg
        slots, positions = self.grow(self.lens0)
        with self._on_stream():
            for l in range(cfg.phys_layers) if layers is None else layers:
                k, v, _ = wl.packed_prefix(cfg, [l], self.lens0, slots.device)
                self.write(l, slots, positions, *(x[0].to(self.pools[l].dtype) for x in (k, v)))
                del k, v

    def begin_step(self):
        kv4.kv_tables_step(self.tables, self.ids, self.ones, self.step_slots, self.index, device_error=self.error,
                           stream=self.stream)
        with self._on_stream():
            self._torch.add(self.index, self.first, out=self.positions)
        kv16.kv16_plan(self.pools[0], self.tables, self.cfg.num_q_heads, self.cfg.batch, self.workspace, seq_ids=self.ids,
                       prefix_ids=self.prefix_ids, device_error=self.error, stream=self.stream)
        self.lens[:self.cfg.batch] += 1

    def phys(self, layer: int) -> int:
        return layer % self.cfg.phys_layers

    def append(self, layer: int, q, k_new, v_new, q_out, positions=None):
        """The new tokens' K and V into their slots; queries for ``attend`` into q_out (which may be q).  positions: others than
        the step's, for instance one row for each axis."""
        if self.rope is None:
            positions = None
        elif positions is None:
            positions = self.positions
        kv16.kv16_write(self.pools[self.phys(layer)], self.step_slots, k_new, v_new, rope=self.rope, positions=positions, q=q,
                        q_out=q_out, q_weight=self.q_weight, k_weight=self.k_weight, eps=self.eps, device_error=self.error,
                        stream=self.stream)

    def attend(self, layer: int, q, out, scale: float = 0.0, lse=None):
        kv16.kv16_attention(self.pools[self.phys(layer)], self.tables, q, out, self.workspace, lse=lse, softmax_scale=scale,
                            device_error=self.error, stream=self.stream)

    def check(self):
        """Wait for the session's stream and raise if a call has found something wrong."""
        with self._on_stream():
            bits = int(self.error.item())
        if bits:
            raise RuntimeError(f"device error bits {bits:#x}")

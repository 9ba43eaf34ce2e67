"""Drive a decode session of a workload through the C ABI: over the bf16 cache
(``DecodeSession``) or over the 4-bit one (``Kv4Session``).

Sets up a cache for a ``WorkloadConfig`` (pool sized for the prefix plus
``extra_tokens`` decode steps, page order and reservation order from the
workload), writes each sequence's cached prefix (vision tokens first, then
text) into every layer pool, and runs decode steps: ``kv_begin_step`` then, per
logical layer, ``kv_append`` and ``decode_attention``.  Torch is used only to
hold device buffers and streams.
"""
from __future__ import annotations

import numpy as np

from . import kv4
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
        """torch's work and memory on the session's stream: a block that is freed is handed out again behind what reads it."""
        cuda, s = self._torch.cuda, self.stream
        if not isinstance(s, cuda.Stream):
            s = cuda.ExternalStream(int(s)) if s else cuda.default_stream()
        return cuda.stream(s)

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

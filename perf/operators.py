"""Cases of the 4-bit paged cache: the operators that a serving step runs when K and V are held in 4 bits.

* ``tables``: a step's block tables and slot map, built on the GPU from request lengths.  Every request of the
  batch grows by some tokens (a prompt chunk, one decoded token), or gives tokens back (rejected drafts, a finished
  request): pages come from and go to a ring of free pages, every new token gets its slot and position.
* ``write``: K and V rows of a packed batch of new tokens quantised to 4 bits and scattered to their slots, then
  read back through the slot map, as a prefill does that attends to what later decode steps will see.
* ``read``: tokens gathered from the cache and returned in 16 bits (a cached prefix before a prompt chunk).
* ``attention``: single-token decode attention over the cache through the block table.

The format.  A page holds 16 tokens; the block of one page and KV head is

    K codes [16 * D / 2 bytes], V codes [16 * D / 2], K scales [16][D / group] words, V scales [16][D / group] words.

A scale word holds s in its low and z in its high half, both in the cache's 16-bit type; a code c of 0 .. 15 stands for
s * (c - 8) + z.  Over the group's values x, s = round16((max - min) / 15), z = round16(min + 8 s) and
c = clamp(rint((x - z) / s) + 8, 0, 15), 8 where s is 0.  Codes lie as 32-bit words of eight: K word [token][j][i]
(j < 4, i < D / 32) holds d = 32 i + 8 j + e, e < 8, at bit 16 (e % 2) + 4 (e / 2); V word [token / 8][g][j][i] (g < 8,
j < 4) holds token 8 (token / 8) + 2 j + h and d = 32 i + 8 n + g, h < 2, n < 4, at bit 16 h + 4 n.

Lengths are a function of the case alone (``lens_seed``), so ``work`` is exact; values and page orders come from
``prepare``'s seed.  The plain forms gather, unpack and compute in 32 bits with elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

P = 16                                       # tokens per page
PREFIXES = (256, 576, 1024, 2048, 4096)      # dynamic-resolution vision prefixes


# ------------------------------------------------------------------- cases
def _attention(name, hq, hkv, d, group, batch, dist, lo, hi, dtype="bf16", fused_qkv=False, scale=0.0, lens_seed=1):
    return {"name": name, "op": "attention", "hq": hq, "hkv": hkv, "d": d, "group": group, "batch": batch, "dist": dist,
            "lo": lo, "hi": hi, "dtype": dtype, "fused_qkv": fused_qkv, "scale": scale, "lens_seed": lens_seed}


def _rows(name, op, hkv, d, group, n, dtype="bf16", fused_qkv=False, order="runs"):
    return {"name": name, "op": op, "hkv": hkv, "d": d, "group": group, "n": n, "dtype": dtype, "fused_qkv": fused_qkv,
            "order": order}


def _tables(name, batch, dist, lo, hi, chunk, prefills, trims, closes, lens_seed=1):
    return {"name": name, "op": "tables", "batch": batch, "dist": dist, "lo": lo, "hi": hi, "chunk": chunk,
            "prefills": prefills, "trims": trims, "closes": closes, "lens_seed": lens_seed}


def listed():
    return [
        # A decode step of the GQA batch: one token each.  Launch latency.
        _tables("tables_decode_b32", 32, "vision", 32, 512, 1, 0, 0, 0),
        # A mixed step of continuous batching: prompt chunks beside decoding requests, some drafts rejected, some closed.
        _tables("tables_mixed_b157", 157, "log", 1, 8192, 1777, 9, 21, 6),
        # A bulk admission: many prompts at once.
        _tables("tables_admit_b1500", 1500, "log", 1, 64, 600, 1500, 0, 0),
        # One decoded token per request of the MHA batch: what a layer appends in every step.
        _rows("write_decode_mha_b64", "write", 32, 128, 128, 64, fused_qkv=True),
        # A ragged prompt chunk on the GQA shape, fine groups, in fp16.
        _rows("write_chunk_gqa_5003", "write", 4, 128, 32, 5003, dtype="fp16"),
        # The MHA batch's prompts: 64 requests of some 900 tokens.
        _rows("write_prompts_mha_57344", "write", 32, 128, 64, 57344),
        # One request's cached vision prefix (576 tokens and a prompt) at d 64.
        _rows("read_prefix_d64_631", "read", 8, 64, 32, 631),
        # A long cached prefix of the GQA shape whose tokens lie in any order.
        _rows("read_prefix_gqa_32768", "read", 4, 128, 128, 32768, order="shuffled"),
        # One interactive request on the GQA shape with a dynamic vision prefix: latency.
        _attention("attn_gqa_b1", 28, 4, 128, 128, 1, "uniform", 2337, 2337, fused_qkv=True),
        # The MHA batch (576 vision tokens, a prompt and what was generated).
        _attention("attn_mha_b64", 32, 32, 128, 128, 64, "uniform", 640, 1344),
        # Long multi-image contexts: few, very long rows, fine groups, fp16.
        _attention("attn_long_b8", 28, 4, 128, 32, 8, "uniform", 32640, 32768, dtype="fp16"),
        # Ragged mixed batch, log-uniform contexts, some rows still empty.
        _attention("attn_ragged_b64", 32, 32, 128, 64, 64, "log0", 0, 8192),
    ]


HEADS = ((8, 8), (32, 32), (28, 4), (14, 2), (16, 2), (5, 5), (12, 4), (7, 1), (24, 3))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = work(listed()[-1])["bytes"]
    while True:
        op = rng.choice(("tables", "write", "read", "attention", "attention"))
        dtype = rng.choice(("bf16", "fp16"))
        d = rng.choice((64, 128))
        group = rng.choice((32, 64, d))
        hq, hkv = rng.choice(HEADS)
        if op == "tables":
            batch = _log(rng, 1, 2000)
            prefills = rng.randint(0, batch)
            trims = rng.randint(0, batch - prefills)
            closes = rng.randint(0, batch - prefills - trims)
            c = _tables("", batch, "log", 1, _log(rng, 16, 16384), _log(rng, 1, max(2, 500000 // batch)), prefills, trims, closes,
                        lens_seed=rng.randint(1, 10 ** 6))
        elif op == "attention":
            hi = _log(rng, 1, 33000)
            c = _attention("", hq, hkv, d, group, _log(rng, 1, 256), rng.choice(("log0", "uniform")), rng.randint(0, hi), hi,
                           dtype, rng.random() < 0.5, rng.choice((0.0, 0.11)), rng.randint(1, 10 ** 6))
            if c["batch"] * hi * hkv * d > 64 * 8192 * 32 * 128:   # what the padded plain form may take
                continue
        else:
            c = _rows("", op, hkv, d, group, _log(rng, 1, 60000), dtype, rng.random() < 0.5, rng.choice(("runs", "shuffled")))
        if work(c)["bytes"] <= most:
            del c["name"]
            return c


# ------------------------------------------------------- lengths and bytes
def _np_rng(case, stream):
    return np.random.Generator(np.random.PCG64([case.get("lens_seed", 1), stream]))


def _lens(case):
    r, n, lo, hi = _np_rng(case, 1), case["batch"], case["lo"], case["hi"]
    if case["dist"] == "uniform":
        return r.integers(lo, hi, size=n, endpoint=True)
    if case["dist"] == "vision":
        return r.choice(np.array(PREFIXES), size=n) + r.integers(lo, hi, size=n, endpoint=True)
    if case["dist"] == "log":
        return np.clip(np.rint(np.exp(r.uniform(math.log(lo), math.log(max(lo, hi)), size=n))).astype(np.int64), lo, max(lo, hi))
    # "log0": from zero on
    return np.clip(np.rint(np.exp(r.uniform(0.0, math.log(hi + 1.0), size=n))).astype(np.int64) - 1, 0, hi)


def _changes(case):
    """What each request of a tables case adds (> 0) or gives back (< 0), in batch order."""
    r, lens = _np_rng(case, 2), _lens(case)
    n = case["batch"]
    new = np.ones(n, np.int64)
    kind = r.permutation(n)
    a, b, c = case["prefills"], case["trims"], case["closes"]
    new[kind[:a]] = r.integers(1, max(1, case["chunk"]), size=a, endpoint=True)
    new[kind[a:a + b]] = -np.minimum(r.integers(1, 7, size=b, endpoint=True), lens[kind[a:a + b]])
    new[kind[a + b:a + b + c]] = -lens[kind[a + b:a + b + c]]
    return lens, new


def _pages(n):
    return (n + P - 1) // P


def work(case):
    if case["op"] == "tables":
        lens, new = _changes(case)
        tokens = int(np.maximum(new, 0).sum())
        taken = int(np.maximum(_pages(lens + new) - _pages(lens), 0).sum())
        back = int(np.maximum(_pages(lens) - _pages(lens + new), 0).sum())
        # ids, lengths and changes read; lengths, offsets, slots (8 bytes) and positions written; pages taken and given back
        return {"bytes": case["batch"] * 20 + 4 + tokens * 12 + (taken + back) * 8, "flops": 0}
    row = case["hkv"] * (case["d"] + 8 * (case["d"] // case["group"]))   # a token's codes and scales, K and V
    full = case["hkv"] * case["d"] * 4                                   # the same in 16 bits
    if case["op"] == "write":     # 16-bit rows in, 4-bit rows out; 4-bit rows in, 16-bit rows out
        return {"bytes": case["n"] * (2 * full + 2 * row + 16), "flops": case["n"] * case["hkv"] * case["d"] * 16}
    if case["op"] == "read":
        return {"bytes": case["n"] * (full + row + 8), "flops": case["n"] * case["hkv"] * case["d"] * 4}
    lens = _lens(case)
    tokens = int(lens.sum())
    q = case["batch"] * case["hq"] * case["d"] * 2
    return {"bytes": tokens * row + int(_pages(lens).sum()) * 4 + 2 * q + case["batch"] * (8 + 4 * case["hq"]),
            "flops": 4 * tokens * case["hq"] * case["d"]}


# ------------------------------------------------------ the format, plainly
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _k_shifts(device):
    e = torch.arange(8, device=device)
    return 16 * (e % 2) + 4 * (e // 2)


def _quantise(x, group):
    """[..., D] -> codes (int32) [..., D], s and z [..., D / group] in x's type."""
    y = x.float().reshape(*x.shape[:-1], -1, group)
    lo, hi = y.amin(-1, keepdim=True), y.amax(-1, keepdim=True)
    s = ((hi * 0.5 - lo * 0.5) / 7.5).to(x.dtype).float()
    z = (lo + 8.0 * s).to(x.dtype).float()
    c = torch.where(s > 0, torch.round((y - z) / s) + 8.0, torch.full_like(y, 8.0)).clamp(0.0, 15.0)
    bad = ~torch.isfinite(hi * 0.5 - lo * 0.5)
    s, z = (torch.where(bad, torch.full_like(t, math.nan), t) for t in (s, z))
    c = torch.where(bad, torch.full_like(c, 8.0), c)
    return c.to(torch.int32).reshape(x.shape), s.squeeze(-1).to(x.dtype), z.squeeze(-1).to(x.dtype)


def _bits(x):
    return x.view(torch.int16).to(torch.int32) & 0xFFFF


def _pack_codes(k, v):
    """Codes [N, H, 16, D] -> words [N, H, 16 * D / 8] of K and of V."""
    n, h, _, d = k.shape
    sh = _k_shifts(k.device)
    kw = (k.reshape(n, h, P, d // 32, 4, 8) << sh).sum(-1, dtype=torch.int32).permute(0, 1, 2, 4, 3).reshape(n, h, -1)
    w = v.reshape(n, h, 2, 4, 2, d // 32, 4, 8)                # [token / 8][j][h][i][n][g]
    sv = 16 * torch.arange(2, device=k.device)[:, None, None, None] + 4 * torch.arange(4, device=k.device)[:, None]
    vw = (w << sv).sum((4, 6), dtype=torch.int32).permute(0, 1, 2, 5, 3, 4).reshape(n, h, -1)   # [token / 8][g][j][i]
    return kw, vw


def _pack(k, v, group):
    """K and V [N, H, 16, D] of whole pages -> blocks uint8 [N, H, bytes]."""
    ck, sk, zk = _quantise(k, group)
    cv, sv, zv = _quantise(v, group)
    kw, vw = _pack_codes(ck, cv)
    n, h = kw.shape[:2]
    words = [kw, vw] + [(_bits(s) | (_bits(z) << 16)).reshape(n, h, -1) for s, z in ((sk, zk), (sv, zv))]
    return torch.cat([w.to(torch.int32) for w in words], -1).contiguous().view(torch.uint8)


def _halves(words, dtype):
    pair = words.contiguous().view(torch.int16).reshape(*words.shape, 2).view(dtype).float()
    return pair[..., 0], pair[..., 1]


def _unpack(blocks, d, group, dtype):
    """Blocks uint8 [N, H, bytes] -> K, V in 32 bits [N, H, 16, D]."""
    w = blocks.contiguous().view(torch.int32)
    n, h, _ = w.shape
    c, g = 16 * d // 8, d // group
    sh = _k_shifts(w.device)
    k = (w[..., :c].reshape(n, h, P, 4, d // 32, 1) >> sh) & 15
    k = k.permute(0, 1, 2, 4, 3, 5).reshape(n, h, P, g, group).float()
    sv = 16 * torch.arange(2, device=w.device)[:, None] + 4 * torch.arange(4, device=w.device)
    v = (w[..., c:2 * c].reshape(n, h, 2, 8, 4, d // 32, 1, 1) >> sv) & 15                     # [.., t/8, g, j, i, h, n]
    v = v.permute(0, 1, 2, 4, 6, 5, 7, 3).reshape(n, h, P, g, group).float()
    sk, zk = _halves(w[..., 2 * c:2 * c + P * g].reshape(n, h, P, g, 1), dtype)
    sv, zv = _halves(w[..., 2 * c + P * g:].reshape(n, h, P, g, 1), dtype)
    return (sk * (k - 8.0) + zk).reshape(n, h, P, d), (sv * (v - 8.0) + zv).reshape(n, h, P, d)


def _block_bytes(d, group):
    return 16 * d + 128 * (d // group)


# ----------------------------------------------------------------- prepare
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 11)


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _kv(gen, shape, dtype):
    """K and V as projections give them: K has channels that stand out, and an offset."""
    ch = 1.0 + 3.0 * (torch.rand(shape[-1], generator=gen, device="cuda") > 0.95).float()
    off = 0.5 * torch.randn(shape[-1], generator=gen, device="cuda")
    k = (torch.randn(shape, generator=gen, device="cuda") * ch + off).to(dtype)
    return k, _randn(gen, shape, dtype)


def _fill(gen, num_pages, hkv, d, group, dtype):
    """Blocks of num_pages pages of such K and V."""
    out = torch.empty((num_pages, hkv, _block_bytes(d, group)), dtype=torch.uint8, device="cuda")
    step = max(1, (1 << 26) // (hkv * P * d))
    for a in range(0, num_pages, step):
        b = min(num_pages, a + step)
        k, v = _kv(gen, (b - a, hkv, P, d), dtype)
        out[a:b] = _pack(k, v, group)
    return out


def prepare(case, seed):
    gen = _gen(seed)
    st = {"case": case}
    if case["op"] == "tables":
        lens, new = _changes(case)
        n = case["batch"]
        rows = n + n // 8 + 1                                   # request slots; the batch holds some of them
        width = int(_pages(np.maximum(lens, lens + new)).max()) + 3
        total = int(_pages(np.maximum(lens, lens + new)).sum()) + 64
        perm = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
        ids = torch.randperm(rows, generator=gen, device="cuda")[:n]
        ctx = torch.from_numpy(lens).cuda()
        held = _pages(ctx)
        table = torch.full((rows, width), -1, dtype=torch.int32, device="cuda")
        used = int(held.sum())
        at = torch.repeat_interleave(torch.arange(n, device="cuda"), held)
        col = torch.arange(used, device="cuda") - (held.cumsum(0) - held)[at]
        table[ids[at], col] = perm[:used]
        head = int(torch.randint(0, total, (1,), generator=gen, device="cuda"))
        ring = torch.full((total,), -1, dtype=torch.int32, device="cuda")
        ring[(head + torch.arange(total - used, device="cuda")) % total] = perm[used:]
        slot_lens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        slot_lens[ids] = ctx.to(torch.int32)
        tokens = int(np.maximum(new, 0).sum())
        st |= {"table": table, "ring": ring, "lens": slot_lens, "ids": ids.to(torch.int32),
               "new": torch.from_numpy(new).to(torch.int32).cuda(),
               "free": torch.tensor([head, total - used, 0, 0], dtype=torch.int32, device="cuda"),
               "slots": torch.empty(tokens, dtype=torch.int64, device="cuda"),
               "positions": torch.empty(tokens, dtype=torch.int32, device="cuda"),
               "cu": torch.empty(n + 1, dtype=torch.int32, device="cuda"),
               "lens_out": torch.empty_like(slot_lens), "free_out": torch.zeros(4, dtype=torch.int32, device="cuda")}
        if own:
            from paper_2603_12707_gb300 import kv4
            st["tables"] = kv4.Tables(st["table"], st["lens"], st["ring"], st["free"])
        return st
    d, group, hkv, dt = case["d"], case["group"], case["hkv"], _dtype(case)
    if case["op"] in ("write", "read"):
        n = case["n"]
        num_pages = _pages(n) + n // 50 + 3
        if case["order"] == "runs":      # consecutive tokens in pages of any order, starting inside a page
            pages = torch.randperm(num_pages, generator=gen, device="cuda")
            pos = torch.arange(n, device="cuda") + 5
            slots = pages[pos // P] * P + pos % P
        else:
            slots = torch.randperm(num_pages * P, generator=gen, device="cuda")[:n]
        st["slots"] = slots
        if case["op"] == "write":
            st["pool"] = torch.zeros((num_pages, hkv, _block_bytes(d, group)), dtype=torch.uint8, device="cuda")
            k, v = _kv(gen, (n, hkv, d), dt)
            if case["fused_qkv"]:        # K and V are slices of a fused projection's rows
                row = torch.zeros((n, 3 * hkv, d), dtype=dt, device="cuda")
                row[:, hkv:2 * hkv], row[:, 2 * hkv:] = k, v
                k, v = row[:, hkv:2 * hkv], row[:, 2 * hkv:]
            st["k"], st["v"] = k, v
        else:
            st["pool"] = _fill(gen, num_pages, hkv, d, group, dt)
        st["k_out"], st["v_out"] = (torch.empty((n, hkv, d), dtype=dt, device="cuda") for _ in range(2))
    else:
        lens, b = _lens(case), case["batch"]
        width = int(_pages(lens).max()) + 1
        used = int(_pages(lens).sum())
        num_pages = used + 2
        st["pool"] = _fill(gen, num_pages, hkv, d, group, dt)
        perm = torch.randperm(num_pages, generator=gen, device="cuda").to(torch.int32)
        held = torch.from_numpy(_pages(lens)).cuda()
        table = torch.full((b, width), -1, dtype=torch.int32, device="cuda")
        at = torch.repeat_interleave(torch.arange(b, device="cuda"), held)
        table[at, torch.arange(used, device="cuda") - (held.cumsum(0) - held)[at]] = perm[:used]
        st |= {"table": table, "lens": torch.from_numpy(lens).to(torch.int32).cuda()}
        q = _randn(gen, (b, case["hq"] + 2 * hkv, d), dt)
        st["q"] = q[:, :case["hq"]] if case["fused_qkv"] else q[:, :case["hq"]].contiguous()
        st["out"] = torch.empty((b, case["hq"], d), dtype=dt, device="cuda")
        st["lse"] = torch.empty((b, case["hq"]), dtype=torch.float32, device="cuda")
    if own:
        from paper_2603_12707_gb300 import kv4
        st["handle"] = kv4.Pool(st["pool"], d, group, dt)
        if case["op"] == "attention":
            st["tables"] = kv4.Tables(st["table"], st["lens"])
            st["work"] = kv4.kv4_workspace(st["handle"], case["hq"])
    return st


# --------------------------------------------------------------------- run
def _run_tables(st):
    ids, new, table, ring = st["ids"].long(), st["new"].long(), st["table"], st["ring"]
    head, count = st["free"][0].long(), st["free"][1].long()
    size, room = ring.numel(), st["slots"].numel()
    ctx = st["lens"][ids].long()
    end = ctx + new
    fine = (end >= 0) & (end <= table.shape[1] * P)
    grow = new.clamp(min=0)
    stop = grow.cumsum(0)
    need = torch.where(fine, (_pages(end) - _pages(ctx)).clamp(min=0), 0)
    take = need.cumsum(0)
    ok = fine & (stop <= room) & ((need == 0) | (take <= count))
    cu = torch.cat([torch.zeros_like(stop[:1]), stop])
    # every new token's request, position and slot
    t = torch.arange(room, device=ids.device)
    r = torch.searchsorted(stop, t, right=True)
    live = r < ids.numel()
    r = r.clamp(max=ids.numel() - 1)
    live = live & ok[r]
    pos = ctx[r] + t - cu[r]
    page = pos // P
    fresh = page >= _pages(ctx)[r]
    col = page.clamp(0, table.shape[1] - 1)
    taken = ring[(head + (take - need)[r] + page - _pages(ctx)[r]).clamp(min=0) % size].long()
    where = torch.where(fresh, taken, table[ids[r], col].long())
    st["slots"].copy_(torch.where(live, where * P + pos % P, -1))
    st["positions"].copy_(torch.where(live, pos, -1))
    st["cu"].copy_(cu)
    # the new entries of the tables
    opens = live & fresh & (pos % P == 0)
    held = torch.where(opens, taken, table[ids[r], col].long())
    row = torch.where(opens, ids[r], table.shape[0])           # a row of its own takes what opens no page
    wide = torch.cat([table, table[:1]])
    wide[row, col] = held.to(torch.int32)
    table.copy_(wide[:-1])
    # pages given back, in batch order, to the end of the ring
    back = torch.where(ok, (_pages(ctx) - _pages(end)).clamp(min=0), 0)
    given = back.cumsum(0)
    total = torch.where(ok, need, 0).sum()
    k = torch.arange(size, device=ids.device)
    rr = torch.searchsorted(given, k, right=True)
    real = rr < ids.numel()
    rr = rr.clamp(max=ids.numel() - 1)
    c2 = (_pages(end)[rr] + k - (given - back)[rr]).clamp(0, table.shape[1] - 1)
    place = torch.where(real, (head + count + k) % size, size)
    longer = torch.cat([ring, ring[:1]])
    longer[place] = table[ids[rr], c2]
    ring.copy_(longer[:-1])
    lens = st["lens"].clone()
    lens[ids] = torch.where(ok, end, ctx).to(torch.int32)
    st["lens_out"].copy_(lens)
    st["free_out"][0] = (head + total) % size
    st["free_out"][1] = count - total + given[-1]


def _slots_read(st, d, group, dt):
    """K and V of every slot in 32 bits, [n][H][D]: the blocks of the slots' pages, unpacked once a page."""
    slots, pool = st["slots"], st["pool"]
    k, v = _unpack(pool, d, group, dt)
    return k[slots // P, :, slots % P], v[slots // P, :, slots % P]


def _run_write(st, d, group):
    slots, pool = st["slots"], st["pool"]
    n_pages, h, _ = pool.shape
    words = pool.view(torch.int32)
    c, g = 2 * d, d // group
    kw = torch.zeros((n_pages, h, P, d), dtype=torch.int32, device=pool.device)
    vw = torch.zeros_like(kw)
    meta = words[..., 2 * c:].reshape(n_pages, h, 2, P, g).clone()
    for x, codes, side in ((st["k"], kw, 0), (st["v"], vw, 1)):
        q, s, z = _quantise(x, group)
        codes[slots // P, :, slots % P] = q
        meta[slots // P, :, side, slots % P] = _bits(s.contiguous()) | (_bits(z.contiguous()) << 16)
    kw, vw = _pack_codes(kw, vw)
    words.copy_(torch.cat([kw, vw, meta.reshape(n_pages, h, -1)], -1))


def _run_attention(st, case, dt):
    d, group, hkv, hq = case["d"], case["group"], case["hkv"], case["hq"]
    b, g = st["q"].shape[0], hq // hkv
    table = st["table"][:, :-1] if st["table"].shape[1] > 1 else st["table"]
    k, v = _unpack(st["pool"], d, group, dt)
    rows = table.clamp(min=0).long()
    k = k[rows].permute(0, 2, 1, 3, 4).reshape(b, hkv, -1, d)
    v = v[rows].permute(0, 2, 1, 3, 4).reshape(b, hkv, -1, d)
    scale = case["scale"] or d ** -0.5
    q = st["q"].float().reshape(b, hkv, g, d) * scale
    s = q @ k.transpose(-1, -2)
    t = torch.arange(s.shape[-1], device=s.device)
    gone = (t >= st["lens"][:, None])[:, None, None]
    s = s.masked_fill(gone, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.zeros_like(top))
    p = torch.exp(s - top)
    l = p.sum(-1, keepdim=True)
    o = (p @ v) / torch.where(l > 0, l, torch.ones_like(l))
    st["out"].copy_(o.reshape(b, hq, d))
    st["lse"].copy_((top + torch.log(l)).reshape(b, hq))


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2603_12707_gb300 import kv4
        if op == "tables":
            kv4.kv_tables_step(st["tables"], st["ids"], st["new"], st["slots"], st["positions"], st["cu"],
                               lens_out=st["lens_out"], free_state_out=st["free_out"])
        elif op == "attention":
            kv4.kv4_decode_attention(st["handle"], st["tables"], st["q"], st["out"], st["work"], lse=st["lse"],
                                     softmax_scale=case["scale"])
        else:
            if op == "write":
                kv4.kv4_write(st["handle"], st["slots"], st["k"], st["v"])
            kv4.kv4_read(st["handle"], st["slots"], st["k_out"], st["v_out"])
    elif op == "tables":
        _run_tables(st)
    elif op == "attention":
        _run_attention(st, case, _dtype(case))
    else:
        if op == "write":
            _run_write(st, case["d"], case["group"])
        k, v = _slots_read(st, case["d"], case["group"], _dtype(case))
        st["k_out"].copy_(k)
        st["v_out"].copy_(v)
    if op == "tables":
        return {n: st[n] for n in ("slots", "positions", "cu", "table", "ring", "lens_out", "free_out")}
    if op == "attention":
        return {"out": st["out"], "lse": st["lse"]}
    return {"k": st["k_out"], "v": st["v_out"]}


# ------------------------------------------------------------------- exact
def _exact_rows(x, group):
    """What x [n, H, D] is held as, in 64 bits, from the definition of the format."""
    y = x.double().unflatten(-1, (-1, group))
    lo, hi = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
    s = ((hi - lo) / 15).to(x.dtype).double()
    z = (lo + 8 * s).to(x.dtype).double()
    c = torch.clamp(torch.round((y - z) / torch.where(s > 0, s, 1.0)) + 8, 0, 15)
    return (s * (c - 8) + z).flatten(-2)


def _exact_tokens(blocks, d, group, dtype):
    """K and V of one KV head's pages [N, bytes] in 64 bits [16 N, D]: byte by byte."""
    n = blocks.shape[0]
    low, high = blocks & 15, blocks >> 4
    nib = torch.stack([low, high], -1).flatten(-2).double()     # codes in the order of their bits
    half = 16 * d
    e, i, j, t = (torch.arange(m, device=blocks.device) for m in (d, d, d, P))
    i, j, e = e // 32, (e // 8) % 4, e % 8
    at_k = (t[:, None] * 4 + j) * (d // 32) * 8 + i * 8 + 4 * (e % 2) + e // 2
    dd = torch.arange(d, device=blocks.device)
    at_v = (((t // 8)[:, None] * 8 + dd % 8) * 4 + ((t % 8) // 2)[:, None]) * (d // 32) * 8 + (dd // 32) * 8 \
        + 4 * (t % 2)[:, None] + (dd // 8) % 4
    meta = blocks[:, 16 * d:].contiguous().view(dtype).double().reshape(n, 2, P, d // group, 2)
    out = []
    for side, at in ((0, at_k), (1, half + at_v)):
        s, z = (meta[:, side, :, :, w].repeat_interleave(group, -1) for w in (0, 1))
        out.append((s * (nib[:, at.flatten()].reshape(n, P, d) - 8) + z).reshape(n * P, d))
    return out


def exact(case, seed):
    if case["op"] == "tables":
        return None
    st = prepare(case, seed)
    d, group, dt = case["d"], case["group"], _dtype(case)
    if case["op"] == "write":
        return {"k": _exact_rows(st["k"], group), "v": _exact_rows(st["v"], group)}
    if case["op"] == "read":
        out = [torch.empty(st["k_out"].shape, dtype=torch.float64, device="cuda") for _ in range(2)]
        for h in range(case["hkv"]):
            for o, x in zip(out, _exact_tokens(st["pool"][:, h], d, group, dt)):
                o[:, h] = x[st["slots"]]
        return {"k": out[0], "v": out[1]}
    if int(_lens(case).sum()) * case["hq"] > 12_000_000:
        return None
    out = torch.zeros(st["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    g = case["hq"] // case["hkv"]
    scale = case["scale"] or 1.0 / math.sqrt(d)
    for b, n in enumerate(int(x) for x in _lens(case)):
        if not n:
            continue
        pages = st["table"][b, :_pages(n)].long()
        for h in range(case["hkv"]):
            k, v = (x[:n] for x in _exact_tokens(st["pool"][pages, h], d, group, dt))
            s = st["q"][b, h * g:(h + 1) * g].double() @ k.T * scale
            w = torch.softmax(s, -1)
            out[b, h * g:(h + 1) * g] = w @ v
            lse[b, h * g:(h + 1) * g] = torch.logsumexp(s, -1)
    return {"out": out, "lse": lse}

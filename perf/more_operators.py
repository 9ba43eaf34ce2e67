"""Cases of a serving step on a 16-bit paged cache: rotation of queries and keys, the write of rotated keys, and decode attention
of requests that share a prefix.

* ``rope``: norms of queries and keys for each head (optional) and their rotation by positions of one or three axes
  (time, height, width), in one pass over the rows of a packed batch.
* ``write``: the same with the rotated keys, and the values, going into their slots of a paged cache.
* ``attention``: one decode step.  Every row attends to the tokens of the prefix that it shares with others (an image or a
  video that several requests ask about, a system prompt), then to its own; the step's plan once, then the layers' calls.

The formulas.  With a norm, y = x / sqrt(mean(x^2) + eps) * w over the elements of a head, else y = x.  Pair j of the first
``rd`` elements (j and j + rd / 2, or 2 j and 2 j + 1) is turned by the angle pos[axis_j] * base^(-2 j / rd).  Attention:
o = sum_t softmax_t(q . k_t / sqrt(d)) v_t, and the natural logarithm of the softmax's denominator.

A pool is K and V of [pages][KV heads][16 tokens][d].  Lengths and groups are a function of the case alone (``lens_seed``), so
``work`` is exact; values, positions and page orders come from ``prepare``'s seed.
"""
import math

import numpy as np
import torch

own = False

P = 16            # tokens per page
EPS = 1e-6


# ------------------------------------------------------------------- cases
def _rows(name, op, hq, hkv, d, n, dtype="bf16", rd=0, pairs="halves", axes="one", norm=False, fused_qkv=False, where="prompt",
          far=0, base=1e6):
    return {"name": name, "op": op, "hq": hq, "hkv": hkv, "d": d, "n": n, "dtype": dtype, "rd": rd or d, "pairs": pairs,
            "axes": axes, "norm": norm, "fused_qkv": fused_qkv, "where": where, "far": far, "base": base}


def _attention(name, hq, hkv, d, batch, groups, plo, phi, olo, ohi, layers=1, dtype="bf16", alone=0, fused_qkv=False, lens_seed=1):
    return {"name": name, "op": "attention", "hq": hq, "hkv": hkv, "d": d, "batch": batch, "groups": groups, "plo": plo, "phi": phi,
            "olo": olo, "ohi": ohi, "layers": layers, "dtype": dtype, "alone": alone, "fused_qkv": fused_qkv, "lens_seed": lens_seed}


def listed():
    return [
        # A decode step of the GQA batch: one token each, three axes, far into long contexts.  Latency.
        _rows("rope_decode_gqa_b32", "rope", 28, 4, 128, 32, axes="sections", where="decode", far=1000000, fused_qkv=True),
        # A ragged prompt chunk of text and images with normed heads, in fp16, axes that take turns.
        _rows("rope_chunk_norm_5003", "rope", 16, 8, 128, 5003, dtype="fp16", axes="turns", norm=True, fused_qkv=True),
        # A request at d 64 of which half a head is rotated, neighbouring pairs.
        _rows("rope_partial_d64_631", "rope", 14, 2, 64, 631, rd=32, pairs="neighbours", base=1e4),
        # The GQA batch's prompts: 32 requests of a vision prefix and text.
        _rows("rope_prompts_gqa_49152", "rope", 28, 4, 128, 49152, axes="sections", fused_qkv=True),
        # One decoded token per request of the MHA batch: what a layer appends in every step.
        _rows("write_decode_mha_b64", "write", 32, 32, 128, 64, where="decode", far=4096, base=1e4, fused_qkv=True),
        # A ragged prompt chunk with normed heads on a GQA shape, fp16.
        _rows("write_chunk_gqa_4999", "write", 24, 3, 128, 4999, dtype="fp16", axes="turns", norm=True),
        # The MHA batch's prompts: 64 requests of 576 vision tokens and some text.
        _rows("write_prompts_mha_40960", "write", 32, 32, 128, 40960, base=1e4, fused_qkv=True),
        # Four questions about one image, just begun: latency, four layers of a step.
        _attention("attn_image_gqa_b4", 28, 4, 128, 4, 1, 1369, 1369, 0, 64, layers=4, fused_qkv=True),
        # The MHA batch: all ask about one picture and share its 576 tokens and the instructions; each has its own text.
        _attention("attn_mha_b64", 32, 32, 128, 64, 1, 701, 701, 64, 768, layers=2),
        # Several documents and pictures, some rows without, ragged, d 64, fp16.
        _attention("attn_groups_b150", 14, 2, 64, 150, 11, 1, 9000, 0, 700, dtype="fp16", alone=17, layers=2),
        # A long multi-image context that the GQA batch shares.
        _attention("attn_long_gqa_b32", 28, 4, 128, 32, 1, 32768, 32768, 32, 512, fused_qkv=True),
        # An hour of video that many ask about: more rows than bytes can hide.
        _attention("attn_video_gqa_b96", 28, 4, 128, 96, 1, 131009, 131009, 1, 300),
    ]


HEADS = ((8, 8), (32, 32), (28, 4), (14, 2), (16, 2), (5, 5), (12, 4), (7, 1), (24, 3), (40, 8))


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    costs = [_cost(c) for c in listed()]
    while True:
        op = rng.choice(("rope", "write", "attention", "attention"))
        dtype = rng.choice(("bf16", "fp16"))
        d = rng.choice((64, 128))
        hq, hkv = rng.choice(HEADS)
        if op == "attention":
            batch = _log(rng, 1, 200)
            groups = min(batch, _log(rng, 1, 24))
            phi = _log(rng, 1, 60000)
            ohi = _log(rng, 1, 4000)
            c = _attention("", hq, hkv, d, batch, groups, rng.randint(0, phi), phi, rng.randint(0, ohi), ohi, rng.choice((1, 2, 4)),
                           dtype, rng.randint(0, batch - groups) if rng.random() < 0.5 else 0, rng.random() < 0.5,
                           rng.randint(1, 10 ** 6))
            lens = _lens(c)
            most = int(np.bincount(lens[1][lens[1] >= 0], minlength=1).max())
            # what the padded plain form may take: scores of every group and row, K and V of both, in 32 bits
            if max(groups * most * hq * phi, groups * phi * hkv * d * 2, batch * ohi * (hq + 2 * hkv * d)) > 2 ** 31:
                continue
        else:
            c = _rows("", op, hq, hkv, d, _log(rng, 1, 50000), dtype, rng.choice((d, d, d // 2)), rng.choice(("halves", "neighbours")),
                      rng.choice(("one", "sections", "turns")), rng.random() < 0.5, rng.random() < 0.5,
                      rng.choice(("prompt", "decode")), rng.choice((0, 4096, 1000000)), rng.choice((1e4, 5e5, 1e6)))
        if _cost(c) <= max(costs):
            del c["name"]
            return c


# ------------------------------------------------------- lengths and bytes
def _pages(n):
    return (n + P - 1) // P


def _lens(case):
    """Prefix lengths [groups], the group of every row (-1: none), own lengths [batch]."""
    r = np.random.Generator(np.random.PCG64([case["lens_seed"], 3]))
    prefix = r.integers(case["plo"], case["phi"], size=case["groups"], endpoint=True)
    shared = case["batch"] - case["alone"]
    cuts = np.sort(r.choice(np.arange(1, shared), size=case["groups"] - 1, replace=False)) if case["groups"] > 1 else np.zeros(0, int)
    group = np.full(case["batch"], -1)
    group[:shared] = np.searchsorted(cuts, np.arange(shared), side="right")
    return prefix, group, r.integers(case["olo"], case["ohi"], size=case["batch"], endpoint=True)


def work(case):
    d, hq, hkv = case["d"], case["hq"], case["hkv"]
    if case["op"] == "attention":
        prefix, group, mine = _lens(case)
        of_row = np.where(group >= 0, prefix[group], 0)
        tokens = int(prefix[np.unique(group[group >= 0])].sum() + mine.sum())
        ids = int(_pages(prefix).sum() + _pages(mine).sum()) * 4
        row = case["batch"] * hq * (4 * d + 4)
        return {"bytes": case["batch"] * 12 + ids + case["layers"] * (tokens * 4 * hkv * d + row),
                "flops": case["layers"] * 4 * hq * d * int((of_row + mine).sum())}
    heads = 2 * hq + 2 * hkv + (2 * hkv if case["op"] == "write" else 0)
    each = 2 * heads * d + 4 * (1 if case["axes"] == "one" else 3) + (8 if case["op"] == "write" else 0)
    return {"bytes": case["n"] * each, "flops": case["n"] * (hq + hkv) * (3 * case["rd"] + (4 * d if case["norm"] else 0))}


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 280)


# ----------------------------------------------------------------- prepare
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 6007 + 29)


def _randn(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32) * scale).to(dtype)


def _keys(gen, shape, dtype):
    """Keys as projections give them: channels that stand out, and an offset."""
    ch = 1.0 + 3.0 * (torch.rand(shape[-1], generator=gen, device="cuda") > 0.95).float()
    off = 0.5 * torch.randn(shape[-1], generator=gen, device="cuda")
    x = torch.empty(shape, dtype=dtype, device="cuda")
    step = max(1, (1 << 27) // max(1, int(np.prod(shape[1:]))))
    for a in range(0, shape[0], step):
        y = torch.randn((min(step, shape[0] - a), *shape[1:]), generator=gen, device="cuda")
        x[a:a + step] = (y * ch + off).to(dtype)
    return x


def _frequencies(case):
    half = case["rd"] // 2
    return [case["base"] ** (-j / half) for j in range(half)]


def _axes(case):
    """The axis of each pair."""
    half = case["rd"] // 2
    if case["axes"] == "one":
        return [0] * half
    if case["axes"] == "turns":
        return [j % 3 for j in range(half)]
    return [0] * (half // 4) + [1] * (3 * half // 8) + [2] * (half - half // 4 - 3 * half // 8)


def _positions(case, seed):
    """Positions [axes][n]: of text and images as a processor lays them out, or of one decoded token per request."""
    r = np.random.Generator(np.random.PCG64([seed, 5]))
    n, axes = case["n"], 1 if case["axes"] == "one" else 3
    if case["where"] == "decode":
        return np.repeat(r.integers(0, case["far"] + 1024, size=(1, n)), axes, 0).astype(np.int32)
    parts, at, have = [], int(r.integers(0, case["far"] + 1)), 0
    while have < n:
        if r.random() < 0.5:
            k = int(r.integers(5, 300))
            block = np.repeat(at + np.arange(k)[None], 3, 0)
        else:
            t, h, w = int(r.choice((1, 1, 4))), int(r.integers(8, 40)), int(r.integers(8, 40))
            block = at + np.stack(np.meshgrid(np.arange(t), np.arange(h), np.arange(w), indexing="ij")).reshape(3, -1)
        parts.append(block)
        have += block.shape[1]
        at = int(block.max()) + 1
    return np.concatenate(parts, 1)[:axes, :n].astype(np.int32)


def _table(gen, lens, pages, free):
    """Block tables of the requests with shuffled pages; the entries past a request's own are -1."""
    held = torch.from_numpy(_pages(lens)).cuda()
    used, width = int(held.sum()), max(1, int(_pages(lens).max()))
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    at = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), held)
    table[at, torch.arange(used, device="cuda") - (held.cumsum(0) - held)[at]] = order[:used]
    return table


def prepare(case, seed):
    gen, dt, d, hq, hkv = _gen(seed), _dtype(case), case["d"], case["hq"], case["hkv"]
    st = {"case": case}
    if case["op"] == "attention":
        prefix, group, mine = _lens(case)
        b, ng = case["batch"], case["groups"]
        lens = np.concatenate([mine, prefix])           # requests: the rows' own, then the prefixes
        pages = int(_pages(lens).sum()) + 3
        st["table"] = _table(gen, lens, pages, 3)
        st["lens"] = torch.from_numpy(lens).to(torch.int32).cuda()
        st["seq_ids"] = torch.arange(b, dtype=torch.int32, device="cuda")
        st["prefix_ids"] = torch.from_numpy(np.where(group >= 0, b + group, -1)).to(torch.int32).cuda()
        # which row is the i-th of its group (the plain form works on padded groups)
        first = np.searchsorted(group[:b - case["alone"]], np.arange(ng))
        place = np.where(group >= 0, np.arange(b) - first[group], 0)
        st |= {"group": torch.from_numpy(group).cuda(), "place": torch.from_numpy(place).cuda(), "most": int(place.max()) + 1,
               "width": [max(1, int(_pages(x).max())) for x in (mine, prefix)]}
        shape = (pages, hkv, P, d)
        st["k"] = [_keys(gen, shape, dt) for _ in range(case["layers"])]
        st["v"] = [_randn(gen, shape, dt) for _ in range(case["layers"])]
        q = [_randn(gen, (b, hq + 2 * hkv, d), dt) for _ in range(case["layers"])]
        st["q"] = [x[:, :hq] if case["fused_qkv"] else x[:, :hq].contiguous() for x in q]
        st["out"] = [torch.empty((b, hq, d), dtype=dt, device="cuda") for _ in range(case["layers"])]
        st["lse"] = [torch.empty((b, hq), dtype=torch.float32, device="cuda") for _ in range(case["layers"])]
        if own:
            from paper_2603_12707_gb300 import kv4, kv16
            st["pools"] = [kv16.Pool(k, v) for k, v in zip(st["k"], st["v"])]
            st["tables"] = kv4.Tables(st["table"], st["lens"])
            st["work"] = kv16.kv16_workspace(st["pools"][0], hq, b)
        return st
    n = case["n"]
    rows = torch.empty((n, hq + 2 * hkv, d), dtype=dt, device="cuda")
    rows[:, :hq] = _randn(gen, (n, hq, d), dt, 2.0)
    rows[:, hq:hq + hkv] = _keys(gen, (n, hkv, d), dt)
    rows[:, hq + hkv:] = _randn(gen, (n, hkv, d), dt)
    q, k, v = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    st["q"], st["k"], st["v"] = (q, k, v) if case["fused_qkv"] else (q.contiguous(), k.contiguous(), v.contiguous())
    st["positions"] = torch.from_numpy(_positions(case, seed)).cuda()
    st["frequencies"] = torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda")
    st["axes"] = torch.tensor(_axes(case), device="cuda")
    st["qw"], st["kw"] = ((1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dt) if case["norm"] else None for _ in range(2))
    st["q_out"] = torch.empty((n, hq, d), dtype=dt, device="cuda")
    st["k_out"] = torch.empty((n, hkv, d), dtype=dt, device="cuda")
    if case["op"] == "write":
        pages = _pages(n + 5) + n // 50 + 3
        order = torch.randperm(pages, generator=gen, device="cuda")
        at = torch.arange(n, device="cuda") + 5        # a run of tokens that starts inside a page
        if case["where"] == "decode":                  # every token in a page of its own request
            pages = n + 3
            order, at = torch.randperm(pages, generator=gen, device="cuda"), torch.arange(n, device="cuda") * P + 7
        st["slots"] = order[at // P] * P + at % P
        st["k_pool"], st["v_pool"] = (torch.zeros((pages, hkv, P, d), dtype=dt, device="cuda") for _ in range(2))
    if own:
        from paper_2603_12707_gb300 import kv16
        st["rope"] = kv16.Rope(_frequencies(case), axes=_axes(case), num_axes=st["positions"].shape[0],
                               neighbours=case["pairs"] == "neighbours")
        if case["op"] == "write":
            st["pool"] = kv16.Pool(st["k_pool"], st["v_pool"])
    return st


# --------------------------------------------------------------------- run
def _turned(st, x, w):
    """Rows x [n][heads][d] normed and rotated, in 32 bits (the angles in 64)."""
    case = st["case"]
    rd, half = case["rd"], case["rd"] // 2
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    angle = st["positions"][st["axes"]].t().double() * st["frequencies"]        # [n][rd / 2]
    c, s = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    if case["pairs"] == "halves":
        a, b = y[..., :half], y[..., half:rd]
        return torch.cat([a * c - b * s, b * c + a * s, y[..., rd:]], -1)
    a, b = y[..., 0:rd:2], y[..., 1:rd:2]
    return torch.cat([torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2), y[..., rd:]], -1)


def _partial(q, k, v, gone):
    """Attention of q [.., R, d] over k, v [.., T, d] in 32 bits where gone [.., 1, T] is false: o unnormalised, top, denominator."""
    s = (q @ k.transpose(-1, -2)).masked_fill_(gone, -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, torch.full_like(top, -1e30))
    p = torch.exp_(s.sub_(top))
    return p @ v, top, p.sum(-1, keepdim=True)


def _tokens(pool, table):
    """Rows of pages -> tokens [rows][KV heads][T][d] in 32 bits."""
    x = pool[table.clamp(min=0).long()]
    return x.permute(0, 2, 1, 3, 4).flatten(2, 3).float()


def _attend(st, layer):
    case = st["case"]
    b, hq, hkv, d, ng = case["batch"], case["hq"], case["hkv"], case["d"], case["groups"]
    g = hq // hkv
    q = st["q"][layer].float().reshape(b, hkv, g, d) * d ** -0.5
    k, v, lens, table = st["k"][layer], st["v"][layer], st["lens"], st["table"]
    t_own, t_pre = table[:b, :st["width"][0]], table[b:, :st["width"][1]]
    t = torch.arange(max(st["width"]) * P, device=q.device)
    # own tokens, row by row
    o1, m1, l1 = _partial(q, _tokens(k, t_own), _tokens(v, t_own), (t[:st["width"][0] * P] >= lens[:b, None])[:, None, None])
    # the prefixes, group by group, over padded groups of rows
    held = st["group"] >= 0
    at, place = st["group"].clamp(min=0), st["place"]
    padded = torch.zeros((ng, st["most"], hkv, g, d), device=q.device)
    padded[at[held], place[held]] = q[held]
    padded = padded.permute(0, 2, 1, 3, 4).reshape(ng, hkv, st["most"] * g, d)
    o2, m2, l2 = _partial(padded, _tokens(k, t_pre), _tokens(v, t_pre), (t[:st["width"][1] * P] >= lens[b:, None])[:, None, None])
    o2, m2, l2 = (x.reshape(ng, hkv, st["most"], g, -1)[at, :, place] for x in (o2, m2, l2))
    l2 = l2 * held[:, None, None, None]
    m2 = torch.where(l2 > 0, m2, torch.full_like(m2, -1e30))
    # both together
    top = torch.maximum(m1, m2)
    w1, w2 = torch.exp(m1 - top), torch.exp(m2 - top) * held[:, None, None, None]
    l = l1 * w1 + l2 * w2
    o = (o1 * w1 + o2 * w2) / torch.where(l > 0, l, torch.ones_like(l))
    st["out"][layer].copy_(o.reshape(b, hq, d))
    st["lse"][layer].copy_((top + torch.log(l)).reshape(b, hq))


def run(st):
    case = st["case"]
    op = case["op"]
    if own:
        from paper_2603_12707_gb300 import kv16
        if op == "rope":
            kv16.kv_qk_rope(st["rope"], st["positions"], st["q"], st["k"], st["q_out"], st["k_out"], q_weight=st["qw"],
                            k_weight=st["kw"], eps=EPS)
        elif op == "write":
            kv16.kv16_write(st["pool"], st["slots"], st["k"], st["v"], rope=st["rope"], positions=st["positions"], q=st["q"],
                            q_out=st["q_out"], q_weight=st["qw"], k_weight=st["kw"], eps=EPS)
        else:
            kv16.kv16_plan(st["pools"][0], st["tables"], case["hq"], case["batch"], st["work"], seq_ids=st["seq_ids"],
                           prefix_ids=st["prefix_ids"])
            for pool, q, out, lse in zip(st["pools"], st["q"], st["out"], st["lse"]):
                kv16.kv16_attention(pool, st["tables"], q, out, st["work"], lse=lse)
    elif op == "attention":
        [_attend(st, layer) for layer in range(case["layers"])]
    else:
        st["q_out"].copy_(_turned(st, st["q"], st["qw"]))
        k = _turned(st, st["k"], st["kw"])
        if op == "rope":
            st["k_out"].copy_(k)
        else:
            page, tok = st["slots"] // P, st["slots"] % P
            st["k_pool"][page, :, tok] = k.to(st["k"].dtype)
            st["v_pool"][page, :, tok] = st["v"]
    if op == "attention":
        return {"out": st["out"], "lse": st["lse"]}
    if op == "write":
        return {"q": st["q_out"], "k": st["k_pool"], "v": st["v_pool"]}
    return {"q": st["q_out"], "k": st["k_out"]}


# ------------------------------------------------------------------- exact
def _exact_rows(st, x, w):
    """The rotation as a product of complex numbers, in 64 bits."""
    case = st["case"]
    half = case["rd"] // 2
    y = x.double()
    if w is not None:
        y = w.double() * y / torch.sqrt(y.pow(2).sum(-1, keepdim=True) / case["d"] + EPS)
    turned = y[..., :case["rd"]]
    pair = turned.unflatten(-1, (2, half)).transpose(-1, -2) if case["pairs"] == "halves" else turned.unflatten(-1, (half, 2))
    f = torch.tensor([case["base"] ** (-2.0 * j / case["rd"]) for j in range(half)], dtype=torch.float64, device="cuda")
    pos = torch.stack([st["positions"][a] for a in _axes(case)], -1)
    turn = torch.polar(torch.ones_like(f), pos.double() * f)[:, None]
    z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    z = z.transpose(-1, -2).flatten(-2) if case["pairs"] == "halves" else z.flatten(-2)
    return torch.cat([z, y[..., case["rd"]:]], -1)


def exact(case, seed):
    st = prepare(case, seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] != "attention":
        q, k = _exact_rows(st, st["q"], st["qw"]), _exact_rows(st, st["k"], st["kw"])
        if case["op"] == "rope":
            return {"q": q, "k": k}
        pools = []
        for rows, pool in ((k, st["k_pool"]), (st["v"], st["v_pool"])):
            flat = pool.double().transpose(1, 2).reshape(-1, hkv, d)
            flat[st["slots"]] = rows.double()
            pools.append(flat.reshape(-1, P, hkv, d).transpose(1, 2))
        return {"q": q, "k": pools[0], "v": pools[1]}
    prefix, group, mine = _lens(case)
    outs, lses, g = [], [], hq // hkv
    for layer in range(case["layers"]):
        out = torch.zeros((case["batch"], hq, d), dtype=torch.float64, device="cuda")
        lse = torch.full((case["batch"], hq), -math.inf, dtype=torch.float64, device="cuda")
        cut = lambda pool, req, n, h: pool[st["table"][req, :_pages(n)].long(), h].reshape(-1, d)[:n].double()  # noqa: E731
        for h in range(hkv):
            heads = slice(h * g, (h + 1) * g)
            shared = {}
            for r in range(case["batch"]):
                q = st["q"][layer][r, heads].double() / math.sqrt(d)
                keys, values = (cut(p[layer], r, int(mine[r]), h) for p in (st["k"], st["v"]))
                s, parts = q @ keys.T, [values]
                if group[r] >= 0:
                    if group[r] not in shared:
                        n, rows = int(prefix[group[r]]), np.flatnonzero(group == group[r])
                        a, z = (cut(p[layer], case["batch"] + int(group[r]), n, h) for p in (st["k"], st["v"]))
                        shared = {group[r]: (a, z, (st["q"][layer][rows[0]:rows[-1] + 1, heads].double() / math.sqrt(d)) @ a.T, rows[0])}
                    _, z, scores, first = shared[group[r]]
                    s, parts = torch.cat([scores[r - first], s], -1), [z, values]
                if s.shape[-1] == 0:
                    continue
                lse[r, heads] = torch.logsumexp(s, -1)
                p = torch.exp(s - lse[r, heads, None])
                n = p.shape[-1] - parts[-1].shape[0]
                out[r, heads] = p[:, n:] @ parts[-1] + (p[:, :n] @ parts[0] if len(parts) == 2 else 0.0)
        outs.append(out)
        lses.append(lse)
    return {"out": outs, "lse": lses}

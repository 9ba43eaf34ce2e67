"""Plain reference of the 16-bit serving step for the tests: norms and rotations in 64 bits, attention over a shared
prefix and a row's own tokens in 64 bits, each with what the arithmetic of kvdecode16.h may differ by."""
import math

import numpy as np
import torch

P = 16
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # a rounding's relative error
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # and its least absolute one


def pages_of(n):
    return (n + P - 1) // P


def inv_freq(half, base=1e4):
    return [base ** (-j / half) for j in range(half)]


def turned(x, positions, freq, axes, neighbours=False, scale=1.0, weight=None, eps=1e-6):
    """x [n, heads, d] (16 bits) -> (normed and rotated, bound) in 64 bits.

    The bound: a norm's sum of d <= 128 squares in 32 bits, its root and two products are off by less than 24 steps of
    2^-24 (16 in a lane, 3 across, 5 after); an angle by 2^-25 of half a turn and 2^-32 of a turn; sine and cosine by two
    steps; four products and sums: together below 2^-18 of the pair's elements."""
    y = x.double()
    n, _, d = y.shape
    if weight is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * weight.double()
    half = len(freq)
    if half == 0:
        return y, 2.0 ** -18 * y.abs()
    pos = torch.as_tensor(np.asarray(positions), dtype=torch.float64).reshape(-1, n)
    ax = [0] * half if axes is None else axes
    angle = pos[ax].T * torch.tensor(freq, dtype=torch.float64)
    c, s = (scale * f(angle)[:, None] for f in (torch.cos, torch.sin))
    ia = torch.arange(half) * (2 if neighbours else 1)
    ib = ia + (1 if neighbours else half)
    out, bound = y.clone(), 2.0 ** -18 * y.abs()
    a, b = y[..., ia], y[..., ib]
    out[..., ia], out[..., ib] = a * c - b * s, b * c + a * s
    bound[..., ia] = bound[..., ib] = 2.0 ** -18 * abs(scale) * (a.abs() + b.abs())
    return out, bound


def assert_rows(got, ref, dtype, what=""):
    out, bound = ref
    got = got.double().cpu()
    assert torch.isfinite(got).all(), (what, "not finite")
    err = (got - out).abs()
    lim = UNIT[dtype] * out.abs() + (1 + UNIT[dtype]) * bound + TINY[dtype]
    assert (err <= lim).all(), (what, float((err - lim).max()), torch.nonzero(err > lim)[:4].tolist())


def attention(k, v, table, lens, seq_ids, prefix_ids, q, scale, dtype):
    """64-bit attention of q [B, Hq, d] over pools k, v [pages, Hkv, 16, d] (torch, one device): (out, lse, bound, lse bound).

    Scores: fp32 sums of d products, each step rounded or truncated at 2^-23 of the running sum: eps <= d 2^-22 times the
    largest sum of |q k| scale (the factor 2 covers the few operations after it).  A relative error e^eps - 1 of every
    weight moves the output by at most 2 eps max|v|.  Weights are rounded to the type: UNIT of the sum of w |v|, and in fp16 no
    finer than 2^-25 / 2^7 of one that is at least 1.  Sums of n terms in fp32, in parts of which none has more than some
    thousands: 2e-5 of max|v|."""
    b, hq, d = q.shape
    hkv = k.shape[1]
    g = hq // hkv
    f64 = dict(dtype=torch.float64, device=q.device)
    out, lse = torch.zeros((b, hq, d), **f64), torch.full((b, hq), -math.inf, **f64)
    bound, lse_bound = torch.zeros((b, hq, 1), **f64), torch.zeros((b, hq), **f64)
    cache = {}

    def tokens(req):
        if req not in cache:
            n = int(lens[req])
            ids = [int(p) for p in table[req][:pages_of(n)]]
            there = torch.tensor([0 <= p < k.shape[0] for p in ids], device=k.device).repeat_interleave(P)[:n]
            pg = torch.tensor(ids, device=k.device).clamp(0, k.shape[0] - 1)
            cache[req] = [x[pg].double().permute(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n][:, there] for x in (k, v)]
        return cache[req]

    for i in range(b):
        parts = []
        pre = -1 if prefix_ids is None else int(prefix_ids[i])
        if pre >= 0 and int(lens[pre]):
            parts.append(tokens(pre))
        own = i if seq_ids is None else int(seq_ids[i])
        if int(lens[own]):
            parts.append(tokens(own))
        if not parts or sum(p[0].shape[1] for p in parts) == 0:
            continue
        kk, vv = (torch.cat([p[s] for p in parts], 1) for s in (0, 1))
        qi = q[i].double().reshape(hkv, g, d)
        x = torch.einsum("hgd,htd->hgt", qi, kk) * scale
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - top)
        l = w.sum(-1, keepdim=True)
        w = w / l
        o = w @ vv
        a = torch.einsum("hgd,htd->hgt", qi.abs(), kk.abs()).amax(-1) * abs(scale)
        eps = d * 2.0 ** -22 * a
        big = vv.abs().amax((1, 2))[:, None]
        u = UNIT[dtype]
        rounding = u * (w @ vv.abs()).amax(-1)
        if dtype is torch.float16:
            rounding = rounding + kk.shape[1] * 2.0 ** -32 / l[..., 0].clamp(min=1.0) * big
        out[i] = o.reshape(hq, d)
        lse[i] = (top + torch.log(l)).reshape(hq)
        bound[i] = ((2 * eps + 2e-5) * big + rounding).reshape(hq, 1)
        lse_bound[i] = eps.reshape(hq) + 2.0 ** -20 * (1 + lse[i].abs())
    return out, lse, bound, lse_bound


def assert_attention(out, lse, ref, dtype, what=""):
    r_out, r_lse, bound, lse_bound = ref
    got = out.double().to(r_out.device)
    assert torch.isfinite(got).all(), (what, "not finite")
    err = (got - r_out).abs()
    lim = UNIT[dtype] * r_out.abs() + (1 + UNIT[dtype]) * bound + TINY[dtype]
    assert (err <= lim).all(), (what, float((err - lim).max()), torch.nonzero(err > lim)[:4].tolist())
    if lse is not None:
        got = lse.double().to(r_lse.device)
        empty = torch.isinf(r_lse)
        assert (got[empty] == -math.inf).all(), what
        err = (got[~empty] - r_lse[~empty]).abs()
        assert (err <= lse_bound[~empty]).all(), (what, float((err - lse_bound[~empty]).max()))


def make_tables(lens, seed, extra_pages=3, width=None):
    """Shuffled tables of requests of these lengths: (numpy table, number of pages); entries past a request's own are -7."""
    rng = np.random.default_rng(seed)
    n = [pages_of(int(x)) for x in lens]
    pages = sum(n) + extra_pages
    order = rng.permutation(pages)
    table = np.full((len(lens), width or max(1, max(n))), -7, np.int32)
    at = 0
    for i, m in enumerate(n):
        table[i, :m] = order[at:at + m]
        at += m
    return table, pages


def make_pool(pages, hkv, d, dtype, seed, table=None, lens=None, poisoned=True, v_mean=0.0):
    """K and V (CPU); with poisoned, slots that no request holds are NaN."""
    g = torch.Generator().manual_seed(seed)
    k, v = (torch.randn((pages, hkv, P, d), generator=g) for _ in range(2))
    v = v + v_mean
    if poisoned and table is not None:
        held = torch.zeros((pages, P), dtype=torch.bool)
        for row, n in zip(table, lens):
            n = int(n)
            t = np.arange(n)
            held[torch.as_tensor(row[t // P].astype(np.int64)), torch.as_tensor(t % P)] = True
        for x in (k, v):
            x.masked_fill_(~held[:, None, :, None], math.nan)
    return k.to(dtype), v.to(dtype)

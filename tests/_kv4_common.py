"""Plain reference of the 4-bit cache for the tests: the block layout bit by
bit, the quantisation of kvdecode4.h, attention in 64 bits, and the block tables
of a step row by row."""
import numpy as np
import torch

P = 16


def block_bytes(d, group):
    return 16 * d + 128 * (d // group)


def k_bit(tok, el, d):
    """Bit of K's code (tok, el) from the start of the K codes."""
    i, j, e = el // 32, (el % 32) // 8, el % 8
    word = (tok * 4 + j) * (d // 32) + i
    return 32 * word + 16 * (e % 2) + 4 * (e // 2)


def v_bit(tok, el, d):
    i, n, g = el // 32, (el % 32) // 8, el % 8
    word = (((tok // 8) * 8 + g) * 4 + (tok % 8) // 2) * (d // 32) + i
    return 32 * word + 16 * (tok % 2) + 4 * n


def _bits(d, fn):
    t, e = np.meshgrid(np.arange(P), np.arange(d), indexing="ij")
    return fn(t, e, d)


def unpack(block, d, group, dtype):
    """Blocks uint8 [..., bytes] (numpy) -> codes int, s, z float64 of K and of V, [..., 16, D] each."""
    out = []
    half, g = 8 * d, d // group
    for side, fn in ((0, k_bit), (1, v_bit)):
        bit = _bits(d, fn)
        codes = (block[..., side * half + bit // 8] >> (bit % 8)) & 15
        meta = np.ascontiguousarray(block[..., 2 * half + side * 64 * g: 2 * half + (side + 1) * 64 * g])
        m = torch.from_numpy(meta.copy()).view(dtype).double().numpy().reshape(*block.shape[:-1], P, g, 2)
        out.append((codes.astype(np.int64), np.repeat(m[..., 0], group, -1), np.repeat(m[..., 1], group, -1)))
    return out


def values(block, d, group, dtype):
    """K and V in 64 bits [..., 16, D], and the scales s that bound a code's step."""
    (ck, sk, zk), (cv, sv, zv) = unpack(block, d, group, dtype)
    return sk * (ck - 8) + zk, sv * (cv - 8) + zv, (sk, zk), (sv, zv)


def quantise(x, group):
    """x [..., D] (CPU tensor) -> codes, s, z (s and z in x's type, [..., D / group])."""
    y = x.float().unflatten(-1, (-1, group))
    lo, hi = y.amin(-1), y.amax(-1)
    half = hi * 0.5 - lo * 0.5
    s = (half / 7.5).to(x.dtype)
    z = (lo.double() + 8.0 * s.double()).float().to(x.dtype)
    c = torch.round((y - z.float()[..., None]) / s.float()[..., None]) + 8.0
    c = torch.where(s[..., None] > 0, c.clamp(0, 15), torch.full_like(c, 8.0))
    bad = ~torch.isfinite(y).all(-1)
    nan = torch.full_like(s, float("nan"))
    s, z = torch.where(bad, nan, s), torch.where(bad, nan, z)
    c = torch.where(bad[..., None], torch.full_like(c, 8.0), c)
    return c.flatten(-2).to(torch.int64).numpy(), s, z


def put(block, tok, side, codes, s, z, d, group):
    """One token's codes [D] and scales [D / group] into a block (numpy uint8 [bytes])."""
    bit = (k_bit if side == 0 else v_bit)(np.full(d, tok), np.arange(d), d)
    at = side * 8 * d + bit // 8
    for a, b, c in zip(at, bit % 8, codes):
        block[a] = (int(block[a]) & ~(15 << int(b))) | (int(c) << int(b))
    g = d // group
    meta = torch.stack([s, z], -1).contiguous().view(torch.uint8).numpy().reshape(-1)
    off = 16 * d + side * 64 * g + tok * 4 * g
    block[off:off + 4 * g] = meta


def random_pool(pages, heads, d, group, dtype, seed, scale=1.0):
    """Blocks with random codes and scales (numpy uint8 [pages, heads, bytes])."""
    rng = np.random.default_rng(seed)
    blocks = rng.integers(0, 256, (pages, heads, block_bytes(d, group)), dtype=np.uint8)
    g = d // group
    s = torch.from_numpy(rng.uniform(0.05, 0.6, (pages, heads, 2 * P * g)) * scale).to(dtype)
    z = torch.from_numpy(rng.normal(0, 0.5, (pages, heads, 2 * P * g)) * scale).to(dtype)
    blocks[..., 16 * d:] = torch.stack([s, z], -1).contiguous().view(torch.uint8).numpy().reshape(pages, heads, -1)
    return blocks


def poison(blocks, table, lens, d, group):
    """Codes and scales of every slot that no request holds: all bits set (a NaN scale)."""
    g = d // group
    held = np.zeros((blocks.shape[0], P), bool)
    for row, n in zip(table, lens):
        for t in range(int(n)):
            held[row[t // P], t % P] = True
    tok = np.arange(P)
    for p in range(blocks.shape[0]):
        free = tok[~held[p]]
        if free.size == P:
            blocks[p] = 255
            continue
        for t in free:
            for side, fn in ((0, k_bit), (1, v_bit)):
                bit = fn(np.full(d, t), np.arange(d), d)
                np.bitwise_or.at(blocks[p], (slice(None), side * 8 * d + bit // 8), (15 << (bit % 8)).astype(np.uint8))
                off = 16 * d + side * 64 * g + t * 4 * g
                blocks[p][:, off:off + 4 * g] = 255


def attention(blocks, table, lens, q, group, dtype, scale):
    """64-bit attention of q [B, Hq, D] (numpy); returns (out, lse, bound): bound is what the
    arithmetic of kvdecode4.h may differ by before the output's own rounding.

    Scores: fp32 sums of D products |q_d| * 8 s plus |q_d| |z|, each step rounded or truncated at
    2^-23 of the running sum: eps <= D * 2^-22 * max_t scale * sum_d |q_d| (8 s + |z|) (the factor 2
    covers the few operations after the sum and the exponential).  A relative error e^eps - 1 of
    every weight moves the normalised output by at most 2 eps max|v|.  Weights times scales are
    rounded to 11 bits before they meet the codes: 2^-11 * 8 max s.  Sums of n terms in fp32 whose
    errors average: 1e-5 of max(8 s + |z|)."""
    b, hq, d = q.shape
    hkv = blocks.shape[1]
    g = hq // hkv
    out, lse = np.zeros((b, hq, d)), np.full((b, hq), -np.inf)
    bound, lse_bound = np.zeros((b, hq, 1)), np.zeros((b, hq))
    for i in range(b):
        n = int(lens[i])
        if n == 0:
            continue
        pages = np.asarray(table[i][:(n + P - 1) // P])
        k, v, (sk, zk), (sv, zv) = values(blocks[pages], d, group, dtype)
        k, v, sk, zk, sv, zv = (x.transpose(1, 0, 2, 3).reshape(hkv, -1, d)[:, :n] for x in (k, v, sk, zk, sv, zv))
        for h in range(hq):
            x = k[h // g] @ q[i, h] * scale
            m = x.max()
            w = np.exp(x - m)
            out[i, h] = w @ v[h // g] / w.sum()
            lse[i, h] = m + np.log(w.sum())
            a = ((8 * sk[h // g] + np.abs(zk[h // g])) @ np.abs(q[i, h])).max() * abs(scale)
            eps = d * 2.0 ** -22 * a
            big = (8 * sv[h // g] + np.abs(zv[h // g])).max()
            bound[i, h] = (2 * eps + 1e-5) * big + 2.0 ** -11 * 8 * sv[h // g].max()
            lse_bound[i, h] = eps + 2.0 ** -20 * (1 + abs(lse[i, h]))
    return out, lse, bound, lse_bound


UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # a rounding's relative error
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # and its least absolute one


def assert_attention(out, lse, ref, dtype, what=""):
    r_out, r_lse, bound, lse_bound = ref
    got = out.double().cpu().numpy()
    assert np.isfinite(got).all(), (what, "not finite")
    err = np.abs(got - r_out)
    lim = UNIT[dtype] * np.abs(r_out) + (1 + UNIT[dtype]) * bound + TINY[dtype]
    assert (err <= lim).all(), (what, float((err - lim).max()), np.argwhere(err > lim)[:4].tolist())
    if lse is not None:
        got = lse.double().cpu().numpy()
        empty = np.isinf(r_lse)
        assert (got[empty] == -np.inf).all(), what
        err = np.abs(got[~empty] - r_lse[~empty])
        assert (err <= lse_bound[~empty]).all(), (what, float((err - lse_bound[~empty]).max()))


class TablesModel:
    """kv_tables_step row by row."""

    def __init__(self, table, lens, ring, head, count):
        self.table, self.lens, self.ring = np.array(table), np.array(lens), np.array(ring)
        self.head, self.count = int(head), int(count)

    def step(self, ids, new, max_tokens):
        size, width = len(self.ring), self.table.shape[1]
        pages = lambda n: (n + P - 1) // P  # noqa: E731
        slots, pos = np.full(max_tokens, -1, np.int64), np.full(max_tokens, -1, np.int32)
        cu, err = [0], 0
        tokens = need = back = taken = 0
        head, count = self.head, self.count
        valid = []
        ids, new = [int(s) for s in ids], [int(n) for n in new]
        for s, n in zip(ids, new):
            ok = 0 <= s < len(self.lens) and 0 <= int(self.lens[s]) + n <= width * P
            valid.append(ok)
            if ok and n < 0:
                back += pages(self.lens[s]) - pages(self.lens[s] + n)
        fits = count + back <= size
        if not fits:
            err |= 1
        back = 0
        for s, n, ok in zip(ids, new, valid):
            grow, first = max(n, 0), tokens
            tokens += grow
            cu.append(tokens)
            if not ok:
                err |= 4
                continue
            ctx = int(self.lens[s])
            if n < 0:
                if fits:
                    for c in range(pages(ctx + n), pages(ctx)):
                        self.ring[(head + count + back) % size] = self.table[s, c]
                        back += 1
                    self.lens[s] = ctx + n
                continue
            u = pages(ctx + n) - pages(ctx)
            at = need
            need += u
            if grow and tokens > max_tokens:
                err |= 4
                continue
            if u and need > count:
                err |= 8
                continue
            for c in range(u):
                self.table[s, pages(ctx) + c] = self.ring[(head + at + c) % size]
            if u:
                taken = need
            for i in range(grow):
                p = ctx + i
                page = int(self.table[s, p // P])
                slots[first + i] = page * P + p % P if 0 <= page < size else -1
                if not 0 <= page < size:
                    err |= 1
                pos[first + i] = p
            self.lens[s] = ctx + n
        self.head, self.count = (head + taken) % size, count - taken + back
        return slots, pos, np.array(cu, np.int32), err

"""Plain 64-bit implementations of the serving operators (numpy, from their
definitions in include/ssd.h), shared by their tests."""
import numpy as np


def bf16_bits(x):
    """Nearest bf16 (ties to even) of float32 values, as uint16."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    r = ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)
    return np.where(np.isnan(x), np.uint16(0x7FC0), r)


def bf16_value(bits):
    return (np.asarray(bits, np.uint16).astype(np.uint32) << 16).view(np.float32)


def _e4m3_table():
    """Value of each e4m3 code (OCP: bias 7, no infinities, 0x7F and 0xFF are NaN)."""
    t = np.zeros(256)
    for c in range(256):
        e, f = (c >> 3) & 15, c & 7
        v = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        t[c] = np.nan if (c & 127) == 127 else (-v if c & 128 else v)
    return t


E4M3 = _e4m3_table()


def e4m3_round(x):
    """Nearest e4m3 value, ties to even; |x| <= 448."""
    x = np.asarray(x, np.float64)
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -30))), -6)
    step = 2.0 ** (e - 3)
    return np.rint(x / step) * step


def exponent(big):
    """Smallest s >= 1 with big <= 448 * 2^(s - 127)."""
    s = 1
    while big > 448.0 * 2.0 ** (s - 127):
        s += 1
    return s


# ---------------------------------------------------------------- block tables and slots
def slots(held, fresh, pool, table, block, n_rows):
    table = table.copy()
    B, W = table.shape
    held, fresh = [max(int(x), 0) for x in held], [max(int(x), 0) for x in fresh]
    lens, cu, taken = [h + f for h, f in zip(held, fresh)], [0], 0
    out_s, out_p = np.full(n_rows, -1, np.int32), np.full(n_rows, -1, np.int32)
    for b in range(B):
        have, want = min(-(-held[b] // block), W), min(-(-lens[b] // block), W)
        for j in range(have, want):
            table[b, j] = pool[taken] if taken < len(pool) else -1
            taken += 1
        for i in range(fresh[b]):
            r, p = cu[-1] + i, held[b] + i
            if r < n_rows:
                out_p[r] = p
                if p // block < W and table[b, p // block] >= 0:
                    out_s[r] = table[b, p // block] * block + p % block
        cu.append(cu[-1] + fresh[b])
    return dict(table=table, lens=np.array(lens, np.int32), cu=np.array(cu, np.int32), slots=out_s, positions=out_p,
                used=np.array([taken], np.int32))


# ---------------------------------------------------------------- rotary positions
def rope(x, positions, section, theta):
    """x [T][heads][D] float64."""
    half, y, j = sum(section), x.copy(), 0
    for axis, n in enumerate(section):
        for _ in range(n):
            a = positions[axis].astype(np.float64) * theta ** (-j / half)
            c, s = np.cos(a)[:, None], np.sin(a)[:, None]
            y[:, :, j] = x[:, :, j] * c - x[:, :, j + half] * s
            y[:, :, j + half] = x[:, :, j + half] * c + x[:, :, j] * s
            j += 1
    return y


# ---------------------------------------------------------------- cache
class Cache:
    """Codes as values: k, v [blocks][heads][block][D] float64 (v by token too), exponents int."""

    def __init__(self, n_blocks, heads, block, D):
        self.block, self.n_blocks = block, n_blocks
        self.k, self.v = np.zeros((n_blocks, heads, block, D)), np.zeros((n_blocks, heads, block, D))
        self.ke, self.ve = np.ones((n_blocks, heads), int), np.ones((n_blocks, heads), int)

    def load(self, k, v, ke, ve):
        """From the device arrays' codes and exponent bytes."""
        self.k, self.v = E4M3[k], E4M3[v].swapaxes(2, 3).copy()
        self.ke, self.ve = ke.astype(int), ve.astype(int)

    def append(self, slots, k, v):
        """Rows k, v [n][heads][D] float64."""
        n = len(slots)
        ok = lambda s: 0 <= s < self.n_blocks * self.block  # noqa: E731
        a = 0
        while a < n:
            if not ok(slots[a]):
                a += 1
                continue
            e = a + 1
            while e < n and slots[e] == slots[e - 1] + 1 and slots[e] % self.block:
                e += 1
            p, o = divmod(int(slots[a]), self.block)
            for val, exps, x in ((self.k, self.ke, k), (self.v, self.ve, v)):
                for h in range(val.shape[1]):
                    rows = x[a:e, h]
                    mag = np.abs(rows)
                    s = exponent(mag[np.isfinite(mag)].max(initial=0.0))
                    if o and exps[p, h] >= s:
                        s = exps[p, h]
                    elif o:
                        val[p, h, :o] = e4m3_round(val[p, h, :o] * 2.0 ** (exps[p, h] - s))
                    exps[p, h] = s
                    y = np.clip(rows * 2.0 ** (127 - s), -448.0, 448.0)
                    val[p, h, o:o + e - a] = e4m3_round(np.where(np.isnan(y), 0.0, y))
            a = e

    def gather(self, table_row, n, h):
        """Keys, values [n][D] of KV head h, whether each position exists, and the largest value its block can hold."""
        D = self.k.shape[3]
        K, V, ok, top = np.zeros((n, D)), np.zeros((n, D)), np.zeros(n, bool), np.zeros(n)
        for p in range(n):
            j = p // self.block
            pg = table_row[j] if j < len(table_row) else -1
            if 0 <= pg < self.n_blocks:
                ok[p] = True
                K[p] = self.k[pg, h, p % self.block] * 2.0 ** (self.ke[pg, h] - 127)
                V[p] = self.v[pg, h, p % self.block] * 2.0 ** (self.ve[pg, h] - 127)
                top[p] = 448.0 * 2.0 ** (self.ve[pg, h] - 127)
        return K, V, ok, top


def attention(cache, q, cu, lens, table, scale, bf16):
    """q [rows][heads][D] float64 -> (out, bound of its error); rows of no request stay NaN.

    The bound: a score is a sum of D products, so fp32 leaves it off by at most d = (D + 16) 2^-24 scale sum |q k|
    plus 4 2^-24 of itself (scaling, the subtraction of the maximum, the exponential's argument); an
    exponential by a few units more; its weight then by a factor of about 1 + d, the normalised one by twice that;
    the weighted sum of n values adds (n + 16) 2^-24 sum p |v|.  bf16 outputs add their own rounding,
    2^-8 |o|, and may carry the weights in a type of 11 bits, 2^-11 sum p |v|: fp16, whose smallest step is
    2^-24, with the largest weight (times its block's value scale) held at 2^6 or above, so that a smaller one is
    off by at most 2^-25 2^-6 of that, and a value by that times its code: n 2^-31 max (p scale) 448.  A weight below 2^-126 of the
    largest, and a result below 2^-126, has no normal fp32 value and may be 0: n 2^-126 max |v| + 2^-126.
    """
    rows, Hq, D = q.shape
    g = Hq // cache.k.shape[1]
    out, tol = np.full(q.shape, np.nan), np.zeros(q.shape)
    u = 2.0 ** -24
    for b in range(len(lens)):
        r0, n = int(cu[b]), int(cu[b + 1] - cu[b])
        if n <= 0:
            continue
        L = max(0, min(int(lens[b]), table.shape[1] * cache.block))
        for h in range(cache.k.shape[1]):
            K, V, ok, top = cache.gather(table[b], L, h)
            for i in range(n):
                if not 0 <= r0 + i < rows:
                    continue
                seen = ok & (np.arange(L) <= int(lens[b]) - n + i)
                for j in range(h * g, (h + 1) * g):
                    if not seen.any():
                        out[r0 + i, j], tol[r0 + i, j] = 0.0, 0.0
                        continue
                    x = q[r0 + i, j]
                    s = (K[seen] @ x) * scale
                    d = ((D + 16) * u * abs(scale) * (np.abs(K[seen]) @ np.abs(x)) + 4 * u * np.abs(s - s.max()) +
                         4 * u * np.abs(s)).max()
                    p = np.exp(s - s.max())
                    p /= p.sum()
                    pv = p @ np.abs(V[seen])
                    o = p @ V[seen]
                    out[r0 + i, j] = o
                    tol[r0 + i, j] = pv * (2 * d + (L + 16) * u) + 2.0 ** -126 * (1 + L * np.abs(V[seen]).max()) + (
                        np.abs(o) * 2.0 ** -8 + pv * 2.0 ** -11 + L * 2.0 ** -31 * (p * top[seen]).max() if bf16 else 0.0)
    return out, tol


# ---------------------------------------------------------------- sampling
def sample(logits, u, temperature, top_k, top_p, min_p):
    """(token, probability) of one row."""
    l = np.where(np.isnan(logits), -np.inf, np.minimum(logits.astype(np.float64), np.finfo(np.float32).max))
    V = len(l)
    order = np.lexsort((np.arange(V), -l))
    if l[order[0]] == -np.inf:
        return -1, 0.0
    if not temperature > 0:
        return int(order[0]), 1.0
    with np.errstate(over="ignore"):  # a tiny temperature: exp(-inf) = 0
        w = np.exp((l[order] - l[order[0]]) / temperature)
    n = min(top_k, V) if top_k > 0 else V
    if top_p < 1:
        c = np.cumsum(w[:n])
        n = min(n, int(np.searchsorted(c, top_p * c[-1], side="left")) + 1)
    if min_p > 0:
        n = int((w[:n] >= min(min_p, 1.0)).sum())  # falling order
    ids = np.sort(order[:n])
    w = np.exp((l[ids] - l[order[0]]) / temperature)
    c = np.cumsum(w)
    live = np.nonzero(w > 2.0 ** -46)[0]
    j = min(int(np.searchsorted(c, max(u, 0.0) * c[-1], side="right")), live[-1])
    return int(ids[j]), w[j] / c[-1]

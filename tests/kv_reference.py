"""Definitions in 64 bits of the operators on the paged bf16 / fp32 cache (``include/rsd_ops.h``), and the places of an entry's values in a page."""
import numpy as np

PAGE = 16


def frequencies(theta, rot, kind="plain", factor=1.0, original=0.0, low=1.0, high=32.0):
    i = np.arange(rot // 2)
    if kind == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = theta ** (-2.0 * i / rot)
    if kind == "linear":
        return f / factor
    if kind == "parts":
        g = np.clip((original * f / (2 * np.pi) - low) / (high - low), 0, 1)
        return f * (g + (1 - g) / factor)
    return f


def turned(x, weight, eps, position, rope):
    """Heads [rows, heads, hd] normed (with a weight) and rotated (rope: freq, interleaved, magnitude; or None)."""
    x = np.asarray(x, np.float64).copy()
    if weight is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * weight
    if rope is None:
        return x
    freq, interleaved, magnitude = rope
    half = len(freq)
    a = np.asarray(position, np.float64)[:, None] * freq
    c, s = (magnitude * np.cos(a))[:, None], (magnitude * np.sin(a))[:, None]
    i = np.arange(half)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    u, w = x[..., p], x[..., q]
    x[..., p], x[..., q] = u * c - w * s, w * c + u * s
    return x


def partner_sums(x, rope):
    """|a| + |b| of the pair that each dimension belongs to, times the magnitude (the dimension itself where it does not turn)."""
    y = np.abs(np.asarray(x, np.float64))
    if rope is None:
        return y
    freq, interleaved, magnitude = rope
    half = len(freq)
    i = np.arange(half)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    s = (y[..., p] + y[..., q]) * max(1.0, abs(magnitude))
    y[..., p], y[..., q] = s, s
    return y


def key_places(size, hd, t):
    """Where the dimensions of token t's key stand among the 16 * hd values of a (page, head), `size` bytes each."""
    e = 16 // size
    d = np.arange(hd)
    return d // (4 * e) * (64 * e) + d % (4 * e) // e * (16 * e) + t * e + d % e


def value_places(size, hd, t):
    e = 16 // size
    d = np.arange(hd)
    return d // (4 * e) * (64 * e) + t // 4 * (16 * e) + d % 16 * e + d % (4 * e) // 16 * 4 + t % 4


def fill(pool, table, size, hd, seq, slot, k, v):
    """Entries into a pool [pages, heads, 2, 16 hd] (numpy, in place); entries that the cache has no place for are left out."""
    for i in range(len(seq)):
        if not (0 <= seq[i] < len(table) and 0 <= slot[i] < table.shape[1] * PAGE):
            continue
        page = table[seq[i], slot[i] // PAGE]
        if 0 <= page < len(pool):
            pool[page][:, 0, key_places(size, hd, slot[i] % PAGE)] = k[i]
            pool[page][:, 1, value_places(size, hd, slot[i] % PAGE)] = v[i]


def entries(pool, table_row, n, size, hd):
    """Keys and values [heads, n, hd] of a sequence's first n slots, and which of them have a page."""
    k, v = np.zeros((2, pool.shape[1], n, hd))
    there = np.zeros(n, bool)
    for s in range(n):
        page = table_row[s // PAGE]
        if 0 <= page < len(pool):
            there[s] = True
            k[:, s] = pool[page][:, 0, key_places(size, hd, s % PAGE)]
            v[:, s] = pool[page][:, 1, value_places(size, hd, s % PAGE)]
    return k, v, there


def seen(n, m, window, sinks):
    """[m rows, n slots]: what the rows of a sequence of n entries see."""
    p = n - m + np.arange(m)[:, None]
    s = np.arange(n)[None]
    return (s <= p) & ((s > p - window) | (s < sinks) if window else True)


def attention(q, k, v, there, scale, window=0, sinks=0):
    """Rows q [m, heads, hd] over entries [kv heads, n, hd]: out, lse, and what bounds their errors: sum p|v|, the largest sum |scale q k| of a row."""
    m, heads, hd = q.shape
    hkv, n, _ = k.shape
    mask = seen(n, m, window, sinks) & there[None]
    out, lse = np.zeros((m, heads, hd)), np.full((m, heads), -np.inf)
    mass, size = np.zeros((m, heads, hd)), np.zeros((m, heads))
    for h in range(heads):
        g = h // (heads // hkv)
        for j in range(m):
            on = mask[j]
            if not on.any():
                continue
            with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                z = k[g][on] @ q[j, h] * scale
                top = z.max()
                if top == -np.inf:
                    continue
                e = np.exp(z - top)
                p = e / e.sum()
                lse[j, h] = top + np.log(e.sum())
                vv = v[g][on]
                out[j, h] = np.sum(np.where(p[:, None] == 0, 0.0, p[:, None] * vv), 0)
                mass[j, h] = np.sum(p[:, None] * np.abs(np.where(np.isfinite(vv), vv, 0)), 0)
                a = np.abs(k[g][on]) @ np.abs(q[j, h]) * abs(scale)
                size[j, h] = np.max(a[np.isfinite(a)], initial=0.0)
    return out, lse, mass, size

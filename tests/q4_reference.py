"""The 4-bit operators by their definitions, in 64 bits and one step at a time (numpy, no shared code with the kernels)."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """[..., 32 g] -> codes (0..15), scale bytes [..., g] and the values they stand for."""
    x = np.asarray(x, np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    amax = np.abs(g).max(-1)
    e = np.full(amax.shape, -125)
    while True:
        more = (e < 125) & (amax > np.ldexp(7.0, e))
        if not more.any():
            break
        e = e + more
    m = np.minimum(np.abs(g) / np.ldexp(1.0, e)[..., None], 6.0)
    code = np.zeros(g.shape, np.int64)
    for j in range(7):                                     # past the midpoint, or on it when the upper code is the even one
        mid = (GRID[j] + GRID[j + 1]) / 2
        code = np.where((m > mid) | ((m == mid) & ((j + 1) % 2 == 0)), j + 1, code)
    code = np.where(bad[..., None], 0, code + 8 * np.signbit(g))
    byte = np.where(bad, 255, e + 127)
    return code.reshape(x.shape).astype(np.uint8), byte.astype(np.uint8), values(code.reshape(x.shape), byte)


def values(code, byte):
    code = np.asarray(code, np.int64)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code & 7]
    with np.errstate(over="ignore"):
        s = np.where(np.asarray(byte) == 255, np.nan, np.ldexp(1.0, np.asarray(byte, np.int64) - 127))
    return v * np.repeat(s, 32, -1)


def tiles(code, byte, n, k):
    """Codes [n][k'], scale bytes [n][k'/32] of a weight matrix -> its tiles, byte by byte."""
    nt, kt, ks = -(-n // 16), -(-k // 128), -(-k // 512)
    codes, scales = np.zeros((nt, kt, 4, 16, 16), np.uint8), np.full((nt, ks, 4, 16, 4), 2, np.uint8)
    for i in range(n):
        for j in range(code.shape[1]):
            codes[i // 16, j // 128, j % 128 // 32, i % 16, j % 32 // 2] |= int(code[i, j]) << (4 * (j % 2))
        for g in range(byte.shape[1]):
            scales[i // 16, g // 16, g % 4, i % 16, g // 4 % 4] = byte[i, g]
    return codes, scales


def entry_places(hd, t):
    """Byte offsets in a (page, kv head) block of token t: keys [hd/2], values [hd/32][16], key and value scales [hd/32]."""
    g = hd // 32
    key = [d // (hd // 4) * 16 * (hd // 8) + t * (hd // 8) + d % (hd // 4) // 2 for d in range(0, hd, 2)]
    val = [[8 * hd + ((t // 4 * 16 + m) * g + q) * 4 + t % 4 for m in range(16)] for q in range(g)]
    ks = [16 * hd + q * 16 + t for q in range(g)]
    vs = [16 * hd + 16 * g + (t // 4 * g + q) * 4 + t % 4 for q in range(g)]
    return np.array(key), np.array(val), np.array(ks), np.array(vs)


def write_entry(block, hd, t, k, v):
    """One entry into the bytes of its (page, kv head) block."""
    key, val, ks, vs = entry_places(hd, t)
    code, byte, _ = quantize(k)
    block[key] = code[0::2] | (code[1::2] << 4)
    block[ks] = byte
    code, byte, _ = quantize(v)
    code = code.reshape(-1, 2, 16)
    block[val] = code[:, 0] | (code[:, 1] << 4)
    block[vs] = byte


def read_entry(block, hd, t):
    key, val, ks, vs = entry_places(hd, t)
    kc = np.stack([block[key] & 15, block[key] >> 4], -1).reshape(-1)
    vc = np.stack([block[val] & 15, block[val] >> 4], 1).reshape(-1)
    return values(kc, block[ks]), values(vc, block[vs])


def entries(pool, table_row, n, head, hd):
    """Keys and values [n][hd] of a sequence's kv head, and which of them exist (their page lies in the pool)."""
    k, v, there = np.zeros((n, hd)), np.zeros((n, hd)), np.zeros(n, bool)
    for s in range(n):
        p = int(table_row[s // 16])
        if 0 <= p < len(pool):
            k[s], v[s] = read_entry(pool[p, head], hd, s % 16)
            there[s] = True
    return k, v, there


def attention(q, k, v, there, scale, count):
    """Rows q [count][heads of the group][hd] of one (sequence, kv head) over its n entries.
    Returns out, lse, weight per entry, and the sum of p |v| and the largest sum of |scale q k| that bound the rounding."""
    n = len(k)
    out, lse = np.zeros(q.shape), np.full(q.shape[:2], -np.inf)
    weight, mass, spread = np.zeros(n), np.zeros(q.shape), 0.0
    for r in range(count):
        seen = there & (np.arange(n) < n - (count - 1 - r))
        if not seen.any():
            continue
        for g in range(q.shape[1]):
            z = scale * (k[seen] @ q[r, g])
            spread = max(spread, float(np.nanmax(abs(scale) * (np.abs(k[seen]) @ np.abs(q[r, g])))))
            top = z.max()
            p = np.exp(z - top)
            lse[r, g] = top + np.log(p.sum())
            p /= p.sum()
            out[r, g] = p @ v[seen]
            mass[r, g] = p @ np.abs(v[seen])
            weight[seen] += p
    return out, lse, weight, mass, spread


def evict(score, pos, n, budget, recent):
    """Kept slots of one (sequence, kv head), and the moves (from, to) in order."""
    if n <= budget:
        return np.arange(n), []
    newest = int(pos[:n].max())
    rank = []
    for s in range(n):
        x = float(score[s])
        rank.append((0 if int(pos[s]) > newest - recent else 1, -(-np.inf if np.isnan(x) else x), s))
    kept = sorted(s for _, _, s in sorted(rank)[:budget])
    free = [s for s in range(budget) if s not in set(kept)]
    return np.array(kept), list(zip([s for s in kept if s >= budget], free))

"""The 4-bit operators where their arguments meet: repeated positions, rows whose scores are all minus infinity, factors of zero, memory that outputs
share, arguments left out.  Definitions and tolerances are those of ``test_gpu_ops``.
"""
import numpy as np
import pytest

import q4_reference as ref
from test_gpu_ops import U, R, dev, host, make_cache, torch, weights  # noqa: F401  (torch and R are its fixtures)

pytestmark = pytest.mark.gpu


def random_pages(torch, R, rng, lens, hkv, hd, cap=0):
    """A cache of arbitrary codes with scales near 1: keys as large as normally distributed ones."""
    need = [-(-n // 16) for n in lens]
    pool = rng.integers(0, 256, (sum(need) + 3, hkv, 17 * hd)).astype(np.uint8)
    pool[:, :, 16 * hd:] = rng.integers(124, 127, (len(pool), hkv, hd))
    order, table = rng.permutation(len(pool)).astype(np.int32), np.full((len(lens), max(need + [-(-cap // 16)])), -1, np.int32)
    for b in range(len(lens)):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
    return R.Kv4Cache(dev(torch, pool), dev(torch, table), dev(torch, np.array(lens, np.int32))), pool, table


def starts_of(rows):
    return np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)


# ---------------------------------------------------------------- eviction

def check_evict(torch, R, rng, lens, budget, recent, score, pos, hd, hkv):
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    want, ws, wp = pool.copy(), score.copy(), pos.copy()
    for b, n in enumerate(lens):
        for h in range(hkv):
            for fr, to in ref.evict(score[b, h], pos[b, h].astype(np.int64), n, budget, recent)[1]:
                for a, c in zip(ref.entry_places(hd, fr % 16), ref.entry_places(hd, to % 16)):
                    want[table[b, to // 16], h][c] = pool[table[b, fr // 16], h][a]
                ws[b, h, to], wp[b, h, to] = score[b, h, fr], pos[b, h, fr]
    ds, dp = dev(torch, score), dev(torch, pos)
    R.rsd_kv4_evict(cache, ds, dp, budget, recent)
    assert np.array_equal(cache.kv_len.cpu().numpy(), np.minimum(lens, budget))
    assert np.array_equal(dp.cpu().numpy(), wp) and np.array_equal(ds.cpu().numpy().view(np.int32), ws.view(np.int32))
    assert np.array_equal(cache.pool.cpu().numpy(), want)


def test_evict_ranks_protected_entries_by_score(torch, R):
    """Four of six entries at the newest position, two places."""
    score = np.array([1, 5, 2, 9, 100, 50] + [0] * 10, np.float32)[None, None]
    pos = np.array([7, 7, 7, 7, 0, 1] + [0] * 10, np.int32)[None, None]
    assert list(ref.evict(score[0, 0], pos[0, 0], 6, 2, 1)[0]) == [1, 3]
    check_evict(torch, R, np.random.default_rng(1), [6], 2, 1, score, pos, 32, 1)


@pytest.mark.parametrize("lens,budget,recent", [([300, 90, 257], 80, 1), ([300, 90], 80, 40), ([1500, 700], 512, 512), ([17000], 600, 3)])
@pytest.mark.parametrize("scores", ["normal", "ties", "odd"])
def test_evict_where_positions_repeat(torch, R, lens, budget, recent, scores):
    """More protected entries than the budget, just as many, and fewer, side by side."""
    rng = np.random.default_rng(sum(lens) + recent)
    hkv, cap = 4, -(-max(lens) // 16) * 16
    shape = (len(lens), hkv, cap)
    score = rng.normal(size=shape).astype(np.float32)
    if scores == "ties":
        score = np.floor(score).astype(np.float32) * rng.choice([1.0, -0.0], shape).astype(np.float32)
    if scores == "odd":
        for x in (np.nan, -np.nan, np.inf, -np.inf, -3e38, 3e38):
            score[rng.random(shape) < 0.15] = x
    pos = np.zeros(shape, np.int32)                        # head 0: positions never set
    pos[:, 1] = rng.integers(0, 3, shape[::2]) - 1
    for b, n in enumerate(lens):                           # head 2: exactly `budget` protected entries, head 3: one more
        for h in (2, 3):
            pos[b, h] = -1000
            pos[b, h, rng.permutation(n)[:budget + h - 2]] = 2 ** 31 - 1
    check_evict(torch, R, rng, lens, budget, recent, score, pos, 32, hkv)

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


# ---------------------------------------------------------------- attention

def check_columns(cache, pool, table, lens, rows, q, scale, out, lse, score0=None, score1=None, dtype="f32"):
    """Every (row, head) by itself, with the bounds of test_gpu_ops.check_attention; a column whose scores are all -inf deals out nothing."""
    hd, hkv = pool.shape[2] // 17, pool.shape[1]
    group, starts = q.shape[1] // hkv, starts_of(rows)
    q, out, lse = host(q), host(out), host(lse)
    for b, n in enumerate(lens):
        for h in range(hkv):
            k, v, there = ref.entries(pool, table[b], n, h, hd)
            total, slack = np.zeros(n), np.zeros(n)
            for r in range(rows[b]):
                m = max(n - (rows[b] - 1 - r), 0)          # entries that the row sees
                for g in range(group):
                    at = (starts[b] + r, h * group + g)
                    with np.errstate(invalid="ignore"):
                        z = scale * (k[:m][there[:m]] @ q[at])
                    if (z == -np.inf).all():               # nothing is seen, or nothing has a weight
                        assert not out[at].any() and lse[at] == -np.inf, at
                        continue
                    if np.isnan(z).any() or (z == np.inf).any():
                        assert np.isnan(out[at]).all() and np.isnan(lse[at]), at
                        total[:m][there[:m]] = np.nan
                        continue
                    want, want_lse, weight, mass, spread = ref.attention(q[at][None, None], k[:m], v[:m], there[:m], scale, 1)
                    rel = 2 * (2 * (3 * hd / 32 + 48) * U * spread + 4 * U * spread) + (n / 64 + 80) * 2 * U + 8 * U
                    bound = rel * mass + U * np.abs(want) * 4 + 1e-37
                    if dtype == "bf16":
                        bound = bound + 2.0 ** -16 * mass + 2.0 ** -8 * np.abs(want)
                    bad = np.isnan(want[0, 0])             # dims of a value that reads as NaN
                    assert np.array_equal(np.isnan(out[at]), bad) and np.all((np.abs(out[at] - want[0, 0]) <= bound)[0, 0][~bad]), at
                    assert abs(lse[at] - want_lse[0, 0]) <= rel + 4 * U * (1 + abs(want_lse[0, 0])), at
                    total[:m] += weight
                    slack[:m] += (2 * rel + 8 * U * spread) * weight
            if score0 is not None:
                got, was = score1[b, h, :n], score0[b, h, :n]
                assert np.array_equal(np.isnan(got), np.isnan(total)), (b, h)
                fine = ~np.isnan(total)
                assert np.all(np.abs(got - was - total)[fine] <= (slack + 2 * U * np.abs(got) + 1e-37)[fine]), (b, h)
                assert np.array_equal(score1[b, h, n:], score0[b, h, n:])


def columns_with_first_dimension_alike(pool, hd):
    """Every key gets 1.5 units as its first number: q with an infinity there scores the same infinity everywhere."""
    for t in range(16):
        pool[:, :, t * (hd // 8)] = (pool[:, :, t * (hd // 8)] & 0xF0) | 3


# heads, kv heads, head dim, lengths, rows: one tile (weights added by the attention kernel itself), in parts, two tiles, many columns, columns in groups
KINDS = [(8, 2, 64, [128, 70, 3], [1, 1, 1]), (8, 2, 128, [2304, 40], [1, 1]), (28, 2, 32, [64, 133], [1, 2]), (10, 1, 128, [192, 90], [9, 7]),
         (8, 1, 128, [400, 130], [34, 40])]


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_whose_scores_are_all_minus_infinity(torch, R, heads, hkv, hd, lens, rows, dtype):
    rng = np.random.default_rng(heads + hd)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    columns_with_first_dimension_alike(pool, hd)
    cache = R.Kv4Cache(dev(torch, pool), cache.table, cache.kv_len)
    starts = starts_of(rows)
    q = rng.normal(size=(int(starts[-1]), heads, hd)).astype(np.float32)
    q[0, 1, 0] = q[starts[1], heads - 1, 0] = q[-1, 0, 0] = -np.inf
    q = dev(torch, q).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    scores = dev(torch, rng.random((len(lens), hkv, table.shape[1] * 16)).astype(np.float32))
    before = host(scores)
    out, lse = R.rsd_kv4_attention(cache, q, 0.125, row_start=dev(torch, starts), max_rows=max(rows), scores=scores, want_lse=True)
    check_columns(cache, pool, table, lens, rows, q, 0.125, out, lse, before, host(scores), dtype)
    assert np.isfinite(host(scores)).all()
    scores.copy_(dev(torch, before))                       # and without the logarithms asked for
    again = R.rsd_kv4_attention(cache, q, 0.125, row_start=dev(torch, starts), max_rows=max(rows), scores=scores)
    assert torch.equal(again, out) and bool(torch.isfinite(scores).all())


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS)
@pytest.mark.parametrize("scale", [0.0, float("nan")])
def test_factor_of_zero_or_nan(torch, R, heads, hkv, hd, lens, rows, scale):
    """0 times an infinite score is NaN, whatever the length; rows that see nothing stay empty; else every entry weighs the same."""
    rng = np.random.default_rng(heads + 2 * hd)
    lens = lens + [2]
    rows = rows + [4]                                      # (two of these rows see nothing)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    columns_with_first_dimension_alike(pool, hd)
    cache = R.Kv4Cache(dev(torch, pool), cache.table, cache.kv_len)
    starts = starts_of(rows)
    q = rng.normal(size=(int(starts[-1]), heads, hd)).astype(np.float32)
    q[0, 0, 0], q[starts[1], 1, 0], q[starts[-2] - 1, heads - 1, 0] = -np.inf, np.inf, -np.inf
    q = dev(torch, q)
    scores = torch.zeros(len(lens), hkv, table.shape[1] * 16, device="cuda")
    out, lse = R.rsd_kv4_attention(cache, q, scale, row_start=dev(torch, starts), max_rows=max(rows), scores=scores, want_lse=True)
    check_columns(cache, pool, table, lens, rows, q, scale, out, lse, np.zeros(scores.shape), host(scores))


# ---------------------------------------------------------------- arguments

def test_an_error_the_caller_has_not_read_stays(torch, R):
    """The runtime's last error belongs to the caller's own call before; an operator that succeeds neither reports nor clears it."""
    import ctypes as C
    rng = np.random.default_rng(3)
    cache, pool, table = make_cache(torch, R, rng, [20], 1, 32)
    x, idx = torch.ones(1, 1, 32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    hip = C.CDLL([line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line][0])
    assert hip.hipGetLastError() == 0
    refused = hip.hipSetDevice(10_000)
    assert refused != 0 and hip.hipPeekAtLastError() == refused
    try:
        R.rsd_kv4_append(cache, x, x, idx, idx)
        assert hip.hipPeekAtLastError() == refused
    finally:
        hip.hipGetLastError()
    k, v = R.rsd_kv4_read(cache, idx, idx)
    assert bool((k == 1).all()) and bool((v == 1).all())


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS)
def test_out_may_be_q_where_no_weights_need_it_again(torch, R, heads, hkv, hd, lens, rows):
    rng = np.random.default_rng(heads + 7 * hd)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    starts = dev(torch, starts_of(rows))
    q = dev(torch, rng.normal(size=(sum(rows), heads, hd)).astype(np.float32))
    kw = dict(row_start=starts, max_rows=max(rows))
    scores = torch.zeros(len(lens), hkv, table.shape[1] * 16, device="cuda")
    want = R.rsd_kv4_attention(cache, q, 0.2, scores=scores, **kw)
    got = q.clone()
    assert R.rsd_kv4_attention(cache, got, 0.2, out=got, **kw).data_ptr() == got.data_ptr() and torch.equal(got, want)
    got, sums = q.clone(), torch.zeros_like(scores)
    try:
        R.rsd_kv4_attention(cache, got, 0.2, out=got, scores=sums, **kw)
    except R.RsdError:
        assert torch.equal(got, q) and not bool(sums.any())
    else:
        assert torch.equal(got, want) and torch.equal(sums, scores)
    more = torch.zeros(sum(rows) + 1, heads, hd, device="cuda")
    with pytest.raises(R.RsdError):                        # a row further on
        R.rsd_kv4_attention(cache, more[1:], 0.2, out=more[:-1], **kw)
    both = torch.zeros(sum(rows), 2 * heads, hd, device="cuda")         # beside each other in one buffer
    both[:, ::2] = q
    assert torch.equal(R.rsd_kv4_attention(cache, both[:, ::2], 0.2, out=both[:, 1::2], scores=sums, **kw), want) and torch.equal(both[:, ::2], q)


def test_rows_bounded_far_above_what_there_is(torch, R):
    """A bound that makes more than 2^16 tiles of columns of a list, and 2^24 (sequence, row, head) triples."""
    rng = np.random.default_rng(17)
    lens, rows, heads = [70, 0, 130, 20], [3, 0, 33, 1], 64
    cache, pool, table = random_pages(torch, R, rng, lens, 1, 32)
    q = dev(torch, rng.normal(size=(sum(rows), heads, 32)).astype(np.float32))
    starts = dev(torch, starts_of(rows))
    out, lse = R.rsd_kv4_attention(cache, q, 0.2, row_start=starts, max_rows=70_000, want_lse=True)
    check_columns(cache, pool, table, lens, rows, q, float(np.float32(0.2)), out, lse)


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS)
def test_rows_without_a_bound_are_all_computed(torch, R, heads, hkv, hd, lens, rows):
    rng = np.random.default_rng(heads + 11 * hd)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    q = dev(torch, rng.normal(size=(sum(rows), heads, hd)).astype(np.float32))
    out, lse = R.rsd_kv4_attention(cache, q, 0.2, row_start=dev(torch, starts_of(rows)), want_lse=True, out=torch.full_like(q, 1e9))
    check_columns(cache, pool, table, lens, rows, q, float(np.float32(0.2)), out, lse)


# ---------------------------------------------------------------- every kernel of the attention with its rarer arguments

GROUPS = [(9, 3, 64, [400, 150], [90, 60]), (3, 1, 32, [300], [100])]      # columns in two groups, the first of which ends inside a step


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS + GROUPS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [0.15, -0.15])
def test_pages_outside_the_pool_and_negative_factors(torch, R, heads, hkv, hd, lens, rows, dtype, scale):
    rng = np.random.default_rng(heads + 3 * hd)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    table[0, 1], table[0, 3], table[-1, 0] = -1, len(pool) + 3, 1 << 30
    cache = R.Kv4Cache(cache.pool, dev(torch, table), cache.kv_len)
    starts = starts_of(rows)
    q = dev(torch, rng.normal(size=(int(starts[-1]), heads, hd)).astype(np.float32)).to(torch.float32 if dtype == "f32" else torch.bfloat16)
    scores = dev(torch, rng.random((len(lens), hkv, table.shape[1] * 16)).astype(np.float32))
    before = host(scores)
    out, lse = R.rsd_kv4_attention(cache, q, scale, row_start=dev(torch, starts), max_rows=max(rows), scores=scores, want_lse=True)
    check_columns(cache, pool, table, lens, rows, q, float(np.float32(scale)), out, lse, before, host(scores), dtype)


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", KINDS + GROUPS)
@pytest.mark.parametrize("what", ["large", "infinite", "nan value", "nan key"])
def test_weights_of_unusual_numbers(torch, R, heads, hkv, hd, lens, rows, what):
    rng = np.random.default_rng(heads + 5 * hd)
    cache, pool, table = random_pages(torch, R, rng, lens, hkv, hd)
    columns_with_first_dimension_alike(pool, hd)
    starts = starts_of(rows)
    q = rng.normal(size=(int(starts[-1]), heads, hd)).astype(np.float32)
    if what == "large":
        q *= 100
    if what == "infinite":
        q[0, 0, 0], q[0, heads - 1, 0] = np.inf, -np.inf
    if "nan" in what:
        for slot in (lens[0] - 2, 5):                      # one that not every row sees where there are several, one that all see
            pool[table[0, slot // 16], 0][ref.entry_places(hd, slot % 16)[3 if "value" in what else 2][0]] = 255
            if "value" not in what and slot != 5:
                break                                      # (a key that all see leaves nothing else to look at)
    cache = R.Kv4Cache(dev(torch, pool), cache.table, cache.kv_len)
    q = dev(torch, q)
    scores = dev(torch, rng.random((len(lens), hkv, table.shape[1] * 16)).astype(np.float32))
    before = host(scores)
    out, lse = R.rsd_kv4_attention(cache, q, 0.25, row_start=dev(torch, starts), max_rows=max(rows), scores=scores, want_lse=True)
    check_columns(cache, pool, table, lens, rows, q, 0.25, out, lse, before, host(scores))

"""The 4-bit operators against their definitions in 64 bits (``q4_reference``).

Tolerances, derived from the number formats.  u = 2^-24.
* A product over k values in fp32: products are exact (an fp32 factor enters as three bf16 numbers), every addition errs by at most 2 u of the
  sum so far (the matrix instruction may cut instead of round); on the way to the result there are at most 3 k / 32 dependent additions across instructions, 32 inside one,
  and 16 across waves and parts: error <= 2 (3 k / 32 + 48) u sum|x w|.
* A score errs by that over the head dimension, plus 4 u of itself for the factors; a softmax weight then errs by twice the scores' error (its own and the sum's),
  relative, plus (n / 64 + 80) u for the sums over n entries (64 to a step, 16 + 64 inside one and across waves and parts) and 8 u for exp.
* A result in bf16 (8 significant bits) errs by 2^-8 of itself more; there the softmax weights are products' operands as two bf16 numbers: 2^-16 of sum p|v|.
What is held in 4 bits, positions, lengths and choices are equal.
"""
import numpy as np
import pytest

import q4_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def torch():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch


@pytest.fixture(scope="module")
def R():
    from paper_2501_19324_amd import binding
    return binding


def dev(torch, a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def host(t):
    return t.detach().double().cpu().numpy()


def bf16(torch, a):
    """a rounded to bf16, as 64-bit numbers."""
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16).double().numpy()


# ---------------------------------------------------------------- weights

def special_values():
    grid = np.concatenate([ref.GRID, (ref.GRID[1:] + ref.GRID[:-1]) / 2, [6.5, 7.0, 7.5]])
    around = np.concatenate([grid, np.nextafter(np.float32(grid), np.float32(100)), np.nextafter(np.float32(grid), np.float32(-100))])
    rows = []
    for e in (-149, -140, -127, -126, -125, -20, 0, 30, 100, 122, 125):
        with np.errstate(over="ignore"):
            r = np.float32(np.ldexp(around, e))
        r[~np.isfinite(r)] = 0
        for top in (7.0, 6.0, 4.0, 3.5000002):
            line = np.zeros(32 * ((len(r) + 14) // 15), np.float32)
            for g in range(len(line) // 32):
                part = r[15 * g:15 * g + 15]
                line[32 * g:32 * g + len(part)], line[32 * g + 15:32 * g + 15 + len(part)] = part, -part
                with np.errstate(over="ignore"):
                    t = np.float32(np.ldexp(top, e))
                line[32 * g + 31] = t if np.isfinite(t) else np.finfo(np.float32).max
            rows.append(line)
    x = np.stack(rows)
    x[3, 5], x[7, 40], x[9, 70] = np.nan, np.inf, -np.inf
    return x


def test_pack_special_values(torch, R):
    x = special_values()
    code, byte, _ = ref.quantize(x)
    want = ref.tiles(code, byte, *x.shape)
    w = R.rsd_w4_pack(dev(torch, x))
    assert np.array_equal(w.codes.cpu().numpy(), want[0]) and np.array_equal(w.scales.cpu().numpy(), want[1])


@pytest.mark.parametrize("n,k", [(1, 1), (1, 32), (17, 31), (16, 128), (33, 129), (5, 513), (40, 700)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pack(torch, R, n, k, dtype):
    rng = np.random.default_rng(n * 1000 + k)
    x = (rng.normal(size=(n, k)) * np.exp(rng.normal(size=(n, 1)))).astype(np.float32)
    if dtype == "bf16":
        x = bf16(torch, x).astype(np.float32)
    wide = torch.full((n, k + 5), 1e30, device="cuda", dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    wide[:, 2:2 + k] = dev(torch, x).to(wide.dtype)
    pad = np.zeros((n, -(-k // 32) * 32))
    pad[:, :k] = x
    code, byte, _ = ref.quantize(pad)
    want = ref.tiles(code, byte, n, k)
    for src in (wide[:, 2:2 + k], wide[:, 2:2 + k].contiguous()):
        w = R.rsd_w4_pack(src)
        assert np.array_equal(w.codes.cpu().numpy(), want[0]) and np.array_equal(w.scales.cpu().numpy(), want[1])


def weights(torch, R, rng, n, k):
    """Packed weights and the numbers they stand for."""
    w = np.zeros((n, -(-k // 32) * 32))
    w[:, :k] = (rng.normal(size=(n, k)) * np.exp(0.5 * rng.normal(size=(n, 1)))).astype(np.float32)
    packed = R.rsd_w4_pack(dev(torch, w[:, :k].astype(np.float32)))
    return packed, ref.quantize(w)[2][:, :k]


def linear_bound(x, w, k, dtype, y):
    return 2 * (3 * k / 32 + 48) * U * (np.abs(x) @ np.abs(w).T) + (2.0 ** -8 if dtype == "bf16" else U) * np.abs(y) + 1e-37


LINEAR = [(1, 1, 1), (1, 16, 32), (1, 17, 33), (2, 15, 128), (3, 64, 129), (7, 100, 512), (1, 300, 1536), (16, 33, 513), (17, 48, 640), (31, 20, 1100), (32, 64, 2048),
          (33, 70, 300), (64, 129, 260), (65, 31, 1536), (100, 40, 96), (128, 256, 384), (130, 33, 700), (257, 17, 130), (1, 40, 9000), (5, 5000, 70), (70, 2100, 1000),
          (20, 101, 5000), (40, 50, 2100), (6, 37, 2600), (12, 2050, 2200), (66, 18, 6200), (100, 600, 520), (3, 20, 7), (40, 300, 5), (20, 33, 8), (9, 64, 15), (70, 40, 9), (8, 8300, 150), (6, 20, 10500)]


@pytest.mark.parametrize("rows,n,k", LINEAR)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_linear(torch, R, rows, n, k, dtype):
    rng = np.random.default_rng(rows + 7 * n + 31 * k)
    packed, w = weights(torch, R, rng, n, k)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = dev(torch, (rng.normal(size=(rows, k)) * np.exp(rng.normal(size=(1, k)))).astype(np.float32)).to(t)
    want = host(x) @ w.T
    got = R.rsd_w4_linear(x, packed)
    assert got.dtype == t and got.shape == (rows, n)
    assert np.all(np.abs(host(got) - want) <= linear_bound(host(x), w, k, dtype, want))
    # the same from rows further apart and off every wider alignment, into such rows; what lies between them stays
    gap = torch.full((rows, k + 3), float("nan"), device="cuda", dtype=t)
    gap[:, 1:1 + k] = x
    out = torch.full((rows, n + 5), 7.0, device="cuda", dtype=t)
    again = R.rsd_w4_linear(gap[:, 1:1 + k], packed, out=out[:, 3:3 + n])
    assert again.data_ptr() == out[:, 3:].data_ptr()
    assert torch.equal(out[:, 3:3 + n], got) and bool((out[:, :3] == 7).all()) and bool((out[:, 3 + n:] == 7).all())
    # no order of the sum that changes from call to call
    assert torch.equal(R.rsd_w4_linear(x, packed), got)


def test_linear_of_no_rows(torch, R):
    packed, _ = weights(torch, R, np.random.default_rng(1), 20, 40)
    assert R.rsd_w4_linear(torch.zeros(0, 40, device="cuda"), packed).shape == (0, 20)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40])
def test_linear_keeps_nan_and_infinity_where_they_belong(torch, R, rows, dtype):
    rng = np.random.default_rng(5)
    n, k = 50, 200
    w = np.abs(rng.normal(size=(n, k))).astype(np.float32) + 1.0        # no zero code: every product with an infinity is one
    w[7, 100] = np.nan
    packed = R.rsd_w4_pack(dev(torch, w))
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = np.abs(rng.normal(size=(rows, k))).astype(np.float32) + 0.1
    x[1, 3] = np.nan
    x[2, 199] = np.inf
    y = host(R.rsd_w4_linear(dev(torch, x).to(t), packed))
    bad = np.zeros((rows, n), bool)
    bad[:, 7] = bad[1] = True
    inf = np.zeros((rows, n), bool)
    inf[2] = True
    assert np.array_equal(np.isnan(y), bad) and np.array_equal(np.isinf(y), inf & ~bad)


def test_linear_extreme_magnitudes(torch, R):
    """fp32 activations near both ends of their range, and weights of every scale."""
    rng = np.random.default_rng(6)
    k = 96
    for e in (-100, -60, 60, 100):
        packed, w = weights(torch, R, rng, 24, k)
        x = (rng.normal(size=(4, k)) * 2.0 ** e).astype(np.float32)
        x[0, :5] = [3.3e38, -3.3e38, 1e-38, 0.0, -0.0]
        x[0, 5:] = 0
        y, want = host(R.rsd_w4_linear(dev(torch, x), packed)), x.astype(np.float64) @ w.T
        fine = np.abs(x.astype(np.float64)) @ np.abs(w).T < 3e38
        assert np.all((np.abs(y - want) <= linear_bound(x.astype(np.float64), w, k, "f32", want) + 2.0 ** -126 * k)[fine])


# ---------------------------------------------------------------- the cache

def make_cache(torch, R, rng, lens, hkv, hd, spare=3, cap=0):
    """A cache with random entries; its bytes on the host.  Everything behind a sequence's entries, and pages of nobody, are arbitrary bytes."""
    need = [-(-max(n, 1) // 16) for n in lens]
    max_pages = max(need + [-(-cap // 16)])
    total = sum(need) + spare
    pool = rng.integers(0, 256, (total, hkv, 17 * hd)).astype(np.uint8)
    pool[:, :, 16 * hd:][rng.random((total, hkv, hd)) < 0.3] = 255
    order = rng.permutation(total)
    table = np.full((len(lens), max_pages), -1, np.int32)
    at = 0
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
        for s in range(n):
            for h in range(hkv):
                ref.write_entry(pool[table[b, s // 16], h], hd, s % 16, rng.normal(size=hd) * 1.3, rng.normal(size=hd))
    return R.Kv4Cache(dev(torch, pool), dev(torch, table), dev(torch, np.array(lens, np.int32))), pool, table


@pytest.mark.parametrize("hd,hkv", [(32, 1), (64, 3), (128, 2)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_append_and_read(torch, R, hd, hkv, dtype):
    rng = np.random.default_rng(hd + hkv)
    cache, pool, table = make_cache(torch, R, rng, [40, 3, 17], hkv, hd)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    seq = np.array([0] * 20 + [2, 2, 1, 0, 2] + [1] * 6, np.int32)
    slot = np.array(list(range(20, 40)) + [0, 31, 9, 47, 16] + list(range(10, 16)), np.int32)
    rows = len(seq)
    x = rng.normal(size=(rows, hkv, 2, hd)) * np.exp(2 * rng.normal(size=(rows, 1, 1, 1)))
    x[3, 0, 0, 5], x[5, hkv - 1, 1, hd - 1], x[6, 0, 1, 0] = np.nan, np.inf, -np.inf
    x = dev(torch, x.astype(np.float32)).to(t)
    k, v = x[:, :, 0], x[:, :, 1]                          # rows and heads further apart than contiguous ones
    cap = table.shape[1] * 16
    scores = torch.full((3, hkv, cap + 7), 5.0, device="cuda")[..., :cap + 2]
    pos = torch.full((3, hkv, cap), -9, dtype=torch.int32, device="cuda")
    position = dev(torch, (1000 + np.arange(rows)).astype(np.int32))
    R.rsd_kv4_append(cache, k, v, dev(torch, seq), dev(torch, slot), position=position, entry_pos=pos, scores=scores)
    want, ws, wp = pool.copy(), np.full((3, hkv, cap + 2), 5.0), np.full((3, hkv, cap), -9)
    hk, hv = host(k), host(v)
    for i in range(rows):
        for h in range(hkv):
            ref.write_entry(want[table[seq[i], slot[i] // 16], h], hd, slot[i] % 16, hk[i, h], hv[i, h])
            ws[seq[i], h, slot[i]], wp[seq[i], h, slot[i]] = 0.0, 1000 + i
    assert np.array_equal(cache.pool.cpu().numpy(), want)
    assert np.array_equal(scores.cpu().numpy(), ws) and np.array_equal(pos.cpu().numpy(), wp)
    for out in (torch.bfloat16, torch.float32):
        gk, gv = R.rsd_kv4_read(cache, dev(torch, seq), dev(torch, slot), dtype=out)
        assert gk.dtype == out and np.array_equal(host(gk), ref.quantize(hk)[2], equal_nan=True) and np.array_equal(host(gv), ref.quantize(hv)[2], equal_nan=True)
    # without the books nothing but the pages changes
    R.rsd_kv4_append(cache, k, v, dev(torch, seq), dev(torch, slot))
    assert np.array_equal(cache.pool.cpu().numpy(), want) and np.array_equal(scores.cpu().numpy(), ws)


def test_append_whole_pages_and_pieces(torch, R):
    """Long runs of consecutive slots, as a prompt leaves them, from any first slot."""
    rng = np.random.default_rng(8)
    hd, hkv = 128, 2
    for first, count in ((0, 64), (5, 59), (1, 14), (15, 2), (3, 61)):
        cache, pool, table = make_cache(torch, R, rng, [0, 0], hkv, hd, spare=9, cap=64)
        table[:] = np.array([[1, 4, 0, 7], [2, 3, 5, 6]])
        cache = R.Kv4Cache(cache.pool, dev(torch, table), cache.kv_len)
        x = rng.normal(size=(2 * count, hkv, hd, 2)).astype(np.float32)
        k, v = dev(torch, x[..., 0]), dev(torch, x[..., 1])
        seq, slot = np.repeat([0, 1], count).astype(np.int32), np.tile(np.arange(first, first + count), 2).astype(np.int32)
        for i in range(2 * count):
            for h in range(hkv):
                ref.write_entry(pool[table[seq[i], slot[i] // 16], h], hd, slot[i] % 16, x[i, h, :, 0], x[i, h, :, 1])
        R.rsd_kv4_append(cache, k, v, dev(torch, seq), dev(torch, slot))
        assert np.array_equal(cache.pool.cpu().numpy(), pool), (first, count)
        gk, gv = R.rsd_kv4_read(cache, dev(torch, seq), dev(torch, slot))
        assert np.array_equal(host(gk), ref.quantize(x[..., 0])[2]) and np.array_equal(host(gv), ref.quantize(x[..., 1])[2])


def test_rows_that_name_no_entry_are_dropped(torch, R):
    rng = np.random.default_rng(9)
    cache, pool, table = make_cache(torch, R, rng, [20, 20], 2, 64)
    table[1, 1] = len(pool)                                # a page outside the pool
    table[0, 1] = -5
    cache = R.Kv4Cache(cache.pool, dev(torch, table), cache.kv_len)
    seq = dev(torch, np.array([-1, 2, 0, 0, 0, 1, 1], np.int32))
    slot = dev(torch, np.array([0, 0, -1, 32, 17, 18, 4], np.int32))
    x = torch.ones(7, 2, 64, device="cuda")
    R.rsd_kv4_append(cache, x, x, seq, slot)
    for h in range(2):
        ref.write_entry(pool[table[1, 0], h], 64, 4, np.ones(64), np.ones(64))
    assert np.array_equal(cache.pool.cpu().numpy(), pool)
    k, v = R.rsd_kv4_read(cache, seq, slot)
    assert bool((k[:6] == 0).all()) and bool((v[:6] == 0).all()) and bool((k[6] == 1).all()) and bool((v[6] == 1).all())


# ---------------------------------------------------------------- attention

def check_attention(torch, R, cache, pool, table, lens, q, scale, starts, got, lse, score0=None, score1=None, dtype="f32"):
    hd, hkv = pool.shape[2] // 17, pool.shape[1]
    group = q.shape[1] // hkv
    q, got, lse = host(q), host(got), host(lse)
    for b, n in enumerate(lens):
        r0, r1 = starts[b], starts[b + 1]
        for h in range(hkv):
            k, v, there = ref.entries(pool, table[b], n, h, hd)
            cols = slice(h * group, (h + 1) * group)
            out, want_lse, weight, mass, spread = ref.attention(q[r0:r1, cols], k, v, there, scale, r1 - r0)
            score_err = 2 * (3 * hd / 32 + 48) * U * spread + 4 * U * spread
            rel = 2 * score_err + (n / 64 + 80) * 2 * U + 8 * U
            bound = rel * mass + U * np.abs(out) * 4 + 1e-37
            if dtype == "bf16":
                bound = bound + 2.0 ** -16 * mass + 2.0 ** -8 * np.abs(out)
            assert np.all(np.abs(got[r0:r1, cols] - out) <= bound), (b, h, np.max(np.abs(got[r0:r1, cols] - out) / bound))
            fine = np.isfinite(want_lse)
            assert np.array_equal(np.isneginf(lse[r0:r1, cols]), ~fine)
            assert np.all(np.abs(lse[r0:r1, cols][fine] - want_lse[fine]) <= (rel + 4 * U * (1 + np.abs(want_lse[fine]))))
            if score0 is not None:
                err = np.abs(score1[b, h, :n] - score0[b, h, :n] - weight)
                assert np.all(err <= 2 * rel * weight + 8 * U * spread * weight + 2 * U * np.abs(score1[b, h, :n]) + 1e-37), (b, h, err.max())
                assert np.array_equal(score1[b, h, n:], score0[b, h, n:])


ATTENTION = [  # heads, kv heads, head dim, lengths, rows of each sequence (None: one each, without row_start)
    (4, 2, 32, [1, 2, 15, 16, 17, 0, 33], None),
    (8, 2, 32, [63, 64, 65, 128, 200], None),
    (1, 1, 64, [5], None),
    (9, 3, 64, [31, 257, 70, 0], None),
    (16, 16, 64, [100, 48], None),
    (12, 2, 128, [1, 300, 64], None),
    (28, 4, 128, [129, 16, 7], None),
    (64, 8, 128, [90], None),
    (20, 1, 128, [70, 33], None),                          # more heads than columns of a tile
    (40, 1, 32, [50], None),
    (7, 1, 128, [1100, 20], None),
    (7, 1, 128, [2300, 20, 1030], None),                   # long enough to be split
    (4, 2, 32, [2100], [3]),
    (4, 2, 32, [20, 64, 5, 0, 90], [3, 1, 5, 0, 17]),
    (12, 2, 128, [40, 100, 16], [5, 33, 16]),              # a sequence that consists of its rows alone
    (28, 4, 128, [300, 65], [9, 2]),
    (9, 3, 64, [70, 7, 130], [8, 7, 1]),
    (16, 16, 64, [80], [40]),
    (8, 1, 128, [700, 66], [20, 3]),
    (8, 1, 128, [1100, 90], [20, 90]),                     # many columns, split; a whole prompt
    (9, 3, 64, [1090, 0, 33], [30, 0, 12]),
    (3, 1, 32, [1300], [40]),
    (6, 2, 64, [5, 3], [9, 4]),                            # more rows than entries: the first ones see nothing
]


@pytest.mark.parametrize("heads,hkv,hd,lens,rows", ATTENTION)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attention(torch, R, heads, hkv, hd, lens, rows, dtype):
    rng = np.random.default_rng(heads * hd + sum(lens))
    cache, pool, table = make_cache(torch, R, rng, lens, hkv, hd)
    counts = [1] * len(lens) if rows is None else rows
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    total = int(starts[-1])
    q = dev(torch, (rng.normal(size=(total, heads, hd)) * 1.5).astype(np.float32)).to(t)
    scale = 1 / np.sqrt(hd)
    kw = {} if rows is None else dict(row_start=dev(torch, starts), max_rows=max(rows))
    scores = dev(torch, rng.random((len(lens), hkv, table.shape[1] * 16 + 3)).astype(np.float32))[..., :table.shape[1] * 16]
    before = host(scores)
    out, lse = R.rsd_kv4_attention(cache, q, scale, scores=scores, want_lse=True, **kw)
    check_attention(torch, R, cache, pool, table, lens, q, float(np.float32(scale)), starts, out, lse, before, host(scores), dtype)
    assert np.array_equal(cache.pool.cpu().numpy(), pool)
    # the same bits without the weights, with a tight bound on the lengths where the parts stay the same, from strided q into strided out
    wide = torch.full((total, 2 * heads + 1, hd + 3), float("nan"), device="cuda", dtype=t)
    wide[:, 1:2 * heads:2, 2:hd + 2] = q
    into = torch.full((total, heads + 2, hd + 1), 3.0, device="cuda", dtype=t)
    R.rsd_kv4_attention(cache, wide[:, 1:2 * heads:2, 2:hd + 2], scale, out=into[:, 1:heads + 1, 1:], **kw)
    assert torch.equal(into[:, 1:heads + 1, 1:], out)
    assert bool((into[:, 0] == 3).all()) and bool((into[:, -1] == 3).all()) and bool((into[:, :, 0] == 3).all())
    out2, lse2 = R.rsd_kv4_attention(cache, q, scale, max_kv=max(max(lens), 1), want_lse=True, **kw)
    check_attention(torch, R, cache, pool, table, lens, q, float(np.float32(scale)), starts, out2, lse2, dtype=dtype)


# more blocks than run at once, lengths from none to long in any order; parts of which short sequences have one
UNEQUAL = [
    ("single tokens", 140, 4, 4, [300, 0, 17, 64, 1], 1),
    ("pieces of steps", 140, 16, 4, [300, 0, 17, 64, 12], 10),
    ("parts", 7, 16, 2, [2700, 0, 1290, 1344, 40, 1345, 2000], 9),
    ("single tokens in parts", 9, 8, 2, [2700, 0, 511, 512, 513, 40, 1025], 1),
]


@pytest.mark.parametrize("batch,heads,hkv,some,most", [u[1:] for u in UNEQUAL], ids=[u[0] for u in UNEQUAL])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scored", [False, True])
def test_attention_over_unequal_sequences(torch, R, batch, heads, hkv, some, most, dtype, scored):
    rng = np.random.default_rng(batch + heads)
    lens = [int(x) for x in rng.permutation(some + [int(n) for n in rng.integers(0, 70, batch - len(some))])]
    hd = 32
    # pages of arbitrary codes; NaN behind the last entry
    need = [-(-n // 16) for n in lens]
    pool = rng.integers(0, 256, (sum(need) + 3, hkv, 17 * hd)).astype(np.uint8)
    pool[:, :, 16 * hd:] = rng.integers(122, 127, (len(pool), hkv, hd))
    order, table = rng.permutation(len(pool)).astype(np.int32), np.full((batch, max(need)), -1, np.int32)
    for b, n in enumerate(lens):
        table[b, :need[b]] = order[sum(need[:b]):sum(need[:b + 1])]
        for s in range(n, 16 * need[b]):
            key, val, ks, vs = ref.entry_places(hd, s % 16)
            pool[table[b, need[b] - 1]][:, np.concatenate([ks, vs])] = 255
    cache = R.Kv4Cache(dev(torch, pool), dev(torch, table), dev(torch, np.array(lens, np.int32)))
    counts = [min(int(rng.integers(0, most + 1)), n) if most > 1 else 1 for n in lens]
    starts = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    q = dev(torch, (rng.normal(size=(int(starts[-1]), heads, hd)) * 1.5).astype(np.float32)).to(t)
    kw = {} if most == 1 else dict(row_start=dev(torch, starts), max_rows=most)
    scores = dev(torch, rng.random((batch, hkv, table.shape[1] * 16)).astype(np.float32)) if scored else None
    before = host(scores) if scored else None
    scale = 1 / np.sqrt(hd)
    out, lse = R.rsd_kv4_attention(cache, q, scale, scores=scores, want_lse=True, **kw)
    check_attention(torch, R, cache, pool, table, lens, q, float(np.float32(scale)), starts, out, lse, before, host(scores) if scored else None, dtype=dtype)


@pytest.mark.parametrize("cap", [64, 4000])
def test_attention_is_cut_to_max_kv_and_to_the_table(torch, R, cap):
    rng = np.random.default_rng(3)
    cache, pool, table = make_cache(torch, R, rng, [50, 90], 2, 64, cap=cap)
    q = dev(torch, rng.normal(size=(2, 4, 64)).astype(np.float32))
    long = R.Kv4Cache(cache.pool, cache.table, dev(torch, np.array([1 << 30, -7], np.int32)))
    out, lse = R.rsd_kv4_attention(long, q, 0.125, max_kv=48, want_lse=True)
    check_attention(torch, R, cache, pool, table, [48, 0], q, 0.125, [0, 1, 2], out, lse)
    # without the bound: every slot of the table counts, but entries without a page (table -1) are not seen
    n = table.shape[1] * 16
    clean = pool.copy()
    for s in range(50, 64):                                # what lies behind the 50 written ones is seen here: give it numbers
        for h in range(2):
            ref.write_entry(clean[table[0, s // 16], h], 64, s % 16, rng.normal(size=64), rng.normal(size=64))
    long = R.Kv4Cache(dev(torch, clean), cache.table, long.kv_len)
    out, lse = R.rsd_kv4_attention(long, q, 0.125, want_lse=True)
    check_attention(torch, R, long, clean, table, [n, 0], q, 0.125, [0, 1, 2], out, lse)


@pytest.mark.parametrize("rows", [1, 6])
def test_pages_outside_the_pool_are_not_seen(torch, R, rows):
    rng = np.random.default_rng(4)
    cache, pool, table = make_cache(torch, R, rng, [100, 60], 2, 128)
    table[0, 2], table[0, 4], table[1, 0], table[1, 1] = -1, len(pool) + 3, 1 << 30, -(1 << 31)
    cache = R.Kv4Cache(cache.pool, dev(torch, table), cache.kv_len)
    starts = np.array([0, rows, 2 * rows], np.int32)
    q = dev(torch, rng.normal(size=(2 * rows, 4, 128)).astype(np.float32))
    scores = torch.zeros(2, 2, table.shape[1] * 16, device="cuda")
    out, lse = R.rsd_kv4_attention(cache, q, 0.1, row_start=dev(torch, starts), max_rows=rows, scores=scores, want_lse=True)
    check_attention(torch, R, cache, pool, table, [100, 60], q, float(np.float32(0.1)), starts, out, lse, np.zeros(scores.shape), host(scores))


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", [5, 12, 40])
def test_nan_entries_reach_only_what_sees_them(torch, R, hd, rows):
    """A value group that reads as NaN: its 32 dims of the rows that see the entry; a key group: those rows whole."""
    rng = np.random.default_rng(hd)
    n, heads = 90, 6
    cache, pool, table = make_cache(torch, R, rng, [n], 2, hd)
    for what, slot in (("v", 85), ("k", 83), ("v", 88), ("v", 89), ("v", 20)):
        mine = pool.copy()
        place = ref.entry_places(hd, slot % 16)
        mine[table[0, slot // 16], 1, place[3 if what == "v" else 2][0]] = 255
        c = R.Kv4Cache(dev(torch, mine), cache.table, cache.kv_len)
        q = dev(torch, rng.normal(size=(rows, heads, hd)).astype(np.float32))
        out = R.rsd_kv4_attention(c, q, 0.2, row_start=dev(torch, np.array([0, rows], np.int32)), max_rows=rows)
        sees = n - (rows - 1 - np.arange(rows)) > slot
        bad = np.zeros((rows, heads, hd), bool)
        bad[np.ix_(sees, range(3, 6), range(32 if what == "v" else hd))] = True
        assert np.array_equal(np.isnan(host(out)), bad), what
        clean = R.rsd_kv4_attention(cache, q, 0.2, row_start=dev(torch, np.array([0, rows], np.int32)), max_rows=rows)
        assert torch.equal(out[:, :3], clean[:, :3])
        unseen = dev(torch, ~sees)
        assert torch.equal(out[unseen], clean[unseen])


def test_large_and_infinite_scores(torch, R):
    rng = np.random.default_rng(12)
    cache, pool, table = make_cache(torch, R, rng, [200, 70], 1, 64)
    q = dev(torch, (rng.normal(size=(2, 4, 64)) * 300).astype(np.float32))
    out, lse = R.rsd_kv4_attention(cache, q, 1.0, want_lse=True)
    check_attention(torch, R, cache, pool, table, [200, 70], q, 1.0, [0, 1, 2], out, lse)
    out, lse = R.rsd_kv4_attention(cache, q, 0.0, want_lse=True)
    check_attention(torch, R, cache, pool, table, [200, 70], q, 0.0, [0, 1, 2], out, lse)
    q[1, 2, 5] = float("nan")
    bad = np.isnan(host(R.rsd_kv4_attention(cache, q, 0.1)))
    assert bad[1, 2].all() and bad.sum() == 64


def test_row_starts_outside_the_rows_are_cut(torch, R):
    rng = np.random.default_rng(13)
    cache, pool, table = make_cache(torch, R, rng, [40, 50, 30], 2, 32)
    q = dev(torch, rng.normal(size=(6, 4, 32)).astype(np.float32))
    starts = np.array([-3, 2, 100, 50], np.int32)          # rows 0-1, 2-5, none
    out = torch.full_like(q, 9.0)
    R.rsd_kv4_attention(cache, q, 0.2, row_start=dev(torch, starts), max_rows=4, out=out)
    good = R.rsd_kv4_attention(cache, q, 0.2, row_start=dev(torch, np.array([0, 2, 6, 6], np.int32)), max_rows=4)
    assert torch.equal(out, good)
    # more rows than max_rows: the first max_rows are computed, as rows of a sequence of that many
    out = torch.full_like(q, 9.0)
    R.rsd_kv4_attention(cache, q, 0.2, row_start=dev(torch, np.array([0, 6, 6, 6], np.int32)), max_rows=2, out=out)
    two = R.rsd_kv4_attention(cache, q[:2].contiguous(), 0.2, row_start=dev(torch, np.array([0, 2, 2, 2], np.int32)), max_rows=2)
    assert torch.equal(out[:2], two) and bool((out[2:] == 9).all())


def test_offsets_beyond_32_bits(torch, R):
    """A pool of more than 4 GiB: entries in its last pages."""
    rng = np.random.default_rng(14)
    hd, hkv, n_pages = 128, 8, 260_000
    pool = torch.empty(n_pages, hkv, 17 * hd, dtype=torch.uint8, device="cuda")
    assert pool.numel() > 1 << 32
    table = np.array([[n_pages - 1, 5, n_pages - 2]], np.int32)
    cache = R.Kv4Cache(pool, dev(torch, table), dev(torch, np.array([40], np.int32)))
    x = rng.normal(size=(40, hkv, hd, 2)).astype(np.float32)
    seq, slot = dev(torch, np.zeros(40, np.int32)), dev(torch, np.arange(40, dtype=np.int32))
    R.rsd_kv4_append(cache, dev(torch, x[..., 0]), dev(torch, x[..., 1]), seq, slot)
    k, v = R.rsd_kv4_read(cache, seq, slot, dtype=torch.float32)
    assert np.array_equal(host(k), ref.quantize(x[..., 0])[2]) and np.array_equal(host(v), ref.quantize(x[..., 1])[2])
    q = dev(torch, rng.normal(size=(1, 16, hd)).astype(np.float32))
    scores, pos = torch.zeros(1, hkv, 48, device="cuda"), torch.arange(48, dtype=torch.int32, device="cuda").expand(1, hkv, 48).contiguous()
    out, lse = R.rsd_kv4_attention(cache, q, 0.1, scores=scores, want_lse=True)
    for h in range(hkv):
        want = ref.attention(host(q)[:, 2 * h:2 * h + 2], host(k)[:, h], host(v)[:, h], np.ones(40, bool), float(np.float32(0.1)), 1)
        assert np.all(np.abs(host(out)[:, 2 * h:2 * h + 2] - want[0]) <= 1e-5 * want[3] + 1e-6) and np.all(np.abs(host(scores)[0, h, :40] - want[2]) <= 1e-5)
    score0 = scores.cpu().numpy().copy()
    R.rsd_kv4_evict(cache, scores, pos, 24, 4)
    k2, v2 = R.rsd_kv4_read(cache, seq[:24].contiguous(), slot[:24].contiguous(), dtype=torch.float32)
    assert int(cache.kv_len[0]) == 24
    for h in range(hkv):
        kept, moves = ref.evict(score0[0, h], np.arange(48), 40, 24, 4)
        source = np.arange(24)
        for fr, to in moves:
            source[to] = fr
        assert np.array_equal(pos[0, h, :24].cpu().numpy(), source)
        assert np.array_equal(host(k2)[:, h], host(k)[source, h]) and np.array_equal(host(v2)[:, h], host(v)[source, h])


# ---------------------------------------------------------------- eviction

EVICT = [([5, 0, 12, 40], 12, 0, "plain"), ([100, 64, 16, 17], 16, 16, "plain"), ([100, 64, 16, 17], 16, 3, "ties"), ([33, 90], 1, 0, "plain"), ([33, 90], 1, 1, "ties"),
         ([300, 257, 256, 255], 200, 64, "ties"), ([300, 40], 290, 10, "odd"), ([1500, 1100], 700, 128, "odd"), ([1500, 2100], 1024, 0, "ties"), ([64], 64, 5, "plain"),
         ([2500], 1500, 0, "equal"), ([70, 90], 50, 20, "positions")]


@pytest.mark.parametrize("lens,budget,recent,kind", EVICT)
@pytest.mark.parametrize("hd,hkv", [(32, 3), (128, 1)])
def test_evict(torch, R, lens, budget, recent, kind, hd, hkv):
    rng = np.random.default_rng(sum(lens) + budget)
    need = [-(-max(n, 1) // 16) for n in lens]
    max_pages, total = max(need), sum(need) + 2
    pool = rng.integers(0, 256, (total, hkv, 17 * hd)).astype(np.uint8)
    table = np.full((len(lens), max_pages), -1, np.int32)
    order, at = rng.permutation(total), 0
    for b in range(len(lens)):
        table[b, :need[b]] = order[at:at + need[b]]
        at += need[b]
    cap = max_pages * 16
    score = rng.normal(size=(len(lens), hkv, cap)).astype(np.float32)
    if kind == "ties":
        score = np.floor(score * 2).astype(np.float32) * rng.choice([1.0, -0.0], score.shape).astype(np.float32)
    if kind == "equal":
        score[:] = 0.5
    if kind == "odd":
        score[rng.random(score.shape) < 0.2] = np.nan
        score[rng.random(score.shape) < 0.2] = np.inf
        score[rng.random(score.shape) < 0.2] = -np.inf
        score[rng.random(score.shape) < 0.1] = 1e-42
        score[rng.random(score.shape) < 0.1] = -1e-42
    pos = np.stack([[rng.permutation(cap) for _ in range(hkv)] for _ in lens]).astype(np.int32) * 3
    if kind == "positions":
        pos = pos - 100
        pos[0, :, 3], pos[1, :, 4] = 2 ** 31 - 1, -2 ** 31
    book = torch.zeros(2, len(lens), hkv, cap + 1, dtype=torch.int32, device="cuda")
    ds, dp = book[0].view(torch.float32)[..., :cap], book[1][..., :cap]
    ds.copy_(dev(torch, score))
    dp.copy_(dev(torch, pos))
    cache = R.Kv4Cache(dev(torch, pool), dev(torch, table), dev(torch, np.array(lens, np.int32)))
    want, ws, wp = pool.copy(), score.copy(), pos.copy()
    for b, n in enumerate(lens):
        for h in range(hkv):
            _, moves = ref.evict(score[b, h], pos[b, h].astype(np.int64), n, budget, recent)
            for fr, to in moves:
                src, dst = pool[table[b, fr // 16], h], want[table[b, to // 16], h]
                for a, c in zip(ref.entry_places(hd, fr % 16), ref.entry_places(hd, to % 16)):
                    dst[c] = src[a]
                ws[b, h, to], wp[b, h, to] = score[b, h, fr], pos[b, h, fr]
    for _ in range(2):                                     # a second call finds nothing to do
        R.rsd_kv4_evict(cache, ds, dp, budget, recent)
        assert np.array_equal(cache.kv_len.cpu().numpy(), np.minimum(lens, budget))
        assert np.array_equal(cache.pool.cpu().numpy(), want)
        assert np.array_equal(ds.cpu().numpy().view(np.int32), ws.view(np.int32)) and np.array_equal(dp.cpu().numpy(), wp)


@pytest.mark.parametrize("n", [12300, 16383, 16384, 16400, 17600])
def test_evict_from_long_lists(torch, R, n):
    """Lists whose keys fill the shared memory, and longer ones, which are read again instead."""
    rng = np.random.default_rng(n)
    hd, budget, recent, pages = 32, 600, 50, -(-n // 16)
    pool = rng.integers(0, 256, (pages, 1, 17 * hd)).astype(np.uint8)
    table = rng.permutation(pages).astype(np.int32)[None]
    score = np.floor(rng.normal(size=(1, 1, pages * 16)) * 50).astype(np.float32)
    pos = rng.permutation(pages * 16).astype(np.int32)[None, None]
    cache = R.Kv4Cache(dev(torch, pool), dev(torch, table), dev(torch, np.array([n], np.int32)))
    ds, dp = dev(torch, score), dev(torch, pos)
    _, moves = ref.evict(score[0, 0], pos[0, 0].astype(np.int64), n, budget, recent)
    want, ws, wp = pool.copy(), score.copy(), pos.copy()
    for fr, to in moves:
        for a, c in zip(ref.entry_places(hd, fr % 16), ref.entry_places(hd, to % 16)):
            want[table[0, to // 16], 0][c] = pool[table[0, fr // 16], 0][a]
        ws[0, 0, to], wp[0, 0, to] = score[0, 0, fr], pos[0, 0, fr]
    R.rsd_kv4_evict(cache, ds, dp, budget, recent)
    assert int(cache.kv_len[0]) == budget
    assert np.array_equal(cache.pool.cpu().numpy(), want)
    assert np.array_equal(ds.cpu().numpy(), ws) and np.array_equal(dp.cpu().numpy(), wp)


def test_evict_with_lengths_outside_the_table(torch, R):
    rng = np.random.default_rng(20)
    cache, pool, table = make_cache(torch, R, rng, [64, 64], 1, 32)
    cache = R.Kv4Cache(cache.pool, cache.table, dev(torch, np.array([1 << 30, -4], np.int32)))
    scores, pos = torch.rand(2, 1, 64, device="cuda"), torch.arange(64, dtype=torch.int32, device="cuda").expand(2, 1, 64).contiguous()
    kept, moves = ref.evict(scores[0, 0].cpu().numpy(), np.arange(64), 64, 40, 0)
    R.rsd_kv4_evict(cache, scores, pos, 40, 0)
    assert cache.kv_len.tolist() == [40, 0] and sorted(pos[0, 0, :40].tolist()) == list(kept)


# ---------------------------------------------------------------- streams, graphs, refusals

def _step(torch, R, seed, hd=64):
    rng = np.random.default_rng(seed)
    cache, pool, table = make_cache(torch, R, rng, [300, 40, 129], 2, hd, cap=640)
    packed, _ = weights(torch, R, rng, 6 * hd, 200)
    x = dev(torch, rng.normal(size=(3, 200)).astype(np.float32))
    scores = torch.zeros(3, 2, table.shape[1] * 16, device="cuda")
    pos = torch.arange(table.shape[1] * 16, dtype=torch.int32, device="cuda").expand(3, 2, -1).contiguous()
    seq, slot = dev(torch, np.arange(3, dtype=np.int32)), dev(torch, np.array([299, 39, 128], np.int32))

    def step():
        y = R.rsd_w4_linear(x, packed).view(3, 6, hd)
        R.rsd_kv4_append(cache, y[:, 4:5].expand(3, 2, hd), y[:, 5:6].expand(3, 2, hd), seq, slot, position=slot, entry_pos=pos, scores=scores)
        out = R.rsd_kv4_attention(cache, y[:, :4], 0.1, scores=scores)
        R.rsd_kv4_evict(cache, scores, pos, 100, 10)
        return out

    state = [cache.pool, cache.kv_len, scores, pos]
    return step, state


def test_another_stream_and_a_recorded_graph(torch, R):
    step, state = _step(torch, R, 30)
    start = [t.clone() for t in state]
    torch.cuda.synchronize()

    def reset():
        for t, s in zip(state, start):
            t.copy_(s)

    want = [step().clone()] + [t.clone() for t in state]
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip([out] + state, want))
    reset()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for i in range(4):
        reset()
        junk = torch.randn(1000 + i, 1000, device="cuda") @ torch.randn(1000, 50, device="cuda")
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([out] + state, want)), i
        assert bool(torch.isfinite(junk).all())


def test_refusals(torch, R):
    rng = np.random.default_rng(40)
    cache, pool, table = make_cache(torch, R, rng, [40, 20], 2, 64)
    cap = table.shape[1] * 16
    q = torch.zeros(2, 4, 64, device="cuda")
    kv = torch.zeros(2, 2, 64, device="cuda")
    idx = torch.zeros(2, dtype=torch.int32, device="cuda")
    book, pos = torch.zeros(2, 2, cap, device="cuda"), torch.zeros(2, 2, cap, dtype=torch.int32, device="cuda")
    packed, _ = weights(torch, R, rng, 20, 40)
    x = torch.zeros(3, 40, device="cuda")
    C = R.Kv4Cache
    bad = [
        lambda: R.rsd_w4_linear(x.half(), packed), lambda: R.rsd_w4_linear(x[:, :39], packed), lambda: R.rsd_w4_linear(x.cpu(), packed),
        lambda: R.rsd_w4_linear(x.t().contiguous().t(), packed), lambda: R.rsd_w4_linear(x, (packed.codes, packed.scales, 40, 40)),
        lambda: R.rsd_w4_linear(x, packed, out=torch.zeros(3, 20, device="cuda", dtype=torch.bfloat16)), lambda: R.rsd_w4_linear(x, packed, out=torch.zeros(3, 21, device="cuda")),
        lambda: R.rsd_w4_linear(x, packed, out=torch.zeros(1, 20, device="cuda").expand(3, 20)),
        lambda: R.rsd_w4_pack(x.half()), lambda: R.rsd_w4_pack(x[0]), lambda: R.rsd_w4_pack(x.t()), lambda: R.rsd_w4_pack(x[:0]),
        lambda: R.rsd_kv4_attention(C(cache.pool.int(), cache.table, cache.kv_len), q, 1.0), lambda: R.rsd_kv4_attention(C(cache.pool[..., 1:], cache.table, cache.kv_len), q, 1.0),
        lambda: R.rsd_kv4_attention(C(cache.pool, cache.table.long(), cache.kv_len), q, 1.0), lambda: R.rsd_kv4_attention(C(cache.pool, cache.table, cache.kv_len[:1]), q, 1.0),
        lambda: R.rsd_kv4_attention(C(cache.pool, cache.table[:, ::2], cache.kv_len), q, 1.0), lambda: R.rsd_kv4_attention(cache, q.half(), 1.0),
        lambda: R.rsd_kv4_attention(cache, q[:, :3], 1.0), lambda: R.rsd_kv4_attention(cache, q[:1], 1.0), lambda: R.rsd_kv4_attention(cache, q[..., :32], 1.0),
        lambda: R.rsd_kv4_attention(cache, q, 1.0, max_rows=2), lambda: R.rsd_kv4_attention(cache, q, 1.0, row_start=idx, max_rows=1),
        lambda: R.rsd_kv4_attention(cache, q, 1.0, scores=book[..., :cap - 1]), lambda: R.rsd_kv4_attention(cache, q, 1.0, scores=pos),
        lambda: R.rsd_kv4_attention(cache, q, 1.0, out=q.bfloat16()), lambda: R.rsd_kv4_attention(cache, q.cpu(), 1.0),
        lambda: R.rsd_kv4_append(cache, kv, kv.bfloat16(), idx, idx), lambda: R.rsd_kv4_append(cache, kv[:, :1], kv[:, :1], idx, idx),
        lambda: R.rsd_kv4_append(cache, kv, kv, idx[:1], idx), lambda: R.rsd_kv4_append(cache, kv, kv, idx, idx.long()),
        lambda: R.rsd_kv4_append(cache, kv, kv, idx, idx, entry_pos=pos), lambda: R.rsd_kv4_append(cache, kv.half(), kv.half(), idx, idx),
        lambda: R.rsd_kv4_read(cache, idx, idx[:1]), lambda: R.rsd_kv4_read(cache, idx, idx, dtype=torch.float16), lambda: R.rsd_kv4_read(cache, idx, idx, 128),
        lambda: R.rsd_kv4_evict(cache, book, pos, 0), lambda: R.rsd_kv4_evict(cache, book, pos, 4, 5), lambda: R.rsd_kv4_evict(cache, book, book, 4),
        lambda: R.rsd_kv4_evict(cache, book[:1], pos, 4),
    ]
    before = cache.pool.clone()
    for i, call in enumerate(bad):
        with pytest.raises(R.RsdError) as e:
            call()
        assert e.value.code == R.RSD_EINVAL, i
    assert torch.equal(cache.pool, before) and cache.kv_len.tolist() == [40, 20]

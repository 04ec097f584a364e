"""The operators on the paged bf16 / fp32 cache against their definitions in 64 bits (``kv_reference``).

Tolerances, derived from the number formats.  u = 2^-24.
* Norm: the sum of squares over one head adds 16 terms in a lane and up to 4 partial sums, 20 u of itself, half of it in the root; root, mean and eps 4 u, the products with the
  root and the weight 2 u: 16 u of a dimension.
* Rotation: the reduced angle is rounded to fp32 (at most half a turn: pi 2^-25 < 2 u), sine and cosine err by 4 u, times the magnitude 2 u; the angle itself comes from 64 bits, 3 * 2^-53 of at most 2^24
  radians: 8 u of each product and 2 u for the products and the sum: 10 u (|a| + |b|) for a pair.  Together at most 28 u (|a| + |b|) and the rounding of the result.
* A rounding of the result: 2^-8 of it in bf16, u in fp32.
* A score: products of bf16 numbers (an fp32 factor is three of them) are exact, each of at most 3 hd / 32 matrix instructions, or hd / 4 in fp32, adds its products and the sum so far with at
  most 2 u for each of 32 (4) additions, cut instead of rounded: 2 (hd + 48) u sum|q k|, and 4 u of the score for its factors.  A weight errs by twice the largest such error (its own and that of the sum's terms),
  relative; sums over n entries add at most 2 (n + 88) u, exp 8 u.
* bf16 activations: a weight is rounded to bf16 before it meets the values, 2^-8 of sum p|v|.
What the cache holds is equal to what was rounded into it; what is not written keeps its bits.
"""
import numpy as np
import pytest

import kv_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
PAIRS = [("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")]      # activations, cache


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


def kind(torch, name):
    return torch.float32 if name == "f32" else torch.bfloat16


def dev(torch, a, dtype):
    """(the array on the GPU, its rounded values in 64 bits)"""
    t = torch.from_numpy(np.ascontiguousarray(a)).to(dtype)
    return t.cuda(), t.double().numpy()


def ints(torch, a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")


def host(t):
    return t.detach().double().cpu().numpy()


def bits(torch, t):
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32).cpu()


def close(got, want, bound, what=""):
    got, want = np.asarray(got), np.asarray(want)
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        bad = ~same & ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(bound, got.shape)[bad][:3])


# ---------------------------------------------------------------- norms and rotation

ROPES = [(32, 32, False), (32, 32, True), (32, 8, False), (32, 16, True), (64, 64, False), (64, 20, False), (64, 20, True), (128, 128, False), (128, 128, True), (128, 64, False),
         (128, 2, True), (128, 126, False), (128, 0, False), (256, 256, False), (256, 128, True), (256, 96, False)]


def rope_of(torch, R, rot, interleaved, magnitude=1.0, theta=1e4):
    if not rot:
        return None, None
    freq = ref.frequencies(theta, rot)
    return (torch.tensor(freq, dtype=torch.float64, device="cuda"), interleaved, magnitude), (freq, interleaved, magnitude)


def rope_bound(x, weight, eps, rope, want, dtype):
    y = ref.turned(x, weight, eps, None, None) if weight is not None else np.asarray(x)
    return 28 * U * ref.partner_sums(y, rope) + HALF[dtype] * np.abs(want) * (1 + 2.0 ** -7) + 1e-44


@pytest.mark.parametrize("hd,rot,interleaved", ROPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope(torch, R, hd, rot, interleaved, dtype):
    rng = np.random.default_rng(hd * 1000 + rot + interleaved)
    for rows, heads, kv_heads, normed in ((1, 1, 1, True), (3, 5, 2, False), (67, 7, 1, True)):
        qkv, exact = dev(torch, rng.normal(size=(rows, heads + kv_heads + 1, hd)) * np.exp(rng.normal(size=(1, heads + kv_heads + 1, hd))), kind(torch, dtype))
        q, k = qkv[:, 1:heads + 1], qkv[:, heads + 1:]
        w = [dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, dtype)) if normed else (None, None) for _ in range(2)]
        position = np.concatenate([[1 << 20], rng.integers(-50, 1 << 17, rows)])[:rows]
        rope, rope64 = rope_of(torch, R, rot, interleaved, 1.25)
        got = R.rsd_qk_rope(q, k, ints(torch, position), rope, q_weight=w[0][0], k_weight=w[1][0], eps=1e-5)
        for g, x, (_, w64) in ((got[0], exact[:, 1:heads + 1], w[0]), (got[1], exact[:, heads + 1:], w[1])):
            want = ref.turned(x, w64, float(np.float32(1e-5)), position, rope64)
            close(host(g), want, rope_bound(x, w64, 1e-5, rope64, want, dtype), (rows, heads))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_in_place_strided_and_alone(torch, R, dtype):
    rng = np.random.default_rng(5)
    rope, rope64 = rope_of(torch, R, 40, False)
    buf, exact = dev(torch, rng.normal(size=(9, 4, 64)), kind(torch, dtype))
    view = buf[:, 1:3]
    before = bits(torch, buf)
    position = np.arange(9) * 977
    out, none = R.rsd_qk_rope(view, None, ints(torch, position), rope, q_out=view)
    want = ref.turned(exact[:, 1:3], None, 0, position, rope64)
    assert none is None and out.data_ptr() == view.data_ptr()
    close(host(view), want, rope_bound(exact[:, 1:3], None, 0, rope64, want, dtype))
    assert torch.equal(bits(torch, buf)[:, [0, 3]], before[:, [0, 3]])
    # rows and heads the other way round, addresses that are no multiple of 16 bytes
    flat, exact = dev(torch, rng.normal(size=(5 * 7 * 64 + 1)), kind(torch, dtype))
    x = flat[1:].view(5, 7, 64).transpose(0, 1)
    got, _ = R.rsd_qk_rope(x, None, ints(torch, position[:7]), rope)
    x64 = exact[1:].reshape(5, 7, 64).transpose(1, 0, 2)
    want = ref.turned(x64, None, 0, position[:7], rope64)
    close(host(got), want, rope_bound(x64, None, 0, rope64, want, dtype))
    # a norm alone, and a copy
    weight, w64 = dev(torch, rng.normal(size=64), kind(torch, dtype))
    got, _ = R.rsd_qk_rope(x, None, None, None, q_weight=weight, eps=0.0)
    want = ref.turned(x64, w64, 0, None, None)
    close(host(got), want, rope_bound(x64, w64, 0, None, want, dtype))
    assert torch.equal(R.rsd_qk_rope(x, None, None, None)[0], x)
    assert R.rsd_qk_rope(x[:0], None, None, None)[0].shape == (0, 5, 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rope_far_sizes_and_infinities(torch, R, dtype):
    rng = np.random.default_rng(6)
    x = rng.normal(size=(10, 2, 128))
    for i, s in enumerate((1e30, 1e19, 3e-20, 1e-30, 1e18)):
        x[i] *= s
    x[5] = 0.0
    x[6, 0, 100] = np.inf               # behind the rotation
    x[7, 1, 3] = np.nan
    x[8, 0, 5] = -np.inf
    t, exact = dev(torch, x, kind(torch, dtype))
    w, w64 = dev(torch, np.ones(128), kind(torch, dtype))
    rope, rope64 = rope_of(torch, R, 64, False)
    position = np.arange(10)
    for eps in (1e-6, 0.0):
        got, _ = R.rsd_qk_rope(t, None, ints(torch, position), rope, q_weight=w, eps=eps)
        with np.errstate(invalid="ignore", divide="ignore"):
            want = ref.turned(exact, w64, float(np.float32(eps)), position, rope64)
            bound = rope_bound(exact, w64, float(np.float32(eps)), rope64, want, dtype)
        fine = [0, 1, 2, 3, 4, 9] + ([5] if eps else [])
        close(host(got)[fine], want[fine], bound[fine], eps)
        assert np.isnan(host(got)[7, 1]).all() and np.isfinite(host(got)[7, 0]).all() and np.isfinite(host(got)[6, 1]).all()
    got, _ = R.rsd_qk_rope(t, None, ints(torch, position), rope)
    want = ref.turned(exact, None, 0, position, rope64)
    g = host(got)
    assert g[6, 0, 100] == np.inf and np.isfinite(np.delete(g[6, 0], 100)).all()
    assert not np.isfinite(g[8, 0, [5, 37]]).any() and np.isfinite(np.delete(g[8, 0], [5, 37])).all()


def test_rope_frequencies(torch, R):
    for rot, kw in ((128, dict()), (64, dict(scaling="linear", factor=4.0)), (128, dict(scaling="base", factor=8.0, theta=5e5)),
                    (128, dict(scaling="parts", factor=16.0, original=8192, theta=1e6)), (64, dict(scaling="parts", factor=8.0, original=8192, low=1, high=4, magnitude=1.0))):
        r = R.rsd_rope(rot, interleaved=True, **kw)
        args = dict(kw)
        theta, name, magnitude = args.pop("theta", 1e4), args.pop("scaling", "plain"), args.pop("magnitude", None)
        want = ref.frequencies(theta, rot, name, **args)
        assert np.allclose(r.freq.cpu().numpy(), want, rtol=1e-14, atol=0) and r.interleaved is True
        assert r.magnitude == (magnitude if magnitude is not None else 0.1 * np.log(16.0) + 1 if name == "parts" else 1.0)
    f = R.rsd_rope(64, scaling="base", factor=8.0).freq.cpu().numpy()
    assert f[0] == 1.0 and np.isclose(f[-1], ref.frequencies(1e4, 64)[-1] / 8)


# ---------------------------------------------------------------- the cache

def make_cache(torch, R, rng, lens, hkv, hd, dtype, spare=3, junk=None):
    """A cache whose pages lie in random order, every value of the pool arbitrary (or `junk`)."""
    need = [-(-n // 16) for n in lens]
    total, width = sum(need) + spare, max(max(need), 1)
    c = R.rsd_kv_cache(len(lens), width, total, hkv, hd, dtype=kind(torch, dtype))
    order = rng.permutation(total)
    table, at = np.full((len(lens), width), -1, np.int32), 0
    for b, m in enumerate(need):
        table[b, :m] = order[at:at + m]
        at += m
    c.table.copy_(ints(torch, table))
    c.kv_len.copy_(ints(torch, lens))
    c.pool.copy_(torch.from_numpy(rng.normal(size=c.pool.shape)) if junk is None else torch.full(c.pool.shape, junk))
    return c, table


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("rot,interleaved,normed", [(0, False, False), (32, False, True), (32, True, False), (10, False, True)])
def test_append_and_read(torch, R, act, held, hd, rot, interleaved, normed):
    rng = np.random.default_rng(hd + rot)
    for hkv, heads, lens in ((1, 1, [5]), (3, 6, [70, 0, 33, 16]), (2, 0, [1, 300])):
        c, table = make_cache(torch, R, rng, lens, hkv, hd, held)
        seq = np.repeat(np.arange(len(lens)), lens)
        slot = np.concatenate([np.arange(n) for n in lens])
        order = rng.permutation(len(seq)) if hkv == 3 else np.arange(len(seq))      # runs of neighbours, and none
        seq, slot = seq[order], slot[order]
        # rows that name no entry
        seq = np.concatenate([seq, [-1, len(lens), 0, 0, 0]])
        slot = np.concatenate([slot, [0, 0, -1, table.shape[1] * 16, 1 << 30]])
        rows = len(seq)
        position = rng.integers(0, 9000, rows)
        qkv, exact = dev(torch, rng.normal(size=(rows, heads + 2 * hkv, hd)), kind(torch, act))
        w, w64 = dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, act)) if normed else (None, None)
        rope, rope64 = rope_of(torch, R, rot, interleaved)
        before, before_bits = host(c.pool), bits(torch, c.pool)
        q = R.rsd_kv_append(c, qkv[:, heads:heads + hkv], qkv[:, heads + hkv:], ints(torch, seq), ints(torch, slot), position=ints(torch, position), rope=rope, k_weight=w,
                            q=qkv[:, :heads] if heads else None, q_weight=w if heads else None)
        if heads:
            want = ref.turned(exact[:, :heads], w64, 1e-6, position, rope64)
            close(host(q), want, rope_bound(exact[:, :heads], w64, 1e-6, rope64, want, act))
        else:
            assert q is None
        size = c.pool.element_size()
        k64, v64 = exact[:, heads:heads + hkv], exact[:, heads + hkv:]
        k64t = ref.turned(k64, w64, 1e-6, position, rope64)
        bound = np.zeros_like(before)
        ref.fill(before, table, size, hd, seq, slot, k64t, v64)
        ref.fill(bound, table, size, hd, seq, slot, rope_bound(k64, w64, 1e-6, rope64, k64t, held), HALF[held] * np.abs(v64) if act != held else 0 * v64)
        close(host(c.pool), before, bound)
        untouched = np.ones(before.shape, bool)
        ref.fill(untouched, table, size, hd, seq, slot, np.zeros_like(k64, bool), np.zeros_like(v64, bool))
        assert torch.equal(bits(torch, c.pool)[torch.from_numpy(untouched)], before_bits[torch.from_numpy(untouched)])
        rk, rv = R.rsd_kv_read(c, ints(torch, seq), ints(torch, slot))
        pool = host(c.pool)
        for i in range(rows):
            if i >= rows - 5:
                assert not host(rk[i]).any() and not host(rv[i]).any()
                continue
            block = pool[table[seq[i], slot[i] // 16]]
            assert np.array_equal(host(rk[i]), block[:, 0, ref.key_places(size, hd, slot[i] % 16)]) and np.array_equal(host(rv[i]), block[:, 1, ref.value_places(size, hd, slot[i] % 16)])
        # a page that the table does not have
        c.table[0, 0] = -1 if hkv != 3 else len(c.pool)
        kept = bits(torch, c.pool)
        R.rsd_kv_append(c, qkv[:, heads:heads + hkv], qkv[:, heads + hkv:], ints(torch, np.zeros(rows)), ints(torch, np.arange(rows) % 16))
        assert torch.equal(bits(torch, c.pool), kept)
        R.rsd_kv_append(c, qkv[:0, heads:heads + hkv], qkv[:0, heads + hkv:], ints(torch, []), ints(torch, []))


# ---------------------------------------------------------------- attention

def check_attention(torch, R, rng, lens, rows, heads, hkv, hd, act, held, window=0, sinks=0, scale=None, missing=(), max_rows=None, junk=np.nan, single=False, tight=True, spike=None,
                    want=None, strided=False, q_size=1.5):
    """Random entries, NaN behind the last one of each sequence; against the definition."""
    c, table = make_cache(torch, R, rng, lens, hkv, hd, held, junk=junk)
    size = c.pool.element_size()
    pool = host(c.pool)
    for b, n in enumerate(lens):
        k, v = rng.normal(size=(n, hkv, hd)) * np.exp(0.5 * rng.normal(size=(1, hkv, hd))), rng.normal(size=(n, hkv, hd))
        if spike:
            spike(b, k, v)
        ref.fill(pool, table, size, hd, np.full(n, b), np.arange(n), k, v)
    c.pool.copy_(torch.from_numpy(pool))
    pool = host(c.pool)
    for b, p in missing:
        table[b, p] = -1 if (b + p) % 2 else len(pool) + 7
    c.table.copy_(ints(torch, table))
    start = np.concatenate([[0], np.cumsum(rows)])
    total = int(start[-1]) + (0 if single else 2)           # two rows that no sequence has
    q, q64 = dev(torch, q_size * rng.normal(size=(total, heads, hd)), kind(torch, act))
    if strided:
        q = q.transpose(0, 1).contiguous().transpose(0, 1)
    scale = 1 / np.sqrt(hd) if scale is None else scale
    out = torch.full((total, heads, hd), 77.0, device="cuda", dtype=q.dtype)
    kw = dict(window=window, sinks=sinks)
    if not single:
        kw.update(row_start=ints(torch, start), max_rows=max_rows or (max(rows) if tight and max(rows) else None), max_kv=max(lens) if tight else None)
    got, lse = R.rsd_kv_attention(c, q, scale, out=out, want_lse=True, **kw)
    again, lse2 = R.rsd_kv_attention(c, q, scale, want_lse=True, **kw)
    g, gl = host(got), host(lse)
    for b, n in enumerate(lens):
        m = rows[b] if max_rows is None else min(rows[b], max_rows)
        r = slice(int(start[b]), int(start[b]) + m)
        if m == 0:
            continue
        assert torch.equal(bits(torch, got[r]), bits(torch, again[r])) and torch.equal(bits(torch, lse[r]), bits(torch, lse2[r]))      # the same call, the same bits
        k, v, there = ref.entries(pool, table[b], n, size, hd)
        o, l, mass, big = ref.attention(q64[r], k, v, there, np.float64(np.float32(scale)), window, sinks)
        ds = 2 * (hd + 48) * U * big + 8 * U * np.abs(np.where(np.isfinite(l), l, 0)) + 8 * U * big
        rel = 2 * ds + 2 * (n + 96) * U
        close(g[r], o, (rel[..., None] + (2.0 ** -8 if act == "bf16" else 0)) * mass * 1.01 + HALF[act] * np.abs(o) + 1e-42, ("out", b, n, m))
        close(gl[r], l, ds + 2 * (n + 96) * U + 4 * U * np.abs(np.where(np.isfinite(l), l, 0)), ("lse", b))
        assert (host(out[int(start[b]) + m:int(start[b + 1])]) == 77.0).all()
    assert (g[int(start[-1]):] == 77.0).all()
    return g, gl, start


GROUPS = [(1, 1), (4, 2), (7, 1), (12, 2), (9, 3), (20, 1)]


@pytest.mark.parametrize("heads,hkv", GROUPS)
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_single_tokens(torch, R, act, held, hd, heads, hkv):
    rng = np.random.default_rng(heads * 10 + hd)
    check_attention(torch, R, rng, [1, 0, 15, 16, 17, 31, 32, 33, 100, 257, 640], [1] * 11, heads, hkv, hd, act, held, single=True)
    check_attention(torch, R, rng, [2300], [1], heads, hkv, hd, act, held, single=True)


@pytest.mark.parametrize("lens,rows", [([1, 2, 40], [1, 2, 3]), ([0, 5, 64, 130], [1, 0, 5, 7]), ([300], [9]), ([33, 50, 90], [33, 20, 40]), ([700, 129], [70, 129]), ([3, 20], [7, 33])],
                         ids=str)
@pytest.mark.parametrize("heads,hkv", [(4, 2), (7, 1), (3, 3)])
@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_chunks(torch, R, act, held, hd, heads, hkv, lens, rows):
    rng = np.random.default_rng(len(lens) * 100 + sum(rows) + hd)
    check_attention(torch, R, rng, lens, rows, heads, hkv, hd, act, held)
    check_attention(torch, R, rng, lens, rows, heads, hkv, hd, act, held, tight=False, strided=True)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 3), (16, 0), (17, 16), (33, 4), (100, 40), (64, 1000), (1 << 30, 2), ((1 << 31) - 1, (1 << 31) - 1)])
@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_windows(torch, R, act, held, window, sinks):
    rng = np.random.default_rng(window % 1000 + sinks % 1000)
    for hd, heads, hkv in ((64, 4, 2), (128, 7, 1)):
        check_attention(torch, R, rng, [1, 0, 31, 200, 515, 130], [1] * 6, heads, hkv, hd, act, held, window, sinks, single=True)
        check_attention(torch, R, rng, [9, 300, 140, 2], [9, 40, 140, 5], heads, hkv, hd, act, held, window, sinks)
        # pages behind the window are gone
        gone = [(0, p) for p in range(sinks // 16 + 1, (900 - 3 - window) // 16)] if sinks < 900 and window < 900 else []
        check_attention(torch, R, rng, [900], [3], heads, hkv, hd, act, held, window, sinks, missing=gone)


@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_missing_pages_and_row_limits(torch, R, act, held):
    rng = np.random.default_rng(3)
    check_attention(torch, R, rng, [100, 64, 40], [5, 30, 1], 6, 2, 64, act, held, missing=[(0, 0), (0, 3), (1, 0), (1, 1), (1, 2), (1, 3), (2, 2)])
    check_attention(torch, R, rng, [100, 64], [9, 3], 6, 2, 32, act, held, max_rows=4)
    check_attention(torch, R, rng, [100, 640], [90, 3], 2, 2, 128, act, held, max_rows=50)


@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("hd", [32, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (20, 3)])
def test_attention_nonfinite_entries_reach_only_rows_that_see_them(torch, R, act, held, hd, window, sinks):
    rng = np.random.default_rng(8)
    bad = {0: (95, np.nan, "v"), 1: (60, np.inf, "v"), 2: (77, -np.inf, "v"), 3: (90, np.nan, "k"), 4: (40, np.nan, "v"), 5: (1, np.inf, "v")}

    def spike(b, k, v):
        at, x, which = bad[b]
        (v if which == "v" else k)[at, 0, 5] = x

    for m in (1, 11, 40):
        lens, rows = [100, 66, 80, 95, 64, 300], [m] * 6
        g, gl, start = check_attention(torch, R, rng, lens, rows, 6, 2, hd, act, held, window, sinks, spike=spike)
        for b, n in enumerate(lens):
            at, x, which = bad[b]
            sees = ref.seen(n, m, window, sinks)[:, at]
            o = g[start[b]:start[b] + m]
            if which == "v":
                assert (np.isfinite(o[:, :3, 5]).all(-1) == ~sees).all() and np.isfinite(np.delete(o, 5, -1)).all()
            else:
                assert (np.isfinite(o[:, :3]).all((-1, -2)) == ~sees).all()
            assert np.isfinite(o[:, 3:]).all()


@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_scores_at_the_ends_of_their_range(torch, R, act, held):
    rng = np.random.default_rng(9)
    for scale in (0.0, -0.3, 4.0):
        check_attention(torch, R, rng, [50, 700], [3, 20], 4, 2, 64, act, held, scale=scale, q_size=0.5)

    def spike(b, k, v):
        k[:] = 0
        k[..., 0] = -np.inf if b == 0 else 0.5
    # q positive: scores -inf with all that a row sees, or finite ones
    c, table = make_cache(torch, R, rng, [40, 40], 1, 64, held, junk=0.0)
    pool = host(c.pool)
    for b in range(2):
        k, v = np.zeros((40, 1, 64)), rng.normal(size=(40, 1, 64))
        spike(b, k, v)
        ref.fill(pool, table, c.pool.element_size(), 64, np.full(40, b), np.arange(40), k, v)
    c.pool.copy_(torch.from_numpy(pool))
    q = torch.zeros(2, 2, 64, device="cuda", dtype=kind(torch, act))
    q[..., 0] = 1.0
    out, lse = R.rsd_kv_attention(c, q, 1.0, want_lse=True)
    assert not host(out[0]).any() and (host(lse[0]) == -np.inf).all() and np.isfinite(host(out[1])).all() and host(out[1]).any()
    # growing scores: the maximum moves in every chunk; two tokens share the weight at last
    c, table = make_cache(torch, R, rng, [512], 1, 32, held, junk=0.0)
    pool = host(c.pool)
    k, v = np.zeros((512, 1, 32)), rng.normal(size=(512, 1, 32))
    k[:, 0, 0] = np.arange(512) // 2
    ref.fill(pool, table, c.pool.element_size(), 32, np.zeros(512, int), np.arange(512), k, v)
    c.pool.copy_(torch.from_numpy(pool))
    q = torch.zeros(1, 1, 32, device="cuda", dtype=kind(torch, act))
    q[..., 0] = 64.0
    pool = host(c.pool)
    want, wl, mass, _ = ref.attention(host(q), *ref.entries(pool, table[0], 512, c.pool.element_size(), 32), 1.0)
    out, lse = R.rsd_kv_attention(c, q, 1.0, want_lse=True)
    close(host(out), want, (2.0 ** -8 if act == "bf16" else 0) * mass * 1.01 + HALF[act] * np.abs(want) + 2000 * U * mass)
    close(host(lse), wl, 8 * U * np.abs(wl) + 1e-6)


@pytest.mark.parametrize("act,held", PAIRS)
def test_attention_into_q_and_long_pools(torch, R, act, held):
    rng = np.random.default_rng(12)
    hd, hkv, heads = 64, 2, 6
    for lens, rows in (([40, 130], [1, 3]), ([3000], [1]), ([400, 77], [60, 70])):
        c, table = make_cache(torch, R, rng, lens, hkv, hd, held)
        q, _ = dev(torch, rng.normal(size=(sum(rows), heads, hd)), kind(torch, act))
        start = ints(torch, np.concatenate([[0], np.cumsum(rows)]))
        want = R.rsd_kv_attention(c, q, 0.125, row_start=start)
        got = R.rsd_kv_attention(c, q, 0.125, row_start=start, out=q)
        assert got.data_ptr() == q.data_ptr() and torch.equal(bits(torch, got), bits(torch, want))
    # a pool whose last pages lie more than 2^32 bytes, and 2^31 values, behind its start
    pages = (1 << 32) // (c.pool[0].numel() * c.pool.element_size()) + (1 << 31) // c.pool[0].numel() + 64
    big = torch.empty(pages, *c.pool.shape[1:], device="cuda", dtype=c.pool.dtype)
    small, table = make_cache(torch, R, rng, [100, 50], hkv, hd, held)
    far = table.copy()
    far[table >= 0] += pages - len(small.pool)
    seq, slot = np.repeat([0, 1], [100, 50]), np.concatenate([np.arange(100), np.arange(50)])
    kv, _ = dev(torch, rng.normal(size=(150, 2 * hkv, hd)), kind(torch, act))
    q, _ = dev(torch, rng.normal(size=(2, heads, hd)), kind(torch, act))
    outs = []
    for cache in (small, (big, ints(torch, far), small.kv_len)):
        R.rsd_kv_append(cache, kv[:, :hkv], kv[:, hkv:], ints(torch, seq), ints(torch, slot))
        outs.append((R.rsd_kv_attention(cache, q, 0.125), *R.rsd_kv_read(cache, ints(torch, seq), ints(torch, slot))))
    for a, b in zip(*outs):
        assert torch.equal(bits(torch, a), bits(torch, b))


# ---------------------------------------------------------------- together, as a program runs them

def run_model(torch, R, act, held, window, sinks, pieces, seed=21, graph=False):
    """Prompts in pieces, then single tokens, of three sequences through norms, rotation, cache and attention; every output, against the definition over all tokens."""
    rng = np.random.default_rng(seed)
    hd, hkv, heads, batch = 64, 2, 6, 3
    total = sum(pieces)
    qkv, exact = dev(torch, rng.normal(size=(total, batch, heads + 2 * hkv, hd)), kind(torch, act))
    qw, qw64 = dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, act))
    kw, kw64 = dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, act))
    rope = R.rsd_rope(hd, 1e4, scaling="parts", factor=4.0, original=64)
    rope64 = (ref.frequencies(1e4, hd, "parts", 4.0, 64), False, 0.1 * np.log(4.0) + 1)
    c, table = make_cache(torch, R, rng, [total] * batch, hkv, hd, held, junk=np.nan)
    c.kv_len.zero_()
    got, at = [], 0
    for m in pieces:
        rows = qkv[at:at + m].transpose(0, 1).reshape(batch * m, heads + 2 * hkv, hd)
        seq, slot = ints(torch, np.repeat(np.arange(batch), m)), ints(torch, np.tile(np.arange(at, at + m), batch))
        q = R.rsd_kv_append(c, rows[:, heads:heads + hkv], rows[:, heads + hkv:], seq, slot, position=slot, rope=rope, k_weight=kw, q=rows[:, :heads], q_weight=qw)
        q2, _ = R.rsd_qk_rope(rows[:, :heads], None, slot, rope, q_weight=qw)
        assert torch.equal(bits(torch, q), bits(torch, q2))
        c.kv_len.fill_(at + m)
        start = None if m == 1 else ints(torch, np.arange(batch + 1) * m)
        o = R.rsd_kv_attention(c, q, 0.125, row_start=start, max_rows=m, window=window, sinks=sinks)
        got.append(o.view(batch, m, heads, hd))
        at += m
    q64 = ref.turned(exact[..., :heads, :].reshape(total * batch, heads, hd), qw64, 1e-6, np.repeat(np.arange(total), batch), rope64)
    size = c.pool.element_size()
    pool = host(c.pool)
    out = host(torch.cat(got, 1))
    for b in range(batch):
        k, v, there = ref.entries(pool, table[b], total, size, hd)
        qb = q64.reshape(total, batch, heads, hd)[:, b]
        want, _, mass, big = ref.attention(qb, k, v, there, 0.125, window, sinks)
        # q is rounded to its type before it scores: half a step of every dimension, 28 u for norm and rotation
        ds = (2 * (hd + 48) * U + HALF[act] + 64 * U) * big
        close(out[b], want, (2 * ds[..., None] * np.exp(2 * ds[..., None]) + 2 * (total + 96) * U + (2.0 ** -8 if act == "bf16" else 0)) * mass * 1.05 + HALF[act] * np.abs(want) * 1.01 + 1e-42)
    return out


@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 4)])
def test_a_run_of_the_operators(torch, R, act, held, window, sinks):
    run_model(torch, R, act, held, window, sinks, [37, 1, 1, 5, 20, 1, 1])


def test_captured_step_and_two_streams(torch, R):
    """A step recorded into a graph, replayed with other inputs between eager calls; two graphs and an eager call at once on streams of their own."""
    rng = np.random.default_rng(30)
    hd, hkv, heads, batch = 128, 2, 8, 4
    rope = R.rsd_rope(hd)

    def program(c, qkv, slot, seq, max_kv):
        q = R.rsd_kv_append(c, qkv[:, heads:heads + hkv], qkv[:, heads + hkv:], seq, slot, position=slot, rope=rope, q=qkv[:, :heads])
        return R.rsd_kv_attention(c, q, 0.1, max_kv=max_kv, window=300, sinks=4)

    lens = [1500, 33, 900, 1200]
    states = []
    for i in range(2):
        c, _ = make_cache(torch, R, rng, [n + 64 for n in lens], hkv, hd, "bf16")
        c.kv_len.copy_(ints(torch, lens))
        qkv = torch.zeros(batch, heads + 2 * hkv, hd, device="cuda", dtype=torch.bfloat16)
        states.append((c, qkv, ints(torch, np.array(lens) - 1), ints(torch, np.arange(batch))))
    for s in states:
        program(*s, 1600)
    torch.cuda.synchronize()
    graphs, outs, streams = [], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for s in states:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(program(*s, 1600))
        graphs.append(g)
    for step in range(4):
        fresh = [torch.from_numpy(rng.normal(size=s[1].shape)).to(torch.bfloat16).cuda() for s in states]
        for s, f in zip(states, fresh):
            s[1].copy_(f)
            s[0].kv_len.add_(1)
            s[2].add_(1)
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s, o in zip(states, outs):
            replayed = o.clone()
            assert torch.equal(bits(torch, replayed), bits(torch, program(*s, 1600)))
            with torch.cuda.stream(streams[step % 2]):
                other = program(*s, 1600)
            torch.cuda.synchronize()
            assert torch.equal(bits(torch, other), bits(torch, replayed))

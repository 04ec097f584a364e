"""Attention and entries of the paged bf16 / fp32 cache at the shapes that choose a kernel, a tile, a number of parts or an order of the blocks; calls at the ends of what the header allows.

The definition and the tolerances are those of ``test_gpu_kv``; where two calls differ in nothing that a result depends on, their bits are equal."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import PAIRS, R, bits, check_attention, dev, host, ints, kind, make_cache, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# 128 columns to a block: two tiles of rows by 16 kv heads and 3 sequences, four parts of 4100 entries; and 384 blocks that are not split
LONG = ([4100, 700, 300], [18, 200, 129], 16, 16)
EVEN = ([900, 0, 1, 40, 77] + [33 + i for i in range(18)] + [850], [40, 3, 1, 40, 5] + [1 + i % 7 for i in range(18)] + [37], 32, 16)


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("sizes", [LONG, EVEN], ids=["parts", "whole"])
def test_tiles_of_128_columns(torch, R, sizes, hd):
    rng = np.random.default_rng(hd)
    lens, rows, heads, hkv = sizes
    check_attention(torch, R, rng, lens, rows, heads, hkv, hd, "bf16", "bf16")


@pytest.mark.parametrize("sizes,window,sinks,scale", [(LONG, 2500, 20, None), (LONG, 150, 0, -0.2), (EVEN, 30, 17, None)], ids=str)
def test_tiles_of_128_columns_windows_missing_pages_and_strides(torch, R, sizes, window, sinks, scale):
    rng = np.random.default_rng(window)
    lens, rows, heads, hkv = sizes
    b = 1 if sizes is LONG else 3
    check_attention(torch, R, rng, lens, rows, heads, hkv, 64, "bf16", "bf16", window, sinks, scale=scale, missing=[(0, 0), (0, 40), (0, 41), (b, 1), (2, 0)], strided=True)


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3)])
@pytest.mark.parametrize("sizes", [LONG, EVEN], ids=["parts", "whole"])
def test_tiles_of_128_columns_nonfinite_entries(torch, R, sizes, window, sinks):
    rng = np.random.default_rng(5)
    lens, rows, heads, hkv = sizes
    bad = {0: (lens[0] - 6, np.nan, "v"), 1: (640, np.inf, "v"), 2: (290, -np.inf, "v"), 3: (20, np.nan, "k"), len(lens) - 1: (830 if sizes is EVEN else 250, np.nan, "k")}

    def spike(b, k, v):
        if b in bad and bad[b][0] < len(k):
            at, x, which = bad[b]
            (v if which == "v" else k)[at, 0, 5] = x

    g, _, start = check_attention(torch, R, rng, lens, rows, heads, hkv, 32, "bf16", "bf16", window, sinks, spike=spike)
    group = heads // hkv
    for b, n in enumerate(lens):
        m, o = rows[b], g[start[b]:start[b + 1]]
        assert np.isfinite(o[:, group:]).all()
        if b in bad and bad[b][0] < n:
            sees = ref.seen(n, m, window, sinks)[:, bad[b][0]]
            assert (np.isfinite(o[:, :group]).all((-1, -2)) == ~sees).all()
        else:
            assert np.isfinite(o).all()


@pytest.mark.parametrize("window,sinks", [(0, 0), (2500, 40), (70, 70)])
@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("hd", [32, 128])
def test_steps_whose_entries_are_split(torch, R, act, held, hd, window, sinks):
    rng = np.random.default_rng(window + hd)
    check_attention(torch, R, rng, [3000, 5, 1400], [6, 5, 3], 14, 2, hd, act, held, window, sinks, missing=[(0, 90), (2, 87)])
    check_attention(torch, R, rng, [5, 2600], [1, 9], 16, 2, hd, act, held, window, sinks, missing=[(1, p) for p in range(70)])


@pytest.mark.parametrize("act,held", PAIRS)
def test_infinite_entries_in_one_of_many_parts(torch, R, act, held):
    rng = np.random.default_rng(6)
    for at, x, which in ((10, np.inf, "v"), (2990, np.nan, "v"), (1500, -np.inf, "v"), (2996, np.nan, "k")):
        def spike(b, k, v):
            if b == 0:
                (v if which == "v" else k)[at, 1, 3] = x

        for rows in ([6, 2], [1, 1]):
            g, _, start = check_attention(torch, R, rng, [3000, 1400], rows, 14, 2, 64, act, held, spike=spike)
            sees = ref.seen(3000, rows[0], 0, 0)[:, at]
            assert (np.isfinite(g[:rows[0], 7:]).all((-1, -2)) == ~sees).all() and np.isfinite(g[:rows[0], :7]).all() and np.isfinite(g[rows[0]:start[-1]]).all()


@pytest.mark.parametrize("batch,heads,hkv,most,rows", [(130, 8, 4, 210, 1), (600, 2, 1, 150, 1), (70, 72, 8, 40, 5), (67, 16, 16, 300, 2)], ids=str)
@pytest.mark.parametrize("act,held", PAIRS)
def test_many_sequences_longest_first(torch, R, act, held, batch, heads, hkv, most, rows):
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, most + 1, batch)
    lens[:4], lens[-3:] = most, 0                           # equal ones at either end
    m = np.ones(batch, int) if rows == 1 else rng.integers(0, rows + 1, batch)
    m[0] = rows
    check_attention(torch, R, rng, lens.tolist(), m.tolist(), heads, hkv, 32, act, held, single=rows == 1)


@pytest.mark.parametrize("batch,heads,hkv,most", [(9, 5, 1, 40), (64, 2, 1, 90), (33, 6, 3, 30), (5, 16, 8, 60), (13, 5, 5, 70), (65, 2, 1, 90), (8, 17, 17, 20)], ids=str)
@pytest.mark.parametrize("act,held", PAIRS)
def test_sequences_with_unlike_numbers_of_rows(torch, R, act, held, batch, heads, hkv, most):
    """Most tiles of columns have no row; none at all, one row, all rows, more rows than entries; long ones in parts."""
    rng = np.random.default_rng(batch * hkv)
    m = rng.integers(0, 9, batch)
    m[1], m[-1] = most, 0
    lens = rng.integers(0, 100, batch)
    lens[0] = 1300 if batch < 10 else 200
    lens[2:5] = lens[1]
    check_attention(torch, R, rng, lens.tolist(), m.tolist(), heads, hkv, 32, act, held, tight=batch % 2 == 0)
    check_attention(torch, R, rng, lens.tolist(), m.tolist(), heads, hkv, 64, act, held, 24, 5, missing=[(0, 3)])


@pytest.mark.parametrize("heads,rows", [(64, 1), (64, 3), (96, 5), (17, 2), (129, 1)])
@pytest.mark.parametrize("act,held", PAIRS)
def test_large_groups(torch, R, act, held, heads, rows):
    rng = np.random.default_rng(heads)
    check_attention(torch, R, rng, [600, 31, rows], [rows, 1, rows], heads, 1, 64, act, held)


@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_addresses_aligned_to_their_type_only(torch, R, act, held, hd):
    rng = np.random.default_rng(hd)
    t, heads, hkv = kind(torch, act), 6, 2
    for lens, rows in (([700, 40], [1, 1]), ([2500, 40], [1, 1]), ([300, 120], [60, 45]), ([3000, 9], [9, 9])):
        c, _ = make_cache(torch, R, rng, lens, hkv, hd, held)
        total, start = sum(rows), ints(torch, np.concatenate([[0], np.cumsum(rows)]))
        q, _ = dev(torch, rng.normal(size=(total, heads, hd)), t)
        want, lse = R.rsd_kv_attention(c, q, 0.1, row_start=start, max_rows=max(rows), want_lse=True)
        step = heads * (hd + 1) + 3
        odd = [torch.full((total * step + 9,), 5.0, device="cuda", dtype=t)[i:i + total * step].view(total, step)[:, :heads * (hd + 1)].view(total, heads, hd + 1)[..., :hd] for i in (1, 3)]
        odd[0].copy_(q)
        got, lse2 = R.rsd_kv_attention(c, odd[0], 0.1, row_start=start, max_rows=max(rows), want_lse=True, out=odd[1])
        assert got.data_ptr() % 16 and torch.equal(bits(torch, got), bits(torch, want)) and torch.equal(bits(torch, lse2), bits(torch, lse))
        whole = odd[1]._base if odd[1]._base is not None else odd[1]
        kept = torch.ones_like(whole, dtype=torch.bool)
        torch.as_strided(kept, odd[1].shape, odd[1].stride(), odd[1].storage_offset()).fill_(False)
        assert (whole[kept] == 5.0).all()


@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("lens,rows", [([300, 40], [1, 1]), ([300, 60], [7, 3]), ([300, 150], [90, 20])], ids=str)
def test_infinite_queries_stay_in_their_rows(torch, R, act, held, lens, rows):
    """A result is off by at most 2^-8 sum p|v| for bf16 weights, 2^-8 of itself for its rounding, and what its scores err by: with 300 entries, |scale q k| sums of at most 60 and
    heads of 64, 4 * 2 * 112 * 2^-24 * 60 < 2^-8 of sum p|v|.  Two results without an infinity beside them differ by at most twice that, and sum p|v| <= max |v|."""
    rng = np.random.default_rng(8)
    hd, hkv, heads, total = 64, 2, 6, sum(rows)
    c, _ = make_cache(torch, R, rng, lens, hkv, hd, held)
    most = float(c.pool[:, :, 1].abs().max())
    q, _ = dev(torch, rng.normal(size=(total, heads, hd)), kind(torch, act))
    assert float(q.abs().max()) * float(c.pool[:, :, 0].abs().max()) * 0.04 * hd < 60
    kw = dict(row_start=ints(torch, np.concatenate([[0], np.cumsum(rows)])), max_rows=max(rows), want_lse=True)
    want, lse = (host(x) for x in R.rsd_kv_attention(c, q, 0.04, **kw))
    at = rng.permutation(total * heads)[:max(total * heads // 5, 3)]
    mark = np.zeros(total * heads, bool)
    mark[at] = True
    mark = mark.reshape(total, heads)
    bad = q.clone()
    for i, x in enumerate(at):
        bad[x // heads, x % heads, int(rng.integers(hd))] = (np.nan, np.inf, -np.inf)[i % 3]
    got, lse2 = (host(x) for x in R.rsd_kv_attention(c, bad, 0.04, **kw))
    assert not np.isfinite(got[mark]).all(-1).any() and np.isfinite(got[~mark]).all()
    assert (np.abs(got[~mark] - want[~mark]) <= (2 ** -5 if act == "bf16" else 2 ** -7) * most).all() and (np.abs(lse2[~mark] - lse[~mark]) <= 2 ** -7).all()


@pytest.mark.parametrize("act,held", PAIRS)
def test_lengths_that_the_device_cuts(torch, R, act, held):
    rng = np.random.default_rng(4)
    hd, hkv, heads, lens = 64, 2, 6, [200, 64, 96]
    c, table = make_cache(torch, R, rng, lens, hkv, hd, held)
    q, _ = dev(torch, rng.normal(size=(9, heads, hd)), kind(torch, act))
    start = ints(torch, [0, 3, 7, 9])

    def run(lengths, q=q, **kw):
        cache = (c.pool, c.table, ints(torch, lengths))
        out = torch.full_like(q, 7.0)
        o, lse = R.rsd_kv_attention(cache, q, 0.1, out=out, want_lse=True, **kw)
        return bits(torch, o), bits(torch, lse)

    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    cap = table.shape[1] * 16
    # no entries: nothing is seen
    for kw in (dict(row_start=start, max_rows=4), dict(q=q[:3])):
        o, lse = R.rsd_kv_attention(c, kw.get("q", q), 0.1, want_lse=True, max_kv=0, **{k: v for k, v in kw.items() if k != "q"})
        assert not host(o).any() and (host(lse) == -np.inf).all()
        assert same(run([0, -5, -(1 << 31)], max_kv=64, **kw), run([0, 0, 0], max_kv=64, **kw))
        # more than the table, or max_kv, has
        assert same(run([cap, cap + 1, (1 << 31) - 1], **kw), run([cap] * 3, **kw))
        assert same(run(lens, max_kv=70, **kw), run([70, 64, 70], max_kv=70, **kw))
        assert same(run(lens, max_kv=1 << 40, **kw), run(lens, **kw))
    # rows that are not there
    o, _ = run(lens, row_start=ints(torch, [-4, 3, 7, 1000]), max_rows=4)
    assert torch.equal(o, run(lens, row_start=start, max_rows=4)[0])
    o, _ = run(lens, row_start=ints(torch, [0, 3, 2, -9]), max_rows=4)      # the second sequence has none, nor the third
    assert torch.equal(o[:2], run(lens, row_start=ints(torch, [0, 3, 3, 3]), max_rows=4)[0][:2])
    # a window longer than all there is
    for rows in (dict(row_start=start, max_rows=4), dict(q=q[:3])):
        assert same(run(lens, window=cap, sinks=3, **rows), run(lens, **rows))


def test_graphs_that_share_a_pool_of_memory(torch, R):
    """Two graphs whose workspaces may lie at the same addresses, replayed in turn with eager calls between."""
    rng = np.random.default_rng(2)
    hd, hkv, heads = 128, 2, 8
    lens = [3000, 700, 2222]
    c, _ = make_cache(torch, R, rng, lens, hkv, hd, "bf16")
    q = [dev(torch, rng.normal(size=(n, heads, hd)), torch.bfloat16)[0] for n in (3, 27)]
    starts = [None, ints(torch, [0, 9, 18, 27])]

    def run(i):
        return R.rsd_kv_attention(c, q[i], 0.1, row_start=starts[i], max_rows=(1, 9)[i])

    want = [bits(torch, run(i)) for i in range(2)]
    graphs, outs, pool = [], [], None
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(run(i))
        graphs.append(g)
        pool = pool or g.pool()
    for step in range(3):
        for i in (0, 1) if step % 2 else (1, 0):
            outs[i].fill_(3.0)
            graphs[i].replay()
            got = bits(torch, outs[i])
            assert torch.equal(got, want[i])
            assert torch.equal(bits(torch, run(1 - i)), want[1 - i])


@pytest.mark.parametrize("act,held", PAIRS)
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (20, False), (0, False)])
def test_queries_in_place_beside_keys_and_values(torch, R, act, held, rot, interleaved):
    """q, k and v side by side in one buffer, q over itself; against the same call into memory of its own, row by row and all at once."""
    rng = np.random.default_rng(rot)
    hd, hkv, heads, lens = 64, 2, 6, [37, 64, 5]
    seq, slot = np.repeat(np.arange(3), lens), np.concatenate([np.arange(n) for n in lens])
    rope = R.rsd_rope(rot, interleaved=interleaved) if rot else None
    w, _ = dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, act))
    qkv, _ = dev(torch, rng.normal(size=(len(seq), heads + 2 * hkv, hd)), kind(torch, act))
    results = []
    for way in ("apart", "in place", "one by one"):
        c, _ = make_cache(torch, R, np.random.default_rng(1), lens, hkv, hd, held)
        x = qkv.clone()
        out = torch.empty_like(x[:, :heads]) if way != "in place" else x[:, :heads]
        kw = dict(rope=rope, q_weight=w, k_weight=w)
        pieces = [slice(i, i + 1) for i in rng.permutation(len(seq))] if way == "one by one" else [slice(None)]
        for r in pieces:
            s, t = ints(torch, seq[r]), ints(torch, slot[r])
            R.rsd_kv_append(c, x[r, heads:heads + hkv], x[r, heads + hkv:], s, t, position=t, q=x[r, :heads], q_out=out[r], **kw)
        results.append((bits(torch, out), bits(torch, c.pool)))
        assert torch.equal(bits(torch, x[:, heads:]), bits(torch, qkv[:, heads:]))
    for r in results[1:]:
        assert torch.equal(r[0], results[0][0]) and torch.equal(r[1], results[0][1])


@pytest.mark.parametrize("act,held", PAIRS)
def test_values_of_neighbours_that_are_no_neighbours(torch, R, act, held):
    """Runs of four that begin anywhere, break off, change sequence, go backwards, lie in missing pages or leave the cache."""
    rng = np.random.default_rng(17)
    hd, hkv = 32, 3
    c, table = make_cache(torch, R, rng, [48, 48, 48], hkv, hd, held)
    c.table[1, 1] = -1
    table[1, 1] = -1
    seq = [0] * 7 + [1] * 6 + [0, 1, 0, 1] + [2] * 4 + [2] * 4 + [1] * 4 + [5] * 4 + [2] * 3
    slot = [1, 2, 3, 4, 5, 6, 7] + [4, 5, 6, 8, 9, 10] + [12, 12, 13, 13] + [7, 6, 5, 4] + [44, 45, 46, 47] + [16, 17, 18, 19] + [0, 1, 2, 3] + [48, 49, (1 << 31) - 1]
    seq, slot = np.array(seq), np.array(slot, np.int64)
    k, k64 = dev(torch, rng.normal(size=(len(seq), hkv, hd)), kind(torch, act))
    v, v64 = dev(torch, rng.normal(size=(len(seq), hkv, hd)), kind(torch, act))
    want, size = host(c.pool), c.pool.element_size()
    to = lambda x: torch.from_numpy(x).to(kind(torch, held)).double().numpy()
    ref.fill(want, table, size, hd, seq, slot, to(k64), to(v64))
    R.rsd_kv_append(c, k, v, ints(torch, seq), ints(torch, slot))
    assert np.array_equal(host(c.pool), want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_keys_without_queries(torch, R, dtype):
    """The entry point takes keys alone, which the binding calls queries."""
    from paper_2501_19324_amd import ops
    rng = np.random.default_rng(3)
    rows, heads, hd = 37, 3, 64
    x, _ = dev(torch, rng.normal(size=(rows, heads, hd)), kind(torch, dtype))
    w, _ = dev(torch, 1 + 0.3 * rng.normal(size=hd), kind(torch, dtype))
    position, rope = ints(torch, rng.integers(0, 5000, rows)), R.rsd_rope(hd)
    want, _ = R.rsd_qk_rope(x, None, position, rope, q_weight=w)
    out = torch.empty_like(x)
    k = ops._Heads(x.data_ptr(), out.data_ptr(), w.data_ptr(), heads * hd, hd, heads * hd, hd, heads)
    turn = ops._Rope(rope.freq.data_ptr(), hd, 0, 1.0)
    assert ops._load().rsd_qk_rope(None, bytes(k), position.data_ptr(), bytes(turn), 1e-6, rows, hd, int(dtype == "bf16"), torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(bits(torch, out), bits(torch, want))

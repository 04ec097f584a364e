"""Calls of the attention over the paged bf16 / fp32 cache that run at the same time, and workspaces of exactly the size that they are said to need."""
import numpy as np
import pytest

from test_gpu_kv import PAIRS, R, bits, dev, ints, kind, make_cache, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# rows of each sequence, lengths: both are split into parts and joined
FORMS = [([1, 1, 1], [3000, 700, 2222]), ([9, 9, 9], [3000, 700, 2222])]


@pytest.mark.parametrize("rows,lens", FORMS, ids=["single tokens", "steps"])
@pytest.mark.parametrize("act,held", PAIRS)
def test_two_graphs_and_an_eager_call_at_once(torch, R, act, held, rows, lens):  # noqa: F811
    """Three caches, three streams, three workspaces: replays of two graphs and an eager call are issued without a wait between them; each result is what the call gives alone."""
    rng = np.random.default_rng(4)
    hd, hkv, heads = 128, 2, 8
    start, m = ints(torch, np.concatenate([[0], np.cumsum(rows)])), max(rows)
    caches = [make_cache(torch, R, rng, lens, hkv, hd, held)[0] for _ in range(3)]
    q = [dev(torch, rng.normal(size=(sum(rows), heads, hd)), kind(torch, act))[0] for _ in range(3)]

    def run(i):
        return R.rsd_kv_attention(caches[i], q[i], 0.1, row_start=start, max_rows=m, want_lse=True)

    alone = [[bits(torch, t) for t in run(i)] for i in range(3)]
    streams, graphs, outs = [torch.cuda.Stream() for _ in range(3)], [], []
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(i))
        graphs.append(g)
    for turn in range(4):
        for o in outs:
            for t in o:
                t.fill_(5.0)
        torch.cuda.synchronize()
        eager = []
        for order in (0, 1, 2, 2, 1, 0) if turn % 2 else (2, 0, 1, 1, 0, 2):
            with torch.cuda.stream(streams[order]):
                if order < 2:
                    graphs[order].replay()
                else:
                    eager.append(run(2))
        torch.cuda.synchronize()
        for got, want in [*zip(outs, alone), *((e, alone[2]) for e in eager)]:
            assert all(torch.equal(bits(torch, a), b) for a, b in zip(got, want))


@pytest.mark.parametrize("window", [0, 2000])
@pytest.mark.parametrize("rows,lens", [*FORMS, ([40, 3, 129], [2500, 300, 1400])], ids=["single tokens", "steps", "chunks"])
@pytest.mark.parametrize("act,held", PAIRS)
def test_workspaces_between_guards(torch, R, act, held, rows, lens, window):  # noqa: F811
    """The C entry point with a workspace of the size that it reports, between bytes that stay as they are; the result is the binding's."""
    import ctypes as C
    from paper_2501_19324_amd import ops
    rng = np.random.default_rng(7)
    hd, hkv, heads, total = 64, 2, 14, sum(rows)
    c, _ = make_cache(torch, R, rng, lens, hkv, hd, held)
    q, _ = dev(torch, rng.normal(size=(total, heads, hd)), kind(torch, act))
    start = ints(torch, np.concatenate([[0], np.cumsum(rows)]))
    want, want_lse = R.rsd_kv_attention(c, q, 0.1, row_start=start, max_rows=max(rows), window=window, sinks=20, want_lse=True)
    out, lse = torch.full_like(q, 9.0), torch.full((total, heads), 9.0, device="cuda")
    n, kv, batch = c.table.numel(), c.pool.shape[1], len(lens)
    cache = ops._KvCache(c.pool.data_ptr(), c.table.data_ptr(), c.kv_len.data_ptr(), c.pool.shape[0], kv, hd, batch, n // batch, 0 if held == "f32" else 1)
    a = ops._KvAttn(q.data_ptr(), out.data_ptr(), lse.data_ptr(), heads * hd, hd, heads * hd, hd, start.data_ptr(), total, max(rows), heads, n // batch * 16, window, 20, 0 if act == "f32" else 1, 0.1)
    lib = ops._load()
    need = lib.rsd_kv_attention_workspace(C.byref(cache), C.byref(a))
    assert need or window or (held == "f32" and max(rows) > 9)          # the others are split
    guard = 4096
    room = torch.randint(0, 256, (need + 2 * guard,), dtype=torch.uint8, device="cuda")
    before = room.cpu()
    assert room.data_ptr() % 256 == 0
    assert lib.rsd_kv_attention(C.byref(cache), C.byref(a), room.data_ptr() + guard, need, torch.cuda.current_stream().cuda_stream) == 0
    after = room.cpu()
    assert torch.equal(after[:guard], before[:guard]) and torch.equal(after[guard + need:], before[guard + need:])
    assert torch.equal(bits(torch, out), bits(torch, want)) and torch.equal(bits(torch, lse), bits(torch, want_lse))
    if need:
        assert lib.rsd_kv_attention(C.byref(cache), C.byref(a), room.data_ptr() + guard, need - 1, None) == -1 and b"workspace" in lib.rsd_op_last_error()

"""The operators' entry points without a GPU: exported symbols, structures, and the refusals that the host decides."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import q4_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2501_19324_amd import binding, ops
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ops._load()


def test_header_symbols_are_exported(lib):
    from paper_2501_19324_amd import binding, ops
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "rsd_ops.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(rsd_[a-z0-9_]+)\s*\(", text)))
    assert names == sorted(ops.OPS_EXPORTED_SYMBOLS)
    debug = C.CDLL(os.path.join(os.path.dirname(binding.LIB_PATH), "librsd_debug.so"))
    for n in names:
        assert hasattr(lib, n) and hasattr(debug, n), n


def test_structures_have_the_headers_sizes():
    from paper_2501_19324_amd import ops
    assert C.sizeof(ops._W4) == 24 and C.sizeof(ops._Cache) == 24 + 20 + 4
    assert C.sizeof(ops._Book) == 48 and C.sizeof(ops._Attn) == 24 + 32 + 8 + 20 + 4


def _cache(ops, **kw):
    c = dict(pool=4096, table=4096, kv_len=4096, n_pages=8, n_kv_heads=2, head_dim=64, batch=3, max_pages=4)
    c.update(kw)
    return ops._Cache(**c)


def _attn(ops, **kw):
    a = dict(q=4096, out=4096, lse=None, q_row=512, q_head=64, out_row=512, out_head=64, row_start=None, rows=3, max_rows=1, n_heads=8, max_kv=64, dtype=1, scale=0.1)
    a.update(kw)
    return ops._Attn(**a)


BAD_CACHE = [dict(pool=None), dict(table=None), dict(kv_len=None), dict(head_dim=48), dict(head_dim=256), dict(head_dim=0), dict(n_pages=0), dict(n_kv_heads=0),
             dict(batch=0), dict(max_pages=0), dict(max_pages=1 << 28), dict(pool=4096 + 8), dict(batch=1 << 20, n_kv_heads=2)]


@pytest.mark.parametrize("kw", BAD_CACHE, ids=str)
def test_bad_caches_are_refused(lib, kw):
    from paper_2501_19324_amd import ops
    c, a = _cache(ops, **kw), _attn(ops)
    book = ops._Book(4096, 4096, 128, 64, 128, 64)
    p = 4096
    assert lib.rsd_kv4_append(C.byref(c), p, 128, 64, p, 128, 64, 1, p, p, p, 3, C.byref(book), None) == -1
    assert lib.rsd_op_last_error().startswith(b"append")
    assert lib.rsd_kv4_read(C.byref(c), p, p, 3, p, p, 1, None) == -1
    assert lib.rsd_kv4_attention(C.byref(c), C.byref(a), None, p * 256, 1 << 30, None) == -1
    assert lib.rsd_kv4_evict(C.byref(c), C.byref(book), 8, 0, p * 256, 1 << 30, None) == -1
    assert lib.rsd_kv4_attention_workspace(C.byref(c), C.byref(a), 0) == 0 and lib.rsd_kv4_evict_workspace(C.byref(c), 8) == 0


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(dtype=2), dict(rows=0), dict(max_rows=0), dict(max_rows=2), dict(max_kv=-1), dict(n_heads=0),
                                dict(n_heads=7), dict(q=4097), dict(out=4097), dict(row_start=4096, max_rows=1 << 28)], ids=str)
def test_bad_attention_arguments_are_refused(lib, kw):
    from paper_2501_19324_amd import ops
    c, a = _cache(ops), _attn(ops, **kw)
    assert lib.rsd_kv4_attention(C.byref(c), C.byref(a), None, 1 << 20, 1 << 30, None) == -1
    assert lib.rsd_op_last_error().startswith(b"attention")
    assert lib.rsd_kv4_attention(C.byref(c), None, None, 1 << 20, 1 << 30, None) == -1


def test_small_or_unaligned_workspaces_are_refused(lib):
    from paper_2501_19324_amd import ops
    c, book = _cache(ops, batch=1, max_pages=512), ops._Book(4096, 4096, 1 << 14, 1 << 13, 1 << 14, 1 << 13)
    a = _attn(ops, rows=1, max_kv=8192)
    need = lib.rsd_kv4_attention_workspace(C.byref(c), C.byref(a), 1)
    assert need > 0
    for ws, n in ((1 << 20, need - 1), (None, need), ((1 << 20) + 16, need)):
        assert lib.rsd_kv4_attention(C.byref(c), C.byref(a), C.byref(book), ws, n, None) == -1
    need = lib.rsd_kv4_evict_workspace(C.byref(c), 100)
    for ws, n in ((1 << 20, need - 1), (None, need), ((1 << 20) + 16, need)):
        assert lib.rsd_kv4_evict(C.byref(c), C.byref(book), 100, 0, ws, n, None) == -1
    w = ops._W4(4096, 4096, 200, 5000)
    need = lib.rsd_w4_linear_workspace(300, 200, 5000, 0)
    assert need > 0
    for ws, n in ((1 << 20, need - 1), (None, need), ((1 << 20) + 16, need)):
        assert lib.rsd_w4_linear(C.byref(w), 4096, 5000, 4096, 200, 300, 0, ws, n, None) == -1


@pytest.mark.parametrize("budget,recent", [(0, 0), (-1, 0), (4, 5), (4, -1)])
def test_bad_budgets_are_refused(lib, budget, recent):
    from paper_2501_19324_amd import ops
    c, book = _cache(ops), ops._Book(4096, 4096, 128, 64, 128, 64)
    assert lib.rsd_kv4_evict(C.byref(c), C.byref(book), budget, recent, 1 << 20, 1 << 30, None) == -1
    assert lib.rsd_kv4_evict(C.byref(c), C.byref(ops._Book(4096, None, 128, 64, 0, 0)), 4, 0, 1 << 20, 1 << 30, None) == -1
    assert lib.rsd_kv4_evict(C.byref(c), None, 4, 0, 1 << 20, 1 << 30, None) == -1


def test_bad_weights_and_rows_are_refused(lib):
    from paper_2501_19324_amd import ops
    p, ws = 4096, 1 << 20
    for w, x, ldx, y, ldy, rows, t in [((None, p, 16, 32), p, 32, p, 16, 1, 0), ((p, None, 16, 32), p, 32, p, 16, 1, 0), ((p, p, 0, 32), p, 32, p, 16, 1, 0),
                                       ((p, p, 16, 0), p, 32, p, 16, 1, 0), ((p, p, 16, 32), None, 32, p, 16, 1, 0), ((p, p, 16, 32), p, 31, p, 16, 1, 0),
                                       ((p, p, 16, 32), p, 32, p, 15, 1, 0), ((p, p, 16, 32), p, 32, p, 16, 0, 0), ((p, p, 16, 32), p, 32, p, 16, 1, 3),
                                       ((p + 8, p, 16, 32), p, 32, p, 16, 1, 0), ((p, p + 4, 16, 32), p, 32, p, 16, 1, 0), ((p, p, 16, 32), p + 2, 32, p, 16, 1, 0),
                                       ((p, p, 16, 32), p, 32, p + 1, 16, 1, 1), ((p, p, 16, 32), p, 32, p, 16, 1 << 21, 1)]:
        assert lib.rsd_w4_linear(C.byref(ops._W4(*w)), x, ldx, y, ldy, rows, t, ws, 1 << 40, None) == -1, (w, rows, t)
        assert lib.rsd_op_last_error().startswith(b"w4_linear")
    for args in [(None, 0, 32, 16, 32, p, p), (p, 0, 32, 16, 32, None, p), (p, 0, 32, 16, 32, p, None), (p, 2, 32, 16, 32, p, p), (p, 0, 31, 16, 32, p, p),
                 (p, 0, 32, 0, 32, p, p), (p, 0, 32, 16, 0, p, p)]:
        assert lib.rsd_w4_pack(*args, None) == -1, args
    c = _cache(ops)
    for args in [(None, p, 1, p, p, p, 3), (p, None, 1, p, p, p, 3), (p, p, 2, p, p, p, 3), (p, p, 1, None, p, p, 3), (p, p, 1, p, None, p, 3), (p, p, 1, p, p, None, 3),
                 (p, p, 1, p, p, p, 0), (p + 1, p, 1, p, p, p, 3)]:
        k, v, t, seq, slot, pos, rows = args
        assert lib.rsd_kv4_append(C.byref(c), k, 128, 64, v, 128, 64, t, seq, slot, pos, rows, C.byref(ops._Book(p, p, 128, 64, 128, 64)), None) == -1, args
    assert lib.rsd_kv4_read(C.byref(c), p, p, 0, p, p, 1, None) == -1 and lib.rsd_kv4_read(C.byref(c), p, p, 3, p, p + 8, 1, None) == -1


def test_reference_grid_and_round_trip():
    """The definitions the GPU tests compare with: nearest values, scale choice, layouts without overlap."""
    x = np.zeros(32)
    x[:9] = [7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.0]
    code, byte, val = ref.quantize(x)
    assert byte[0] == 127 and list(code[:9]) == [7, 0, 2, 2, 4, 4, 6, 6, 8] and list(val[:8]) == [6, 0, 1, 1, 2, 2, 4, 4]
    x[0] = np.nextafter(7.0, 8)
    assert ref.quantize(x)[1][0] == 128
    x[0] = 2.0 ** 127 * 1.9
    assert ref.quantize(x)[1][0] == 252 and ref.quantize(np.full(32, 1e-40))[1][0] == 2
    rng = np.random.default_rng(0)
    y = rng.normal(size=(64,)) * np.exp(rng.normal(size=64))
    _, byte, val = ref.quantize(y)
    step = np.repeat(np.ldexp(1.0, byte.astype(int) - 127), 32)
    assert np.all(np.abs(y - val) <= step * np.where(np.abs(y) > 4 * step, 1.0, np.where(np.abs(y) > 2 * step, 0.5, 0.25)))
    for hd in (32, 64, 128):
        used = np.concatenate([np.concatenate([p.reshape(-1) for p in ref.entry_places(hd, t)]) for t in range(16)])
        assert sorted(used) == list(range(17 * hd))
        block = rng.integers(0, 256, 17 * hd).astype(np.uint8)
        k, v = rng.normal(size=hd), rng.normal(size=hd)
        ref.write_entry(block, hd, 5, k, v)
        a, b = ref.read_entry(block, hd, 5)
        assert np.array_equal(a, ref.quantize(k)[2]) and np.array_equal(b, ref.quantize(v)[2])

"""The entry points of the paged bf16 / fp32 cache and of the rotation without a GPU: structures, frequencies, and the refusals that the host decides."""
import ctypes as C
import os

import numpy as np
import pytest

import kv_reference as ref


@pytest.fixture(scope="module")
def lib():
    from paper_2501_19324_amd import binding, ops
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ops._load()


@pytest.fixture(scope="module")
def ops():
    from paper_2501_19324_amd import ops
    return ops


def test_structures_have_the_headers_sizes(ops):
    assert C.sizeof(ops._KvCache) == 24 + 24 and C.sizeof(ops._KvAttn) == 24 + 32 + 8 + 32
    assert C.sizeof(ops._Heads) == 24 + 32 + 8 and C.sizeof(ops._Rope) == 24
    # the bytes that the binding packs are those of the structures
    for kind, pack, values in ((ops._KvCache, ops._KV_CACHE_BYTES, (16, 17, 18, 1, 2, 3, 4, 5, 1)), (ops._Rope, ops._ROPE_BYTES, (16, 64, 1, 1.25, 0)),
                               (ops._Heads, ops._HEADS_BYTES, (16, 17, 18, -5, 6, 1 << 40, 8, 9, 0)),
                               (ops._KvAttn, ops._KV_ATTN_BYTES, (16, 17, 18, -1, 2, 3, 1 << 40, 19, 4, 5, 6, 7, 8, 9, 1, -0.5))):
        made = kind(*values[:len(kind._fields_)])
        assert bytes(made)[:sum(C.sizeof(f) for _, f in kind._fields_)] == pack(*values)[:sum(C.sizeof(f) for _, f in kind._fields_)] and C.sizeof(kind) == len(pack(*values))


def cache(ops, **kw):
    c = dict(pool=1 << 30, table=4096, kv_len=8192, n_pages=8, n_kv_heads=2, head_dim=64, batch=3, max_pages=4, dtype=1)
    c.update(kw)
    return ops._KvCache(**c)


def attn(ops, **kw):
    a = dict(q=1 << 20, out=1 << 21, lse=None, q_row=512, q_head=64, out_row=512, out_head=64, row_start=None, rows=3, max_rows=1, n_heads=8, max_kv=64, window=0, sinks=0,
             dtype=1, scale=0.1)
    a.update(kw)
    return ops._KvAttn(**a)


def heads(ops, **kw):
    h = dict(x=1 << 20, out=1 << 21, weight=None, row=512, head=64, out_row=512, out_head=64, n_heads=8)
    h.update(kw)
    return ops._Heads(**h)


WS = 1 << 28


@pytest.mark.parametrize("kw", [dict(pool=None), dict(table=None), dict(kv_len=None), dict(head_dim=48), dict(head_dim=256), dict(head_dim=0), dict(n_pages=0), dict(n_kv_heads=0),
                                dict(batch=0), dict(max_pages=0), dict(max_pages=1 << 28), dict(pool=4096 + 8), dict(batch=1 << 20, n_kv_heads=2), dict(dtype=2), dict(dtype=-1)],
                         ids=str)
def test_bad_caches_are_refused(lib, ops, kw):
    c, k = cache(ops, **kw), heads(ops, n_heads=2, out=None)
    p = 4096
    assert lib.rsd_kv_append(C.byref(c), C.byref(k), 1 << 22, 128, 64, None, p, p, None, None, 1e-6, 3, 1, None) == -1
    assert lib.rsd_op_last_error().startswith(b"append")
    assert lib.rsd_kv_read(C.byref(c), p, p, 3, p, p, None) == -1
    assert lib.rsd_kv_attention(C.byref(c), C.byref(attn(ops)), WS, 1 << 30, None) == -1
    assert lib.rsd_kv_attention_workspace(C.byref(c), C.byref(attn(ops))) == 0
    assert lib.rsd_kv_attention(None, C.byref(attn(ops)), WS, 1 << 30, None) == -1


@pytest.mark.parametrize("kw", [dict(q=None), dict(out=None), dict(dtype=2), dict(rows=0), dict(max_rows=0), dict(max_rows=2), dict(max_kv=-1), dict(n_heads=0), dict(n_heads=7),
                                dict(q=4097), dict(out=4097), dict(row_start=4096, max_rows=1 << 28), dict(window=-1), dict(sinks=-1), dict(out_row=500), dict(out_head=63),
                                dict(out=(1 << 20) + 128), dict(out=1 << 20, out_row=1024), dict(out_row=0)], ids=str)
def test_bad_attention_arguments_are_refused(lib, ops, kw):
    c = cache(ops)
    assert lib.rsd_kv_attention(C.byref(c), C.byref(attn(ops, **kw)), WS, 1 << 30, None) == -1
    assert lib.rsd_op_last_error().startswith(b"attention")
    assert lib.rsd_kv_attention(C.byref(c), None, WS, 1 << 30, None) == -1


def test_types_that_do_not_go_together_are_refused(lib, ops):
    c = cache(ops, dtype=0)
    assert lib.rsd_kv_attention(C.byref(c), C.byref(attn(ops, dtype=1)), WS, 1 << 30, None) == -1
    k = heads(ops, n_heads=2, out=None)
    assert lib.rsd_kv_append(C.byref(c), C.byref(k), 1 << 22, 128, 64, None, 4096, 4096, None, None, 1e-6, 3, 1, None) == -1


def test_small_or_unaligned_workspaces_are_refused(lib, ops):
    c, a = cache(ops, batch=1, max_pages=512), attn(ops, rows=1, max_kv=8192)
    need = lib.rsd_kv_attention_workspace(C.byref(c), C.byref(a))
    assert need > 0
    for ws, n in ((WS, need - 1), (None, need), (WS + 16, need)):
        assert lib.rsd_kv_attention(C.byref(c), C.byref(a), ws, n, None) == -1


ROPE = dict(freq=4096, rot_dim=64, interleaved=0, magnitude=1.0)


@pytest.mark.parametrize("change", [dict(q=dict(x=None)), dict(q=dict(out=None)), dict(q=dict(n_heads=0)), dict(q=dict(x=(1 << 20) + 1)), dict(q=dict(out=(1 << 21) + 1)),
                                    dict(q=dict(weight=4097)), dict(q=dict(out_head=63)), dict(q=dict(out_row=511)), dict(q=dict(out=(1 << 20) + 64)),
                                    dict(q=dict(out=1 << 20, out_row=1024)), dict(k=dict(x=(1 << 21) + 512)), dict(k=dict(out=1 << 20)), dict(k=dict(out=1 << 21)), dict(hd=48),
                                    dict(hd=512), dict(rows=0), dict(rows=1 << 24), dict(dtype=3), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                                    dict(rope=dict(rot_dim=0)), dict(rope=dict(rot_dim=66)), dict(rope=dict(rot_dim=33)), dict(rope=dict(freq=None)), dict(rope=dict(freq=4100)),
                                    dict(position=None), dict(position=(1 << 21) + 64), dict(q=dict(weight=(1 << 21) + 64)), dict(rope=dict(freq=(1 << 21) + 64)), dict(none=True)], ids=str)
def test_bad_heads_and_rotations_are_refused(lib, ops, change):
    q = heads(ops, **change.get("q", {}))
    k = heads(ops, **{**dict(x=1 << 22, out=1 << 23, n_heads=2, row=128, out_row=128), **change.get("k", {})})
    r = ops._Rope(**{**ROPE, **change.get("rope", {})})
    args = (change.get("position", 8192), C.byref(r), change.get("eps", 1e-6), change.get("rows", 3), change.get("hd", 64), change.get("dtype", 1), None)
    both = (None, None) if change.get("none") else (C.byref(q), C.byref(k))
    assert lib.rsd_qk_rope(*both, *args) == -1
    assert lib.rsd_op_last_error().startswith(b"qk_rope")


@pytest.mark.parametrize("change", [dict(k=dict(x=None)), dict(k=dict(n_heads=3)), dict(v=None), dict(v=4097), dict(seq=None), dict(slot=None), dict(rows=0), dict(dtype=2),
                                    dict(rope=dict(rot_dim=66)), dict(position=None), dict(q=dict(out=1 << 22)), dict(q=dict(out=1 << 23)), dict(q=dict(out=(1 << 30) + 4096)), dict(q=dict(out=4096)),
                                    dict(q=dict(out=8192 * 2)), dict(eps=-0.5)], ids=str)
def test_bad_entries_are_refused(lib, ops, change):
    c = cache(ops)
    q = heads(ops, **change.get("q", {}))
    k = heads(ops, **{**dict(x=1 << 22, out=None, n_heads=2, row=128), **change.get("k", {})})
    r = ops._Rope(**{**ROPE, "freq": 4096 * 7, **change.get("rope", {})})
    rc = lib.rsd_kv_append(C.byref(c), C.byref(k), change.get("v", 1 << 23), 128, 64, C.byref(q), change.get("seq", 16384), change.get("slot", 16640), change.get("position", 16896),
                           C.byref(r), change.get("eps", 1e-6), change.get("rows", 3), change.get("dtype", 1), None)
    assert rc == -1 and lib.rsd_op_last_error().startswith(b"append")


def test_heads_side_by_side_in_a_buffer_do_not_meet(lib, ops):
    """What the host says of views of one buffer is what an enumeration of their elements says (calls that pass the check reach the launch, so only refusals are looked at: an
    invalid rotation behind the check of the heads tells the two apart)."""
    rng = np.random.default_rng(1)
    base, hd, size = 1 << 24, 32, 4
    refused = 0
    for _ in range(400):
        rows, nq, nk = int(rng.integers(1, 4)), int(rng.integers(1, 4)), int(rng.integers(1, 3))
        row = int(rng.choice([hd * (nq + nk), hd * (2 * nq + nk), hd * (nq + nk) + 7]))
        off_k = int(rng.integers(0, 2 * row))
        # q in place, k read only, into a cache far away
        e = lambda off, n: {off + i * row + h * hd + d for i in range(rows) for h in range(n) for d in range(hd)}  # noqa: E731
        q = heads(ops, x=base, out=base, row=row, head=hd, out_row=row, out_head=hd, n_heads=nq)
        k = heads(ops, x=base + off_k * size, out=None, row=row, head=hd, n_heads=nk)
        c = cache(ops, head_dim=hd, n_kv_heads=nk, dtype=0)
        r = ops._Rope(4096 * 7, 32, 0, 1.0)
        rc = lib.rsd_kv_append(C.byref(c), C.byref(k), 1 << 26, hd * nk, hd, C.byref(q), 16384, 16640, base + 4 if not e(0, nq) & e(off_k, nk) else 16896, C.byref(r), 1e-6, rows, 0, None)
        text = lib.rsd_op_last_error()
        assert rc == -1
        if e(0, nq) & e(off_k, nk):
            refused += 1
            assert b"shares memory with k" in text
        elif rows == 1 or off_k % row + hd * nk <= row:     # inside the rows of the buffer
            assert b"shares memory with weights" in text
    assert refused > 50


@pytest.mark.parametrize("args", [(1e4, 0, 0, 1, 0, 1, 32), (1e4, 5, 0, 1, 0, 1, 32), (0.0, 8, 0, 1, 0, 1, 32), (float("nan"), 8, 0, 1, 0, 1, 32), (1e4, 8, 4, 1, 0, 1, 32), (1e4, 8, -1, 1, 0, 1, 32),
                                  (1e4, 8, 1, 0.0, 0, 1, 32), (1e4, 2, 2, 4.0, 0, 1, 32), (1e4, 8, 3, 4.0, 0.0, 1, 32), (1e4, 8, 3, 4.0, 8192, 2, 2), (1e4, 8, 3, float("inf"), 8192, 1, 32)])
def test_bad_frequencies_are_refused(lib, args):
    assert lib.rsd_rope_frequencies(*args, (C.c_double * 8)()) == -1
    assert lib.rsd_op_last_error().startswith(b"rope_frequencies")
    assert lib.rsd_rope_frequencies(1e4, 8, 0, 1, 0, 1, 32, None) == -1


def test_frequencies(lib):
    for rot, code, name, kw in ((8, 0, "plain", {}), (128, 1, "linear", dict(factor=4.0)), (64, 2, "base", dict(factor=8.0)), (128, 3, "parts", dict(factor=16.0, original=8192.0, low=1.0, high=32.0))):
        f = (C.c_double * (rot // 2))()
        a = dict(factor=1.0, original=0.0, low=1.0, high=32.0)
        a.update(kw)
        assert lib.rsd_rope_frequencies(1e6, rot, code, a["factor"], a["original"], a["low"], a["high"], f) == 0
        assert np.allclose(list(f), ref.frequencies(1e6, rot, name, **kw), rtol=1e-14, atol=0)


def test_places_cover_a_page():
    for size in (2, 4):
        for hd in (32, 64, 128):
            for places in (ref.key_places, ref.value_places):
                assert sorted(np.concatenate([places(size, hd, t) for t in range(16)])) == list(range(16 * hd))


def test_binding_refuses_what_it_can_see(ops):
    import torch
    from paper_2501_19324_amd.binding import RsdError
    c = ops.rsd_kv_cache(2, 3, 8, 2, 64, device="cpu")
    assert c.pool.shape == (8, 2, 2, 1024) and c.pool.dtype is torch.bfloat16 and (c.table == -1).all() and not c.kv_len.any()
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: ops.rsd_kv_attention(c, x, 1.0), lambda: ops.rsd_kv_append(c, x, x, i, i), lambda: ops.rsd_kv_read(c, i, i), lambda: ops.rsd_qk_rope(x, None, i)):
        with pytest.raises(RsdError, match="current device"):
            call()
    for bad in (dict(scaling="other"), dict(factor=0.0, scaling="linear"), dict(theta=-1.0)):
        with pytest.raises(RsdError):
            ops.rsd_rope(64, device="cpu", **bad)
    for rot in (0, 3, 258, 1.5):
        with pytest.raises(RsdError):
            ops.rsd_rope(rot, device="cpu")
    r = ops.rsd_rope(64, 1e4, scaling="parts", factor=4.0, original=64, device="cpu")
    assert r.freq.shape == (32,) and abs(r.magnitude - (0.1 * np.log(4.0) + 1)) < 1e-12


def test_arrays_that_share_memory_are_refused(lib, ops):
    big = dict(batch=1, max_pages=512, pool=1 << 30)
    c, a = cache(ops, **big), dict(rows=1, max_kv=8192)
    need = lib.rsd_kv_attention_workspace(C.byref(c), C.byref(attn(ops, **a)))
    line = 8 * 64 * 2                                       # bytes of q, and of out
    for kw, ws in ((dict(out=(1 << 30) + 2), WS), (dict(lse=(1 << 30) + 4), WS), (dict(lse=(1 << 21) + line - 4), WS), (dict(lse=(1 << 20) - 28), WS), (dict(out=4096), WS), (dict(lse=8192 - 28), WS),
                   (dict(row_start=(1 << 21) - 4), WS), (dict(lse=(1 << 21) + 4096, row_start=(1 << 21) + 4096 + 28), WS), (dict(out=WS + need - 2), WS), (dict(q=WS + need - 2), WS), (dict(lse=WS), WS),
                   (dict(), (1 << 30) - 256), (dict(), (1 << 21) - 256), (dict(lse=1 << 22 | 2), WS)):
        assert lib.rsd_kv_attention(C.byref(c), C.byref(attn(ops, **a, **kw)), ws, 1 << 30, None) == -1, (kw, ws)
        assert b"share" in lib.rsd_op_last_error() or b"aligned" in lib.rsd_op_last_error(), lib.rsd_op_last_error()
    rows = 3 * 2 * 64 * 2                                   # bytes of k, and of v
    for k, v, seq in ((1 << 20, (1 << 20) + rows - 16, 1 << 16), ((1 << 30) + 16, 1 << 20, 1 << 16), (1 << 20, 4096, 1 << 16), (1 << 20, 1 << 21, (1 << 20) + rows - 4)):
        assert lib.rsd_kv_read(C.byref(c), seq, 1 << 17, 3, k, v, None) == -1 and b"shares" in lib.rsd_op_last_error()
    k, q = heads(ops, n_heads=2, out=None), heads(ops, x=1 << 23, out=1 << 30)
    assert lib.rsd_kv_append(C.byref(c), C.byref(k), 1 << 22, 128, 64, C.byref(q), 1 << 16, 1 << 17, None, None, 1e-6, 3, 1, None) == -1 and b"cache" in lib.rsd_op_last_error()


@pytest.mark.parametrize("rows,batch,kv,heads_", [(1, 1, 1279, 12), (64, 64, 5120, 28), (2048, 1, 8192, 28), (1, 1, 1, 1), (130, 3, 4096, 16), (7, 2, 1 << 20, 64), (512, 512, 70, 8)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1000, 4), (5, 1 << 20)])
def test_workspaces_hold_the_parts(lib, ops, rows, batch, kv, heads_, window, sinks):
    """A part of a row's head is head_dim sums and two numbers, and there are no more parts than the entries have chunks."""
    for hd in (32, 64, 128):
        for held, act in ((1, 1), (1, 0), (0, 0)):
            c = cache(ops, batch=batch, max_pages=-(-kv // 16), n_kv_heads=1, head_dim=hd, dtype=held)
            a = attn(ops, rows=rows, max_rows=max(rows // batch, 1), row_start=1 << 16, n_heads=heads_, max_kv=kv, window=window, sinks=sinks, dtype=act)
            need = lib.rsd_kv_attention_workspace(C.byref(c), C.byref(a))
            most = -(-kv // 16) * rows * heads_ * (4 * hd + 8) + 512
            assert need % 256 == 0 and need <= most and (need == 0 or need >= 2 * rows * heads_ * (4 * hd + 8))

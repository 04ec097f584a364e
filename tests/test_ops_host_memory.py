"""Which memory the operators may be given, as far as the host decides it: strides that overlap, memory that outputs share, sizes beyond 32 bits.  No call
here reaches a launch."""
import ctypes as C
import os

import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2501_19324_amd import binding, ops
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return ops._load()


@pytest.fixture
def on_host(lib, monkeypatch):
    """The binding on tensors in host memory: for calls that are refused."""
    from paper_2501_19324_amd import ops
    monkeypatch.setattr(ops, "_stream", lambda t: 0)
    return ops


def refused(call, ops):
    with pytest.raises(ops._b.RsdError) as e:
        call()
    return e.value.code == ops._b.RSD_EINVAL


@pytest.mark.parametrize("shape,strides", [((48, 64), (0, 1)), ((48, 64), (1, 1)), ((2, 64), (63, 1)), ((5, 1), (0, 1))], ids=str)
def test_weights_whose_rows_overlap_are_refused(on_host, shape, strides):
    """A row stride below the row's length was once taken for that length: a read behind the tensor's memory."""
    import torch
    w = torch.zeros(4096).as_strided(shape, strides)
    assert refused(lambda: on_host.rsd_w4_pack(w), on_host)


def _cache(ops, batch=3, n_kv_heads=2, max_pages=4):
    return ops._Cache(4096, 4096, 4096, 8, n_kv_heads, 64, batch, max_pages)


def _attn(ops, **kw):
    a = dict(q=1 << 20, out=1 << 24, lse=None, q_row=512, q_head=64, out_row=512, out_head=64, row_start=4096, rows=3, max_rows=2, n_heads=8, max_kv=64, dtype=1, scale=0.1)
    a.update(kw)
    return ops._Attn(**a)


def _no_workspace(lib, call):
    """What a call without room for its workspace says: the last refusal before a launch."""
    assert call() == -1
    return b"workspace" in lib.rsd_op_last_error()


# rows, heads, strides of both in elements, pieces of 64
STRIDES = [(3, 8, 512, 64), (3, 8, 64, 192), (3, 8, 1000, 70), (1, 8, 0, 64), (3, 1, 64, 0), (1, 1, 0, 0), (3, 8, -512, 64), (2, 2, 192, 128), (3, 2, 128, 192), (4, 3, 150, 230),
           (3, 8, 0, 64), (3, 8, 512, 0), (3, 8, 511, 64), (3, 8, 512, 63), (3, 8, 64, 64), (3, 8, 64, 128), (3, 8, 128, 192), (2, 8, 400, 100), (3, 1, 63, 0), (1, 2, 0, -63),
           (8, 3, 64, 500)]


def _share(rows, heads, row, head, length):
    taken = set()
    for r in range(rows):
        for h in range(heads):
            piece = set(range(r * row + h * head, r * row + h * head + length))
            if taken & piece:
                return True
            taken |= piece
    return False


@pytest.mark.parametrize("rows,heads,row,head", STRIDES)
def test_outputs_whose_rows_overlap_are_refused(lib, rows, heads, row, head):
    """Blocks would write to one place in any order."""
    from paper_2501_19324_amd import ops
    # (accepted: as far as the workspace, which is not there)
    c = _cache(ops, batch=1, n_kv_heads=1, max_pages=512)
    a = _attn(ops, rows=rows, n_heads=heads, out_row=row, out_head=head, max_kv=8192, max_rows=rows)
    good = _no_workspace(lib, lambda: lib.rsd_kv4_attention(C.byref(c), C.byref(a), None, None, 0, None))
    assert good != _share(rows, heads, row, head, 64), lib.rsd_op_last_error()


@pytest.mark.parametrize("batch,heads,b,h", STRIDES)
def test_lists_that_overlap_are_refused(lib, batch, heads, b, h):
    from paper_2501_19324_amd import ops
    c, fine = _cache(ops, batch, heads, 4), (heads * 64, 64)
    ok = not _share(batch, heads, b, h, 64)
    for scores, positions in (((b, h), fine), (fine, (b, h))):
        book = ops._Book(1 << 20, 1 << 24, *scores, *positions)
        assert _no_workspace(lib, lambda: lib.rsd_kv4_evict(C.byref(c), C.byref(book), 5, 0, None, 0, None)) == ok
    # attention: scores alone; positions are not looked at
    c = _cache(ops, batch, heads, 4)
    a = _attn(ops, rows=batch, n_heads=17 * heads, out_row=17 * heads * 64, max_kv=64, max_rows=batch)
    book = ops._Book(1 << 20, None, b, h, 0, 0)
    assert _no_workspace(lib, lambda: lib.rsd_kv4_attention(C.byref(c), C.byref(a), C.byref(book), None, 0, None)) == ok


def test_expanded_outputs_are_refused_by_the_binding(on_host):
    import torch
    ops = on_host
    cache = ops.Kv4Cache(torch.zeros(8, 2, 17 * 64, dtype=torch.uint8), torch.zeros(3, 4, dtype=torch.int32), torch.zeros(3, dtype=torch.int32))
    q = torch.zeros(3, 4, 64)
    lists, pos = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64, dtype=torch.int32)
    for out in (q[:1].clone().expand(3, 4, 64), q[:, :1].clone().expand(3, 4, 64)):
        assert refused(lambda: ops.rsd_kv4_attention(cache, q, 1.0, out=out), ops)
    for bad in (lists[:1].expand(3, 2, 64), lists[:, :1].expand(3, 2, 64)):
        assert refused(lambda: ops.rsd_kv4_attention(cache, q, 1.0, scores=bad), ops)
        assert refused(lambda: ops.rsd_kv4_evict(cache, bad, pos, 8), ops)
    for bad in (pos[:1].expand(3, 2, 64), pos[:, :1].expand(3, 2, 64)):
        assert refused(lambda: ops.rsd_kv4_evict(cache, lists, bad, 8), ops)


# out's start behind q's, strides of q, strides of out (rows, heads), rows, heads; pieces of 64
PAIRS = [(0, (512, 64), (512, 64), 3, 8), (1024, (2048, 64), (2048, 64), 3, 8), (64, (1024, 128), (1024, 128), 3, 8), (63, (1024, 128), (1024, 128), 3, 8),
         (65, (1024, 128), (1024, 128), 3, 8), (-64, (1024, 128), (1024, 128), 3, 8), (1536, (512, 64), (512, 64), 3, 8), (1535, (512, 64), (512, 64), 3, 8),
         (-1536, (512, 64), (512, 64), 3, 8), (-1473, (512, 64), (512, 64), 3, 8), (512, (1024, 64), (1024, 64), 3, 8), (448, (1024, 64), (1024, 64), 3, 8),
         (0, (512, 64), (64, 192), 3, 8), (1024, (2048, 64), (2048, 128), 2, 8), (1024, (2048, 64), (2048, 120), 2, 9), (960, (2048, 64), (2048, 128), 2, 8),
         (0, (0, 64), (512, 64), 3, 8), (1536, (0, 64), (512, 64), 3, 8), (64, (0, 64), (0, 128), 1, 1), (63, (7, 9), (0, 128), 1, 1), (2, (64, 192), (64, 192), 3, 2),
         (2048, (1024, -64), (1024, 64), 2, 8), (192, (64, 300), (64, 300), 3, 2), (130, (64, 300), (64, 300), 3, 2), (172, (64, 300), (64, 300), 2, 2),
         (448, (1024, 64), (1024, 64), 3, 7), (-448, (1024, 64), (1024, 64), 3, 7), (1500, (1024, 64), (1024, 64), 4, 7), (1536, (1024, 64), (1024, 70), 4, 8),
         (576, (1024, 64), (1024, 64), 4, 8), (512, (1024, 64), (1024, 73), 4, 8), (1984, (1024, 64), (1024, 0), 3, 9), (1023, (512, 64), (512, 64), 4, 8)]


@pytest.mark.parametrize("d,q,out,rows,heads", PAIRS)
@pytest.mark.parametrize("scored", [False, True])
def test_out_that_shares_memory_with_q_is_refused(lib, d, q, out, rows, heads, scored):
    """Elsewhere a block would read what another has written.  q itself is read before it is written, except where the weights need it again."""
    from paper_2501_19324_amd import ops
    at = 1 << 24

    def elements(first, strides):
        return {first + r * strides[0] + h * strides[1] + i for r in range(rows) for h in range(heads) for i in range(64)}

    shared = elements(0, q) & elements(d, out)
    if (d, q) == (0, out):
        shared = shared if scored else set()               # (in parts: the weights are added by a kernel of their own)
    c = _cache(ops, batch=1, n_kv_heads=1, max_pages=512)
    a = _attn(ops, q=at, out=at + 2 * d, q_row=q[0], q_head=q[1], out_row=out[0], out_head=out[1], rows=rows, n_heads=heads, max_kv=8192, max_rows=rows)
    book = ops._Book(1 << 30, None, 8192, 8192, 0, 0)
    good = _no_workspace(lib, lambda: lib.rsd_kv4_attention(C.byref(c), C.byref(a), C.byref(book) if scored else None, None, 0, None))
    assert good == (not shared) or _share(rows, heads, *out, 64), lib.rsd_op_last_error()


# y's start behind x's, n, distance of the rows of y and of x; 20 rows of 1024 (long enough for a workspace)
PRODUCTS = [(0, 1024, 1024, 1024), (1024, 1024, 2048, 2048), (1023, 1024, 2048, 2048), (-1024, 1024, 2048, 2048), (-1023, 1024, 2048, 2048), (20480, 16, 16, 1024),
            (20479, 16, 16, 1024), (-320, 16, 16, 1024), (-319, 16, 16, 1024), (1024, 10, 1034, 1034), (1025, 10, 1034, 1034), (-10, 10, 1034, 1034), (2000, 20, 1044, 1044)]


@pytest.mark.parametrize("d,n,ldy,ldx", PRODUCTS)
@pytest.mark.parametrize("dtype,size", [(0, 4), (1, 2)])
def test_products_into_memory_of_x_are_refused(lib, d, n, ldy, ldx, dtype, size):
    """Every block reads all of x while others write."""
    from paper_2501_19324_amd import ops
    w, at, rows, k = ops._W4(4096, 4096, n, 1024), 1 << 24, 20, 1024
    shared = {r * ldx + i for r in range(rows) for i in range(k)} & {d + r * ldy + i for r in range(rows) for i in range(n)}
    good = _no_workspace(lib, lambda: lib.rsd_w4_linear(C.byref(w), at, ldx, at + size * d, ldy, rows, dtype, None, 0, None))
    assert good == (not shared), lib.rsd_op_last_error()


def test_products_into_their_activations_are_refused_by_the_binding(on_host):
    import torch
    ops = on_host
    w = ops.W4(torch.zeros(2, 1, 4, 16, 16, dtype=torch.uint8), torch.zeros(2, 1, 4, 16, 4, dtype=torch.uint8), 32, 32)
    x = torch.zeros(6, 32)
    assert refused(lambda: ops.rsd_w4_linear(x, w, out=x), ops)
    assert refused(lambda: ops.rsd_w4_linear(x[1:], w, out=x[:-1]), ops)


# ---- sizes beyond 32 bits: ctypes takes them modulo 2^32

def small_cache(ops, batch=3, pages=4):
    import torch
    return ops.Kv4Cache(torch.zeros(8, 2, 17 * 64, dtype=torch.uint8), torch.zeros(batch, pages, dtype=torch.int32), torch.zeros(batch, dtype=torch.int32))


@pytest.mark.parametrize("big", [(1 << 32) + 2, 1 << 31, -(1 << 32) + 2, 2.0, 2.5, None], ids=str)
def test_sizes_beyond_32_bits_are_refused(on_host, big):
    import torch
    ops = on_host
    cache, q = small_cache(ops), torch.zeros(3, 4, 64)
    lists, pos, starts = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    assert refused(lambda: ops.rsd_kv4_evict(cache, lists, pos, big), ops)
    assert refused(lambda: ops.rsd_kv4_evict(cache, lists, pos, 60, big), ops)
    if big is not None:
        assert refused(lambda: ops.rsd_kv4_attention(cache, q, 1.0, row_start=starts, max_rows=big), ops)
    if isinstance(big, int) and big < 0:
        assert refused(lambda: ops.rsd_kv4_attention(cache, q, 1.0, max_kv=big), ops)


def test_whole_numbers_of_other_types_are_taken(on_host):
    """A budget that holds every entry of the table leaves nothing to launch."""
    import numpy as np
    import torch
    ops = on_host
    lists, pos = torch.zeros(3, 2, 64), torch.zeros(3, 2, 64, dtype=torch.int32)
    for budget, recent in ((64, 0), (np.int64(64), np.int32(3)), (torch.tensor(64), torch.tensor(3)), ((1 << 31) - 1, 5)):
        ops.rsd_kv4_evict(small_cache(ops), lists, pos, budget, recent)


@pytest.mark.parametrize("budget", [64, 65, 10 ** 6, (1 << 31) - 1])
def test_a_budget_beyond_the_table_needs_no_workspace(lib, budget):
    """It once grew with the budget: 1 GB for a million on 256 lists, for a call that has nothing to do."""
    from paper_2501_19324_amd import ops
    c, book = _cache(ops, batch=64, n_kv_heads=4, max_pages=4), ops._Book(1 << 20, 1 << 24, 256, 64, 256, 64)
    assert lib.rsd_kv4_evict_workspace(C.byref(c), budget) == 0
    assert lib.rsd_kv4_evict(C.byref(c), C.byref(book), budget, 0, None, 0, None) == 0
    most = max(lib.rsd_kv4_evict_workspace(C.byref(c), b) for b in range(1, 64))
    assert 0 < most <= 64 * 4 * (4 + 64 + 2 * 3) * 4 + 255     # an entry for each slot: those below the budget and those that move, each in whole fours
    assert _no_workspace(lib, lambda: lib.rsd_kv4_evict(C.byref(c), C.byref(book), 63, 0, None, 0, None))


# batch, heads, kv heads, most rows of a sequence: prompts of large batches, and the bounds that the header names
SIZES = [(128, 64, 8, 4096, True), (1024, 64, 8, 1000, True), (2, 64, 1, 1 << 20, True), (16383, 16, 16, 4096, True), (16384, 16, 16, 4096, False), (1, 64, 1, (1 << 21) - 1, True),
         (1, 64, 1, 1 << 21, False), (1 << 20, 1, 1, 64 * 15, True), (1 << 20, 1, 1, 64 * 15 + 1, False)]


@pytest.mark.parametrize("batch,heads,hkv,most,good", SIZES)
def test_prompts_of_large_batches_are_taken(lib, batch, heads, hkv, most, good):
    """batch x rows x heads was once held below 2^24, for a launch that such sizes do not make."""
    from paper_2501_19324_amd import ops
    c = _cache(ops, batch=batch, n_kv_heads=hkv)
    a = _attn(ops, rows=5, max_rows=most, n_heads=heads, q_row=heads * 64, out_row=heads * 64)
    book = ops._Book(1 << 30, None, hkv * 64, 64, 0, 0)
    assert (lib.rsd_kv4_attention_workspace(C.byref(c), C.byref(a), 1) > 0) == good
    assert _no_workspace(lib, lambda: lib.rsd_kv4_attention(C.byref(c), C.byref(a), C.byref(book), None, 0, None)) == good

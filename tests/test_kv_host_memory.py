"""Entries into the paged bf16 / fp32 cache: what a call reads may not lie in the pool that it writes.  Decided on the host, by addresses alone."""
import ctypes as C

import pytest

from test_kv_host import cache, heads, lib, ops  # noqa: F401

PAGE = 8 * 2 * 2 * 16 * 64 * 2                              # bytes of the pool: pages, kv heads, keys and values, 16 tokens of 64, bf16
POOL = 1 << 30
ROW = 2 * 64 * 2                                            # bytes of a token's keys, and of its values


def append(lib, ops, **kw):  # noqa: F811
    """An append of 3 tokens whose arrays lie apart from each other, but for those given; the out of q lies in the pool, which is refused last."""
    at = dict(k=1 << 22, v=1 << 23, q=1 << 24, k_weight=1 << 25, q_weight=(1 << 25) + 4096, seq=1 << 16, slot=(1 << 16) + 256, position=(1 << 16) + 512, freq=(1 << 16) + 1024, table=1 << 14, q_out=POOL)
    at.update(kw)
    c = cache(ops, table=at["table"], pool=POOL)
    k, q = heads(ops, x=at["k"], out=None, weight=at["k_weight"], n_heads=2, row=128), heads(ops, x=at["q"], out=at["q_out"], weight=at["q_weight"])
    r = ops._Rope(at["freq"], 64, 0, 1.0)
    rc = lib.rsd_kv_append(C.byref(c), C.byref(k), at["v"], 128, 64, C.byref(q), at["seq"], at["slot"], at["position"], C.byref(r), 1e-6, 3, 1, None)
    return rc, lib.rsd_op_last_error()


# bytes of each array that the call reads
SIZES = dict(k=3 * ROW, v=3 * ROW, q=3 * 8 * 64 * 2, k_weight=128, q_weight=128, seq=12, slot=12, position=12, freq=256, table=3 * 4 * 4)


@pytest.mark.parametrize("name", SIZES)
def test_arrays_in_the_pool_are_refused(lib, ops, name):  # noqa: F811
    for at in (POOL, POOL + PAGE // 2, POOL + PAGE - 8, POOL - SIZES[name] + 8):
        rc, text = append(lib, ops, **{name: at, "q_out": 1 << 27})
        assert rc == -1 and b"lies in the pool" in text, (at, rc, text)
    for at in (POOL + PAGE, POOL - SIZES[name]):            # side by side
        rc, text = append(lib, ops, **{name: at})
        assert rc == -1 and b"out of q shares memory with the cache" in text, (at, rc, text)

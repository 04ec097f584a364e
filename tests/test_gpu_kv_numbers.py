"""Attention over the paged bf16 / fp32 cache where numbers are what a kernel could get wrong: scores far beyond the range of the exponential.

Every form (few columns, many, 128 to a block, with and without parts) is set against the definition in 64 bits of ``kv_reference``.  u = 2^-24."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import HALF, PAIRS, R, U, bits, close, dev, host, ints, kind, make_cache, torch  # noqa: F401

pytestmark = pytest.mark.gpu

# lengths, rows, heads, kv heads
FORMS = {
    "single tokens": ([1, 40, 700], [1, 1, 1], 12, 2),
    "a single token in parts": ([3000], [1], 12, 2),
    "few columns": ([5, 90], [2, 3], 6, 2),
    "many columns": ([300, 90, 1], [40, 40, 1], 16, 2),
    "many columns in parts": ([2500, 9], [48, 3], 14, 2),
    "128 columns in parts": ([4100, 700, 300], [18, 200, 129], 16, 16),
    "128 columns": ([900, 0, 1, 40, 77] + [33 + i for i in range(18)] + [850], [40, 3, 1, 40, 5] + [1 + i % 7 for i in range(18)] + [37], 32, 16),
}


def call(torch, R, rng, form, hd, act, held, entries, queries, scale):
    """The form's call over keys and values ``entries(n, kv heads)`` with ``queries(rows, heads)``: for every sequence (out, lse, what the reference says of it, its length)."""
    lens, rows, heads, hkv = FORMS[form]
    c, table = make_cache(torch, R, rng, lens, hkv, hd, held, junk=np.nan)
    pool, size = host(c.pool), c.pool.element_size()
    for b, n in enumerate(lens):
        ref.fill(pool, table, size, hd, np.full(n, b), np.arange(n), *entries(n, hkv))
    c.pool.copy_(torch.from_numpy(pool))
    pool = host(c.pool)
    start = np.concatenate([[0], np.cumsum(rows)])
    q, q64 = dev(torch, queries(int(start[-1]), heads), kind(torch, act))
    out, lse = R.rsd_kv_attention(c, q, scale, row_start=ints(torch, start), max_rows=max(rows), max_kv=max(lens), want_lse=True)
    for b, n in enumerate(lens):
        r = slice(int(start[b]), int(start[b + 1]))
        yield host(out[r]), host(lse[r]), ref.attention(q64[r], *ref.entries(pool, table[b], n, size, hd), np.float64(np.float32(scale))), n


@pytest.mark.parametrize("scale", [1.0, 0.0884, -0.3, 2.0 ** 60])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("act,held", PAIRS)
def test_scores_beyond_the_range_of_the_exponential(torch, R, act, held, form, scale):
    """Products of one dimension, exact in fp32, from 2^10 to beyond what fp32 holds after the scale.  Unlike ones differ by 2^16 / 4 * scale > 1000 at least, so weights are 1 for the largest score of a
    row and its equals and 0 for all others: out errs by its sums, 2 (n + 96) u sum p|v|, and its rounding, lse by the rounding of a product and its logarithm."""
    rng = np.random.default_rng(len(form))
    held_bits, act_bits = (8 if held == "bf16" else 12), (8 if act == "bf16" else 12)

    def some(bits_, shape):
        return rng.integers(1 << (bits_ - 1), 1 << bits_, shape) / 2.0 ** (bits_ - 1)

    def entries(n, hkv):
        k, v = np.zeros((n, hkv, 64)), rng.normal(size=(n, hkv, 64))
        top = some(held_bits, hkv) * 2.0 ** rng.integers(8, 31, hkv)
        k[..., 0] = top * rng.choice([1.0, 0.5, -1.0, -0.5], (n, hkv))
        k[:, -1, 0] = top[-1] * 2.0 ** (np.arange(n) * 8 // max(n, 1) - 7)         # larger and larger ones
        return k, v

    def queries(rows, heads):
        q = np.zeros((rows, heads, 64))
        q[..., 0] = some(act_bits, (rows, heads)) * 2.0 ** rng.integers(8, 39, (rows, heads)) * rng.choice([1.0, -1.0], (rows, heads))
        return q

    for out, lse, (o, l, mass, _), n in call(torch, R, rng, form, 64, act, held, entries, queries, scale):
        close(out, o, 2 * (n + 96) * U * mass * 1.01 + HALF[act] * np.abs(o), (form, n))
        with np.errstate(over="ignore"):
            close(lse, l.astype(np.float32), 8 * U * np.abs(np.where(np.isfinite(l), l, 0)) + 2 * (n + 96) * U, ("lse", form, n))


@pytest.mark.parametrize("hd", [32, 128])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("act,held", PAIRS)
def test_weights_that_nearly_cancel(torch, R, act, held, form, hd):
    """Neighbours with values of opposite sign and nearly the same weight: the result is small beside sum p|v|, and so is its rounding, so the bits that weights are held in show.  bf16 activations: two bf16
    numbers, the first cut to 8 bits and the second rounded, 2^-16 of a weight; fp32: as the tolerances of ``test_gpu_kv``."""
    rng = np.random.default_rng(hd)

    def entries(n, hkv):
        v = rng.choice([-2.0, -1.5, -1.0, 1.0, 1.25, 2.0], (n, hkv, hd))
        v[1::2] = -v[:n // 2 * 2:2]
        return rng.normal(size=(n, hkv, hd)), v

    for out, lse, (o, l, mass, big), n in call(torch, R, rng, form, hd, act, held, entries, lambda rows, heads: 0.03 * rng.normal(size=(rows, heads, hd)), 1 / np.sqrt(hd)):
        ds = 2 * (hd + 48) * U * big + 8 * U * np.abs(np.where(np.isfinite(l), l, 0)) + 8 * U * big
        rel = 2 * ds + 2 * (n + 96) * U
        close(out, o, (rel[..., None] + (2.0 ** -16 if act == "bf16" else 0)) * mass * 1.01 + HALF[act] * np.abs(o), (form, n))

"""Attention over the 4-bit cache, and the weights that it deals out, where scores lie far beyond the range of the exponential; against the definition in 64 bits of ``q4_reference``.  u = 2^-24."""
import numpy as np
import pytest

import q4_reference as ref

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HD = 64
# heads, kv heads, lengths, rows
FORMS = {
    "single tokens": (12, 2, [1, 40, 700], [1, 1, 1]),
    "a single token in parts": (7, 1, [2300], [1]),
    "two tiles": (20, 1, [70, 33], [1, 1]),
    "many columns": (16, 2, [300, 90, 1], [9, 20, 1]),
    "many columns in parts": (8, 1, [1100, 90], [20, 90]),
}


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


def host(t):
    return t.detach().double().cpu().numpy()


@pytest.mark.parametrize("scale", [1.0, 0.0884, -0.3, 2.0 ** 60])
@pytest.mark.parametrize("scored", [True, False])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_beyond_the_range_of_the_exponential(torch, R, dtype, form, scored, scale):
    """Products of one dimension, exact in fp32, from 2^10 to beyond what fp32 holds after the scale.  Unlike ones differ by 2^16 / 4 * scale > 1000 at least, so a row deals its weight out evenly among the
    largest scores: out errs by its sums, 2 (n + 96) u sum p|v|, and its rounding, lse by the rounding of a product and its logarithm, a weight by 64 u (its logarithm is at most 12), a sum of weights
    by u for each of them."""
    rng = np.random.default_rng(len(form))
    heads, hkv, lens, rows = FORMS[form]
    start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    need = [-(-n // 16) for n in lens]
    cache = R.rsd_kv4_cache(len(lens), max(need), sum(need), hkv, HD)
    table = np.full((len(lens), max(need)), -1, np.int32)
    for b, m in enumerate(need):
        table[b, :m] = sum(need[:b]) + np.arange(m)
    cache.table.copy_(torch.from_numpy(table))
    cache.kv_len.copy_(torch.tensor(lens, dtype=torch.int32))
    top = rng.choice([1.0, 1.5], hkv) * 2.0 ** rng.integers(8, 31, hkv)
    for b, n in enumerate(lens):
        k, v = np.zeros((n, hkv, HD)), rng.choice([-6.0, -4.0, -1.5, -0.5, 0.5, 1.0, 2.0, 3.0], (n, hkv, HD))      # exact in four bits
        k[..., 0] = top * rng.choice([1.0, 0.5, -1.0, -0.5], (n, hkv))
        k[:, -1, 0] = top[-1] * 2.0 ** (np.arange(n) * 8 // n - 7)                 # larger and larger ones
        seq, slot = torch.full((n,), b, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")
        R.rsd_kv4_append(cache, torch.from_numpy(k).float().cuda(), torch.from_numpy(v).float().cuda(), seq, slot)
    fine = 8 if dtype == "bf16" else 12
    q64 = np.zeros((int(start[-1]), heads, HD))
    q64[..., 0] = rng.integers(1 << (fine - 1), 1 << fine, q64.shape[:2]) / 2.0 ** (fine - 1) * 2.0 ** rng.integers(8, 39, q64.shape[:2]) * rng.choice([1.0, -1.0], q64.shape[:2])
    q = torch.from_numpy(q64).to(torch.bfloat16 if dtype == "bf16" else torch.float32).cuda()
    assert np.array_equal(host(q), q64)
    scores = torch.rand(len(lens), hkv, max(need) * 16, device="cuda") if scored else None
    before = host(scores) if scored else None
    out, lse = R.rsd_kv4_attention(cache, q, scale, row_start=torch.from_numpy(start).cuda(), max_rows=max(rows), max_kv=max(lens), scores=scores, want_lse=True)
    out, lse, after, pool = host(out), host(lse), host(scores) if scored else None, cache.pool.cpu().numpy()
    group, exact = heads // hkv, float(np.float32(scale))
    for b, n in enumerate(lens):
        r = slice(start[b], start[b + 1])
        for h in range(hkv):
            cols = slice(h * group, (h + 1) * group)
            k, v, there = ref.entries(pool, table[b], n, h, HD)
            o, l, weight, mass, _ = ref.attention(q64[r, cols], k, v, there, exact, rows[b])
            assert np.all(np.abs(out[r, cols] - o) <= 2 * (n + 96) * U * mass + (2.0 ** -8 if dtype == "bf16" else 4 * U) * np.abs(o)), (b, h)
            with np.errstate(over="ignore", invalid="ignore"):
                want = l.astype(np.float32).astype(np.float64)
                assert np.all((lse[r, cols] == want) | (np.abs(lse[r, cols] - want) <= 8 * U * np.abs(l) + 2 * (n + 96) * U)), (b, h)
            if scored:
                error = np.abs(after[b, h, :n] - before[b, h, :n] - weight)
                assert np.all(error <= (64 + 2 * (n + 96) + rows[b] * group) * U * weight + 2 * U * np.abs(after[b, h, :n])), (b, h, error.max())
                assert np.array_equal(after[b, h, n:], before[b, h, n:])

"""The kernel of 128 columns to a block at each head dimension: with windows, missing pages and other strides, which are its steps with a mask, and with infinities and NaN among the entries."""
import numpy as np
import pytest

import kv_reference as ref
from test_gpu_kv import R, check_attention, torch  # noqa: F401
from test_gpu_kv_shapes import EVEN, LONG

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes,window,sinks,scale", [(LONG, 2500, 20, None), (LONG, 150, 0, -0.2), (EVEN, 30, 17, None), (EVEN, 800, 0, -0.2)], ids=str)
@pytest.mark.parametrize("hd", [32, 128])
def test_windows_missing_pages_and_strides(torch, R, hd, sizes, window, sinks, scale):  # noqa: F811
    rng = np.random.default_rng(window + hd)
    lens, rows, heads, hkv = sizes
    b = 1 if sizes is LONG else 3
    check_attention(torch, R, rng, lens, rows, heads, hkv, hd, "bf16", "bf16", window, sinks, scale=scale, missing=[(0, 0), (0, 40), (0, 41), (b, 1), (2, 0)], strided=True)


@pytest.mark.parametrize("window,sinks", [(0, 0), (60, 3), (700, 0)])
@pytest.mark.parametrize("sizes", [LONG, EVEN], ids=["parts", "whole"])
@pytest.mark.parametrize("hd", [64, 128])
def test_nonfinite_entries(torch, R, hd, sizes, window, sinks):  # noqa: F811
    """Keys and values of one kv head that are infinite or NaN, in steps with and without a mask: they reach the rows that see them and no others."""
    rng = np.random.default_rng(hd)
    lens, rows, heads, hkv = sizes
    last = len(lens) - 1
    bad = {0: (lens[0] - 6, np.nan, "v"), 1: (640, np.inf, "v"), 2: (290, -np.inf, "v"), 3: (20, np.nan, "k"), last: (830 if sizes is EVEN else 250, np.nan, "k")}

    def spike(b, k, v):
        if b in bad and bad[b][0] < len(k):
            at, x, which = bad[b]
            (v if which == "v" else k)[at, 0, hd - 3] = x

    g, _, start = check_attention(torch, R, rng, lens, rows, heads, hkv, hd, "bf16", "bf16", window, sinks, spike=spike)
    group = heads // hkv
    for b, n in enumerate(lens):
        m, o = rows[b], g[start[b]:start[b + 1]]
        assert np.isfinite(o[:, group:]).all()
        if b in bad and bad[b][0] < n:
            at, _, which = bad[b]
            sees = ref.seen(n, m, window, sinks)[:, at]
            hit = o[:, :group, hd - 3] if which == "v" else o[:, :group].reshape(m, -1)
            assert (np.isfinite(hit).all(-1) == ~sees).all()
            assert which == "k" or np.isfinite(np.delete(o[:, :group], hd - 3, -1)).all()
        else:
            assert np.isfinite(o).all()

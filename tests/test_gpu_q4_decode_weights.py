"""What the 4-bit decoder (``q4_decode``) keeps of its attention weights, and what its evictions choose by them.

Tolerance: a row's weights sum to 1 within twice their relative error, which test_gpu_ops derives: with u = 2^-24, head dimension 32, scores whose sums of
|q k| stay below 30 and up to 48 entries, 2 (2 * 51 * 30 + 4 * 30) u + 2 * 81 u + 8 u < 2^-11; every addition to a score errs by 2 u of it more."""
import numpy as np
import pytest

import q4_reference as ref

pytestmark = pytest.mark.gpu


def test_entries_receive_what_the_rows_deal_out(monkeypatch):
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2501_19324_amd import binding as R
    from paper_2501_19324_amd.q4_decode import Q4Decoder
    from rsd_inputs import model_blob_torch, workload

    w = workload("cfg0")
    s, batch, budget, recent = w.draft, 3, 24, 6
    m = Q4Decoder(s, model_blob_torch(w.seed, 0, s, torch.device("cuda:0")), batch, 48, budget, recent)
    rng = np.random.default_rng(4)
    evict, seen = R.rsd_kv4_evict, []

    def watched(cache, scores, entry_pos, budget_, recent_):
        before, pos, lens = scores.cpu().numpy(), entry_pos.cpu().numpy(), cache.kv_len.tolist()
        evict(cache, scores, entry_pos, budget_, recent_)
        after, left = scores.cpu().numpy(), entry_pos.cpu().numpy()
        for b, n in enumerate(lens):
            for h in range(s.n_kv_heads):
                kept, moves = ref.evict(before[b, h], pos[b, h].astype(np.int64), n, budget, recent)
                place = {slot: slot for slot in kept}
                place.update(moves)
                for fr, to in place.items():
                    assert left[b, h, to] == pos[b, h, fr] and after[b, h, to] == before[b, h, fr]
        seen.append(lens)

    monkeypatch.setattr(R, "rsd_kv4_evict", watched)
    feeds = [[rng.integers(0, 1023, n).tolist() for n in (20, 7, 24)]] + [[[int(t)] for t in rng.integers(0, 1023, batch)] for _ in range(30)]
    for tokens in feeds:
        m.feed(tokens)
        if seen:
            continue
        for scores, cache in zip(m.scores, m.caches):
            got = scores.double().sum((1, 2)).cpu().numpy()
            want = m.seen * s.n_heads                      # the weights of a row and head sum to 1
            assert np.all(np.abs(got - want) <= 2.0 ** -10 * want), (got, want)
    assert len(seen) >= s.n_layers                         # an eviction in every layer, of more entries than the budget
    assert all(max(lens) > budget for lens in seen)

"""The 4-bit decoder (``q4_decode``) against the same model evaluated in 64 bits from what its weights and cache hold."""
import numpy as np
import pytest

import q4_reference as ref

pytestmark = pytest.mark.gpu


def test_decoder_matches_the_model_it_holds():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2501_19324_amd import binding as R
    from paper_2501_19324_amd.q4_decode import Q4Decoder
    from rsd_inputs import blob_layout, model_blob_torch, prompt_tokens, workload

    w = workload("cfg0")
    s = w.draft
    blob = model_blob_torch(w.seed, 0, s, torch.device("cuda:0"))
    B, budget, recent = 3, 24, 6
    m = Q4Decoder(s, blob, B, 48, budget, recent)
    raw = {n: blob.view(torch.float32)[o:o + r * c].view(r, c).double().cpu().numpy() for n, r, c, o in blob_layout(s)[0]}
    q4 = {n: (ref.quantize(v)[2] if v.shape[0] > 1 and n != "embed" else v) for n, v in raw.items()}
    hd, h, hk = s.d_model // s.n_heads, s.n_heads, s.n_kv_heads
    rng = np.random.default_rng(3)
    prompts = prompt_tokens(w)

    def norm(x, g):
        return x / np.sqrt((x * x).mean(-1, keepdims=True) + s.rms_eps) * g

    def rotate(x, pos):
        ang = pos * s.rope_theta ** (-np.arange(0, hd, 2) / hd)
        a, b = x[..., :hd // 2], x[..., hd // 2:]
        return np.concatenate([a * np.cos(ang) - b * np.sin(ang), b * np.cos(ang) + a * np.sin(ang)], -1)

    def check(tokens, logits, entries_before, seen_before):
        """Every row from its embedding on, with the entries the cache holds now (written by this pass too): errors of earlier
        layers and roundings of entries near the middle of two codes stay out of the comparison."""
        row = 0
        pools = [c.pool.cpu().numpy() for c in m.caches]
        table = m.caches[0].table.cpu().numpy()
        for b, toks in enumerate(tokens):
            kv = [[ref.entries(pools[l], table[b], int(m.entries[b]), g, hd) for g in range(hk)] for l in range(s.n_layers)]
            for j, tok in enumerate(toks):
                x = raw["embed"][tok]
                pos = seen_before[b] + j
                for l in range(s.n_layers):
                    p = f"l{l}."
                    y = norm(x, raw[p + "attn_norm"][0])
                    q = rotate((q4[p + "wq"] @ y).reshape(h, hd), pos)
                    seen = int(entries_before[b]) + j + 1
                    att = np.zeros((h, hd))
                    for g in range(hk):
                        k, v, there = kv[l][g]
                        part, *_ = ref.attention(q[None, g * h // hk:(g + 1) * h // hk], k[:seen], v[:seen], there[:seen], hd ** -0.5, 1)
                        att[g * h // hk:(g + 1) * h // hk] = part[0]
                        # the entry itself: the rotated key and the value, within a step of the format
                        for got, want in ((k[seen - 1], rotate((q4[p + "wk"] @ y).reshape(hk, hd), pos)[g]), (v[seen - 1], (q4[p + "wv"] @ y).reshape(hk, hd)[g])):
                            step = np.abs(want).reshape(-1, 32).max(-1).repeat(32) / 3.5
                            assert np.all(np.abs(got - want) <= step)
                    x = x + q4[p + "wo"] @ att.reshape(-1)
                    y = norm(x, raw[p + "ffn_norm"][0])
                    gate, up = q4[p + "w_gate"] @ y, q4[p + "w_up"] @ y
                    x = x + q4[p + "w_down"] @ (gate / (1 + np.exp(-gate)) * up)
                want = q4["lm_head"] @ norm(x, raw["final_norm"][0])
                assert np.max(np.abs(logits[row] - want)) < 1e-4        # the framework's tolerance for fp32 logits
                row += 1
        assert row == len(logits)

    lens, evictions = [20, 7, 24], 0
    feeds = [[prompts[b, :lens[b]].tolist() for b in range(B)]]
    feeds += [[[int(t)] for t in rng.integers(0, 1023, B)] for _ in range(30)] + [[[1, 2, 3, 4, 5], [], [9]]]
    for i, tokens in enumerate(feeds):
        entries, seen = m.entries.copy(), m.seen.copy()
        logits = m.feed(tokens).double().cpu().numpy()
        if (m.entries < entries + [len(t) for t in tokens]).any():
            evictions += 1
            entries = np.minimum(entries, budget)
            for l in range(s.n_layers):                    # the newest tokens have survived
                for b in range(B):
                    for g in range(hk):
                        kept = set(m.entry_pos[l][b, g, :int(m.entries[b])].tolist())
                        assert kept >= set(range(int(m.seen[b]) - len(tokens[b]) - min(recent, int(entries[b])), int(m.seen[b])))
                        assert len(kept) == m.entries[b]
        if i < 3 or i % 7 == 0 or i > 28:
            check(tokens, logits, entries, seen)
    assert evictions >= 1
    # what every row has dealt out is what the entries have received, less what evicted entries took with them
    total = float(sum(sc[1, :, :int(m.entries[1])].sum() for sc in m.scores))
    assert total <= m.seen[1] * s.n_layers * h * (1 + 1e-5)

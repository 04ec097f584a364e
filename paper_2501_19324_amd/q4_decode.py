"""A decoder whose weights and KV cache are held in 4 bits, and whose cache keeps to a budget of entries: the operators of
``include/rsd_ops.h`` as a decode loop uses them.

``Q4Decoder`` takes one of the framework's models (a shape and its weight blob, the layout of ``rsd_inputs.blob_layout``), packs the
projections into 4-bit tiles and feeds ragged batches of tokens: one token per sequence (decoding), several (a step to be scored or
verified) or whole prompts.  Per layer the queries, keys and values come from one product with 4-bit weights, keys are rotated and
written with their positions, attention reads the cache and adds up the weight every entry receives; when some sequence
would outgrow its pages, every sequence with more than ``budget`` entries falls back to that many, each kv head by its own weights.  Norms, rotation and the
activation are plain torch, and activations are fp32 whatever the model's type: the products and the attention run in their fp32 forms.

    python -m paper_2501_19324_amd.q4_decode --workload cfg1 --layers 4 --tokens 64
"""
from __future__ import annotations

import argparse
from typing import List, Sequence

import numpy as np
import torch

from . import binding as R


class Q4Decoder:
    def __init__(self, shape, blob: torch.Tensor, batch: int, capacity: int, budget: int, recent: int):
        """``capacity`` entries of room per sequence; ``budget`` of them survive an eviction, the ``recent`` newest among them.  An eviction cuts back
        every sequence that holds more, whichever of them ran out of room."""
        from rsd_inputs import blob_layout

        if not 0 < budget < capacity or not 0 <= recent <= budget:
            raise ValueError(f"budget {budget}, recent {recent}, capacity {capacity}")
        self.s, self.batch, self.budget, self.recent = shape, batch, budget, recent
        self.dtype = torch.float32 if shape.dtype == "f32" else torch.bfloat16
        w = {n: blob.view(self.dtype)[off:off + r * c].view(r, c) for n, r, c, off in blob_layout(shape)[0]}
        self.embed = w["embed"]
        self.layers = []
        for i in range(shape.n_layers):
            p = f"l{i}."
            self.layers.append(dict(attn_norm=w[p + "attn_norm"][0].float(), ffn_norm=w[p + "ffn_norm"][0].float(),
                                    qkv=R.rsd_w4_pack(torch.cat([w[p + "wq"], w[p + "wk"], w[p + "wv"]])), o=R.rsd_w4_pack(w[p + "wo"]),
                                    gate_up=R.rsd_w4_pack(torch.cat([w[p + "w_gate"], w[p + "w_up"]])), down=R.rsd_w4_pack(w[p + "w_down"])))
        self.final_norm, self.head = w["final_norm"][0].float(), R.rsd_w4_pack(w["lm_head"])
        self.hd = shape.d_model // shape.n_heads
        pages = -(-capacity // 16)
        self.capacity = 16 * pages
        table = torch.arange(batch * pages, dtype=torch.int32, device=blob.device).view(batch, pages)
        self.caches: List[R.Kv4Cache] = []
        self.scores, self.entry_pos = [], []
        for _ in range(shape.n_layers):
            c = R.rsd_kv4_cache(batch, pages, batch * pages, shape.n_kv_heads, self.hd, blob.device)
            self.caches.append(R.Kv4Cache(c.pool, table, c.kv_len))
            self.scores.append(torch.zeros(batch, shape.n_kv_heads, self.capacity, device=blob.device))
            self.entry_pos.append(torch.zeros(batch, shape.n_kv_heads, self.capacity, dtype=torch.int32, device=blob.device))
        self.entries = np.zeros(batch, np.int64)           # entries of each sequence, tokens seen so far
        self.seen = np.zeros(batch, np.int64)
        inv = shape.rope_theta ** (-torch.arange(0, self.hd, 2, dtype=torch.float64, device=blob.device) / self.hd)
        self.inv = inv

    def _norm(self, x, gain):
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.s.rms_eps) * gain

    def _rotate(self, x, cos, sin):
        a, b = x.float().chunk(2, -1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

    def feed(self, tokens: Sequence[Sequence[int]]) -> torch.Tensor:
        """The next tokens of every sequence (ragged, possibly none); fp32 logits [rows, vocab], a row per token, sequence by sequence."""
        count = np.array([len(t) for t in tokens])
        if len(count) != self.batch or count.max() > self.capacity - self.budget:
            raise ValueError(f"{len(count)} sequences with up to {count.max()} tokens; room for {self.batch} and {self.capacity - self.budget}")
        dev = self.embed.device
        if (self.entries + count).max() > self.capacity:
            for c, score, pos in zip(self.caches, self.scores, self.entry_pos):
                R.rsd_kv4_evict(c, score, pos, self.budget, self.recent)
            self.entries = np.minimum(self.entries, self.budget)
        rows, start = int(count.sum()), np.concatenate([[0], np.cumsum(count)])
        within = np.arange(rows) - np.repeat(start[:-1], count)
        seq = np.repeat(np.arange(self.batch), count)
        index = torch.from_numpy(np.stack([seq, self.entries[seq] + within, self.seen[seq] + within, np.concatenate([np.asarray(t) for t in tokens])]).astype(np.int32)).to(dev)
        seq_d, slot_d, pos_d, tok = index
        self.entries, self.seen = self.entries + count, self.seen + count
        lens = torch.from_numpy(self.entries.astype(np.int32)).to(dev)
        row_start = torch.from_numpy(start.astype(np.int32)).to(dev)
        angle = pos_d.double()[:, None] * self.inv[None]
        cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
        x = self.embed[tok.long()].float()
        h, hk, hd = self.s.n_heads, self.s.n_kv_heads, self.hd
        for i, w in enumerate(self.layers):
            cache = self.caches[i]
            qkv = R.rsd_w4_linear(self._norm(x, w["attn_norm"]), w["qkv"]).view(rows, h + 2 * hk, hd)
            qk = self._rotate(qkv[:, :h + hk], cos, sin)
            cache.kv_len.copy_(lens)
            R.rsd_kv4_append(cache, qk[:, h:], qkv[:, h + hk:], seq_d, slot_d, position=pos_d, entry_pos=self.entry_pos[i], scores=self.scores[i])
            att = R.rsd_kv4_attention(cache, qk[:, :h], hd ** -0.5, row_start=row_start, max_rows=int(count.max()), max_kv=int(self.entries.max()), scores=self.scores[i])
            x = x + R.rsd_w4_linear(att.view(rows, h * hd), w["o"])
            gate, up = R.rsd_w4_linear(self._norm(x, w["ffn_norm"]), w["gate_up"]).chunk(2, -1)
            x = x + R.rsd_w4_linear(torch.nn.functional.silu(gate) * up, w["down"])
        return R.rsd_w4_linear(self._norm(x, self.final_norm), self.head)


def main() -> None:
    import time

    from rsd_inputs import model_blob_torch, prompt_lengths, prompt_tokens, workload

    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--workload", default="cfg0")
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=48, help="tokens to decode")
    ap.add_argument("--budget", type=int, default=64)
    ap.add_argument("--room", type=int, default=32, help="entries beyond the budget before a sequence is cut back")
    a = ap.parse_args()
    w = workload(a.workload, n_layers=a.layers)
    blob = model_blob_torch(w.seed, 0, w.draft, torch.device("cuda:0"))
    m = Q4Decoder(w.draft, blob, w.batch, a.budget + a.room, a.budget, min(16, a.budget))
    prompts, lens = prompt_tokens(w), prompt_lengths(w)
    for at in range(0, int(lens.max()), a.room):           # prompts in pieces that fit
        piece = [prompts[b, at:min(at + a.room, lens[b])].tolist() for b in range(w.batch)]
        logits = m.feed(piece)
        ends = np.cumsum([len(p) for p in piece]) - 1
        nxt = [int(t) for t in R.rsd_sample_static(logits[torch.from_numpy(ends).clamp(min=0)], None, 0.0, 1.0).tolist()]
        last = nxt if at == 0 else [n if p else o for n, o, p in zip(nxt, last, piece)]
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    for _ in range(a.tokens):
        last = R.rsd_sample_static(m.feed([[t] for t in last]), None, 0.0, 1.0).tolist()
    dt = time.perf_counter() - t0
    print(f"{w.name}: {w.batch} sequences, {a.layers} layers, {a.tokens} tokens each in {dt:.3f} s; {m.seen[0]} tokens seen, {m.entries[0]} entries kept; last tokens {last[:8]}")


if __name__ == "__main__":
    main()

"""What the operators on the paged bf16 / fp32 cache are measured on, with their plain forms.

Three operators of a decoding step, in the order in which a layer calls them: queries and keys normed for each head and rotated by their
position in one pass (``rope``), the same with keys and values written into a paged cache on the way (``append``), and attention of new
tokens over that cache, optionally with a sliding window and a few first tokens that stay visible (``attention``).

Norm of a head: x / sqrt(mean(x^2) + eps) * weight.  Rotation: the first ``rot`` dimensions form pairs, (2 i, 2 i + 1) where they are interleaved,
(i, i + rot / 2) otherwise; pair i of a token at position p turns by p * freq[i], and is multiplied by ``magnitude``.  The other dimensions stay.

A cache is (pool, table, kv_len): pool ``[n_pages][kv heads][2][16 * hd]``, keys and values of 16 tokens, E = 16 bytes / size of a value:
keys ``[hd / 4E][4][16 tokens][E]`` (dims 4E j + E c + i), values ``[hd / 4E][4][16 dims][E / 4][4 tokens]`` (dims 4E j + 16 x + d, tokens 4 c + i).
Row j of a sequence's q rows stands at slot p = n - q + j of its n entries and sees the slots s <= p with s > p - window (window 0: all) or s < sinks.

Widths, batch sizes, prompt and step lengths are those of the workload definitions (the 1.5B, 7B and 72B shapes, the tiny fp32 configuration; batches of 1,
4, 16, 64, 256; contexts up to 8192; steps of up to 128 tokens); windows and rotations are generic.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

PAGE = 16
EPS = 1e-6
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # ---- norms and rotation of queries and keys
        # the tiny configuration's batch of single tokens: latency only
        dict(name="rope_tiny_b4_f32", op="rope", rows=4, heads=4, kv_heads=2, hd=32, rot=32, interleaved=False, scaled=False, normed=False, far=96, dtype="f32"),
        # steps of 128 tokens of 64 sequences, 7B heads, before a cache of another kind
        dict(name="rope_7b_steps", op="rope", rows=8192, heads=28, kv_heads=4, hd=128, rot=128, interleaved=False, scaled=False, normed=True, far=5120, dtype="bf16"),
        # half of a head rotates, neighbours in pairs, frequencies scaled for a long context; fp32 activations of 16 prompts
        dict(name="rope_72b_partial_far_f32", op="rope", rows=7937, heads=64, kv_heads=8, hd=128, rot=64, interleaved=True, scaled=True, normed=True, far=131072, dtype="f32"),
        # ---- the same on the way into the cache
        # one new token of 64 sequences
        dict(name="append_7b_b64", op="append", batch=64, heads=28, kv_heads=4, hd=128, rot=128, interleaved=False, scaled=False, normed=True, tok_lo=1, tok_hi=1,
             dtype="bf16", cache="bf16"),
        # prompts of 16 sequences, fp32 activations into a bf16 cache
        dict(name="append_72b_prompts_f32", op="append", batch=16, heads=64, kv_heads=8, hd=128, rot=128, interleaved=False, scaled=True, normed=False, tok_lo=480, tok_hi=512,
             dtype="f32", cache="bf16"),
        # ---- attention
        # one sequence, 1.5B shape, at the end of a run of 16 steps
        dict(name="attn_1p5b_b1", op="attention", batch=1, heads=12, kv_heads=2, hd=128, kv_lo=1279, kv_hi=1279, q_lo=1, q_hi=1, window=0, sinks=0, dtype="bf16", cache="bf16"),
        # 64 ragged sequences of the 7B shape with four drafted tokens and one of their own each: verification
        dict(name="attn_7b_b64_verify", op="attention", batch=64, heads=28, kv_heads=4, hd=128, kv_lo=128, kv_hi=5120, q_lo=5, q_hi=5, window=0, sinks=0, dtype="bf16", cache="bf16"),
        # the long-context configuration: single tokens of 256 sequences, up to 8192 tokens
        dict(name="attn_7b_b256_8k", op="attention", batch=256, heads=28, kv_heads=4, hd=128, kv_lo=4096, kv_hi=8192, q_lo=1, q_hi=1, window=0, sinks=0, dtype="bf16", cache="bf16"),
        # the same lengths where a token sees the last 1024 and the first 4
        dict(name="attn_7b_b256_8k_window", op="attention", batch=256, heads=28, kv_heads=4, hd=128, kv_lo=4096, kv_hi=8192, q_lo=1, q_hi=1, window=1024, sinks=4, dtype="bf16", cache="bf16"),
        # a chunk of a long prompt
        dict(name="attn_7b_chunk_2k_of_8k", op="attention", batch=1, heads=28, kv_heads=4, hd=128, kv_lo=8192, kv_hi=8192, q_lo=2048, q_hi=2048, window=0, sinks=0, dtype="bf16", cache="bf16"),
        # steps of up to 128 tokens of 16 sequences through the 72B shape (catch-up and scoring passes), windowed, fp32 activations over a bf16 cache
        dict(name="attn_72b_b16_steps_window_f32", op="attention", batch=16, heads=64, kv_heads=8, hd=128, kv_lo=512, kv_hi=2560, q_lo=17, q_hi=128, window=1000, sinks=16,
             dtype="f32", cache="bf16"),
        # everything in fp32, heads of 64, steps of 16 sequences
        dict(name="attn_hd64_b16_steps_f32", op="attention", batch=16, heads=16, kv_heads=16, hd=64, kv_lo=300, kv_hi=1025, q_lo=17, q_hi=128, window=0, sinks=0, dtype="f32", cache="f32"),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention"])
    heads, kv_heads, hd = rng.choice([(12, 2, 128), (28, 4, 128), (64, 8, 128), (4, 2, 32), (8, 2, 32), (16, 16, 64), (9, 3, 64), (20, 1, 128)])
    dtype = rng.choice(["bf16", "f32"])
    if op != "attention":
        c = dict(op=op, heads=heads, kv_heads=kv_heads, hd=hd, rot=rng.choice([hd, hd, hd // 2, hd // 4, 2 * rng.randint(1, hd // 2)]), interleaved=rng.random() < 0.5,
                 scaled=rng.random() < 0.5, normed=rng.random() < 0.5, dtype=dtype)
        if op == "rope":
            return dict(c, rows=_spread(rng, 1, 7936), far=_spread(rng, 16, 1 << 20))
        hi = 1 if rng.random() < 0.4 else _spread(rng, 2, 1024)
        return dict(c, batch=max(1, min(_spread(rng, 1, 256), 7936 // hi)), tok_lo=max(1, hi // 2), tok_hi=hi, cache=rng.choice(["bf16", dtype]))
    hi = _spread(rng, 1, 8192)
    batch = _spread(rng, 1, 256)
    q = rng.choice([1, 1, _spread(rng, 2, 16), _spread(rng, 2, 128), _spread(rng, 2, 2048)])
    while batch > 1 and (batch * hi * kv_heads * hd > 128 * 6144 * 4 * 128 or batch * q * heads * hi > 16 * 128 * 64 * 2048):
        batch //= 2
    q = max(1, min(q, hi, 16 * 128 * 64 * 2048 // (batch * heads * hi)))
    window = 0 if rng.random() < 0.5 else _spread(rng, 1, 2048)
    return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, hd=hd, kv_lo=rng.choice([hi, max(1, hi // 8)]), kv_hi=hi, q_lo=max(1, q // 4), q_hi=q,
                window=window, sinks=rng.choice([0, 4, 17]) if window else 0, dtype=dtype, cache=rng.choice(["bf16", dtype]))


# ---------------------------------------------------------------- layout of the cache, in elementary operations

def _views(pool, hd):
    """Keys [..., hd/4E, 4, 16 tokens, E] and values [..., hd/4E, 4, 16 dims, E/4, 4 tokens] of every (page, kv head)."""
    e = 16 // pool.element_size()
    return pool[..., 0, :].unflatten(-1, (hd // (4 * e), 4, PAGE, e)), pool[..., 1, :].unflatten(-1, (hd // (4 * e), 4, 16, e // 4, 4))


def _write(pool, table, hd, seq, slot, k, v):
    """Entries k, v [rows][kv heads][hd] into slot[i] of sequence seq[i]."""
    page, t = table[seq, slot // PAGE].long(), slot % PAGE
    pk, pv = _views(pool, hd)
    e = pk.shape[-1]
    pk[page, :, :, :, t] = k.to(pool.dtype).unflatten(-1, (-1, 4, e))
    pv[page, :, :, t // 4, :, :, t % 4] = v.to(pool.dtype).unflatten(-1, (-1, e // 4, 16)).transpose(-1, -2)


def _values(pages, hd):
    """Pages [..., kv heads, 2, 16 hd] -> keys and values [..., kv heads, 16, hd] in 32 bits."""
    pk, pv = _views(pages, hd)
    k = pk.movedim(-2, -4).flatten(-3)                                     # [..., t, j, c, i]
    d = pv.dim()
    v = pv.permute(*range(d - 5), d - 4, d - 1, d - 5, d - 2, d - 3)       # [..., t/4, t%4, j, x, dim]
    return k.float(), v.flatten(-3).flatten(-3, -2).float()


# ---------------------------------------------------------------- inputs

def _frequencies(case):
    """Radians a position for every pair, and the magnitude: plain, or scaled by parts for a context 16 times an original one of 8192 (pairs that turn
    more than 32 times over it stay, those that turn less than once are slowed down 16 times, with a ramp between)."""
    freq = [1e6 ** (-2 * i / case["rot"]) for i in range(case["rot"] // 2)]
    if not case["scaled"]:
        return freq, 1.0
    out = []
    for f in freq:
        keep = max(0.0, min(1.0, (8192 * f / (2 * math.pi) - 1) / (32 - 1)))
        out.append(f * keep + f / 16 * (1 - keep))
    return out, 0.1 * math.log(16) + 1


def _ragged(lo, hi, count, odd):
    """Lengths of a batch: the same multiset for every seed (the inputs' order and values come from the seed)."""
    v = np.random.RandomState((lo * 31 + hi * 7 + count) * 4 + odd).randint(lo, hi + 1, count)
    v[0] = hi
    return v


def _pages(gen, lens):
    """A table over a pool with a quarter of spare pages, in random order; the number of pages."""
    need = [-(-n // PAGE) for n in lens]
    total = sum(need) + max(1, sum(need) // 4)
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(lens), max(need)), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max(need), device="cuda")[None] < torch.tensor(need, device="cuda")[:, None]] = order[:sum(need)]
    return table, total


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 31))
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    ints = lambda a: torch.tensor(np.asarray(a), dtype=torch.int32, device="cuda")  # noqa: E731
    s = SimpleNamespace(op=case["op"], hd=case["hd"], heads=case["heads"], kv_heads=case["kv_heads"])
    dtype = TYPES[case["dtype"]]
    if s.op != "attention":
        rows = case.get("rows")
        if s.op == "append":
            count = [int(x) for x in rs.permutation(_ragged(case["tok_lo"], case["tok_hi"], case["batch"], 0))]
            at = [int(x) for x in rs.randint(0, 64, len(count))]
            slots = [64 + case["tok_hi"]] * len(count)                     # (a pool's size does not depend on the seed)
            s.table, total = _pages(gen, slots)
            s.kv_len = ints([a + c for a, c in zip(at, count)])
            s.pool = rand(total, s.kv_heads, 2, PAGE * s.hd).to(TYPES[case["cache"]])
            s.seq = ints(np.repeat(np.arange(len(count)), count))
            s.slot = ints(np.concatenate([np.arange(a, a + c) for a, c in zip(at, count)]))
            s.position = s.slot
            rows = sum(count)
        else:
            s.position = torch.randint(0, case["far"], (rows,), generator=gen, device="cuda", dtype=torch.int32)
            s.position[0] = case["far"] - 1
        # queries, keys and values as a fused projection leaves them, with a few strong channels
        qkv = rand(rows, s.heads + 2 * s.kv_heads, s.hd) * torch.exp(0.5 * rand(1, s.heads + 2 * s.kv_heads, s.hd))
        qkv = qkv.to(dtype)
        s.q, s.k, s.v = qkv[:, :s.heads], qkv[:, s.heads:s.heads + s.kv_heads], qkv[:, s.heads + s.kv_heads:]
        s.q_weight = s.k_weight = None
        if case["normed"]:
            s.q_weight, s.k_weight = (1 + 0.3 * rand(s.hd)).to(dtype), (1 + 0.3 * rand(s.hd)).to(dtype)
        freq, magnitude = _frequencies(case)
        s.rope = (torch.tensor(freq, dtype=torch.float64, device="cuda"), case["interleaved"], magnitude)
        return s
    order = rs.permutation(case["batch"])
    lens = [int(x) for x in _ragged(case["kv_lo"], case["kv_hi"], case["batch"], 0)[order]]
    rows = [min(int(r), n) for r, n in zip(_ragged(case["q_lo"], case["q_hi"], case["batch"], 1)[order], lens)]
    s.table, total = _pages(gen, lens)
    s.kv_len = ints(lens)
    # keys with a few strong channels, values of unit size; what lies behind a sequence's last entry is as the memory was: anything, NaN among it
    s.pool = torch.empty(total, s.kv_heads, 2, PAGE * s.hd, dtype=TYPES[case["cache"]], device="cuda")
    for p in range(0, total, 8192):
        s.pool[p:p + 8192] = rand(*s.pool[p:p + 8192].shape)
    pk, pv = _views(s.pool, s.hd)
    pk *= torch.exp(0.5 * rand(s.kv_heads, pk.shape[2], 4, 1, pk.shape[-1])).to(s.pool.dtype)
    last = s.table.gather(1, ((s.kv_len.long() - 1) // PAGE)[:, None])[:, 0].long()
    behind = torch.arange(PAGE, device="cuda")[None] > ((s.kv_len.long() - 1) % PAGE)[:, None]
    pk[last] = torch.where(behind[:, None, None, None, :, None], math.nan, pk[last])
    pv[last] = torch.where(behind.view(-1, 1, 1, 4, 1, 1, 4), math.nan, pv[last])
    s.max_rows, s.max_kv, s.window, s.sinks = max(rows), max(lens), case["window"], case["sinks"]
    s.row_start = ints(np.concatenate([[0], np.cumsum(rows)]))
    s.q = (1.5 * rand(sum(rows), s.heads, s.hd)).to(dtype)
    s.factor = 1.0 / math.sqrt(s.hd)
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    if s.op == "attention":
        return _plain_attention(s)
    q, k = _plain_rope(s, s.q, s.q_weight), _plain_rope(s, s.k, s.k_weight)
    if s.op == "rope":
        return {"q": q.to(s.q.dtype), "k": k.to(s.k.dtype)}
    _write(s.pool, s.table, s.hd, s.seq.long(), s.slot.long(), k, s.v)
    return {"q": q.to(s.q.dtype), "pool": s.pool}


def _run_own(s):
    from paper_2501_19324_amd import binding as R

    if s.op == "rope":
        q, k = R.rsd_qk_rope(s.q, s.k, s.position, s.rope, q_weight=s.q_weight, k_weight=s.k_weight, eps=EPS)
        return {"q": q, "k": k}
    cache = (s.pool, s.table, s.kv_len)
    if s.op == "append":
        q = R.rsd_kv_append(cache, s.k, s.v, s.seq, s.slot, position=s.position, rope=s.rope, k_weight=s.k_weight, eps=EPS, q=s.q, q_weight=s.q_weight)
        return {"q": q, "pool": s.pool}
    out, lse = R.rsd_kv_attention(cache, s.q, s.factor, row_start=s.row_start, max_rows=s.max_rows, max_kv=s.max_kv, window=s.window, sinks=s.sinks, want_lse=True)
    return {"out": out, "lse": lse}


def _plain_rope(s, x, weight):
    """Heads [rows, heads, hd] normed and rotated, in 32 bits."""
    freq, interleaved, magnitude = s.rope
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    angle = s.position.double()[:, None] * freq
    cos, sin = (torch.cos(angle) * magnitude).float()[:, None], (torch.sin(angle) * magnitude).float()[:, None]
    rot = 2 * freq.shape[0]
    turn, stay = x[..., :rot], x[..., rot:]
    if interleaved:
        a, b = turn[..., 0::2], turn[..., 1::2]
        turn = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = turn[..., :rot // 2], turn[..., rot // 2:]
        turn = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turn, stay], -1)


def _plain_attention(s):
    dev, (rows, heads, hd) = s.q.device, s.q.shape
    batch, group = len(s.kv_len), heads // s.kv_heads
    k, v = _values(s.pool[s.table.clamp(min=0).long()], hd)                # [b, page, kv head, 16, hd]
    k, v = k.transpose(1, 2).flatten(2, 3), v.transpose(1, 2).flatten(2, 3)
    slot = torch.arange(k.shape[2], device=dev)
    there = (slot[None] < s.kv_len[:, None])[:, None, :, None]
    k, v = torch.where(there, k, 0.0), torch.where(there, v, 0.0)
    # rows of every sequence, padded to max_rows
    r = torch.arange(s.max_rows, device=dev)
    count = (s.row_start[1:] - s.row_start[:-1]).long()
    at = (s.row_start[:-1].long()[:, None] + r[None]).clamp(max=rows - 1)
    used = r[None] < count[:, None]
    q = s.q.float()[at].view(batch, s.max_rows, s.kv_heads, group, hd).permute(0, 2, 1, 3, 4).flatten(2, 3)
    p = (s.kv_len.long()[:, None] - count[:, None] + r[None])[:, :, None]
    seen = (slot <= p) & used[:, :, None]                                  # [b, row, slot]
    if s.window:
        seen &= (slot > p - s.window) | (slot < s.sinks)
    logit = (q @ k.transpose(-1, -2) * s.factor).unflatten(2, (s.max_rows, group))
    logit = torch.where(seen[:, None, :, None], logit, -math.inf)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    w = torch.exp(logit - top)
    total = w.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    w = torch.where(total > 0, w / total, torch.zeros_like(w))
    out = (w.flatten(2, 3) @ v).unflatten(2, (s.max_rows, group))          # [b, kv head, row, g, hd]
    line = torch.arange(rows, device=dev)
    b = (line[:, None] >= s.row_start[None, 1:]).sum(-1)
    i = line - s.row_start[b]
    out = out.permute(0, 2, 1, 3, 4)[b, i].flatten(1, 2)
    return {"out": out.to(s.q.dtype), "lse": lse[..., 0].permute(0, 2, 1, 3)[b, i].flatten(1, 2)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size, hd, heads, kv_heads = 4 if case["dtype"] == "f32" else 2, case["hd"], case["heads"], case["kv_heads"]
    held = 4 if case.get("cache") == "f32" else 2
    if case["op"] != "attention":
        rows = case["rows"] if case["op"] == "rope" else int(_ragged(case["tok_lo"], case["tok_hi"], case["batch"], 0).sum())
        flops = rows * (heads + kv_heads) * (3 * case["rot"] + (4 * hd if case["normed"] else 0))
        if case["op"] == "rope":
            return {"bytes": rows * (2 * (heads + kv_heads) * hd * size + 4), "flops": flops}
        return {"bytes": rows * ((2 * heads + 2 * kv_heads) * hd * size + 2 * kv_heads * hd * held + 12), "flops": flops}
    lens = _ragged(case["kv_lo"], case["kv_hi"], case["batch"], 0)
    rows = np.minimum(_ragged(case["q_lo"], case["q_hi"], case["batch"], 1), lens)
    window, sinks, entries, pairs = case["window"], case["sinks"], 0, 0
    for n, q in zip(lens.tolist(), rows.tolist()):
        p = np.arange(n - q, n)
        first = np.maximum(0, p - window + 1) if window else np.zeros_like(p)
        extra = np.minimum(sinks, first) if window else np.zeros_like(p)
        pairs += int((p + 1 - first + extra).sum())
        entries += int(n - first[0] + extra[0])
    return {"bytes": entries * 2 * kv_heads * hd * held + int(rows.sum()) * heads * (2 * hd * size + 4), "flops": pairs * 4 * heads * hd}


# ---------------------------------------------------------------- the definitions in 64 bits

def _turned(x, weight, s):
    """A head's dimensions as the products of complex numbers that they are, in 64 bits."""
    freq, interleaved, magnitude = s.rope
    x = x.double()
    if weight is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / s.hd + EPS) * weight.double()
    half = freq.numel()
    i = torch.arange(half, device=x.device)
    re, im = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    z = torch.complex(x[..., re], x[..., im]) * torch.polar(torch.full_like(freq, magnitude).expand(len(x), half), s.position.double()[:, None] * freq)[:, None]
    x[..., re], x[..., im] = z.real, z.imag
    return x


def _entries(pool, table_row, n, hd):
    """The first n entries of one sequence: keys and values [kv head][n][hd] in 64 bits, element by element."""
    e, heads = 16 // pool.element_size(), pool.shape[1]
    raw = pool[table_row[:-(-n // PAGE)].long()].transpose(0, 1).reshape(heads, -1)      # pages of a head one after the other
    t, d = torch.arange(n, device=pool.device)[:, None], torch.arange(hd, device=pool.device)[None]
    page, i = t // PAGE * (2 * PAGE * hd), t % PAGE
    key = raw[:, page + d // e * (16 * e) + i * e + d % e]
    x = d % (4 * e) // 16
    val = raw[:, page + PAGE * hd + d // (4 * e) * (64 * e) + i // 4 * (16 * e) + d % 16 * e + x * 4 + i % 4]
    return key.double(), val.double()


def exact(case, seed):
    s = prepare(case, seed)
    if s.op != "attention":
        q, k = _turned(s.q, s.q_weight, s), _turned(s.k, s.k_weight, s)
        if s.op == "rope":
            return {"q": q, "k": k}
        e, pool = 16 // s.pool.element_size(), s.pool.double()
        line = pool.view(len(pool), s.kv_heads, -1)
        page, t = s.table[s.seq.long(), s.slot.long() // PAGE].long(), s.slot.long() % PAGE
        for d in range(s.hd):
            line[page, :, d // e * (16 * e) + t * e + d % e] = k[..., d]
            line[page, :, PAGE * s.hd + d // (4 * e) * (64 * e) + t // 4 * (16 * e) + d % 16 * e + d % (4 * e) // 16 * 4 + t % 4] = s.v[..., d].double()
        return {"q": q, "pool": pool}
    outs, lses, start = [], [], s.row_start.tolist()
    for b, n in enumerate(s.kv_len.tolist()):
        q = s.q[start[b]:start[b + 1]].double()
        rows, heads, hd = q.shape
        k, v = _entries(s.pool, s.table[b], n, hd)
        out, lse = torch.empty_like(q), q.new_empty(rows, heads)
        hidden = torch.zeros(rows, n, dtype=torch.bool, device=q.device)
        for j in range(rows):
            p = n - rows + j
            hidden[j, p + 1:] = True
            if s.window and p - s.window >= s.sinks:
                hidden[j, s.sinks:p - s.window + 1] = True
        for h in range(heads):
            z = (q[:, h] @ k[h // (heads // s.kv_heads)].T * s.factor).masked_fill(hidden, -math.inf)
            lse[:, h] = torch.logsumexp(z, -1)
            out[:, h] = torch.softmax(z, -1) @ v[h // (heads // s.kv_heads)]
        outs.append(out)
        lses.append(lse)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}

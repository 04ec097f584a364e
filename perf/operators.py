"""What the 4-bit operators are measured on, with their plain forms.

Four operators of a decode step whose memory is 4 bits wide: products with 4-bit weights (``w4``), writing keys and values
into a paged 4-bit cache and reading entries back (``append``), attention over that cache (``attention``), and eviction
from it by accumulated attention weight (``evict``).

Format of weights and cache: groups of 32 values along the contracted axis (the head dimension in the cache) share a scale
2^(s - 127), one byte s per group, 255 for a group that held NaN or infinity; a value is a sign and one of 0, .5, 1, 1.5, 2,
3, 4, 6.  The scale exponent is the least e with max|x| <= 7 * 2^e, within -125 .. 125; values are rounded to nearest, ties to the
even code.  Bytes hold two values, the first in the low half.

Weights [N][K] are kept in tiles of 16 rows x 128 columns, zero beyond N and K: codes ``[N/16][K/128][4 groups][16 rows][16
bytes]``, scales ``[N/16][K/512][4 groups][16 rows][4 tiles]``.  A cache page holds 16 tokens of every kv head, hd * 17 bytes each: key
codes ``[4 quarters of the head dimension][16 tokens][hd/8 bytes]``, value codes ``[token/4][dim % 16][dim/32][token % 4]`` (a byte: the
dims m and m + 16 of its group), key scales ``[dim/32][16 tokens]``, value scales ``[token/4][dim/32][token % 4]``.

Widths, batch sizes, prompt and step lengths are those of the workload definitions (the 1.5B, 7B and 72B shapes, the tiny
fp32 configuration; batches of 1, 4, 16, 64, 256; contexts up to 8192; steps of up to 128 tokens).
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False

PAGE = 16
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # ---- products with 4-bit weights
        # the tiny configuration's widest product at its batch of 4: latency only
        dict(name="w4_tiny_b4_f32", op="w4", rows=4, n=1024, k=256, dtype="f32"),
        # one sequence, gate and up projection of the 7B shape: interactive decoding
        dict(name="w4_7b_gate_up_b1", op="w4", rows=1, n=37888, k=3584, dtype="bf16"),
        # down projection of the 72B shape, 16 sequences of which three have finished, fp32 activations
        dict(name="w4_72b_down_b13_f32", op="w4", rows=13, n=8192, k=29568, dtype="f32"),
        # the largest serving batch through the 7B shape's down projection
        dict(name="w4_7b_down_b256", op="w4", rows=256, n=3584, k=18944, dtype="bf16"),
        # ---- attention
        # one sequence, 1.5B shape, at the end of a run of 16 steps
        dict(name="attn_1p5b_b1", op="attention", batch=1, heads=12, kv_heads=2, hd=128, kv_lo=1279, kv_hi=1279, q_lo=1, q_hi=1, dtype="bf16", scored=False),
        # 64 ragged sequences of the 7B shape; the weights are accumulated for eviction
        dict(name="attn_7b_b64_scored", op="attention", batch=64, heads=28, kv_heads=4, hd=128, kv_lo=128, kv_hi=5120, q_lo=1, q_hi=1, dtype="bf16", scored=True),
        # steps of up to 128 tokens of 16 sequences through the 72B shape (catch-up and scoring passes), fp32 activations
        dict(name="attn_72b_b16_steps_f32", op="attention", batch=16, heads=64, kv_heads=8, hd=128, kv_lo=512, kv_hi=2560, q_lo=17, q_hi=128, dtype="f32", scored=False),
        # the long-context configuration: 256 sequences, up to 8192 tokens
        dict(name="attn_7b_b256_8k", op="attention", batch=256, heads=28, kv_heads=4, hd=128, kv_lo=4096, kv_hi=8192, q_lo=1, q_hi=1, dtype="bf16", scored=False),
        # ---- writing and reading entries
        # one new token of 64 sequences
        dict(name="append_7b_b64", op="append", batch=64, kv_heads=4, hd=128, tok_lo=1, tok_hi=1, dtype="bf16"),
        # prompts of 16 sequences, fp32
        dict(name="append_72b_prompts_f32", op="append", batch=16, kv_heads=8, hd=128, tok_lo=480, tok_hi=512, dtype="f32"),
        # ---- eviction
        # one sequence falls back to a budget of 1024 after a step
        dict(name="evict_1p5b_b1", op="evict", batch=1, kv_heads=2, hd=128, kv_lo=1152, kv_hi=1152, budget=1024, recent=128),
        # 64 ragged sequences fall back to 2048 entries
        dict(name="evict_7b_b64", op="evict", batch=64, kv_heads=4, hd=128, kv_lo=128, kv_hi=5120, budget=2048, recent=128),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    op = rng.choice(["w4", "attention", "append", "evict"])
    if op == "w4":
        wide = [(1536, 2048), (1536, 1536), (1536, 17920), (8960, 1536), (3584, 4608), (3584, 3584), (3584, 37888), (18944, 3584),
                (8192, 10240), (8192, 8192), (29568, 8192), (1536, 151936), (128, 1024), (256, 1024)]
        k, n = rng.choice(wide) if rng.random() < 0.6 else (_spread(rng, 33, 12000), _spread(rng, 17, 20000))
        rows = _spread(rng, 1, 256)
        while rows > 1 and (rows * n * k > 256 * 3584 * 18944 or rows * n > 4 * 10 ** 7):
            rows //= 2
        return dict(op=op, rows=rows, n=n, k=k, dtype=rng.choice(["bf16", "f32"]))
    heads, kv_heads, hd = rng.choice([(12, 2, 128), (28, 4, 128), (64, 8, 128), (4, 2, 32), (8, 2, 32), (16, 16, 64), (9, 3, 64), (20, 1, 128)])
    if op == "attention":
        batch = _spread(rng, 1, 256)
        hi = _spread(rng, 1, 8192)
        q = 1 if rng.random() < 0.5 else _spread(rng, 2, 128)
        while batch > 1 and (batch * hi * kv_heads * hd > 128 * 6144 * 4 * 128 or batch * q * heads * hi > 16 * 128 * 64 * 1280):
            batch //= 2
        return dict(op=op, batch=batch, heads=heads, kv_heads=kv_heads, hd=hd, kv_lo=rng.choice([hi, max(1, hi // 8)]), kv_hi=hi,
                    q_lo=max(1, q // 4), q_hi=q, dtype=rng.choice(["bf16", "f32"]), scored=rng.random() < 0.5)
    if op == "append":
        hi = 1 if rng.random() < 0.4 else _spread(rng, 2, 1024)
        batch = max(1, min(_spread(rng, 1, 256), 8192 // hi))
        return dict(op=op, batch=batch, kv_heads=kv_heads, hd=hd, tok_lo=max(1, hi // 2), tok_hi=hi, dtype=rng.choice(["bf16", "f32"]))
    hi = _spread(rng, 24, 8192)
    batch = max(1, min(_spread(rng, 1, 128), 64 * 2624 * 4 * 128 // (hi * kv_heads * hd)))
    budget = max(1, round(hi * rng.uniform(0.3, 0.95)))
    return dict(op=op, batch=batch, kv_heads=kv_heads, hd=hd, kv_lo=max(1, hi // 4), kv_hi=hi, budget=budget, recent=rng.choice([0, 1, min(64, budget)]))


# ---------------------------------------------------------------- the format, in elementary operations

def _quantize(x):
    """[..., 32 g] numbers -> codes 0..15 of the same shape and scale bytes [..., g]."""
    x = x.float()
    x = x.reshape(*x.shape[:-1], -1, 32)
    amax = x.abs().amax(-1)
    fine = torch.isfinite(x).all(-1)
    s = ((torch.where(fine, amax, torch.zeros_like(amax)).view(torch.int32) + 0x1FFFFF) >> 23).sub(2).clamp(2, 252)
    v = torch.where(fine[..., None], x * ((254 - s) << 23).view(torch.float32)[..., None], torch.zeros_like(x))
    m = v.abs()
    code = (m > 0.25).to(torch.uint8)
    above = (m >= 0.75, m > 1.25, m >= 1.75, m > 2.5, m >= 3.5, m > 5.0)
    code = code + above[0] + above[1] + above[2] + above[3] + above[4] + above[5]
    code = code + 8 * (torch.signbit(v) & fine[..., None]).to(torch.uint8)
    return code.flatten(-2), torch.where(fine, s, torch.full_like(s, 255)).to(torch.uint8)


def _pairs(device):
    """[256][2]: the two values of a byte."""
    g = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float32, device=device)
    return torch.stack([g.repeat(16), g.repeat_interleave(16)], -1)


def _scale(s):
    """Scale bytes -> 32-bit scales."""
    v = torch.where(s == 0, 0x400000, s.to(torch.int32) << 23)
    return torch.where(s == 255, 0x7FC00000, v).view(torch.float32)


def _w4_tiles(codes, scales, n, k):
    """Codes [n][k], scale bytes [n][k/32] -> the tiled layout."""
    nt, kt, ks = -(-n // 16), -(-k // 128), -(-k // 512)
    c = codes.new_zeros(nt * 16, kt * 128)
    c[:n, :codes.shape[1]] = codes
    c = (c[:, 0::2] | (c[:, 1::2] << 4)).view(nt, 16, kt, 4, 16).permute(0, 2, 3, 1, 4).contiguous()
    s = scales.new_full((nt * 16, ks * 16), 2)
    s[:n, :scales.shape[1]] = scales
    return c, s.view(nt, 16, ks, 4, 4).permute(0, 2, 4, 1, 3).contiguous()


def _views(pool, hd):
    """The four parts of every (page, kv head): key codes, value codes, key scales, value scales."""
    g = hd // 32
    return (pool[..., :8 * hd].unflatten(-1, (4, 16, hd // 8)), pool[..., 8 * hd:16 * hd].unflatten(-1, (4, 16, g, 4)),
            pool[..., 16 * hd:16 * hd + 16 * g].unflatten(-1, (g, 16)), pool[..., 16 * hd + 16 * g:].unflatten(-1, (4, g, 4)))


def _entry_bytes(codes, scales):
    """Codes [..., hd] and scale bytes [..., hd/32] of keys or values -> key bytes [..., 4, hd/8], value bytes [..., dim%16, group]."""
    kb = (codes[..., 0::2] | (codes[..., 1::2] << 4)).unflatten(-1, (4, -1))
    v = codes.unflatten(-1, (-1, 2, 16))
    vb = (v[..., 0, :] | (v[..., 1, :] << 4)).transpose(-1, -2)
    return kb, vb


def _write(pool, table, hd, seq, slot, k, v):
    """Entries k, v [rows][kv heads][hd] into slot[i] of sequence seq[i]."""
    page, t = table[seq, slot // PAGE].long(), slot % PAGE
    pk, pv, sk, sv = _views(pool, hd)
    (ck, ek), (cv, ev) = _quantize(k), _quantize(v)
    pk[page, :, :, t] = _entry_bytes(ck, ek)[0]
    pv[page, :, t // 4, :, :, t % 4] = _entry_bytes(cv, ev)[1]
    sk[page, :, :, t] = ek
    sv[page, :, t // 4, :, t % 4] = ev


def _values(pages, hd):
    """Pages [..., kv heads, hd * 17] -> keys and values [..., kv heads, 16, hd] in 32 bits."""
    pk, pv, sk, sv = _views(pages, hd)
    pairs = _pairs(pages.device)
    g = hd // 32
    k = pairs[pk.long()].movedim(-4, -3).flatten(-3).unflatten(-1, (g, 32)) * _scale(sk).transpose(-1, -2)[..., None]
    v = pairs[pv.long()]                                                   # [..., t/4, m, g, t%4, half]
    d = v.dim()
    v = v.permute(*range(d - 5), d - 5, d - 2, d - 3, d - 1, d - 4)        # [..., t/4, t%4, g, half, m]
    v = v.flatten(-2) * _scale(sv).transpose(-1, -2)[..., None]
    return k.flatten(-2), v.flatten(-2).flatten(-3, -2)


# ---------------------------------------------------------------- inputs

def _cache(gen, lens, slots, hd, kv_heads, device="cuda"):
    """A pool with a quarter of spare pages in random order, every byte of it arbitrary where nothing was written."""
    batch = len(lens)
    max_pages = -(-max(slots) // PAGE)
    need = [-(-s // PAGE) for s in slots]
    total = sum(need) + max(1, sum(need) // 4)
    pool = torch.randint(0, 256, (total, kv_heads, 17 * hd), generator=gen, device=device, dtype=torch.uint8)
    order = torch.randperm(total, generator=gen, device=device).to(torch.int32)
    table = torch.full((batch, max_pages), -1, dtype=torch.int32, device=device)
    own_pages = torch.arange(max_pages, device=device)[None] < torch.tensor(need, device=device)[:, None]
    table[own_pages] = order[:sum(need)]
    return SimpleNamespace(pool=pool, table=table, kv_len=torch.tensor(lens, dtype=torch.int32, device=device))


def _fill(gen, c, slots, hd, kv_heads):
    """Keys with a few strong channels, values of unit size, written page by page (a cache as prefill leaves it)."""
    dev = c.pool.device
    channel = torch.exp(0.5 * torch.randn(kv_heads, hd, generator=gen, device=dev))
    pages = c.table[c.table >= 0].long()
    pk, pv, sk, sv = _views(c.pool, hd)
    for at in range(0, pages.numel(), 8192):
        p = pages[at:at + 8192]
        k = torch.randn(p.numel(), kv_heads, PAGE, hd, generator=gen, device=dev) * channel[None, :, None]
        v = torch.randn(p.numel(), kv_heads, PAGE, hd, generator=gen, device=dev)
        (ck, ek), (cv, ev) = _quantize(k), _quantize(v)
        kb, vb = _entry_bytes(ck, ek)[0], _entry_bytes(cv, ev)[1]
        pk[p] = kb.movedim(2, 3)                                           # [p, h, 4, 16, hd/8]
        pv[p] = vb.unflatten(2, (4, 4)).permute(0, 1, 2, 4, 5, 3)          # [p, h, t/4, m, g, t%4]
        sk[p] = ek.movedim(2, 3)
        sv[p] = ev.unflatten(2, (4, 4)).movedim(3, 4)
    # what lies behind the last entry of a sequence is arbitrary
    last = c.table.gather(1, ((c.kv_len.long() - 1).clamp(min=0) // PAGE)[:, None])[:, 0].long()
    junk = torch.randint(0, 256, (len(last), kv_heads, 17 * hd), generator=gen, device=dev, dtype=torch.uint8)
    free = torch.arange(PAGE, device=dev)[None] > ((c.kv_len.long() - 1) % PAGE)[:, None]
    for view, rubbish, axis in zip(_views(c.pool, hd), _views(junk, hd), (1, 2, 3, 4)):
        mask = {1: free[:, None, None, :, None], 2: free.view(-1, 1, 4, 1, 1, 4), 3: free[:, None, None, :], 4: free.view(-1, 1, 4, 1, 4)}[axis]
        view[last] = torch.where(mask, rubbish, view[last])


def _ragged(lo, hi, count, odd):
    """Lengths of a batch: the same multiset for every seed (the inputs' order and values come from the seed)."""
    v = np.random.RandomState((lo * 31 + hi * 7 + count) * 4 + odd).randint(lo, hi + 1, count)
    v[0] = hi
    return v


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rs = np.random.RandomState(seed % (1 << 31))
    s = SimpleNamespace(op=case["op"])
    rand = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")  # noqa: E731
    if s.op == "w4":
        n, k = case["n"], case["k"]
        codes, scales = [], []
        for at in range(0, n, 16384):
            w = torch.zeros(min(16384, n - at), -(-k // 32) * 32, device="cuda")
            w[:, :k] = 0.02 * rand(w.shape[0], k)
            c, e = _quantize(w)
            codes.append(c)
            scales.append(e)
        s.codes, s.scales = _w4_tiles(torch.cat(codes), torch.cat(scales), n, k)
        s.n, s.k = n, k
        s.x = (rand(case["rows"], k) * torch.exp(0.5 * rand(1, k))).to(TYPES[case["dtype"]])
        return s
    s.hd, s.kv_heads = case["hd"], case["kv_heads"]
    if s.op == "append":
        count = [int(x) for x in rs.permutation(_ragged(case["tok_lo"], case["tok_hi"], case["batch"], 0))]
        at = [64 + case["tok_hi"] - c - int(x) for c, x in zip(count, rs.permutation(len(count)) % 64)]
        slots = [a + c for a, c in zip(at, count)]
        c = _cache(gen, at, slots, s.hd, s.kv_heads)
        rows = sum(count)
        s.seq = torch.tensor(np.repeat(np.arange(len(count)), count), dtype=torch.int32, device="cuda")
        s.slot = torch.tensor(np.concatenate([np.arange(a, b) for a, b in zip(at, slots)]), dtype=torch.int32, device="cuda")
        s.position = s.slot + 1000
        heads = 7 * s.kv_heads
        # keys and values as a fused projection leaves them: columns behind the queries'
        qkv = rand(rows, heads + 2 * s.kv_heads, s.hd)
        qkv[:, heads:heads + s.kv_heads] *= torch.exp(0.5 * rand(s.kv_heads, s.hd))
        s.qkv = qkv.to(TYPES[case["dtype"]])
        s.k, s.v = s.qkv[:, heads:heads + s.kv_heads], s.qkv[:, heads + s.kv_heads:]
    else:
        order = rs.permutation(case["batch"])
        lens = [int(x) for x in _ragged(case["kv_lo"], case["kv_hi"], case["batch"], 0)[order]]
        c = _cache(gen, lens, lens, s.hd, s.kv_heads)
        _fill(gen, c, lens, s.hd, s.kv_heads)
    s.pool, s.table, s.kv_len = c.pool, c.table, c.kv_len
    cap = c.table.shape[1] * PAGE
    s.score = torch.rand(case["batch"], s.kv_heads, cap, generator=gen, device="cuda") ** 4 * 8
    if s.op == "attention":
        rows = [min(int(r), n) for r, n in zip(_ragged(case["q_lo"], case["q_hi"], case["batch"], 1)[order], lens)]
        s.max_rows, s.max_kv = max(rows), max(lens)
        s.row_start = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
        s.q = (1.5 * rand(sum(rows), case["heads"], s.hd)).to(TYPES[case["dtype"]])
        s.factor = 1.0 / math.sqrt(s.hd)
        s.scored = case["scored"]
    else:
        s.pos = torch.argsort(torch.rand(case["batch"], s.kv_heads, cap, generator=gen, device="cuda"), -1).to(torch.int32)
    if s.op == "evict":
        # few different scores among the smallest: ties decide
        s.score = torch.where(s.score < 0.25, torch.zeros_like(s.score), s.score)
        s.budget, s.recent = case["budget"], case["recent"]
    return s


# ---------------------------------------------------------------- one pass

def run(s):
    if own:
        return _run_own(s)
    return {"w4": _plain_w4, "append": _plain_append, "attention": _plain_attention, "evict": _plain_evict}[s.op](s)


def _run_own(s):
    from paper_2501_19324_amd import binding as R

    if s.op == "w4":
        return R.rsd_w4_linear(s.x, (s.codes, s.scales, s.n, s.k))
    cache = (s.pool, s.table, s.kv_len)
    if s.op == "append":
        R.rsd_kv4_append(cache, s.k, s.v, s.seq, s.slot, position=s.position, entry_pos=s.pos, scores=s.score)
        k, v = R.rsd_kv4_read(cache, s.seq, s.slot, s.hd)
        return {"k": k, "v": v, "pos": s.pos, "score": s.score}
    if s.op == "attention":
        score = s.score.clone() if s.scored else None
        out, lse = R.rsd_kv4_attention(cache, s.q, s.factor, row_start=s.row_start, max_rows=s.max_rows, max_kv=s.max_kv, scores=score, want_lse=True)
        return {"out": out, "lse": lse, "score": score}
    score, pos, kv_len = s.score.clone(), s.pos.clone(), s.kv_len.clone()
    R.rsd_kv4_evict((s.pool, s.table, kv_len), score, pos, s.budget, s.recent)
    return {"pool": s.pool, "score": score, "pos": pos, "kv_len": kv_len}


def _plain_w4(s):
    w = _pairs(s.x.device)[s.codes.long()]                                 # [n/16, k/128, group, row, byte, half]
    nt, kt = s.codes.shape[:2]
    e = _scale(s.scales).permute(0, 1, 4, 2, 3).reshape(nt, -1, 4, 16)[:, :kt]
    w = (w.flatten(-2) * e[..., None]).permute(0, 3, 1, 2, 4).reshape(nt * 16, kt * 128)[:s.n, :s.k]
    return (s.x.float() @ w.T).to(s.x.dtype)


def _plain_append(s):
    seq, slot = s.seq.long(), s.slot.long()
    _write(s.pool, s.table, s.hd, seq, slot, s.k, s.v)
    s.pos[seq, :, slot] = s.position[:, None].expand(-1, s.kv_heads)
    s.score[seq, :, slot] = 0.0
    k, v = _values(s.pool[s.table[seq, slot // PAGE].long()], s.hd)
    at = torch.arange(len(slot), device=slot.device)
    return {"k": k[at, :, slot % PAGE].to(torch.bfloat16), "v": v[at, :, slot % PAGE].to(torch.bfloat16), "pos": s.pos, "score": s.score}


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
    limit = s.kv_len.long()[:, None] - (count[:, None] - 1 - r[None])
    seen = (slot[None, None] < limit[:, :, None]) & used[:, :, None]       # [b, row, slot]
    logit = (q @ k.transpose(-1, -2) * s.factor).unflatten(2, (s.max_rows, group))
    logit = torch.where(seen[:, None, :, None], logit, -math.inf)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = torch.exp(logit - top)
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + top
    p = torch.where(total > 0, p / total, torch.zeros_like(p))
    out = (p.flatten(2, 3) @ v).unflatten(2, (s.max_rows, group))          # [b, kv head, row, g, hd]
    line = torch.arange(rows, device=dev)
    b = (line[:, None] >= s.row_start[None, 1:]).sum(-1)
    i = line - s.row_start[b]
    out = out.permute(0, 2, 1, 3, 4)[b, i].flatten(1, 2)
    lse = lse[..., 0].permute(0, 2, 1, 3)[b, i].flatten(1, 2)
    return {"out": out.to(s.q.dtype), "lse": lse, "score": s.score + _padded(p.sum((2, 3)), s.score.shape[-1]) if s.scored else None}


def _padded(x, width):
    return torch.cat([x, x.new_zeros(*x.shape[:-1], width - x.shape[-1])], -1) if width > x.shape[-1] else x


def _plain_evict(s):
    dev, cap = s.pool.device, s.score.shape[-1]
    slot = torch.arange(cap, device=dev)
    n = s.kv_len.long()[:, None, None]
    there = slot < n
    newest = torch.where(there, s.pos, torch.full_like(s.pos, -1)).amax(-1, keepdim=True)
    safe = there & (s.pos > newest - s.recent)
    value = torch.where(there, torch.where(torch.isnan(s.score), -math.inf, s.score + 0.0), -math.inf)
    order = torch.sort(value, dim=-1, descending=True, stable=True).indices
    tier = torch.where(safe, 2, there.to(torch.int64)).gather(-1, order)
    order = order.gather(-1, torch.sort(tier, dim=-1, descending=True, stable=True).indices)
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order).contiguous())
    keep = there & ((rank < s.budget) | (n <= s.budget))
    hole = (slot < s.budget) & (slot < n) & ~keep
    extra = (slot >= s.budget) & keep & (n > s.budget)
    source = torch.zeros_like(order)
    source = source.scatter_add(-1, torch.where(extra, extra.cumsum(-1) - 1, cap - 1), torch.where(extra, slot.expand_as(order), torch.zeros_like(order)))
    b, h, to = hole.nonzero(as_tuple=True)
    fr = source[b, h, (hole.cumsum(-1) - 1)[b, h, to]]
    p1, p0, t1, t0 = s.table[b, fr // PAGE].long(), s.table[b, to // PAGE].long(), fr % PAGE, to % PAGE
    pk, pv, sk, sv = _views(s.pool, s.hd)
    pk[p0, h, :, t0] = pk[p1, h, :, t1]
    pv[p0, h, t0 // 4, :, :, t0 % 4] = pv[p1, h, t1 // 4, :, :, t1 % 4]
    sk[p0, h, :, t0] = sk[p1, h, :, t1]
    sv[p0, h, t0 // 4, :, t0 % 4] = sv[p1, h, t1 // 4, :, t1 % 4]
    score, pos = s.score.clone(), s.pos.clone()
    score[b, h, to], pos[b, h, to] = s.score[b, h, fr], s.pos[b, h, fr]
    return {"pool": s.pool, "score": score, "pos": pos, "kv_len": s.kv_len.clamp(max=s.budget)}


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 4 if case.get("dtype") == "f32" else 2
    if case["op"] == "w4":
        r, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": n * k * 17 // 32 + r * (n + k) * size, "flops": 2 * r * n * k}
    entry = case["hd"] * 17 // 16 * case["kv_heads"]
    if case["op"] == "append":
        rows = case["batch"] * (case["tok_lo"] + case["tok_hi"]) // 2
        return {"bytes": rows * (2 * case["kv_heads"] * case["hd"] * (size + 2) + 2 * entry + 8 * case["kv_heads"] + 12), "flops": rows * 8 * case["kv_heads"] * case["hd"]}
    mean = (case["kv_lo"] + case["kv_hi"]) / 2
    if case["op"] == "attention":
        q = min((case["q_lo"] + case["q_hi"]) / 2, mean)
        b, io = case["batch"], 2 * case["heads"] * case["hd"] * size
        return {"bytes": int(b * (mean * (entry + (8 * case["kv_heads"] if case["scored"] else 0)) + q * io)),
                "flops": int(b * q * (mean - q / 2 + 0.5) * 4 * case["heads"] * case["hd"])}
    # entries seen: score and position; entries moved: an equal share of those above the budget is kept
    over = max(0.0, min(1.0, (case["kv_hi"] - case["budget"]) / max(1, case["kv_hi"] - case["kv_lo"] + 1)))
    above = (case["kv_hi"] - case["budget"]) / 2 if case["kv_hi"] > case["kv_lo"] else case["kv_hi"] - case["budget"]
    above = max(0.0, above)
    long = (case["budget"] + above) if over > 0 else mean
    moved = above * case["budget"] / max(1.0, case["budget"] + above)
    seen = case["batch"] * case["kv_heads"] * over * long
    return {"bytes": int(8 * seen + case["batch"] * case["kv_heads"] * over * moved * 2 * (entry // case["kv_heads"] + 8)) + 8 * case["batch"], "flops": int(seen)}


# ---------------------------------------------------------------- the definitions in 64 bits

def _number(code):
    """A 4-bit code's value from its fields: sign, two exponent bits, one fraction bit."""
    code = code.to(torch.int64)
    e, f = (code >> 1) & 3, (code & 1).double()
    v = torch.where(e == 0, 0.5 * f, (1 + 0.5 * f) * torch.pow(2.0, (e - 1).double()))
    return torch.where(code >= 8, -v, v)


def _power(byte):
    return torch.where(byte == 255, math.nan, torch.pow(2.0, byte.double() - 127.0))


def _entries(pool, table_row, n, hd):
    """The first n entries of one sequence: keys and values [kv head][n][hd] in 64 bits."""
    g, heads = hd // 32, pool.shape[1]
    raw = pool[table_row[:-(-n // PAGE)].long()]                           # [pages, head, bytes]
    t = torch.arange(n, device=pool.device)
    d = torch.arange(hd, device=pool.device)
    line = raw.transpose(0, 1).reshape(heads, -1)                          # bytes of a head, page after page
    base = (t // PAGE * 17 * hd)[:, None]
    i = (t % PAGE)[:, None]
    quarter = hd // 4
    key = line[:, base + (d // quarter) * 2 * hd + i * (hd // 8) + d % quarter // 2]
    key = torch.where(d % 2 == 0, key & 15, key >> 4)
    key_scale = line[:, base + 16 * hd + (d // 32) * 16 + i]
    val = line[:, base + 8 * hd + (i // 4) * 2 * hd + (d % 16) * (hd // 8) + (d // 32) * 4 + i % 4]
    val = torch.where(d % 32 < 16, val & 15, val >> 4)
    val_scale = line[:, base + 16 * hd + 16 * g + (i // 4) * 4 * g + (d // 32) * 4 + i % 4]
    return _number(key) * _power(key_scale), _number(val) * _power(val_scale)


def _nearest(x):
    """Numbers -> what 4 bits hold of them, in 64 bits."""
    x = x.double().unflatten(-1, (-1, 32))
    frac, exp = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(frac <= 0.875, exp - 3, exp - 2).clamp(-125, 125).double()
    e = torch.where(frac == 0, -125.0, e)
    m = x.abs() / torch.pow(2.0, e)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    best = torch.full_like(m, math.inf)
    pick = torch.zeros_like(m)
    for j in (0, 2, 4, 6, 1, 3, 5, 7):                                     # even codes first: they win ties
        d = (m - grid[j]).abs()
        pick = torch.where(d < best, grid[j], pick)
        best = torch.minimum(best, d)
    return (torch.sign(x) * pick * torch.pow(2.0, e)).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    if s.op == "w4":
        x, parts = s.x.double(), []
        for at in range(0, s.codes.shape[0], 512):
            c, e = s.codes[at:at + 512], s.scales[at:at + 512]
            tiles, kt = c.shape[:2]
            both = torch.stack([_number(c & 15), _number(c >> 4)], -1).reshape(tiles, kt, 4, 16, 32)
            power = _power(e)                                              # [tile, k/512, group, row, k/128 % 4]
            power = torch.movedim(power, 4, 2).reshape(tiles, -1, 4, 16)[:, :kt]
            w = torch.einsum("tkgrb,tkgr->trkgb", both, power).reshape(tiles * 16, -1)
            parts.append(x @ w[:, :s.k].T.contiguous())
        return torch.cat(parts, 1)[:, :s.n]
    if s.op == "append":
        score = s.score.double()
        score[s.seq.long(), :, s.slot.long()] = 0.0
        return {"k": _nearest(s.k.float()), "v": _nearest(s.v.float()), "pos": None, "score": score}
    if s.op == "attention":
        outs, lses, score = [], [], s.score.double() if s.scored else None
        start = s.row_start.tolist()
        for b, n in enumerate(s.kv_len.tolist()):
            q = s.q[start[b]:start[b + 1]].double()
            rows, heads, hd = q.shape
            k, v = _entries(s.pool, s.table[b], n, hd)
            z = torch.matmul(q.reshape(rows, s.kv_heads, -1, hd).permute(1, 2, 0, 3).reshape(s.kv_heads, -1, hd), k.transpose(1, 2).contiguous()) * s.factor
            z = z.view(s.kv_heads, -1, rows, n)
            hidden = torch.arange(n, device=z.device)[None] >= n - (rows - 1 - torch.arange(rows, device=z.device))[:, None]
            z = z.masked_fill(hidden, -math.inf)
            lse = torch.logsumexp(z, -1)
            p = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
            o = torch.matmul(p.flatten(1, 2), v).view(s.kv_heads, -1, rows, hd)
            outs.append(o.permute(2, 0, 1, 3).reshape(rows, heads, hd))
            lses.append(lse.permute(2, 0, 1).reshape(rows, heads))
            if s.scored:
                score[b, :, :n] += p.sum((1, 2))
        return {"out": torch.cat(outs), "lse": torch.cat(lses), "score": score}
    score, pos = s.score.cpu().numpy().copy(), s.pos.cpu().numpy().copy()
    lens = s.kv_len.cpu().numpy()
    for b, n in enumerate(lens):
        for h in range(s.kv_heads if n > s.budget else 0):
            value, where = score[b, h, :n].astype(np.float64), pos[b, h, :n]
            safe = where > where.max() - s.recent
            kept = np.sort(np.lexsort((np.arange(n), -value, ~safe))[:s.budget])
            stays = np.zeros(n, bool)
            stays[kept] = True
            to, fr = np.flatnonzero(~stays[:s.budget]), kept[kept >= s.budget]
            score[b, h, to], pos[b, h, to] = score[b, h, fr], pos[b, h, fr]
    return {"pool": None, "score": score.astype(np.float64), "pos": pos, "kv_len": np.minimum(lens, s.budget)}

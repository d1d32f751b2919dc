"""The key-value cache operators in numbers: what is measured, in a plain form and through the library.

Four operators work on one cache.  A cache holds, for each sequence, full blocks of tokens in 8 bits (one page of the
pool per block, one scale per block, head and K or V) and its last, unfinished block in 16 bits:

  rotary     turns pairs of channels of q or k by an angle that grows with the position; its gradient turns them back
  append     stores new tokens' K (turned) and V, and quantises every block that they complete
  attention  softmax(q K^T) V over the cache, for one new token per sequence or many, optionally with the attention
             weight that each block received
  evict      drops the blocks with the least accumulated weight and closes the gaps in the page table

``run`` computes an operator in elementary torch operations where ``own`` is false, and through
``paper_2410_15240_b200.kv`` where it is true.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
TOP = {"int8": 127.0, "e4m3": 448.0}
TINY = 2.0 ** -100          # blocks whose largest magnitude is below this are held as zeros


# ------------------------------------------------------------------------------------------------ cases ----

def listed():
    return [
        # one user's short chat, one token at a time: latency
        dict(name="attend_one_short", op="attention", dtype="bf16", fmt="int8", seqs=1, new=1, len_min=700, len_max=700, q_heads=32, kv_heads=8,
             dim=128, block=64, window=0, mass=False),
        # a serving batch of unequal lengths, with the weights that eviction goes by
        dict(name="attend_batch_ragged", op="attention", dtype="bf16", fmt="e4m3", seqs=61, new=1, len_min=130, len_max=4096, q_heads=32, kv_heads=8,
             dim=128, block=64, window=0, mass=True),
        # few sequences with very long contexts: one axis to split
        dict(name="attend_long", op="attention", dtype="f16", fmt="int8", seqs=4, new=1, len_min=70001, len_max=131072, q_heads=64, kv_heads=8,
             dim=128, block=64, window=0, mass=True),
        # a few drafted tokens checked at once, every head with its own K and V, a sliding window, small blocks
        dict(name="attend_drafts_window", op="attention", dtype="f16", fmt="e4m3", seqs=23, new=5, len_min=3, len_max=2777, q_heads=16, kv_heads=16,
             dim=64, block=16, window=1000, mass=False),
        # a long prompt taken in pieces: many new tokens against what is cached already
        dict(name="attend_prompt_piece", op="attention", dtype="bf16", fmt="e4m3", seqs=3, new=1024, len_min=1500, len_max=6100, q_heads=32, kv_heads=8,
             dim=128, block=64, window=0, mass=True),
        # one new token for each sequence of a batch
        dict(name="append_one_each", op="append", dtype="bf16", fmt="e4m3", seqs=64, new=1, len_min=130, len_max=2048, q_heads=32, kv_heads=8,
             dim=128, block=64, rotary="half", rotary_dim=128, read=False),
        # prompts that start a cache or lengthen it
        dict(name="append_prompts", op="append", dtype="bf16", fmt="e4m3", seqs=7, new=2500, len_min=2500, len_max=9001, q_heads=32, kv_heads=8,
             dim=128, block=64, rotary="half", rotary_dim=128, read=False),
        # the same with part of the head turned, 8-bit integers, and the values read back out of the cache
        dict(name="append_read_partial", op="append", dtype="f16", fmt="int8", seqs=5, new=333, len_min=333, len_max=1100, q_heads=12, kv_heads=4,
             dim=96, block=32, rotary="interleaved", rotary_dim=48, read=True),
        # a batch at its budget: every sequence gives up what it attends to least
        dict(name="evict_batch", op="evict", seqs=16, blocks=150, kv_heads=8, budget=128, first=1, last=4, block=64),
        # many long contexts cut to a fraction
        dict(name="evict_long", op="evict", seqs=64, blocks=4001, kv_heads=8, budget=1024, first=4, last=16, block=32),
        # q of a decoding batch, partly turned, far into a lengthened context
        dict(name="rotary_few", op="rotary", dtype="f16", tokens=48, heads=32, dim=128, rotary="interleaved", rotary_dim=64, factor=16.0,
             positions=131072, inverse=False),
        # the gradient of q in a training step
        dict(name="rotary_gradient", op="rotary", dtype="bf16", tokens=32768, heads=32, dim=128, rotary="half", rotary_dim=128, factor=1.0,
             positions=8192, inverse=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "append", "append", "evict", "rotary"])
    dtype, fmt = rng.choice(["bf16", "f16"]), rng.choice(["int8", "e4m3"])
    block = rng.choice([16, 32, 64, 128])
    dim = rng.choice([64, 96, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    group = rng.choice([1, 3, 4, 7, 8])
    if op == "attention":
        new = rng.choice([1, 1, rng.randint(2, 12), _spread(rng, 16, 1024)])
        rows = new * kv_heads * group
        len_max = _spread(rng, max(new, 40), 65000)
        # K and V of at most 3e8 values (the listed cases' largest: 9e8), and no more scores than the listed cases have
        most = min(3e8 / (len_max * kv_heads * dim), 5e8 / (len_max * rows))
        if most < 1:
            len_max = max(new, int(len_max * most))
            most = 1
        seqs = rng.randint(1, max(1, min(96, int(most))))
        return dict(op=op, dtype=dtype, fmt=fmt, seqs=seqs, new=new, len_min=rng.randint(new, len_max), len_max=len_max, q_heads=kv_heads * group,
                    kv_heads=kv_heads, dim=dim, block=block, window=rng.choice([0, 0, 0, rng.randint(1, len_max)]), mass=rng.random() < 0.5)
    if op == "append":
        new = rng.choice([1, _spread(rng, 2, 4000)])
        len_max = rng.randint(new, new + 4000)
        seqs = rng.randint(1, max(1, min(128, 16000 // new)))
        layout = rng.choice(["half", "interleaved"])
        return dict(op=op, dtype=dtype, fmt=fmt, seqs=seqs, new=new, len_min=rng.randint(new, len_max), len_max=len_max, q_heads=kv_heads * group,
                    kv_heads=kv_heads, dim=dim, block=block, rotary=layout, rotary_dim=rng.choice([dim, dim // 2]), read=fmt == "int8")
    if op == "evict":
        blocks = _spread(rng, 9, 4000)
        budget = rng.randint(max(1, blocks // 5), blocks)
        return dict(op=op, seqs=rng.randint(1, 64), blocks=blocks, kv_heads=kv_heads, budget=budget, first=rng.randint(0, 4), last=rng.randint(0, 8),
                    block=block)
    return dict(op=op, dtype=dtype, tokens=_spread(rng, 1, 30000), heads=rng.choice([1, 5, 8, 32]), dim=dim, rotary=rng.choice(["half", "interleaved"]),
                rotary_dim=rng.choice([dim, dim // 2]), factor=rng.choice([1.0, 4.0, 16.0]), positions=_spread(rng, 100, 200000),
                inverse=rng.random() < 0.5)


def _lens(c):
    """Tokens held by each sequence after the call: from len_min to len_max, unequal, the same for every seed."""
    n = c["seqs"]
    return [c["len_max"] if i == 0 else c["len_min"] + int((c["len_max"] - c["len_min"]) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _news(c):
    """New tokens of each sequence: the full number for the first, fewer for some others, never none."""
    return [c["new"] if i % 3 == 0 else max(1, c["new"] - (i * 7) % max(1, c["new"] // 2)) for i in range(c["seqs"])]


def work(c):
    if c["op"] == "rotary":
        n = c["tokens"] * c["heads"] * c["dim"]
        return {"bytes": 2 * 2 * n + 8 * c["tokens"], "flops": 3 * c["tokens"] * c["heads"] * c["rotary_dim"]}
    if c["op"] == "evict":
        entries = c["seqs"] * (c["blocks"] + 1)
        return {"bytes": entries * (2 * 4 * c["kv_heads"] + 2 * 4) + c["seqs"] * 4 * (3 + max(0, c["blocks"] - c["budget"])),
                "flops": entries * c["kv_heads"]}
    lens, news = _lens(c), _news(c)
    d, kh, qh, bt = c["dim"], c["kv_heads"], c["q_heads"], c["block"]
    if c["op"] == "append":
        new = sum(news)
        done = sum(L // bt - (L - n) // bt for L, n in zip(lens, news))
        tail = sum(min(n, L % bt) for L, n in zip(lens, news)) + sum((L - n) % bt for L, n in zip(lens, news) if L // bt > (L - n) // bt)
        total = 2 * new * kh * d * 2 + 2 * done * bt * kh * d + 8 * done * kh + 2 * tail * kh * d * 2 + 2 * 2 * new * qh * d + 8 * new
        if c["read"]:
            total += 2 * sum(lens) * kh * d + 2 * 2 * c["seqs"] * c["len_max"] * kh * d
        return {"bytes": total, "flops": 3 * new * (qh + kh) * c["rotary_dim"] + 4 * new * kh * d}
    pairs, tokens, tails = 0, 0, 0
    for L, n in zip(lens, news):
        w = c["window"] or L
        seen = [min(L - n + j + 1, w) for j in range(n)]
        pairs += sum(seen)
        span = min(L, w + n - 1)
        tails += min(span, L % bt)
        tokens += span - min(span, L % bt)
    total = 2 * tokens * kh * d + 2 * 2 * tails * kh * d + 2 * 2 * sum(news) * qh * d + 4 * sum(news) * qh
    total += sum(-(-L // bt) for L in lens) * (4 + 8 * kh + (8 * kh if c["mass"] else 0))
    return {"bytes": total, "flops": 4 * pairs * qh * d}


# ------------------------------------------------------------------------------------------------ inputs ----

def _frequencies(rotary_dim, base=10000.0, factor=1.0):
    """Radians per position of each pair; for a context lengthened `factor` times the slow pairs are slowed down by it, the
    fast ones are left, and a ramp over the wavelength joins them."""
    plain = [base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]
    if factor == 1.0:
        return plain, 1.0
    turns = [4096 * f / (2 * math.pi) for f in plain]
    keep = [min(1.0, max(0.0, (t - 1.0) / (32.0 - 1.0))) for t in turns]
    return [f * k + f / factor * (1 - k) for f, k in zip(plain, keep)], 0.1 * math.log(factor) + 1.0


class State:
    pass


def _page(c):
    """Byte offsets inside a page: K codes of all heads, V codes, then (K scale, V scale) per head; padded to 128 bytes."""
    codes = c["kv_heads"] * c["block"] * c["dim"]
    return codes, 2 * codes, -(-(2 * codes + 8 * c["kv_heads"]) // 128) * 128


def _normal(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype)


def prepare(c, seed):
    s, gen = State(), torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s.c = c
    if c["op"] == "evict":
        nb = c["blocks"] + 1
        stride = nb + 3
        lens = [c["blocks"] * c["block"] + 1 + (7 * i) % c["block"] if i % 4 != 1 else max(1, c["blocks"] * c["block"] * (i % 7) // 7) for i in range(c["seqs"])]
        lens = [min(n, nb * c["block"]) for n in lens]
        s.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        s.mass = (2.5 * _normal(gen, c["seqs"], c["kv_heads"], stride)).exp()        # weights: many small, few large
        s.mass[:, :, 3::11] = 0.0                                                     # and blocks that nobody looked at: ties
        s.table = torch.rand(c["seqs"], stride, generator=gen, device=DEV).argsort(1).to(torch.int32) + 5
        s.new_table, s.new_mass, s.new_lens = torch.empty_like(s.table), torch.empty_like(s.mass), torch.empty_like(s.lens)
        s.evicted, s.count = torch.empty_like(s.table), torch.empty_like(s.lens)
        if own:
            from paper_2410_15240_b200 import kv
            s.cache = kv.KvCache(kv.BF16, kv.INT8, c["kv_heads"], c["kv_heads"], 64, c["block"])
            s.call = kv.Eviction(n_seqs=c["seqs"], table_stride=stride, mass_stride=stride, budget=c["budget"], keep_first=c["first"], keep_last=c["last"],
                                 d_table=s.table.data_ptr(), d_lens=s.lens.data_ptr(), d_mass=s.mass.data_ptr(), d_table_out=s.new_table.data_ptr(),
                                 d_lens_out=s.new_lens.data_ptr(), d_mass_out=s.new_mass.data_ptr(), d_evicted=s.evicted.data_ptr(),
                                 d_n_evicted=s.count.data_ptr())
        return s
    t = TYPES[c["dtype"]]
    if c["op"] == "rotary":
        s.freq, s.gain = _frequencies(c["rotary_dim"], factor=c["factor"])
        s.x = _normal(gen, c["tokens"], c["heads"], c["dim"]).to(t)
        s.out = torch.empty_like(s.x)
        s.pos = torch.randint(0, c["positions"], (c["tokens"],), generator=gen, device=DEV)
        _tables(s, c["positions"])
        if own:
            from paper_2410_15240_b200 import kv
            s.cache = kv.KvCache(getattr(kv, c["dtype"].upper()), kv.INT8, c["heads"], 1, c["dim"], 64,
                                 rotary=getattr(kv, "ROTARY_" + c["rotary"].upper()), frequencies=s.freq, rotary_gain=s.gain)
            s.rows_in, s.rows_out = _rows(kv, s.x), _rows(kv, s.out)
        return s

    kh, d, bt = c["kv_heads"], c["dim"], c["block"]
    lens, news = _lens(c), _news(c)
    s.total, s.max_new, s.max_len = sum(news), max(news), max(lens)
    s.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s.news = torch.tensor(news, dtype=torch.int32, device=DEV)
    s.starts = torch.cat([torch.zeros_like(s.news[:1]), s.news.cumsum(0).to(torch.int32)])
    s.blocks = -(-s.max_len // bt)
    full = [n // bt for n in lens]
    s.pages = sum(full) + 3
    table = torch.full((c["seqs"], s.blocks + 1), -1, dtype=torch.int32)
    order = torch.randperm(s.pages, generator=torch.Generator().manual_seed(seed + 1)).to(torch.int32)
    at = 0
    for i, n in enumerate(full):
        table[i, :n] = order[at:at + n]
        at += n
    s.table = table.to(DEV)
    codes, scales, page = _page(c)
    s.pool = torch.zeros(s.pages, page, dtype=torch.uint8, device=DEV)
    s.tail = _normal(gen, c["seqs"], kh, 2, bt, d).to(t)
    s.pos = torch.cat([torch.arange(L - n, L, device=DEV) for L, n in zip(lens, news)])
    s.seq = torch.repeat_interleave(torch.arange(c["seqs"], device=DEV), s.news.long(), output_size=s.total)
    s.slot = torch.arange(s.total, device=DEV) - s.starts[:-1].long()[s.seq]            # which of its sequence's new tokens
    s.q = (2 * _normal(gen, s.total, c["q_heads"], d)).to(t)
    s.q_out = torch.empty_like(s.q)
    if c["op"] == "attention":
        for h in range(2):                                                              # K, then V: normal values as codes
            x = _normal(gen, s.pages, codes, dtype=torch.float16 if codes * s.pages > 1 << 28 else torch.float32)
            x *= TOP[c["fmt"]] / 4
            x.clamp_(-TOP[c["fmt"]], TOP[c["fmt"]])
            s.pool[:, h * codes:(h + 1) * codes] = (x.round_().to(torch.int8) if c["fmt"] == "int8" else x.to(torch.float8_e4m3fn)).view(torch.uint8)
            del x
        spread = (0.25 * _normal(gen, s.pages, kh, 2)).exp() * (4 / TOP[c["fmt"]])
        s.pool[:, scales:scales + 8 * kh] = spread.view(s.pages, 2 * kh).view(torch.uint8)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(s.total, c["q_heads"], device=DEV)
        s.mass = torch.rand(c["seqs"], kh, s.blocks, generator=gen, device=DEV) if c["mass"] else None
        s.new_mass = torch.zeros_like(s.mass) if c["mass"] else None
    else:
        s.freq, s.gain = _frequencies(c["rotary_dim"])
        _tables(s, s.max_len)
        s.qkv = _normal(gen, s.total, c["q_heads"] + 2 * kh, d).to(t)                   # as one projection gives them
        s.q, s.k, s.v = s.qkv.split([c["q_heads"], kh, kh], 1)
        s.kept_tail = s.tail.clone() if c["new"] > 1 else None                          # a second pass needs the tokens that the first replaces
        done = [(i, b) for i, (L, n) in enumerate(zip(lens, news)) for b in range((L - n) // bt, L // bt)]
        s.done = torch.tensor(done, dtype=torch.int64, device=DEV).reshape(-1, 2)       # which blocks get complete
        if c["read"]:
            s.k_read, s.v_read = (torch.empty(c["seqs"], s.max_len, kh, d, dtype=t, device=DEV) for _ in range(2))
    if own:
        from paper_2410_15240_b200 import kv
        rotary = dict(rotary=getattr(kv, "ROTARY_" + c["rotary"].upper()), frequencies=s.freq, rotary_gain=s.gain) if "rotary" in c else {}
        s.cache = kv.KvCache(getattr(kv, c["dtype"].upper()), getattr(kv, c["fmt"].upper()), c["q_heads"], kh, d, bt, **rotary)
        s.batch = kv.Batch(n_seqs=c["seqs"], total_new=s.total, max_new=s.max_new, max_len=s.max_len, pool_pages=s.pages, table_stride=s.table.stride(0),
                           d_pool=s.pool.data_ptr(), d_tail=s.tail.data_ptr(), d_table=s.table.data_ptr(), d_lens=s.lens.data_ptr(),
                           d_starts=s.starts.data_ptr(), d_positions=s.pos.data_ptr())
        s.rq, s.rq_out = _rows(kv, s.q), _rows(kv, s.q_out)
        if c["op"] == "attention":
            s.r_out = _rows(kv, s.out)
            s.workspace = torch.zeros(s.cache.workspace_bytes(s.batch, c["mass"]), dtype=torch.uint8, device=DEV)
        else:
            s.rk, s.rv = _rows(kv, s.k), _rows(kv, s.v)
            if c["read"]:
                s.rk_read, s.rv_read = (_rows(kv, x.view(-1, kh, d)) for x in (s.k_read, s.v_read))
    return s


def _rows(kv, x):
    return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1))


def _tables(s, positions):
    """Cosines and sines of every position, made once in 64 bits and kept in 32."""
    angle = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * torch.tensor(s.freq, device=DEV, dtype=torch.float64)
    s.cos, s.sin = (angle.cos() * s.gain).float(), (angle.sin() * s.gain).float()


# ------------------------------------------------------------------------------------------------ the operators ----

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    c, stream = s.c, torch.cuda.current_stream().cuda_stream
    if c["op"] == "rotary":
        s.cache.rotary(c["tokens"], c["heads"], s.rows_in, s.rows_out, s.pos.data_ptr(), c["inverse"], stream)
        return s.out
    if c["op"] == "evict":
        s.cache.evict(s.call, stream)
        return {"table": s.new_table, "lens": s.new_lens, "mass": s.new_mass, "evicted": s.evicted, "count": s.count}
    if c["op"] == "attention":
        if c["mass"]:
            s.cache.attention(s.batch, s.rq, s.r_out, s.workspace.data_ptr(), s.workspace.numel(), d_lse=s.lse.data_ptr(), window=c["window"],
                              d_mass_in=s.mass.data_ptr(), d_mass_out=s.new_mass.data_ptr(), mass_stride=s.blocks, stream=stream)
            return {"out": s.out, "lse": s.lse, "mass": s.new_mass}
        s.cache.attention(s.batch, s.rq, s.r_out, s.workspace.data_ptr(), s.workspace.numel(), d_lse=s.lse.data_ptr(), window=c["window"], stream=stream)
        return {"out": s.out, "lse": s.lse}
    if s.kept_tail is not None:
        s.tail.copy_(s.kept_tail)
    s.cache.append(s.batch, s.rk, s.rv, s.rq, s.rq_out, stream)
    if c["read"]:
        s.cache.read(s.batch, s.rk_read, s.rv_read, stream)
    return _appended(s)


def _appended(s):
    c = s.c
    if c["read"]:
        return {"q": s.q_out, "k": s.k_read, "v": s.v_read}
    codes, scales, _ = _page(c)
    return {"q": s.q_out, "codes": s.pool[:, :scales].view(torch.float8_e4m3fn) if c["fmt"] == "e4m3" else s.pool[:, :scales].view(torch.int8),
            "scales": s.pool[:, scales:scales + 8 * c["kv_heads"]].view(torch.float32), "tail": s.tail}


def _turn(x, cos, sin, layout, inverse=False):
    """x [tokens, heads, dim], 32 bits; cos and sin [tokens, pairs]."""
    r = 2 * cos.shape[1]
    cos, sin = cos[:, None], -sin[:, None] if inverse else sin[:, None]
    a, b = (x[..., :r // 2], x[..., r // 2:r]) if layout == "half" else (x[..., 0:r:2], x[..., 1:r:2])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([u, w], -1) if layout == "half" else torch.stack([u, w], -1).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _codes(x, fmt):
    return x.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


def _held(s, which):
    """K (0) or V (1) of every sequence in 32 bits, [seqs, kv heads, tokens, dim], from the pages and the unfinished blocks."""
    c = s.c
    kh, d, bt, n = c["kv_heads"], c["dim"], c["block"], c["seqs"]
    codes, scales, _ = _page(c)
    page = s.table[:, :s.blocks].clamp(min=0).long()
    x = _codes(s.pool[:, which * codes:(which + 1) * codes][page], c["fmt"]).view(n, s.blocks, kh, bt, d)
    x = x * s.pool[:, scales:scales + 8 * kh].view(torch.float32)[page].view(n, s.blocks, kh, 2)[..., which, None, None]
    last = (s.lens // bt).long()
    ragged = torch.arange(s.blocks, device=DEV)[None] == last[:, None]
    x = torch.where(ragged[:, :, None, None, None], s.tail[:, None, :, which].float(), x)
    x = x.permute(0, 2, 1, 3, 4).reshape(n, kh, s.blocks * bt, d)[:, :, :s.max_len]
    held = torch.arange(s.max_len, device=DEV)[None] < s.lens[:, None]
    return torch.where(held[:, None, :, None], x, 0.0)


def _run_plain(s):
    c = s.c
    if c["op"] == "rotary":
        s.out.copy_(_turn(s.x.float(), s.cos[s.pos], s.sin[s.pos], c["rotary"], c["inverse"]))
        return s.out
    if c["op"] == "evict":
        return _plain_evict(s)
    t = TYPES[c["dtype"]]
    n, kh, d, bt = c["seqs"], c["kv_heads"], c["dim"], c["block"]
    if c["op"] == "append":
        return _plain_append(s)
    g = c["q_heads"] // kh
    q = torch.zeros(n, s.max_new, c["q_heads"], d, device=DEV)
    q[s.seq, s.slot] = s.q.float()
    q = q.view(n, s.max_new, kh, g, d).permute(0, 2, 3, 1, 4).reshape(n, kh, g * s.max_new, d)
    k = _held(s, 0)
    score = torch.matmul(q, k.transpose(2, 3)).view(n, kh, g, s.max_new, s.max_len)
    del k
    score *= d ** -0.5
    index = (s.lens - s.news)[:, None] + torch.arange(s.max_new, device=DEV)[None]       # where each query stands in its sequence
    token = torch.arange(s.max_len, device=DEV)
    sees = (token <= index[..., None]) & (index < s.lens[:, None])[..., None]
    if c["window"]:
        sees &= token > index[..., None] - c["window"]
    score.masked_fill_(~sees[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp(min=-3e38)
    score -= top
    p = score.exp_()
    total = p.sum(-1, keepdim=True)
    lse = (top + total.log()).squeeze(-1)
    p /= total.clamp(min=1e-38)
    v = _held(s, 1)
    out = torch.matmul(p.view(n, kh, g * s.max_new, s.max_len), v).view(n, kh, g, s.max_new, d)
    s.out.copy_(out.permute(0, 3, 1, 2, 4).reshape(n, s.max_new, c["q_heads"], d)[s.seq, s.slot].to(t))
    s.lse.copy_(lse.permute(0, 3, 1, 2).reshape(n, s.max_new, c["q_heads"])[s.seq, s.slot])
    if not c["mass"]:
        return {"out": s.out, "lse": s.lse}
    weight = p.sum((2, 3))
    weight = torch.nn.functional.pad(weight, (0, s.blocks * bt - s.max_len)).view(n, kh, s.blocks, bt).sum(-1)
    inside = torch.arange(s.blocks, device=DEV)[None] * bt < s.lens[:, None]
    s.new_mass.copy_(torch.where(inside[:, None], s.mass + weight, s.new_mass))
    return {"out": s.out, "lse": s.lse, "mass": s.new_mass}


def _plain_append(s):
    c, t = s.c, TYPES[s.c["dtype"]]
    kh, d, bt = c["kv_heads"], c["dim"], c["block"]
    codes, scales, _ = _page(c)
    if s.kept_tail is not None:
        s.tail.copy_(s.kept_tail)
    cos, sin = s.cos[s.pos], s.sin[s.pos]
    s.q_out.copy_(_turn(s.q.float(), cos, sin, c["rotary"]))
    new = torch.stack([_turn(s.k.float(), cos, sin, c["rotary"]), s.v.float()], 2)       # [tokens, kv heads, 2, dim]
    first = (s.lens - s.news).long()
    if s.done.shape[0]:
        seq, blk = s.done[:, 0], s.done[:, 1]
        token = blk[:, None] * bt + torch.arange(bt, device=DEV)                         # [blocks, block tokens]
        fresh = token >= first[seq][:, None]
        row = (s.starts[:-1].long()[seq][:, None] + token - first[seq][:, None]).clamp(min=0)
        x = torch.where(fresh[..., None, None, None], new[row], s.tail.float()[seq].permute(0, 3, 1, 2, 4))
        x = x.permute(0, 3, 2, 1, 4)                                                     # [blocks, 2, kv heads, block tokens, dim]
        amax = x.abs().amax((3, 4))
        amax = torch.where(amax < TINY, 0.0, amax)
        factor = torch.where(amax > 0, TOP[c["fmt"]] / amax, 0.0)
        x = (x * factor[..., None, None]).clamp(-TOP[c["fmt"]], TOP[c["fmt"]])
        x = (x.round().to(torch.int8) if c["fmt"] == "int8" else x.to(torch.float8_e4m3fn)).view(torch.uint8).reshape(-1, scales)
        page = s.table[seq, blk].long()
        s.pool[:, :scales].index_copy_(0, page, x)
        s.pool[:, scales:scales + 8 * kh].index_copy_(0, page, (amax / TOP[c["fmt"]]).transpose(1, 2).reshape(-1, 2 * kh).view(torch.uint8))
    at = first[s.seq] + s.slot
    keep = at >= (s.lens.long() // bt * bt)[s.seq]                                       # into the block that stays unfinished
    old = s.tail[s.seq, :, :, at % bt]
    # tokens of finished blocks write back what is there, or what the unfinished block's own token there gets
    owner = (s.starts[1:].long()[s.seq] - 1) - (s.lens.long()[s.seq] - 1 - (s.lens.long() // bt * bt)[s.seq] - at % bt)
    has = (owner < s.starts[1:].long()[s.seq]) & (owner >= s.starts[:-1].long()[s.seq])
    s.tail[s.seq, :, :, at % bt] = torch.where((keep | has)[:, None, None, None], new[torch.where(has, owner, 0)].to(t), old)
    if c["read"]:
        for which, x in ((0, s.k_read), (1, s.v_read)):
            x.copy_(_held(s, which).transpose(1, 2))
    return _appended(s)


def _plain_evict(s):
    c = s.c
    stride = s.table.shape[1]
    n = torch.arange(stride, device=DEV)[None]
    full, held = (s.lens // c["block"])[:, None], -(-s.lens // c["block"])[:, None]
    score = s.mass.double().sum(1).float()
    safe = (n < c["first"]) | (n >= full - c["last"])
    free = (~safe & (n < full)).sum(1, keepdim=True)
    drop = torch.minimum((full - c["budget"]).clamp(min=0), free)
    order = torch.where(safe, math.inf, score).argsort(dim=1, stable=True)
    rank = torch.empty_like(order).scatter_(1, order, n.expand_as(order))
    out = (rank < drop) & ~safe
    stay = ~out & (n < held)
    order = (~stay).to(torch.int8).argsort(dim=1, stable=True)
    kept = stay.sum(1, keepdim=True)
    s.new_table.copy_(torch.where(n < kept, s.table.gather(1, order), -1))
    s.new_mass.copy_(torch.where((n < kept)[:, None], s.mass.gather(2, order[:, None].expand_as(s.mass)), 0.0))
    order = (~out).to(torch.int8).argsort(dim=1, stable=True)
    s.evicted.copy_(torch.where(n < drop, s.table.gather(1, order), -1))
    s.count.copy_(drop[:, 0])
    s.new_lens.copy_(s.lens - drop[:, 0] * c["block"])
    return {"table": s.new_table, "lens": s.new_lens, "mass": s.new_mass, "evicted": s.evicted, "count": s.count}


# ------------------------------------------------------------------------------------------------ 64 bits ----

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "evict":
        return _exact_evict(s)
    if c["op"] == "rotary":
        return _exact_turn(s.x, s.pos, s.freq, s.gain, c["rotary"], -1.0 if c["inverse"] else 1.0)
    lens, news, starts = s.lens.tolist(), s.news.tolist(), s.starts.tolist()
    kh, d, bt = c["kv_heads"], c["dim"], c["block"]
    codes, scales, _ = _page(c)
    if c["op"] == "attention":
        out = torch.zeros(s.total, c["q_heads"], d, dtype=torch.float64, device=DEV)
        lse = torch.zeros(s.total, c["q_heads"], dtype=torch.float64, device=DEV)
        mass = s.mass.double() if c["mass"] else None
        for i, (L, n) in enumerate(zip(lens, news)):
            values = []
            for which in range(2):
                parts = [s.tail[i, :, which, :L % bt].double()]
                if L >= bt:
                    page = s.table[i, :L // bt].long()
                    raw = s.pool[page][:, which * codes:(which + 1) * codes].view(torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn).double()
                    by = s.pool[page][:, scales:scales + 8 * kh].view(torch.float32).double().view(-1, kh, 2)[..., which]
                    parts.insert(0, (raw.view(-1, kh, bt, d) * by[..., None, None]).transpose(0, 1).reshape(kh, -1, d))
                values.append(torch.cat(parts, 1))
            k, v = values
            at = torch.arange(L - n, L, device=DEV)[:, None]
            token = torch.arange(L, device=DEV)[None]
            hidden = token > at
            if c["window"]:
                hidden = hidden | (token <= at - c["window"])
            for h in range(c["q_heads"]):
                a = h // (c["q_heads"] // kh)
                z = (s.q[starts[i]:starts[i + 1], h].double() @ k[a].T) / math.sqrt(d)
                z = z.masked_fill(hidden, -math.inf)
                lse[starts[i]:starts[i + 1], h] = torch.logsumexp(z, 1)
                p = torch.softmax(z, 1)
                out[starts[i]:starts[i + 1], h] = p @ v[a]
                if c["mass"]:
                    full = torch.zeros(-(-L // bt) * bt, dtype=torch.float64, device=DEV)
                    full[:L] = p.sum(0)
                    mass[i, a, :-(-L // bt)] += full.view(-1, bt).sum(1)
            if c["mass"]:
                mass[i, :, -(-L // bt):] = 0
        return {"out": out, "lse": lse, "mass": mass} if c["mass"] else {"out": out, "lse": lse}
    q = _exact_turn(s.q, s.pos, s.freq, s.gain, c["rotary"], 1.0)
    k = _exact_turn(s.k, s.pos, s.freq, s.gain, c["rotary"], 1.0)
    tail = s.tail.double()
    kept = s.pool[:, :scales].view(torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn).double()
    by = s.pool[:, scales:scales + 8 * kh].view(torch.float32).double()
    held = [torch.zeros(c["seqs"], s.max_len, kh, d, dtype=torch.float64, device=DEV) for _ in range(2)] if c["read"] else None
    for i, (L, n) in enumerate(zip(lens, news)):
        if L - n and c["read"]:                         # blocks that were there
            for b in range((L - n) // bt):
                p = int(s.table[i, b])
                for which in range(2):
                    held[which][i, b * bt:(b + 1) * bt] = (kept[p].view(2, kh, bt, d)[which] * by[p].view(kh, 2)[:, which, None, None]).transpose(0, 1)
        first = (L - n) // bt * bt
        for which, x in ((0, k), (1, s.v.double())):
            run_of = torch.cat([s.tail[i, :, which, :L - n - first].double().transpose(0, 1), x[starts[i]:starts[i + 1]]])
            whole = run_of.shape[0] // bt
            blocks = run_of[:whole * bt].view(whole, bt, kh, d).permute(0, 2, 1, 3)
            amax = blocks.abs().amax((2, 3))
            unit = torch.where(amax < TINY, torch.zeros_like(amax), amax) / TOP[c["fmt"]]
            z = torch.where(unit[..., None, None] > 0, blocks / unit[..., None, None], 0.0)
            z = torch.round(z) if c["fmt"] == "int8" else _nearest_e4m3(z)
            page = s.table[i, first // bt:first // bt + whole].long()
            kept.view(-1, 2, kh, bt * d)[page, which] = z.reshape(whole, kh, bt * d)
            by.view(-1, kh, 2)[page, :, which] = unit
            rest = run_of[whole * bt:]
            tail[i, :, which, :rest.shape[0]] = rest.transpose(0, 1)
            if c["read"]:
                held[which][i, first:first + whole * bt] = (z * unit[..., None, None]).transpose(1, 2).reshape(whole * bt, kh, d)
                held[which][i, first + whole * bt:L] = rest
    if c["read"]:
        return {"q": q, "k": held[0], "v": held[1]}
    return {"q": q, "codes": kept, "scales": by, "tail": tail}


def _exact_evict(s):
    c, stride = s.c, s.table.shape[1]
    table, mass, lens = s.table.tolist(), s.mass.double().cpu(), s.lens.tolist()
    score = mass.sum(1).float().tolist()
    got = {k: torch.full((c["seqs"], stride), -1, dtype=torch.int32) for k in ("table", "evicted")}
    got["mass"], got["lens"], got["count"] = torch.zeros_like(mass), s.lens.cpu().clone(), torch.zeros_like(s.lens).cpu()
    for i, held in enumerate(lens):
        full = held // c["block"]
        free = sorted(range(min(c["first"], full), max(c["first"], full - c["last"])), key=lambda b: (score[i][b], b))
        free = [b for b in free if b < full]
        out = sorted(free[:max(0, full - c["budget"])])
        gone = set(out)
        stay = [b for b in range(-(-held // c["block"])) if b not in gone]
        got["table"][i, :len(stay)] = torch.tensor([table[i][b] for b in stay], dtype=torch.int32)
        got["evicted"][i, :len(out)] = torch.tensor([table[i][b] for b in out], dtype=torch.int32)
        got["mass"][i, :, :len(stay)] = mass[i][:, stay]
        got["lens"][i] -= len(out) * c["block"]
        got["count"][i] = len(out)
    return {k: v.to(DEV) for k, v in got.items()}


def _exact_turn(x, pos, freq, gain, layout, sign):
    angle = sign * pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    z = gain * torch.polar(torch.ones_like(angle), angle)[:, None]
    out, r = x.double(), 2 * len(freq)
    if layout == "half":
        w = torch.complex(out[..., :r // 2].contiguous(), out[..., r // 2:r].contiguous()) * z
        out[..., :r // 2], out[..., r // 2:r] = w.real, w.imag
    else:
        w = torch.complex(out[..., 0:r:2].contiguous(), out[..., 1:r:2].contiguous()) * z
        out[..., 0:r:2], out[..., 1:r:2] = w.real, w.imag
    return out


def _nearest_e4m3(z):
    """To the nearest of the numbers with 3 fraction bits and exponents from 2^-6 (below: multiples of 2^-9) to 448, ties to even."""
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(z / step) * step

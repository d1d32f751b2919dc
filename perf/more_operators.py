"""The latent cache operators in numbers: what is measured, in a plain form and through the library.

A latent cache holds ONE vector per token for all heads, in pages of 16-bit values: `latent` channels, normed, from which every head's
keys and values can be made by a matrix, and `rope` channels of a key that all heads share and that turns with the position.

  append   norms new tokens' latents, turns their shared keys, stores both in the pages, and turns the queries' part
  attend   attention in the latent space (the matrices are absorbed into the queries and the answers): one new token per sequence,
           several, or a tree of drafted ones, each of which sees the cache and its ancestors
  expand   keys and values of every head for the cached tokens: a matrix product that reads the pages
  prompt   attention of many new tokens over expanded keys and values, with the shared keys from the pages
  accept   walks a drafted tree along the model's choices and moves the accepted tokens together in the pages

``run`` computes an operator in elementary torch operations where ``own`` is false, and through
``paper_2410_15240_b200.latent`` where it is true.  ``exact`` is the definition in 64 bits.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases ----

def listed():
    return [
        # one new token for each sequence of a serving batch
        dict(name="append_one_each", op="append", dtype="bf16", seqs=64, new=1, len_min=130, len_max=4096, heads=128, latent=512, rope=64, block=64,
             rotary="interleaved", norm=True),
        # prompts that start a cache or lengthen it
        dict(name="append_prompts", op="append", dtype="bf16", seqs=7, new=2500, len_min=2500, len_max=9001, heads=128, latent=512, rope=64, block=64,
             rotary="interleaved", norm=True),
        # one user's short chat, one token at a time: latency
        dict(name="attend_one_short", op="attend", dtype="bf16", seqs=1, new=1, len_min=700, len_max=700, heads=16, latent=512, rope=64, block=64, tree=False),
        # a serving batch of unequal lengths, many heads
        dict(name="attend_batch_ragged", op="attend", dtype="bf16", seqs=61, new=1, len_min=130, len_max=4096, heads=128, latent=512, rope=64, block=64,
             tree=False),
        # few sequences with very long contexts: one axis to split
        dict(name="attend_long", op="attend", dtype="f16", seqs=4, new=1, len_min=70001, len_max=131072, heads=64, latent=512, rope=64, block=128, tree=False),
        # trees of drafted tokens checked at once, small blocks
        dict(name="attend_tree", op="attend", dtype="bf16", seqs=15, new=25, len_min=333, len_max=5000, heads=16, latent=512, rope=64, block=16, tree=True),
        # the cached part of a short prompt expanded for a small model
        dict(name="expand_short", op="expand", dtype="f16", seqs=3, new=1, len_min=333, len_max=1100, heads=16, latent=256, rope=32, key=64, value=64, block=32),
        # long contexts expanded for a large one
        dict(name="expand_long", op="expand", dtype="bf16", seqs=2, new=1, len_min=4500, len_max=7777, heads=64, latent=512, rope=64, key=128, value=128,
             block=64),
        # a long prompt taken in pieces: many new tokens against what is cached already
        dict(name="prompt_piece", op="prompt", dtype="bf16", seqs=3, new=1000, len_min=1500, len_max=6100, heads=32, latent=512, rope=64, key=128, value=128,
             block=64),
        # whole prompts at once
        dict(name="prompt_whole", op="prompt", dtype="f16", seqs=2, new=8000, len_min=8000, len_max=8000, heads=16, latent=512, rope=64, key=128, value=128,
             block=128),
        # drafts of a few sequences: stored, then the accepted ones kept
        dict(name="accept_few", op="accept", dtype="bf16", seqs=4, new=12, len_min=100, len_max=3000, heads=16, latent=512, rope=64, block=64,
             rotary="half", norm=True),
        # drafts of a large batch
        dict(name="accept_batch", op="accept", dtype="bf16", seqs=128, new=63, len_min=100, len_max=3000, heads=16, latent=512, rope=64, block=64,
             rotary="half", norm=True),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "attend", "expand", "prompt", "prompt", "accept"])
    c = dict(op=op, dtype=rng.choice(["bf16", "f16"]), block=rng.choice([16, 32, 64, 128]), latent=rng.choice([128, 256, 384, 512, 512]),
             rope=rng.choice([32, 64, 64]))
    if op == "attend":
        heads, tree = rng.choice([1, 5, 12, 16, 40, 64, 128]), rng.random() < 0.3
        new = rng.randint(2, 64) if tree else rng.choice([1, 1, rng.randint(2, 12), _spread(rng, 16, 200)])
        len_max = _spread(rng, max(new, 40), 100000)
        most = min(2.6e5 / len_max, 2.5e7 / (len_max * heads * new), 1e5 / (heads * new))       # tokens, scores, and queries
        if most < 1:
            len_max, most = max(new, int(len_max * most)), 1
        return dict(c, seqs=rng.randint(1, max(1, min(96, int(most)))), new=new, len_min=rng.randint(new, len_max), len_max=len_max, heads=heads, tree=tree)
    if op in ("append", "accept"):
        new = rng.choice([1, _spread(rng, 2, 4000)]) if op == "append" else rng.randint(1, 128)
        len_max = rng.randint(new, new + 4000)
        seqs = rng.randint(1, max(1, min(128, (16000 if op == "append" else 8000) // new)))
        return dict(c, seqs=seqs, new=new, len_min=rng.randint(new, len_max), len_max=len_max, heads=rng.choice([1, 5, 16, 64, 128]) if op == "append" else 16,
                    rotary=rng.choice(["half", "interleaved"]), norm=op == "accept" or rng.random() < 0.7)
    heads, key, value = rng.choice([1, 5, 8, 16, 32, 64]), rng.choice([64, 128]), rng.choice([64, 128])
    if op == "expand":
        len_max = _spread(rng, 1, 30000)
        seqs = rng.randint(1, max(1, min(32, int(2e5 / len_max), int(5e5 / (len_max * heads)))))
        len_max = max(1, min(len_max, int(5e5 / (seqs * heads))))
        return dict(c, seqs=seqs, new=1, len_min=rng.randint(1, len_max), len_max=len_max, heads=heads, key=key, value=value)
    new = _spread(rng, 1, 4000)
    len_max = rng.randint(new, new + rng.choice([0, 100, 6000]))
    heads = max(1, min(heads, int(7e8 / (new * len_max)), int(5e5 / len_max)))            # scores, and keys
    most = min(7e8 / (new * len_max * heads), 5e5 / (len_max * heads))
    return dict(c, seqs=rng.randint(1, max(1, min(24, int(most)))), new=new, len_min=rng.randint(new, len_max), len_max=len_max, heads=heads, key=key,
                value=value)


def _lens(c):
    """Tokens held by each sequence after the call: from len_min to len_max, unequal, the same for every seed."""
    n = c["seqs"]
    return [c["len_max"] if i == 0 else c["len_min"] + int((c["len_max"] - c["len_min"]) * ((i * 0.6180339887498949) % 1.0)) for i in range(n)]


def _news(c):
    """New tokens of each sequence: the full number for the first, fewer for some others, never none."""
    if c["new"] == c["len_min"] == c["len_max"]:
        return [c["new"]] * c["seqs"]
    return [c["new"] if i % 3 == 0 else max(1, c["new"] - (i * 7) % max(1, c["new"] // 2)) for i in range(c["seqs"])]


def work(c):
    lens, news = _lens(c), _news(c)
    new, held, h = sum(news), sum(lens), c["heads"]
    row = c["latent"] + c["rope"]
    if c["op"] in ("append", "accept"):
        total = 2 * 2 * new * row + 8 * new + (2 * c["latent"] if c["norm"] else 0)
        if c["op"] == "append":
            return {"bytes": total + 2 * 2 * new * h * c["rope"], "flops": new * (4 * c["latent"] + 3 * c["rope"] * (1 + h))}
        moved = 3 * c["seqs"]                                                          # some three tokens of a tree are accepted
        return {"bytes": total + 2 * 2 * moved * row + 4 * 4 * new + 16 * c["seqs"], "flops": new * (4 * c["latent"] + 3 * c["rope"])}
    table = sum(4 * -(-n // c["block"]) for n in lens)
    if c["op"] == "expand":
        out = h * (c["key"] + c["value"])
        return {"bytes": 2 * held * c["latent"] + table + 2 * out * c["latent"] + 2 * held * out, "flops": 2 * held * out * c["latent"]}
    pairs = sum(sum(range(L - n + 1, L + 1)) for L, n in zip(lens, news))
    if c["op"] == "prompt":
        each = c["key"] + c["rope"] + c["value"]
        return {"bytes": 2 * held * (h * (c["key"] + c["value"]) + c["rope"]) + table + 2 * new * h * each + 4 * new * h, "flops": 2 * pairs * h * each}
    if c["tree"]:                                                                      # a drafted token sees some four others
        pairs = sum((L - n + 4) * n for L, n in zip(lens, news))
    return {"bytes": 2 * held * row + table + 2 * new * h * (row + c["latent"]) + 4 * new * h + (4 * new if c["tree"] else 0),
            "flops": 2 * pairs * h * (row + c["latent"])}


# ------------------------------------------------------------------------------------------------ inputs ----

class State:
    pass


def _normal(gen, *shape, dtype=torch.float32):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=dtype)


def _trees(news, seed):
    """A drafted tree for each sequence: row 0 is the last token that is certain, the others are drafted children of earlier rows, tokens out
    of a small vocabulary; and the model's choice behind every row, mostly one of its children's tokens.
    -> parents, tokens, choices, depths of all rows."""
    gen = torch.Generator().manual_seed(seed)
    parents, tokens, choices, depths = [], [], [], []
    for n in news:
        r = torch.rand(4, n, generator=gen).tolist()
        parent = [-1] + [max(0, j - 6) + int(r[0][j] * (j - max(0, j - 6))) for j in range(1, n)]
        token = [int(997 * x) for x in r[1]]
        depth = [0] * n
        for j in range(1, n):
            depth[j] = depth[parent[j]] + 1
        choice = []
        for j in range(n):
            kids = [i for i in range(j + 1, n) if parent[i] == j]
            choice.append(token[kids[int(r[3][j] * len(kids))]] if kids and r[2][j] < 0.75 else int(997 * r[3][j]))
        parents += parent
        tokens += token
        choices += choice
        depths += depth
    return parents, tokens, choices, depths


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def prepare(c, seed):
    s, gen = State(), torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s.c = c
    t, h, latent, rope, bt = TYPES[c["dtype"]], c["heads"], c["latent"], c["rope"], c["block"]
    s.row = latent + rope
    s.l, s.n = _lens(c), _news(c)
    s.total, s.max_len = sum(s.n), max(s.l)
    s.scale = 1.0 / math.sqrt(c.get("key", 128) + rope)
    s.lens, s.news = _ints(s.l), _ints(s.n)
    s.starts = torch.cat([torch.zeros_like(s.news[:1]), s.news.cumsum(0).to(torch.int32)])
    s.st = s.starts.tolist()
    blocks = [-(-n // bt) for n in s.l]
    s.pages = sum(blocks) + 3
    table = torch.full((c["seqs"], max(blocks) + 1), -1, dtype=torch.int32)
    order = torch.randperm(s.pages, generator=torch.Generator().manual_seed(seed + 1)).to(torch.int32)
    at = 0
    for i, n in enumerate(blocks):
        table[i, :n] = order[at:at + n]
        at += n
    s.table = table.to(DEV)
    s.pool = _normal(gen, s.pages, bt, s.row).to(t)
    # where token t of sequence i lies: row of the pool's tokens
    s.where = [(s.table[i, :b].long()[:, None] * bt + torch.arange(bt, device=DEV)).flatten()[:n] for i, (b, n) in enumerate(zip(blocks, s.l))]
    new_at = torch.cat([w[L - n:] for w, L, n in zip(s.where, s.l, s.n)])
    s.new_at = new_at
    depths = None
    if c["op"] == "accept" or c.get("tree"):
        parents, tokens, choices, depths = _trees(s.n, seed)
        s.p, s.parents, s.tokens, s.choices = parents, _ints(parents), _ints(tokens), _ints(choices)
        s.tok, s.cho = tokens, choices
        s.levels = max(depths) + 1
    if c["op"] in ("append", "accept"):
        s.freq = [10000.0 ** (-2.0 * i / rope) for i in range(rope // 2)]
        pos = [torch.arange(L - n, L) for L, n in zip(s.l, s.n)]
        s.pos = torch.cat(pos).to(DEV) if depths is None else torch.cat([torch.full((n,), L - n) for L, n in zip(s.l, s.n)]).to(DEV) + torch.tensor(depths, device=DEV)
        angle = torch.arange(s.max_len + 1, device=DEV, dtype=torch.float64)[:, None] * torch.tensor(s.freq, device=DEV, dtype=torch.float64)
        s.cos, s.sin = angle.cos().float(), angle.sin().float()
        s.down = (3 * _normal(gen, s.total, s.row)).to(t)                             # as one projection gives them
        s.c_new, s.k_new = s.down.split([latent, rope], 1)
        s.weight = (1 + 0.2 * _normal(gen, latent)).to(t) if c["norm"] else None
        s.q = s.q_out = None
        s.out = {"pool": s.pool}
        if c["op"] == "append":
            q = _normal(gen, s.total, h, 128 + rope).to(t)                            # a head's query: 128 channels without position, then these
            s.q, s.q_out = q[..., 128:], torch.empty(s.total, h, rope, dtype=t, device=DEV)
            s.out["q"] = s.q_out
        else:
            s.path, s.count, s.next, s.lens_out = _ints([0] * s.total), torch.empty_like(s.lens), torch.empty_like(s.lens), torch.empty_like(s.lens)
            s.out.update(path=s.path, count=s.count, next=s.next, lens=s.lens_out)
    elif c["op"] == "attend":
        s.q = _normal(gen, h, s.total, latent).to(t).transpose(0, 1)                  # as a product per head gives them
        s.q_rope = _normal(gen, s.total, h, rope).to(t)
        s.answer = torch.empty(s.total, h, latent, dtype=t, device=DEV)
    else:
        s.key_starts = [0]
        for L in s.l:
            s.key_starts.append(s.key_starts[-1] + L)
        s.keys = s.key_starts[-1]
        if c["op"] == "expand":
            s.weights = (_normal(gen, h, c["key"] + c["value"], latent) * latent ** -0.5).to(t)
            s.k, s.v = torch.empty(s.keys, h, c["key"], dtype=t, device=DEV), torch.empty(s.keys, h, c["value"], dtype=t, device=DEV)
            s.out = {"k": s.k, "v": s.v}
        else:
            s.k, s.v = _normal(gen, s.keys, h, c["key"]).to(t), _normal(gen, s.keys, h, c["value"]).to(t)
            s.q_all = (1.5 * _normal(gen, s.total, h, c["key"] + rope)).to(t)
            s.q, s.q_rope = s.q_all[..., :c["key"]], s.q_all[..., c["key"]:]
            s.answer = torch.empty(s.total, h, c["value"], dtype=t, device=DEV)
    if c["op"] in ("attend", "prompt"):
        s.lse = torch.empty(s.total, h, device=DEV)
        s.out = {"out": s.answer, "lse": s.lse}
    if own:
        _prepare_own(s)
    return s


def _prepare_own(s):
    from paper_2410_15240_b200 import kv, latent
    c = s.c

    def rows(x):
        return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1) if x.dim() > 2 else 0)

    rotary = dict(rotary=getattr(kv, "ROTARY_" + c["rotary"].upper()), frequencies=s.freq) if "rotary" in c else {}
    s.cache = latent.LatentCache(getattr(kv, c["dtype"].upper()), c["heads"], c["latent"], c["rope"], c.get("key", 128), c.get("value", 128), c["block"],
                                 norm_eps=EPS, **rotary)
    s.batch = latent.Batch(n_seqs=c["seqs"], total_new=s.total, max_new=max(s.n), max_len=s.max_len, pool_pages=s.pages, table_stride=s.table.stride(0),
                           d_pool=s.pool.data_ptr(), d_table=s.table.data_ptr(), d_lens=s.lens.data_ptr(), d_starts=s.starts.data_ptr(),
                           d_positions=s.pos.data_ptr() if "rotary" in c else 0)
    if c["op"] in ("append", "accept"):
        s.rows = rows(s.c_new), rows(s.k_new), s.weight.data_ptr() if c["norm"] else 0
        s.q_rows = (rows(s.q), rows(s.q_out)) if s.q is not None else (None, None)
    if c["op"] == "accept":
        s.call = latent.Acceptance(d_parents=s.parents.data_ptr(), d_tokens=s.tokens.data_ptr(), d_choices=s.choices.data_ptr(), d_path=s.path.data_ptr(),
                                   d_n_accepted=s.count.data_ptr(), d_next=s.next.data_ptr(), d_lens_out=s.lens_out.data_ptr())
    if c["op"] == "attend":
        s.rows = rows(s.q), rows(s.q_rope), rows(s.answer)
        s.workspace = torch.zeros(s.cache.workspace_bytes(s.batch), dtype=torch.uint8, device=DEV)
    if c["op"] in ("expand", "prompt"):
        s.d_key_starts = _ints(s.key_starts)
        s.rows = rows(s.k), rows(s.v)
    if c["op"] == "prompt":
        s.q_rows = rows(s.q), rows(s.q_rope), rows(s.answer)
        s.workspace = torch.zeros(s.cache.prompt_workspace_bytes(s.batch), dtype=torch.uint8, device=DEV)


# ------------------------------------------------------------------------------------------------ the operators ----

def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    op, stream = s.c["op"], torch.cuda.current_stream().cuda_stream
    if op == "attend":
        q, q_rope, out = s.rows
        s.cache.attention(s.batch, q, q_rope, out, s.workspace.data_ptr(), s.workspace.numel(), d_lse=s.lse.data_ptr(),
                          d_parents=s.parents.data_ptr() if s.c["tree"] else 0, stream=stream)
    elif op == "prompt":
        (q, q_rope, out), (k, v) = s.q_rows, s.rows
        s.cache.prompt(s.batch, q, q_rope, k, v, s.d_key_starts.data_ptr(), s.keys, out, s.workspace.data_ptr(), s.workspace.numel(),
                       d_lse=s.lse.data_ptr(), stream=stream)
    elif op == "expand":
        s.cache.expand(s.batch, s.weights.data_ptr(), s.rows[0], s.rows[1], s.d_key_starts.data_ptr(), s.keys, stream=stream)
    else:
        s.cache.append(s.batch, s.rows[0], s.rows[1], s.rows[2], s.q_rows[0], s.q_rows[1], stream=stream)
        if op == "accept":
            s.cache.accept(s.batch, s.call, stream=stream)
    return s.out


def _turn(x, cos, sin, layout):
    """x [..., rope], 32 bits; cos and sin as x with half the channels."""
    r = x.shape[-1]
    a, b = (x[..., :r // 2], x[..., r // 2:]) if layout == "half" else (x[..., 0::2], x[..., 1::2])
    u, w = a * cos - b * sin, b * cos + a * sin
    return torch.cat([u, w], -1) if layout == "half" else torch.stack([u, w], -1).flatten(-2)


def _ancestors(s, i):
    """Which drafted rows each drafted row of sequence i sees: itself, its parent, and so on."""
    n, st = s.n[i], s.st[i]
    parent = s.parents[st:st + n].long()
    seen = torch.eye(n, dtype=torch.bool, device=DEV)
    up = seen.clone()
    for _ in range(s.levels):
        has = (parent >= 0)[:, None]
        up = torch.where(has, up[parent.clamp(min=0)], False)
        seen = seen | up
    return seen


def _run_plain(s):
    c = s.c
    flat = s.pool.view(-1, s.row)
    if c["op"] in ("append", "accept"):
        return _plain_append(s, flat)
    if c["op"] == "expand":
        w = s.weights.float().view(-1, c["latent"])
        x = torch.cat([flat[at, :c["latent"]] for at in s.where]).float()
        x = torch.matmul(x, w.T).view(s.keys, c["heads"], -1)
        s.k.copy_(x[..., :c["key"]])
        s.v.copy_(x[..., c["key"]:])
        return s.out
    token = torch.arange(s.max_len, device=DEV)
    for i, (L, n) in enumerate(zip(s.l, s.n)):
        here = slice(s.st[i], s.st[i] + n)
        held = flat[s.where[i]].float()
        sees = token[None, :L] <= torch.arange(L - n, L, device=DEV)[:, None]
        if c.get("tree"):
            sees[:, L - n:] = _ancestors(s, i)
        keys = slice(s.key_starts[i], s.key_starts[i] + L) if c["op"] == "prompt" else None
        # some heads at a time: a GB or two of scores
        step = max(1, min(c["heads"], int(4e8 / (n * L))))
        for h in range(0, c["heads"], step):
            some = slice(h, min(c["heads"], h + step))
            q, q_rope = s.q[here, some].float().transpose(0, 1), s.q_rope[here, some].float().transpose(0, 1)
            if keys is None:
                k = held[None, :, :c["latent"]]
                v = k
            else:
                k, v = s.k[keys, some].float().transpose(0, 1), s.v[keys, some].float().transpose(0, 1)
            score = torch.matmul(q, k.transpose(1, 2))
            score += torch.matmul(q_rope, held[:, c["latent"]:].T)
            score *= s.scale
            score.masked_fill_(~sees, -math.inf)
            top = score.amax(-1, keepdim=True)
            p = score.sub_(top).exp_()
            total = p.sum(-1, keepdim=True)
            s.lse[here, some] = (top + total.log()).squeeze(-1).T
            p /= total
            s.answer[here, some] = torch.matmul(p, v).transpose(0, 1).to(s.answer.dtype)
    return s.out


def _plain_append(s, flat):
    c = s.c
    cos, sin = s.cos[s.pos], s.sin[s.pos]
    x = s.c_new.float()
    if c["norm"]:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s.weight.float()
    flat[s.new_at] = torch.cat([x, _turn(s.k_new.float(), cos, sin, c["rotary"])], 1).to(flat.dtype)
    if s.q is not None:
        s.q_out.copy_(_turn(s.q.float(), cos[:, None], sin[:, None], c["rotary"]))
        return s.out
    # every level of all trees at once: from each sequence's last accepted row to the first child that holds the chosen token
    n = c["seqs"]
    start, news = s.starts[:-1].long(), s.news.long()
    at = torch.zeros(n, dtype=torch.long, device=DEV)
    live = news > 0
    s.path.fill_(-1)
    s.count.zero_()
    seq = torch.repeat_interleave(torch.arange(n, device=DEV), news, output_size=s.total)
    slot = torch.arange(s.total, device=DEV) - start[seq]
    far = s.total
    chosen = [at]
    alive = [live]
    for _ in range(s.levels - 1):
        fits = (s.parents.long() == at[seq]) & (s.tokens == s.choices[(start + at)[seq]]) & (slot > 0)
        best = torch.full((n,), far, dtype=torch.long, device=DEV).scatter_reduce_(0, seq, torch.where(fits, slot, far), "amin")
        live = live & (best < far)
        at = torch.where(live, best, at)
        chosen.append(at)
        alive.append(live)
    chosen, alive = torch.stack(chosen, 1), torch.stack(alive, 1)
    s.count.copy_(alive.sum(1))
    s.next.copy_(s.choices[start + at])
    s.lens_out.copy_(s.lens.long() - news + alive.sum(1))
    level = torch.arange(chosen.shape[1], device=DEV)[None]
    to = (start[:, None] + level)
    where = to[alive]
    s.path[where] = chosen[alive].to(torch.int32)
    flat[s.new_at[where]] = flat[s.new_at[(start[:, None] + chosen)[alive]]]
    return s.out


# ------------------------------------------------------------------------------------------------ 64 bits ----

def exact(c, seed):
    s = prepare(c, seed)
    flat = s.pool.view(-1, s.row).double()
    if c["op"] in ("append", "accept"):
        return _exact_append(s, flat)
    if c["op"] == "expand":
        k, v = s.k.double(), s.v.double()
        w = s.weights.double()
        for i in range(c["seqs"]):
            x = flat[s.where[i], :c["latent"]]
            at = slice(s.key_starts[i], s.key_starts[i + 1])
            for h in range(c["heads"]):
                k[at, h] = x @ w[h, :c["key"]].T
                v[at, h] = x @ w[h, c["key"]:].T
        return {"k": k, "v": v}
    out = torch.zeros(s.answer.shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s.lse.shape, dtype=torch.float64, device=DEV)
    for i in range(c["seqs"]):
        L, n, st = s.l[i], s.n[i], s.st[i]
        x = flat[s.where[i]]
        hidden = torch.ones(n, L, dtype=torch.bool).tril(L - n).logical_not()
        if c.get("tree"):
            hidden[:, L - n:] = True
            for j in range(n):
                a = j
                while a >= 0:
                    hidden[j, L - n + a] = False
                    a = s.p[st + a]
        hidden = hidden.to(DEV)
        for h in range(c["heads"]):
            if c["op"] == "prompt":
                at = slice(s.key_starts[i], s.key_starts[i + 1])
                key, value = torch.cat([s.k[at, h].double(), x[:, c["latent"]:]], 1), s.v[at, h].double()
            else:
                key, value = x, x[:, :c["latent"]]
            q = torch.cat([s.q[st:st + n, h], s.q_rope[st:st + n, h]], 1).double()
            z = (q @ key.T) / math.sqrt(c.get("key", 128) + c["rope"])
            z = z.masked_fill(hidden, -math.inf)
            lse[st:st + n, h] = torch.logsumexp(z, 1)
            out[st:st + n, h] = torch.softmax(z, 1) @ value
    return {"out": out, "lse": lse}


def _exact_turn(x, pos, freq, layout):
    angle = pos.double()[:, None] * torch.tensor(freq, dtype=torch.float64, device=DEV)
    z = torch.polar(torch.ones_like(angle), angle)
    if x.dim() == 3:
        z = z[:, None]
    x, r = x.double(), x.shape[-1]
    out = torch.empty_like(x)
    if layout == "half":
        w = torch.complex(x[..., :r // 2].contiguous(), x[..., r // 2:].contiguous()) * z
        out[..., :r // 2], out[..., r // 2:] = w.real, w.imag
    else:
        w = torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous()) * z
        out[..., 0::2], out[..., 1::2] = w.real, w.imag
    return out


def _exact_append(s, flat):
    c = s.c
    x = s.c_new.double()
    if c["norm"]:
        x = x / torch.sqrt(x.pow(2).sum(1, keepdim=True) / c["latent"] + EPS) * s.weight.double()
    row = torch.cat([x, _exact_turn(s.k_new, s.pos, s.freq, c["rotary"])], 1)
    flat[s.new_at] = row
    if c["op"] == "append":
        return {"pool": flat.view(s.pool.shape), "q": _exact_turn(s.q, s.pos, s.freq, c["rotary"])}
    path, count, following = torch.full((s.total,), -1, dtype=torch.int32), [], []
    for i in range(c["seqs"]):
        st, n = s.st[i], s.n[i]
        walk = [0]
        while True:
            kids = [j for j in range(1, n) if s.p[st + j] == walk[-1] and s.tok[st + j] == s.cho[st + walk[-1]]]
            if not kids:
                break
            walk.append(kids[0])
        path[st:st + len(walk)] = torch.tensor(walk, dtype=torch.int32)
        count.append(len(walk))
        following.append(s.cho[st + walk[-1]])
        flat[s.new_at[st:st + len(walk)]] = row[[st + j for j in walk]]
    lens = [L - n + k for L, n, k in zip(s.l, s.n, count)]
    return {"pool": flat.view(s.pool.shape), "path": path.to(DEV), "count": _ints(count), "next": _ints(following), "lens": _ints(lens)}

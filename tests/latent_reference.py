"""The latent cache operators in 64 bits on the CPU, and a cache made of random pages to run the library on."""
from __future__ import annotations

import math

import torch

from paper_2410_15240_b200 import kv, latent

TYPES = {kv.BF16: torch.bfloat16, kv.F16: torch.float16}
UNIT = {kv.BF16: 2.0 ** -8, kv.F16: 2.0 ** -11}         # half a step of a rounding, relative
LEAST = {kv.BF16: 0.0, kv.F16: 2.0 ** -25}              # and absolute, where f16 has its smallest steps


def rows(x):
    return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1) if x.dim() > 2 else 0)


def strided(x, gap=8):
    """The same values with room between tokens and heads."""
    if x.dim() == 2:
        room = torch.full((x.shape[0], x.shape[1] + gap), -7.0, dtype=x.dtype, device=x.device)
        room[:, :x.shape[1]] = x
        return room[:, :x.shape[1]]
    room = torch.full((x.shape[0], x.shape[1] + 1, x.shape[2] + gap), -7.0, dtype=x.dtype, device=x.device)
    room[:, :x.shape[1], :x.shape[2]] = x
    return room[:, :x.shape[1], :x.shape[2]]


class Cache:
    """lens and news per sequence; pages in random order; `absent`: (sequence, block) pairs without a page."""

    def __init__(self, dtype, heads, dim, rope, block, lens, news, seed=0, key=128, value=128, absent=(), positions=None, spare=2, max_new=None, max_len=None,
                 **config):
        self.dtype, self.t, self.heads, self.dim, self.rope, self.block, self.key, self.value = dtype, TYPES[dtype], heads, dim, rope, block, key, value
        self.lens, self.news = list(lens), list(news)
        self.gen = torch.Generator().manual_seed(seed)
        self.row = dim + rope
        self.starts = [0]
        for n in self.news:
            self.starts.append(self.starts[-1] + n)
        self.total = self.starts[-1]
        self.max_len = max_len or max([1] + self.lens)
        blocks = -(-self.max_len // block)
        self.stride = blocks + 1
        count = sum(-(-n // block) for n in self.lens)
        self.pages = count + spare
        order = torch.randperm(self.pages, generator=self.gen).tolist()
        table = torch.full((len(self.lens), self.stride), -1, dtype=torch.int32)
        for i, n in enumerate(self.lens):
            for b in range(-(-n // block)):
                table[i, b] = order.pop() if (i, b) not in set(absent) else (-1 if b % 2 else self.pages + 5)
        self.table = table
        self.scale = config.get("softmax_scale", 0.0) or 1.0 / math.sqrt(key + rope)
        self.pool = torch.randn(self.pages, block, self.row, generator=self.gen).to(self.t)
        self.handle = latent.LatentCache(dtype, heads, dim, rope, key, value, block, **config)
        self.d_pool, self.d_table = self.pool.cuda(), table.cuda()
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.d_starts = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.d_pos = positions.cuda() if positions is not None else None
        self.batch = latent.Batch(n_seqs=len(self.lens), total_new=self.total, max_new=max_new or max([0] + self.news), max_len=self.max_len,
                                  pool_pages=self.pages, table_stride=self.stride, d_pool=self.d_pool.data_ptr(), d_table=self.d_table.data_ptr(),
                                  d_lens=self.d_lens.data_ptr(), d_starts=self.d_starts.data_ptr(), d_positions=positions is not None and self.d_pos.data_ptr() or 0)

    def upload(self):
        self.d_pool.copy_(self.pool)

    def page(self, i, place):
        p = int(self.table[i, place // self.block])
        return p if 0 <= p < self.pages else -1

    def held(self, i):
        """-> vectors of the sequence's tokens [len, row] in 64 bits, and whether each is there."""
        x, there = torch.zeros(self.lens[i], self.row, dtype=torch.float64), torch.zeros(self.lens[i], dtype=torch.bool)
        for place in range(0, self.lens[i], self.block):
            n, p = min(self.block, self.lens[i] - place), self.page(i, place)
            if p >= 0:
                x[place:place + n] = self.pool[p, :n].double()
                there[place:place + n] = True
        return x, there

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.gen).to(self.t)


def visible(n, length, parents=None):
    """[new tokens, tokens held]: what each new token sees."""
    sees = torch.ones(n, length, dtype=torch.bool).tril(length - n)
    if parents is not None:
        sees[:, length - n:] = False
        for j in range(n):
            a = j
            while True:
                sees[j, length - n + a] = True
                if not 0 <= parents[a] < a:
                    break
                a = parents[a]
    return sees


def attend(q, k, v, sees, scale):
    """One head in 64 bits: -> answers, lse, and for the bounds sum of p |v|, the largest sum of |q k| that a row sees."""
    z = scale * (q @ k.T)
    z = z.masked_fill(~sees, -math.inf)
    some = sees.any(1)
    lse = torch.logsumexp(z, 1)
    p = torch.where(some[:, None], torch.exp(z - lse[:, None]), 0.0)
    p = torch.where(sees, p, 0.0)
    size = (q.abs() @ k.abs().T).masked_fill(~sees, 0.0).amax(1) * scale
    return p @ v, lse, p @ v.abs(), size


def bounds(dtype, want, weighed, size, spread, tokens):
    """How far an answer may be off: its own rounding and the weights' (half a step each, and f16's smallest steps, which a weight's reference
    keeps at 1 or less of the sum); scores summed in 32 bits, one addition per 16 channels that may cut off instead of rounding, with the
    products' sum of magnitudes `size` as what is cut from (2^-23 of it per addition, 40 additions), whose error counts twice, once in the
    weight and once in the sum; the exponential (2^-21) and the answer's own sum, an addition per 16 tokens."""
    score = 40 * 2.0 ** -23 * size
    relative = UNIT[dtype] + 2 * score[:, None] + 2.0 ** -20 + (tokens / 16 + 2) * 2.0 ** -23
    return UNIT[dtype] * want.abs() + relative * weighed + LEAST[dtype] * (1 + spread)

"""The key-value cache operators in 64 bits, from their definitions, and a cache to run them on.  Test infrastructure."""
from __future__ import annotations

import math
import random
from fractions import Fraction

import numpy as np
import torch

from paper_2410_15240_b200 import kv

TYPES = {kv.BF16: torch.bfloat16, kv.F16: torch.float16}
UNIT = {kv.BF16: 2.0 ** -8, kv.F16: 2.0 ** -11}         # rounding to nearest is off by at most this share of the value
TOP = {kv.INT8: 127.0, kv.E4M3: 448.0}
TURN = 2 * Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49)


def rows(x):
    return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1))


def turn(x, positions, freq, gain, layout, inverse=False):
    """x [tokens, heads, dim] float64, any positions: the angle is reduced in exact arithmetic."""
    if not freq:
        return x.clone()
    angle = torch.tensor([[float(Fraction(int(p)) * Fraction(f) % TURN) for f in freq] for p in positions.tolist()], dtype=torch.float64).reshape(-1, len(freq))
    c, s = gain * angle.cos()[:, None], gain * angle.sin()[:, None] * (-1 if inverse else 1)
    out, r = x.clone(), 2 * len(freq)
    i, j = (slice(0, r // 2), slice(r // 2, r)) if layout == kv.ROTARY_HALF else (slice(0, r, 2), slice(1, r, 2))
    out[..., i] = x[..., i] * c - x[..., j] * s
    out[..., j] = x[..., j] * c + x[..., i] * s
    return out


class Cache:
    """A cache on the GPU, its contents in float64 on the host, and sequences of given lengths with their new tokens."""

    def __init__(self, dtype, fmt, q_heads, kv_heads, dim, block, lens, news, seed=0, rotary=kv.ROTARY_NONE, freq=None, gain=1.0, spare=2, page_base=0,
                 scale=0.0, poison=True):
        self.dtype, self.fmt, self.qh, self.kh, self.d, self.bt = dtype, fmt, q_heads, kv_heads, dim, block
        self.lens, self.news, self.layout, self.freq, self.gain = list(lens), list(news), rotary, list(freq or []), gain
        self.scale = scale or 1 / math.sqrt(dim)
        self.gen = torch.Generator().manual_seed(seed)
        self.kv = kv.KvCache(dtype, fmt, q_heads, kv_heads, dim, block, rotary=rotary, frequencies=self.freq, rotary_gain=gain, softmax_scale=scale)
        self.t = TYPES[dtype]
        self.n, self.total, self.max_new, self.max_len = len(lens), sum(news), max(news, default=0), max(lens, default=0)
        self.codes = kv_heads * block * dim
        full = [n // block for n in lens]
        self.stride = max(full, default=0) + 1
        used = sum(full)
        self.pages = page_base + used + spare
        order = torch.randperm(used + spare, generator=self.gen).tolist()
        self.table = torch.full((self.n, self.stride), 0x7fffffff, dtype=torch.int32)      # entries that no one may follow
        at = 0
        for i, n in enumerate(full):
            self.table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32) + page_base
            at += n
        fill = torch.full if not poison else lambda shape, _, **k: torch.full(shape, 255, **k)
        self.pool = fill((self.pages, self.kv.page_bytes), 0, dtype=torch.uint8, device="cuda")   # 255: NaN scales, NaN codes
        self.tail = torch.full((self.n, kv_heads, 2, block, dim), math.nan if poison else 0.0, dtype=self.t, device="cuda")
        self.d_table = self.table.cuda()
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32).cuda()
        self.starts = [0]
        for k in news:
            self.starts.append(self.starts[-1] + k)
        self.d_starts = torch.tensor(self.starts, dtype=torch.int32).cuda()
        self.positions = torch.cat([torch.arange(L - k, L) for L, k in zip(lens, news)] or [torch.zeros(0)]).long()
        self.d_positions = self.positions.cuda()

    def batch(self, **change):
        b = dict(n_seqs=self.n, total_new=self.total, max_new=self.max_new, max_len=self.max_len, pool_pages=self.pages, table_stride=self.stride,
                 d_pool=self.pool.data_ptr(), d_tail=self.tail.data_ptr(), d_table=self.d_table.data_ptr(), d_lens=self.d_lens.data_ptr(),
                 d_starts=self.d_starts.data_ptr(), d_positions=self.d_positions.data_ptr())
        return kv.Batch(**{**b, **change})

    def fill(self, spread=1.0):
        """Random contents for every full block and the held part of every tail; returns nothing, see held()."""
        for i, L in enumerate(self.lens):
            for b in range(L // self.bt):
                p = int(self.table[i, b])
                x = torch.randn(2 * self.codes, generator=self.gen) * TOP[self.fmt] / 4
                x = x.clamp(-TOP[self.fmt], TOP[self.fmt])
                raw = (x.round().to(torch.int8) if self.fmt == kv.INT8 else x.to(torch.float8_e4m3fn)).view(torch.uint8)
                self.pool[p, :2 * self.codes] = raw.cuda()
                s = (spread * torch.randn(2 * self.kh, generator=self.gen)).exp() * 4 / TOP[self.fmt]
                self.pool[p, 2 * self.codes:2 * self.codes + 8 * self.kh] = s.view(torch.uint8).cuda()
            rest = L % self.bt
            self.tail[i, :, :, :rest] = torch.randn(self.kh, 2, rest, self.d, generator=self.gen).to(self.t).cuda()

    def page(self, p):
        """(codes as numbers [2][kv_heads][block][dim], scales [2][kv_heads]) of a page, float64."""
        raw = self.pool[p].cpu()
        codes = raw[:2 * self.codes].view(torch.int8 if self.fmt == kv.INT8 else torch.float8_e4m3fn).to(torch.float64)
        scales = raw[2 * self.codes:2 * self.codes + 8 * self.kh].clone().view(torch.float32).double().view(self.kh, 2).T
        return codes.view(2, self.kh, self.bt, self.d), scales

    def held(self, i):
        """(k, v, there) of sequence i: [kv_heads][len][dim] float64, and which tokens are not on absent pages."""
        L = self.lens[i]
        x, there = torch.zeros(2, self.kh, L, self.d, dtype=torch.float64), torch.ones(L, dtype=torch.bool)
        for b in range(L // self.bt):
            p = int(self.table[i, b])
            if not 0 <= p < self.pages:
                there[b * self.bt:(b + 1) * self.bt] = False
                continue
            codes, scales = self.page(p)
            x[:, :, b * self.bt:(b + 1) * self.bt] = codes * scales[:, :, None, None]
        full = L // self.bt * self.bt
        x[:, :, full:] = self.tail[i, :, :, :L - full].double().cpu().transpose(0, 1)
        return x[0], x[1], there

    def attention(self, q, window=0):
        """-> out, lse, weights per sequence [kv_heads][blocks], and |p v| sums and the largest |score| for the error bounds."""
        out = torch.zeros(self.total, self.qh, self.d, dtype=torch.float64)
        spread, lse, top = torch.zeros_like(out), torch.full((self.total, self.qh), -math.inf, dtype=torch.float64), torch.zeros(self.total, self.qh, dtype=torch.float64)
        mass, group = [], self.qh // self.kh
        for i, (L, n) in enumerate(zip(self.lens, self.news)):
            k, v, there = self.held(i)
            w = torch.zeros(self.kh, -(-L // self.bt), dtype=torch.float64)
            sl = slice(self.starts[i], self.starts[i + 1])
            place, token = torch.arange(L - n, L)[:, None], torch.arange(L)[None]
            sees = (token <= place) & there[None]
            if window:
                sees &= token > place - window
            for h in range(self.qh):
                a = h // group
                s = (q[sl, h].double() @ k[a].T) * self.scale
                s = torch.where(sees, s, -math.inf)
                m = s.amax(1, keepdim=True) if L else torch.full((n, 1), -math.inf, dtype=torch.float64)
                e = torch.where(sees, (s - torch.where(m == -math.inf, 0.0, m)).exp(), 0.0)
                z = e.sum(1, keepdim=True)
                p = torch.where(z == 0, 0.0, e / z)
                vv = torch.where(there[:, None], v[a], 0.0)
                seen = sees.any(0)[:, None]
                vv = torch.where(seen, vv, 0.0)
                out[sl, h] = torch.where(p[..., None] == 0, torch.where(sees[..., None], p[..., None] * vv[None], 0.0), p[..., None] * vv[None]).sum(1) if n * L <= 4096 else p @ vv
                spread[sl, h] = p @ vv.abs()
                lse[sl, h] = (m + z.log())[:, 0]
                top[sl, h] = torch.where(sees, s.abs(), 0.0).amax(1) if L else 0.0
                full = torch.zeros(w.shape[1] * self.bt, dtype=torch.float64)
                full[:L] = p.sum(0)
                w[a] += full.view(-1, self.bt).sum(1)
            mass.append(w)
        return out, lse, mass, spread, top

    def run_attention(self, q, out, window=0, mass_in=None, mass_out=None, want_lse=True, stream=None, batch=None):
        b = batch or self.batch()
        need = self.kv.workspace_bytes(b, mass_out is not None)
        ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")         # contents must not matter
        lse = torch.full((self.total, self.qh), 777.0, device="cuda") if want_lse else None
        st = stream or torch.cuda.current_stream()
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        self.kv.attention(b, rows(q), rows(out), ws.data_ptr(), need, d_lse=lse.data_ptr() if want_lse else 0, window=window,
                          d_mass_in=mass_in.data_ptr() if mass_in is not None else 0, d_mass_out=mass_out.data_ptr() if mass_out is not None else 0,
                          mass_stride=mass_out.shape[2] if mass_out is not None else 0, stream=st.cuda_stream)
        st.synchronize()
        return lse

    def check_attention(self, q, out, lse, window=0, mass_in=None, mass_out=None, ref=None):
        """The bounds.  A score is a sum of head_dim products in 32 bits (and, for bf16 queries, of values that were brought to
        11 bits below the row's largest): off by at most 2^-17 (1 + its size).  A probability is off by that share from its
        score, from lse, and by 2^-11 from its rounding to 16 bits (2^-10 is allowed: f16 numbers below the running maximum's
        range are rounded to a fixed step); the answer is then rounded once to the 16-bit type."""
        r_out, r_lse, r_mass, spread, top = ref or self.attention(q.cpu(), window)
        u = UNIT[self.dtype]
        got = out.double().cpu()
        slack = 2.0 ** -17 * (1 + top)
        bound = u * r_out.abs() + (2.0 ** -10 + 4 * slack)[..., None] * spread + 2.0 ** -24 + 2.0 ** -16 * spread.amax(-1, keepdim=True)
        # what the type cannot hold becomes infinite (within the bound of its largest number: either)
        most = torch.finfo(self.t).max
        over = r_out.abs() - bound > most
        assert bool((torch.isinf(got) & (got.sign() == r_out.sign()))[over].all())
        bad = ((got - r_out).abs() > bound) & ~over & ~(torch.isinf(got) & (r_out.abs() + bound > most) & (got.sign() == r_out.sign()))
        assert not bool(bad.any()) and not bool(torch.isnan(got[~torch.isnan(r_out)]).any()), \
            (int(bad.sum()), float(((got - r_out).abs() / bound).max()), bad.nonzero()[:4])
        assert bool((torch.isnan(got) == torch.isnan(r_out)).all())
        if lse is not None:
            g = lse.double().cpu()
            empty = r_lse == -math.inf
            assert bool((g[empty] == -math.inf).all()), "a row that sees nothing"
            fine = ~empty & ~torch.isnan(r_lse)
            assert bool(((g - r_lse).abs() <= slack + 2.0 ** -22 * r_lse.abs())[fine].all()), float((g - r_lse)[fine].abs().max())
        if mass_out is not None:
            for i, w in enumerate(r_mass):
                want = mass_in[i, :, :w.shape[1]].double().cpu() + w
                got = mass_out[i, :, :w.shape[1]].double().cpu()
                worst = float(top[self.starts[i]:self.starts[i + 1]].max()) if self.news[i] else 0.0
                assert bool(((got - want).abs() <= 2.0 ** -15 * (1 + worst) * w + 2.0 ** -22 * want.abs() + 1e-30).all()), (i, float((got - want).abs().max()))
                assert bool((mass_out[i, :, w.shape[1]:] == -5.0).all()), "entries behind the last block were written"


def nearest_code(z, fmt):
    if fmt == kv.INT8:
        return torch.round(z).clamp(-127, 127)
    step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
    return (torch.round(z / step) * step).clamp(-448, 448)


def evict(table, lens, mass, block, budget, first, last):
    """Plain eviction of one batch on the host -> table, lens, mass, evicted, counts."""
    n, stride = table.shape
    t, m, ev = np.full_like(table, -1), np.zeros_like(mass), np.full_like(table, -1)
    new_lens, counts = lens.copy(), np.zeros_like(lens)
    for i in range(n):
        full, held = lens[i] // block, -(-lens[i] // block)
        score = [np.float32(sum(float(mass[i, h, b]) for h in range(mass.shape[1]))) for b in range(full)]
        order = sorted((b for b in range(full) if first <= b < full - last), key=lambda b: (1, 0, b) if np.isnan(score[b]) else (0, score[b], b))
        gone = set(order[:max(0, full - budget)])
        stay = [b for b in range(held) if b not in gone]
        t[i, :len(stay)] = table[i, stay]
        m[i, :, :len(stay)] = mass[i][:, stay]
        ev[i, :len(gone)] = table[i, sorted(gone)]
        new_lens[i] -= len(gone) * block
        counts[i] = len(gone)
    return t, new_lens, m, ev, counts


def ragged(rng: random.Random, n, low, high):
    return [rng.randint(low, high) for _ in range(n)]

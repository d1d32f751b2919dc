"""A key-value cache that gives up its least attended blocks to host memory, sealed, and takes them back:

    python examples/sealed_cache.py

Sequences of random prompts are appended to an 8-bit cache and decoded token by token (rotary positions, append, attention with the
weight that every block received).  Then each sequence is cut to a budget of blocks.  The pages that leave are gathered and go to
page-locked host memory through one ``pipelined_d2h`` call: the context's chunk is one page, so that every page has its own IV and
tag.  A page is quantised once and never changes, so one IV covers one content.  Decoding goes on without them; at the end the pages
are brought back by ``pipelined_h2d``, verified, and the full cache answers bit for bit as it did before.
"""
from __future__ import annotations

import os
import secrets
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_15240_b200 import fastrack, kv  # noqa: E402

SEQS, Q_HEADS, KV_HEADS, DIM, BLOCK, PROMPT, STEPS, BUDGET = 4, 16, 4, 128, 32, 1500, 40, 24


def rows(x):
    return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1))


def main(verbose=True):
    torch.manual_seed(0)
    dev, t = "cuda", torch.bfloat16
    stream = torch.cuda.current_stream().cuda_stream
    frequencies, gain = kv.rotary_frequencies(DIM, 10000.0, kv.FREQ_RAMP, 4.0, 1024.0)
    cache = kv.KvCache(kv.BF16, kv.E4M3, Q_HEADS, KV_HEADS, DIM, BLOCK, rotary=kv.ROTARY_HALF, frequencies=frequencies, rotary_gain=gain)
    lens = [PROMPT - 97 * i for i in range(SEQS)]
    most = max(lens) + STEPS
    stride = -(-most // BLOCK)
    pages = SEQS * stride
    pool = torch.zeros(pages, cache.page_bytes, dtype=torch.uint8, device=dev)
    tail = torch.zeros(SEQS, cache.tail_bytes, dtype=torch.uint8, device=dev)
    table = torch.randperm(pages, dtype=torch.int64).to(torch.int32).view(SEQS, stride).to(dev)      # every block has its page in advance
    d_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    mass = torch.zeros(SEQS, KV_HEADS, stride, device=dev)

    def batch(new):
        starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).to(dev)
        positions = torch.cat([torch.arange(p - n, p) for p, n in zip(lens, new)]).to(dev)
        b = kv.Batch(n_seqs=SEQS, total_new=sum(new), max_new=max(new), max_len=most, pool_pages=pages, table_stride=stride, d_pool=pool.data_ptr(),
                     d_tail=tail.data_ptr(), d_table=table.data_ptr(), d_lens=d_lens.data_ptr(), d_starts=starts.data_ptr(),
                     d_positions=positions.data_ptr())
        return b, (starts, positions)

    def step(new):
        """New tokens of every sequence: q, k, v as one projection would give them -> their answers."""
        b, keep = batch(new)
        qkv = torch.randn(sum(new), Q_HEADS + 2 * KV_HEADS, DIM, device=dev).to(t)
        q, k, v = qkv.split([Q_HEADS, KV_HEADS, KV_HEADS], 1)
        turned, out = torch.empty(sum(new), Q_HEADS, DIM, dtype=t, device=dev), torch.empty(sum(new), Q_HEADS, DIM, dtype=t, device=dev)
        cache.append(b, rows(k), rows(v), rows(q), rows(turned), stream)
        attend(b, turned, out, mass)
        return turned, out, keep

    def attend(b, q, out, weights=None):
        ws = torch.empty(cache.workspace_bytes(b, weights is not None), dtype=torch.uint8, device=dev)
        at = weights.data_ptr() if weights is not None else 0
        cache.attention(b, rows(q), rows(out), ws.data_ptr(), ws.numel(), d_mass_in=at, d_mass_out=at, mass_stride=stride if at else 0, stream=stream)

    step(lens)                                          # the prompts
    for _ in range(STEPS):
        lens = [n + 1 for n in lens]
        d_lens += 1
        q, out, _ = step([1] * SEQS)
    full_table, full_lens = table.clone(), d_lens.clone()

    # the least attended blocks leave
    evicted, count = torch.empty_like(table), torch.empty_like(d_lens)
    cache.evict(kv.Eviction(n_seqs=SEQS, table_stride=stride, mass_stride=stride, budget=BUDGET, keep_first=1, keep_last=2, d_table=table.data_ptr(),
                            d_lens=d_lens.data_ptr(), d_mass=mass.data_ptr(), d_table_out=table.data_ptr(), d_lens_out=d_lens.data_ptr(),
                            d_mass_out=mass.data_ptr(), d_evicted=evicted.data_ptr(), d_n_evicted=count.data_ptr()), stream)
    gone = evicted[evicted >= 0].long()
    n = gone.numel()
    key, iv = secrets.token_bytes(32), secrets.token_bytes(12)
    with fastrack.Context(key, cache.page_bytes) as seal:
        staged = pool.index_select(0, gone)
        cipher, host = torch.empty_like(staged), torch.empty(n, cache.page_bytes, dtype=torch.uint8).pin_memory()
        tags = torch.empty(n, 16, dtype=torch.uint8)
        torch.cuda.synchronize()
        seal.pipelined_d2h(iv, staged.data_ptr(), staged.numel(), cipher.data_ptr(), host.data_ptr(), tags.data_ptr())
        pool[gone] = 0xff                               # the pages may be used for something else

        # decoding goes on over what is left
        b, keep = batch([1] * SEQS)
        small = torch.empty_like(out)
        attend(b, q, small)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(small).all())

        # back again, verified page by page; a byte that the host changed is noticed
        back, ok = torch.empty_like(staged), torch.zeros(n, dtype=torch.int32, device=dev)
        host[n // 2, 1234] ^= 1
        seal.pipelined_h2d(iv, host.data_ptr(), back.numel(), tags.data_ptr(), back.data_ptr(), ok.data_ptr())
        refused = (ok == 0).nonzero().flatten().tolist()
        host[n // 2, 1234] ^= 1
        seal.pipelined_h2d(iv, host.data_ptr(), back.numel(), tags.data_ptr(), back.data_ptr(), ok.data_ptr())
        accepted = bool((ok == 1).all())
        pool[gone] = back
    table.copy_(full_table)
    d_lens.copy_(full_lens)
    b, keep2 = batch([1] * SEQS)
    again = torch.empty_like(out)
    attend(b, q, again)
    torch.cuda.synchronize()
    result = dict(evicted=n, page_bytes=cache.page_bytes, refused=refused, accepted=accepted, same=bool(torch.equal(again, out)),
                  kept_weight=float(mass.sum() / (SEQS * Q_HEADS * STEPS + Q_HEADS * sum(PROMPT - 97 * i for i in range(SEQS)))))
    if verbose:
        print(result)
    return result


if __name__ == "__main__":
    main()

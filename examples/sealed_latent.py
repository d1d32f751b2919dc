"""A latent cache that is decoded with drafted trees and whose full pages leave for host memory, sealed:

    python examples/sealed_latent.py

Prompts are stored (norm, rotary positions), expanded to every head's keys and values, and attended.  Then every step drafts a tree of
tokens per sequence: they are stored behind the cache at the positions of their depths, attended in the latent space, each seeing the
cache and its ancestors, and the path that the (here random) model agrees with is kept.  A page whose tokens are all certain does not
change any more: such pages go to page-locked host memory through one ``pipelined_d2h`` call, a chunk with its own IV and tag each, are
overwritten on the device, come back by ``pipelined_h2d``, verified, and the last step's queries get the same answers, bit for bit.
"""
from __future__ import annotations

import os
import secrets
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2410_15240_b200 import fastrack, kv, latent  # noqa: E402

SEQS, HEADS, LATENT, ROPE, KEY, VALUE, BLOCK, PROMPT, STEPS, DRAFTS = 3, 16, 256, 64, 128, 128, 32, 700, 12, 9


def rows(x):
    return kv.Rows(x.data_ptr(), x.stride(0), x.stride(1) if x.dim() > 2 else 0)


def main(verbose=True):
    torch.manual_seed(0)
    dev, t = "cuda", torch.bfloat16
    stream = torch.cuda.current_stream().cuda_stream
    frequencies, gain = kv.rotary_frequencies(ROPE, 10000.0)
    cache = latent.LatentCache(kv.BF16, HEADS, LATENT, ROPE, KEY, VALUE, BLOCK, rotary=kv.ROTARY_INTERLEAVED, frequencies=frequencies, rotary_gain=gain)
    lens = [PROMPT - 61 * i for i in range(SEQS)]
    most = max(lens) + STEPS * DRAFTS
    stride = -(-most // BLOCK)
    pages = SEQS * stride
    pool = torch.zeros(pages, cache.page_bytes, dtype=torch.uint8, device=dev)
    table = torch.randperm(pages, dtype=torch.int64).to(torch.int32).view(SEQS, stride).to(dev)      # every block has its page in advance
    d_lens = torch.tensor(lens, dtype=torch.int32, device=dev)
    norm = torch.ones(LATENT, dtype=t, device=dev)
    weights = (torch.randn(HEADS, KEY + VALUE, LATENT, device=dev) * LATENT ** -0.5).to(t)

    def batch(new, positions):
        starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32).to(dev)
        b = latent.Batch(n_seqs=SEQS, total_new=sum(new), max_new=max(new), max_len=most, pool_pages=pages, table_stride=stride, d_pool=pool.data_ptr(),
                         d_table=table.data_ptr(), d_lens=d_lens.data_ptr(), d_starts=starts.data_ptr(), d_positions=positions.data_ptr())
        return b, (starts, positions)

    def store(b, total):
        """A projection's output for the new tokens: latents and shared keys are stored, the queries' part is turned."""
        down = torch.randn(total, LATENT + ROPE, device=dev).to(t)
        q = torch.randn(total, HEADS, KEY + ROPE, device=dev).to(t)
        turned = torch.empty(total, HEADS, ROPE, dtype=t, device=dev)
        cache.append(b, rows(down[:, :LATENT]), rows(down[:, LATENT:]), norm.data_ptr(), rows(q[..., KEY:]), rows(turned), stream)
        return down, q[..., :KEY], turned

    def attend(b, q, turned, parents=None):
        """In the latent space: the keys' half of the matrix goes into the queries, the values' half would follow the answers."""
        absorbed = torch.einsum("thk,hkd->thd", q.float(), weights[:, :KEY].float()).to(t)
        out = torch.empty_like(absorbed)
        ws = torch.empty(cache.workspace_bytes(b), dtype=torch.uint8, device=dev)
        cache.attention(b, rows(absorbed), rows(turned), rows(out), ws.data_ptr(), ws.numel(), d_parents=parents.data_ptr() if parents is not None else 0,
                        stream=stream)
        return out

    # the prompts, over expanded keys and values
    b, keep = batch(lens, torch.cat([torch.arange(n) for n in lens]).to(dev))
    _, q, turned = store(b, sum(lens))
    k, v = torch.empty(sum(lens), HEADS, KEY, dtype=t, device=dev), torch.empty(sum(lens), HEADS, VALUE, dtype=t, device=dev)
    key_starts = torch.tensor([sum(lens[:i]) for i in range(SEQS)], dtype=torch.int32, device=dev)
    cache.expand(b, weights.data_ptr(), rows(k), rows(v), key_starts.data_ptr(), sum(lens), stream)
    answers = torch.empty(sum(lens), HEADS, VALUE, dtype=t, device=dev)
    ws = torch.empty(max(16, cache.prompt_workspace_bytes(b)), dtype=torch.uint8, device=dev)
    cache.prompt(b, rows(q), rows(turned), rows(k), rows(v), key_starts.data_ptr(), sum(lens), rows(answers), ws.data_ptr(), ws.numel(), stream=stream)

    # drafted trees: row 0 is the last certain token, the others are children of earlier rows
    kept = 0
    n = [DRAFTS] * SEQS
    for step in range(STEPS):
        parents, depths = [], []
        for _ in range(SEQS):
            p = [-1] + [int(torch.randint(max(0, j - 3), j, ())) for j in range(1, DRAFTS)]
            d = [0]
            for j in range(1, DRAFTS):
                d.append(d[p[j]] + 1)
            parents += p
            depths += d
        old = d_lens.clone()
        d_lens += DRAFTS
        d_parents = torch.tensor(parents, dtype=torch.int32, device=dev)
        b, keep = batch(n, (old.repeat_interleave(DRAFTS) + torch.tensor(depths, device=dev)).long())
        down, q, turned = store(b, sum(n))
        out = attend(b, q, turned, d_parents)
        tokens = torch.randint(0, 3, (sum(n),), dtype=torch.int32, device=dev)
        choices = torch.randint(0, 3, (sum(n),), dtype=torch.int32, device=dev)
        path, count, following = torch.empty_like(tokens), torch.empty_like(d_lens), torch.empty_like(d_lens)
        cache.accept(b, latent.Acceptance(d_parents=d_parents.data_ptr(), d_tokens=tokens.data_ptr(), d_choices=choices.data_ptr(), d_path=path.data_ptr(),
                                          d_n_accepted=count.data_ptr(), d_next=following.data_ptr(), d_lens_out=d_lens.data_ptr()), stream)
        kept += int(count.sum())
    # what is left of the last tree is a chain at the end of the cache: the accepted rows' queries see it as they saw their ancestors
    news = count.tolist()
    accepted = torch.cat([path[DRAFTS * i:DRAFTS * i + c].long() + DRAFTS * i for i, c in enumerate(news)])
    b, keep2 = batch(news, torch.zeros(sum(news), dtype=torch.int64, device=dev))
    again = attend(b, q[accepted], turned[accepted])
    chain_error = float((again.float() - out[accepted].float()).abs().max())

    # full pages of certain tokens leave, sealed, and come back
    gone = torch.cat([table[i, :int(d_lens[i]) // BLOCK] for i in range(SEQS)]).long()
    count_gone = gone.numel()
    key, iv = secrets.token_bytes(32), secrets.token_bytes(12)
    with fastrack.Context(key, cache.page_bytes) as seal:
        staged = pool.index_select(0, gone)
        cipher, host = torch.empty_like(staged), torch.empty(count_gone, cache.page_bytes, dtype=torch.uint8).pin_memory()
        tags = torch.empty(count_gone, 16, dtype=torch.uint8)
        torch.cuda.synchronize()
        seal.pipelined_d2h(iv, staged.data_ptr(), staged.numel(), cipher.data_ptr(), host.data_ptr(), tags.data_ptr())
        pool[gone] = 0xff
        back, ok = torch.empty_like(staged), torch.zeros(count_gone, dtype=torch.int32, device=dev)
        host[count_gone // 2, 77] ^= 1                  # a byte that the host changed is noticed
        seal.pipelined_h2d(iv, host.data_ptr(), back.numel(), tags.data_ptr(), back.data_ptr(), ok.data_ptr())
        refused = (ok == 0).nonzero().flatten().tolist()
        host[count_gone // 2, 77] ^= 1
        seal.pipelined_h2d(iv, host.data_ptr(), back.numel(), tags.data_ptr(), back.data_ptr(), ok.data_ptr())
        pool[gone] = back
    b, keep2 = batch(news, torch.zeros(sum(news), dtype=torch.int64, device=dev))
    last = attend(b, q[accepted], turned[accepted])
    torch.cuda.synchronize()
    result = dict(pages=count_gone, page_bytes=cache.page_bytes, kept=kept, refused=refused, accepted=bool((ok == 1).all()), same=bool(torch.equal(last, again)),
                  chain_error=chain_error, finite=bool(torch.isfinite(answers).all()))
    if verbose:
        print(result)
    return result


if __name__ == "__main__":
    main()

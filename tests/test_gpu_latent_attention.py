"""Attention in the latent space against its definition."""
import math
import random

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from latent_reference import Cache, attend, bounds, rows, strided, visible  # noqa: E402
from paper_2410_15240_b200 import kv, latent  # noqa: E402

pytestmark = pytest.mark.gpu
GUARD = -3.0


def trees(news, seed):
    r = random.Random(seed)
    return [[-1] + [r.randint(max(0, j - 5), j - 1) for j in range(1, n)] for n in news]


def run(c, q, q_rope, parents=None, stream=None):
    """-> answers and lse on the CPU; what lies around them stays as it was."""
    total = c.total
    room = torch.full((total + 2, c.heads + 1, c.dim + 8), GUARD, dtype=c.t, device="cuda")
    out = room[1:-1, :c.heads, :c.dim]
    lse_room = torch.full((total * c.heads + 2,), GUARD, device="cuda")
    ws = torch.full((c.handle.workspace_bytes(c.batch) + 64,), 0xff, dtype=torch.uint8, device="cuda")
    d_parents = torch.tensor(sum(parents, []), dtype=torch.int32, device="cuda") if parents else None
    c.handle.attention(c.batch, rows(q), rows(q_rope), rows(out), ws.data_ptr(), ws.numel() - 64, d_lse=lse_room[1:].data_ptr(),
                       d_parents=d_parents.data_ptr() if parents else 0, stream=stream or torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    kept = out.clone()
    out.fill_(GUARD)
    assert bool((room == GUARD).all()) and float(lse_room[0]) == GUARD and float(lse_room[-1]) == GUARD and bool((ws[-64:] == 0xff).all())
    return kept.cpu(), lse_room[1:-1].view(total, c.heads).cpu()


def check(c, q, q_rope, out, lse, parents=None, seqs=None):
    qf = torch.cat([q, q_rope], 2).double().cpu()
    for i in seqs if seqs is not None else range(len(c.lens)):
        n, L, st = c.news[i], c.lens[i], c.starts[i]
        if n == 0:
            continue
        x, there = c.held(i)
        sees = visible(n, L, parents[i] if parents else None) & there
        spread = x[:, :c.dim].abs().sum(0)
        for h in range(c.heads):
            want, want_lse, weighed, size = attend(qf[st:st + n, h], x, x[:, :c.dim], sees, c.scale)
            bound = bounds(c.dtype, want, weighed, size, spread, L)
            got = out[st:st + n, h].double()
            assert bool(((got - want).abs() <= bound).all()), (i, h, float(((got - want).abs() / bound).max()))
            some = sees.any(1)
            assert bool((lse[st:st + n, h][~some] == -math.inf).all()) and bool((got[~some] == 0).all())
            # the sum's error, and the logarithm's rounding
            off = (lse[st:st + n, h].double() - want_lse)[some].abs()
            assert bool((off <= (40 * 2.0 ** -23 * size + 2.0 ** -19 + 2.0 ** -23 * want_lse.abs() + L * 2.0 ** -26)[some]).all()), float(off.max())


def queries(c, size=1.0):
    q = strided((size * torch.randn(c.total, c.heads, c.dim, generator=c.gen)).to(c.t).cuda())
    return q, strided((size * torch.randn(c.total, c.heads, c.rope, generator=c.gen)).to(c.t).cuda(), 16)


CASES = [
    # heads, dim, rope, block, lens, news
    (16, 512, 64, 64, [700], [1]),
    (128, 512, 64, 64, [1, 63, 64, 65, 300], [1, 1, 1, 1, 1]),
    (1, 128, 32, 16, [5, 1, 200], [1, 1, 1]),
    (5, 256, 64, 32, [33, 0, 90, 17], [3, 0, 0, 17]),
    (12, 384, 32, 128, [129, 1000], [7, 2]),
    (40, 512, 32, 16, [100, 31], [9, 31]),
    (64, 128, 64, 64, [4000], [1]),
    (7, 512, 64, 128, [260, 2, 77], [70, 2, 1]),
    (100, 256, 32, 32, [95], [13]),
    (1024, 128, 32, 16, [50], [2]),
]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,dim,rope,block,lens,news", CASES)
def test_chain(dtype, heads, dim, rope, block, lens, news):
    c = Cache(dtype, heads, dim, rope, block, lens, news, seed=heads + dim)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    check(c, q, q_rope, out, lse)


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,dim,rope,block,lens,news", [
    (16, 512, 64, 16, [333, 25, 90], [25, 25, 1]), (3, 128, 32, 64, [200, 150], [130, 150]), (128, 256, 64, 128, [64, 65, 200], [4, 9, 17]),
    (2, 512, 64, 32, [700], [300])])
def test_tree(dtype, heads, dim, rope, block, lens, news):
    c = Cache(dtype, heads, dim, rope, block, lens, news, seed=heads)
    parents = trees(news, heads)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope, parents)
    check(c, q, q_rope, out, lse, parents)


def test_parents_that_are_none():
    """Anything but an earlier row makes a root: no call walks in circles or out of the tree."""
    c = Cache(kv.BF16, 4, 128, 32, 16, [40], [6])
    parents = [[5, -9, 2, 1, 1000, 4]]
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope, parents)
    check(c, q, q_rope, out, lse, parents)
    chain = [[-1, 0, 1, 2, 3, 4]]
    out, lse = run(c, q, q_rope, chain)
    plain, plain_lse = run(c, q, q_rope)
    assert torch.equal(out, plain) and torch.equal(lse, plain_lse)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_absent_pages(block):
    lens, news = [400, 300, 2 * block, block], [1, 5, 2, 1]
    absent = [(0, 0), (0, 300 // block), (1, 299 // block), (2, 0), (3, 0)]
    c = Cache(kv.BF16, 16, 256, 64, block, lens, news, absent=absent, seed=block)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    check(c, q, q_rope, out, lse)


@pytest.mark.parametrize("heads,tree", [(16, False), (128, False), (16, True)])
@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
def test_what_is_hidden_does_not_count(dtype, heads, tree):
    """Unused rows of pages hold NaN and infinities, and so do new tokens that some queries do not see."""
    lens, news = [150, 70, 130], [9, 6, 1]
    c = Cache(dtype, heads, 512, 64, 32, lens, news, seed=3)
    parents = trees(news, 5) if tree else None
    for p in range(c.pages):
        if p not in set(c.table.flatten().tolist()):
            c.pool[p] = math.nan
    for i, n in enumerate(lens):
        if n % 32:
            c.pool[c.page(i, n - 1), n % 32:] = torch.tensor([math.nan, math.inf, -math.inf, 1.0]).repeat(c.row // 4).to(c.t)
    # new tokens 4 and 7 of the first sequence
    for j, value in ((4, math.inf), (7, math.nan)):
        place = lens[0] - news[0] + j
        c.pool[c.page(0, place), place % 32, 17 + j] = value
    c.upload()
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope, parents)
    check(c, q, q_rope, out, lse, parents, seqs=[1, 2])
    x, _ = c.held(0)
    sees = visible(news[0], lens[0], parents[0] if tree else None)
    qf = torch.cat([q, q_rope], 2).double().cpu()
    at = lens[0] - news[0]
    for j in range(news[0]):
        seen = sees[j]
        hit = [t for t in (4, 7) if bool(seen[at + t])]
        for h in range(heads):
            if not hit:
                want, _, weighed, size = attend(qf[j:j + 1, h], x[seen], x[seen, :512], torch.ones(1, int(seen.sum()), dtype=torch.bool), c.scale)
                bound = bounds(dtype, want, weighed, size, x[seen, :512].abs().sum(0), lens[0])
                assert bool(((out[j, h].double() - want[0]).abs() <= bound[0]).all()), (j, h)
            elif 7 in hit:
                assert bool(out[j, h].isnan().all()) and math.isnan(float(lse[j, h])), (j, h)
            else:
                # a score of +infinity, which has no softmax, or -infinity, which counts for nothing
                score = float(qf[j, h] @ x[at + 4])
                if score > 0:
                    assert bool(out[j, h].isnan().all()), (j, h)
                else:
                    there = seen.clone()
                    there[at + 4] = False
                    want, _, weighed, size = attend(qf[j:j + 1, h], x[there], x[there, :512], torch.ones(1, int(there.sum()), dtype=torch.bool), c.scale)
                    bound = bounds(dtype, want, weighed, size, x[there, :512].abs().sum(0), lens[0])
                    off = (out[j, h].double() - want[0]).abs() <= bound[0]
                    off[17 + 4] = True
                    assert bool(off.all()), (j, h)


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
def test_large_scores_and_rising_ones(dtype):
    """References that rise tile by tile, and scores of some thousands: one token takes all."""
    c = Cache(dtype, 16, 256, 64, 64, [1500, 64 * 9], [1, 3], seed=8, softmax_scale=0.5)
    for i in range(2):
        for b in range(c.lens[i] // 64):
            c.pool[c.page(i, 64 * b)] *= 0.2 + 0.15 * b
    c.upload()
    q, q_rope = queries(c, 2.0)
    out, lse = run(c, q, q_rope)
    check(c, q, q_rope, out, lse)


def test_a_query_that_is_not_finite_spoils_only_its_own_answer():
    c = Cache(kv.BF16, 16, 512, 64, 64, [300], [5])
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    q[2, 3, 100] = math.nan
    q_rope[4, 15, 0] = math.inf
    again, lse2 = run(c, q, q_rope)
    bad = torch.zeros(5, 16, dtype=torch.bool)
    bad[2, 3] = bad[4, 15] = True
    assert torch.equal(again[~bad], out[~bad]) and torch.equal(lse2[~bad], lse[~bad])
    assert bool(again[bad].isnan().all())


def test_odd_numbers_from_the_device():
    """Lengths, starts and pages out of bounds touch nothing outside the buffers; other sequences answer as before."""
    c = Cache(kv.BF16, 16, 128, 32, 16, [100, 60, 33], [2, 3, 1])
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    c.d_lens[1] = 1 << 30
    c.d_table[1, 2] = 1 << 30
    again, _ = run(c, q, q_rope)
    assert torch.equal(again[:2], out[:2]) and torch.equal(again[5:], out[5:])
    c.d_lens[1] = -5                    # queries in front of every token
    again, again_lse = run(c, q, q_rope)
    assert torch.equal(again[:2], out[:2]) and torch.equal(again[5:], out[5:])
    assert bool((again[2:5] == 0).all()) and bool((again_lse[2:5] == -math.inf).all())


@pytest.mark.parametrize("lens", [[20000], [9000, 17, 4000, 1, 12345], [700] * 40])
def test_cut_work_is_the_same_in_every_run_and_company(lens):
    """Long sequences are cut into pieces; the answer does not change from run to run."""
    c = Cache(kv.BF16, 16, 512, 64, 64, lens, [1] * len(lens), seed=1)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    check(c, q, q_rope, out, lse, seqs=range(min(5, len(lens))))
    again, lse2 = run(c, q, q_rope)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_bounds_larger_than_the_batch():
    """max_new, max_len and total_new are bounds: graphs are captured with them."""
    c = Cache(kv.F16, 16, 256, 32, 32, [300, 45], [3, 1], seed=2)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    d = Cache(kv.F16, 16, 256, 32, 32, [300, 45], [3, 1], seed=2, max_new=4, max_len=1024)
    d.batch.max_new, d.batch.max_len = 4, 1024
    again, lse2 = run(d, q, q_rope)
    check(d, q, q_rope, again, lse2)


def test_many_sequences():
    lens = [(37 * i) % 90 for i in range(2500)]
    news = [1 if n else 0 for n in lens]
    c = Cache(kv.BF16, 8, 128, 64, 32, lens, news, seed=6)
    q, q_rope = queries(c)
    out, lse = run(c, q, q_rope)
    check(c, q, q_rope, out, lse, seqs=range(0, 2500, 97))


def test_captured_and_on_another_stream():
    c = Cache(kv.BF16, 128, 512, 64, 64, [3000, 500], [1, 1], seed=4)
    q, q_rope = queries(c)
    want, want_lse = run(c, q, q_rope)
    out, lse = torch.empty(c.total, c.heads, c.dim, dtype=c.t, device="cuda"), torch.empty(c.total, c.heads, device="cuda")
    ws = torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda")
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        c.handle.attention(c.batch, rows(q), rows(q_rope), rows(out), ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(),
                           stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.cpu(), want) and torch.equal(lse.cpu(), want_lse)
    c.d_lens.copy_(torch.tensor([1200, 64], dtype=torch.int32))            # the graph reads the lengths again
    graph.replay()
    torch.cuda.synchronize()
    c.lens = [1200, 64]
    check(c, q, q_rope, out.cpu(), lse.cpu())

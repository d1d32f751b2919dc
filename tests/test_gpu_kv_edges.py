"""The cache operators where they can go wrong: what a query does not see must not reach it, whatever stands there; sizes and
windows at the ends of what the header allows."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from kv_reference import UNIT, Cache, rows  # noqa: E402
from paper_2410_15240_b200 import kv  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim", [64, 128])
def test_read_of_more_than_2_31_pieces(dim):
    """A sequence whose rows count more pieces of 8 channels than 31 bits do.  Rows 8 channels apart (what they share holds the same
    number): 16 bytes a token.  All pages are absent but the last, whose codes are all alike."""
    block, held_page = 128, 3
    max_len = (1 << 31) * 8 // dim + 1000
    cache = kv.KvCache(kv.BF16, kv.INT8, 1, 1, dim, block)
    blocks = max_len // block
    table = torch.full((1, blocks), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = held_page
    pool = torch.full((5, cache.page_bytes), 255, dtype=torch.uint8, device="cuda")
    codes = block * dim
    pool[held_page, :2 * codes] = 3
    pool[held_page, 2 * codes:2 * codes + 8].view(torch.float32)[:] = 0.5
    tail = torch.full((cache.tail_bytes // 2,), 1.5, dtype=torch.bfloat16, device="cuda")
    lens, starts = torch.tensor([max_len], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    guard, size = 1 << 20, 8 * (max_len - 1) + dim
    out = torch.full((guard + size + guard,), -7.0, dtype=torch.bfloat16, device="cuda")
    b = kv.Batch(n_seqs=1, total_new=0, max_new=0, max_len=max_len, pool_pages=5, table_stride=blocks, d_pool=pool.data_ptr(), d_tail=tail.data_ptr(),
                 d_table=table.data_ptr(), d_lens=lens.data_ptr(), d_starts=starts.data_ptr())
    to = kv.Rows(out[guard:].data_ptr(), 8, 8)
    cache.read(b, to, to)
    torch.cuda.synchronize()
    assert bool((out[:guard] == -7).all()) and bool((out[guard + size:] == -7).all())
    rows_ = out[guard:guard + size]
    page, rest = 8 * (blocks - 1) * block, 8 * blocks * block   # first values of the page's tokens and of the unfinished block's
    assert bool((rows_[:page] == 0).all())                      # absent
    assert bool((rows_[page + dim:rest] == 1.5).all())          # 3 x 0.5
    assert bool((rows_[rest + dim:] == 1.5).all())


@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("window", [900, 1 << 30, (1 << 31) - 1])
def test_window_that_hides_nothing(new, window):
    """A window of max_len tokens or more, up to the largest number, is none: same answers, same weights."""
    c = Cache(kv.BF16, kv.INT8, 8, 2, 64, 32, [900, new + 3], [new, new])
    c.fill()
    gen = torch.Generator().manual_seed(1)
    q = torch.randn(c.total, c.qh, c.d, generator=gen).to(c.t).cuda()
    got = []
    for w in (0, window):
        out, m_out = torch.empty_like(q), torch.full((c.n, c.kh, 30), -5.0, device="cuda")
        m_in = torch.zeros_like(m_out)
        lse = c.run_attention(q, out, w, m_in, m_out)
        got.append((out, lse, m_out))
    c.check_attention(q, got[0][0], got[0][1], 0, m_in, got[0][2])
    for a, b in zip(*got):
        assert torch.equal(a, b)


def test_one_handle_on_several_threads_and_streams():
    """A handle holds constants only: threads with streams, batches and workspaces of their own use it at the same time."""
    import threading
    c = Cache(kv.BF16, kv.E4M3, 8, 2, 128, 64, [5000, 1200, 333], [5, 5, 5])
    c.fill()
    gen = torch.Generator().manual_seed(3)
    qs = [torch.randn(c.total, c.qh, c.d, generator=gen).to(c.t).cuda() for _ in range(4)]
    want = [torch.empty_like(q) for q in qs]
    for q, w in zip(qs, want):
        c.run_attention(q, w)
    outs, failed = [[torch.empty_like(q) for _ in range(20)] for q in qs], []
    need = c.kv.workspace_bytes(c.batch(), False)
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    torch.cuda.synchronize()

    def work(i):
        try:
            b = c.batch()
            for o in outs[i]:
                c.kv.attention(b, rows(qs[i]), rows(o), spaces[i].data_ptr(), need, stream=streams[i].cuda_stream)
            streams[i].synchronize()
        except Exception as e:                          # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(qs))]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert not failed and not any(t.is_alive() for t in threads)
    torch.cuda.synchronize()
    for w, got in zip(want, outs):
        assert all(torch.equal(w, o) for o in got)


def definition(c, q, window=0):
    """Attention in 64 bits where values may be infinite or NaN: a token counts for the rows that see it, and for no other.
    -> out, lse, the sums of |p v| over finite values, the largest |score|."""
    out, spread = (torch.zeros(c.total, c.qh, c.d, dtype=torch.float64) for _ in range(2))
    lse, top = torch.full((c.total, c.qh), -math.inf, dtype=torch.float64), torch.zeros(c.total, c.qh, dtype=torch.float64)
    for i, (L, n) in enumerate(zip(c.lens, c.news)):
        k, v, there = c.held(i)
        sl = slice(c.starts[i], c.starts[i + 1])
        place, token = torch.arange(L - n, L)[:, None], torch.arange(L)[None]
        sees = (token <= place) & there[None]
        if window:
            sees &= token > place - window
        for h in range(c.qh):
            a = h // (c.qh // c.kh)
            s = torch.where(sees, (q[sl, h].double().cpu() @ k[a].T) * c.scale, -math.inf)
            p = torch.softmax(s, 1)
            fine = torch.where(torch.isfinite(v[a]), v[a], 0.0)
            o = p @ fine
            for t in (~torch.isfinite(v[a])).any(1).nonzero().flatten().tolist():
                o = torch.where(sees[:, t, None] & ~torch.isfinite(v[a, t])[None], o + v[a, t][None], o)
            out[sl, h], spread[sl, h] = o, p @ fine.abs()
            lse[sl, h] = torch.logsumexp(s, 1)
            top[sl, h] = torch.where(torch.isfinite(s), s.abs(), 0.0).amax(1)
    return out, lse, spread, top


def compare(c, got, lse, want, least=2.0 ** -24):
    """The bounds of Cache.check_attention, but for its share of the row's largest |p v|; `least`: what the type's smallest step may add.
    Infinities and NaN have to be where the definition has them."""
    r_out, r_lse, spread, top = want
    g, slack = got.double().cpu(), 2.0 ** -17 * (1 + top)
    assert torch.equal(torch.isnan(g), torch.isnan(r_out)), "NaN"
    assert torch.equal(torch.isinf(g), torch.isinf(r_out)) and bool((g.sign() == r_out.sign())[torch.isinf(r_out)].all()), "infinite"
    fine = torch.isfinite(r_out)
    bound = UNIT[c.dtype] * r_out.abs() + (2.0 ** -10 + 4 * slack)[..., None] * spread + least + 2.0 ** -16 * spread.amax(-1, keepdim=True)
    bad = ((g - r_out).abs() > bound) & fine
    assert not bool(bad.any()), (int(bad.sum()), bad.nonzero()[:4].tolist(), float(((g - r_out).abs() / bound)[fine].max()))
    fine = torch.isfinite(r_lse)
    assert torch.equal(torch.isnan(lse.double().cpu()), torch.isnan(r_lse))
    assert bool(((lse.double().cpu() - r_lse).abs() <= slack + 2.0 ** -22 * r_lse.abs())[fine].all())


def attend(c, seed=5, scale=2.0, window=0):
    gen = torch.Generator().manual_seed(seed)
    q = (scale * torch.randn(c.total, c.qh, c.d, generator=gen)).to(c.t).cuda()
    out = torch.full_like(q, -7.0)
    return q, out, c.run_attention(q, out, window)


@pytest.mark.parametrize("new", [1, 5, 150])
@pytest.mark.parametrize("size", [2.0 ** -100, 2.0 ** -119, 1e-37, 1e-40])
def test_tiny_values_in_the_unfinished_block(new, size):
    """V far below what a page would hold, alone in the cache and beside pages: small answers, not infinite ones."""
    c = Cache(kv.BF16, kv.INT8, 4, 2, 128, 64, [new + 40, new + 64 - new % 64 + 9], [new, new])
    c.fill()
    c.tail[:, :, 1] *= size
    if new < 24:
        c.pool[:, 2 * c.codes:2 * c.codes + 8 * c.kh].view(torch.float32).view(c.pages, c.kh, 2)[..., 1] = 2.0 ** -100
    q, out, lse = attend(c)
    # where all of V is small: steps of 2^-133, and 16 bits of f16 at 2^-25 of a page's smallest power
    compare(c, out, lse, definition(c, q), least=2.0 ** -118 if new < 24 else 2.0 ** -24)


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("new,group,block", [(1, 4, 64), (5, 1, 16), (5, 8, 32), (150, 2, 64)])
def test_zeros_in_the_unfinished_block_cost_nothing(dtype, new, group, block):
    """V of zeros (no matter at what power of two they are held) beside pages with small scales, whose answers keep their bits."""
    c = Cache(dtype, kv.INT8, 2 * group, 2, 128, block, [new + 6 * block - new % block + 9] * 2, [new] * 2)
    c.fill(spread=0.3)
    c.tail[:, :, 1] = 0
    small = 2.0 ** (-46 if dtype == kv.BF16 else -17)
    c.pool[:, 2 * c.codes:2 * c.codes + 8 * c.kh].view(torch.float32).view(c.pages, c.kh, 2)[..., 1] *= small
    q, out, lse = attend(c)
    compare(c, out, lse, definition(c, q), least=2.0 ** -25 if dtype == kv.F16 else 2.0 ** -90)


@pytest.mark.parametrize("dtype,ratio", [(kv.BF16, 2.0 ** 45), (kv.BF16, 2.0 ** 80), (kv.F16, 2.0 ** 24)])
@pytest.mark.parametrize("fmt", [kv.INT8, kv.E4M3])
@pytest.mark.parametrize("new,group,window", [(5, 1, 100), (16, 1, 100), (5, 3, 100), (8, 8, 100), (150, 2, 0), (150, 2, 100), (300, 1, 0)])
def test_a_page_that_some_rows_do_not_see(dtype, ratio, fmt, new, group, window):
    """One page's V is larger than all others' by orders of magnitude: rows that do not see it answer as without it."""
    block = 16
    L = 320 + new
    first = L - new                                     # place of the first new token
    # the page is at the first row's window's edge (its last token is seen by the first row only), or full of new tokens
    big = (first - window + 1) // block if window else (first + new // 2) // block
    if window:
        L += (big * block + block - 1) - (first - window + 1)
    c = Cache(dtype, fmt, 2 * group, 2, 64, block, [L, L], [new] * 2, seed=4)
    c.fill(spread=0.3)
    scales = c.pool[:, 2 * c.codes:2 * c.codes + 8 * c.kh].view(torch.float32).view(c.pages, c.kh, 2)
    scales[..., 1] *= 2.0 ** -14 if dtype == kv.F16 else 2.0 ** -20
    scales[int(c.table[0, big]), :, 1] *= ratio
    q, out, lse = attend(c, window=window)
    want = definition(c, q, window)
    block_seen = want[2].amax((1, 2))[:new] > 2 * want[2].amax((1, 2))[new:].max()
    assert bool(block_seen.any()) and not bool(block_seen.all())         # the case is what it says
    got = out
    if dtype == kv.F16:                                 # what the type cannot hold
        over = want[0].abs() > 60000
        got = torch.where(over.cuda(), want[0].cuda(), out.double())
    compare(c, got, lse, want, least=2.0 ** -25 if dtype == kv.F16 else 2.0 ** -90)


@pytest.mark.parametrize("new", [1, 5, 150])
def test_a_page_of_large_values_and_little_weight(new):
    """One page's V is larger by 2^60, and its tokens' weights are smaller by more than that."""
    c = Cache(kv.BF16, kv.E4M3, 4, 2, 64, 16, [new + 300] * 2, [new] * 2, seed=6)
    c.fill(spread=0.3)
    q = torch.ones(c.total, c.qh, c.d, dtype=c.t, device="cuda")
    page, scales = int(c.table[0, 5]), c.pool[:, 2 * c.codes:2 * c.codes + 8 * c.kh].view(torch.float32).view(c.pages, c.kh, 2)
    scales[page, :, 1] *= 2.0 ** 60
    scales[page, :, 0] = 1.0
    codes = torch.full((c.codes,), -8.0).to(torch.float8_e4m3fn)         # scores of -64 (the others': within a few of 0)
    c.pool[page, :c.codes] = codes.view(torch.uint8).cuda()
    out = torch.full_like(q, -7.0)
    lse = c.run_attention(q, out)
    compare(c, out, lse, definition(c, q), least=2.0 ** -90)


SPOIL = [math.nan, math.inf, -math.inf, 2.0 ** 60]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("value", SPOIL)
@pytest.mark.parametrize("new,group,block", [(5, 1, 64), (3, 5, 16), (5, 8, 64), (150, 2, 128), (100, 1, 128)])
def test_k_of_later_tokens(dtype, value, new, group, block):
    """An infinite, NaN or huge K of the last new token reaches no query that does not see it."""
    if dtype == kv.F16 and value == 2.0 ** 60:
        value = 65504.0
    c = Cache(dtype, kv.E4M3, 2 * group, 2, 64, block, [3 * block + block - 1, max(new, block + 7)], [new, new])
    c.fill()
    for i, L in enumerate(c.lens):
        c.tail[i, :, 0, L % block - 1] = value
    q, out, lse = attend(c)
    want = definition(c, q)
    last = torch.tensor([s - 1 for s in c.starts[1:]])
    keep = torch.ones(c.total, dtype=torch.bool)
    keep[last] = False
    assert bool(torch.isfinite(want[0][keep]).all())
    sub = tuple(x[keep] for x in want)
    compare(c, out[keep.cuda()], lse[keep.cuda()], sub)
    if math.isnan(value):
        assert bool(torch.isnan(out[last.cuda()]).all())


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("new,group", [(1, 4), (5, 8), (150, 1)])
def test_a_score_of_minus_infinity(dtype, new, group):
    """A seen token whose score is -infinity has no weight, and the others have the weights that they have without it."""
    c = Cache(dtype, kv.INT8, 2 * group, 2, 64, 64, [64 + 40 + new - new % 64 if new > 24 else 104, 20 + new], [new, new])
    c.fill()
    q = torch.full((c.total, c.qh, c.d), 0.25, dtype=c.t, device="cuda")
    c.tail[:, :, 0, 3, 5] = -math.inf
    out = torch.full_like(q, -7.0)
    lse = c.run_attention(q, out)
    compare(c, out, lse, definition(c, q))


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 2.0 ** 100])
@pytest.mark.parametrize("new,group,block", [(1, 4, 64), (5, 1, 64), (3, 5, 16), (5, 8, 64), (150, 2, 128), (100, 1, 128)])
def test_v_of_later_tokens(dtype, value, new, group, block):
    """An infinite, NaN or huge V of the last new token reaches no query that does not see it, and shows in those that do, in its
    channels."""
    if dtype == kv.F16 and value == 2.0 ** 100:
        value = 65504.0
    c = Cache(dtype, kv.E4M3, 2 * group, 2, 64, block, [3 * block + block - 1, max(new, block + 7)], [new, new])
    c.fill()
    for i, L in enumerate(c.lens):
        c.tail[i, :, 1, L % block - 1, 3:50] = value
    q, out, lse = attend(c)
    compare(c, out, lse, definition(c, q))


@pytest.mark.parametrize("new,group", [(5, 2), (150, 1)])
def test_infinities_of_both_signs(new, group):
    """Where a query sees both, NaN; where it sees one, that one."""
    c = Cache(kv.F16, kv.INT8, 2 * group, 2, 96, 32, [new + 96 - new % 32 + 20] * 2, [new, new])
    c.fill()
    rest = c.lens[0] % 32
    c.tail[:, :, 1, rest - 3, 7] = math.inf
    c.tail[:, :, 1, rest - 2, 7] = -math.inf
    c.tail[:, :, 1, rest - 2, 90] = -math.inf
    c.tail[1, :, 1, 0, 33] = math.nan
    q, out, lse = attend(c)
    compare(c, out, lse, definition(c, q))


@pytest.mark.parametrize("new,group,block", [(1, 4, 64), (5, 8, 128), (150, 2, 128)])
def test_values_of_very_different_sizes(new, group, block):
    """V of tokens that a query does not see may be larger by any power."""
    c = Cache(kv.BF16, kv.INT8, 2 * group, 2, 64, block, [block + block - 3, max(new, block - 2)], [new, new], seed=9)
    c.fill()
    power = torch.exp2(torch.arange(block, device="cuda").float() * 0.5)[:, None]      # later ones larger, up to 2^63
    c.tail[:, :, 1] = torch.where(torch.isnan(c.tail[:, :, 1]), c.tail[:, :, 1], c.tail[:, :, 1] * power)
    q, out, lse = attend(c)
    compare(c, out, lse, definition(c, q))


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("new,group,block,window", [(1, 4, 64, 0), (5, 2, 16, 0), (150, 2, 128, 0), (150, 1, 64, 0), (100, 3, 16, 0), (140, 1, 32, 90)])
def test_weights_beside_tokens_of_very_different_sizes(dtype, new, group, block, window):
    """Answers, sums and block weights where the unfinished block's tokens differ by up to 2^12 in K and in V."""
    c = Cache(dtype, kv.E4M3, 2 * group, 2, 64, block, [3 * block + new - new % block + block - 2, max(new, block - 1)], [new, new], seed=12)
    c.fill()
    gen = torch.Generator().manual_seed(2)
    for which in range(2):
        power = torch.exp2(-torch.randint(0, 13, (c.n, 1, block, 1), generator=gen).float()).cuda()
        c.tail[:, :, which] *= power
    q = torch.randn(c.total, c.qh, c.d, generator=gen).to(c.t).cuda()
    out, stride = torch.full_like(q, -7.0), -(-c.max_len // block) + 1
    m_in = torch.rand(c.n, c.kh, stride, device="cuda")
    m_out = torch.full_like(m_in, -5.0)
    lse = c.run_attention(q, out, window, m_in, m_out)
    c.check_attention(q, out, lse, window, m_in, m_out)


@pytest.mark.parametrize("new,window", [(1, 0), (140, 0), (140, 200)])
def test_scores_beyond_the_last_whole_number(new, window):
    """Scores up to 2^28, where a float's steps are whole numbers: one token takes all, and no weight leaves f16's range."""
    c = Cache(kv.BF16, kv.INT8, 4, 2, 128, 32, [800, 333], [new, new], scale=3.0, seed=3)
    c.fill(spread=4.0)
    gen = torch.Generator().manual_seed(2)
    q = (3 * torch.randn(c.total, c.qh, c.d, generator=gen)).to(c.t).cuda()
    out = torch.full_like(q, -7.0)
    m_in = torch.rand(c.n, c.kh, 26, device="cuda")
    m_out = torch.full_like(m_in, -5.0)
    lse = c.run_attention(q, out, window, m_in, m_out)
    c.check_attention(q, out, lse, window, m_in, m_out)


@pytest.mark.parametrize("new,lens,window", [(1, [70000, 65000], 0), (1, [30000], 2000), (5, [3000, 2500], 0), (150, [2000], 0), (150, [900, 800], 300)])
def test_graph_capture_with_joins_and_weights(new, lens, window):
    """The paths whose later launches start under the earlier ones, replayed in a graph behind kernels that change their input."""
    c = Cache(kv.BF16, kv.INT8, 8, 1, 128, 64, lens, [new] * len(lens))
    c.fill()
    gen = torch.Generator().manual_seed(3)
    inputs = [torch.randn(c.total, c.qh, c.d, generator=gen).to(c.t).cuda() for _ in range(2)]
    q, out, lse = inputs[0].clone(), torch.empty_like(inputs[0]), torch.empty(c.total, c.qh, device="cuda")
    stride = -(-c.max_len // c.bt)
    m_in, m_out = torch.rand(c.n, c.kh, stride, device="cuda"), torch.empty(c.n, c.kh, stride, device="cuda")
    b = c.batch()
    ws = torch.empty(c.kv.workspace_bytes(b, True), dtype=torch.uint8, device="cuda")
    plain = []
    for x in inputs:
        o, m = torch.empty_like(out), torch.full_like(m_out, -5.0)
        plain.append((o, c.run_attention(x, o, window, m_in, m), m))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph, fresh = torch.cuda.CUDAGraph(), torch.empty_like(q)
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            q.copy_(fresh)
            c.kv.attention(b, rows(q), rows(out), ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(), window=window, d_mass_in=m_in.data_ptr(),
                           d_mass_out=m_out.data_ptr(), mass_stride=stride, stream=stream.cuda_stream)
            kept = [x.clone() for x in (out, lse, m_out)]
    for k in (0, 1, 0, 1):
        fresh.copy_(inputs[k])
        m_out.fill_(-5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, w in zip(kept, plain[k]):
            assert torch.equal(a, w)


@pytest.mark.parametrize("new", [3, 150])
def test_no_tokens_at_all(new):
    """max_len 0: nothing is held, every query sees nothing."""
    c = Cache(kv.F16, kv.INT8, 4, 2, 64, 16, [0, 0], [new, new])
    q, out, lse = attend(c)
    assert bool((out == 0).all()) and bool((lse == -math.inf).all())


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("value", [math.nan, math.inf, 2.0 ** 100])
@pytest.mark.parametrize("new,group", [(5, 2), (150, 1)])
def test_a_query_that_is_not_finite(dtype, value, new, group):
    """It is NaN (or huge) for itself: the other rows' bits stay."""
    c = Cache(dtype, kv.INT8, 2 * group, 2, 128, 64, [300 + new, new], [new, new])
    c.fill()
    q, out, lse = attend(c)
    bad = c.total - 2
    q[bad, 1] = value if dtype == kv.BF16 or not math.isfinite(value) else 60000.0
    again = torch.full_like(q, -7.0)
    lse2 = c.run_attention(q, again)
    keep = torch.ones(c.total, c.qh, dtype=torch.bool, device="cuda")
    keep[bad, 1] = False
    if math.isfinite(value):                            # beside a huge one, others may go another way to the same answer
        compare(c, torch.where(keep[..., None], again, 0), torch.where(keep, lse2, 0.0), tuple(torch.where(keep.cpu()[..., None] if x.dim() == 3 else keep.cpu(), x, 0.0) for x in definition(c, q)))
    else:
        assert torch.equal(out[keep], again[keep]) and torch.equal(lse[keep], lse2[keep])
        assert bool(torch.isnan(again[bad, 1]).all())

"""Attention over the 8-bit cache against the definition in 64 bits."""
import math
import random

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from kv_reference import TYPES, Cache, ragged  # noqa: E402
from paper_2410_15240_b200 import fastrack, kv  # noqa: E402

pytestmark = pytest.mark.gpu
SHAPES = [(kv.BF16, kv.INT8), (kv.BF16, kv.E4M3), (kv.F16, kv.INT8), (kv.F16, kv.E4M3)]


def queries(c, scale=2.0, seed=5):
    gen = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(c.total, c.qh, c.d, generator=gen)).to(c.t).cuda()


def check(c, q=None, window=0, mass=True):
    q = queries(c) if q is None else q
    pad = 64                                            # rows before and behind the answers that stay as they are
    room = torch.full((c.total + 2 * pad, c.qh, c.d), -7.0, dtype=c.t, device="cuda")
    out = room[pad:pad + c.total]
    stride = -(-c.max_len // c.bt) + 3
    m_in = torch.rand(c.n, c.kh, stride, device="cuda") if mass else None
    m_out = torch.full_like(m_in, -5.0) if mass else None
    lse = c.run_attention(q, out, window, m_in, m_out)
    assert bool((room[:pad] == -7).all()) and bool((room[pad + c.total:] == -7).all())
    c.check_attention(q, out, lse, window, m_in, m_out)
    return out, lse, m_out


@pytest.mark.parametrize("dtype,fmt", SHAPES)
@pytest.mark.parametrize("dim,block,q_heads,kv_heads", [(128, 64, 8, 2), (128, 16, 4, 4), (64, 32, 14, 2), (96, 128, 8, 1), (128, 128, 40, 2)])
def test_single_tokens(dtype, fmt, dim, block, q_heads, kv_heads):
    lens = [1, 2, block - 1, block, block + 1, 2 * block, 5 * block + 3, 15, 16, 17, 700]
    c = Cache(dtype, fmt, q_heads, kv_heads, dim, block, lens, [1] * len(lens))
    c.fill()
    check(c)


@pytest.mark.parametrize("dtype,fmt", SHAPES)
@pytest.mark.parametrize("dim,block,q_heads,kv_heads,new", [(128, 64, 8, 2, 7), (64, 16, 3, 3, 33), (96, 32, 6, 2, 129), (128, 128, 8, 1, 70), (128, 64, 4, 4, 300),
                                                             (64, 64, 16, 2, 200), (128, 32, 12, 2, 150)])
@pytest.mark.parametrize("window", [0, 50])
def test_many_new_tokens(dtype, fmt, dim, block, q_heads, kv_heads, new, window):
    news = [new, 1, new // 2, new]
    lens = [new, 400, new // 2 + 37, new + 511]
    c = Cache(dtype, fmt, q_heads, kv_heads, dim, block, lens, news, seed=1)
    c.fill()
    check(c, window=window)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(seed):
    rng = random.Random(seed)
    dtype, fmt = rng.choice(SHAPES)
    block, dim, kvh, group = rng.choice([16, 32, 64, 128]), rng.choice([64, 96, 128]), rng.choice([1, 2, 3]), rng.choice([1, 2, 3, 5, 8, 17])
    n = rng.randint(1, 5)
    lens = ragged(rng, n, 0, rng.choice([40, 300, 1500]))
    news = [rng.randint(0, rng.choice([1, 4, 40, 260])) for _ in lens]
    if rng.random() < 0.7:
        news = [min(a, b) for a, b in zip(news, lens)]
    c = Cache(dtype, fmt, kvh * group, kvh, dim, block, lens, news, seed=seed)
    c.fill(spread=rng.choice([0.1, 3.0]))
    for i in range(n):                                  # absent pages
        for b in range(lens[i] // block):
            if rng.random() < 0.1:
                c.table[i, b] = rng.choice([-1, c.pages, -2 ** 31, 2 ** 31 - 1])
    c.d_table.copy_(c.table)
    check(c, window=rng.choice([0, 0, 1, 7, 64, 300]), mass=rng.random() < 0.7)


@pytest.mark.parametrize("new", [1, 5, 200])
def test_rows_that_see_nothing(new):
    # sequences of length zero, shorter than their new tokens, and with every page absent
    c = Cache(kv.BF16, kv.INT8, 8, 2, 128, 64, [0, new - 1, 128, 130, 300], [new] * 5)
    c.fill()
    c.table[2, :2] = -1
    c.table[4, :1] = -1
    c.d_table.copy_(c.table)
    out, lse, _ = check(c)
    assert bool((out[:new] == 0).all()) and bool((lse[:new] == -math.inf).all())


@pytest.mark.parametrize("new", [1, 130])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_non_finite_blocks(new, bad):
    """A block whose scale is not finite turns the rows that see it to NaN and leaves the others alone."""
    c = Cache(kv.BF16, kv.E4M3, 4, 2, 128, 16, [200 + new] * 3, [new] * 3, poison=True)
    c.fill()
    if new > 1:
        p = int(c.table[1, (200 + new - 16) // 16])     # seen by the last new tokens only
    else:
        p = int(c.table[1, 3])
    at = 2 * c.codes
    c.pool[p, at:at + 8 * c.kh].view(torch.float32)[:] = bad
    q = queries(c)
    out = torch.empty(c.total, c.qh, c.d, dtype=c.t, device="cuda")
    c.run_attention(q, out)
    first = c.lens[1] - c.news[1]
    block = [int(x) for x in c.table[1]].index(p)
    sees = [first + j >= block * 16 for j in range(new)]
    nan = torch.isnan(out.float()).any(-1).cpu()
    for i in range(3):
        for j in range(new):
            want = i == 1 and sees[j]
            assert bool((nan[c.starts[i] + j] == want).all()), (i, j)
    # the same inputs with the block in order: rows that do not see it keep their bits
    c.pool[p, at:at + 8 * c.kh].view(torch.float32)[:] = 0.01
    again = torch.empty_like(out)
    c.run_attention(q, again)
    assert bool((again == out)[~nan.cuda()].all())


@pytest.mark.parametrize("new", [1, 3, 140])
def test_scores_far_apart(new):
    """Large scores, of both signs, and V scales many orders apart: the running maximum and V's reference both move."""
    c = Cache(kv.F16, kv.E4M3, 8, 2, 64, 16, [900, 333], [new, new], scale=3.0)
    c.fill(spread=4.0)
    check(c, queries(c, 3.0))


def test_bf16_range():
    """bf16 queries and tails beyond f16's range."""
    c = Cache(kv.BF16, kv.INT8, 4, 2, 128, 64, [90, 40, 700], [1, 1, 1], scale=1e-30)
    c.fill()
    c.tail.mul_(1e5)
    q = queries(c, 1e23)
    check(c, q, mass=False)


@pytest.mark.parametrize("new", [1, 6, 150])
def test_strides(new):
    """q as a slice of one projection, out with heads outermost."""
    c = Cache(kv.F16, kv.INT8, 6, 2, 96, 32, [new + 200, new + 5], [new, new])
    c.fill()
    fused = torch.randn(c.total, 10, 96, device="cuda").to(c.t)
    q = fused[:, 2:8]
    out = torch.empty(6, c.total, 96, dtype=c.t, device="cuda").transpose(0, 1)
    lse = c.run_attention(q, out)
    c.check_attention(q, out, lse)


@pytest.mark.parametrize("new", [1, 150])
def test_same_bits_again_and_on_another_stream(new):
    c = Cache(kv.BF16, kv.E4M3, 8, 2, 128, 64, [3000, 1, 777], [new, 1, new])
    c.fill()
    q = queries(c)
    out, lse, mass = check(c, q)
    stream = torch.cuda.Stream()
    other = torch.empty_like(out)
    m_in = torch.zeros(c.n, c.kh, mass.shape[2], device="cuda")
    m1, m2 = m_in.clone(), m_in.clone()
    torch.cuda.synchronize()
    lse2 = c.run_attention(q, other, mass_in=m_in, mass_out=m1, stream=stream)
    assert torch.equal(out, other) and torch.equal(lse, lse2)
    c.run_attention(q, other, mass_in=m2, mass_out=m2)  # in place
    assert torch.equal(m1, m2)


@pytest.mark.parametrize("new", [1, 150])
def test_other_sequences_do_not_matter(new):
    """A sequence's answers keep their bits when the others' contents change."""
    c = Cache(kv.BF16, kv.INT8, 8, 2, 128, 64, [500, 900, 260], [new] * 3)
    c.fill()
    q = queries(c)
    a, b = (torch.empty(c.total, c.qh, c.d, dtype=c.t, device="cuda") for _ in range(2))
    c.run_attention(q, a)
    keep = [int(x) for x in c.table[1, :900 // 64]]
    other = [p for p in range(c.pages) if p not in keep]
    c.pool[other] = 255
    c.tail[0] = math.nan
    c.tail[2] = math.nan
    c.run_attention(q, b)
    s = slice(c.starts[1], c.starts[2])
    assert torch.equal(a[s], b[s])


@pytest.mark.parametrize("new", [1, 140])
def test_pages_behind_4_gib(new):
    """Offsets that pass 32 bits."""
    page = kv.KvCache(kv.BF16, kv.INT8, 8, 8, 128, 128).page_bytes
    c = Cache(kv.BF16, kv.INT8, 8, 8, 128, 128, [new + 1000], [new], page_base=(1 << 32) // page + 3, poison=False)
    c.fill()
    assert int(c.table[0, 0]) * page > 1 << 32
    check(c)


def test_long_sequence():
    """One sequence split over many CTAs, and its weights."""
    c = Cache(kv.BF16, kv.E4M3, 8, 1, 128, 128, [40001, 5], [1, 1], poison=False)
    c.fill()
    check(c)
    check(c, window=20000)


def test_graph_capture_with_lengths_that_change():
    """A captured call follows lengths, pages and tails as they are at replay."""
    c = Cache(kv.BF16, kv.INT8, 8, 2, 128, 64, [2000, 1999], [1, 1])
    c.fill()
    q = queries(c)
    out, lse = torch.empty(c.total, c.qh, c.d, dtype=c.t, device="cuda"), torch.empty(c.total, c.qh, device="cuda")
    b = c.batch()
    ws = torch.empty(c.kv.workspace_bytes(b, False), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    from kv_reference import rows
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            c.kv.attention(b, rows(q), rows(out), ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(), stream=stream.cuda_stream)
    for lens in ([2000, 1999], [1, 64], [700, 1024]):
        c.lens = lens
        c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.tail.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check_attention(q, out, lse)


def test_device_values_beyond_the_bounds_are_clamped():
    """Lengths and starts that break the struct's bounds reach nothing outside the buffers: they are cut to the bounds."""
    c = Cache(kv.BF16, kv.INT8, 4, 2, 64, 16, [100, 90], [2, 2])
    c.fill()
    q = queries(c)
    c.d_lens.copy_(torch.tensor([2 ** 30, -4], dtype=torch.int32))
    c.d_starts.copy_(torch.tensor([-3, 2, 2 ** 30], dtype=torch.int32))
    out = torch.empty(c.total, c.qh, c.d, dtype=c.t, device="cuda")
    lse = c.run_attention(q, out)
    c.lens = [100, 0]                                   # max_len, and nothing
    c.check_attention(q, out, lse)


def test_refusals():
    c = Cache(kv.BF16, kv.INT8, 4, 2, 64, 16, [100, 90], [1, 1])
    c.fill()
    q, out = queries(c), torch.empty(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    mass = torch.zeros(2, 2, 7, device="cuda")
    from kv_reference import rows
    R = rows

    def refused(batch=None, q=R(q), out=R(out), ws_ptr=ws.data_ptr(), ws_bytes=ws.numel(), **more):
        with pytest.raises(fastrack.FastrackError) as e:
            c.kv.attention(batch or c.batch(), q, out, ws_ptr, ws_bytes, **more)
        assert e.value.code == fastrack.ERR_ARG
    refused(batch=c.batch(n_seqs=-1))
    refused(batch=c.batch(max_new=3))                   # more than total_new
    refused(batch=c.batch(max_len=8 * 16))              # beyond the table's rows
    refused(batch=c.batch(max_len=-1))
    refused(batch=c.batch(d_lens=0))
    refused(batch=c.batch(d_starts=0))
    refused(batch=c.batch(d_tail=0))
    refused(batch=c.batch(d_pool=c.pool.data_ptr() + 8))
    refused(batch=c.batch(d_table=0))
    refused(q=kv.Rows(q.data_ptr() + 2, 256, 64))
    refused(q=kv.Rows(q.data_ptr(), 252, 64))
    refused(out=kv.Rows(out.data_ptr(), 256, 63))
    refused(out=kv.Rows(0, 256, 64))
    refused(window=-1)
    refused(ws_bytes=c.kv.workspace_bytes(c.batch(), False) // 4)
    refused(ws_ptr=0)
    refused(ws_ptr=ws.data_ptr() + 8)
    refused(d_mass_in=mass.data_ptr())
    refused(d_mass_in=mass.data_ptr(), d_mass_out=mass.data_ptr(), mass_stride=6)
    assert c.kv.workspace_bytes(c.batch(n_seqs=-1), True) == 0
    c.kv.attention(c.batch(n_seqs=0), R(q), R(out), ws.data_ptr(), ws.numel())      # nothing to do
    assert c.kv.launches == 0

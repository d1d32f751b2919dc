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

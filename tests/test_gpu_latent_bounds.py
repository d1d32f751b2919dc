"""The latent cache at the ends of its ranges: offsets beyond 32 bits, bounds larger than the batch, the largest numbers of heads and drafts."""
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from latent_reference import Cache, rows  # noqa: E402
from paper_2410_15240_b200 import kv, latent  # noqa: E402

pytestmark = pytest.mark.gpu
GUARD = -3.0


def test_pages_beyond_32_bits():
    """The same cache in the first pages of a pool and in the last ones of a pool of more than 2^31 values: the same answers, bit for bit."""
    freq = kv.rotary_frequencies(64, 10000.0)[0]
    c = Cache(kv.BF16, 16, 512, 64, 64, [500, 130], [9, 5], seed=3, key=64, value=64, positions=torch.arange(14), rotary=kv.ROTARY_HALF, frequencies=freq)
    x, key, weight = c.normal(14, 512).cuda(), c.normal(14, 64).cuda(), c.normal(512).cuda()
    q, q_rope = c.normal(14, 16, 512).cuda(), c.normal(14, 16, 64).cuda()
    w, qk = c.normal(16, 128, 512).cuda(), c.normal(14, 16, 64).cuda()
    ints = torch.zeros(128, dtype=torch.int32, device="cuda")
    ints[16:30] = torch.arange(14)
    ints[32:46] = torch.tensor([3, 9, 9, 6, 9, 9, 9, 9, 9, 12, 9, 9, 9, 9])
    starts = torch.tensor([0, 500], dtype=torch.int32, device="cuda")
    parents = torch.tensor([-1, 0, 0, 0, 1, 2, 3, 6, 6, -1, 0, 0, 0, 3], dtype=torch.int32, device="cuda")

    def everything(batch):
        out, lse = torch.zeros(14, 16, 512, dtype=c.t, device="cuda"), torch.zeros(14, 16, device="cuda")
        k, v, po = (torch.zeros(n, 16, 64, dtype=c.t, device="cuda") for n in (630, 630, 14))
        ws = torch.empty(c.handle.workspace_bytes(batch), dtype=torch.uint8, device="cuda")
        results = ints.clone()
        at = results.data_ptr()
        c.handle.append(batch, rows(x), rows(key), weight.data_ptr())
        c.handle.attention(batch, rows(q), rows(q_rope), rows(out), ws.data_ptr(), ws.numel(), d_lse=lse.data_ptr(), d_parents=parents.data_ptr())
        c.handle.expand(batch, w.data_ptr(), rows(k), rows(v), starts.data_ptr(), 630)
        c.handle.prompt(batch, rows(qk), rows(q_rope), rows(k), rows(v), starts.data_ptr(), 630, rows(po))
        c.handle.accept(batch, latent.Acceptance(parents.data_ptr(), at + 64, at + 128, at + 256, at + 320, at + 328, at + 336))
        torch.cuda.synchronize()
        return out, lse, k, v, po, results

    pages = (1 << 31) // (64 * 576) + 100
    big = torch.empty(pages, 64, 576, dtype=c.t, device="cuda")
    far = c.table.clone()
    far[(c.table >= 0)] += pages - c.pages
    big[pages - c.pages:] = c.d_pool
    batch = latent.Batch.from_buffer_copy(c.batch)
    d_far = far.cuda()
    batch.d_pool, batch.d_table, batch.pool_pages = big.data_ptr(), d_far.data_ptr(), pages
    want, got = everything(c.batch), everything(batch)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert torch.equal(big[pages - c.pages:], c.d_pool)
    assert want[5][80:82].tolist() != [0, 0]


def test_rows_beyond_32_bits():
    """Expanded keys and values whose rows lie 2^22 values apart."""
    c = Cache(kv.F16, 2, 128, 32, 32, [600], [40], key=64, value=128)
    w, q, q_rope = c.normal(2, 192, 128).cuda(), c.normal(40, 2, 64).cuda(), c.normal(40, 2, 32).cuda()
    starts = torch.zeros(1, dtype=torch.int32, device="cuda")
    answers = []
    for stride in (256, 1 << 22):
        k, v = (torch.empty(600 * stride, dtype=c.t, device="cuda").view(600, stride)[:, :2 * n].view(600, 2, n) if stride == 2 * n else
                torch.empty(600 * stride, dtype=c.t, device="cuda").as_strided((600, 2, n), (stride, n, 1)) for n in (64, 128))
        out = torch.empty(40, 2, 128, dtype=c.t, device="cuda")
        c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), starts.data_ptr(), 600)
        c.handle.prompt(c.batch, rows(q), rows(q_rope), rows(k), rows(v), starts.data_ptr(), 600, rows(out))
        torch.cuda.synchronize()
        answers.append((k.clone(), v.clone(), out))
        del k, v
    assert all(torch.equal(a, b) for a, b in zip(*answers))


def test_rows_of_no_sequence_stay():
    """total_new and max_new are bounds: rows behind the last sequence are left as they were, by every call."""
    freq = kv.rotary_frequencies(32, 10000.0)[0]
    c = Cache(kv.BF16, 3, 128, 32, 16, [50, 20], [4, 2], key=64, value=64, positions=torch.arange(9), rotary=kv.ROTARY_INTERLEAVED, frequencies=freq)
    x, key, q, q_rope, qk = (c.normal(9, *s).cuda() for s in ((128,), (32,), (3, 128), (3, 32), (3, 64)))
    k, v = c.normal(70, 3, 64).cuda(), c.normal(70, 3, 64).cuda()
    starts = torch.tensor([0, 50], dtype=torch.int32, device="cuda")

    def run(total, most):
        batch = latent.Batch.from_buffer_copy(c.batch)
        batch.total_new, batch.max_new = total, most
        turned = torch.full((9, 3, 32), GUARD, dtype=c.t, device="cuda")
        out, po = torch.full((9, 3, 128), GUARD, dtype=c.t, device="cuda"), torch.full((9, 3, 64), GUARD, dtype=c.t, device="cuda")
        lse, path = torch.full((2, 9, 3), GUARD, device="cuda"), torch.full((9,), -7, dtype=torch.int32, device="cuda")
        tokens = torch.zeros(9, dtype=torch.int32, device="cuda")
        few = torch.zeros(6, dtype=torch.int32, device="cuda")
        ws = torch.empty(c.handle.workspace_bytes(batch), dtype=torch.uint8, device="cuda")
        c.handle.append(batch, rows(x), rows(key), 0, rows(q_rope), rows(turned))
        c.handle.attention(batch, rows(q), rows(q_rope), rows(out), ws.data_ptr(), ws.numel(), d_lse=lse[0].data_ptr())
        c.handle.prompt(batch, rows(qk), rows(q_rope), rows(k), rows(v), starts.data_ptr(), 70, rows(po), d_lse=lse[1].data_ptr())
        at = few.data_ptr()
        c.handle.accept(batch, latent.Acceptance(0, tokens.data_ptr(), tokens.data_ptr(), path.data_ptr(), at, at + 8, at + 16))
        torch.cuda.synchronize()
        return turned, out, po, lse[0], lse[1], path, few

    exact, loose = run(6, 4), run(9, 9)
    for a, b in zip(exact[:6], loose[:6]):
        assert torch.equal(a[:6], b[:6]) and bool((b[6:] == a[6:]).all())
        assert bool((a[6:] == (GUARD if a.is_floating_point() else -7)).all())
    assert torch.equal(exact[6], loose[6])


def test_the_largest_tree_and_many_heads():
    """1024 drafts in one chain of parents answer as a chain does; 1024 heads of one token as 1024 tokens of one head."""
    c = Cache(kv.BF16, 1, 128, 32, 64, [1100], [1024], seed=2)
    q, q_rope = c.normal(1024, 1, 128).cuda(), c.normal(1024, 1, 32).cuda()
    out, again = (torch.zeros(1024, 1, 128, dtype=c.t, device="cuda") for _ in range(2))
    ws = torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda")
    parents = torch.arange(-1, 1023, dtype=torch.int32, device="cuda")
    c.handle.attention(c.batch, rows(q), rows(q_rope), rows(out), ws.data_ptr(), ws.numel())
    c.handle.attention(c.batch, rows(q), rows(q_rope), rows(again), ws.data_ptr(), ws.numel(), d_parents=parents.data_ptr())
    torch.cuda.synchronize()
    # cut at other places, since a tree's rows all go to the end: the same to a rounding of values of size 1 and their weights'
    assert float((out.float() - again.float()).abs().max()) <= 4 * 2.0 ** -8
    one = Cache(kv.BF16, 1024, 128, 32, 64, [76], [1], seed=2)
    qh, qh_rope = q.view(1, 1024, 128), q_rope.view(1, 1024, 32)
    wide = torch.zeros(1, 1024, 128, dtype=c.t, device="cuda")
    ws = torch.empty(one.handle.workspace_bytes(one.batch), dtype=torch.uint8, device="cuda")
    one.handle.attention(one.batch, rows(qh), rows(qh_rope), rows(wide), ws.data_ptr(), ws.numel())
    x, _ = one.held(0)
    z = one.scale * (torch.cat([qh[0], qh_rope[0]], 1).double().cpu() @ x.T)
    want = torch.softmax(z, 1) @ x[:, :128]
    torch.cuda.synchronize()
    # its own rounding and its weights' (half a step each of values of 4 at most)
    assert bool(((wide[0].double().cpu() - want).abs() <= 2.0 ** -8 * (want.abs() + torch.softmax(z, 1) @ x[:, :128].abs()) + 2.0 ** -12).all())

"""The latent cache's calls: what is refused, threads, streams, memory, and all operators together as examples/sealed_latent.py uses them."""
import importlib.util
import os
import threading

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from latent_reference import Cache, rows  # noqa: E402
from paper_2410_15240_b200 import fastrack, kv, latent  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Calls:
    """Good arguments for every call of one cache."""

    def __init__(self):
        freq = kv.rotary_frequencies(64, 10000.0)[0]
        self.c = c = Cache(kv.BF16, 4, 128, 64, 32, [70, 40], [3, 2], key=64, value=64, positions=torch.arange(5), rotary=kv.ROTARY_HALF, frequencies=freq)
        self.x, self.key = c.normal(5, 128).cuda(), c.normal(5, 64).cuda()
        self.weight, self.w = c.normal(128).cuda(), c.normal(4, 128, 128).cuda()
        self.q, self.q_rope, self.out = c.normal(5, 4, 128).cuda(), c.normal(5, 4, 64).cuda(), torch.empty(5, 4, 128, dtype=c.t, device="cuda")
        self.qk, self.po = c.normal(5, 4, 64).cuda(), torch.empty(5, 4, 64, dtype=c.t, device="cuda")
        self.k, self.v = c.normal(110, 4, 64).cuda(), c.normal(110, 4, 64).cuda()
        self.starts = torch.tensor([0, 70], dtype=torch.int32, device="cuda")
        self.ints = torch.zeros(64, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda")
        at = self.ints.data_ptr()
        self.call = latent.Acceptance(at, at, at, at + 64, at + 128, at + 144, at + 160)

    def append(self, batch=None, x=None, key=None, weight=None, q=0, q_out=0):
        self.c.handle.append(batch or self.c.batch, x or rows(self.x), key or rows(self.key), self.weight.data_ptr() if weight is None else weight,
                             rows(self.q_rope) if q == 0 else q, rows(self.q_rope) if q_out == 0 else q_out)

    def attention(self, batch=None, q=None, q_rope=None, out=None, ws=None, size=None, lse=0, parents=0):
        self.c.handle.attention(batch or self.c.batch, q or rows(self.q), q_rope or rows(self.q_rope), out or rows(self.out), self.ws.data_ptr() if ws is None else ws,
                                self.ws.numel() if size is None else size, d_lse=lse, d_parents=parents)

    def expand(self, batch=None, w=None, k=None, v=None, starts=None, keys=110):
        self.c.handle.expand(batch or self.c.batch, self.w.data_ptr() if w is None else w, k or rows(self.k), v or rows(self.v),
                             self.starts.data_ptr() if starts is None else starts, keys)

    def prompt(self, batch=None, q=None, q_rope=None, k=None, v=None, starts=None, keys=110, out=None, lse=0):
        self.c.handle.prompt(batch or self.c.batch, q or rows(self.qk), q_rope or rows(self.q_rope), k or rows(self.k), v or rows(self.v),
                             self.starts.data_ptr() if starts is None else starts, keys, out or rows(self.po), d_lse=lse)

    def accept(self, batch=None, **change):
        call = latent.Acceptance.from_buffer_copy(self.call)
        for name, value in change.items():
            setattr(call, name, value)
        self.c.handle.accept(batch or self.c.batch, call)

    def batch(self, **change):
        b = latent.Batch.from_buffer_copy(self.c.batch)
        for name, value in change.items():
            setattr(b, name, value)
        return b


@pytest.fixture(scope="module")
def calls():
    return Calls()


NAMES = ("append", "attention", "expand", "prompt", "accept")
BAD_BATCHES = [dict(n_seqs=-1), dict(n_seqs=65536), dict(max_len=-1), dict(max_len=(1 << 30) + 1), dict(pool_pages=-1), dict(table_stride=2), dict(d_pool=0),
               dict(d_pool=264), dict(d_table=0), dict(d_table=2), dict(d_lens=0), dict(d_lens=6)]
BAD_NEWS = [dict(total_new=-1), dict(max_new=-1), dict(max_new=6), dict(total_new=1 << 29), dict(d_starts=0), dict(d_starts=10)]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("change", BAD_BATCHES + BAD_NEWS, ids=str)
def test_bad_batches(calls, name, change):
    if name == "expand" and change in BAD_NEWS:
        return                                           # new tokens do not count there
    before = calls.c.handle.launches
    with pytest.raises(fastrack.FastrackError) as e:
        getattr(calls, name)(batch=calls.batch(**change))
    assert e.value.code == fastrack.ERR_ARG and calls.c.handle.launches == before


def bad_rows(x):
    good = rows(x)
    return [kv.Rows(0, good.token_stride, good.head_stride), kv.Rows(good.data + 8, good.token_stride, good.head_stride),
            kv.Rows(good.data, good.token_stride + 4, good.head_stride), kv.Rows(good.data, good.token_stride, good.head_stride + 1)]


def test_bad_arguments(calls):
    bad = []
    for k in range(4):
        bad += [lambda k=k: calls.append(x=bad_rows(calls.x)[k]), lambda k=k: calls.append(key=bad_rows(calls.key)[k]), lambda k=k: calls.append(q=bad_rows(calls.q)[k]),
                lambda k=k: calls.append(q_out=bad_rows(calls.q)[k]), lambda k=k: calls.attention(q=bad_rows(calls.q)[k]),
                lambda k=k: calls.attention(q_rope=bad_rows(calls.q_rope)[k]), lambda k=k: calls.attention(out=bad_rows(calls.out)[k]),
                lambda k=k: calls.expand(k=bad_rows(calls.k)[k]), lambda k=k: calls.expand(v=bad_rows(calls.v)[k]), lambda k=k: calls.prompt(q=bad_rows(calls.qk)[k]),
                lambda k=k: calls.prompt(q_rope=bad_rows(calls.q_rope)[k]), lambda k=k: calls.prompt(k=bad_rows(calls.k)[k]), lambda k=k: calls.prompt(v=bad_rows(calls.v)[k]),
                lambda k=k: calls.prompt(out=bad_rows(calls.po)[k])]
    at = calls.ws.data_ptr()
    bad += [lambda: calls.append(q=None), lambda: calls.append(q_out=None), lambda: calls.append(weight=calls.weight.data_ptr() + 8),
            lambda: calls.append(batch=calls.batch(d_positions=0)), lambda: calls.append(batch=calls.batch(d_positions=12)),
            lambda: calls.append(q_out=kv.Rows(calls.q_rope.data_ptr(), calls.q_rope.stride(0), 128)),
            lambda: calls.attention(ws=0), lambda: calls.attention(ws=at + 8), lambda: calls.attention(size=calls.ws.numel() - 1), lambda: calls.attention(lse=at + 2),
            lambda: calls.attention(parents=at + 1),
            lambda: calls.attention(batch=calls.batch(total_new=1025, max_new=1025), parents=calls.ints.data_ptr(), size=1 << 40),
            lambda: calls.expand(w=0), lambda: calls.expand(w=at + 8), lambda: calls.expand(starts=0), lambda: calls.expand(starts=at + 2), lambda: calls.expand(keys=-1),
            lambda: calls.prompt(starts=0), lambda: calls.prompt(starts=at + 1), lambda: calls.prompt(keys=-1), lambda: calls.prompt(lse=at + 1),
            lambda: calls.prompt(k=kv.Rows(calls.k.data_ptr(), -256, 64)), lambda: calls.prompt(k=kv.Rows(calls.k.data_ptr(), 0, 64)),
            lambda: calls.prompt(v=kv.Rows(calls.v.data_ptr(), 256, -64)), lambda: calls.prompt(v=kv.Rows(calls.v.data_ptr(), 1 << 40, 64)),
            lambda: calls.accept(batch=calls.batch(total_new=1025, max_new=1025))]
    bad += [lambda n=n, v=v: calls.accept(**{n: v}) for n in ("d_tokens", "d_choices", "d_path", "d_n_accepted", "d_next", "d_lens_out") for v in (0, at + 2)]
    bad += [lambda: calls.accept(d_parents=at + 2)]
    before = calls.c.handle.launches
    for i, call in enumerate(bad):
        with pytest.raises(fastrack.FastrackError) as e:
            call()
        assert e.value.code == fastrack.ERR_ARG, i
    assert calls.c.handle.launches == before


def test_nothing_to_do(calls):
    before = calls.c.handle.launches
    for name in NAMES:
        getattr(calls, name)(batch=calls.batch(n_seqs=0))
    for name in ("append", "attention", "prompt"):
        getattr(calls, name)(batch=calls.batch(total_new=0, max_new=0))
    calls.expand(keys=0)
    assert calls.c.handle.launches == before
    assert latent._lib.fastrack_latent_attention_workspace(calls.c.handle.handle, calls.batch(n_seqs=-1)) == 0


def test_good_calls_and_no_memory(calls):
    for name in NAMES:                                   # once, for what the driver sets up
        getattr(calls, name)()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    for _ in range(3):
        for name in NAMES:
            getattr(calls, name)()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free


def test_first_calls_from_a_new_thread():
    made = Calls()
    fine = []

    def work():
        for name in ("attention", "expand", "prompt"):
            getattr(made, name)()
        fine.append(True)

    thread = threading.Thread(target=work)
    thread.start()
    thread.join()
    torch.cuda.synchronize()
    assert fine == [True]


def test_two_streams_at_once():
    """Two attentions on two streams, each with its workspace, beside an expansion on a third."""
    c = Cache(kv.BF16, 16, 512, 64, 64, [5000, 300], [1, 1], seed=9)
    w = c.normal(16, 256, 512).cuda()
    k, v = torch.empty(5300, 16, 128, dtype=c.t, device="cuda"), torch.empty(5300, 16, 128, dtype=c.t, device="cuda")
    starts = torch.tensor([0, 5000], dtype=torch.int32, device="cuda")
    qs = [(c.normal(2, 16, 512).cuda(), c.normal(2, 16, 64).cuda()) for _ in range(2)]
    ws = [torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda") for _ in range(2)]

    def one(i, out, stream):
        c.handle.attention(c.batch, rows(qs[i][0]), rows(qs[i][1]), rows(out), ws[i].data_ptr(), ws[i].numel(), stream=stream)

    want = [torch.empty(2, 16, 512, dtype=c.t, device="cuda") for _ in range(2)]
    for i in range(2):
        one(i, want[i], 0)
    c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), starts.data_ptr(), 5300)
    torch.cuda.synchronize()
    want_k = k.clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[torch.zeros_like(want[0]) for _ in range(10)] for _ in range(2)]
    k.zero_()
    torch.cuda.synchronize()
    for r in range(10):
        for i in range(2):
            one(i, outs[i][r], streams[i].cuda_stream)
        c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), starts.data_ptr(), 5300, stream=streams[2].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(outs[i][r], want[i]) for i in range(2) for r in range(10)) and torch.equal(k, want_k)


def test_a_step_in_one_graph():
    """Store, attend and accept drafts captured together; replayed with other lengths and another tree."""
    freq = kv.rotary_frequencies(64, 10000.0)[0]

    def make():
        c = Cache(kv.BF16, 16, 256, 64, 32, [200, 90], [6, 6], seed=5, positions=torch.arange(12), rotary=kv.ROTARY_HALF, frequencies=freq, max_len=256)
        c.x, c.key, c.weight = c.normal(12, 256).cuda(), c.normal(12, 64).cuda(), c.normal(256).cuda()
        c.q, c.q_rope, c.out = c.normal(12, 16, 256).cuda(), c.normal(12, 16, 64).cuda(), torch.empty(12, 16, 256, dtype=c.t, device="cuda")
        c.parents = torch.tensor([-1, 0, 0, 1, 2, 3] * 2, dtype=torch.int32, device="cuda")
        c.tokens = torch.tensor([0, 1, 2, 3, 4, 5] * 2, dtype=torch.int32, device="cuda")
        c.choices = torch.tensor([2, 9, 4, 9, 8, 9, 1, 3, 9, 5, 9, 7], dtype=torch.int32, device="cuda")
        c.path, c.count, c.next = torch.zeros(12, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        c.after = torch.zeros(2, dtype=torch.int32, device="cuda")
        c.ws = torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda")
        return c

    def step(c, stream):
        c.handle.append(c.batch, rows(c.x), rows(c.key), c.weight.data_ptr(), stream=stream)
        c.handle.attention(c.batch, rows(c.q), rows(c.q_rope), rows(c.out), c.ws.data_ptr(), c.ws.numel(), d_parents=c.parents.data_ptr(), stream=stream)
        c.handle.accept(c.batch, latent.Acceptance(c.parents.data_ptr(), c.tokens.data_ptr(), c.choices.data_ptr(), c.path.data_ptr(), c.count.data_ptr(),
                                                   c.next.data_ptr(), c.after.data_ptr()), stream)

    a, b = make(), make()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, torch.cuda.current_stream().cuda_stream)
    for lens, parents in (([200, 90], None), ([150, 70], [-1, 0, 1, 2, 3, 4] * 2)):
        for c in (a, b):
            c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
            if parents:
                c.parents.copy_(torch.tensor(parents, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        step(b, 0)
        torch.cuda.synchronize()
        for name in ("out", "path", "count", "next", "after", "d_pool"):
            assert torch.equal(getattr(a, name), getattr(b, name)), name
    assert a.count.tolist() == [1, 2]


def test_sealed_latent():
    spec = importlib.util.spec_from_file_location("sealed_latent", os.path.join(ROOT, "examples", "sealed_latent.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    r = module.main(verbose=False)
    assert r["refused"] == [r["pages"] // 2] and r["accepted"] and r["same"] and r["finite"]
    assert module.SEQS * module.STEPS <= r["kept"] <= module.SEQS * module.STEPS * module.DRAFTS
    # the same scores and weights, added up in another order: a few roundings of answers of size 1 or less
    assert r["chain_error"] <= 4 * 2.0 ** -8

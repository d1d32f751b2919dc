"""Prompts of few heads, sequences and new tokens over a long cache: the tokens are shared out, and the answers joined."""
import math

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from latent_reference import Cache, rows  # noqa: E402
from paper_2410_15240_b200 import fastrack, kv, latent  # noqa: E402
from test_gpu_latent_cache import check_prompt, prompt_inputs, run_prompt  # noqa: E402

pytestmark = pytest.mark.gpu

# heads, rope, key, value, block, lens, news
PARTS = [
    (1, 64, 128, 128, 64, [5000], [600]),
    (2, 32, 64, 64, 16, [897], [1]),
    (2, 64, 128, 64, 32, [2050, 3, 0, 1200], [513, 3, 0, 1200]),                    # most sequences leave parts empty
    (16, 64, 64, 128, 128, [1500, 1030], [20, 257]),
    (9, 32, 128, 128, 16, [2000], [2000]),
]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,rope,key,value,block,lens,news", PARTS)
def test_parts(dtype, heads, rope, key, value, block, lens, news):
    c = Cache(dtype, heads, 128, rope, block, lens, news, key=key, value=value, seed=heads)
    assert c.handle.prompt_workspace_bytes(c.batch) > 0
    q, q_rope, k, v, starts = prompt_inputs(c, 1.5)
    before = c.handle.launches
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    assert c.handle.launches == before + 2
    check_prompt(c, q, q_rope, k, v, starts, out, lse, heads=sorted({0, heads - 1}))
    again, lse2 = run_prompt(c, q, q_rope, k, v, starts)
    assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_parts_with_absent_pages():
    """Of one sequence all pages are absent; of another those of one part and more; a third sees only its last tokens."""
    lens, news = [1000, 1500, 1300], [70, 300, 5]
    absent = [(0, i) for i in range(16)] + [(1, i) for i in range(3, 14)] + [(2, i) for i in range(20)]
    c = Cache(kv.BF16, 2, 128, 64, 64, lens, news, absent=absent, seed=5)
    q, q_rope, k, v, starts = prompt_inputs(c)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)
    assert bool((out[:70] == 0).all()) and bool((lse[:70] == -math.inf).all())


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
def test_parts_large_scores(dtype):
    """Scores that rise from part to part, and fall again."""
    c = Cache(dtype, 2, 128, 64, 64, [1800], [300], softmax_scale=0.5, seed=4)
    q, q_rope, k, v, starts = prompt_inputs(c, 2.0)
    for b in range(18):
        k[starts[0] + 100 * b] *= 0.2 + 0.3 * min(b, 18 - b)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)


def test_parts_hidden_values_do_not_count():
    """Rows that do not see a token are the same bits whatever it holds; rows that see it have its NaN or infinity, in its channel alone."""
    c = Cache(kv.BF16, 2, 128, 64, 32, [1700], [700], seed=11)
    q, q_rope, k, v, starts = prompt_inputs(c)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    first = 1700 - 700
    vk = v.clone()
    put = ((1023, 5, math.nan), (1024, 6, -math.inf), (1400, 7, math.inf), (1699, 8, math.nan))
    for token, channel, x in put:
        vk[starts[0] + token, 1, channel] = 0
    want, _ = run_prompt(c, q, q_rope, k, vk, starts)
    for token, channel, x in put:
        vk[starts[0] + token, 1, channel] = x
        want[token - first:, 1, channel] = x
    vk[starts[0] + 1700:] = math.nan
    got, lse2 = run_prompt(c, q, q_rope, k, vk, starts)
    assert torch.equal(lse2, lse) and torch.equal(got[:, 0], out[:, 0])
    assert torch.equal(got.nan_to_num(nan=1e4), want.nan_to_num(nan=1e4))


def test_loose_bounds_captured_and_two_streams():
    """Bounds above what there is share out otherwise, within the same tolerances; a captured call repeats bit for bit; two streams have a workspace each."""
    c = Cache(kv.F16, 3, 128, 64, 64, [1300, 900], [100, 40], seed=2, max_len=4000)
    q, q_rope, k, v, starts = prompt_inputs(c)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)
    exact = latent.Batch.from_buffer_copy(c.batch)
    exact.max_len = 1300
    assert c.handle.prompt_workspace_bytes(c.batch) > c.handle.prompt_workspace_bytes(exact) > 0
    c.batch = exact
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)
    d_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    outs = [torch.zeros(c.total, c.heads, c.value, dtype=c.t, device="cuda") for _ in range(3)]
    spaces = [torch.full((c.handle.prompt_workspace_bytes(exact),), 0xff, dtype=torch.uint8, device="cuda") for _ in range(3)]

    def call(i, stream):
        c.handle.prompt(exact, rows(q), rows(q_rope), rows(k), rows(v), d_starts.data_ptr(), k.shape[0], rows(outs[i]), spaces[i].data_ptr(), spaces[i].numel(),
                        stream=stream.cuda_stream)

    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i, s in enumerate(streams):
            call(i, s)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        call(2, torch.cuda.current_stream())
    spaces[2].fill_(0x7f)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(o.cpu(), out) for o in outs)


def test_workspace_is_wanted():
    c = Cache(kv.BF16, 2, 128, 64, 64, [1300], [100])
    q, q_rope, k, v, starts = prompt_inputs(c)
    d_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    out = torch.full((c.total, c.heads, c.value), 7.0, dtype=c.t, device="cuda")
    size = c.handle.prompt_workspace_bytes(c.batch)
    ws = torch.empty(size + 16, dtype=torch.uint8, device="cuda")
    before = c.handle.launches
    for at, n in ((0, 0), (0, size), (ws.data_ptr(), size - 1), (ws.data_ptr() + 8, size)):
        with pytest.raises(fastrack.FastrackError):
            c.handle.prompt(c.batch, rows(q), rows(q_rope), rows(k), rows(v), d_starts.data_ptr(), k.shape[0], rows(out), at, n)
    torch.cuda.synchronize()
    assert c.handle.launches == before and bool((out == 7).all())

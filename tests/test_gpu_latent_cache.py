"""Append, accept, expand and the attention over what was expanded, against their definitions."""
import math
import random

import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from kv_reference import turn  # noqa: E402
from latent_reference import LEAST, UNIT, Cache, attend, bounds, rows, strided, visible  # noqa: E402
from paper_2410_15240_b200 import kv, latent  # noqa: E402

pytestmark = pytest.mark.gpu
GUARD = -3.0
# a turned channel: cos and sin from 32 bits of a turn, two products and a sum
TURN_ERROR = 2.0 ** -21
# the norm in 32 bits: 16 squares added by a lane and 5 sums across lanes, a division, an addition, a root, a reciprocal and two products
NORM_ERROR = (16 + 5 + 6) * 2.0 ** -24


def pair_sizes(x, layout):
    s, r = x.abs(), x.shape[-1]
    out = torch.empty_like(s)
    if layout == kv.ROTARY_HALF:
        out[..., :r // 2] = out[..., r // 2:] = s[..., :r // 2] + s[..., r // 2:]
    else:
        out[..., 0::2] = out[..., 1::2] = s[..., 0::2] + s[..., 1::2]
    return out


def turned_bound(dtype, x, want, layout, gain):
    return UNIT[dtype] * want.abs() + gain * TURN_ERROR * pair_sizes(x, layout) + LEAST[dtype]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,dim,rope,block,lens,news,layout,norm", [
    (128, 512, 64, 64, [1, 65, 300], [1, 2, 300], kv.ROTARY_INTERLEAVED, True), (5, 128, 32, 16, [33, 0, 90], [3, 0, 17], kv.ROTARY_HALF, True),
    (16, 384, 64, 128, [129, 7], [7, 7], kv.ROTARY_HALF, False), (1, 256, 32, 32, [1000], [999], kv.ROTARY_NONE, True)])
def test_append(dtype, heads, dim, rope, block, lens, news, layout, norm):
    total = sum(news)
    positions = torch.randint(0, 100000, (total,), generator=torch.Generator().manual_seed(dim))
    rotary = dict(rotary=layout) if layout == kv.ROTARY_NONE else dict(rotary=layout, rotary_gain=1.25, frequencies=kv.rotary_frequencies(rope, 10000.0)[0])
    c = Cache(dtype, heads, dim, rope, block, lens, news, absent=[(len(lens) - 1, 0)], positions=positions, norm_eps=1e-3, **rotary)
    freq, gain = rotary.get("frequencies", []), rotary.get("rotary_gain", 1.0)
    down = strided((3 * torch.randn(total, dim + rope, generator=c.gen)).to(c.t).cuda())
    x, key = down.split([dim, rope], 1)
    weight = c.normal(dim).cuda()
    q = strided(c.normal(total, heads, rope).cuda())
    room = torch.full((total + 2, heads + 1, rope + 8), GUARD, dtype=c.t, device="cuda")
    q_out = room[1:-1, :heads, :rope]
    kept = q.clone()
    c.handle.append(c.batch, rows(x), rows(key), weight.data_ptr() if norm else 0, rows(q), rows(q_out), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(q, kept)
    got_q = q_out.clone()
    q_out.fill_(GUARD)
    assert bool((room == GUARD).all())
    xd, kd = x.double().cpu(), key.double().cpu()
    want = xd / torch.sqrt(xd.pow(2).mean(1, keepdim=True) + float(torch.tensor(1e-3))) * weight.double().cpu() if norm else xd
    want_k = turn(kd[:, None], positions, freq, gain, layout)[:, 0] if freq else kd
    pool, mine = c.d_pool.cpu(), torch.zeros(c.pages, block, dtype=torch.bool)
    for i, (L, n) in enumerate(zip(lens, news)):
        for j in range(n):
            place, row = L - n + j, c.starts[i] + j
            p = c.page(i, place)
            if p < 0:
                continue
            mine[p, place % block] = True
            got = pool[p, place % block].double()
            bound = (UNIT[dtype] + 2 * NORM_ERROR) * want[row].abs() + LEAST[dtype] if norm else torch.zeros(dim)
            assert bool(((got[:dim] - want[row]).abs() <= bound).all()), (i, j)
            bound = turned_bound(dtype, kd[row], want_k[row], layout, gain) if freq else torch.zeros(rope)
            assert bool(((got[dim:] - want_k[row]).abs() <= bound).all()), (i, j)
    assert torch.equal(pool[~mine], c.pool[~mine])           # nothing else was touched
    want_q = turn(q.double().cpu(), positions, freq, gain, layout) if freq else q.double().cpu()
    bound = turned_bound(dtype, q.double().cpu(), want_q, layout, gain) if freq else torch.zeros(1)
    assert bool(((got_q.double().cpu() - want_q).abs() <= bound).all())
    c.handle.append(c.batch, rows(x), rows(key), weight.data_ptr() if norm else 0, rows(q), rows(q), torch.cuda.current_stream().cuda_stream)   # in place
    torch.cuda.synchronize()
    assert torch.equal(q, got_q)


@pytest.mark.parametrize("value", [0.0, 1e-20, 1e4])
def test_norm_of_odd_sizes(value):
    """Rows of zeros, rows whose squares end below the smallest number, and large ones."""
    c = Cache(kv.BF16, 1, 128, 32, 16, [2], [2], norm_eps=1e-6)
    x = torch.full((2, 128), value).to(c.t).cuda()
    weight = torch.ones(128, dtype=c.t, device="cuda")
    key = torch.zeros(2, 32, dtype=c.t, device="cuda")
    c.handle.append(c.batch, rows(x), rows(key), weight.data_ptr())
    torch.cuda.synchronize()
    v = float(x[0, 0])
    want = v / math.sqrt(v * v + 1e-6)
    got = c.d_pool[c.page(0, 0), :2, :128].double().cpu()
    assert bool(((got - want).abs() <= (2.0 ** -8 + 2.0 ** -18) * abs(want)).all())


def test_accept():
    r = random.Random(7)
    for dim, rope, block, tokens in ((512, 64, 16, 25), (128, 32, 64, 200), (256, 64, 32, 1)):
        lens, news = [300, tokens + 3, tokens, 90, 400], [tokens, tokens, tokens, 0, min(9, tokens)]
        c = Cache(kv.BF16, 4, dim, rope, block, lens, news, absent=[(0, 17)], seed=tokens)
        parents, token, choice = [], [], []
        for i, n in enumerate(news):
            p = [-1] + [r.randint(max(0, j - 4), j - 1) for j in range(1, n)] if i != 2 else [j - 1 for j in range(n)]
            if n > 4 and i == 4:
                p[3] = -1                                    # a root that is not row 0
            parents.append(p[:n])
            t = [r.randint(0, 2) for _ in range(n)]
            token.append(t)
            choice.append([r.choice([t[k] for k in range(n) if k and p[k] == j] or [77]) if r.random() < 0.9 else 55 for j in range(n)])
        total = sum(news)
        ints = lambda x: torch.tensor(sum(x, []), dtype=torch.int32, device="cuda")  # noqa: E731
        d_parents, d_tokens, d_choices = ints(parents), ints(token), ints(choice)
        path = torch.full((total + 1,), -9, dtype=torch.int32, device="cuda")
        out = torch.full((3, len(lens) + 1), -9, dtype=torch.int32, device="cuda")
        call = latent.Acceptance(d_parents=d_parents.data_ptr(), d_tokens=d_tokens.data_ptr(), d_choices=d_choices.data_ptr(), d_path=path.data_ptr(),
                                 d_n_accepted=out[0].data_ptr(), d_next=out[1].data_ptr(), d_lens_out=out[2].data_ptr())
        before = c.d_pool.cpu()
        c.handle.accept(c.batch, call, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        want_pool, want_path = before.clone(), []
        for i, n in enumerate(news):
            walk = [0] if n else []
            while walk:
                kids = [j for j in range(walk[-1] + 1, n) if parents[i][j] == walk[-1] and token[i][j] == choice[i][walk[-1]]]
                if not kids:
                    break
                walk.append(kids[0])
            base = lens[i] - n
            for k, j in enumerate(walk):
                src, dst = c.page(i, base + j), c.page(i, base + k)
                if src >= 0 and dst >= 0:
                    want_pool[dst, (base + k) % block] = before[src, (base + j) % block]
            want_path += walk + [-1] * (n - len(walk))
            assert out[:, i].tolist() == [len(walk), choice[i][walk[-1]] if walk else -1, base + len(walk)], i
        assert path.tolist() == want_path + [-9] and bool((out[:, -1] == -9).all())
        assert torch.equal(c.d_pool.cpu(), want_pool)


def test_accept_a_chain_in_place():
    """Without parents the drafts are a chain; the new lengths may replace the old ones."""
    c = Cache(kv.F16, 4, 128, 32, 16, [40, 60], [6, 6])
    tokens = torch.tensor([9, 1, 2, 3, 4, 5] * 2, dtype=torch.int32, device="cuda")
    choices = torch.tensor([1, 2, 9, 4, 5, 6, 1, 2, 3, 4, 5, 6], dtype=torch.int32, device="cuda")
    path, n, following = (torch.zeros(k, dtype=torch.int32, device="cuda") for k in (12, 2, 2))
    before = c.d_pool.clone()
    c.handle.accept(c.batch, latent.Acceptance(d_tokens=tokens.data_ptr(), d_choices=choices.data_ptr(), d_path=path.data_ptr(), d_n_accepted=n.data_ptr(),
                                               d_next=following.data_ptr(), d_lens_out=c.d_lens.data_ptr()))
    torch.cuda.synchronize()
    assert n.tolist() == [3, 6] and following.tolist() == [9, 6] and c.d_lens.tolist() == [37, 60]
    assert path.tolist() == [0, 1, 2, -1, -1, -1, 0, 1, 2, 3, 4, 5] and torch.equal(before, c.d_pool)


SHAPES = [(16, 512, 64, 128, 128, 64, [1, 127, 128, 129, 300]), (5, 128, 32, 64, 64, 16, [33, 0, 200]), (3, 256, 64, 64, 128, 128, [400, 5]),
          (40, 384, 32, 128, 64, 32, [130]), (1, 512, 32, 64, 64, 16, [1])]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,dim,rope,key,value,block,lens", SHAPES)
def test_expand(dtype, heads, dim, rope, key, value, block, lens):
    absent = [(0, 0)] if lens[0] > 2 * block else []
    c = Cache(dtype, heads, dim, rope, block, lens, [0] * len(lens), key=key, value=value, absent=absent, seed=dim)
    for i, n in enumerate(lens):
        if n % block:
            c.pool[c.page(i, n - 1), n % block:] = math.nan  # behind the last token
    c.upload()
    w = (torch.randn(heads, key + value, dim, generator=c.gen) * dim ** -0.5).to(c.t).cuda()
    starts, at = [], 2
    for n in lens:                                           # rows between the sequences belong to nobody
        starts.append(at)
        at += n + 3
    room_k = torch.full((at + 1, heads + 1, key + 8), GUARD, dtype=c.t, device="cuda")
    room_v = torch.full((at + 1, heads + 1, value + 16), GUARD, dtype=c.t, device="cuda")
    k, v = room_k[:, :heads, :key], room_v[:, :heads, :value]
    d_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.batch.d_starts, c.batch.total_new, c.batch.max_new = 0, 0, 0
    c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), d_starts.data_ptr(), at, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    wd = w.double().cpu()
    for i, n in enumerate(lens):
        x, _ = c.held(i)
        x = x[:, :dim]
        here = slice(starts[i], starts[i] + n)
        for got, part in ((k[here], wd[:, :key]), (v[here], wd[:, key:])):
            want = torch.einsum("td,hcd->thc", x, part)
            size = torch.einsum("td,hcd->thc", x.abs(), part.abs())
            # its rounding; an addition in 32 bits per 16 products that may cut off, and the products brought to one size before it
            bound = UNIT[dtype] * want.abs() + 2 * (dim / 16) * 2.0 ** -23 * size + LEAST[dtype]
            assert bool(((got.double().cpu() - want).abs() <= bound).all()), i
        k[here] = GUARD
        v[here] = GUARD
    assert bool((room_k == GUARD).all()) and bool((room_v == GUARD).all())


def test_expand_into_too_little_room():
    """Rows outside the buffers are dropped: starts come from the device."""
    c = Cache(kv.BF16, 2, 128, 32, 16, [200, 50], [0, 0], key=64, value=64)
    w = c.normal(2, 128, 128).cuda()
    full_k, full_v = (torch.zeros(260, 2, 64, dtype=c.t, device="cuda") for _ in range(2))
    starts = torch.tensor([5, 205], dtype=torch.int32, device="cuda")
    c.handle.expand(c.batch, w.data_ptr(), rows(full_k), rows(full_v), starts.data_ptr(), 260)
    room = torch.full((2, 300, 2, 64), GUARD, dtype=c.t, device="cuda")
    k, v = room[0, 100:], room[1, 100:]
    starts = torch.tensor([-50, 100], dtype=torch.int32, device="cuda")
    c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), starts.data_ptr(), 120)
    torch.cuda.synchronize()
    assert torch.equal(k[:100], full_k[55:155]) and torch.equal(v[:100], full_v[55:155])
    # rows 100 .. 119 are both sequences': one of the two
    same = (k[100:120] == full_k[155:175]) | (k[100:120] == full_k[205:225])
    assert bool(same.all()) and bool((room[:, :100] == GUARD).all()) and bool((room[:, 220:] == GUARD).all())


def run_prompt(c, q, q_rope, k, v, starts, stream=None):
    room = torch.full((c.total + 2, c.heads + 1, c.value + 8), GUARD, dtype=c.t, device="cuda")
    out = room[1:-1, :c.heads, :c.value]
    lse_room = torch.full((c.total * c.heads + 2,), GUARD, device="cuda")
    d_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    ws = torch.full((c.handle.prompt_workspace_bytes(c.batch) + 64,), 0xff, dtype=torch.uint8, device="cuda")
    c.handle.prompt(c.batch, rows(q), rows(q_rope), rows(k), rows(v), d_starts.data_ptr(), k.shape[0], rows(out), ws.data_ptr(), ws.numel() - 64,
                    d_lse=lse_room[1:].data_ptr(), stream=stream or torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    kept = out.clone()
    out.fill_(GUARD)
    assert bool((room == GUARD).all()) and float(lse_room[0]) == GUARD and float(lse_room[-1]) == GUARD and bool((ws[-64:] == 0xff).all())
    return kept.cpu(), lse_room[1:-1].view(c.total, c.heads).cpu()


def check_prompt(c, q, q_rope, k, v, starts, out, lse, heads=None):
    qf = torch.cat([q, q_rope], 2).double().cpu()
    kd, vd = k.double().cpu(), v.double().cpu()
    for i, (L, n) in enumerate(zip(c.lens, c.news)):
        if n == 0:
            continue
        x, there = c.held(i)
        here = slice(starts[i], starts[i] + L)
        sees = visible(n, L) & there
        for h in heads or range(c.heads):
            hk, hv = (h if t.stride(1) else 0 for t in (k, v))
            want, want_lse, weighed, size = attend(qf[c.starts[i]:c.starts[i] + n, h], torch.cat([kd[here, hk], x[:, c.dim:]], 1), vd[here, hv], sees, c.scale)
            bound = bounds(c.dtype, want, weighed, size, vd[here, hv].abs().sum(0), L)
            got = out[c.starts[i]:c.starts[i] + n, h].double()
            assert bool(((got - want).abs() <= bound).all()), (i, h, float(((got - want).abs() / bound).max()))
            some = sees.any(1)
            got_lse = lse[c.starts[i]:c.starts[i] + n, h]
            assert bool((got_lse[~some] == -math.inf).all()) and bool((got[~some] == 0).all())
            off = (got_lse.double() - want_lse)[some].abs()
            assert bool((off <= (40 * 2.0 ** -23 * size + 2.0 ** -19 + 2.0 ** -23 * want_lse.abs() + L * 2.0 ** -26)[some]).all()), float(off.max())


def prompt_inputs(c, size=1.0, gap=3):
    starts, at = [], gap
    for n in c.lens:
        starts.append(at)
        at += n
    keys = at + gap
    k, v = strided(c.normal(keys, c.heads, c.key).cuda()), strided(c.normal(keys, c.heads, c.value).cuda(), 16)
    q = strided((size * torch.randn(c.total, c.heads, c.key, generator=c.gen)).to(c.t).cuda(), 16)
    return q, strided((size * torch.randn(c.total, c.heads, c.rope, generator=c.gen)).to(c.t).cuda()), k, v, starts


PROMPTS = [
    # heads, rope, key, value, block, lens, news
    (4, 64, 128, 128, 64, [300, 128, 1], [300, 128, 1]),
    (3, 32, 64, 64, 16, [700, 129, 0, 50], [257, 1, 0, 50]),
    (2, 64, 64, 128, 32, [1000], [130]),
    (5, 32, 128, 64, 128, [260, 515], [255, 256]),
    (1, 64, 128, 128, 16, [1, 2, 127, 130], [1, 2, 127, 129]),
]


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("heads,rope,key,value,block,lens,news", PROMPTS)
def test_prompt(dtype, heads, rope, key, value, block, lens, news):
    c = Cache(dtype, heads, 128, rope, block, lens, news, key=key, value=value, seed=heads)
    q, q_rope, k, v, starts = prompt_inputs(c, 1.5)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)


@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_prompt_with_absent_pages(block):
    lens, news = [400, 300, 2 * block, block], [20, 300, 2, 1]
    c = Cache(kv.BF16, 2, 128, 64, block, lens, news, absent=[(0, 0), (0, 300 // block), (1, 299 // block), (2, 0), (3, 0)], seed=block)
    q, q_rope, k, v, starts = prompt_inputs(c)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
def test_prompt_hidden_values_do_not_count(dtype):
    """NaN and infinities in tokens that some queries do not see, behind the sequence, and in values that some do see."""
    lens, news = [290, 200], [270, 150]
    c = Cache(dtype, 2, 128, 64, 32, lens, news, seed=11)
    q, q_rope, k, v, starts = prompt_inputs(c)
    out, _ = run_prompt(c, q, q_rope, k, v, starts)
    late = starts[0] + 280                                   # seen by the last 10 queries of the first sequence
    k[late] = math.nan
    v[late + 2, 0, 5] = math.nan
    v[late + 3, 0, 6] = -math.inf
    v[late + 4, 1, 7] = math.inf
    v[starts[1] + 200:] = math.nan                           # behind everything
    k[starts[1] + 200:] = math.inf
    v[:starts[0]] = math.inf
    again, _ = run_prompt(c, q, q_rope, k, v, starts)
    at = 280 - 20
    assert torch.equal(again[:at], out[:at]) and torch.equal(again[270:], out[270:])
    assert bool(again[at:270].isnan().all())
    k[late] = 0.5
    again, lse = run_prompt(c, q, q_rope, k, v, starts)
    vk = v.clone()
    vk[late + 2, 0, 5] = vk[late + 3, 0, 6] = vk[late + 4, 1, 7] = 0
    want, want_lse = run_prompt(c, q, q_rope, k, vk, starts)
    assert torch.equal(lse, want_lse)
    want[at + 2:270, 0, 5] = math.nan
    want[at + 3:270, 0, 6] = -math.inf
    want[at + 4:270, 1, 7] = math.inf
    assert torch.equal(again.nan_to_num(nan=1e4), want.nan_to_num(nan=1e4))


def test_prompt_keys_out_of_the_buffers():
    c = Cache(kv.BF16, 2, 128, 32, 16, [200, 60], [50, 60], key=64, value=64)
    q, q_rope, k, v, starts = prompt_inputs(c, gap=0)
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    # the first 7 tokens of the first sequence lie in front of the buffers, and the last 10 of the second behind them
    again, lse2 = run_prompt(c, q, q_rope, k[7:250], v[7:250], [-7, 193])
    assert torch.equal(again[50:100], out[50:100])
    qf, kd, vd = torch.cat([q, q_rope], 2).double().cpu(), k.double().cpu(), v.double().cpu()
    x, _ = c.held(0)
    for h in range(2):
        sees = visible(50, 200)
        sees[:, :7] = False
        want, _, weighed, size = attend(qf[:50, h], torch.cat([kd[:200, h], x[:, 128:]], 1), vd[:200, h], sees, c.scale)
        bound = bounds(kv.BF16, want, weighed, size, vd[:200, h].abs().sum(0), 200)
        assert bool(((again[:50, h].double() - want).abs() <= bound).all())
    none, none_lse = run_prompt(c, q, q_rope, k[:0], v[:0], [0, 0])
    assert bool((none == 0).all()) and bool((none_lse == -math.inf).all())


def test_prompt_heads_that_share_keys():
    """A head stride of 0: one head's rows for all."""
    c = Cache(kv.BF16, 4, 128, 64, 64, [300], [200])
    q, q_rope, k, v, starts = prompt_inputs(c)
    shared = k[:, :1].expand(-1, 4, -1)
    assert shared.stride(1) == 0
    out, lse = run_prompt(c, q, q_rope, shared, v, starts)
    check_prompt(c, q, q_rope, shared, v, starts, out, lse)


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
def test_prompt_large_scores(dtype):
    c = Cache(dtype, 2, 128, 64, 64, [900], [700], softmax_scale=0.5, seed=4)
    q, q_rope, k, v, starts = prompt_inputs(c, 2.0)
    for b in range(9):
        k[starts[0] + 100 * b] *= 0.2 + 0.3 * b
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    check_prompt(c, q, q_rope, k, v, starts, out, lse)


def test_expanded_and_absorbed_agree():
    """The two ways to attend: expanding the cache, or taking the matrices into the queries and the answers."""
    heads, dim, rope, key, value = 8, 256, 64, 64, 128
    lens, news = [500, 70], [9, 3]
    c = Cache(kv.F16, heads, dim, rope, 32, lens, news, key=key, value=value)
    w = (torch.randn(heads, key + value, dim, generator=c.gen) * dim ** -0.5).to(c.t).cuda()
    starts, keys = [0, 500], 570
    k, v = torch.empty(keys, heads, key, dtype=c.t, device="cuda"), torch.empty(keys, heads, value, dtype=c.t, device="cuda")
    d_starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.handle.expand(c.batch, w.data_ptr(), rows(k), rows(v), d_starts.data_ptr(), keys)
    q, q_rope = c.normal(c.total, heads, key).cuda(), c.normal(c.total, heads, rope).cuda()
    out, lse = run_prompt(c, q, q_rope, k, v, starts)
    absorbed = torch.einsum("thk,hkd->thd", q.float(), w[:, :key].float()).to(c.t)
    answer, lse2 = torch.empty(c.total, heads, dim, dtype=c.t, device="cuda"), torch.empty(c.total, heads, device="cuda")
    ws = torch.empty(c.handle.workspace_bytes(c.batch), dtype=torch.uint8, device="cuda")
    c.handle.attention(c.batch, rows(absorbed), rows(q_rope), rows(answer), ws.data_ptr(), ws.numel(), d_lse=lse2.data_ptr())
    back = torch.einsum("thd,hvd->thv", answer.float(), w[:, key:].float())
    # Each side rounds some vectors to 11 bits (keys, values and weights; queries, weights and answers) and sums products with random signs: scores
    # of size 1 are off by some 2^-11, and answers, of size 0.1 to 1, by some roundings of values of size 1 to 3 that are averaged: 8 half steps of 1
    assert float((lse.cuda() - lse2).abs().max()) <= 8 * 2.0 ** -11
    assert float((out.cuda().float() - back).abs().max()) <= 8 * 2.0 ** -11

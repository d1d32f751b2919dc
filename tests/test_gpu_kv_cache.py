"""Rotary positions, append, read and eviction against their definitions."""
import math
import random

import numpy as np
import pytest

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no CUDA device", allow_module_level=True)

from kv_reference import TOP, TYPES, UNIT, Cache, evict, nearest_code, rows, turn  # noqa: E402
from paper_2410_15240_b200 import fastrack, kv  # noqa: E402

pytestmark = pytest.mark.gpu
LAYOUTS = [kv.ROTARY_HALF, kv.ROTARY_INTERLEAVED]
# cos and sin come from a half turn held in 24 bits and a function good to 2 units: 2^-21 of the pair's size covers both products and their sum
TURN_ERROR = 2.0 ** -21


def handle(dtype, dim, layout, freq, gain=1.0):
    return kv.KvCache(dtype, kv.INT8, 4, 4, dim, 64, rotary=layout, frequencies=freq, rotary_gain=gain)


def pair_size(x, freq, layout):
    r, s = 2 * len(freq), x.abs()
    if layout == kv.ROTARY_HALF:
        n = s[..., :r // 2] + s[..., r // 2:r]
        s[..., :r // 2] = s[..., r // 2:r] = n
    else:
        n = s[..., 0:r:2] + s[..., 1:r:2]
        s[..., 0:r:2] = s[..., 1:r:2] = n
    return s


def check_turned(got, x, positions, freq, gain, layout, dtype, inverse=False):
    want = turn(x.double().cpu(), positions, freq, gain, layout, inverse)
    bound = UNIT[dtype] * want.abs() + gain * TURN_ERROR * pair_size(x.double().cpu(), freq, layout) + 2.0 ** -25 * (dtype == kv.F16)
    assert bool(((got.double().cpu() - want).abs() <= bound).all()), float(((got.double().cpu() - want).abs() / bound).max())
    r = 2 * len(freq)
    assert torch.equal(got[..., r:].cpu(), x[..., r:].cpu())


@pytest.mark.parametrize("dtype", [kv.BF16, kv.F16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim,part,tokens,heads", [(128, 128, 1, 1), (128, 64, 5, 32), (64, 16, 301, 3), (96, 96, 17, 7), (96, 48, 2000, 9), (64, 64, 3, 65)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rotary(dtype, layout, dim, part, tokens, heads, inverse):
    gen = torch.Generator().manual_seed(dim + tokens)
    freq, gain = kv.rotary_frequencies(part, 10000.0, kv.FREQ_RAMP, 8.0, 2048.0)
    x = torch.randn(tokens, heads, dim, generator=gen).to(TYPES[dtype]).cuda()
    positions = torch.randint(0, 100000, (tokens,), generator=gen)
    room = torch.full((tokens + 2, heads, dim), -3.0, dtype=x.dtype, device="cuda")
    out, kept, d_pos = room[1:-1], x.clone(), positions.cuda()
    h = handle(dtype, dim, layout, freq, gain)
    h.rotary(tokens, heads, rows(x), rows(out), d_pos.data_ptr(), inverse)
    torch.cuda.synchronize()
    assert torch.equal(x, kept) and bool((room[0] == -3).all()) and bool((room[-1] == -3).all())
    check_turned(out, x, positions, freq, gain, layout, dtype, inverse)
    h.rotary(tokens, heads, rows(x), rows(x), d_pos.data_ptr(), inverse)         # in place
    torch.cuda.synchronize()
    assert torch.equal(x, out)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotary_far_positions(layout):
    """The angle is as exact at 2^40 as at 1, and negative positions turn back."""
    freq = kv.rotary_frequencies(64, 10000.0)[0]
    positions = torch.tensor([0, 1, -1, 2 ** 20 + 1, 2 ** 31 + 12345, 2 ** 40 - 1, -(2 ** 33)])
    x = torch.randn(len(positions), 2, 64).to(torch.float16).cuda()
    out, d_pos = torch.empty_like(x), positions.cuda()
    handle(kv.F16, 64, layout, freq).rotary(len(positions), 2, rows(x), rows(out), d_pos.data_ptr())
    torch.cuda.synchronize()
    check_turned(out, x, positions, freq, 1.0, layout, kv.F16)
    assert torch.equal(out[0], x[0])


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotary_strides(layout):
    """A slice of one projection in, heads outermost out."""
    freq = kv.rotary_frequencies(64, 500.0)[0]
    fused = torch.randn(40, 11, 128).to(torch.bfloat16).cuda()
    x, out = fused[:, 3:8], torch.empty(5, 40, 128, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    positions = torch.arange(40) * 3
    d_pos = positions.cuda()
    handle(kv.BF16, 128, layout, freq).rotary(40, 5, rows(x), rows(out), d_pos.data_ptr())
    torch.cuda.synchronize()
    check_turned(out, x, positions, freq, 1.0, layout, kv.BF16)


@pytest.mark.parametrize("layout", LAYOUTS)
def test_rotary_gradient(layout):
    """The map is linear, so differences with any step give its matrix; the inverse turn has to be the transpose."""
    dim, part, gain = 64, 48, 1.25
    freq = kv.rotary_frequencies(part, 10000.0)[0]
    h, positions = handle(kv.F16, dim, layout, freq, gain), torch.full((dim,), 77, device="cuda")
    eye = torch.eye(dim, device="cuda").half()[:, None]
    base = torch.randint(-8, 9, (1, 1, dim), device="cuda").half() / 8
    up, down, back = (torch.empty_like(eye) for _ in range(3))
    h.rotary(dim, 1, rows((base + eye).contiguous()), rows(up), positions.data_ptr())
    h.rotary(dim, 1, rows((base - eye).contiguous()), rows(down), positions.data_ptr())
    h.rotary(dim, 1, rows(eye), rows(back), positions.data_ptr(), inverse=True)
    torch.cuda.synchronize()
    matrix = (up.double() - down.double())[:, 0] / 2    # row i: the map of channel i's unit vector
    # each of up and down is at most 4 in size (two products of at most 2 x 1.25), rounded by 2^-11 of it; back by 2^-11 of at most 1.25
    assert float((matrix - back.double()[:, 0].T).abs().max()) <= 5 * 2.0 ** -11 + 1.25 * 2.0 ** -11


def test_rotary_refusals():
    h = handle(kv.BF16, 64, kv.ROTARY_HALF, [1.0] * 16)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int64, device="cuda")
    good = dict(tokens=4, heads=2, x=rows(x), out=rows(x), d_positions=pos.data_ptr())
    for bad in (dict(tokens=-1), dict(heads=-1), dict(d_positions=0), dict(d_positions=pos.data_ptr() + 4), dict(x=kv.Rows(0, 128, 64)),
                dict(x=kv.Rows(x.data_ptr() + 8, 128, 64)), dict(out=kv.Rows(x.data_ptr(), 130, 64)), dict(out=kv.Rows(x.data_ptr(), 256, 64))):
        with pytest.raises(fastrack.FastrackError) as e:
            h.rotary(**{**good, **bad})
        assert e.value.code == fastrack.ERR_ARG, bad
    h.rotary(**{**good, "tokens": 0})
    assert h.launches == 0


# ------------------------------------------------------------------------------------------------ append and read ----

def append(c, seed=0, spread=1.0):
    gen = torch.Generator().manual_seed(seed)
    qkv = (torch.randn(c.total, c.qh + 2 * c.kh, c.d, generator=gen) * spread).to(c.t).cuda()
    q, k, v = qkv.split([c.qh, c.kh, c.kh], 1)
    q_out = torch.full((c.total, c.qh, c.d), -3.0, dtype=c.t, device="cuda")
    c.kv.append(c.batch(), rows(k), rows(v), rows(q), rows(q_out), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return q, k, v, q_out


def check_append(c, before_tail, before_pool, q, k, v, q_out):
    if c.freq:
        check_turned(q_out, q, c.positions, c.freq, c.gain, c.layout, c.dtype)
    else:
        assert torch.equal(q_out, q)
    new_k, new_v = turn(k.double().cpu(), c.positions, c.freq, c.gain, c.layout), v.double().cpu()
    size = pair_size(k.double().cpu(), c.freq, c.layout) if c.freq else torch.zeros_like(new_k)
    touched = set()
    for i, (L, n) in enumerate(zip(c.lens, c.news)):
        if n == 0:
            assert torch.equal(c.tail[i], before_tail[i], ) or bool(torch.isnan(before_tail[i]).any())
            continue
        L0 = max(L - n, 0)
        skip = max(n - L, 0)                            # new tokens that would stand before the first place
        base = L0 // c.bt * c.bt
        sl = slice(c.starts[i] + skip, c.starts[i + 1])
        old = before_tail[i].double().cpu().transpose(0, 1)[:, :, :L0 - base]             # [2][kv heads][tokens][dim]
        new = torch.stack([new_k[sl], new_v[sl]]).transpose(1, 2)
        x = torch.cat([old, new], 2)
        # a new K may be off by the turn; old ones and V are exact
        loose = torch.cat([torch.zeros_like(old), torch.stack([size[sl] * c.gain * TURN_ERROR, torch.zeros_like(new_v[sl])]).transpose(1, 2)], 2)
        for b in range(L0 // c.bt, L // c.bt):
            p = int(c.table[i, b])
            if not 0 <= p < c.pages:
                continue
            touched.add(p)
            part = slice(b * c.bt - base, (b + 1) * c.bt - base)
            codes, scales = c.page(p)
            for w in range(2):
                y, slack = x[w, :, part], loose[w, :, part]
                amax = y.abs().amax((1, 2))
                top, wide = TOP[c.fmt], slack.amax((1, 2))
                assert bool(((scales[w] - amax / top).abs() <= 2.0 ** -23 * amax / top + wide / top).all())
                zero = amax < 2.0 ** -100
                assert bool((scales[w][zero] == 0).all()) and bool((codes[w][zero] == 0).all())
                s = scales[w][:, None, None]
                half = s / 2 if c.fmt == kv.INT8 else torch.maximum(y.abs() * 2.0 ** -4, s * 2.0 ** -10)
                # the nearest code, but for the scale's and the product's rounding
                assert bool(((codes[w] * s - y).abs() <= half * (1 + 2.0 ** -12) + y.abs() * 2.0 ** -21 + slack + 1e-30)[~zero].all()), (i, b, w)
                if w == 1 and not bool(zero.any()):     # V has no turn: the same 32-bit steps give the same codes
                    y32 = y.float()
                    z = y32 * (torch.tensor(top, dtype=torch.float32) / y32.abs().amax((1, 2), keepdim=True))
                    assert torch.equal(codes[w], nearest_code(z.double().clamp(-top, top), c.fmt))
                    assert torch.equal(scales[w].float(), y32.abs().amax((1, 2)) / top)
        rest = x[:, :, (L // c.bt * c.bt) - base:] if L // c.bt * c.bt >= base else x[:, :, :0]
        got = c.tail[i].double().cpu().transpose(0, 1)[:, :, :L % c.bt]
        slack = loose[:, :, (L // c.bt * c.bt) - base:]
        assert bool(((got - rest).abs() <= UNIT[c.dtype] * rest.abs() * (slack > 0) + slack + 2.0 ** -25 * (slack > 0)).all())
    same = [p for p in range(c.pages) if p not in touched]
    assert torch.equal(c.pool[same], before_pool[same]), "a page that got no block was written"


@pytest.mark.parametrize("dtype,fmt", [(kv.BF16, kv.INT8), (kv.BF16, kv.E4M3), (kv.F16, kv.INT8), (kv.F16, kv.E4M3)])
@pytest.mark.parametrize("dim,block,part,layout", [(128, 64, 128, kv.ROTARY_HALF), (96, 16, 48, kv.ROTARY_INTERLEAVED), (64, 128, 0, kv.ROTARY_NONE),
                                                   (128, 32, 16, kv.ROTARY_INTERLEAVED)])
def test_append(dtype, fmt, dim, block, part, layout):
    freq, gain = kv.rotary_frequencies(part, 10000.0, kv.FREQ_RAMP, 4.0, 100.0) if part else (None, 1.0)
    # single tokens that do and do not complete a block; many that start, cross, fill and overfill blocks; none at all
    lens = [1, block, block + 1, 3 * block - 1, 5, 2 * block, 4 * block + 7, 3 * block, 77, 2 * block + 3]
    news = [1, 1, 1, 1, 5, 2 * block, 3 * block + 9, block + 5, 0, block]
    c = Cache(dtype, fmt, 6, 2, dim, block, lens, news, rotary=layout, freq=freq, gain=gain, seed=3)
    c.fill()
    c.tail.normal_()
    tail, pool = c.tail.clone(), c.pool.clone()
    check_append(c, tail, pool, *append(c))


@pytest.mark.parametrize("seed", range(12))
def test_append_random(seed):
    rng = random.Random(seed)
    block, n = rng.choice([16, 32, 64, 128]), rng.randint(1, 6)
    lens = [rng.randint(0, 400) for _ in range(n)]
    news = [rng.randint(0, rng.choice([1, 20, 300])) for _ in lens]        # may exceed the length: the first of them fall away
    dim = rng.choice([64, 96, 128])
    layout = rng.choice(LAYOUTS)
    c = Cache(rng.choice([0, 1]), rng.choice([0, 1]), 8, rng.choice([1, 2, 8]), dim, block, lens, news, rotary=layout,
              freq=kv.rotary_frequencies(rng.choice([16, 32, dim]), 10000.0)[0], seed=seed)
    c.fill()
    c.tail.normal_()
    if c.stride > 1 and rng.random() < 0.5:
        c.table[0, 0] = -1
        c.d_table.copy_(c.table)
    tail, pool = c.tail.clone(), c.pool.clone()
    check_append(c, tail, pool, *append(c, seed, rng.choice([1e-3, 1.0, 300.0])))


def test_append_then_steps_equal_one_append():
    """A prompt at once and the same tokens one by one leave the same V and the same tails.  K of a block that was a tail before
    was rounded to 16 bits there: its codes are at most the neighbours of those of the unrounded values."""
    freq = kv.rotary_frequencies(128, 10000.0)[0]
    make = lambda n: Cache(kv.BF16, kv.E4M3, 4, 2, 128, 16, [53, 20], [n[0], n[1]], rotary=kv.ROTARY_HALF, freq=freq, seed=9, poison=False)  # noqa: E731
    a = make([53, 20])
    _, k, v, _ = append(a, 4)
    b = make([1, 1])
    pos = torch.zeros(2, dtype=torch.int64, device="cuda")
    for t in range(53):
        live = [min(t + 1, 53), min(t + 1, 20)]
        b.d_lens.copy_(torch.tensor(live, dtype=torch.int32))
        one = [1, 1 if t < 20 else 0]
        b.d_starts.copy_(torch.tensor([0, 1, 1 + one[1]], dtype=torch.int32))
        pos.fill_(t)
        at = [t, 53 + t] if one[1] else [t, t]
        kk, vv = k[at].contiguous(), v[at].contiguous()
        b.kv.append(b.batch(d_positions=pos.data_ptr()), rows(kk), rows(vv))
        torch.cuda.synchronize()
    for i, L in enumerate(a.lens):
        for block in range(L // 16):
            (ca, sa), (cb, sb) = a.page(int(a.table[i, block])), b.page(int(b.table[i, block]))
            assert torch.equal(ca[1], cb[1]) and torch.equal(sa[1], sb[1])
            # one step of 2^-3 of a code, and what 2^-8 of scale and value can add to it
            assert bool(((ca[0] - cb[0]).abs() <= torch.maximum(ca[0].abs(), cb[0].abs()).clamp(min=2.0 ** -6) * (2.0 ** -3 + 2.0 ** -7)).all())
            assert bool(((sa[0] - sb[0]).abs() <= 2.0 ** -8 * sa[0]).all())
        assert torch.equal(a.tail[i, :, :, :L % 16], b.tail[i, :, :, :L % 16])


@pytest.mark.parametrize("fmt", [kv.INT8, kv.E4M3])
def test_append_small_zero_and_non_finite(fmt):
    c = Cache(kv.BF16, fmt, 2, 2, 64, 16, [16 * 6], [16 * 6], poison=False)
    k = torch.randn(96, 2, 64).to(torch.bfloat16)
    k[0:16] = 0
    k[16:32] *= 2.0 ** -110
    k[32:48] *= 2.0 ** -95
    k[48:64] *= 2.0 ** 100
    k[64, 0, 3] = math.nan
    k[80, 1, 5] = -math.inf
    k = k.cuda()
    c.kv.append(c.batch(), rows(k), rows(k))
    torch.cuda.synchronize()
    pages = [c.page(int(c.table[0, b])) for b in range(6)]
    for b in (0, 1):
        assert bool((pages[b][0] == 0).all()) and bool((pages[b][1] == 0).all())
    for b in (2, 3):
        y = k[16 * b:16 * b + 16].double().cpu().transpose(0, 1)
        s = pages[b][1][0][:, None, None]
        assert bool(((pages[b][0][0] * s - y).abs() <= (s / 2 if fmt == kv.INT8 else torch.maximum(y.abs() / 16, s * 2.0 ** -10)) * (1 + 2.0 ** -10)).all())
    assert bool(torch.isnan(pages[4][1][:, 0]).all()) and bool(torch.isfinite(pages[4][1][:, 1]).all())
    assert bool(torch.isinf(pages[5][1][:, 1]).all()) and bool(torch.isfinite(pages[5][1][:, 0]).all())
    assert all(bool(torch.isfinite(p[0]).all()) for p in pages)       # no code is a NaN


@pytest.mark.parametrize("dtype,fmt", [(kv.BF16, kv.INT8), (kv.F16, kv.E4M3)])
@pytest.mark.parametrize("dim,block", [(128, 64), (96, 16), (64, 128)])
def test_read(dtype, fmt, dim, block):
    c = Cache(dtype, fmt, 4, 2, dim, block, [1, 300, block, 0, 2 * block + 9], [1] * 5, seed=2)
    c.fill()
    if block == 16:
        c.table[1, 2] = -1
        c.d_table.copy_(c.table)
    k, v = (torch.full((5, c.max_len, 2, dim), -3.0, dtype=c.t, device="cuda") for _ in range(2))
    c.kv.read(c.batch(), rows(k.view(-1, 2, dim)), rows(v.view(-1, 2, dim)))
    torch.cuda.synchronize()
    for i, L in enumerate(c.lens):
        hk, hv, there = c.held(i)
        for got, want in ((k, hk), (v, hv)):
            want = torch.where(there[:, None], want, 0.0).transpose(0, 1)
            # code times scale is rounded to 32 bits, then to the type
            assert bool(((got[i, :L].double().cpu() - want).abs() <= want.abs() * (UNIT[dtype] + 2.0 ** -23) + 2.0 ** -25).all())
            assert bool((got[i, L:] == 0).all())


def test_append_and_read_refusals():
    c = Cache(kv.BF16, kv.INT8, 4, 2, 64, 16, [100, 90], [1, 1], rotary=kv.ROTARY_HALF, freq=[1.0] * 8)
    x = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    r = rows(x)
    bad_rows = (kv.Rows(0, 256, 64), kv.Rows(x.data_ptr() + 2, 256, 64), kv.Rows(x.data_ptr(), 257, 64))
    bad_batches = (c.batch(n_seqs=-1), c.batch(max_new=3), c.batch(d_lens=0), c.batch(d_tail=c.tail.data_ptr() + 4), c.batch(d_positions=0),
                   c.batch(max_len=8 * 16), c.batch(n_seqs=65536), c.batch(max_len=(1 << 30) + 1))
    calls = [lambda b=b: c.kv.append(b, r, r) for b in bad_batches] + [lambda b=b: c.kv.append(c.batch(), b, r) for b in bad_rows]
    calls += [lambda b=b: c.kv.append(c.batch(), r, b) for b in bad_rows] + [lambda b=b: c.kv.append(c.batch(), r, r, r, b) for b in bad_rows]
    calls += [lambda: c.kv.append(c.batch(), r, r, r), lambda: c.kv.append(c.batch(), r, r, None, r)]
    calls += [lambda b=b: c.kv.read(c.batch(), r, b) for b in bad_rows] + [lambda: c.kv.read(c.batch(n_seqs=-1), r, r)]
    for call in calls:
        with pytest.raises(fastrack.FastrackError) as e:
            call()
        assert e.value.code == fastrack.ERR_ARG
    c.kv.append(c.batch(n_seqs=0), r, r)
    c.kv.append(c.batch(total_new=0, max_new=0), r, r)
    assert c.kv.launches == 0


# ------------------------------------------------------------------------------------------------ evict ----

def run_evict(table, lens, mass, block, budget, first, last, in_place=False):
    n, stride = table.shape
    h = kv.KvCache(kv.BF16, kv.INT8, mass.shape[1], mass.shape[1], 64, block)
    t, l, m = torch.from_numpy(table).cuda(), torch.from_numpy(lens).cuda(), torch.from_numpy(mass).cuda()
    to, lo, mo = (t, l, m) if in_place else (torch.full_like(t, 99), torch.full_like(l, 99), torch.full_like(m, 99.0))
    ev, cnt = torch.full_like(t, 99), torch.full_like(l, 99)
    h.evict(kv.Eviction(n_seqs=n, table_stride=stride, mass_stride=mass.shape[2], budget=budget, keep_first=first, keep_last=last, d_table=t.data_ptr(),
                        d_lens=l.data_ptr(), d_mass=m.data_ptr(), d_table_out=to.data_ptr(), d_lens_out=lo.data_ptr(), d_mass_out=mo.data_ptr(),
                        d_evicted=ev.data_ptr(), d_n_evicted=cnt.data_ptr()), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return [x.cpu().numpy() for x in (to, lo, mo, ev, cnt)]


def check_evict(table, lens, mass, block, budget, first, last):
    want = evict(table, lens, mass, block, budget, first, last)
    for in_place in (False, True):
        for name, g, w in zip(("table", "lens", "mass", "evicted", "count"), run_evict(table, lens, mass, block, budget, first, last, in_place), want):
            assert np.array_equal(g, w, equal_nan=True), (name, in_place)


@pytest.mark.parametrize("seed", range(16))
def test_evict(seed):
    rng = np.random.default_rng(seed)
    n, heads, block = int(rng.integers(1, 9)), int(rng.choice([1, 2, 8])), int(rng.choice([16, 64]))
    blocks = int(rng.choice([1, 5, 40, 1023, 1024, 1025, 3001]))
    stride, m_stride = blocks + int(rng.integers(1, 4)), blocks + int(rng.integers(1, 4))
    lens = rng.integers(0, blocks * block + block, n).astype(np.int32)
    lens[0] = blocks * block + block - 1
    mass = rng.choice([rng.random((n, heads, m_stride)), rng.integers(0, 3, (n, heads, m_stride)) / 4.0]).astype(np.float32)
    table = rng.permutation(n * stride).reshape(n, stride).astype(np.int32)
    check_evict(table, lens, mass, block, int(rng.integers(0, blocks + 2)), int(rng.integers(0, 4)), int(rng.integers(0, 6)))


@pytest.mark.parametrize("heads,blocks", [(9, 40), (20, 1500), (8, 1024), (8, 1025), (8, 4096), (3, 4097), (2, 9000)])
def test_evict_on_either_side_of_what_registers_hold(heads, blocks):
    rng = np.random.default_rng(heads * blocks)
    stride = blocks                                     # the unfinished block has no entry of its own: every table ends exactly here
    table = rng.permutation(2 * stride).reshape(2, stride).astype(np.int32)
    mass = (rng.integers(0, 5, (2, heads, stride)) / 4.0).astype(np.float32)
    check_evict(table, np.array([blocks * 16, blocks * 16 // 3], np.int32), mass, 16, blocks // 2, 2, 3)


def test_evict_ties_and_odd_weights():
    table = np.arange(2 * 40, dtype=np.int32).reshape(2, 40)
    mass = np.ones((2, 3, 40), np.float32)              # all the same: the lowest index first
    check_evict(table, np.array([39 * 16 + 2, 38 * 16], np.int32), mass, 16, 20, 1, 2)
    mass[:, 1, 5] = np.nan
    mass[:, 0, 7] = np.inf
    mass[:, 2, 9] = -np.inf
    mass[:, :, 11] = 0.0
    mass[:, :, 12] = -0.0
    mass[:, :, 13] = 1e-45
    for budget in (0, 1, 10, 30, 36):
        check_evict(table, np.array([39 * 16 + 2, 38 * 16], np.int32), mass, 16, budget, 0, 0)


def test_evict_more_is_protected_than_the_budget_allows():
    table = np.arange(30, dtype=np.int32).reshape(1, 30)
    mass = np.random.default_rng(1).random((1, 2, 30)).astype(np.float32)
    for first, last in ((0, 0), (30, 0), (0, 30), (20, 20), (10, 10), (1 << 30, 1 << 30)):
        check_evict(table, np.array([29 * 16 + 5], np.int32), mass, 16, 5, first, last)


def test_evict_beyond_shared_memory():
    """More blocks than scores are kept for."""
    rng = np.random.default_rng(7)
    blocks = 60001
    table = rng.permutation(blocks + 2).reshape(1, -1).astype(np.int32)
    mass = rng.random((1, 2, blocks + 2)).astype(np.float32)
    check_evict(table, np.array([blocks * 16 + 3], np.int32), mass, 16, 5000, 3, 9)


def test_evict_refusals():
    h = kv.KvCache(kv.BF16, kv.INT8, 2, 2, 64, 16)
    t = torch.zeros(64, dtype=torch.int32, device="cuda")
    good = dict(n_seqs=1, table_stride=4, mass_stride=4, budget=1, keep_first=0, keep_last=0, **{k: t.data_ptr() for k, _ in kv.Eviction._fields_ if k[:2] == "d_"})
    for key, _ in kv.Eviction._fields_:
        for value in ([-1] if key[:2] != "d_" else [0, t.data_ptr() + 2]):
            with pytest.raises(fastrack.FastrackError) as e:
                h.evict(kv.Eviction(**{**good, key: value}))
            assert e.value.code == fastrack.ERR_ARG, key
    h.evict(kv.Eviction(**{**good, "n_seqs": 0}))
    assert h.launches == 0

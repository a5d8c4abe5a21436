"""GPU parity of the operators around a served sequence's cache against their plain
definitions (oracle/cache_oracle.py): page tables and slots, rotary positions and
their gradient, the writers of the bf16 and the 8-bit cache, decode over the 8-bit
cache, and all of them together.

Bars.  Integers, codes, copied values: equal.  Rotary values: the final rounding
(half a step: 2^-8 relative in bf16, 2^-24 in fp32) and, of |x| + |y| of the pair, what
fp32 cosines and sines may be off: 2^-24 of an angle up to pi (1.9e-7), the function
(4 ulp, 2.4e-7), the products' roundings (2^-23): 6e-7 together; beside it the 64-bit
angle, 2 pi turns 2^-51.  Decode: `decode_bars` below."""

import math

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import bf1_oracle as orc
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu

CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bf1.load()
    yield
    torch.cuda.synchronize()


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


def f64(t):
    return t.detach().double().cpu().numpy()


def normal(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


# ---- page_step ------------------------------------------------------------------------

def check_page_step(old, new, table, free, head, max_tokens, B):
    t = i32(table)
    s = bf1.page_step(i32(old), i32(new), t, i32(free), i32([head]), max_tokens, B)
    want = co.page_step(old, new, table, free, head, max_tokens, B)
    names = ("page_table",) + bf1.PageStep._fields
    got = (t,) + tuple(s)
    order = {"page_table": 0, "seq_lens": 1, "token_start": 2, "block_start": 3, "positions": 4, "slots": 5, "free_head": 6}
    for name, x in zip(names, got):
        w = np.atleast_1d(want[order[name]])
        assert np.array_equal(x.cpu().numpy(), w), name
    return s


@pytest.mark.parametrize("batch,most,B", [(1, 1, 64), (3, 200, 64), (65, 300, 128), (1024, 5, 64), (1025, 70, 64),
                                          (2500, 3, 128)])
def test_page_step_matches_the_oracle(batch, most, B):
    rng = np.random.default_rng(batch + most)
    old, new = rng.integers(0, 400, batch), rng.integers(0, most + 1, batch)
    old[rng.random(batch) < 0.2] = 0
    max_pages = (400 + most) // B + 2
    order = rng.permutation(batch * max_pages + 9)
    table = np.full((batch, max_pages), -1)
    at = 0
    for b in range(batch):
        have = -(-old[b] // B)
        table[b, :have] = order[at:at + have]
        at += have
    for extra in (0, 70):
        check_page_step(old, new, table, order, at, int(new.sum()) + extra, B)
    check_page_step(np.zeros(batch), np.zeros(batch), table, order, at, 3, B)


def test_page_step_shortages():
    B, rng = 64, np.random.default_rng(5)
    old, new = np.array([10, 64, 0, 130, 0, -3]), np.array([300, 64, 0, 500, 5, -9])
    table = rng.permutation(60).reshape(6, 10)
    for num_free in range(0, 18):  # from no free page to all that are needed
        check_page_step(old, new, table, np.arange(100, 100 + num_free), 0, 900, B)
    for head in (-4, 3, 17, 18, 40):  # a head outside the list counts as its end
        check_page_step(old, new, table, np.arange(100, 118), head, 900, B)
    for rows in (0, 1, 300, 301, 700, 1500):  # fewer rows than tokens, and more than a workgroup's
        check_page_step(old, new, table, np.arange(100, 118), 0, rows, B)
    check_page_step([0, 500], [700, 300], np.full((2, 10), -1), np.arange(30), 0, 1000, B)  # past the table
    check_page_step([2 ** 31 - 3], [9], np.full((1, 3), -1), np.arange(4), 0, 9, B)
    check_page_step([5], [2], np.array([[-1, 2]]), np.arange(4), 0, 2, B)  # a page that is missing
    check_page_step(np.zeros(0), np.zeros(0), np.zeros((0, 4)), np.arange(4), 1, 5, B)


def test_page_step_sums_past_32_bits():
    big = 2 ** 31 - 1
    s = bf1.page_step(i32([0, 0, 5, 0]), i32([big, big, big, 7]), i32(np.full((4, 2), -1)), i32(range(9)), i32([0]), 200)
    assert s.token_start.tolist() == [0, big, big, big, big]  # 2^31 - 1 at most
    assert s.seq_lens.tolist() == [128, 0, 5, 0] and s.block_start.tolist() == [0, 2, 2, 2, 2] and int(s.free_head) == 2
    assert s.positions.tolist() == list(range(128)) + [-1] * 72


def test_page_step_into_buffers_and_refusals():
    old, new, free, head = i32([3, 60]), i32([2, 9]), i32(range(9)), i32([0])
    a = bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, 20)
    b = bf1.PageStep(*(torch.full_like(t, 7) for t in a))
    assert bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, 20, out=b).slots is b.slots
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    with pytest.raises(bf1.BF1Error):  # written while every workgroup reads it
        bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, 20, out=b._replace(seq_lens=old))
    with pytest.raises(bf1.BF1Error):
        bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, 20, out=b._replace(free_head=head))
    with pytest.raises(ValueError, match="positions"):
        bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, 21, out=b)
    with pytest.raises(ValueError, match="new_lens"):
        bf1.page_step(old, i32([1]), i32(np.full((2, 4), 1)), free, head, 20)
    with pytest.raises(ValueError, match="negative"):
        bf1.page_step(old, new, i32(np.full((2, 4), 1)), free, head, -1)


# ---- rope -------------------------------------------------------------------------------

def rope_bars(x, ref, pos, freqs, amplitude, interleaved, dtype):
    """Elementwise bound of the error of rope's output (x, ref: [..., n, d])."""
    r = len(freqs)
    mag = np.zeros_like(x)
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        angle = np.abs(pos.astype(np.float64)) * freqs[i] * 2.0 ** -51
        mag[..., a] = mag[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(amplitude) * (6e-7 + angle)
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 2.0 ** -24
    return mag + half * (np.abs(ref) + mag)


def check_rope(q, k, pos, freqs, interleaved, amplitude, bwd=False, dtype=None, tokens=False):
    fn = bf1.rope_bwd if bwd else bf1.rope
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    got = fn(q, k, i32(pos), f, interleaved=interleaved, amplitude=amplitude, dtype=dtype)
    for x, y in zip((q, k), got):
        if x is None:
            assert y is None
            continue
        assert y.is_contiguous() and y.shape == x.shape and y.dtype == (dtype or x.dtype)
        xs, ys = f64(x), f64(y)
        if tokens:  # [tokens, heads, d] -> heads first
            xs, ys = xs.transpose(1, 0, 2), ys.transpose(1, 0, 2)
            p = np.asarray(pos)
        else:
            p = np.broadcast_to(np.asarray(pos), (x.shape[0], x.shape[2]))[:, None]
        ref = co.rope(xs, p, freqs, interleaved, amplitude, -1 if bwd else 1)
        bad = np.abs(ys - ref) > rope_bars(xs, ref, p, freqs, amplitude, interleaved, y.dtype)
        assert not bad.any(), (bad.sum(), np.abs(ys - ref).max())
        r = 2 * len(freqs)
        if dtype is None:
            assert np.array_equal(ys[..., r:], xs[..., r:])
    return got


@pytest.mark.parametrize("batch,n,Hq,Hkv,d,r,dtype", [
    (1, 1, 16, 8, 128, 128, torch.bfloat16), (2, 37, 4, 1, 64, 64, torch.bfloat16), (1, 300, 8, 8, 128, 64, torch.bfloat16),
    (2, 33, 3, 1, 64, 16, torch.bfloat16), (1, 50, 2, 1, 80, 20, torch.bfloat16), (1, 9, 1, 1, 10, 6, torch.bfloat16),
    (1, 5, 2, 2, 1024, 2, torch.bfloat16), (2, 129, 8, 2, 64, 32, torch.float32), (1, 77, 4, 4, 128, 128, torch.float32),
    (1, 20, 2, 1, 36, 12, torch.float32), (3, 3, 40, 5, 128, 128, torch.bfloat16), (1, 9000, 16, 8, 128, 128, torch.bfloat16),
])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_matches_the_oracle(batch, n, Hq, Hkv, d, r, dtype, interleaved):
    rng = np.random.default_rng(n + d)
    freqs = list(1e6 ** (-np.arange(0, r, 2) / r))
    pos = rng.integers(-5, 200000, (batch, n)).astype(np.int32)
    q, k = normal(1, batch, Hq, n, d, dtype=dtype), normal(2, batch, Hkv, n, d, dtype=dtype)
    check_rope(q, k, pos, freqs, interleaved, 1.0)
    check_rope(q, k, pos, freqs, interleaved, 1.139, bwd=True)
    if dtype is torch.float32:
        check_rope(q, k, pos, freqs, interleaved, 1.0, bwd=True, dtype=torch.bfloat16)


def test_rope_positions_far_and_shared():
    freqs = list(1e4 ** (-np.arange(0, 64, 2) / 64))
    pos = np.array([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6 + 1, 123456789], dtype=np.int32)
    check_rope(normal(1, 3, 2, 7, 64, dtype=torch.float32), None, pos, freqs, False, 1.0)
    check_rope(None, normal(2, 3, 1, 7, 64), pos, freqs, True, 1.0)


@pytest.mark.parametrize("d,shift", [(128, 0), (128, 1), (64, 4), (72, 8)])
def test_rope_strided_rows(d, shift):
    """Views of joined rows, aligned to 16 bytes or not, as rows and split into heads."""
    n, H, Hkv = 41, 6, 2
    flat = normal(3, n * ((H + 2 * Hkv) * d + 8) + 16)
    rows = flat[shift:shift + n * ((H + 2 * Hkv) * d + 8)].view(n, -1)
    q = rows[:, :H * d].unflatten(1, (H, d))
    k = rows[:, H * d:(H + Hkv) * d].unflatten(1, (Hkv, d))
    freqs = list(1e6 ** (-np.arange(0, d, 2) / d))
    pos = np.arange(7, 7 + n, dtype=np.int32)
    tok = check_rope(q, k, pos, freqs, False, 1.0, tokens=True)
    head = check_rope(q.transpose(0, 1)[None], k.transpose(0, 1)[None], pos, freqs, False, 1.0)
    for a, b in zip(tok, head):
        assert torch.equal(a.transpose(0, 1), b[0])


def test_rope_in_place_and_refusals():
    q, k, pos = normal(1, 1, 4, 50, 128), normal(2, 1, 2, 50, 128), i32(range(50))
    freqs, amp = bf1.rope_freqs(64, scaling="bands", factor=4.0)
    a = bf1.rope(q, k, pos, freqs, amplitude=amp)
    q2, k2 = q.clone(), k.clone()
    b = bf1.rope(q2, k2, pos, freqs, amplitude=amp, q_out=q2, k_out=k2)
    assert b[0] is q2 and torch.equal(a[0], q2) and torch.equal(a[1], k2)
    for bad, why in [(dict(positions=i32(range(49))), "positions"), (dict(positions=pos.long()), "dtype"),
                     (dict(freqs=freqs.float()), "dtype"), (dict(freqs=freqs.cpu()), "device"),
                     (dict(freqs=torch.ones(65, dtype=torch.float64, device="cuda")), "d / 2"),
                     (dict(k=k[:, :, :49]), "agree"), (dict(k=k.float()), "k must"), (dict(q=q.half()), "bf16"),
                     (dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), "side by side"),
                     (dict(q_out=torch.empty(1, 4, 50, 64, device="cuda")), "q_out"), (dict(dtype=torch.float32), "dtype")]:
        with pytest.raises(ValueError, match=why):
            bf1.rope(**{**dict(q=q, k=k, positions=pos, freqs=freqs), **bad})
    with pytest.raises(bf1.BF1Error):  # an odd head cannot be paired
        bf1.rope(normal(1, 1, 1, 3, 63), None, i32(range(3)), torch.ones(2, dtype=torch.float64, device="cuda"))
    empty = bf1.rope(q[:, :, :0], k[:, :, :0], pos[:0], freqs)
    assert empty[0].shape == (1, 4, 0, 128)


def test_rope_trains_through_attention():
    """Gradients of rope -> attn_fwd -> attn_bwd -> rope_bwd: against the formulas, and
    the loss's differences along a direction."""
    B, L, n, Hq, Hkv, d = 64, 2, 300, 4, 2, 64
    freqs, amp = bf1.rope_freqs(32, 1e4)
    pos = i32(range(1000, 1000 + n))
    q, k, v, do = (normal(s, 1, h, n, d) for s, h in ((1, Hq), (2, Hkv), (3, Hkv), (4, Hq)))

    qr, kr = bf1.rope(q, k, pos, freqs)
    o, lse = bf1.attn_fwd(qr, kr, v, B, L)
    g = bf1.attn_bwd(qr, kr, v, o, do, lse, B, L)
    dq, dk = bf1.rope_bwd(g[0], g[1], pos, freqs)

    fr = freqs.cpu().numpy()
    p = np.arange(1000, 1000 + n)
    turn = lambda t, s=1: co.rope(t, p, fr, False, amp, s)  # noqa: E731
    ref = orc.attn_bwd_gathered_fp64(turn(f64(q)), turn(f64(k)), f64(v), f64(do), B, L)
    for got, want in ((dq, turn(ref[0], -1)), (dk, turn(ref[1], -1))):
        # rounding of the turned bf16 operands and of P and dS: a few 2^-8 of the largest
        assert np.abs(f64(got) - want).max() <= 2e-2 * np.abs(want).max()

    def loss(a, b):
        out = orc.attn_gathered_fp64(turn(a), turn(b), f64(v), B, L)[0]
        return (out * f64(do)).sum()

    rng = np.random.default_rng(0)
    eq, ek, h = rng.standard_normal(q.shape), rng.standard_normal(k.shape), 1e-4
    diff = (loss(f64(q) + h * eq, f64(k) + h * ek) - loss(f64(q) - h * eq, f64(k) - h * ek)) / (2 * h)
    along = (f64(dq) * eq).sum() + (f64(dk) * ek).sum()
    size = math.sqrt((f64(dq) ** 2).sum() + (f64(dk) ** 2).sum())
    assert abs(diff - along) <= 2e-2 * size  # a direction of unit variance sees the gradient's norm


# ---- kv_append --------------------------------------------------------------------------

@pytest.mark.parametrize("T,Hkv,d,B", [(1, 1, 64, 64), (77, 8, 128, 64), (300, 3, 64, 128), (200, 2, 128, 128)])
def test_kv_append_scatters_rows(T, Hkv, d, B):
    rng = np.random.default_rng(T)
    P = T // B + 5
    slots = rng.permutation(P * B)[:T].astype(np.int64)
    slots[rng.random(T) < 0.2] = -1
    if T > 2:
        slots[:2] = [P * B, 2 ** 62]  # past the cache: left out
    kv = normal(1, T, 2 * Hkv, d)  # K and V of a token side by side
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    kp, vp = normal(2, P, Hkv, B, d), normal(3, P, Hkv, B, d)
    want = [kp.clone(), vp.clone()]
    for t, s in enumerate(slots):
        if 0 <= s < P * B:
            want[0][s // B, :, s % B], want[1][s // B, :, s % B] = k[t], v[t]
    bf1.kv_append(k, v, torch.from_numpy(slots).cuda(), kp, vp)
    assert torch.equal(kp, want[0]) and torch.equal(vp, want[1])


def test_kv_append_refusals():
    k, pages, slots = normal(1, 5, 2, 64), normal(2, 3, 2, 64, 64), torch.arange(5, device="cuda")
    for kw, why in [(dict(slots=slots.int()), "dtype"), (dict(slots=slots[:4]), "shape"), (dict(v=k[:4]), "v must"),
                    (dict(k=k.float()), "k must"), (dict(v_pages=pages[:2]), "v_pages"), (dict(k=k[:, :1]), "k must")]:
        with pytest.raises(ValueError, match=why):
            bf1.kv_append(**{**dict(k=k, v=k, slots=slots, k_pages=pages, v_pages=pages.clone()), **kw})
    odd = normal(1, 5 * 130 + 8)[1:651].view(5, 130)[:, :128].unflatten(1, (2, 64))
    with pytest.raises(bf1.BF1Error):
        bf1.kv_append(odd, odd, slots, pages, pages.clone())


# ---- kv_append_q8 -----------------------------------------------------------------------

def host(cache, fmt):
    """A CacheQ8 as the oracle's arrays (codes as bytes or int8)."""
    raw = torch.uint8 if fmt == "e4m3" else torch.int8
    out = {n: t.view(raw).cpu().numpy() if "pages" in n else t.double().cpu().numpy() if "tail" in n else t.cpu().numpy()
           for n, t in cache._asdict().items()}
    return out


def filled_cache(fmt, P, batch, Hkv, d, B, seed=9):
    """A cache that holds something everywhere, so that stray writes show."""
    c = bf1.cache_q8(P, batch, Hkv, d, B, CODES[fmt])
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in c[:2]:
        t.view(torch.int8).copy_(torch.randint(-100, 100, t.shape, generator=g, device="cuda", dtype=torch.int8))
    for t in c[2:4]:
        t.copy_(torch.rand(t.shape, generator=g, device="cuda") * 0.05 + 0.01)
    for t in c[4:]:
        t.copy_(torch.randn(t.shape, generator=g, device="cuda").to(torch.bfloat16))
    return c


def plan_step(before, new, B, seed=0, spare=3):
    """(table, after, token_start, block_start, num_pages) of a step, on the host."""
    rng = np.random.default_rng(seed)
    before, new = np.asarray(before), np.asarray(new)
    after = before + new
    blocks = -(-after // B)
    P = int(blocks.sum()) + spare
    order, at = rng.permutation(P), 0
    table = np.full((len(before), max(1, int(blocks.max()))), -1)
    for b, m in enumerate(blocks):
        table[b, :m] = order[at:at + m]
        at += m
    touched = np.where(new > 0, (after - 1) // B - before // B + 1, 0)
    z = [0]
    return table, after, np.concatenate([z, np.cumsum(new)]), np.concatenate([z, np.cumsum(touched)]), P


def check_append_q8(k, v, before, new, B, fmt, extra=0):
    table, after, ts, bs, P = plan_step(before, new, B)
    Hkv, d = k.shape[1:]
    cache = filled_cache(fmt, P, len(before), Hkv, d, B)
    ref = co.append_q8(f64(k), f64(v), before, after, ts, table, host(cache, fmt), fmt, B)
    bf1.kv_append_q8(k, v, i32(before), i32(after), i32(ts), i32(bs), i32(table), cache)
    got = host(cache, fmt)
    for n in got:
        assert np.array_equal(got[n], ref[n], equal_nan="pages" not in n), n
    return cache


STEPS = [([0], [1]), ([63], [1]), ([64], [1]), ([5, 127, 0, 63, 200], [1, 1, 0, 1, 1]), ([0, 0, 0], [64, 300, 65]),
         ([10, 64, 100, 0], [54, 200, 27, 0]), ([30, 129, 5], [500, 1, 123]), ([0] * 70, [1] * 35 + [64] * 35),
         ([0, 0], [0, 0]), (list(range(0, 390, 3)), [1] * 130)]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d,B", [(64, 64), (128, 64), (64, 128), (128, 128)])
@pytest.mark.parametrize("step", range(len(STEPS)))
def test_append_q8_matches_the_oracle(fmt, d, B, step):
    before, new = STEPS[step]
    T = sum(new)
    scale = torch.tensor([0.01, 1.0, 300.0], device="cuda")[:, None].to(torch.bfloat16)
    kv = normal(step, T + 2, 6, d)  # two rows behind the last sequence
    check_append_q8(kv[:, :3] * scale, kv[:, 3:], before, new, B, fmt)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_q8_special_blocks(fmt):
    """Ties, zeros, tiny, huge, subnormal, infinite and NaN values, each in a block of
    its own."""
    d, B = 64, 64
    g = np.random.default_rng(2)
    ties = np.concatenate([np.arange(-254, 255) / 2.0, [127.0], np.arange(-15, 16) / 16.0, [0.0] * 3])
    blocks = [np.zeros(B * d), np.full(B * d, -0.0), np.resize(np.concatenate([[254.0], ties]), B * d),
              np.resize(np.concatenate([[448.0], np.arange(1, 448) + 0.0]), B * d),
              np.resize([449.0, 1.0, 2.0 ** -9, 2.0 ** -10, 1.5 * 2.0 ** -9, -0.75], B * d),
              g.standard_normal(B * d) * 2.0 ** 120, g.standard_normal(B * d) * 2.0 ** -99,
              g.standard_normal(B * d) * 2.0 ** -110, np.resize([2.0 ** -130, 2.0 ** -100, 2.0 ** -133], B * d),
              np.resize([3.3e38, -3.3e38, 1e38, 1.0], B * d)]
    for bad in (np.inf, -np.inf, np.nan):
        x = g.standard_normal(B * d)
        x[37] = bad
        blocks.append(x)
    x = torch.tensor(np.concatenate(blocks), dtype=torch.float32).to(torch.bfloat16).cuda().view(-1, 1, d)
    n = len(blocks) * B
    check_append_q8(x, x.flip(0), [0], [n], B, fmt)


def test_append_q8_amounts_to_one_append():
    """Token by token, in chunks, or at once: the same cache."""
    B, d, Hkv, n = 64, 128, 2, 200
    k, v = normal(1, n, Hkv, d), normal(2, n, Hkv, d)
    table = i32([[3, 0, 2, 1]])
    done = []
    for cuts in ([n], [1] * n, [50, 14, 1, 70, 65], [64, 64, 64, 8]):
        cache, at = bf1.cache_q8(4, 1, Hkv, d, B), 0
        for m in cuts:
            touched = (at + m - 1) // B - at // B + 1
            bf1.kv_append_q8(k[at:at + m], v[at:at + m], i32([at]), i32([at + m]), i32([0, m]), i32([0, touched]), table,
                             cache)
            at += m
        done.append(cache)
    last = n % B
    for c in done[1:]:
        for a, b in zip(done[0][:4], c[:4]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        for a, b in zip(done[0][4:], c[4:]):
            assert torch.equal(a[:, :, :last], b[:, :, :last])


def test_append_q8_foreign_tables_stay_inside():
    """Pages outside the pool, rows past the tensors, sums that are none: nothing is
    written outside the cache, and what the tables do not name keeps its bits."""
    B, d, Hkv, P = 64, 64, 2, 6
    k, v = normal(1, 64, Hkv, d), normal(2, 64, Hkv, d)
    cases = [([0], [64], [0, 64], [0, 1], [[P]]), ([0], [64], [0, 64], [0, 1], [[-1]]),
             ([0], [128], [1000, 64], [0, 2], [[0, 1]]), ([0], [64], [-70, 64], [0, 1], [[2]]),
             ([5], [-5], [0, 64], [0, 1], [[0]]), ([0, 0], [64, 64], [0, 64, 128], [5, 2, 1], [[0], [1]]),
             ([0], [2 ** 31 - 1], [0, 64], [0, 2 ** 31 - 1], [[1]]), ([-9], [64], [0, 64], [-4, 1], [[3]])]
    for before, after, ts, bs, table in cases:
        cache = filled_cache("int8", P, len(before), Hkv, d, B)
        old = host(cache, "int8")
        bf1.kv_append_q8(k, v, i32(before), i32(after), i32(ts), i32(bs), i32(table), cache)
        new = host(cache, "int8")
        named = {p for r in table for p in r if 0 <= p < P}
        for p in set(range(P)) - named:
            assert np.array_equal(old["k_pages"][p], new["k_pages"][p]) and np.array_equal(old["v_pages"][p], new["v_pages"][p])


def test_append_q8_refusals():
    c = bf1.cache_q8(3, 2, 2, 64)
    k = normal(1, 4, 2, 64)
    ok = dict(k=k, v=k, lens_before=i32([0, 0]), seq_lens=i32([2, 2]), token_start=i32([0, 2, 4]), block_start=i32([0, 1, 2]),
              page_table=i32([[0], [1]]), cache=c)
    for kw, why in [(dict(block_start=i32([0, 1])), "block_start"), (dict(token_start=i32([0, 2])), "token_start"),
                    (dict(seq_lens=i32([1])), "seq_lens"), (dict(k=normal(1, 4, 2, 128)), "k must"),
                    (dict(cache=c._replace(v_pages=c.k_pages[:2])), "v_pages"), (dict(page_table=i32([0])), "page_table"),
                    (dict(cache=c._replace(k_scale=c.k_scale.double())), "k_scale"),
                    (dict(cache=c._replace(k_tail=c.k_tail[:1])), "k_tail"),
                    (dict(cache=c._replace(k_pages=c.k_pages.view(torch.uint8))), "k_pages")]:
        with pytest.raises(ValueError, match=why):
            bf1.kv_append_q8(**{**ok, **kw})


# ---- attn_decode_q8 -----------------------------------------------------------------------

def decode_bars(q, keys, ref):
    """(bar of o, bar of lse) of one head: o = [d], mass = sum of p |v|.  A score's fp32
    sum of d products is off by at most d 2^-24 of the sum of their magnitudes, and by
    2^-22 of itself (scales, log2 e, the subtraction of the largest); a weight by twice
    that (its own and the sum's), exp2 and the two parts of 8 bits by 2^-16; sums over
    n keys by n 2^-24; the output by half a step, 2^-8."""
    o, lse, mass = ref
    d, n = q.shape[0], keys.shape[0]
    big = (np.abs(keys) @ np.abs(q)).max() / np.sqrt(d)
    ds = big * (d * 2.0 ** -24 + 2.0 ** -22)
    rel = 2 * ds + 2.0 ** -16 + 2 * n * 2.0 ** -24
    return 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * mass * rel + 1e-30, ds + n * 2.0 ** -23 + 1e-6 + 2.0 ** -22 * abs(lse)


def decode_case(fmt, lens, Hq, Hkv, d, B, L, dense, seed, spare=4):
    """(q, cache, table): pages and scales that are used hold numbers, everything else
    (spare pages, tails past the newest token) NaN or infinity."""
    rng = np.random.default_rng(seed)
    batch = len(lens)
    blocks = -(-np.asarray(lens) // B)
    P = int(blocks.sum()) + spare
    cache = bf1.cache_q8(P, batch, Hkv, d, B, CODES[fmt])
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in cache[:2]:
        x = torch.randn(t.shape, generator=g, device="cuda")
        t.copy_((x * 40).round().clamp(-127, 127).to(CODES[fmt]))
    for t in cache[2:4]:
        t.copy_(torch.rand(t.shape, generator=g, device="cuda") * 0.03 + 0.005)
    for t in cache[4:]:
        t.copy_(torch.randn(t.shape, generator=g, device="cuda").to(torch.bfloat16))
    order, at = rng.permutation(P), 0
    table = np.zeros((batch, max(1, int(blocks.max()))), dtype=np.int32)
    for b, m in enumerate(blocks):
        table[b, :m] = order[at:at + m]
        at += m
    unused = torch.from_numpy(order[at:]).cuda()
    own = torch.tensor([table[b, m - 1] for b, m in enumerate(blocks) if m], device="cuda", dtype=torch.int64)
    for p in (unused, own):  # the newest block's page is not read either
        for t in cache[:2]:
            t.view(torch.uint8)[p] = 0x7f
        for t in cache[2:4]:
            t[p] = float("nan")
    for b, n in enumerate(lens):
        cache.k_tail[b, :, (n - 1) % B + 1 if n else 0:] = float("inf")
        cache.v_tail[b, :, (n - 1) % B + 1 if n else 0:] = float("nan")
    return normal(seed + 1, batch, Hq, d), cache, table


def keys_of(cache, table, b, h, n, B, L, dense):
    """Float64 keys and values of sequence b, kv-head h, that its newest token sees."""
    j = (n - 1) // B
    blocks = list(range(j)) if dense else [i for i in orc.route(j, L) if i < j]
    ks, vs = [], []
    for i in blocks:
        p = int(table[b][i])
        ks.append(f64(cache.k_pages[p, h].float()) * float(cache.k_scale[p, h]))
        vs.append(f64(cache.v_pages[p, h].float()).T * float(cache.v_scale[p, h]))
    m = (n - 1) % B + 1
    ks.append(f64(cache.k_tail[b, h, :m]))
    vs.append(f64(cache.v_tail[b, h, :m]))
    return np.concatenate(ks), np.concatenate(vs)


def run_decode(q, cache, table, lens, B, L, dense, stride=None, **kw):
    stride = stride or bf1.decode_plan_stride(int(max(lens)), B, L, dense)
    plan = bf1.decode_plan(i32(lens), i32(table), cache.k_pages.shape[0], stride, B, L, dense)
    return bf1.attn_decode_q8(q, cache, i32(lens), plan, B=B, **kw), plan


def check_decode(q, cache, table, lens, B, L, dense, heads=None, stride=None):
    (o, lse), _ = run_decode(q, cache, table, lens, B, L, dense, stride)
    o, lse, qd = f64(o), f64(lse), f64(q)
    Hkv, G = cache.k_pages.shape[1], q.shape[1] // cache.k_pages.shape[1]
    for b, n in enumerate(lens):
        for h in range(Hkv) if heads is None else heads:
            k, v = keys_of(cache, table, b, h, n, B, L, dense)
            for x in range(h * G, (h + 1) * G):
                ref = co.decode(qd[b, x], k, v)
                bo, bl = decode_bars(qd[b, x], k, ref)
                assert (np.abs(o[b, x] - ref[0]) <= bo).all(), (b, n, x, np.abs(o[b, x] - ref[0]).max())
                assert abs(lse[b, x] - ref[1]) <= bl, (b, n, x)


LENS = [1, 2, 63, 64, 65, 127, 128, 129, 193, 600, 1000]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("B", [64, 128])
def test_decode_q8_matches_the_oracle(fmt, d, G, B):
    for L, dense in ((2, False), (2, True)):
        q, cache, table = decode_case(fmt, LENS, 2 * G, 2, d, B, L, dense, G + d)
        check_decode(q, cache, table, LENS, B, L, dense)


@pytest.mark.parametrize("fmt,lens,Hq,Hkv,d,B,L,dense", [
    ("e4m3", [32768], 16, 8, 128, 64, 2, False), ("int8", [20001, 5], 8, 1, 128, 64, 2, True),
    ("e4m3", [30000, 29999, 64, 1], 4, 2, 64, 128, 3, True), ("int8", [9000] * 40 + [77], 16, 16, 64, 64, 1, False),
    ("e4m3", [3000] * 300, 4, 2, 64, 64, 2, False), ("int8", [1], 1, 1, 64, 64, 0, False),
])
def test_decode_q8_long_and_many(fmt, lens, Hq, Hkv, d, B, L, dense):
    q, cache, table = decode_case(fmt, lens, Hq, Hkv, d, B, L, dense, 7)
    pick = range(len(lens)) if len(lens) < 5 else [0, 1, len(lens) // 2, len(lens) - 1]
    (o, lse), _ = run_decode(q, cache, table, lens, B, L, dense)
    G = Hq // Hkv
    for b in pick:
        for h in {0, Hkv - 1}:
            k, v = keys_of(cache, table, b, h, lens[b], B, L, dense)
            for x in {h * G, h * G + G - 1}:
                ref = co.decode(f64(q)[b, x], k, v)
                bo, bl = decode_bars(f64(q)[b, x], k, ref)
                assert (np.abs(f64(o)[b, x] - ref[0]) <= bo).all() and abs(f64(lse)[b, x] - ref[1]) <= bl
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_decode_q8_many_rows_of_long_lists():
    """320 (sequence, kv-head) rows, cut so that the compute units fill evenly."""
    lens = [7000 + 13 * i for i in range(40)]
    q, cache, table = decode_case("e4m3", lens, 8, 8, 64, 64, 2, True, 8)
    assert bf1.decode_q8_workspace_size(40, 8, 8, 64, 64, 122) > 0
    (o, lse), _ = run_decode(q, cache, table, lens, 64, 2, True)
    for b, h in ((0, 0), (17, 3), (39, 7)):
        k, v = keys_of(cache, table, b, h, lens[b], 64, 2, True)
        ref = co.decode(f64(q)[b, h], k, v)
        bo, bl = decode_bars(f64(q)[b, h], k, ref)
        assert (np.abs(f64(o)[b, h] - ref[0]) <= bo).all() and abs(f64(lse)[b, h] - ref[1]) <= bl
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_decode_q8_into_buffers():
    """The caller's outputs and a workspace that holds anything: the same bits; without
    an LSE the outputs alone."""
    lens = [5000, 900]
    q, cache, table = decode_case("e4m3", lens, 4, 2, 128, 128, 2, True, 9)
    (a, la), plan = run_decode(q, cache, table, lens, 128, 2, True)
    need = bf1.decode_q8_workspace_size(2, 4, 2, 128, 128, plan.shape[1])
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    out, lse = torch.full_like(a, 7), torch.full_like(la, 7)
    got = bf1.attn_decode_q8(q, cache, i32(lens), plan, B=128, out=out, lse=lse, workspace=ws)
    assert got[0] is out and got[1] is lse and torch.equal(out, a) and torch.equal(lse, la)
    assert (ws[need:] == 255).all()


def test_nothing_to_do():
    none = i32([])
    cache = bf1.cache_q8(3, 0, 2, 64)
    o, lse = bf1.attn_decode_q8(normal(1, 0, 4, 64), cache, none, i32(np.zeros((0, 5))))
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)
    k = normal(1, 0, 2, 64)
    bf1.kv_append_q8(k, k, none, none, i32([0]), i32([0]), i32(np.zeros((0, 3))), cache)
    pages = normal(2, 3, 2, 64, 64)
    want = pages.clone()
    bf1.kv_append(k, k, torch.empty(0, dtype=torch.int64, device="cuda"), pages, pages.clone())
    assert torch.equal(pages, want)


def test_decode_q8_short_lists_in_wide_rows():
    """Lists far shorter than their plan row could hold, down to one block."""
    lens = [1, 64, 65, 4000, 700]
    q, cache, table = decode_case("e4m3", lens, 8, 2, 128, 64, 2, True, 3)
    for stride in (66, 300, 2051):
        check_decode(q, cache, table, lens, 64, 2, True, stride=stride)


def test_decode_q8_agrees_with_the_bf16_decode():
    """Codes under powers of two are exact in bf16, so pages written out in bf16 hold
    the same numbers."""
    B, L, d, Hkv, lens = 64, 2, 128, 2, [1, 64, 700, 1500]
    q, cache, table = decode_case("e4m3", lens, 8, Hkv, d, B, L, False, 5)
    for t in cache[2:4]:
        t.copy_(torch.exp2(torch.round(torch.log2(t.nan_to_num(1.0)))))
    kp = (cache.k_pages.float() * cache.k_scale[..., None, None]).to(torch.bfloat16)
    vp = (cache.v_pages.float() * cache.v_scale[..., None, None]).transpose(2, 3).to(torch.bfloat16).contiguous()
    for b, n in enumerate(lens):
        p = int(table[b, (n - 1) // B])
        kp[p], vp[p] = cache.k_tail[b], cache.v_tail[b]
    (o, lse), plan = run_decode(q, cache, table, lens, B, L, False)
    o2, lse2 = bf1.attn_decode(q, kp, vp, i32(lens), plan, B)
    assert torch.isfinite(o).all()
    # both are within their weights' 16 or 24 bits of the same numbers, then rounded
    assert (o.float() - o2.float()).abs().max() <= 2.0 ** -7 * o2.float().abs().max()
    assert (lse - lse2).abs().max() <= 2e-5


def test_decode_q8_special_values():
    B, L, d = 64, 2, 64
    lens = [200, 200, 0, 130, 200]
    q, cache, table = decode_case("e4m3", [max(n, 1) for n in lens], 4, 2, d, B, L, False, 11)
    (base, lse0), plan = run_decode(q, cache, table, lens, B, L, False)
    assert torch.isnan(base[2]).all() and torch.isnan(lse0[2]).all()  # an empty place
    assert torch.isfinite(base[[0, 1, 3, 4]]).all()
    plan = plan.clone()
    plan[3, 0] = 0  # made for another block
    plan[4, 1] = plan.shape[1]  # more pages than the row holds
    cache.v_tail[0, 1, 3, 5] = float("inf")  # shows as itself, in its own column and kv-head
    cache.v_tail[0, 1, 4, 7] = -float("inf")
    cache.k_scale[int(table[1][0]), 0] = float("nan")  # a block that held no numbers
    o, lse = bf1.attn_decode_q8(q, cache, i32(lens), plan, B=B)
    assert torch.equal(o[0, :2], base[0, :2]) and (o[0, 2:, 5] == float("inf")).all()
    assert (o[0, 2:, 7] == -float("inf")).all()
    rest = torch.ones(d, dtype=torch.bool, device="cuda")
    rest[[5, 7]] = False
    assert torch.equal(o[0, 2:][:, rest], base[0, 2:][:, rest])
    assert torch.isnan(o[1, :2]).all() and torch.equal(o[1, 2:], base[1, 2:])
    assert torch.isnan(o[3:]).all() and torch.isnan(lse[3:]).all()
    cache.k_tail[0, 0, 2] = float("inf")  # a score without a value
    q[0, 0, 0] = -q[0, 0, 1].abs() - 1
    assert torch.isnan(bf1.attn_decode_q8(q, cache, i32(lens), plan, B=B)[0][0, 0]).all()


def test_decode_q8_infinite_value_at_the_smallest_weight():
    """A key 100 natural units below the largest has a weight of e^-100, under the
    normal range of exp2: its infinity still counts."""
    d = 64
    cache = bf1.cache_q8(1, 1, 1, d, 64)
    q = torch.full((1, 1, d), 1.0, dtype=torch.bfloat16, device="cuda")
    cache.k_tail[0, 0, 0, 0] = 800.0   # score 100
    cache.k_tail[0, 0, 1, 0] = 0.0     # score 0
    cache.v_tail[0, 0, 1, 3] = float("inf")
    o, lse = bf1.attn_decode_q8(q, cache, i32([2]), i32([[0, 0, 0]]))
    assert o[0, 0, 3] == float("inf") and (o[0, 0, [0, 1, 2, 4]] == 0).all() and abs(float(lse) - 100) < 1e-4


def test_decode_q8_offsets_past_32_bits():
    """The last pages of a cache of 5 GB."""
    Hkv, d, B = 8, 128, 64
    P = 5 * 2 ** 30 // (Hkv * d * B)
    pages = [torch.empty((P, Hkv) + s, dtype=torch.int8, device="cuda") for s in ((B, d), (d, B))]
    lens = [300]
    q, small, table = decode_case("int8", lens, 16, Hkv, d, B, 2, False, 2)
    n = small.k_pages.shape[0]
    scales = [torch.full((P, Hkv), float("nan"), device="cuda") for _ in range(2)]
    for i in range(2):
        pages[i][P - n:] = small[i]
        scales[i][P - n:] = small[2 + i]
    big = bf1.CacheQ8(*pages, *scales, *small[4:])
    (a, la), _ = run_decode(q, small, table, lens, B, 2, False)
    (b, lb), _ = run_decode(q, big, table + (P - n), lens, B, 2, False)
    assert torch.equal(a, b) and torch.equal(la, lb) and torch.isfinite(a).all()
    # and the writer there
    k, v = normal(1, 64, Hkv, d), normal(2, 64, Hkv, d)
    args = (k, v, i32([0]), i32([64]), i32([0, 64]), i32([0, 1]))
    bf1.kv_append_q8(*args, i32([[0]]), small)
    bf1.kv_append_q8(*args, i32([[P - n]]), big)
    assert torch.equal(big.k_pages[P - n], small.k_pages[0]) and torch.equal(big.v_pages[P - n], small.v_pages[0])


def test_decode_q8_repeats_its_bits_and_refuses():
    lens = [5000, 100]
    q, cache, table = decode_case("int8", lens, 8, 2, 128, 64, 2, True, 4)
    (a, la), plan = run_decode(q, cache, table, lens, 64, 2, True)
    for _ in range(3):
        b, lb = bf1.attn_decode_q8(q, cache, i32(lens), plan)
        assert torch.equal(a, b) and torch.equal(la, lb)
    for kw, why in [(dict(B=128), "pages of B"), (dict(q=q[:1]), "k_tail"), (dict(seq_lens=i32([1])), "batch"),
                    (dict(plan=plan[:1]), "batch"), (dict(out=torch.empty_like(q).float()), "out"),
                    (dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), "workspace"),
                    (dict(lse=torch.empty(2, 4, device="cuda")), "lse"), (dict(q=q[..., :64].contiguous()), "cache")]:
        with pytest.raises(ValueError, match=why):
            bf1.attn_decode_q8(**{**dict(q=q, cache=cache, seq_lens=i32(lens), plan=plan), **kw})


# ---- all of them together -----------------------------------------------------------------

def serve(fmt, B, L, prompts, steps, graph, seed=1):
    """Prompts, then `steps` single tokens for every sequence; after each step the cache's
    decode is checked against float64 attention over what the cache holds, and the
    cache against the oracle's."""
    rng = np.random.default_rng(seed)
    Hq, Hkv, d, batch = 4, 2, 64, len(prompts)
    freqs, amp = bf1.rope_freqs(d, 1e4, "bands", 2.0, 4096)
    fr = freqs.cpu().numpy()
    max_pages = (max(prompts) + steps) // B + 1
    P = batch * max_pages
    table, free = torch.full((batch, max_pages), -1, dtype=torch.int32, device="cuda"), i32(rng.permutation(P))
    lens, head, new = i32([0] * batch), i32([0]), i32(prompts)
    cache = bf1.cache_q8(P, batch, Hkv, d, B, CODES[fmt]) if fmt != "bf16" else None
    kp = torch.zeros((P, Hkv, B, d), dtype=torch.bfloat16, device="cuda")
    vp = torch.zeros_like(kp)
    stride = bf1.decode_plan_stride(max(prompts) + steps, B, L)
    hist_k = [np.zeros((0, Hkv, d)) for _ in prompts]  # the turned keys and the values, as written
    hist_v = [np.zeros((0, Hkv, d)) for _ in prompts]

    def step(rows, out=None):
        """One step of joined rows [tokens, (Hq + 2 Hkv), d]."""
        q, k, v = rows.split((Hq, Hkv, Hkv), 1)
        s = bf1.page_step(lens, new, table, free, head, rows.shape[0], B, out=out)
        q, k = bf1.rope(q, k, s.positions, freqs, amplitude=amp)
        if cache is None:
            bf1.kv_append(k, v, s.slots, kp, vp)
        else:
            bf1.kv_append_q8(k, v, lens, s.seq_lens, s.token_start, s.block_start, table, cache)
        plan = bf1.decode_plan(s.seq_lens, table, P, stride, B, L)
        last = (s.token_start[1:] - 1).clamp(min=0).long()
        qn = q[last]
        if cache is None:
            o, lse = bf1.attn_decode(qn, kp, vp, s.seq_lens, plan, B)
        else:
            o, lse = bf1.attn_decode_q8(qn, cache, s.seq_lens, plan, B=B)
        lens.copy_(s.seq_lens)
        head.copy_(s.free_head)
        return s, qn, k, v, o, lse

    def check(got, m):
        s, qn, k, v, o, lse = got
        at = 0
        for b in range(batch):
            hist_k[b] = np.concatenate([hist_k[b], f64(k)[at:at + m[b]]])
            hist_v[b] = np.concatenate([hist_v[b], f64(v)[at:at + m[b]]])
            at += m[b]
            n = len(hist_k[b])
            assert int(s.seq_lens[b]) == n
            j = (n - 1) // B
            for h in range(Hkv):
                ks, vs = [], []
                for i in [i for i in orc.route(j, L) if i < j]:
                    x, y = hist_k[b][i * B:(i + 1) * B, h], hist_v[b][i * B:(i + 1) * B, h]
                    if cache is not None:
                        x, y = (co.dequantise(*co.quantise(t, fmt), fmt) for t in (x, y))
                    ks.append(x)
                    vs.append(y)
                ks = np.concatenate(ks + [hist_k[b][j * B:, h]])
                vs = np.concatenate(vs + [hist_v[b][j * B:, h]])
                for x in (2 * h, 2 * h + 1):
                    ref = co.decode(f64(qn)[b, x], ks, vs)
                    bo, bl = decode_bars(f64(qn)[b, x], ks, ref)
                    assert (np.abs(f64(o)[b, x] - ref[0]) <= bo).all(), (b, n, x)
                    assert abs(f64(lse)[b, x] - ref[1]) <= bl, (b, n, x)

    T = sum(prompts)
    rows = normal(seed, T + 5, Hq + 2 * Hkv, d)  # padded behind the last sequence
    got = step(rows)
    p = f64(got[0].positions)[:T]
    want = co.rope(f64(rows)[:T, Hq:Hq + Hkv].transpose(1, 0, 2), p, fr, False, amp)
    bars = rope_bars(f64(rows)[:T, Hq:Hq + Hkv].transpose(1, 0, 2), want, p, fr, amp, False, torch.bfloat16)
    assert (np.abs(f64(got[2])[:T].transpose(1, 0, 2) - want) <= bars).all()
    assert (got[0].slots[T:] == -1).all()
    check(got, prompts)
    new.fill_(1)
    rows = normal(seed + 1, batch, Hq + 2 * Hkv, d)
    if graph:
        keep = [t.clone() for t in (lens, head, table)] + [t.view(torch.uint8).clone() for t in (cache or (kp, vp))]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(rows)  # a first pass outside the capture
        torch.cuda.current_stream().wait_stream(side)
        for t, x in zip((lens, head, table), keep):
            t.copy_(x)
        for t, x in zip(cache or (kp, vp), keep[3:]):
            t.view(torch.uint8).copy_(x)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = step(rows)
    for i in range(steps):
        rows.copy_(normal(seed + 2 + i, batch, Hq + 2 * Hkv, d))
        if graph:
            g.replay()
            torch.cuda.synchronize()
        else:
            got = step(rows)
        check(got, [1] * batch)
    taken = sum(-(-(n + steps) // B) for n in prompts)
    assert int(head[0]) == taken


@pytest.mark.parametrize("fmt", ["bf16", "e4m3", "int8"])
def test_serving_steps(fmt):
    serve(fmt, 64, 2, [130, 1, 63, 700], 4, graph=False)


@pytest.mark.parametrize("fmt,B", [("e4m3", 128), ("int8", 64), ("bf16", 64)])
def test_serving_steps_captured_and_replayed(fmt, B):
    serve(fmt, B, 2, [125, 62, 300], 6, graph=True)


def test_both_ways_of_marshalling_agree():
    """The usual call goes through native code, one that names a stream (or is unusual
    otherwise) through Python: the same results, on the same stream."""
    here = torch.cuda.current_stream()
    lens, new, free, head = i32([3, 60, 0]), i32([2, 9, 700]), i32(range(30)), i32([2])
    tables = [i32(np.full((3, 12), 1)) for _ in range(3)]
    a = bf1.page_step(lens, new, tables[0], free, head, 720)
    b = bf1.page_step(lens, new, tables[1], free, head, 720, stream=here)
    c = bf1.page_step(lens, new, tables[2], free, head, np.int64(720))
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z) and x.dtype == y.dtype and x.shape == y.shape
    assert torch.equal(tables[0], tables[1]) and torch.equal(tables[0], tables[2])

    freqs, amp = bf1.rope_freqs(64, scaling="bands", factor=2.0)
    for dtype in (torch.bfloat16, torch.float32):
        rows = normal(1, 2, 37, 6, 128, dtype=dtype)
        for q, k, pos in ((rows[0, :, :4], rows[0, :, 4:], i32(range(37))),
                          (rows[:, :, :4].transpose(1, 2), rows[:, :, 4:].transpose(1, 2), i32(range(37))),
                          (rows[:, :, :4].transpose(1, 2), rows[:, :, 4:].transpose(1, 2), i32(np.arange(74).reshape(2, 37)))):
            for fn in (bf1.rope, bf1.rope_bwd):
                for inter in (False, True):
                    x = fn(q, k, pos, freqs, interleaved=inter, amplitude=amp)
                    y = fn(q, k, pos, freqs, interleaved=inter, amplitude=amp, stream=here)
                    assert all(torch.equal(u, v) and u.is_contiguous() for u, v in zip(x, y))
        p = torch.nn.Parameter(q.clone(), requires_grad=True)  # served, and no graph is made
        assert torch.equal(bf1.rope(p, k, pos, freqs, amplitude=amp)[0], bf1.rope(q, k, pos, freqs, amplitude=amp)[0])
        assert torch.equal(bf1.rope(q, k, pos, freqs, amplitude=1)[0], bf1.rope(q, k, pos, freqs, amplitude=1.0)[0])

    kv = normal(3, 720, 4, 64)
    pages = [normal(4, 32, 2, 64, 64) for _ in range(4)]
    bf1.kv_append(kv[:, :2], kv[:, 2:], a.slots, pages[0], pages[1])
    bf1.kv_append(kv[:, :2], kv[:, 2:], a.slots, pages[2], pages[3], stream=here)
    assert torch.equal(pages[0], pages[2]) and torch.equal(pages[1], pages[3])

    caches = [filled_cache("e4m3", 32, 3, 2, 64, 64) for _ in range(2)]
    bf1.kv_append_q8(kv[:, :2], kv[:, 2:], lens, a.seq_lens, a.token_start, a.block_start, tables[0], caches[0])
    bf1.kv_append_q8(kv[:, :2], kv[:, 2:], lens, a.seq_lens, a.token_start, a.block_start, tables[0], caches[1], stream=here)
    for x, y in zip(*caches):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))

    for many, dense in (([200, 9], False), ([9000, 70], True)):  # without and with splits
        q, cache, table = decode_case("int8", many, 4, 2, 64, 64, 2, dense, 12)
        (x, lx), plan = run_decode(q, cache, table, many, 64, 2, dense)
        y, ly = bf1.attn_decode_q8(q, tuple(cache), i32(many), plan, stream=here)
        assert torch.equal(x, y) and torch.equal(lx, ly) and lx.shape == ly.shape
    side = torch.cuda.Stream()
    side.wait_stream(here)
    with torch.cuda.stream(side):  # the current stream, whichever it is
        torch.cuda._sleep(10 ** 7)
        z, lz = bf1.attn_decode_q8(q, cache, i32(many), plan)
        z, lz = z.clone(), lz.clone()
    side.synchronize()
    assert torch.equal(x, z) and torch.equal(lx, lz)


def test_another_stream():
    """On a stream of the caller's, with memory of the operators' own: the same bits."""
    lens = [5000, 321, 64]
    q, cache, table = decode_case("e4m3", lens, 8, 2, 128, 64, 2, True, 6)
    freqs, _ = bf1.rope_freqs(128)
    pos = i32(range(3))
    (a, la), plan = run_decode(q, cache, table, lens, 64, 2, True)
    r = bf1.rope(q, None, pos, freqs)[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = []
    for _ in range(20):
        got.append((bf1.attn_decode_q8(q, cache, i32(lens), plan, stream=s), bf1.rope(q, None, pos, freqs, stream=s)[0]))
    torch.cuda.synchronize()
    for (b, lb), x in got:
        assert torch.equal(a, b) and torch.equal(la, lb) and torch.equal(r, x)

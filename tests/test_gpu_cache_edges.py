"""GPU tests of the cache's operators where their size or their inputs change the
path: precision of the decode's weights, searches over many sequences, lanes that own
two heads, far positions, guards around every buffer.  Against the plain definitions
(oracle/cache_oracle.py); helpers and bars are tests/test_gpu_cache.py's."""

import gc
import operator
import sys
import threading
import time
from functools import partial

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import cache_oracle as co
from test_gpu_cache import (CODES, check_rope, decode_case, f64, filled_cache, host, i32, normal, plan_step,
                            run_decode)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bf1.load()
    yield
    torch.cuda.synchronize()


# ---- attn_decode_q8: bits of the weights -------------------------------------------------

@pytest.mark.parametrize("fmt", ["e4m3", "int8", "tail"])
@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d,B", [(64, 64), (128, 64), (64, 128), (128, 128)])
def test_decode_q8_weights_keep_their_bits(fmt, G, d, B):
    """Pairs of keys whose weights differ by 2^-16 of themselves, with opposite values: an
    output is the difference.  Weights of w bits put an error of up to 2^-w of the pair's
    mass on it.  In fp32: four roundings of a score below 1.5 (4 |s| 2^-24 of the weight),
    exp2 (2^-23), the value's scale (2^-24), six sums (6 2^-24): below 2^-20; then half
    a bf16 step of the output."""
    tail, Hkv = fmt == "tail", 2
    Hq = G * Hkv
    cache = bf1.cache_q8(2, 1, Hkv, d, B, CODES["int8" if tail else fmt])
    code = torch.zeros((B, d))
    value = torch.zeros((B, d))
    for i in range(B // 2):
        code[2 * i:2 * i + 2, 0] = -(1 + i % 15)
        code[2 * i + 1, 1] = 1
        value[2 * i, i], value[2 * i + 1, i] = 1, -1
    ks, vs = (0.5, 0.75) if not tail else (1.0, 1.0)
    q = torch.zeros((1, Hq, d))
    for h in range(Hq):
        q[0, h, 0] = (0.5 + h / 32) * (0.5 if tail else 1)
        q[0, h, 1] = 2.0 ** -13 if tail else 2.0 ** -12
    q = q.to(torch.bfloat16).cuda()
    if tail:
        cache.k_tail.copy_(code.cuda().expand(1, Hkv, B, d))
        cache.v_tail.copy_(value.cuda().expand(1, Hkv, B, d))
        n, plan = B, [[0, 0, 0]]
        keys, values = code, value
    else:
        cache.k_pages[1] = code.cuda().to(CODES[fmt])
        cache.v_pages[1] = value.t().contiguous().cuda().to(CODES[fmt])
        cache.k_scale.fill_(ks)
        cache.v_scale.fill_(vs)
        n, plan = B + 1, [[1, 1, 1, 0]]  # and one key of the tail: zeros
        keys, values = (torch.cat([x * s, torch.zeros(1, d)]) for x, s in ((code, ks), (value, vs)))
    o, _ = bf1.attn_decode_q8(q, cache, i32([n]), i32(plan), B=B)
    o = f64(o)
    for h in range(Hq):
        ref, _, mass = co.decode(f64(q)[0, h], f64(keys), f64(values))
        assert (np.abs(ref[:B // 2]) > 0).all()
        bad = np.abs(o[0, h] - ref) > 2.0 ** -8 * np.abs(ref) + 2.0 ** -20 * mass
        assert not bad.any(), (h, bad.sum(), np.abs(o[0, h] - ref).max() / mass.max())


@pytest.mark.parametrize("G", [1, 2, 4, 8])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_q8_infinite_values_under_every_part(G, d):
    """An infinite value shows as itself whatever the parts of its key's weight: under a
    weight of 1 (two of them are 0), of e^-100, and of any other size."""
    cache = bf1.cache_q8(1, 1, 1, d, 64)
    q = torch.ones((1, G, d), dtype=torch.bfloat16, device="cuda")
    for key, score in enumerate((100.0, 0.0, 99.3, 99.9, 95.0)):
        cache.k_tail[0, 0, key, 0] = round(score * d ** 0.5)
        cache.v_tail[0, 0, key] = 1.0
        cache.v_tail[0, 0, key, 2 * key] = float("inf")
        cache.v_tail[0, 0, key, 2 * key + 1] = -float("inf")
    cache.v_tail[0, 0, 3, 20] = float("nan")
    cache.v_tail[0, 0, 1, 21], cache.v_tail[0, 0, 2, 21] = float("inf"), -float("inf")
    o, lse = bf1.attn_decode_q8(q, cache, i32([5]), i32([[0, 0, 0]]))
    o = o[0].float()
    assert (o[:, 0:10:2] == float("inf")).all() and (o[:, 1:10:2] == -float("inf")).all()
    assert torch.isnan(o[:, 20:22]).all() and (o[:, 10:20] == 1).all() and (o[:, 22:] == 1).all()
    assert torch.isfinite(lse).all()


# ---- rope: far positions, two heads per lane ---------------------------------------------

@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_far_positions_keep_fp32(interleaved):
    """Turns of (1, 0) and (0, 1) are cosines and sines alone.  Theirs may be off by the
    function's 4 ulp (4 * 2^-24 of at most 1) and two more roundings of what is turned
    back and of the output (2^-24 each): 6 * 2^-24, whatever the position."""
    d, n = 128, 4096
    rng = np.random.default_rng(1)
    freqs = rng.uniform(0.3, 1.0, d // 2)
    pos = np.concatenate([rng.integers(2 ** 30, 2 ** 31, n - 6), [2 ** 31 - 1, -2 ** 31, 0, 1, -1, 2 ** 27]]).astype(np.int32)
    x = torch.zeros((1, 2, n, d))
    first = torch.arange(0, d, 2) if interleaved else torch.arange(d // 2)
    x[0, 0, :, first] = 1
    x[0, 1, :, first + (1 if interleaved else d // 2)] = 1
    f = torch.as_tensor(freqs, device="cuda")
    for fn, sign in ((bf1.rope, 1), (bf1.rope_bwd, -1)):
        y, _ = fn(x.cuda(), None, i32(pos), f, interleaved=interleaved)
        off = np.abs(f64(y) - co.rope(f64(x), pos, freqs, interleaved, 1.0, sign))
        assert off.max() <= 6 * 2.0 ** -24, off.max()


# ---- binding: other threads ----------------------------------------------------------------

def _calls():
    """The usual call of each operator that is marshalled natively, as a function of no
    arguments."""
    m = bf1._native()
    k, pages = normal(1, 3, 2, 64), normal(2, 3, 2, 64, 64)
    lens, new, table = i32([0, 0, 0]), i32([1, 1, 1]), i32([[0], [1], [2]])
    start = i32([0, 1, 2, 3])
    cache = bf1.cache_q8(3, 3, 2, 64)
    freqs = torch.ones(32, dtype=torch.float64, device="cuda")
    return {"page_step": partial(m.page_step, lens, new, table, i32(range(9)), i32([0]), 3, 64),
            "rope": partial(m.rope, k, k, lens, freqs, False, 1.0, 0),
            "kv_append": partial(m.kv_append, k, k, torch.arange(3, device="cuda"), pages, pages.clone()),
            "kv_append_q8": partial(m.kv_append_q8, k, k, lens, new, start, start, table, cache),
            "attn_decode_q8": partial(m.attn_decode_q8, normal(3, 3, 4, 64), cache, new, i32(np.zeros((3, 4))), 64)}


@pytest.mark.parametrize("name", ["page_step", "rope", "kv_append", "kv_append_q8", "attn_decode_q8"])
def test_other_threads_run_during_a_native_call(name):
    """A row of calls with no Python code between them: another thread gets ahead only
    where a call releases the interpreter's lock."""
    call = _calls()[name]
    assert call() is not None
    ticks, stop = [], threading.Event()

    def tick():
        while not stop.is_set():
            ticks.append(None)
            time.sleep(0)

    other = threading.Thread(target=tick)
    interval = sys.getswitchinterval()
    gc.disable()
    sys.setswitchinterval(1e-5)
    try:
        other.start()
        while not ticks:
            time.sleep(0.001)
        row = [ticks.__len__] + [call] * 1000 + [ticks.__len__]
        got = list(map(operator.methodcaller("__call__"), row))
    finally:
        stop.set()
        sys.setswitchinterval(interval)
        gc.enable()
        other.join()
    torch.cuda.synchronize()
    assert got[-1] > got[0]


# ---- strides that nothing uses ---------------------------------------------------------------

@pytest.mark.parametrize("shape,strides", [((1, 2, 64), (131, 64, 1)), ((5, 1, 64), (64, 33, 1)), ((1, 1, 128), (1, 7, 1))])
def test_strides_of_a_single_row_or_head_are_not_used(shape, strides):
    """One row, or one kv-head, whose stride is no multiple of what a load takes."""
    T, Hkv, d = shape
    x, y = normal(1, 2048), normal(2, 2048)
    odd = [t.as_strided(shape, strides) for t in (x, y)]
    even = [t.as_strided(shape, strides).clone(memory_format=torch.contiguous_format).view(shape) for t in (x, y)]
    pos, freqs = i32(range(100, 100 + T)), torch.linspace(0.01, 1.0, d // 2, dtype=torch.float64, device="cuda")
    got = []
    for k, v in (odd, even):
        pages = [normal(3, 2, Hkv, 64, d) for _ in range(2)]
        bf1.kv_append(k, v, torch.arange(60, 60 + T, device="cuda"), *pages)
        cache = bf1.cache_q8(2, 1, Hkv, d)
        bf1.kv_append_q8(k, v, i32([64 - T]), i32([64]), i32([0, T]), i32([0, 1]), i32([[1]]), cache)
        turned = bf1.rope(k, v, pos, freqs)
        heads = bf1.rope(k.transpose(0, 1)[None], v.transpose(0, 1)[None], pos, freqs)
        got.append([*pages, *cache, *turned, *heads])
    for a, b in zip(*got):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ---- kv_append_q8: what a repeated step needs ------------------------------------------------

def _bytes(cache):
    return [t.view(torch.uint8).clone() for t in cache]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("before,new", [(3, 20), (0, 64), (64, 200), (10, 54), (128, 1), (63, 1)])
def test_append_q8_repeats_inside_a_block_or_from_its_start(fmt, before, new):
    d, B, Hkv = 64, 64, 2
    k, v = normal(1, new, Hkv, d), normal(2, new, Hkv, d)
    cache = filled_cache(fmt, 6, 1, Hkv, d, B)
    touched = (before + new - 1) // B - before // B + 1
    args = (k, v, i32([before]), i32([before + new]), i32([0, new]), i32([0, touched]), i32([[4, 1, 0, 5, 2]]), cache)
    bf1.kv_append_q8(*args)
    once = _bytes(cache)
    bf1.kv_append_q8(*args)
    assert all(torch.equal(a, b) for a, b in zip(once, _bytes(cache)))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("before,new", [([50], [40]), ([63, 5, 100], [2, 300, 27]), ([20], [64])])
def test_append_q8_repeats_across_blocks_with_its_tails_put_back(fmt, before, new):
    d, B, Hkv = 64, 64, 2
    k, v = normal(1, sum(new), Hkv, d), normal(2, sum(new), Hkv, d)
    table, after, ts, bs, P = plan_step(before, new, B)
    cache = filled_cache(fmt, P, len(before), Hkv, d, B)
    tails = [t.clone() for t in cache[4:]]
    args = (k, v, i32(before), i32(after), i32(ts), i32(bs), i32(table), cache)
    bf1.kv_append_q8(*args)
    once = _bytes(cache)
    for t, x in zip(cache[4:], tails):
        t.copy_(x)
    bf1.kv_append_q8(*args)
    assert all(torch.equal(a, b) for a, b in zip(once, _bytes(cache)))


# ---- kv_append_q8: many sequences ------------------------------------------------------------

@pytest.mark.parametrize("fmt,batch,active", [("int8", 256, 200), ("e4m3", 257, 257), ("int8", 513, 300),
                                              ("e4m3", 3000, 900), ("int8", 66000, 150)])
def test_append_q8_finds_its_sequence_among_many(fmt, batch, active):
    """A block's sequence is searched 256 table entries at a time: one pass, two, and for
    more than 65536 sequences three.  Places without rows, rows that complete a block or
    none, blocks on both sides of every 256.  Against the oracle over the active places;
    the others keep what they had."""
    d, B = 64, 64
    rng = np.random.default_rng(batch)
    edges = [i for i in (0, 255, 256, 257, 511, 512, batch - 2, batch - 1) if i < batch]
    at = np.unique(np.concatenate([edges, rng.permutation(batch)[:active]]))
    before, new = np.zeros(batch, dtype=np.int64), np.zeros(batch, dtype=np.int64)
    before[rng.random(batch) < 0.3] = 70  # also of places without rows
    before[at] = rng.choice([0, 10, 63, 64, 127], len(at))
    new[at] = rng.choice([1, 1, 54, 64, 65, 130], len(at))
    new[edges], before[edges] = 1, 63  # each completes a block
    table, after, ts, bs, P = plan_step(before, new, B)
    T = int(ts[-1])
    k, v = normal(1, T, 1, d), normal(2, T, 1, d)
    cache = filled_cache(fmt, P, batch, 1, d, B)
    first = cache._replace(k_tail=cache.k_tail[at], v_tail=cache.v_tail[at])
    ref = co.append_q8(f64(k), f64(v), before[at], after[at], ts[:-1][at], table[at], host(first, fmt), fmt, B)
    rest = torch.ones(batch, dtype=torch.bool)
    rest[at] = False
    old = [t[rest.cuda()] for t in cache[4:]]
    bf1.kv_append_q8(k, v, i32(before), i32(after), i32(ts), i32(bs), i32(table), cache)
    got = host(cache._replace(k_tail=cache.k_tail[at], v_tail=cache.v_tail[at]), fmt)
    for n in got:
        assert np.array_equal(got[n], ref[n]), n
    assert all(torch.equal(t[rest.cuda()], x) for t, x in zip(cache[4:], old))


# ---- rope: two heads per lane ----------------------------------------------------------------

# the lanes of these calls own two heads each (256 workgroups and more with one), the last
# of an odd number of heads one
TWO_HEADS = [(1, 1700, 3, 2, 128, 128, torch.bfloat16), (1, 1200, 7, 0, 128, 128, torch.bfloat16),
             (1, 1200, 3, 2, 128, 64, torch.bfloat16), (2, 500, 3, 2, 128, 128, torch.float32),
             (1, 330, 2, 1, 80, 20, torch.bfloat16), (1, 800, 1, 2, 36, 12, torch.float32),
             (3, 300, 4, 3, 64, 32, torch.float32)]


@pytest.mark.parametrize("batch,n,Hq,Hkv,d,r,dtype", TWO_HEADS)
@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_two_heads_per_lane(batch, n, Hq, Hkv, d, r, dtype, interleaved):
    """Against the oracle, and the same bits as calls on few tokens (a head per lane)."""
    rng = np.random.default_rng(n)
    freqs = list(1e6 ** (-np.arange(0, r, 2) / r))
    pos = rng.integers(-5, 200000, (batch, n)).astype(np.int32)
    q = normal(1, batch, Hq, n, d, dtype=dtype)
    k = normal(2, batch, Hkv, n, d, dtype=dtype) if Hkv else None
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    for bwd, out in ((False, None), (True, None)) + (((True, torch.bfloat16),) if dtype is torch.float32 else ()):
        big = check_rope(q, k, pos, freqs, interleaved, 1.139, bwd=bwd, dtype=out)
        fn = bf1.rope_bwd if bwd else bf1.rope
        for a in (0, n // 2, n - 17):
            part = [None if x is None else x[:, :, a:a + 17] for x in (q, k)]
            small = fn(*part, i32(pos[:, a:a + 17]), f, interleaved=interleaved, amplitude=1.139, dtype=out)
            for x, y in zip(big, small):
                assert x is None or torch.equal(x[:, :, a:a + 17], y)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rope_two_heads_per_lane_in_place(interleaved, dtype):
    q, k, pos = normal(1, 1, 3, 1700, 128, dtype=dtype), normal(2, 1, 2, 1700, 128, dtype=dtype), i32(range(1700))
    freqs, amp = bf1.rope_freqs(64, scaling="bands", factor=4.0)
    a = bf1.rope(q, k, pos, freqs, interleaved, amp)
    b = bf1.rope(q, k, pos, freqs, interleaved, amp, q_out=q, k_out=k)
    assert b[0] is q and b[1] is k and torch.equal(a[0], q) and torch.equal(a[1], k)


# ---- guards around the buffers ---------------------------------------------------------------

GUARD = 1 << 16


def guarded(t):
    """A copy of t between two guards; (copy, all of its memory)."""
    raw = torch.full((2 * GUARD + t.numel() * t.element_size(),), 0xa5, dtype=torch.uint8, device="cuda")
    inner = raw[GUARD:GUARD + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
    inner.copy_(t)
    return inner, raw


def untouched(raw):
    return bool((raw[:GUARD] == 0xa5).all()) and bool((raw[-GUARD:] == 0xa5).all())


FOREIGN = [([0], [64], [0, 64], [0, 1], [[6]]), ([0], [64], [0, 64], [0, 1], [[-1]]), ([0], [64], [0, 64], [0, 1], [[7]]),
           ([0], [128], [1000, 64], [0, 2], [[0, 1]]), ([0], [64], [-70, 64], [0, 1], [[2]]),
           ([5], [-5], [0, 64], [0, 1], [[0]]), ([0, 0], [64, 64], [0, 64, 128], [5, 2, 1], [[0], [1]]),
           ([0], [2 ** 31 - 1], [0, 64], [0, 2 ** 31 - 1], [[1]]), ([-9], [64], [0, 64], [-4, 1], [[3]]),
           ([30, 0], [70, 64], [0, 40, 64], [0, 2, 3], [[6, 4], [5, 6]])]


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("case", range(len(FOREIGN)))
def test_append_q8_foreign_tables_change_nothing_else(fmt, case):
    """Six pages; tables that name others, rows past the tensors, sums that are none.
    Around every buffer nothing is written, pages that no table names keep codes and
    scales, and a row of a tail keeps what it held or takes the row that the tables
    give it."""
    before, after, ts, bs, table = FOREIGN[case]
    B, d, Hkv, P, T = 64, 64, 2, 6, 64
    k, v = normal(1, T, Hkv, d), normal(2, T, Hkv, d)
    old = filled_cache(fmt, P, len(before), Hkv, d, B)
    both = [guarded(t) for t in old]
    cache = bf1.CacheQ8(*(t for t, _ in both))
    bf1.kv_append_q8(k, v, i32(before), i32(after), i32(ts), i32(bs), i32(table), cache)
    assert all(untouched(raw) for _, raw in both)
    named = {p for r in table for p in r if 0 <= p < P}
    for p in set(range(P)) - named:
        for x, y in zip(old[:4], cache[:4]):
            assert torch.equal(x[p].view(torch.uint8), y[p].view(torch.uint8))
    for x, was, now in ((k, old.k_tail, cache.k_tail), (v, old.v_tail, cache.v_tail)):
        for b in range(len(before)):
            start = max(before[b], 0)
            end = max(after[b], start)
            last = (end - 1) // B * B
            for r in range(B):
                row = ts[b] + last + r - start
                given = start <= last + r < end and 0 <= row < T
                assert torch.equal(now[b, :, r], was[b, :, r]) or (given and torch.equal(now[b, :, r], x[row]))


@pytest.mark.parametrize("lens,splits", [([200, 70], False), ([9000, 70], True)])
def test_decode_q8_without_an_lse(lens, splits):
    """O alone, with one split and with several, between guards: the same bits, and
    nothing beside them or behind the workspace."""
    q, cache, table = decode_case("int8", lens, 4, 2, 64, 64, 2, True, 9)
    (want, _), plan = run_decode(q, cache, table, lens, 64, 2, True)
    need = bf1.decode_q8_workspace_size(2, 4, 2, 64, 64, plan.shape[1])
    assert (need > 0) == splits
    o, o_raw = guarded(torch.zeros_like(want))
    ws, ws_raw = guarded(torch.zeros(need, dtype=torch.uint8, device="cuda"))
    lens = i32(lens)
    status = bf1.load().bf1_decode_attn_q8(
        q.data_ptr(), *(t.data_ptr() for t in cache), lens.data_ptr(), cache.k_pages.shape[0], plan.data_ptr(),
        plan.shape[1], o.data_ptr(), None, 2, 4, 2, 64, 64, 1, ws.data_ptr() if need else None, need,
        torch.cuda.current_stream().cuda_stream)
    assert status == bf1.BF1_OK
    torch.cuda.synchronize()
    assert torch.equal(o, want) and untouched(o_raw) and untouched(ws_raw)

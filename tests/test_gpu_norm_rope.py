"""GPU parity of the norm of queries and keys with their rotary positions, and of its
gradient, against float64 (oracle/serve_oracle.py).

Bars, as parts of 2^-24 (U, half an fp32 step): a sum of squares over d <= 512 elements
is a chain of 16 in a lane and six lane moves, so 22 U of itself, r then 11 U and 3 more
for the mean, the root and the quotient; x r g two products more: 16 U of a value, 1e-6.
The turn: 6e-7 of |a| + |b| of the pair (an angle up to pi off by U, cosine and sine 4 ulp,
the products), and 2 pi turns 2^-51 of the 64-bit angle.  The result is rounded once: 2^-8
relative in bf16, 2^-24 in fp32."""

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import bf1_oracle as orc
from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: U}


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


def heads_first(x, tokens):
    """[..., heads, n, d] of [tokens, heads, d] or [batch, heads, n, d]."""
    return f64(x).transpose(1, 0, 2) if tokens else f64(x)


def spread(mag, pos, freqs, interleaved, amplitude):
    """What the turn adds to the error of elements of size mag: of |a| + |b| of a pair."""
    out = np.zeros_like(mag)
    r = len(freqs)
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        part = 6e-7 + np.abs(np.asarray(pos, dtype=np.float64)) * freqs[i] * 2.0 ** -51
        out[..., a] = out[..., b] = (mag[..., a] + mag[..., b]) * abs(amplitude) * part
    return out


def widest(mag, freqs, interleaved, amplitude):
    """Bound of a turned element: amplitude times |a| + |b| of its pair."""
    out = mag.copy()
    r = len(freqs)
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        out[..., a] = out[..., b] = (mag[..., a] + mag[..., b]) * abs(amplitude)
    return out


def check_forward(x, y, gain, pos, freqs, interleaved, amplitude, eps, tokens=False):
    xs, ys = heads_first(x, tokens), heads_first(y, tokens)
    g = np.ones(x.shape[-1]) if gain is None else f64(gain)
    p = np.asarray(pos) if tokens else np.broadcast_to(np.asarray(pos), (x.shape[0], x.shape[2]))[:, None]
    ref = so.norm_rope(xs, g, p, freqs, interleaved, amplitude, eps)
    mag = np.abs(xs) / np.sqrt((xs * xs).mean(-1, keepdims=True) + eps) * np.abs(g)
    bar = spread(mag, p, freqs, interleaved, amplitude) + 16 * U * widest(mag, freqs, interleaved, amplitude)
    bar = bar + HALF[y.dtype] * (np.abs(ref) + bar) + 1e-40
    bad = np.abs(ys - ref) > bar
    assert not bad.any(), (bad.sum(), np.abs(ys - ref).max())


def check_backward(dy, x, gain, pos, freqs, interleaved, amplitude, eps, dx, tokens=False):
    """Checks dx; returns the gain's gradient and its bar without the sum over rows."""
    xs, ds = heads_first(x, tokens), heads_first(dy, tokens)
    g = np.ones(x.shape[-1]) if gain is None else f64(gain)
    p = np.asarray(pos) if tokens else np.broadcast_to(np.asarray(pos), (x.shape[0], x.shape[2]))[:, None]
    ref, share = so.norm_rope_bwd(ds, xs, g, p, freqs, interleaved, amplitude, eps)
    r = 1 / np.sqrt((xs * xs).mean(-1, keepdims=True) + eps)
    n = np.abs(xs) * r
    dn = widest(np.abs(ds), freqs, interleaved, amplitude)
    off = spread(np.abs(ds), p, freqs, interleaved, amplitude) + 2 * U * dn  # of dn
    u, du = dn * np.abs(g), off * np.abs(g)
    along, dalong = (u * n).mean(-1, keepdims=True), ((du + 44 * U * u) * n).mean(-1, keepdims=True)
    bar = r * (du + n * dalong + 20 * U * (u + n * along))
    bar = bar + HALF[dx.dtype] * (np.abs(ref) + bar) + 1e-40
    bad = np.abs(heads_first(dx, tokens) - ref) > bar
    assert not bad.any(), (bad.sum(), np.abs(heads_first(dx, tokens) - ref).max())
    axes = tuple(range(share.ndim - 1))
    return share.sum(axes), ((off + 18 * U * dn) * n).sum(axes), (dn * n).sum(axes)


SIZES = [
    (1, 1, 16, 8, 128, 128, torch.bfloat16), (2, 37, 4, 1, 64, 64, torch.bfloat16), (1, 300, 8, 8, 128, 64, torch.bfloat16),
    (2, 33, 3, 1, 64, 16, torch.bfloat16), (1, 50, 2, 1, 80, 20, torch.bfloat16), (1, 9, 1, 1, 10, 6, torch.bfloat16),
    (1, 5, 2, 2, 512, 2, torch.bfloat16), (2, 129, 8, 2, 64, 32, torch.float32), (1, 77, 4, 4, 128, 128, torch.float32),
    (1, 20, 2, 1, 36, 12, torch.float32), (3, 3, 40, 5, 128, 128, torch.bfloat16), (1, 3, 3, 2, 512, 512, torch.float32),
    (1, 41, 2, 3, 96, 96, torch.bfloat16), (1, 17, 3, 2, 2, 2, torch.bfloat16), (1, 2500, 16, 8, 128, 128, torch.bfloat16),
]


def case(batch, n, Hq, Hkv, d, r, dtype):
    rng = np.random.default_rng(n + d)
    freqs = list(1e6 ** (-np.arange(0, r, 2) / r))
    pos = rng.integers(-5, 200000, (batch, n)).astype(np.int32)
    q, k = normal(1, batch, Hq, n, d, dtype=dtype), 3 * normal(2, batch, Hkv, n, d, dtype=dtype)
    gains = [(1 + 0.3 * normal(s, d, dtype=torch.float32)).to(dtype) for s in (3, 4)]
    return q, k, *gains, pos, freqs, torch.tensor(freqs, dtype=torch.float64, device="cuda")


@pytest.mark.parametrize("batch,n,Hq,Hkv,d,r,dtype", SIZES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_matches_the_oracle(batch, n, Hq, Hkv, d, r, dtype, interleaved):
    q, k, qg, kg, pos, freqs, f = case(batch, n, Hq, Hkv, d, r, dtype)
    for gains, amp, kw in [((qg, kg), 1.0, {}), ((None, kg), 1.139, {}), ((qg.float(), None), 1.0, {})] + \
            ([((qg, kg), 1.0, {"dtype": torch.bfloat16})] if dtype is torch.float32 else []):
        got = bf1.qk_norm_rope(q, k, *gains, i32(pos), f, eps=1e-5, interleaved=interleaved, amplitude=amp, **kw)
        for x, y, g in zip((q, k), got, gains):
            assert y.is_contiguous() and y.dtype == kw.get("dtype", dtype)
            check_forward(x, y, g, pos, freqs, interleaved, amp, 1e-5)


@pytest.mark.parametrize("batch,n,Hq,Hkv,d,r,dtype", SIZES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_gradient_matches_the_oracle(batch, n, Hq, Hkv, d, r, dtype, interleaved):
    q, k, qg, kg, pos, freqs, f = case(batch, n, Hq, Hkv, d, r, dtype)
    ways = [(torch.float32, None, (qg, kg))] + ([(torch.bfloat16, torch.float32, (None, kg))]
                                                if dtype is torch.bfloat16 else [(torch.float32, torch.bfloat16, (qg, None))])
    for grad, out, gains in ways:
        dq, dk = normal(5, *q.shape, dtype=grad), normal(6, *k.shape, dtype=grad)
        got = bf1.qk_norm_rope_bwd(dq, dk, q, k, *gains, i32(pos), f, eps=1e-5, interleaved=interleaved, amplitude=1.139,
                                   dtype=out)
        for x, dy, g, dx, dg in zip((q, k), (dq, dk), gains, got[:2], got[2:]):
            assert dx.dtype == (out or dtype) and dx.is_contiguous()
            want, off, mag = check_backward(dy, x, g, pos, freqs, interleaved, 1.139, 1e-5, dx)
            if g is None:
                assert dg is None
                continue
            # a lane sums the rows of its tiles (up to 16 heads of a token each, for these sizes
            # one tile a workgroup), then the teams of a workgroup (256 lanes, d / 16 or d / 8 a
            # team, a power of two), 32 records and 32 threads follow one after the other
            teams = 256 // 2 ** max(0, int(np.ceil(np.log2(d / (16 if dtype is torch.bfloat16 else 8) + 1))) - 1)
            bar = off + (16 + teams + 32 + 32) * U * mag + U * np.abs(want)
            assert (np.abs(f64(dg) - want) <= bar).all(), np.abs(f64(dg) - want).max()


@pytest.mark.parametrize("d,r", [(512, 2), (512, 12), (512, 508), (510, 4), (508, 2), (512, 8), (506, 2), (504, 252)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_of_wide_float32_rows(d, r, interleaved):
    """Rows of four elements a lane and half that take all of a wave, or more than there is of
    it: turning parts and tails that both leave a remainder.  The sums' chains are those of the
    other rows, at most 16 elements of a lane and six moves."""
    q, k, qg, kg, pos, freqs, f = case(2, 9, 3, 2, d, r, torch.float32)
    for out in (None, torch.bfloat16):
        got = bf1.qk_norm_rope(q, k, qg, kg, i32(pos), f, eps=1e-5, interleaved=interleaved, amplitude=1.139, dtype=out)
        for x, y, g in zip((q, k), got, (qg, kg)):
            check_forward(x, y, g, pos, freqs, interleaved, 1.139, 1e-5)
        dq, dk = normal(5, *q.shape, dtype=torch.float32), normal(6, *k.shape, dtype=torch.float32)
        got = bf1.qk_norm_rope_bwd(dq, dk, q, k, qg, kg, i32(pos), f, eps=1e-5, interleaved=interleaved, amplitude=1.139,
                                   dtype=out)
        for x, dy, g, dx, dg in zip((q, k), (dq, dk), (qg, kg), got[:2], got[2:]):
            want, off, mag = check_backward(dy, x, g, pos, freqs, interleaved, 1.139, 1e-5, dx)
            bar = off + (3 + 8 + 32 + 32) * U * mag + U * np.abs(want)  # three heads, teams of 32 lanes or more
            assert (np.abs(f64(dg) - want) <= bar).all(), np.abs(f64(dg) - want).max()


@pytest.mark.parametrize("batch,n,Hq,Hkv,d,r,dtype", [(1, 30, 1, 1, 128, 128, torch.bfloat16), (2, 300, 4, 2, 64, 16, torch.bfloat16),
                                                      (1, 700, 5, 2, 128, 64, torch.float32), (1, 260, 2, 1, 512, 2, torch.float32),
                                                      (1, 33000, 1, 1, 128, 128, torch.bfloat16),
                                                      (1, 16500, 2, 1, 128, 32, torch.float32)])
def test_gains_gradient_is_summed_in_64_bits(batch, n, Hq, Hkv, d, r, dtype):
    """Rows of +-1 (their norm is 1) at position 0 with gradients that are whole numbers: each
    row's share is one, below 2^24, and a sum in 64 bits is exact.  The large ones cancel, wherever
    they lie: what is left is a number that float32 holds, and has to be equal.  One workgroup a
    side, several, and more tiles than workgroups."""
    f = torch.ones(r // 2, dtype=torch.float64, device="cuda")
    pos, gain = i32([0] * n), torch.ones(d, device="cuda")
    sides, want = [], []
    for i, heads in enumerate((Hq, Hkv)):
        g = torch.Generator().manual_seed(i)
        rows = batch * heads * n
        share = torch.randint(-2 ** 23, 2 ** 23, (rows, d), generator=g)
        share[rows - rows // 2:] = -share[:rows // 2][torch.randperm(rows // 2, generator=g)]
        if rows % 2:
            share[rows // 2] = 0
        share += torch.randint(-3, 4, (rows, d), generator=g)
        x = 2 * torch.randint(0, 2, (rows, d), generator=g) - 1
        want.append(share.sum(0))
        assert want[-1].abs().max() < 2 ** 24
        sides.append([t.view(batch, heads, n, d).cuda() for t in ((share * x).float(), x.to(dtype))])
    (dq, q), (dk, k) = sides
    _, _, dqg, dkg = bf1.qk_norm_rope_bwd(dq, dk, q, k, gain, gain, pos, f, eps=1e-30)
    assert torch.equal(dqg.cpu().double(), want[0].double()) and torch.equal(dkg.cpu().double(), want[1].double())


@pytest.mark.parametrize("tokens,batch,n,Hq,Hkv,d,r,dtype", [(True, 1, 33000, 1, 1, 128, 128, torch.bfloat16),
                                                            (False, 2, 16500, 3, 1, 128, 64, torch.bfloat16),
                                                            (False, 1, 16500, 1, 1, 128, 128, torch.float32),
                                                            (True, 1, 41, 6, 2, 128, 128, torch.bfloat16),
                                                            (True, 1, 333, 3, 1, 80, 20, torch.float32)])
def test_norm_rope_gradient_of_packed_and_of_many_rows(tokens, batch, n, Hq, Hkv, d, r, dtype):
    """Gradients of packed rows [tokens, heads, d], parts of joined ones, and of so many rows
    that a workgroup goes over several tiles (more than 2048 of them), gains included: their
    sums, in 64 bits, add half a step to what the rows' own errors come to."""
    freqs = list(1e6 ** (-np.arange(0, r, 2) / r))
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    pos = np.random.default_rng(n).integers(0, 100000, n if tokens else (batch, n)).astype(np.int32)
    gains = [1 + 0.3 * normal(s, d, dtype=torch.float32) for s in (3, 4)]
    if tokens:
        joined = normal(1, n, Hq + Hkv + 1, d, dtype=dtype)
        x = joined[:, :Hq], joined[:, Hq:Hq + Hkv]
        dy = normal(5, n, Hq + 1, d, dtype=torch.float32)[:, 1:], normal(6, n, Hkv, d, dtype=torch.float32)
    else:
        x = normal(1, batch, Hq, n, d, dtype=dtype), normal(2, batch, Hkv, n, d, dtype=dtype)
        dy = tuple(normal(5 + i, *t.shape, dtype=torch.float32) for i, t in enumerate(x))
    got = bf1.qk_norm_rope_bwd(*dy, *x, *gains, i32(pos), f, amplitude=1.139)
    for a, b, g, dx, dg in zip(x, dy, gains, got[:2], got[2:]):
        assert dx.shape == a.shape and dx.is_contiguous()
        want, off, _ = check_backward(b, a, g, pos, freqs, False, 1.139, 1e-6, dx, tokens=tokens)
        assert (np.abs(f64(dg) - want) <= off + U * (np.abs(want) + off)).all(), np.abs(f64(dg) - want).max()


def test_norm_rope_gradient_by_differences():
    # the loss sum(w y) along a direction: the central difference in float32 at h = 2^-6 of
    # size-1 rows is off by h^2 / 6 times the third derivative (some 10 per row, times the
    # direction's size cubed) and by 2^-24 |y| / h per element, taken as a random walk
    n, H, d = 40, 3, 64
    x = normal(1, 1, H, n, d, dtype=torch.float32)
    v, w = normal(2, *x.shape, dtype=torch.float32), normal(3, *x.shape, dtype=torch.float32)
    gain = 1 + 0.2 * normal(4, d, dtype=torch.float32)
    pos, (f, amp) = i32(range(n)), bf1.rope_freqs(32, 1e4)
    v = v / v.square().sum(-1, keepdim=True).sqrt()  # rows of size 1 next to rows of size 8
    h = 2.0 ** -6

    def loss(t, g):
        return (bf1.qk_norm_rope(t, None, g, None, pos, f)[0].double() * w).sum()

    dx, _, dg, _ = bf1.qk_norm_rope_bwd(w, None, x, None, gain, None, pos, f)
    rows = H * n
    got = float((dx.double() * v).sum())
    diff = float(loss(x + h * v, gain) - loss(x - h * v, gain)) / (2 * h)
    # y is a function of x / 8: the third derivative of a row's w y is at most 15 |w| |y| / 8^3
    third = 15 * 8 * 8 / 8 ** 3
    assert abs(got - diff) < rows * third * h * h / 6 + 8 * np.sqrt(rows * d) * 8 * U / h
    vg = normal(7, d, dtype=torch.float32)
    diff = float(loss(x, gain + h * vg) - loss(x, gain - h * vg)) / (2 * h)
    assert abs(float((dg.double() * vg).sum()) - diff) < 8 * np.sqrt(rows * d) * 8 * U / h


@pytest.mark.parametrize("d,shift", [(128, 0), (128, 1), (64, 4), (72, 8)])
def test_norm_rope_strided_rows(d, shift):
    """Views of joined rows, aligned to 16 bytes or not, as rows and split into heads; the
    same bits as of contiguous tensors; gradients back into joined rows."""
    n, H, Hkv = 41, 6, 2
    width = (H + 2 * Hkv) * d + 8

    def joined(seed, dtype=torch.bfloat16):
        flat = normal(seed, n * width + 16, dtype=dtype)
        rows = flat[shift:shift + n * width].view(n, -1)
        return rows, rows[:, :H * d].unflatten(1, (H, d)), rows[:, H * d:(H + Hkv) * d].unflatten(1, (Hkv, d))

    _, q, k = joined(3)
    r = d // 2 * 2
    freqs = list(1e6 ** (-np.arange(0, r, 2) / r))
    f = torch.tensor(freqs, dtype=torch.float64, device="cuda")
    pos = np.arange(7, 7 + n, dtype=np.int32)
    qg, kg = 1 + 0.3 * normal(4, d, dtype=torch.float32), 1 + 0.3 * normal(5, d, dtype=torch.float32)
    tok = bf1.qk_norm_rope(q, k, qg, kg, i32(pos), f)
    split = q.transpose(0, 1)[None], k.transpose(0, 1)[None]
    head = bf1.qk_norm_rope(*split, qg, kg, i32(pos), f)
    whole = bf1.qk_norm_rope(*(x.contiguous() for x in split), qg, kg, i32(pos), f)
    for x, y, z, w, g in zip((q, k), tok, head, whole, (qg, kg)):
        check_forward(x, y, g, pos, freqs, False, 1.0, 1e-6, tokens=True)
        assert torch.equal(y.transpose(0, 1), z[0]) and torch.equal(z, w)
    # gradients into the q and k parts of joined rows, whose other part stays
    dq, dk = normal(6, 1, H, n, d, dtype=torch.float32), normal(7, 1, Hkv, n, d, dtype=torch.float32)
    rows, oq, ok = joined(8)
    keep = rows[:, (H + Hkv) * d:].clone()
    outs = oq.transpose(0, 1)[None], ok.transpose(0, 1)[None]
    got = bf1.qk_norm_rope_bwd(dq, dk, *split, qg, kg, i32(pos), f, dq_out=outs[0], dk_out=outs[1])
    want = bf1.qk_norm_rope_bwd(dq, dk, *(x.contiguous() for x in split), qg, kg, i32(pos), f)
    assert got[0] is outs[0] and torch.equal(rows[:, (H + Hkv) * d:], keep)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norm_rope_strides_past_32_bits():
    flat = torch.zeros(3 * 2 ** 30 + 4096, dtype=torch.bfloat16, device="cuda")
    q = flat.as_strided((4, 2, 128), (2 ** 30, 128, 1))
    k = flat[1024:].as_strided((4, 1, 128), (2 ** 30, 128, 1))
    q.copy_(normal(1, 4, 2, 128))
    k.copy_(normal(2, 4, 1, 128))
    gain, (f, _) = 1 + 0.3 * normal(3, 128, dtype=torch.float32), bf1.rope_freqs(128)
    pos = i32([5, 6, 7, 8])
    want = bf1.qk_norm_rope(q.contiguous(), k.contiguous(), gain, gain, pos, f)
    got = bf1.qk_norm_rope(q, k, gain, gain, pos, f, q_out=flat[2048:].as_strided(q.shape, q.stride()), k_out=k)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_norm_rope_in_place():
    q, k, qg, kg, pos, freqs, f = case(2, 51, 5, 2, 128, 64, torch.float32)
    a = bf1.qk_norm_rope(q, k, qg, kg, i32(pos), f)
    q2, k2 = q.clone(), k.clone()
    b = bf1.qk_norm_rope(q2, k2, qg, kg, i32(pos), f, q_out=q2, k_out=k2)
    assert b[0] is q2 and torch.equal(a[0], q2) and torch.equal(a[1], k2)
    dq, dk = normal(5, *q.shape, dtype=torch.float32), normal(6, *k.shape, dtype=torch.float32)
    a = bf1.qk_norm_rope_bwd(dq, dk, q, k, qg, kg, i32(pos), f)
    for over_x in (False, True):
        dq2, dk2, q2, k2 = dq.clone(), dk.clone(), q.clone(), k.clone()
        outs = (q2, k2) if over_x else (dq2, dk2)
        b = bf1.qk_norm_rope_bwd(dq2, dk2, q2, k2, qg, kg, i32(pos), f, dq_out=outs[0], dk_out=outs[1])
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_norm_rope_rows_of_zeros_and_extremes():
    d = 64
    x = torch.zeros(1, 1, 6, d, dtype=torch.float32, device="cuda")
    x[0, 0, 1] = 1e-30
    x[0, 0, 2] = 1e15
    x[0, 0, 3, 5] = float("nan")
    x[0, 0, 4, 7] = 1e18
    f, pos = torch.ones(2, dtype=torch.float64, device="cuda"), i32(range(6))
    y, none = bf1.qk_norm_rope(x, None, None, None, pos, f)
    assert none is None and not y[0, 0, 0].any() and not y[0, 0, 5].any() and y[0, 0, 3].isnan().all()
    assert torch.allclose(y[0, 0, 2, 4:], torch.ones(d - 4, device="cuda"), atol=2e-6)
    assert abs(float(y[0, 0, 4, 7]) - 8) < 1e-5 and abs(float(y[0, 0, 1, 9]) / 1e-27 - 1) < 1e-5
    dx, _, _, _ = bf1.qk_norm_rope_bwd(torch.ones_like(x), None, x, None, None, None, pos, f)
    assert torch.allclose(dx[0, 0, 0, 4:], torch.full((d - 4,), 1e3, device="cuda"), rtol=1e-5)  # eps^-1/2


def test_norm_rope_empty_and_refusals():
    q, k, qg, kg, pos, freqs, f = case(1, 50, 4, 2, 128, 128, torch.bfloat16)
    e = bf1.qk_norm_rope(q[:, :, :0], k[:, :, :0], qg, kg, i32([]), f)
    assert e[0].shape == (1, 4, 0, 128)
    e = bf1.qk_norm_rope_bwd(q[:, :, :0].float(), k[:, :, :0].float(), q[:, :, :0], k[:, :, :0], qg, kg, i32([]), f)
    assert e[2].shape == (128,) and not e[2].any() and not e[3].any()  # sums over nothing
    ok = dict(q=q, k=k, q_gain=qg, k_gain=kg, positions=i32(pos), freqs=f)
    for bad, why in [(dict(positions=i32(range(49))), "positions"), (dict(positions=i32(pos).long()), "dtype"),
                     (dict(freqs=f.float()), "dtype"), (dict(freqs=f.cpu()), "device"), (dict(k=k[:, :, :49]), "agree"),
                     (dict(k=k.float()), "k must"), (dict(q=q.half()), "bf16"), (dict(q_gain=qg[:64]), "q_gain"),
                     (dict(k_gain=kg.float()), "dtype"), (dict(q_gain=qg.half()), "gains"), (dict(q_gain=qg.cpu()), "device"),
                     (dict(q=q.transpose(2, 3).contiguous().transpose(2, 3)), "side by side"),
                     (dict(q_out=torch.empty(1, 4, 50, 64, device="cuda")), "q_out"),
                     (dict(q=q.float(), k=k.float(), dtype=torch.float16), "dtype")]:
        with pytest.raises(ValueError, match=why):
            bf1.qk_norm_rope(**{**ok, **bad})
    for bad in (dict(eps=0.0), dict(dtype=torch.float32), dict(q_out=torch.empty(1, 4, 1, 128, device="cuda",
                                                                                 dtype=torch.bfloat16).expand(1, 4, 50, 128))):
        with pytest.raises(bf1.BF1Error):
            bf1.qk_norm_rope(**{**ok, **bad})
    dq, dk = q.float(), k.float()
    for bad, why in [(dict(dq=dq[:, :3]), "dq must"), (dict(dk=k), "dk must"), (dict(dq=q.half(), dk=k.half()), "float32"),
                     (dict(k=None), "dk without k"), (dict(dtype=torch.float16), "dtype"),
                     (dict(workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), "workspace")]:
        with pytest.raises(ValueError, match=why):
            bf1.qk_norm_rope_bwd(**{**ok, **dict(dq=dq, dk=dk), **bad})
    with pytest.raises(ValueError, match="float32"):  # bf16 gradients of float32 rows
        bf1.qk_norm_rope_bwd(**{**ok, **dict(q=dq, k=dk, dq=q, dk=k)})


def test_both_ways_of_marshalling_agree():
    q, k, qg, kg, pos, freqs, f = case(2, 70, 4, 2, 64, 32, torch.bfloat16)
    here = torch.cuda.current_stream()
    a, b = (bf1.qk_norm_rope(q, k, qg, kg, i32(pos), f, stream=s) for s in (None, here))
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    dq, dk = q.float(), k.float()
    a, b = (bf1.qk_norm_rope_bwd(dq, dk, q, k, qg, kg, i32(pos), f, stream=s) for s in (None, here))
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_gradient_is_the_same_each_time_and_in_a_graph():
    q, k, qg, kg, pos, freqs, f = case(1, 3000, 4, 2, 128, 128, torch.bfloat16)
    p = i32(pos)
    dq, dk = normal(5, *q.shape, dtype=torch.float32), normal(6, *k.shape, dtype=torch.float32)

    def step():
        y = bf1.qk_norm_rope(q, k, qg, kg, p, f)
        return (*y, *bf1.qk_norm_rope_bwd(dq, dk, q, k, qg, kg, p, f))

    first = step()
    assert all(torch.equal(a, b) for a, b in zip(first, step()))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = step()
    for i in range(4):
        dq.copy_(normal(10 + i, *dq.shape, dtype=torch.float32))
        q.copy_(normal(20 + i, *q.shape))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, step()))
        torch.cuda.synchronize()


def test_trains_through_the_attention():
    """Gradients of norm + rope -> attn_fwd -> attn_bwd -> norm + rope's gradient, into the
    rows of joined projections, and differences of the loss along them, against the same
    formulas in 64 bits.  (Along the gradient the loss is far from linear: its difference
    at h = 2^-4 is 6% from its derivative in 64 bits too, so like is compared with like.)

    The operators round to bf16 on the way (q, k, v, o), each value by up to 2^-9 of itself
    and at random: the difference by sqrt of the sum of (o w)^2, twice 2^-9 of it, over h; the
    derivative, a sum over all rows, by less than 2^-8 of itself."""
    n, Hq, Hkv, d = 300, 4, 2, 64
    qkv = normal(1, n, Hq + 2 * Hkv, d, dtype=torch.float32)
    gains = [1 + 0.2 * normal(s, d, dtype=torch.float32) for s in (2, 3)]
    f, amp = bf1.rope_freqs(32, 1e4)
    pos, w = i32(range(1000, 1000 + n)), normal(4, 1, Hq, n, d)

    def forward(x):
        h = x.transpose(0, 1)[None]
        q, k = bf1.qk_norm_rope(h[:, :Hq], h[:, Hq:Hq + Hkv], *gains, pos, f, amplitude=amp, dtype=torch.bfloat16)
        v = h[:, Hq + Hkv:].contiguous().bfloat16()
        o, lse = bf1.attn_fwd(q, k, v)
        return q, k, v, o, lse

    angle = pos.cpu().double()[:, None] * f.cpu()
    mask = torch.as_tensor(orc.token_mask(n, 64, 2))

    def loss64(x):
        def side(y, g):
            y = y / (y.square().mean(-1, keepdim=True) + 1e-6).sqrt() * g.cpu().double()
            a, b = y[..., :16], y[..., 16:32]
            return torch.cat([a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin(), y[..., 32:]], -1)

        h = x.transpose(0, 1)
        q, k, v = side(h[:Hq], gains[0]), side(h[Hq:Hq + Hkv], gains[1]), h[Hq + Hkv:]
        k, v = k.repeat_interleave(2, 0), v.repeat_interleave(2, 0)
        s = (q @ k.transpose(1, 2)) / 8
        return ((s.masked_fill(~mask, -1e300).softmax(-1) @ v) * w[0].cpu().double()).sum()

    q, k, v, o, lse = forward(qkv)
    dq, dk, dv = bf1.attn_bwd(q, k, v, o, w, lse)
    grad = torch.empty_like(qkv)
    gh, xh = grad.transpose(0, 1)[None], qkv.transpose(0, 1)[None]
    bf1.qk_norm_rope_bwd(dq, dk, xh[:, :Hq], xh[:, Hq:Hq + Hkv], *gains, pos, f, amplitude=amp, dq_out=gh[:, :Hq],
                         dk_out=gh[:, Hq:Hq + Hkv])
    gh[:, Hq + Hkv:] = dv
    step = grad / grad.square().mean().sqrt()
    h = 2.0 ** -4
    plus, minus = (float((forward(qkv + s * h * step)[3].double() * w.double()).sum()) for s in (1, -1))
    got = float((grad.double() * step.double()).sum())
    x64, step64 = qkv.cpu().double().requires_grad_(), step.cpu().double()
    grad64, = torch.autograd.grad(loss64(x64), x64)
    along = float((grad64 * step64).sum())
    with torch.no_grad():
        diff64 = float(loss64(x64 + h * step64) - loss64(x64 - h * step64)) / (2 * h)
    noise = float((o.double() * w.double()).square().sum().sqrt()) * 2.0 ** -8 / h
    assert abs(got - along) < 2.0 ** -8 * abs(along)
    assert abs((plus - minus) / (2 * h) - diff64) < 8 * noise

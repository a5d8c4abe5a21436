"""The operators around a served sequence's cache without a GPU: pins of their
oracle, rotary frequencies, workspace sizes, and refusals by the library (before any
device call) and by the binding (before any pointer is taken)."""

import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import cache_oracle as co

FAKE = 1 << 20
INVALID, UNSUPPORTED, SMALL = bf1.BF1_ERR_INVALID_ARG, bf1.BF1_ERR_UNSUPPORTED, bf1.BF1_ERR_BUFFER_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    return bf1.load()


# ---- oracle pins ----------------------------------------------------------------

def test_page_step_by_hand():
    # B = 4; sequence 0 holds 3 tokens and gets 3 (one more page), 1 gets nothing, 2 starts
    table = np.array([[7, -1, -1], [-1, -1, -1], [-1, -1, -1]])
    t, lens, ts, bs, pos, slots, head = co.page_step([3, 0, 0], [3, 0, 5], table, [9, 5, 6, 8], 1, 10, 4)
    assert t.tolist() == [[7, 5, -1], [-1, -1, -1], [6, 8, -1]]
    assert lens.tolist() == [6, 0, 5] and ts.tolist() == [0, 3, 3, 8] and bs.tolist() == [0, 2, 2, 4] and head == 4
    assert pos.tolist() == [3, 4, 5, 0, 1, 2, 3, 4, -1, -1]
    assert slots.tolist() == [31, 20, 21, 24, 25, 26, 27, 32, -1, -1]


def test_page_step_without_pages_by_hand():
    # one free page: sequence 0 needs two and keeps what fits the first; 1 needs none, 2 gets none
    table = np.array([[-1, -1, -1], [3, -1, -1], [-1, -1, -1]])
    t, lens, ts, bs, pos, slots, head = co.page_step([0, 1, 0], [6, 2, 1], table, [5], 0, 9, 4)
    assert t.tolist() == [[5, -1, -1], [3, -1, -1], [-1, -1, -1]]
    assert lens.tolist() == [4, 3, 0] and bs.tolist() == [0, 1, 2, 2] and head == 1
    assert slots.tolist() == [20, 21, 22, 23, -1, -1, 13, 14, -1]


def test_e4m3_table_and_rounding():
    v = co.E4M3
    assert v[0x7e] == 448 and v[0x08] == 2.0 ** -6 and v[0x01] == 2.0 ** -9 and np.isnan(v[0x7f]) and v[0xc0] == -2
    every = np.array([c for c in range(256) if not np.isnan(v[c])], dtype=np.uint8)
    assert np.array_equal(v[co.to_e4m3(v[every])], v[every])
    assert np.array_equal(v[every], torch.from_numpy(every.copy()).view(torch.float8_e4m3fn).float().numpy())
    mids = (v[:126] + v[1:127]) / 2  # ties go to the even code
    assert all(c % 2 == 0 for c in co.to_e4m3(mids))
    x = np.random.default_rng(0).standard_normal(4000) * 60
    assert np.array_equal(co.to_e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_quantise_by_hand():
    codes, scale = co.quantise([[448.0, -1.0], [0.5, 7.0]], "e4m3")
    assert scale == 1 and co.E4M3[codes].tolist() == [[448, -1], [0.5, 7]]
    assert co.quantise([[449.0]], "e4m3")[1] == 2 and co.quantise([[0.875]], "e4m3")[1] == 2.0 ** -9
    codes, scale = co.quantise([[254.0, 1.0, 3.0, -5.0]], "int8")  # 1/2, 3/2 and -5/2 go to even
    assert scale == 2 and codes.tolist() == [[127, 0, 2, -2]]
    for fmt in ("e4m3", "int8"):
        assert np.isnan(co.quantise([[1.0, np.inf]], fmt)[1]) and not co.quantise([[np.nan, 1.0]], fmt)[0].any()
        assert co.quantise([[0.0, 2.0 ** -101]], fmt)[1] == 1


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_gradient_by_differences(interleaved):
    # the map is linear, so central differences give its matrix to the last bits
    rng = np.random.default_rng(3)
    n, d, r = 3, 10, 6
    freqs = 10.0 ** -np.arange(r // 2)
    pos = np.array([0, 5, -7])
    x, dy = rng.standard_normal((n, d)), rng.standard_normal((n, d))
    dx = co.rope(dy, pos, freqs, interleaved, 1.25, sign=-1)
    for i in range(n):
        for j in range(d):
            e = np.zeros((n, d))
            e[i, j] = 0.5
            up = co.rope(x + e, pos, freqs, interleaved, 1.25) - co.rope(x - e, pos, freqs, interleaved, 1.25)
            assert abs((up * dy).sum() - dx[i, j]) < 1e-13 * 40
    assert np.array_equal(co.rope(x, pos, freqs, interleaved, 1.0)[:, r:], x[:, r:])


def test_rope_keeps_products_of_distances():
    # q at p and k at p + 5 have the same product for every p
    rng = np.random.default_rng(4)
    q, k = rng.standard_normal((1, 8)), rng.standard_normal((1, 8))
    f = [1.0, 0.3, 0.01, 1e-4]
    got = [float((co.rope(q, [p], f, False, 1.0) * co.rope(k, [p + 5], f, False, 1.0)).sum()) for p in (0, 17, 10 ** 6)]
    assert max(got) - min(got) < 1e-9


# ---- frequencies -------------------------------------------------------------------

def test_rope_freqs():
    f, a = bf1.rope_freqs(8, theta=10000.0, device="cpu")
    assert f.dtype == torch.float64 and a == 1.0
    assert np.allclose(f.numpy(), [1, 10000 ** -0.25, 10000 ** -0.5, 10000 ** -0.75], rtol=1e-14)
    g, a = bf1.rope_freqs(8, 10000.0, "linear", 4.0, device="cpu")
    assert a == 1.0 and np.allclose(g * 4, f, rtol=1e-14)
    g, a = bf1.rope_freqs(8, 10000.0, "base", 4.0, device="cpu")
    assert a == 1.0 and g[0] == 1 and np.allclose(g[-1] * 4, f[-1], rtol=1e-13)
    g, a = bf1.rope_freqs(128, 1e6, "bands", 4.0, 32768, device="cpu")
    f, _ = bf1.rope_freqs(128, 1e6, device="cpu")
    turns = 32768 * f / (2 * math.pi)
    assert torch.equal(g[turns > 32], f[turns > 32]) and torch.equal(g[turns < 1], f[turns < 1] / 4)
    mid = (turns > 1) & (turns < 32)
    assert mid.any() and (g[mid] < f[mid]).all() and (g[mid] > f[mid] / 4).all()
    assert abs(a - (0.1 * math.log(4) + 1)) < 1e-15
    assert bf1.rope_freqs(2, scaling="base", factor=8.0, device="cpu")[0].tolist() == [1.0]


@pytest.mark.parametrize("kw", [dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, scaling="other"),
                                dict(rot_dim=8, factor=0.5), dict(rot_dim=8, theta=0.0),
                                dict(rot_dim=8, fast=1.0, slow=2.0), dict(rot_dim=8, original_len=0)])
def test_rope_freqs_refuses(kw):
    with pytest.raises(ValueError):
        bf1.rope_freqs(device="cpu", **kw)


# ---- refusals of the library ----------------------------------------------------------

def _with(args, at):
    out = list(args)
    for i, x in at.items():
        out[i] = x
    return out


def test_page_step_refusals(lib):
    ok = [4, FAKE, FAKE + 64, FAKE, 8, FAKE, 9, FAKE, 64, 100, FAKE + 256, FAKE, FAKE, FAKE, FAKE, FAKE + 512, None]
    for at, want in [({0: -1}, INVALID), ({4: 0}, INVALID), ({6: -1}, INVALID), ({9: -1}, INVALID), ({8: 32}, UNSUPPORTED),
                     ({9: 1 << 31}, UNSUPPORTED), ({1: None}, INVALID), ({2: FAKE + 2}, INVALID), ({3: None}, INVALID),
                     ({5: None}, INVALID), ({7: None}, INVALID), ({10: FAKE}, INVALID), ({10: FAKE + 64}, INVALID),
                     ({11: None}, INVALID), ({12: None}, INVALID), ({13: None}, INVALID), ({14: FAKE + 4}, INVALID),
                     ({15: FAKE}, INVALID)]:
        assert lib.bf1_page_step(*_with(ok, at)) == want, at


def test_rope_refusals(lib):
    st = (ctypes.c_int64 * 12)(*[4096, 128, 256] * 4)
    ok = [FAKE, FAKE + 8192, FAKE, 0, FAKE, FAKE + 4096, FAKE + 12288, 2, 10, 4, 2, 128, 128, 0, 0, 0, 1.0, 0, st, None]
    for at, want in [({7: -1}, INVALID), ({8: -1}, INVALID), ({9: -1}, INVALID), ({18: None}, INVALID),
                     ({13: 2}, INVALID), ({14: -1}, INVALID), ({15: 2}, INVALID), ({17: 3}, INVALID),
                     ({11: 127}, UNSUPPORTED), ({11: 2048, 12: 64}, UNSUPPORTED), ({12: 0}, UNSUPPORTED),
                     ({12: 130}, UNSUPPORTED), ({12: 63}, UNSUPPORTED), ({14: 1}, UNSUPPORTED), ({3: 5}, INVALID),
                     ({2: None}, INVALID), ({4: None}, INVALID), ({4: FAKE + 4}, INVALID), ({0: FAKE + 1}, INVALID),
                     ({5: None}, INVALID), ({8: 1 << 31}, UNSUPPORTED), ({9: 65535}, UNSUPPORTED),
                     ({18: (ctypes.c_int64 * 12)(-1)}, INVALID),
                     # in place with other strides, or another type
                     ({5: FAKE, 18: (ctypes.c_int64 * 12)(*[4096, 128, 256, 4096, 256, 128] * 2)}, INVALID),
                     ({5: FAKE, 13: 1, 14: 0}, INVALID),
                     # one side's output over the other side
                     ({1: FAKE + 8192, 6: FAKE + 4096}, INVALID), ({1: FAKE + 4096, 6: FAKE + 8192}, INVALID),
                     ({1: FAKE + 8192, 6: FAKE}, INVALID),
                     ({18: (ctypes.c_int64 * 12)(*[1 << 60] * 12)}, INVALID)]:
        assert lib.bf1_rope(*_with(ok, at)) == want, at
    for at in ({7: 0}, {8: 0}, {9: 0, 10: 0}):  # nothing to do
        assert lib.bf1_rope(*_with(ok, at)) == bf1.BF1_OK


def test_append_refusals(lib):
    ok = [FAKE, FAKE, 1024, 128, 1024, 128, FAKE, FAKE, FAKE, 5, 7, 8, 128, 64, None]
    for at, want in [({9: -1}, INVALID), ({10: 0}, INVALID), ({11: 0}, INVALID), ({12: 96}, UNSUPPORTED),
                     ({13: 16}, UNSUPPORTED), ({0: None}, INVALID), ({1: FAKE + 8}, INVALID), ({6: FAKE + 4}, INVALID),
                     ({7: None}, INVALID), ({2: 1022}, INVALID), ({5: -8}, INVALID), ({9: 1 << 31}, UNSUPPORTED)]:
        assert lib.bf1_kv_append(*_with(ok, at)) == want, at
    assert lib.bf1_kv_append(*_with(ok, {9: 0, 0: None})) == bf1.BF1_OK


def test_append_q8_refusals(lib):
    ok = [FAKE, FAKE, 1024, 128, 1024, 128, 5, 3] + [FAKE] * 5 + [9, 7] + [FAKE] * 6 + [8, 128, 64, 1, None]
    for at, want in [({6: -1}, INVALID), ({7: -1}, INVALID), ({13: 0}, INVALID), ({14: 0}, INVALID), ({21: 0}, INVALID),
                     ({22: 32}, UNSUPPORTED), ({23: 65}, UNSUPPORTED), ({24: 2}, INVALID), ({24: -1}, INVALID),
                     ({0: None}, INVALID), ({3: 4}, INVALID), ({8: None}, INVALID), ({12: FAKE + 1}, INVALID),
                     ({15: FAKE + 8}, INVALID), ({17: None}, INVALID), ({20: None}, INVALID), ({21: 65536}, UNSUPPORTED)]:
        assert lib.bf1_kv_append_q8(*_with(ok, at)) == want, at
    assert lib.bf1_kv_append_q8(*_with(ok, {6: 0})) == bf1.BF1_OK
    assert lib.bf1_kv_append_q8(*_with(ok, {7: 0})) == bf1.BF1_OK


def test_decode_q8_refusals(lib):
    ok = [FAKE] * 8 + [7, FAKE, 19, FAKE, FAKE, 3, 16, 8, 128, 64, 0, FAKE, 1 << 40, None]
    for at, want in [({8: 0}, INVALID), ({10: 2}, INVALID), ({13: -1}, INVALID), ({14: 0}, INVALID), ({14: 17}, INVALID),
                     ({14: 24}, UNSUPPORTED), ({14: 128}, UNSUPPORTED), ({16: 96}, UNSUPPORTED), ({17: 32}, UNSUPPORTED),
                     ({18: 2}, INVALID), ({13: 1 << 20}, INVALID), ({13: 1, 14: 65536, 15: 65536}, UNSUPPORTED), ({0: FAKE + 8}, INVALID), ({2: None}, INVALID),
                     ({3: FAKE + 2}, INVALID), ({5: None}, INVALID), ({7: None}, INVALID), ({9: None}, INVALID),
                     ({11: None}, INVALID), ({12: FAKE + 1}, INVALID), ({20: 0}, SMALL), ({19: FAKE + 4}, INVALID)]:
        assert lib.bf1_decode_attn_q8(*_with(ok, at)) == want, at
    assert lib.bf1_decode_attn_q8(*_with(ok, {13: 0})) == bf1.BF1_OK
    size = ctypes.c_int64()
    assert lib.bf1_decode_q8_workspace_size(3, 16, 8, 128, 64, 19, None) == INVALID
    assert lib.bf1_decode_q8_workspace_size(3, 16, 8, 96, 64, 19, ctypes.byref(size)) == UNSUPPORTED


def test_decode_q8_workspace_holds_every_split():
    for batch, Hq, Hkv, d, B, stride in [(1, 16, 8, 128, 64, 19), (300, 8, 8, 64, 64, 500), (2, 8, 1, 128, 128, 5000)]:
        got = bf1.decode_q8_workspace_size(batch, Hq, Hkv, d, B, stride)
        record = batch * Hkv * (Hq // Hkv) * (d + 2) * 4
        assert got % record == 0 and got // record != 1 and got // record <= 256


# ---- refusals of the binding ----------------------------------------------------------

def test_host_tensors_are_refused():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pages = torch.zeros((3, 2, 64, 128), dtype=torch.bfloat16)
    cache = bf1.cache_q8(3, 2, 2, device="cpu")
    calls = [lambda: bf1.page_step(i(2), i(2), i(2, 3), i(4), i(1), 5),
             lambda: bf1.rope(x, x, i(4), torch.ones(64, dtype=torch.float64)),
             lambda: bf1.kv_append(x, x, torch.zeros(4, dtype=torch.int64), pages, pages),
             lambda: bf1.kv_append_q8(x, x, i(2), i(2), i(3), i(3), i(2, 3), cache),
             lambda: bf1.attn_decode_q8(x[:2], cache, i(2), i(2, 19))]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="needs q or k"):
        bf1.rope(None, None, i(4), torch.ones(64, dtype=torch.float64))
    with pytest.raises(ValueError, match="needs dq or dk"):
        bf1.rope_bwd(None, None, i(4), torch.ones(64, dtype=torch.float64))
    with pytest.raises(ValueError, match="dtype"):
        bf1.cache_q8(3, 2, 2, dtype=torch.uint8, device="cpu")

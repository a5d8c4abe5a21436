"""The operators around speculative and parallel decoding without a GPU: pins of their
oracle, workspace sizes, and refusals by the library (before any device call) and by the
binding (before any pointer is taken)."""

import ctypes
import re

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import bf1_oracle as orc
from oracle import serve_oracle as so

FAKE = 1 << 20
INVALID, UNSUPPORTED, SMALL = bf1.BF1_ERR_INVALID_ARG, bf1.BF1_ERR_UNSUPPORTED, bf1.BF1_ERR_BUFFER_TOO_SMALL


@pytest.fixture(scope="module")
def lib():
    return bf1.load()


# ---- oracle pins ----------------------------------------------------------------------

@pytest.mark.parametrize("interleaved", [False, True])
def test_norm_rope_gradient_by_differences(interleaved):
    # central differences of h: their own error is h^2 / 6 times the third derivative (some
    # 30 here, rows are of size 1) and 2^-52 / h of the values (some 10): 1e-9 at h = 1e-5
    rng = np.random.default_rng(3)
    n, d, r, h = 3, 10, 6, 1e-5
    freqs, pos = 10.0 ** -np.arange(r // 2), np.array([0, 5, -7])
    x, dy, gain = rng.standard_normal((n, d)), rng.standard_normal((n, d)), 1 + 0.3 * rng.standard_normal(d)
    args = (pos, freqs, interleaved, 1.25, 1e-3)
    dx, dg = so.norm_rope_bwd(dy, x, gain, *args)
    for i in range(n):
        for j in range(d):
            e = np.zeros((n, d))
            e[i, j] = h
            up = so.norm_rope(x + e, gain, *args) - so.norm_rope(x - e, gain, *args)
            assert abs((up * dy).sum() / (2 * h) - dx[i, j]) < 2e-8
    for j in range(d):
        e = np.zeros(d)
        e[j] = 1.0
        assert abs((so.norm_rope(x, e, *args) * dy).sum() - dg[:, j].sum()) < 1e-12  # linear in the gain


def test_norm_rope_by_hand():
    y = so.norm_rope(np.array([[3.0, 4.0, 0.0, 0.0]]), np.array([1, 2, 1, 1.0]), [0], [1.0], False, 1.0, 0.0)
    assert np.allclose(y, [[1.2, 3.2, 0, 0]], atol=1e-15)  # mean square 6.25, position 0


def test_tree_step_by_hand():
    #  0 - 1 - 3      a second tree: one node; a third with a parent that is not before it
    #    \ 2   4 (new root)
    masks, pos = so.tree_step([-1, 0, 0, 1, 7, -1, 1, 0], [0, 5, 6, 8], [10, 0, 3], [15, 1, 5])
    assert masks == [1, 3, 5, 11, 16, 1, 1, 3] and pos == [10, 11, 11, 12, 10, 0, 3, 4]
    masks, pos = so.tree_step([-1, 0, 1], [0, 3], [5], [7])  # the last node has no place
    assert masks == [1, 3, 0] and pos == [5, 6, -1]


def test_tree_chain_reads_what_decode_reads():
    # a chain's row reads exactly row p of the prefill mask
    B, L = 4, 2
    for held in (0, 3, 4, 30, 31, 63):
        n = 6
        masks, pos = so.tree_step([-1] + list(range(n - 1)), [0, n], [held], [held + n])
        mask = orc.token_mask(held + n, B, L) if hasattr(orc, "token_mask") else None
        for i in range(n):
            keys = sorted(so.tree_keys(0, i, masks, pos, [held], [0, n], B, L, False))
            p = held + i
            want = sorted(t for j in so.route(p // B, L) + [p // B] for t in range(j * B, min(j * B + B, p + 1)))
            assert keys == want
            if mask is not None:
                assert keys == list(np.nonzero(mask[p])[0])


def test_route_is_the_route():
    for L in (0, 1, 2, 3, 5, 32):
        for j in (0, 1, 2, 3, 4, 5, 8, 9, 33, 64, 65, 100):
            rp, ci = bf1.plan_variant("bf1", (j + 1) * 64, 64, L)
            assert list(ci[rp[j]:rp[j + 1]][:-1]) == so.route(j, L)


def test_compact_by_hand():
    moves, lens = so.compact([[0, 2, 5, -1], [1, 1, 2, 3], [-1, 0, 1, 2], [3, 9, 10, 11]], [10, 0, 5, 7], [16, 4, 9, 17])
    assert moves == [(0, 10, 10), (0, 12, 11), (0, 15, 12), (1, 1, 0), (3, 10, 7), (3, 16, 8)]
    assert lens == [13, 1, 5, 9]


def test_page_fork_by_hand():
    B = 4
    # place 0 holds 10 tokens, 1 holds 3, 2 nothing; 2 starts from 0, 1 goes on from 0 too, 0 stays
    table = [[7, 5, 3, -1], [2, -1, -1, -1], [-1, -1, -1, -1]]
    new, lens, head, shares, free, copies = so.page_fork([10, 3, 0], [0, 0, 0], [10, 9, 8], table, [0] * 8,
                                                         [9, 9, 6, 4, 1, 0], 2, B)
    assert new == [[7, 5, 3, -1], [7, 5, 6, -1], [7, 5, -1, -1]] and lens == [10, 9, 8]
    assert copies == [(-1, -1, 0), (3, 6, 1), (-1, -1, 0)]
    assert shares == [0, 0, 0, 0, 0, 2, 0, 2] and head == 2 and free == [9, 9, 2, 4, 1, 0]  # page 2 is free again
    # no free page: the second sequence goes on without its partial block
    new, lens, head, shares, free, copies = so.page_fork([10, 3, 0], [0, 0, -1], [10, 9, 8], table, [0] * 8, [6], 1, B)
    assert lens == [10, 8, 0] and new[1] == [7, 5, -1, -1] and head == 0 and free == [2]
    # tokens taken back into a block that another sequence holds: copied, not written over
    table = [[1, 2], [1, -1]]
    new, lens, head, shares, free, copies = so.page_fork([7, 4], [0, 1], [3, 4], table, [0, 1, 0], [5, 6, 0], 2, B)
    assert copies == [(1, 0, 3), (-1, -1, 0)] and new == [[0, -1], [1, -1]] and shares == [0, 0, 0]
    assert head == 2 and free == [5, 6, 2]  # page 2 is free, page 0 is taken


# ---- refusals of the library -----------------------------------------------------------

def _with(args, at):
    out = list(args)
    for i, x in at.items():
        out[i] = x
    return out


def test_qk_norm_rope_refusals(lib):
    st = (ctypes.c_int64 * 12)(*[5120, 1280, 128] * 4)
    ok = [FAKE, FAKE + (1 << 16), FAKE, FAKE, 0, FAKE, 0, FAKE, FAKE + (1 << 17), FAKE + (1 << 18), 2, 10, 4, 2, 128, 128, 0, 0,
          0, 1e-6, 1.0, st, None]
    for at, want in [({10: -1}, INVALID), ({11: -1}, INVALID), ({12: -1}, INVALID), ({21: None}, INVALID), ({4: 2}, INVALID),
                     ({16: 2}, INVALID), ({17: -1}, INVALID), ({18: 2}, INVALID), ({19: 0.0}, INVALID),
                     ({19: float("nan")}, INVALID), ({14: 127}, UNSUPPORTED), ({14: 514, 15: 64}, UNSUPPORTED),
                     ({15: 0}, UNSUPPORTED), ({15: 130}, UNSUPPORTED), ({15: 63}, UNSUPPORTED), ({17: 1}, UNSUPPORTED),
                     ({6: 5}, INVALID), ({5: None}, INVALID), ({7: FAKE + 4}, INVALID), ({0: FAKE + 1}, INVALID),
                     ({2: FAKE + 1}, INVALID), ({3: FAKE + 2, 4: 1}, INVALID), ({8: None}, INVALID),
                     ({11: 1 << 31}, UNSUPPORTED), ({12: 65535}, UNSUPPORTED), ({11: 1 << 28}, UNSUPPORTED),
                     ({21: (ctypes.c_int64 * 12)(-1)}, INVALID), ({21: (ctypes.c_int64 * 12)(*[1 << 60] * 12)}, INVALID),
                     # an output that writes elements twice: overlapping rows, heads over tokens, one row for all
                     ({21: (ctypes.c_int64 * 12)(*[5120, 1280, 128, 5120, 1280, 64] * 2)}, INVALID),
                     ({21: (ctypes.c_int64 * 12)(*[5120, 1280, 128, 5120, 128, 128] * 2)}, INVALID),
                     ({21: (ctypes.c_int64 * 12)(*[5120, 1280, 128, 0, 1280, 128] * 2)}, INVALID),
                     # in place with other strides, or another type; one side's output over the other side
                     ({8: FAKE, 21: (ctypes.c_int64 * 12)(*[5120, 1280, 128, 5120, 128, 512] * 2)}, INVALID),
                     ({8: FAKE, 16: 1, 17: 0}, INVALID), ({8: FAKE + (1 << 18)}, INVALID), ({8: FAKE + (1 << 16)}, INVALID),
                     ({9: FAKE}, INVALID)]:
        assert lib.bf1_qk_norm_rope(*_with(ok, at)) == want, at
    for at in ({10: 0}, {11: 0}, {12: 0, 13: 0}):  # nothing to do
        assert lib.bf1_qk_norm_rope(*_with(ok, at)) == bf1.BF1_OK


def test_qk_norm_rope_bwd_refusals(lib):
    st = (ctypes.c_int64 * 18)(*[5120, 1280, 128] * 6)
    far = [FAKE + (i << 18) for i in range(1, 8)]
    ok = [far[0], far[1], 1, far[2], far[3], FAKE, FAKE, 0, FAKE, 0, FAKE, far[4], far[5], FAKE + 64, FAKE + 1024, 2, 10, 4, 2,
          128, 128, 0, 0, 0, 1e-6, 1.0, st, FAKE, 1 << 30, None]
    for at, want in [({2: 2}, INVALID), ({7: -1}, INVALID), ({15: -1}, INVALID), ({21: 3}, INVALID), ({22: 2}, INVALID),
                     ({23: 2}, INVALID), ({24: -1.0}, INVALID), ({26: None}, INVALID), ({19: 600}, UNSUPPORTED),
                     ({20: 3}, UNSUPPORTED), ({21: 1, 2: 0}, UNSUPPORTED), ({9: 3}, INVALID), ({0: None}, INVALID),
                     ({3: FAKE + 1}, INVALID), ({11: None}, INVALID), ({13: FAKE + 2}, INVALID), ({14: FAKE + 64}, INVALID),
                     ({28: 100}, SMALL), ({27: FAKE + 8}, INVALID), ({27: None}, INVALID),
                     ({11: far[5]}, INVALID), ({11: far[1]}, INVALID), ({12: far[2]}, INVALID),
                     ({11: far[0]}, INVALID),  # over dq, of another type
                     ({11: far[0], 22: 1, 26: (ctypes.c_int64 * 18)(*[5120, 1280, 128] * 2 + [5120, 128, 512] * 4)}, INVALID),
                     ({26: (ctypes.c_int64 * 18)(*[5120, 1280, 128] * 2 + [5120, 1280, 64] + [5120, 1280, 128] * 3)}, INVALID)]:
        assert lib.bf1_qk_norm_rope_bwd(*_with(ok, at)) == want, at
    assert lib.bf1_qk_norm_rope_bwd(*_with(ok, {15: 0, 13: None, 14: None})) == bf1.BF1_OK
    size = ctypes.c_int64()
    assert lib.bf1_qk_norm_rope_bwd_workspace_size(2, 10, 4, 2, 128, 128, 0, None) == INVALID
    assert lib.bf1_qk_norm_rope_bwd_workspace_size(2, 10, 4, 2, 130, 132, 0, ctypes.byref(size)) == UNSUPPORTED
    assert bf1.qk_norm_rope_bwd_workspace_size(1, 1, 1, 1, 64, 64, torch.bfloat16) == 0  # one workgroup
    assert 0 < bf1.qk_norm_rope_bwd_workspace_size(4, 100000, 16, 8, 128, 128, torch.bfloat16) <= 1 << 22
    for other in (torch.float16, torch.float64, None):
        with pytest.raises(ValueError, match="dtype"):
            bf1.qk_norm_rope_bwd_workspace_size(1, 1, 1, 1, 64, 64, other)


def test_tree_step_refusals(lib):
    ok = [FAKE, FAKE, FAKE, FAKE, 3, 20, FAKE + 4096, FAKE + 8192, None]
    for at, want in [({4: -1}, INVALID), ({5: -1}, INVALID), ({5: 1 << 31}, UNSUPPORTED), ({4: (1 << 24) + 1}, UNSUPPORTED),
                     ({5: (1 << 30) + 1}, UNSUPPORTED), ({1: FAKE + 8192}, INVALID), ({3: FAKE + 8192}, INVALID),
                     ({0: None}, INVALID), ({1: FAKE + 2}, INVALID), ({2: None}, INVALID), ({3: None}, INVALID),
                     ({6: FAKE + 4}, INVALID), ({7: None}, INVALID), ({7: FAKE}, INVALID)]:
        assert lib.bf1_tree_step(*_with(ok, at)) == want, at
    assert lib.bf1_tree_step(*_with(ok, {5: 0, 0: None})) == bf1.BF1_OK


def test_tree_step_writes_buffers_of_its_own(lib):
    """Masks over what other trees' waves still read, or over the positions."""
    ok = [FAKE, FAKE + 64, FAKE + 128, FAKE + 192, 3, 20, FAKE + 4096, FAKE + 8192, None]
    for over in (0, 1, 2, 3, 7):
        assert lib.bf1_tree_step(*_with(ok, {6: ok[over]})) == INVALID, over
        if over < 7:
            assert lib.bf1_tree_step(*_with(ok, {7: ok[over]})) == INVALID, over


def test_attn_tree_refusals(lib):
    ok = [FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 900, 7, FAKE + 4096, FAKE + 8192, 3, 20, 16, 16, 8, 128, 64, 2, 0, FAKE,
          1 << 40, None]
    for at, want in [({12: -1}, INVALID), ({13: -1}, INVALID), ({14: 0}, INVALID), ({14: 65}, UNSUPPORTED), ({15: 0}, INVALID),
                     ({15: 17}, INVALID), ({15: 24}, UNSUPPORTED), ({15: 128}, UNSUPPORTED), ({17: 96}, UNSUPPORTED),
                     ({18: 32}, UNSUPPORTED), ({19: -1}, INVALID), ({19: 33}, UNSUPPORTED), ({20: 2}, INVALID),
                     ({8: 0}, INVALID), ({9: 0}, INVALID), ({13: 1 << 31}, UNSUPPORTED), ({0: FAKE + 8}, INVALID),
                     ({13: (1 << 30) + 1}, UNSUPPORTED),
                     ({1: None}, INVALID), ({3: FAKE + 4}, INVALID), ({4: None}, INVALID), ({5: FAKE + 2}, INVALID),
                     ({6: None}, INVALID), ({7: None}, INVALID), ({10: FAKE}, INVALID), ({11: FAKE + 1}, INVALID),
                     ({22: 0}, SMALL), ({21: FAKE + 4}, INVALID), ({12: (1 << 15) + 1}, UNSUPPORTED),
                     ({12: 1, 15: 65536, 16: 65536}, UNSUPPORTED)]:
        assert lib.bf1_attn_tree(*_with(ok, at)) == want, at
    for at in ({12: 0}, {13: 0}):
        assert lib.bf1_attn_tree(*_with(ok, at)) == bf1.BF1_OK
    assert lib.bf1_attn_tree(*_with(ok, {20: 1, 19: 1000, 22: 0})) == SMALL  # L is not used
    size = ctypes.c_int64()
    assert lib.bf1_attn_tree_workspace_size(3, 16, 16, 8, 128, 64, 9, 2, 0, None) == INVALID
    assert lib.bf1_attn_tree_workspace_size(3, 16, 16, 8, 128, 96, 9, 2, 0, ctypes.byref(size)) == UNSUPPORTED
    assert bf1.attn_tree_workspace_size(0, 16, 16, 8, 128, 64, 9) == 0
    assert bf1.attn_tree_workspace_size(1 << 15, 64, 8, 8, 128, 64, 9) == 0  # rows enough without splits


def test_page_refusals(lib):
    far = [FAKE + (i << 12) for i in range(10)]
    ok = [3, far[0], far[1], far[2], far[3], 9, far[4], 40, far[5], 40, far[6], 64, far[7], far[8], far[6], FAKE + 64, FAKE + 128,
          FAKE + 256, None]
    for at, want in [({0: -1}, INVALID), ({5: 0}, INVALID), ({7: 0}, INVALID), ({9: -1}, INVALID), ({11: 32}, UNSUPPORTED),
                     ({0: (1 << 22) + 1}, UNSUPPORTED), ({7: (1 << 30) + 1}, UNSUPPORTED), ({1: None}, INVALID),
                     ({2: FAKE + 2}, INVALID), ({3: None}, INVALID), ({4: None}, INVALID), ({6: None}, INVALID),
                     ({8: None}, INVALID), ({10: None}, INVALID), ({12: None}, INVALID), ({13: None}, INVALID),
                     ({14: None}, INVALID), ({15: None}, INVALID), ({16: None}, INVALID), ({17: FAKE + 1}, INVALID),
                     ({12: far[3]}, INVALID), ({13: far[0]}, INVALID), ({13: far[1]}, INVALID), ({13: far[2]}, INVALID),
                     ({15: far[0]}, INVALID), ({15: FAKE + 128}, INVALID), ({17: far[8]}, INVALID), ({8: far[4]}, INVALID),
                     ({14: FAKE + 64}, INVALID), ({16: far[6]}, INVALID)]:
        assert lib.bf1_page_fork(*_with(ok, at)) == want, at
    ok = [FAKE, FAKE * 2, FAKE, FAKE, FAKE, 5, 7, 8, 128, 64, None]
    for at, want in [({5: -1}, INVALID), ({6: 0}, INVALID), ({7: 0}, INVALID), ({8: 96}, UNSUPPORTED), ({9: 32}, UNSUPPORTED),
                     ({0: FAKE + 8}, INVALID), ({1: FAKE}, INVALID), ({2: None}, INVALID), ({4: FAKE + 2}, INVALID),
                     ({5: 1 << 24, 7: 1 << 10}, UNSUPPORTED)]:
        assert lib.bf1_kv_copy(*_with(ok, at)) == want, at
    assert lib.bf1_kv_copy(*_with(ok, {5: 0, 0: None})) == bf1.BF1_OK
    ok = [FAKE, FAKE * 2, FAKE, 16, FAKE, FAKE + 64, FAKE, 3, 9, 7, 8, 128, 64, FAKE + 128, None]
    for at, want in [({3: -1}, INVALID), ({3: 65}, UNSUPPORTED), ({7: -1}, INVALID), ({8: 0}, INVALID), ({9: 0}, INVALID),
                     ({10: 0}, INVALID), ({11: 32}, UNSUPPORTED), ({12: 16}, UNSUPPORTED), ({0: None}, INVALID),
                     ({1: FAKE}, INVALID), ({2: None}, INVALID), ({4: None}, INVALID), ({5: FAKE + 1}, INVALID),
                     ({6: None}, INVALID), ({13: None}, INVALID), ({13: FAKE}, INVALID), ({13: FAKE + 64}, INVALID),
                     ({2: FAKE + 128}, INVALID),
                     ({7: 1 << 24, 10: 1 << 10}, UNSUPPORTED)]:
        assert lib.bf1_kv_compact(*_with(ok, at)) == want, at
    assert lib.bf1_kv_compact(*_with(ok, {7: 0, 0: None})) == bf1.BF1_OK


def test_kernels_of_trees_are_those_that_calls_reach():
    """64 nodes of groups of one head are 64 columns: none run 128; and lists are dealt by length
    (a merge that looks up slots) at 64 columns or more."""
    with open(bf1.lib_path(), "rb") as f:
        names = f.read()
    kernels = {tuple(map(int, m)) for m in re.findall(
        rb"attn_tree_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", names)}
    assert kernels == {(d, g, B, nt, cw, waves) for d in (64, 128) for g in (1, 2, 4, 8) for B in (64, 128)
                       for nt, cw, waves in ((1, 1, 4), (2, 1, 4), (2, 2, 4), (2, 2, 8), (2, 4, 4)) if g > 1 or cw < 4}
    merges = {tuple(map(int, m)) for m in re.findall(rb"merge_tree_kernelILi(\d+)ELi(\d+)ELi(\d+)ELb(\d)E", names)}
    assert merges == {(d, g, cols, slots) for d in (64, 128) for g in (1, 2, 4, 8) for cols in (16, 32, 64, 128)
                      for slots in (0, 1) if (g > 1 or cols < 128) and (cols >= 64 or not slots)}


# ---- refusals of the binding -----------------------------------------------------------

def test_host_tensors_are_refused():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    f, g = torch.ones(64, dtype=torch.float64), torch.ones(128)
    pages = torch.zeros((3, 2, 64, 128), dtype=torch.bfloat16)
    calls = [lambda: bf1.qk_norm_rope(x, x, g, g, i(4), f),
             lambda: bf1.qk_norm_rope_bwd(x, x, x, x, g, g, i(4), f),
             lambda: bf1.tree_step(i(4), i(3), i(2), i(2)),
             lambda: bf1.attn_tree(x, pages, pages, torch.zeros(4, dtype=torch.int64), i(4), i(2), i(3), i(2, 3)),
             lambda: bf1.kv_compact(pages, pages, i(2, 4), i(2), i(2), i(2, 3)),
             lambda: bf1.page_fork(i(2), i(2), i(2), i(2, 3), i(9), i(9), i(1)),
             lambda: bf1.kv_copy(pages, pages, i(2), i(2), i(2))]
    for call in calls:
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="needs q or k"):
        bf1.qk_norm_rope(None, None, None, None, i(4), f)

"""How the operators around speculative and parallel decoding are called: on another stream,
from several threads at once, in graphs that replay in turn, with NaN in what a call must
not read."""

import threading

import numpy as np
import pytest
import torch

import paper_2608_20427_amd as bf1
from oracle import serve_oracle as so

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bf1.load()
    yield
    torch.cuda.synchronize()


def i32(x):
    return torch.as_tensor(np.asarray(x, dtype=np.int32), device="cuda")


def normal(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(shape, generator=g).to(dtype).cuda()


def calls(seed):
    """name -> (call, the tensors that it updates); call(**kw) returns a tuple of tensors."""
    rng = np.random.default_rng(seed)
    H, Hkv, d, B, n = 8, 4, 128, 64, 700
    f, amp = bf1.rope_freqs(d)
    q, k, dq, dk = (normal(seed + i, 1, h, n, d, dtype=t) for i, (h, t) in enumerate(
        ((H, torch.bfloat16), (Hkv, torch.bfloat16), (H, torch.float32), (Hkv, torch.float32))))
    gain, pos = 1 + 0.2 * normal(seed + 5, d), i32(range(n))
    held, counts = [3000, 64, 1500], [33, 5, 12]
    start = [0, 33, 38, 50]
    parents = [int(rng.integers(-1, i)) if i else -1 for c in counts for i in range(c)]
    after = [h + c for h, c in zip(held, counts)]
    pages = [-(-a // B) for a in after]
    P = sum(pages) + 9
    order = rng.permutation(P)
    table = np.full((3, max(pages) + 1), -1)
    at = 0
    for b, p in enumerate(pages):
        table[b, :p] = order[at:at + p]
        at += p
    kp, vp, rows = normal(seed + 6, P, Hkv, B, d), normal(seed + 7, P, Hkv, B, d), normal(seed + 8, 50, H, d)
    tree = i32(parents), i32(start), i32(held), i32(after)
    masks, tp = so.tree_step(parents, start, held, after)
    masks, tp = torch.as_tensor(np.array(masks, dtype=np.uint64).view(np.int64), device="cuda"), i32(tp)
    t = i32(table)
    shares, free, head = i32([0] * P), i32(order), i32([at])
    acc = i32([[1, 2, 4, -1], [0, 1, 2, 3], [5, 6, 7, 9]])
    src, keep = i32([1, 1, 0]), i32([70, 66, 2999])
    lists = i32([0, 1]), i32([2, 3]), i32([64, 5])
    return {
        "qk_norm_rope": (lambda **kw: bf1.qk_norm_rope(q, k, gain, gain, pos, f, amplitude=amp, **kw), ()),
        "qk_norm_rope_bwd": (lambda **kw: bf1.qk_norm_rope_bwd(dq, dk, q, k, gain, gain, pos, f, **kw), ()),
        "tree_step": (lambda **kw: bf1.tree_step(*tree, **kw), ()),
        "attn_tree": (lambda **kw: bf1.attn_tree(rows, kp, vp, masks, tp, tree[2], tree[1], t, B=B, **kw), ()),
        "attn_tree dense": (lambda **kw: bf1.attn_tree(rows, kp, vp, masks, tp, tree[2], tree[1], t, B=B, dense=True, **kw), ()),
        "kv_compact": (lambda **kw: (bf1.kv_compact(kp, vp, acc, tree[2], tree[3], t, **kw), kp, vp), (kp, vp)),
        "page_fork": (lambda **kw: (*bf1.page_fork(tree[3], src, keep, t, shares, free, head, B, **kw), shares, free),
                      (shares, free)),
        "kv_copy": (lambda **kw: (bf1.kv_copy(kp, vp, *lists, **kw), kp, vp)[1:], (kp, vp)),
    }


NAMES = ["qk_norm_rope", "qk_norm_rope_bwd", "tree_step", "attn_tree", "attn_tree dense", "kv_compact", "page_fork", "kv_copy"]


def run(call, state, **kw):
    """The call's results as copies; what it updates is put back."""
    keep = [x.clone() for x in state]
    out = [x.clone() for x in call(**kw)]
    for x, y in zip(state, keep):
        x.copy_(y)
    return out


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream(name):
    call, state = calls(1)[name]
    want = run(call, state)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    keep = [x.clone() for x in state]
    torch.cuda.synchronize()
    got = call(stream=side)  # the current stream is another one
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for x, y in zip(state, keep):
        x.copy_(y)
    with torch.cuda.stream(side):
        got = run(call, state)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_graphs_that_replay_in_turn(name):
    """Two captured calls with their own inputs, replayed in turn between eager ones: nothing
    of one call, its workspace least of all, is another's."""
    cases = [calls(s)[name] for s in (2, 3)]
    want = [run(*c) for c in cases]
    graphs = []
    for call, state in cases:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            run(call, state)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        keep = [x.clone() for x in state]
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = call()
        graphs.append((g, got, state, keep))
    for turn in range(6):
        g, got, state, keep = graphs[turn % 2]
        for x, y in zip(state, keep):
            x.copy_(y)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[turn % 2])), turn
        for x, y in zip(state, keep):
            x.copy_(y)
        eager = run(*cases[turn % 2])
        assert all(torch.equal(a, b) for a, b in zip(eager, want[turn % 2])), turn
        torch.cuda.synchronize()


def test_threads_at_once():
    names = [n for n in NAMES if n not in ("kv_compact", "page_fork", "kv_copy")]
    work = {s: calls(s) for s in (4, 5, 6)}
    want = {s: {n: run(*work[s][n]) for n in names} for s in work}
    torch.cuda.synchronize()
    wrong = []

    def go(s):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(5):
                for n in names:
                    got = run(*work[s][n])
                    torch.cuda.current_stream().synchronize()
                    if not all(torch.equal(a, b) for a, b in zip(got, want[s][n])):
                        wrong.append((s, n))

    threads = [threading.Thread(target=go, args=(s,)) for s in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_unused_strides_and_transposed_rows():
    """Dimensions of one entry may have any stride; heads and tokens may lie in any order."""
    d, f = 128, bf1.rope_freqs(128)[0]
    gain = 1 + 0.2 * normal(1, d)
    x = normal(2, 1, 1, 1, d)
    odd = x.as_strided((1, 1, 1, d), (7, 3, 5, 1))
    a, b = (bf1.qk_norm_rope(t, t.clone(), gain, gain, i32([9]), f)[0] for t in (x, odd))
    assert torch.equal(a, b)
    y = normal(3, 5, 3, 40, d)  # [heads, batch, n, d] seen as [batch, heads, n, d]
    z = y.transpose(0, 1)
    a = bf1.qk_norm_rope(z, None, gain, None, i32(range(40)), f)[0]
    out = torch.empty(40, 3, 5, d, dtype=torch.bfloat16, device="cuda").permute(1, 2, 0, 3)
    b = bf1.qk_norm_rope(z, None, gain, None, i32(range(40)), f, q_out=out)[0]
    assert b is out and torch.equal(a, b)
    # one gradient for every token (a stride of 0) is one like any other
    dy = normal(4, 3, 5, 1, d, dtype=torch.float32)
    a = bf1.qk_norm_rope_bwd(dy.expand(3, 5, 40, d), None, z, None, gain, None, i32(range(40)), f)
    b = bf1.qk_norm_rope_bwd(dy.expand(3, 5, 40, d).contiguous(), None, z.contiguous(), None, gain, None, i32(range(40)), f)
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2])

"""GPU parity of pages held by several sequences against their plain definition
(oracle/serve_oracle.py), copies of pages, and all of the operators of a step that
verifies drafts together.  Integers and copied rows: equal."""

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


def check_fork(lens, sources, keep, table, shares, free, head, B, **kw):
    s, f = i32(shares), i32(free)
    t = i32(table)
    got = bf1.page_fork(i32(lens), i32(sources), i32(keep), t, s, f, i32([head]), B, **kw)
    new, n, start, refs, free, copies = so.page_fork(list(map(int, lens)), list(map(int, sources)), list(map(int, keep)),
                                                     np.asarray(table).tolist(), shares, free, head, B)
    assert np.array_equal(got.page_table.cpu().numpy(), np.array(new).reshape(t.shape)) and got.seq_lens.tolist() == n
    assert int(got.free_head) == start and s.tolist() == refs and f.tolist() == list(free)
    assert list(zip(got.copy_from.tolist(), got.copy_to.tolist(), got.copy_rows.tolist())) == copies
    return got, s, f


class Pool:
    """Sequences that grow, fork and end: the operators beside their plain definitions, and
    what every sequence's cells hold."""

    def __init__(self, batch, width, pages, B, seed):
        self.rng = np.random.default_rng(seed)
        self.B, self.batch, self.width = B, batch, width
        self.lens, self.table = [0] * batch, [[-1] * width for _ in range(batch)]
        self.shares, self.free, self.head = [0] * pages, self.rng.permutation(pages).tolist(), 0
        self.cells = np.full((pages, B), -1)
        self.text = [[] for _ in range(batch)]  # what each sequence should read
        self.next = 0

    def append(self, new):
        t, f, h = i32(self.table), i32(self.free), i32([self.head])
        s = bf1.page_step(i32(self.lens), i32(new), t, f, h, int(sum(new)) + 3, self.B)
        slots, start, lens = s.slots.tolist(), s.token_start.tolist(), s.seq_lens.tolist()
        for b in range(self.batch):
            for i in range(lens[b] - self.lens[b]):
                slot = slots[start[b] + i]
                self.cells[slot // self.B, slot % self.B] = self.next
                self.text[b].append(self.next)
                self.next += 1
        self.table, self.lens, self.head = t.tolist(), lens, int(s.free_head)

    def fork(self, sources, keep):
        got, s, f = check_fork(self.lens, sources, keep, self.table, self.shares, self.free, self.head, self.B)
        text = []
        for b, src in enumerate(sources):
            text.append(self.text[src][:max(0, keep[b])] if 0 <= src < self.batch else [])
        for src, dst, rows in zip(got.copy_from.tolist(), got.copy_to.tolist(), got.copy_rows.tolist()):
            if dst >= 0:
                self.cells[dst, :rows] = self.cells[src, :rows]
        self.table, self.lens, self.head = got.page_table.tolist(), got.seq_lens.tolist(), int(got.free_head)
        self.shares, self.free = s.tolist(), f.tolist()
        self.text = [t[:n] for t, n in zip(text, self.lens)]

    def check(self):
        held = {}
        for b in range(self.batch):
            for i in range(-(-self.lens[b] // self.B)):
                held[self.table[b][i]] = held.get(self.table[b][i], 0) + 1
            read = [self.cells[self.table[b][p // self.B], p % self.B] for p in range(self.lens[b])]
            assert read == self.text[b], b
        # every page is free once or held as often as it counts
        left = self.free[self.head:]
        assert sorted(left + list(held)) == list(range(len(self.shares)))
        assert all(self.shares[p] == n - 1 for p, n in held.items()) and not any(self.shares[p] for p in left)


@pytest.mark.parametrize("batch,pages,B,seed", [(6, 60, 64, 0), (6, 40, 64, 1), (40, 200, 64, 2), (17, 400, 128, 3)])
def test_sequences_fork_grow_and_end(batch, pages, B, seed):
    """Random forks, reorders, rollbacks and ends between appended tokens: every sequence
    reads its own tokens, every page is held as often as it counts or is free."""
    pool = Pool(batch, 8, pages, B, seed)
    rng = pool.rng
    for step in range(25):
        pool.append([int(x) for x in rng.integers(0, 2 * B, batch) * (rng.random(batch) < 0.5)])
        pool.check()
        sources = [int(x) if rng.random() < 0.5 else b for b, x in enumerate(rng.integers(-1, batch, batch))]
        keep = [max(0, (pool.lens[s] if s >= 0 else 0) - int(rng.integers(0, B) * (rng.random() < 0.4))) for s in sources]
        pool.fork(sources, keep)
        pool.check()
    pool.fork([-1] * batch, [0] * batch)
    assert pool.head == 0 and sorted(pool.free) == list(range(pages))


@pytest.mark.parametrize("batch,width", [(1, 1), (1, 300), (255, 3), (1023, 2), (1024, 3), (1025, 2), (2100, 3),
                                         (180, 100), (1100, 20)])
def test_page_fork_matches_the_oracle(batch, width):
    rng = np.random.default_rng(batch)
    B = 64
    pages = batch * width + 40
    for kind in range(3):
        lens = rng.integers(0, width * B + 1, batch)
        table = rng.permutation(pages)[:batch * width].reshape(batch, width)
        used = {int(table[b, i]) for b in range(batch) for i in range(-(-lens[b] // B))}
        free = [p for p in rng.permutation(pages).tolist() if p not in used]
        free = list(used) + free  # room for every page
        shares = [0] * pages
        for p in list(used)[:5]:
            shares[p] = 1  # a caller holds it too
        sources = rng.integers(-2, batch + 2, batch) if kind == 0 else np.arange(batch) if kind == 1 \
            else rng.integers(0, max(1, batch // 9), batch)
        keep = rng.integers(-5, width * B + 9, batch)
        check_fork(lens, sources, keep, table, shares, free, len(used), B)


def test_page_fork_shortages_and_odd_arguments():
    B = 64
    table = [[3, 1, 4], [5, 9, 2], [6, -1, -1], [-1, -1, -1]]
    lens = [150, 130, 10, 0]
    for num_free in range(4):  # none of, some of and all of the pages for copies
        free = [0] * 7 + [7, 8, 10][:num_free]
        check_fork(lens, [0, 0, 0, 0], [150, 149, 148, 147], table, [0] * 12, free, 7, B)
    for head in (-5, 0, 3, 9, 10, 50):  # a head outside the list; fewer places below it than pages that come free
        check_fork(lens, [-1, 1, 1, 1], [0, 129, 129, 20], table, [0] * 12, [11, 10, 8, 7, 0, 0, 0, 0, 0], head, B)
    check_fork([0, 0, 0, 0], [0, 1, 2, 3], [5, 5, 5, 5], table, [0] * 12, [0], 0, B)
    check_fork([], [], [], np.zeros((0, 3)), [0, 0], [1, 0], 1, B)
    check_fork([500, -3, 10, 0], [0, 1, 2, 2], [500, 3, 2 ** 31 - 1, -7], table, [0] * 12, [0] * 9, 4, B)  # past the table
    check_fork([150, 70, 0, 0], [1, 0, 0, 9], [70, 150, 140, 3], [[3, 99, 4], [5, -1, 2], [0] * 3, [0] * 3], [0] * 12,
               [0] * 9, 4, B)  # entries that are no pages
    # every place starts again from one, whose page a caller holds: all copy
    check_fork([70, 0, 0, 0], [0] * 4, [70] * 4, table, [0, 2, 0, 1] + [0] * 8, [0] * 4 + [7, 8, 10, 11, 0], 4, B)


def test_page_fork_into_buffers_and_refusals():
    args = i32([70, 3]), i32([0, 0]), i32([70, 70]), i32([[1, 2, -1], [0, -1, -1]])
    state = lambda: (i32([0] * 6), i32([9, 9, 9, 3, 4, 5]), i32([3]))  # noqa: E731
    s1, s2, s3 = state(), state(), state()
    a = bf1.page_fork(*args, *s1)
    out = bf1.PageFork(*(torch.full_like(t, 7) for t in a))._replace(free_head=s2[2])  # the head in place
    b = bf1.page_fork(*args, *s2, out=out)
    c = bf1.page_fork(*args, *s3, stream=torch.cuda.current_stream())
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z) and x.shape == y.shape == z.shape
    assert torch.equal(s1[0], s2[0]) and torch.equal(s1[1], s2[1]) and b.free_head is s2[2]
    for bad in (dict(page_table=args[3]), dict(seq_lens=args[0]), dict(seq_lens=args[2])):
        with pytest.raises(bf1.BF1Error):
            bf1.page_fork(*args, *state(), out=out._replace(**bad))
    for i, x, why in [(0, i32([1]), "seq_lens"), (1, args[1].long(), "sources"), (2, i32([1]), "keep_lens"),
                      (3, i32([1]), "page_table"), (4, i32([[1]]), "shares"), (5, s1[1].float(), "free_pages"),
                      (6, i32([1, 2]), "free_head")]:
        bad = [*args, *state()]
        bad[i] = x
        with pytest.raises(ValueError, match=why):
            bf1.page_fork(*bad)
    with pytest.raises(bf1.BF1Error):
        bf1.page_fork(*args, *state(), B=16)


@pytest.mark.parametrize("Hkv,d,B", [(8, 128, 64), (1, 64, 64), (3, 64, 128), (2, 128, 128)])
def test_kv_copy(Hkv, d, B):
    P = 23
    k, v = normal(1, P, Hkv, B, d), normal(2, P, Hkv, B, d)
    src, dst = [0, 1, 2, 3, 0, -1, 4, 30, 5, 6], [10, 11, 12, 13, 14, 15, -1, 16, 40, 6]
    rows = [B, 1, 0, B // 2 + 1, B + 9, B, B, B, B, B]
    want = k.clone(), v.clone()
    for x, old in zip(want, (k, v)):
        for s, t, r in list(zip(src, dst, rows))[:5]:
            x[t, :, :min(r, B)] = old[s, :, :min(r, B)]
    k2, v2 = k.clone(), v.clone()
    bf1.kv_copy(k, v, i32(src), i32(dst), i32(rows))
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    bf1.kv_copy(k2, v2, i32(src), i32(dst), i32(rows), stream=torch.cuda.current_stream())
    assert torch.equal(k2, want[0]) and torch.equal(v2, want[1])
    bf1.kv_copy(k, v, i32([]), i32([]), i32([]))
    assert torch.equal(k, want[0])
    for bad, why in [((k, v, i32([1]), i32([1, 2]), i32([1])), "length"), ((k, v.float(), i32([1]), i32([1]), i32([1])), "v_pages"),
                     ((k, v, i32([1]).long(), i32([1]), i32([1])), "copy_from"), ((k[0], v[0], i32([1]), i32([1]), i32([1])), "4-D")]:
        with pytest.raises(ValueError, match=why):
            bf1.kv_copy(*bad)
    with pytest.raises(bf1.BF1Error):
        bf1.kv_copy(k, k, i32([1]), i32([2]), i32([3]))


def test_forked_8_bit_sequences():
    """Samples of one prompt over the 8-bit cache: pages shared, the growing block's tail
    copied (kv_copy takes tails as pages); each decodes as if it stood alone."""
    B, L, Hq, Hkv, d, batch, n = 64, 2, 4, 2, 64, 3, 150
    fork = [0, 0, 0]

    def serve(alone):
        cache = bf1.cache_q8(40, batch, Hkv, d, B)
        table = i32(np.full((batch, 8), -1))
        shares, free, head = i32([0] * 40), i32(range(40)), i32([0])
        lens = i32([0] * batch)

        def step(new, k, v):
            nonlocal head, lens
            s = bf1.page_step(lens, i32(new), table, free, head, sum(new), B)
            bf1.kv_append_q8(k, v, lens, s.seq_lens, s.token_start, s.block_start, table, cache)
            lens, head = s.seq_lens, s.free_head

        k, v = normal(1, n, Hkv, d), normal(2, n, Hkv, d)
        if alone:
            step([n] * batch, k.repeat(batch, 1, 1), v.repeat(batch, 1, 1))
        else:
            step([n, 0, 0], k, v)
            f = bf1.page_fork(lens, i32(fork), i32([n] * batch), table, shares, free, head)
            lens, head = f.seq_lens, f.free_head
            table.copy_(f.page_table)
            bf1.kv_copy(cache.k_tail, cache.v_tail, i32([0, 0, 0]), i32([-1, 1, 2]), i32([n % B] * 3))
        out = []
        for i in range(60):  # past the block's end: each sequence completes its own
            step([1] * batch, normal(10 + i, batch, Hkv, d), normal(90 + i, batch, Hkv, d))
            plan = bf1.decode_plan(lens, table, 40, bf1.decode_plan_stride(8 * B, B, L), B, L)
            out.append(bf1.attn_decode_q8(normal(200 + i, batch, Hq, d), cache, lens, plan, B)[0].clone())
        return torch.stack(out), int(head)

    (a, pages_alone), (b, pages) = serve(True), serve(False)
    assert torch.equal(a, b) and pages_alone == 3 * 4 and pages == 2 + 3 * 2


@pytest.mark.parametrize("sources,keep", [([1, 0, 0], [100, 150, 150]), ([2, 0, 1], [67, 140, 97]), ([1, -1, 2], [100, 0, 70]), ([1, 0, 9], [100, 150, 0]),
                                          ([0, 0, 1], [128, 128, 65])])
def test_8_bit_sequences_change_places(sources, keep):
    """Places of the 8-bit cache that change with each other, follow each other round, end, or
    go on from a full block: pages by page_fork, tails gathered, and each sequence decodes as if
    it had always been there."""
    B, L, Hq, Hkv, d, batch, lens0 = 64, 2, 4, 2, 64, 3, [150, 100, 70]
    if 128 in keep:
        lens0 = [128, 100, 70]
    rows = [(normal(7 + b, n, Hkv, d), normal(17 + b, n, Hkv, d)) for b, n in enumerate(lens0)]

    def serve(moved):
        cache = bf1.cache_q8(40, batch, Hkv, d, B)
        table = i32(np.full((batch, 8), -1))
        shares, free, head = i32([0] * 40), i32(range(40)), i32([0])
        lens = i32([0] * batch)

        def step(new, k, v):
            nonlocal head, lens
            s = bf1.page_step(lens, i32(new), table, free, head, sum(new), B)
            bf1.kv_append_q8(k, v, lens, s.seq_lens, s.token_start, s.block_start, table, cache)
            lens, head = s.seq_lens, s.free_head

        if moved:
            step(lens0, *(torch.cat([r[i] for r in rows]) for i in (0, 1)))
            f = bf1.page_fork(lens, i32(sources), i32(keep), table, shares, free, head)
            lens, head = f.seq_lens, f.free_head
            table.copy_(f.page_table)
            for tail in (cache.k_tail, cache.v_tail):
                tail.copy_(tail[i32(sources).clamp(0, batch - 1)])
            assert lens.tolist() == keep
        else:
            step(keep, *(torch.cat([rows[s % batch][i][:n] for s, n in zip(sources, keep)]) for i in (0, 1)))
        out = []
        for i in range(66):  # past the block's end: each sequence completes its own
            step([1] * batch, normal(30 + i, batch, Hkv, d), normal(130 + i, batch, Hkv, d))
            plan = bf1.decode_plan(lens, table, 40, bf1.decode_plan_stride(8 * B, B, L), B, L)
            out.append(bf1.attn_decode_q8(normal(230 + i, batch, Hq, d), cache, lens, plan, B)[0].clone())
        return torch.stack(out)

    a, b = serve(False), serve(True)
    assert a.isfinite().all() and torch.equal(a, b)


def draft_steps(graph, steps=5):
    """Speculative decoding as a program runs it: trees of drafted tokens appended, normed and
    turned, verified, the accepted path kept, the rest taken back; one sequence starts again
    from another on the way.  Attention of every node against float64 over the history of
    its own path."""
    B, L, Hq, Hkv, d = 64, 2, 4, 2, 64
    prompts, nodes = [130, 1, 63, 250], 7
    batch, rng = len(prompts), np.random.default_rng(5)
    parents = [-1, 0, 0, 1, 1, 3, 4]
    P = 60
    freqs, amp = bf1.rope_freqs(d, 1e4)
    qg, kg = 1 + 0.3 * normal(3, d, dtype=torch.float32), 1 + 0.3 * normal(4, d, dtype=torch.float32)
    kp, vp = torch.zeros((P, Hkv, B, d), dtype=torch.bfloat16, device="cuda"), torch.zeros((P, Hkv, B, d), dtype=torch.bfloat16, device="cuda")
    table, shares = i32(np.full((batch, 10), -1)), i32([0] * P)
    free, head, lens = i32(rng.permutation(P)), i32([0]), i32([0] * batch)
    hist = [(np.zeros((0, Hkv, d)), np.zeros((0, Hkv, d))) for _ in prompts]

    def place(new, rows, q, k, v, positions=None):
        s = bf1.page_step(lens, new, table, free, head, rows, B)
        q, k = bf1.qk_norm_rope(q, k, qg, kg, s.positions if positions is None else positions(s), freqs, amplitude=amp)
        bf1.kv_append(k, v, s.slots, kp, vp)
        return s, q, k

    rows = sum(prompts)
    x = normal(1, rows, Hq + 2 * Hkv, d)
    s, _, k = place(i32(prompts), rows, *x.split((Hq, Hkv, Hkv), 1))
    at = 0
    for b, n in enumerate(prompts):
        hist[b] = tuple(t[at:at + n].double().cpu().numpy() for t in (k, x[:, Hq + Hkv:]))
        at += n
    lens.copy_(s.seq_lens)
    head.copy_(s.free_head)

    T = batch * nodes
    x = torch.zeros((T, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    par, new = i32(parents * batch), i32([nodes] * batch)
    accepted, sources = i32(np.full((batch, nodes), -1)), i32(range(batch))

    def verify():
        tree = []

        def positions(s):
            tree.extend(bf1.tree_step(par, s.token_start, lens, s.seq_lens))
            return tree[1]

        s, q, k = place(new, T, *x.split((Hq, Hkv, Hkv), 1), positions=positions)
        o, lse = bf1.attn_tree(q, kp, vp, *tree, lens, s.token_start, table, B, L, max_nodes=nodes)
        kept = bf1.kv_compact(kp, vp, accepted, lens, s.seq_lens, table)
        keep = kept[sources.long()]
        f = bf1.page_fork(s.seq_lens, sources, keep, table, shares, free, s.free_head, B)
        bf1.kv_copy(kp, vp, f.copy_from, f.copy_to, f.copy_rows)
        table.copy_(f.page_table)
        lens.copy_(f.seq_lens)
        head.copy_(f.free_head)
        return q, k, o, lse

    def inputs(i):
        x.copy_(normal(10 + i, *x.shape))
        paths = [[0, 2], [0, 1, 4, 6], [], [0, 1, 3, 5]]
        paths = [paths[(b + i) % 4] for b in range(batch)]
        accepted.copy_(i32([p + [-1] * (nodes - len(p)) for p in paths]))
        src = list(range(batch))
        if i % 2:
            src[i % batch] = (i + 2) % batch
        sources.copy_(i32(src))
        return paths, src

    state = (lens, head, table, shares, free, kp, vp)
    if graph:
        keep = [t.clone() for t in state]
        inputs(0)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            verify()
        torch.cuda.current_stream().wait_stream(side)
        for t, y in zip(state, keep):
            t.copy_(y)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got = verify()
    masks, _ = so.tree_step(parents, [0, nodes], [0], [nodes])
    for i in range(steps):
        paths, src = inputs(i)
        held = lens.tolist()
        if graph:
            g.replay()
            torch.cuda.synchronize()
        else:
            got = verify()
        q, k, o, lse = (t.double().cpu().numpy() for t in got)
        v = x[:, Hq + Hkv:].double().cpu().numpy()
        for b in range(batch):
            assert held[b] == len(hist[b][0])
            for n in range(nodes):
                path = [b * nodes + a for a in range(nodes) if masks[n] >> a & 1]
                p = held[b] + len(path) - 1
                keys, values = (np.concatenate([hist[b][j], y[path]]) for j, y in ((0, k), (1, v)))
                sel = [t for j in so.route(p // B, L) + [p // B] for t in range(j * B, min(j * B + B, p + 1))]
                for h in range(Hq):
                    ref, l, mass = so.attend(q[b * nodes + n, h], keys[sel, h // 2], values[sel, h // 2])
                    assert np.abs(o[b * nodes + n, h] - ref).max() < 2.0 ** -8 * np.abs(ref).max() + 2e-4 * mass.max()
                    assert abs(lse[b * nodes + n, h] - l) < 1e-4
        after = [tuple(np.concatenate([hist[b][j], y[[b * nodes + a for a in paths[b]]]]) for j, y in ((0, k), (1, v)))
                 for b in range(batch)]
        hist = [after[s] for s in src]
        # every sequence's cells hold its history
        for b in range(batch):
            n = int(lens[b])
            assert n == len(hist[b][0])
            pg, off = table[b, torch.arange(n, device="cuda") // B].long(), torch.arange(n, device="cuda") % B
            for j, pages in ((0, kp), (1, vp)):
                assert np.array_equal(pages[pg, :, off].double().cpu().numpy(), hist[b][j])
    held = {}
    for b in range(batch):
        for p in table[b, :-(-int(lens[b]) // B)].tolist():
            held[p] = held.get(p, 0) + 1
    assert sorted(free[int(head):].tolist() + list(held)) == list(range(P))
    assert all(shares[p] == n - 1 for p, n in held.items())


def test_draft_steps():
    draft_steps(graph=False, steps=8)


def test_draft_steps_captured_and_replayed():
    draft_steps(graph=True)

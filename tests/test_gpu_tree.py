"""GPU parity of drafted trees over the paged cache against their plain definitions
(oracle/serve_oracle.py): masks and positions, the attention of all nodes, the accepted
nodes' rows moved together.

Bars.  Integers and moved rows: equal.  Attention: `tree_bars`."""

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


def f64(t):
    return t.detach().double().cpu().numpy()


def signed(masks):
    return torch.as_tensor(np.array([m for m in masks], dtype=np.uint64).view(np.int64), device="cuda")


def random_parents(rng, nodes, deep=False):
    return [-1 if i == 0 or rng.random() < 0.08 else i - 1 if deep else int(rng.integers(max(0, i - 6), i))
            for i in range(nodes)]


# ---- masks and positions ---------------------------------------------------------------

@pytest.mark.parametrize("counts,spare", [([1], 0), ([0], 3), ([64], 1), ([5, 0, 64, 1, 17, 33], 0), ([3] * 301, 70), ([70, 2], 5),
                                          ([], 4)])
def test_tree_step_matches_the_oracle(counts, spare):
    rng = np.random.default_rng(len(counts) + spare)
    start = np.concatenate([[0], np.cumsum(counts)]).astype(int)
    held = rng.integers(0, 5000, len(counts))
    parents = [p for n in counts for p in random_parents(rng, n)] + [7] * spare
    for lost in (0, 2):  # nodes at the end without a place
        after = held + np.maximum(0, np.array(counts, dtype=int) - lost)
        masks, pos = bf1.tree_step(i32(parents), i32(start), i32(held), i32(after))
        want, wpos = so.tree_step(parents, start, held, after)
        assert torch.equal(masks, signed(want)) and pos.tolist() == wpos


def test_tree_step_chains_roots_and_odd_parents():
    # a chain of 64 (every generation), all roots, and parents that are no earlier node's
    parents = list(range(-1, 63)) + [-1] * 64 + [64, 1, 2, 3, -9, 2 ** 31 - 1, -2 ** 31, 0]
    start = [0, 64, 128, 136]
    masks, pos = bf1.tree_step(i32(parents), i32(start), i32([3, 0, 2 ** 31 - 3]), i32([67, 64, 2 ** 31 - 1]))
    want, wpos = so.tree_step(parents, start, [3, 0, 2 ** 31 - 3], [67, 64, 2 ** 31 - 1])
    assert torch.equal(masks, signed(want)) and pos.tolist() == wpos
    # lengths that cannot be: negative ones count as 0, fewer after than before as no nodes
    masks, pos = bf1.tree_step(i32([-1, 0, -1]), i32([0, 2, 3]), i32([-5, 9]), i32([2, 4]))
    assert masks.tolist() == [1, 3, 0] and pos.tolist() == [0, 1, -1]


def test_tree_step_into_buffers_and_refusals():
    args = i32([-1, 0, 0]), i32([0, 2, 3]), i32([4, 5]), i32([6, 6])
    a = bf1.tree_step(*args)
    m, p = torch.full((3,), 7, device="cuda"), i32([7] * 3)
    b = bf1.tree_step(*args, masks=m, positions=p)
    assert b[0] is m and torch.equal(a[0], m) and torch.equal(a[1], p)
    c = bf1.tree_step(*args, stream=torch.cuda.current_stream())
    assert torch.equal(a[0], c[0]) and torch.equal(a[1], c[1])
    for at, why in [((0, i32([[1]])), "parents"), ((1, i32([0, 1])), "token_start"), ((2, args[2].long()), "lens_before"),
                    ((3, i32([1])), "seq_lens")]:
        bad = list(args)
        bad[at[0]] = at[1]
        with pytest.raises(ValueError, match=why):
            bf1.tree_step(*bad)
    with pytest.raises(ValueError, match="masks"):
        bf1.tree_step(*args, masks=i32([1] * 3))


# ---- attention -------------------------------------------------------------------------

def tree_bars(q, keys, ref):
    """(bar of o, bar of lse) of one row.  A score's fp32 sum of d products is off by at
    most d 2^-24 of the sum of their magnitudes, and by 2^-22 of itself (log2 e, the
    subtraction of the largest); a weight by twice that (its own and the sum's), exp2 2^-22,
    and its two bf16 parts leave out 2^-17 (half a step of the second, 2^-9 of the first's
    rest 2^-8); sums over n keys n 2^-24; the quotient 2^-23; the output half a step, 2^-8."""
    o, lse, mass = ref
    d, n = q.shape[0], len(keys)
    if n == 0:
        return np.zeros(d), 0.0
    big = (np.abs(keys) @ np.abs(q)).max() / np.sqrt(d)
    ds = big * (d * 2.0 ** -24 + 2.0 ** -22)
    rel = 2 * ds + 2.0 ** -17 + 2.0 ** -21 + 2 * n * 2.0 ** -24
    return 2.0 ** -8 * np.abs(o) + (1 + 2.0 ** -8) * mass * rel + 1e-30, ds + n * 2.0 ** -23 + 1e-6 + 2.0 ** -22 * abs(lse)


class Case:
    """A batch of trees over a cache whose unread places hold NaN or infinity."""

    def __init__(self, held, counts, Hq, Hkv, d, B, seed, spare=3, deep=False, masks=None, width=0, scale=1.0):
        rng = np.random.default_rng(seed)
        self.held, self.counts, self.B, self.G = [int(x) for x in held], counts, B, Hq // Hkv
        self.start = [0] + [int(x) for x in np.cumsum(counts)]
        rows = self.start[-1]
        parents = [p for n in counts for p in random_parents(rng, n, deep)]
        self.masks, self.pos = so.tree_step(parents, self.start, self.held, [h + n for h, n in zip(self.held, counts)])
        if masks is not None:
            self.masks = masks(self, rng)
        blocks = [-(-(h + n) // B) for h, n in zip(self.held, counts)]
        P = sum(blocks) + spare
        order = rng.permutation(P)
        self.width = max(blocks + [1]) + 1 + width
        self.table = np.full((len(held), self.width), -1)
        at = 0
        for b, n in enumerate(blocks):
            self.table[b, :n] = order[at:at + n]
            at += n
        g = torch.Generator().manual_seed(seed)
        self.k, self.v = ((torch.randn((P, Hkv, B, d), generator=g) * s).bfloat16() for s in (scale, 1.0))
        lost = torch.ones((P, B), dtype=torch.bool)
        for b, n in enumerate(blocks):
            for p in range(self.held[b] + counts[b]):
                lost[self.table[b, p // B], p % B] = False
        for x in (self.k, self.v):
            x[:] = torch.where(lost[:, None, :, None], torch.where(torch.rand(x.shape, generator=g) < 0.5, np.nan, np.inf), x)
        self.q = torch.randn((rows, Hq, d), generator=g).bfloat16()

    def run(self, L=2, dense=False, **kw):
        return bf1.attn_tree(self.q.cuda(), self.k.cuda(), self.v.cuda(), signed(self.masks), i32(self.pos), i32(self.held),
                             i32(self.start), i32(self.table), B=self.B, L=L, dense=dense, **kw)

    def check(self, got, L=2, dense=False, most=64):
        o, lse = f64(got[0]), f64(got[1])
        q = f64(self.q)
        k, v = f64(self.k), f64(self.v)
        for b in range(len(self.held)):
            for r in range(self.start[b], self.start[b + 1]):
                keys = so.tree_keys(b, r, self.masks, self.pos, self.held, self.start, self.B, L, dense, most)
                if keys is None or r - self.start[b] >= most:
                    assert np.isnan(o[r]).all() and np.isnan(lse[r]).all(), (b, r)
                    continue
                at, off = self.table[b, np.array(keys, dtype=int) // self.B], np.array(keys, dtype=int) % self.B
                for h in range(q.shape[1]):
                    kk, vv = k[at, h // self.G, off], v[at, h // self.G, off]
                    ref = so.attend(q[r, h], kk, vv)
                    bo, bl = tree_bars(q[r, h], kk, ref)
                    assert (np.abs(o[r, h] - ref[0]) <= bo).all(), (b, r, h, np.abs(o[r, h] - ref[0]).max())
                    assert lse[r, h] == ref[1] or abs(lse[r, h] - ref[1]) <= bl, (b, r, h, lse[r, h], ref[1])


@pytest.mark.parametrize("Hq,Hkv,d,B", [(16, 8, 128, 64), (4, 4, 64, 64), (8, 2, 128, 128), (8, 1, 64, 128), (8, 1, 128, 64),
                                        (2, 1, 64, 128), (3, 3, 128, 128), (4, 1, 64, 64)])
def test_attn_tree_matches_the_oracle(Hq, Hkv, d, B):
    c = Case([0, 1, B - 1, B, 5 * B + 7, 9 * B - 3, 700], [3, 1, 17, 0, 33, 64, 6], Hq, Hkv, d, B, seed=Hq + d + B)
    for L, dense in ((2, False), (1, False), (0, True)):
        c.check(c.run(L, dense), L, dense)


@pytest.mark.parametrize("L", [0, 1, 2, 3, 5, 32])
def test_attn_tree_routes(L):
    # blocks around powers of two, trees that reach into the next block
    B = 64
    held = [j * B + o for j in (0, 1, 2, 3, 4, 5, 7, 8, 9, 16, 31, 35) for o in (50, 63)]
    c = Case(held, [16] * len(held), 2, 1, 64, B, seed=L, deep=True)
    c.check(c.run(L), L)


@pytest.mark.parametrize("nodes", [1, 2, 7, 8, 9, 15, 16, 17, 31, 32, 33, 48, 63, 64])
@pytest.mark.parametrize("G", [1, 2, 8])
def test_attn_tree_sizes(nodes, G):
    c = Case([200, 61, 320], [nodes, max(0, nodes - 3), 1], G, 1, 64, 64, seed=nodes + G)
    c.check(c.run(max_nodes=nodes))
    c.check(c.run())
    if nodes > 2:  # fewer than there are: the rest is NaN
        c.check(c.run(max_nodes=nodes - 2), most=nodes - 2)


@pytest.mark.parametrize("L", [0, 2])
@pytest.mark.parametrize("copies,Hq,Hkv,nodes,d,B", [(5, 16, 2, 64, 64, 64), (5, 8, 4, 64, 64, 64), (2, 8, 4, 64, 128, 64),
                                                     (5, 8, 4, 16, 64, 128), (4, 8, 1, 64, 128, 128),
                                                     (4, 4, 1, 64, 128, 128)])
def test_attn_tree_columns(copies, Hq, Hkv, nodes, d, B, L):
    """Batches whose rows run 128, 64 (in workgroups of four and of eight waves) and 32 columns
    at a time: trees that reach into the next block, sequences at blocks' ends."""
    rng = np.random.default_rng(copies + nodes)
    held = [j * B + o for j in (0, 1, 2, 3, 5, 9, 16) for o in (3, B - 1)] * copies
    counts = [int(rng.integers(nodes * 3 // 4, nodes + 1)) if rng.random() < 0.5 else int(rng.integers(0, 4)) for _ in held]
    counts[0] = nodes
    c = Case(held, counts, Hq, Hkv, d, B, seed=nodes, deep=True, width=20000 if Hq // Hkv == 8 else 0)
    c.check(c.run(L, max_nodes=nodes), L)


@pytest.mark.parametrize("batch,Hq,Hkv,nodes,d,B", [(14, 8, 8, 3, 128, 64), (28, 8, 8, 16, 64, 64), (14, 16, 8, 8, 64, 64),
                                                    (16, 8, 2, 12, 64, 128), (14, 16, 4, 9, 128, 128), (10, 8, 1, 20, 128, 64)])
def test_attn_tree_short_lists(batch, Hq, Hkv, nodes, d, B):
    """16 columns at a time, as many sequences, heads and nodes as leave room for two splits or
    none; also with a value that is not finite, which sends its columns over their keys once more."""
    rng = np.random.default_rng(batch + nodes)
    held = [int(j * B + o) for j, o in zip(rng.integers(0, 10, batch), rng.choice([0, 1, 40, B - 2, B - 1], batch))]
    held[:2] = [9 * B + B - 1, 8 * B + 5]
    c = Case(held, [nodes, nodes, 0] + [int(x) for x in rng.integers(1, nodes + 1, batch - 3)], Hq, Hkv, d, B, seed=nodes,
             deep=True)
    for L, dense in ((2, False), (0, False), (2, True)):
        c.check(c.run(L, dense, max_nodes=nodes), L, dense)
    x, page = c.v, c.table[1, 8]
    clean = c.run(max_nodes=nodes)
    x[page, 0, 2, 5] = float("inf")  # position 8 B + 2: committed, every node of sequence 1 reads it
    o = c.run(max_nodes=nodes)[0]
    hit = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    hit[c.start[1]:c.start[2], :Hq // Hkv, 5] = True
    # the others of its rows are sums over 500 keys, below 2: both within a step, 2^-7, at most
    assert (o[hit] == float("inf")).all() and (o[~hit].float() - clean[0][~hit].float()).abs().max() < 2.0 ** -6


@pytest.mark.parametrize("width", [20, 200, 2000, 20000])
@pytest.mark.parametrize("G,nodes", [(1, 40), (4, 16), (8, 33)])
def test_attn_tree_wide_tables(width, G, nodes):
    """The same lists under ever wider tables, that is with every number of columns and splits."""
    c = Case([700, 64, 200, 0], [nodes, 3, nodes // 2, 5], 2 * G, 2, 64, 64, seed=width, width=width)
    for dense in (True, False):
        c.check(c.run(dense=dense, max_nodes=nodes), dense=dense)


def test_attn_tree_long_lists_split():
    c = Case([9000, 4097, 64], [5, 16, 2], 8, 4, 128, 64, seed=4)
    for kw in (dict(dense=True, L=0), dict(L=2)):
        c.check(c.run(**kw), **kw)
    # one long list among short ones, in a wide table
    c = Case([6000, 3, 70, 0], [9, 9, 9, 9], 2, 2, 64, 64, seed=5, width=300)
    c.check(c.run(dense=True), dense=True)
    c.check(c.run())


@pytest.mark.parametrize("batch,G,Hkv,nodes,d,B", [(5, 8, 1, 64, 64, 64), (5, 4, 2, 16, 128, 128), (2, 8, 1, 33, 128, 64),
                                                   (64, 8, 1, 8, 64, 64), (65, 8, 1, 8, 64, 64), (19, 2, 3, 40, 64, 128)])
def test_attn_tree_unequal_dense_lists(batch, G, Hkv, nodes, d, B):
    """Dense lists under a wide table, whose splits go by each sequence's length: one long one
    among short and empty ones, sequences that draft nothing or lack a page."""
    rng = np.random.default_rng(batch + nodes)
    held = [2500] + [int(x) for x in rng.choice([0, 1, B - 1, B, 300, 900], batch - 1)]
    counts = [nodes] + [int(x) for x in rng.integers(0, nodes + 1, batch - 1)]
    counts[-1] = 0 if batch > 2 else 1
    for h in (held, held[::-1]):
        n = counts if h is held else counts[::-1]
        c = Case(h, n, G * Hkv, Hkv, d, B, seed=batch, width=2000)
        assert bf1.attn_tree_workspace_size(batch, nodes, G * Hkv, Hkv, d, B, c.width, dense=True) > 0
        got = c.run(dense=True, max_nodes=nodes)
        c.check(got, dense=True)
        assert all(torch.equal(x, y) for x, y in zip(got, c.run(dense=True, max_nodes=nodes)))
    c.table[-1, 3] = -1  # of the long one
    o, lse = c.run(dense=True, max_nodes=nodes)
    assert o[c.start[-2]:].isnan().all() and lse[c.start[-2]:].isnan().all()
    assert torch.equal(o[:c.start[-2]], got[0][:c.start[-2]]) and o[:c.start[-2]].isfinite().all()


def test_attn_tree_wide_batch():
    rng = np.random.default_rng(8)
    c = Case(rng.integers(0, 400, 150), list(rng.integers(0, 20, 150)), 4, 2, 64, 64, seed=8)
    c.check(c.run(max_nodes=19))


def test_attn_tree_any_masks():
    """Masks that are no tree's: rows that read nothing, nodes that read later ones or
    not themselves, bits of nodes that are not there."""
    def odd(c, rng):
        return [0 if i % 5 == 0 else int(rng.integers(0, 2 ** 63)) * 2 + int(rng.integers(0, 2)) for i in range(len(c.masks))]

    for L in (0, 2):
        c = Case([0, 60, 130, 300], [20, 20, 64, 5], 4, 2, 64, 64, seed=3, masks=odd, deep=True)
        got = c.run(L)
        c.check(got, L)
        empty = [r for r in range(20) if c.masks[r] == 0]
        assert empty and not got[0][empty].any() and (got[1][empty] == float("-inf")).all()


def test_attn_tree_rows_without_a_place():
    c = Case([100, 10], [8, 6], 4, 2, 64, 64, seed=6)
    for r, p in ((3, -1), (5, 99), (7, 164), (9, 74), (12, 2 ** 31 - 1)):
        c.pos[r] = p
    c.check(c.run())
    c.pos = [-1] * 14  # no node at all
    assert c.run()[0].isnan().all()


@pytest.mark.parametrize("Hq,nodes,width", [(4, 16, 0), (2, 20, 440), (2, 20, 20000), (4, 20, 20000), (8, 40, 20000)])  # 16 to 128
@pytest.mark.parametrize("where", ["k", "v"])
def test_attn_tree_values_that_are_not_finite(where, Hq, nodes, width):
    """A key or value that is not finite reaches the rows that read it, as the formula has
    it, and no other."""
    B, d, G = 64, 64, Hq // 2
    make = lambda: Case([300, 127], [nodes, 16], Hq, 2, d, B, seed=7, width=width)  # noqa: E731
    c, clean = make(), make()
    x = c.k if where == "k" else c.v
    # drafted node 5 of sequence 0 and node 3 of sequence 1
    x[c.table[0, 305 // B], 1, 305 % B, 3] = float("inf")
    x[c.table[1, 130 // B], 0, 130 % B, 9] = float("nan") if where == "v" else float("inf")
    dense = width > 0
    got, want = c.run(dense=dense), clean.run(dense=dense)
    o, lse, w = f64(got[0]), f64(got[1]), f64(want[0])
    for b, node, head, dim in ((0, 5, 1, 3), (1, 3, 0, 9)):
        for r in range(c.start[b], c.start[b + 1]):
            reads = c.masks[r] >> node & 1
            for h in range(Hq):
                hit = reads and h // G == head
                if not hit:
                    assert np.isfinite(o[r, h]).all() and np.abs(o[r, h] - w[r, h]).max() < 2.0 ** -6, (b, r, h)
                elif where == "v":
                    bad = np.isnan(o[r, h, dim]) if b else o[r, h, dim] == np.inf
                    assert bad and np.isfinite(np.delete(o[r, h], dim)).all() and np.isfinite(lse[r, h]), (b, r, h)
                else:  # a score that is +-infinity (or NaN): all of the row, or none of it
                    assert np.isnan(o[r, h]).all() or np.abs(o[r, h]).max() < 10


@pytest.mark.parametrize("Hq,nodes,width", [(2, 4, 0), (2, 16, 30000), (2, 32, 30000), (4, 64, 30000)])
def test_attn_tree_infinity_under_a_small_weight(Hq, nodes, width):
    """An infinite value is there at any weight, also across units, waves and splits."""
    c = Case([5000], [nodes], Hq, 1, 128, 64, seed=9, scale=4.0, width=width)
    page = c.table[0, 7]
    c.v[page, 0, 20, 5] = float("-inf")
    got = c.run(dense=True)
    assert (got[0][:, :, 5] == float("-inf")).all()
    rest = torch.cat([got[0][:, :, :5], got[0][:, :, 6:]], 2)
    assert rest.isfinite().all() and got[1].isfinite().all()


def bf16(x):
    return f64(torch.as_tensor(x).bfloat16())


@pytest.mark.parametrize("batch,Hq,nodes,width,d,B", [(2, 2, 8, 0, 64, 64), (2, 4, 16, 0, 128, 128), (2, 2, 20, 20000, 64, 128),
                                                      (2, 4, 20, 20000, 128, 64), (130, 4, 20, 200, 64, 64),
                                                      (2, 8, 40, 20000, 64, 64), (2, 8, 33, 20000, 128, 128)])  # 16 to 128 columns
def test_attn_tree_weights_keep_their_24_bits(batch, Hq, nodes, width, d, B):
    """Values that cancel all of a weight but what two bf16 parts leave out of it.

    Rows read three committed keys: two of 0 and one whose score, -t / sqrt(d), gives it the
    weight p in [0.5, 1), another one for each row.  Dim i of the values is -hi, -mid and 1, hi and mid the
    rounded parts of row i's p: row i's output is (p - hi - mid) / (2 + p), below 2^-18.

    Bar: the largest score is 0, so a weight's exponent, of size 0.73 at most, is off by three
    roundings of log2(e) / sqrt(d) and its own, 3.2 * 2^-24, times ln 2 of p, and exp2 by one
    step: 3.3 * 2^-24.  Parts and values are whole numbers of 2^-24, but for the tiniest middle
    parts, and partial sums below 1: they round by 2^-24 in all.  The quotient is off by 2^-22 of
    itself, and rounded once, 2^-8."""
    none = lambda c, rng: [0] * len(c.masks)  # noqa: E731
    c = Case([3] * batch, [nodes] * batch, Hq, 2, d, B, seed=1, width=width, masks=none)
    rows = batch * nodes
    at = (np.arange(rows * Hq) % d).reshape(rows, Hq)
    t = (2 + at / 64) * (1 if d == 64 else 1.25)  # bf16 numbers
    t = bf16(t)
    c.q[:] = 0
    c.q[:, :, 0] = torch.as_tensor(t).bfloat16()
    p = np.exp(-t / np.sqrt(d))
    assert (p >= 0.5).all() and (p < 1).all()
    parts = np.zeros((3, d))
    parts[0][at] = -bf16(p)
    parts[1][at] = -bf16(p - bf16(p))
    parts[2] = 1
    first = c.table[:, 0]
    for i in range(3):
        c.k[first, :, i] = 0
        c.v[first, :, i] = torch.as_tensor(parts[i]).bfloat16()
    c.k[first, :, 2, 0] = -1
    o, lse = c.run(dense=width > 0, max_nodes=nodes)
    want = (p[..., None] + parts[0] + parts[1]) / (2 + p[..., None])
    bar = 4.3 * 2.0 ** -24 / (2 + p[..., None]) + 2.0 ** -22 * np.abs(want)
    bar = bar + 2.0 ** -8 * (np.abs(want) + bar)
    off = np.abs(f64(o) - want)
    assert (off <= bar).all(), (off - bar).max()
    assert np.abs(f64(lse) - np.log(2 + p)).max() < 2.0 ** -21


def test_attn_tree_missing_pages():
    for entry, dense in ((0, False), (3, True), (8, False), (9, False)):
        c = Case([600, 100], [40, 4], 4, 2, 64, 64, seed=10, deep=True)
        for bad in (-1, 10 ** 6):
            c.table[0, entry] = bad  # block 0, an earlier one, the two that hold the nodes
            o, lse = c.run(dense=dense)
            assert o[:40].isnan().all() and lse[:40].isnan().all() and o[40:].isfinite().all()
    c = Case([600], [4], 4, 2, 64, 64, seed=11)
    c.table[0, 3] = -1  # off the route of block 9: {0, 1, 5, 7, 8}
    assert c.run()[0].isfinite().all()
    c.held, c.pos = [2 ** 31 - 100], [2 ** 31 - 100 + i for i in range(4)]  # past the table
    assert c.run()[0].isnan().all()


def test_attn_tree_leaves_rows_behind_and_guards():
    c = Case([100, 40], [7, 5], 4, 2, 64, 64, seed=12)
    rows = 12
    o = torch.full((rows + 9, 4, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((rows + 9, 4), 7.0, device="cuda")
    q = torch.cat([c.q, c.q[:9]]).cuda()
    masks, pos = torch.cat([signed(c.masks), signed([1] * 9)]), torch.cat([i32(c.pos), i32([40] * 9)])
    need = bf1.attn_tree_workspace_size(2, 64, 4, 2, 64, 64, c.width + 400, dense=True)
    assert need > 0
    table = torch.full((2, c.width + 400), -1, dtype=torch.int32, device="cuda")
    table[:, :c.width] = i32(c.table)
    ws = torch.full((need + 64,), 9, dtype=torch.uint8, device="cuda")
    got = bf1.attn_tree(q, c.k.cuda(), c.v.cuda(), masks, pos, i32(c.held), i32(c.start), table, dense=True, out=o, lse=lse,
                        workspace=ws)
    assert got[0] is o and (o[rows:] == 7).all() and (lse[rows:] == 7).all() and (ws[need:] == 9).all()
    c.check((o[:rows], lse[:rows]), dense=True)
    again = c.run(dense=True, stream=torch.cuda.current_stream())
    assert all(torch.equal(x, y) for x, y in zip(again, c.run(dense=True)))


def test_attn_tree_is_a_chain_of_decodes():
    """A chain of drafted tokens gives what one decode step after the other gives, within
    both kernels' bars (twice the larger)."""
    B, L, held, n, Hq, Hkv, d = 64, 2, 700, 5, 8, 4, 128
    c = Case([held], [n], Hq, Hkv, d, B, seed=13)
    c.masks, c.pos = so.tree_step([-1, 0, 1, 2, 3], [0, n], [held], [held + n])
    o, lse = c.run(L)
    k, v, table = c.k.cuda(), c.v.cuda(), i32(c.table)
    for i in range(n):
        lens = i32([held + i + 1])
        stride = bf1.decode_plan_stride(held + n, B, L)
        plan = bf1.decode_plan(lens, table, k.shape[0], stride, B, L)
        od, ld = bf1.attn_decode(c.q[i:i + 1].cuda(), k, v, lens, plan, B)
        assert (o[i].float() - od[0].float()).abs().max() < 2.0 ** -7 and (lse[i] - ld[0]).abs().max() < 1e-4


def test_attn_tree_refusals():
    c = Case([100], [3], 4, 2, 64, 64, seed=14)
    ok = dict(q=c.q.cuda(), k_pages=c.k.cuda(), v_pages=c.v.cuda(), masks=signed(c.masks), positions=i32(c.pos),
              lens_before=i32(c.held), token_start=i32(c.start), page_table=i32(c.table))
    for bad, why in [(dict(q=ok["q"].float()), "q must"), (dict(q=ok["q"][:, :, :32]), "q must"), (dict(B=128), "B tokens"),
                     (dict(masks=i32([1, 1, 1])), "masks"), (dict(positions=i32([1, 2])), "positions"),
                     (dict(lens_before=i32([1, 2])), "lens_before"), (dict(token_start=i32([0])), "token_start"),
                     (dict(page_table=i32([1])), "page_table"), (dict(v_pages=ok["v_pages"][1:]), "v_pages"),
                     (dict(k_pages=ok["k_pages"].cpu()), "CUDA"), (dict(lse=torch.empty(3, 4)), "lse"),
                     (dict(out=torch.empty(3, 4, 64, device="cuda")), "out")]:
        with pytest.raises(ValueError, match=why):
            bf1.attn_tree(**{**ok, **bad})
    for bad in (dict(max_nodes=65), dict(max_nodes=0), dict(L=33), dict(L=-1), dict(q=ok["q"][:, :3].contiguous())):
        with pytest.raises(bf1.BF1Error):
            bf1.attn_tree(**{**ok, **bad})


# ---- the accepted nodes' rows ------------------------------------------------------------

@pytest.mark.parametrize("Hkv,d,B", [(8, 128, 64), (3, 64, 128), (1, 64, 64), (2, 128, 128)])
def test_kv_compact_matches_the_oracle(Hkv, d, B):
    rng = np.random.default_rng(Hkv + d)
    held = [0, 1, B - 1, B - 5, 3 * B, 5 * B + 13, 77, 9, 30]
    counts = [64, 5, 64, 9, 0, 33, 64, 4, 64]
    paths = [sorted(rng.choice(n, rng.integers(0, n + 1), replace=False).tolist()) if n else [] for n in counts]
    paths[0], paths[2], paths[7], paths[8] = list(range(64)), list(range(1, 64)), [0, 2, 2, 3], [63]
    accepted = np.full((len(held), 64), -1)
    for b, p in enumerate(paths):
        accepted[b, :len(p)] = p
    accepted[1] = np.arange(64) + 2  # runs past the nodes
    c = Case(held, counts, Hkv, Hkv, d, B, seed=1)
    moves, lens = so.compact(accepted.tolist(), held, [h + n for h, n in zip(held, counts)])
    for width in (64, 13, 0):
        k, v = torch.nan_to_num(c.k, nan=5.0, posinf=6.0).cuda(), torch.nan_to_num(c.v, nan=5.0, posinf=6.0).cuda()
        want = k.clone(), v.clone()
        acc = accepted[:, :width]
        moves, lens = so.compact(acc.tolist(), held, [h + n for h, n in zip(held, counts)])
        src = [(int(c.table[b, x // B]), x % B) for b, x, _ in moves]
        dst = [(int(c.table[b, y // B]), y % B) for b, _, y in moves]
        for old, new in zip((k, v), want):
            for (p, o), (p2, o2) in zip(src, dst):
                new[p2, :, o2] = old[p, :, o]
        got = bf1.kv_compact(k, v, i32(acc), i32(held), i32([h + n for h, n in zip(held, counts)]), i32(c.table))
        assert got.tolist() == lens and torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_kv_compact_missing_pages_buffers_and_refusals():
    B = 64
    c = Case([60], [10], 2, 2, 64, B, seed=2)
    k, v = (torch.nan_to_num(x, nan=1.0, posinf=2.0).cuda() for x in (c.k, c.v))
    table = i32(c.table)
    table[0, 1] = -1  # nodes 4.. have no page: rows from there and to there are left out
    want = k.clone()
    p = int(c.table[0, 0])
    want[p, :, 61] = k[p, :, 63]
    out = i32([0])
    got = bf1.kv_compact(k, v, i32([[0, 3, 5, 6, 7, 8, 9]]), i32([60]), i32([70]), table, out=out)
    assert got is out and out.tolist() == [67] and torch.equal(k, want)
    ok = dict(k_pages=k, v_pages=v, accepted=i32([[0]]), lens_before=i32([60]), seq_lens=i32([70]), page_table=table)
    a = bf1.kv_compact(**ok, stream=torch.cuda.current_stream())
    assert a.tolist() == [61]
    for bad, why in [(dict(accepted=i32([0])), "accepted"), (dict(accepted=i32([[0], [0]])), "accepted"),
                     (dict(seq_lens=i32([70, 1])), "seq_lens"), (dict(page_table=i32([1])), "page_table"),
                     (dict(v_pages=v.float()), "v_pages"), (dict(out=i32([1, 2])), "out")]:
        with pytest.raises(ValueError, match=why):
            bf1.kv_compact(**{**ok, **bad})
    with pytest.raises(bf1.BF1Error):
        bf1.kv_compact(**{**ok, "accepted": torch.zeros((1, 65), dtype=torch.int32, device="cuda")})
    with pytest.raises(bf1.BF1Error):
        bf1.kv_compact(**ok, out=ok["lens_before"])


def test_caches_past_32_bits():
    """Pages behind 2^32 elements: attention, moved rows and copies there as at the front."""
    Hkv, d, B, P = 8, 128, 64, 66000  # 4.3e9 elements each
    k, v = (torch.empty((P, Hkv, B, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c = Case([500, 70], [9, 6], 16, Hkv, d, B, seed=21, spare=0)
    n = c.k.shape[0]
    k[P - n:], v[P - n:] = torch.nan_to_num(c.k, nan=9.0, posinf=9.0).cuda(), torch.nan_to_num(c.v, nan=9.0, posinf=9.0).cuda()
    far = np.where(c.table < 0, c.table, c.table + P - n)
    args = signed(c.masks), i32(c.pos), i32(c.held), i32(c.start)
    got = bf1.attn_tree(c.q.cuda(), k, v, *args, i32(far))
    c.check(got)
    front = k[P - n:].clone(), v[P - n:].clone()
    acc, lens, after = i32([[0, 3, 8], [1, 2, -1]]), i32(c.held), i32([509, 76])
    a = bf1.kv_compact(k, v, acc, lens, after, i32(far))
    b = bf1.kv_compact(*front, acc, lens, after, i32(c.table))
    assert torch.equal(a, b) and torch.equal(k[P - n:], front[0]) and torch.equal(v[P - n:], front[1])
    bf1.kv_copy(k, v, i32([P - 1, P - 2]), i32([P - n - 1, 0]), i32([64, 33]))
    assert torch.equal(k[P - n - 1], k[P - 1]) and torch.equal(v[0, :, :33], v[P - 2, :, :33])

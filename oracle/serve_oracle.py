"""Plain definitions of the operators around speculative and parallel decoding, in float64
and integers on the CPU, written row by row and place by place (test infrastructure only)."""

import numpy as np

from .cache_oracle import rope


def norm_rope(x, gain, positions, freqs, interleaved, amplitude, eps):
    """x [..., n, d] float64; gain [d]; positions broadcastable to x's leading sizes."""
    x = np.asarray(x, dtype=np.float64)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return rope(x * r * gain, positions, freqs, interleaved, amplitude)


def norm_rope_bwd(dy, x, gain, positions, freqs, interleaved, amplitude, eps):
    """(dx, the rows' shares [..., n, d] of the gain's gradient)."""
    x = np.asarray(x, dtype=np.float64)
    dn = rope(dy, positions, freqs, interleaved, amplitude, -1)
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    u, n = dn * gain, x * r
    return r * (u - n * (u * n).mean(-1, keepdims=True)), dn * n


def tree_step(parents, token_start, before, after):
    """(masks, positions) of the packed rows; masks as Python ints."""
    rows = len(parents)
    masks, pos = [0] * rows, [-1] * rows
    for b in range(len(before)):
        start = token_start[b]
        for i in range(min(token_start[b + 1] - start, after[b] - before[b], 64)):
            p = parents[start + i]
            up = p if 0 <= p < i else None
            masks[start + i] = (1 << i) | (masks[start + up] if up is not None else 0)
            pos[start + i] = before[b] + bin(masks[start + i]).count("1") - 1
    return masks, pos


def route(j, L):
    """P(j) without j."""
    return sorted({i for i in {0} | set(range(j - L, j)) | {j - 2 ** r for r in range(2, 40)} if 0 <= i < j})


def tree_keys(b, r, masks, positions, before, token_start, B, L, dense, most=64):
    """Positions in the cache that row r of sequence b reads; None if it has no place."""
    start, held = token_start[b], before[b]
    count = min(token_start[b + 1] - start, most)

    def placed(i):
        return i < count and held <= positions[start + i] < held + 64

    if not placed(r - start):
        return None
    j = positions[r] // B
    blocks = (list(range(j)) if dense else route(j, L)) + [j]
    keys = [p for i in blocks for p in range(i * B, min((i + 1) * B, held))]
    for i in range(64):
        if masks[r] >> i & 1 and placed(i):
            ka = positions[start + i] // B
            if dense or ka == j or min(ka, j) in route(max(ka, j), L):
                keys.append(held + i)
    return keys


def attend(q, keys, values):
    """One head over keys [n, d]: (o, lse, mass); zeros and -inf over nothing."""
    if len(keys) == 0:
        return np.zeros(q.shape[0]), -np.inf, np.zeros(q.shape[0])
    s = keys @ q / np.sqrt(q.shape[0])
    m = s.max()
    p = np.exp(s - m)
    l = p.sum()
    return p @ values / l, m + np.log(l), p @ np.abs(values) / l


def compact(accepted, before, after):
    """Moves [(sequence, from position, to position)] and the new lengths."""
    moves, lens = [], []
    for b, row in enumerate(accepted):
        last, n = -1, 0
        for k, node in enumerate(row):
            if node <= last or node >= min(after[b] - before[b], 64):
                break
            moves.append((b, before[b] + node, before[b] + k))
            last, n = node, k + 1
        lens.append(before[b] + n)
    return moves, lens


def page_fork(lens, sources, keep, table, shares, free, head, B):
    """One place after the other; returns (table, lens, head, shares, free, copies), copies
    [(from, to, rows)] per place, (-1, -1, 0) without one."""
    nb, width, pages = len(lens), len(table[0]) if len(table) else 0, len(shares)
    lens = [min(max(int(x), 0), width * B) for x in lens]
    refs = [int(x) + 1 for x in shares]
    touched = set()
    n = []
    for b in range(nb):
        s = sources[b]
        n.append(min(max(int(keep[b]), 0), lens[s]) if 0 <= s < nb else 0)
    for b in range(nb):
        for i in range(-(-lens[b] // B)):
            p = table[b][i]
            if 0 <= p < pages:
                refs[p] -= 1
                touched.add(p)
    for b in range(nb):
        for i in range(n[b] // B):
            p = table[sources[b]][i]
            if 0 <= p < pages:
                refs[p] += 1
    new = [[-1] * width for _ in range(nb)]
    copies = []
    free = list(free)
    head = min(max(int(head), 0), len(free))
    asked = head
    for b in range(nb):
        full, rows = n[b] // B, n[b] % B
        for i in range(full):
            new[b][i] = table[sources[b]][i]
        copies.append((-1, -1, 0))
        if rows == 0:
            continue
        p = table[sources[b]][full]
        new[b][full] = p
        if not 0 <= p < pages:
            continue
        if refs[p] <= 0:
            refs[p] = 1
        elif asked < len(free):
            new[b][full] = free[asked]
            copies[b] = (p, free[asked], rows)
            asked += 1
        else:
            new[b][full] = -1
            n[b] -= rows
    freed = sorted(p for p in touched if refs[p] <= 0)
    start = max(asked - len(freed), 0)
    for i, p in enumerate(freed):
        if start + i < asked:
            free[start + i] = p
    return new, n, start, [max(x - 1, 0) for x in refs], free, copies

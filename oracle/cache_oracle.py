"""Plain definitions of the operators around a served sequence's cache, in float64
and integers on the CPU, written token by token (test infrastructure only)."""

import numpy as np


def page_step(seq_lens, new_lens, page_table, free_pages, head, max_tokens, B):
    """One token after the other; returns (table, lens, token_start, block_start,
    positions, slots, head)."""
    table = np.array(page_table, dtype=np.int64)
    F = len(free_pages)
    head = min(max(int(head), 0), F)
    lens, tstart, bstart = [], [0], [0]
    pos = np.full(max_tokens, -1, dtype=np.int64)
    slots = np.full(max_tokens, -1, dtype=np.int64)
    asked = head  # where the sequence's pages would start, had all before it got theirs
    taken = 0
    for b in range(len(seq_lens)):
        old, want = max(int(seq_lens[b]), 0), max(int(new_lens[b]), 0)
        first = tstart[-1]
        n, blocks = 0, set()
        full = False
        for i in range(want):
            p = old + i
            if p >= table.shape[1] * B or p >= 2 ** 31 - 1 or first + i >= max_tokens:
                break
            if p % B == 0:  # a block's first token takes a page
                if asked >= F:
                    full = True
                if not full:
                    table[b, p // B] = free_pages[asked]
                    taken += 1
                asked += 1
            if full:
                continue  # its pages are still counted as asked for
            page = int(table[b, p // B])
            pos[first + i] = p
            slots[first + i] = page * B + p % B if page >= 0 else -1
            blocks.add(p // B)
            n += 1
        lens.append(old + n)
        tstart.append(first + want)
        bstart.append(bstart[-1] + len(blocks))
    return table, np.array(lens), np.array(tstart), np.array(bstart), pos, slots, head + taken


def rope(x, positions, freqs, interleaved, amplitude, sign=1):
    """x [..., n, d] float64, positions [n] or broadcastable to x's leading sizes;
    angles in extended precision, so that far positions are exact."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    r2 = len(freqs)
    for i in range(r2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r2)
        ang = np.asarray(positions, dtype=np.longdouble) * np.longdouble(freqs[i])
        c = np.asarray(amplitude * np.cos(ang), dtype=np.float64)
        s = np.asarray(sign * amplitude * np.sin(ang), dtype=np.float64)
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def e4m3_values():
    """The 256 numbers of the 1-4-3 format (bias 7, no infinities)."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        if e == 15 and m == 7:
            v = np.nan
        out[c] = -v if c & 128 else v
    return out


E4M3 = e4m3_values()
_POS = E4M3[:127]  # 0 .. 448, ascending


def to_e4m3(y):
    """Codes (uint8) nearest to y, |y| <= 448, ties to the even code."""
    a = np.abs(y)
    hi = np.searchsorted(_POS, a)           # first entry >= a
    hi = np.minimum(hi, 126)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def quantise(block, fmt):
    """(codes, scale) of one block of one kv-head: codes uint8 (e4m3) or int8, scale
    a float32."""
    x = np.asarray(block, dtype=np.float64)
    empty = np.zeros(x.shape, dtype=np.uint8 if fmt == "e4m3" else np.int8)
    if not np.isfinite(x).all():
        return empty, np.float32(np.nan)
    a = np.abs(x).max()
    if a < 2.0 ** -100:
        return empty, np.float32(1)
    if fmt == "e4m3":
        e = -300
        while a > 448 * 2.0 ** e:
            e += 1
        return to_e4m3(x / 2.0 ** e), np.float32(2.0 ** e)
    return np.rint(127 * x / a).astype(np.int8), np.float32(a / 127)


def dequantise(codes, scale, fmt):
    c = E4M3[np.asarray(codes, dtype=np.uint8)] if fmt == "e4m3" else np.asarray(codes, dtype=np.float64)
    return c * float(scale)


def append_q8(k, v, before, after, token_start, page_table, cache, fmt, B):
    """The cache (dict of float64 / code arrays, as the tensors lie) after a step,
    token by token through each sequence's newest block."""
    out = {n: a.copy() for n, a in cache.items()}
    for b in range(len(before)):
        for i in range(int(after[b]) - int(before[b])):
            p, row = int(before[b]) + i, int(token_start[b]) + i
            for name, x in (("k", k), ("v", v)):
                out[name + "_tail"][b, :, p % B] = x[row]
            if p % B == B - 1:  # the block is complete
                page = int(page_table[b, p // B])
                for name in ("k", "v"):
                    for h in range(k.shape[1]):
                        codes, scale = quantise(out[name + "_tail"][b, h], fmt)
                        out[name + "_pages"][page, h] = codes if name == "k" else codes.T
                        out[name + "_scale"][page, h] = scale
    # rows of the tail that do not belong to the newest block keep what they had
    for b in range(len(before)):
        if after[b] > before[b]:
            last = (int(after[b]) - 1) // B * B
            for r in range(B):
                if not int(before[b]) <= last + r < int(after[b]):
                    for name in ("k", "v"):
                        out[name + "_tail"][b, :, r] = cache[name + "_tail"][b, :, r]
    return out


def decode(q, keys, values):
    """One head's softmax over keys [n, d], values [n, d]: (o, lse, mass) with mass =
    sum of p |v|, what roundings of weights scale with."""
    s = keys @ q / np.sqrt(q.shape[0])
    m = s.max()
    p = np.exp(s - m)
    l = p.sum()
    return p @ values / l, m + np.log(l), p @ np.abs(values) / l

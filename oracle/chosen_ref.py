"""CPU oracle for attention over chosen pages: digests, scores, choices, and the maps of a ragged batch, written out token by token.

TEST INFRASTRUCTURE ONLY, like the rest of oracle/.  Whole numbers are Python integers or int64; the one thing in 32 bits is the sum of queries over the heads
that share a kv head, which is defined there.

    digest   hi = sat8(ceil(max_t K_t 2^-e)), lo = sat8(floor(min_t K_t 2^-e)); a channel with a key that is no number: 127, -128
    score    sum_d p_d hi_d + n_d lo_d, p and n the codes of the queries' positive and negative parts
    choice   of the pages 0 .. o that are there the first, the last, and the highest scores, equal ones from the lowest page on
"""
import math

import numpy as np


def digest(keys, exponents):
    """keys [H, n, D] of one full page, exponents [H, D].  int8 [H, 2, D]."""
    H, n, D = keys.shape
    got = np.zeros((H, 2, D), dtype=np.int8)
    for h in range(H):
        for d in range(D):
            column, e = [float(x) for x in keys[h, :, d]], int(exponents[h, d])
            if any(math.isnan(x) for x in column):
                got[h, :, d] = 127, -128
                continue
            top, low = max(column), min(column)

            def scaled(x):
                if math.isinf(x):
                    return x
                try:
                    return math.ldexp(x, -e)                 # doubles reach far beyond what 16-bit values and int8 exponents need
                except OverflowError:
                    return math.copysign(math.inf, x)

            hi, lo = scaled(top), scaled(low)
            hi = hi if math.isinf(hi) else math.ceil(hi)
            lo = lo if math.isinf(lo) else math.floor(lo)
            got[h, 0, d], got[h, 1, d] = max(-128, min(127, hi)), max(-128, min(127, lo))
    return got


def codes(q, exponents):
    """q [R, D] float32, exponents [D].  Integers p [D], n [D]."""
    R, D = q.shape
    above, below = np.zeros(D, dtype=np.float32), np.zeros(D, dtype=np.float32)
    most = np.finfo(np.float32).max
    with np.errstate(all="ignore"):
        for r in range(R):
            x = np.where(np.isnan(q[r]), np.float32(0), q[r]).astype(np.float32)
            above, below = (above + np.maximum(x, 0)).astype(np.float32), (below + np.minimum(x, 0)).astype(np.float32)
    above, below = np.minimum(above, most), np.maximum(below, -most)
    heights = [math.frexp(max(float(above[d]), -float(below[d])))[1] - 1 + int(exponents[d]) for d in range(D) if above[d] > 0 or below[d] < 0]
    p, n = np.zeros(D, dtype=np.int64), np.zeros(D, dtype=np.int64)
    if heights:
        x = max(heights)
        for d in range(D):
            by = int(exponents[d]) - x + 6
            p[d] = min(127, round(math.ldexp(float(above[d]), by)))          # Python rounds halves to even
            n[d] = max(-127, round(math.ldexp(float(below[d]), by)))
    return p, n


def choose(q, place, size, entries, pages, digests, exponents, most, first, last):
    """One query token and kv head: q [R, D], entries of its row, digests [pages, 2, D].  The set of page numbers of the sequence."""
    if place < 0:
        return set()
    o = place // size
    there = [j for j in range(o + 1) if 0 <= entries[j] < pages]
    always = [j for j in there if j < first or j > o - last]
    p, n = codes(q, exponents)
    rest = [j for j in there if j not in set(always)]
    score = {j: int(p @ digests[entries[j], 0].astype(np.int64) + n @ digests[entries[j], 1].astype(np.int64)) for j in rest}
    rest.sort(key=lambda j: (-score[j], j))
    return set(always) | set(rest[: max(0, most - len(always))])


def words(chosen, row_pages):
    got = np.zeros((row_pages + 31) // 32, dtype=np.uint32)
    for j in chosen:
        got[j // 32] |= np.uint32(1 << (j % 32))
    return got


def slots(more, lens, table, pages, size, tokens):
    """starts, row, place, slot as lists; 0x20 / 0x10 for numbers that may not be and entries that name no page."""
    status, starts, row, place, slot = 0, [0], [], [], []
    full = False
    for b, n in enumerate(lens):
        count = (1 if n else 0) if more is None else more[b]
        if count < 0 or count > n:
            status, count = status | 0x20, 0
        if full or starts[-1] + count > tokens:
            full, status, count = True, status | 0x20, 0
        starts.append(starts[-1] + count)
        for p in range(n - count, n):
            page = table[b][p // size]
            row.append(b)
            place.append(p)
            if 0 <= page < pages:
                slot.append(page * size + p % size)
            else:
                slot.append(-1)
                status |= 0x10
    behind = [-1] * (tokens - len(row))
    return starts, row + behind, place + behind, slot + behind, status

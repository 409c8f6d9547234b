"""Oracle of the cache in pages (include/vico_pages.h): the page table's operations entry by entry on
Python lists, and attention over pages in float64, sequence by sequence.

Test infrastructure; shares no code with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np


def pages_of(tokens: int, page: int) -> int:
    return -(-tokens // page)


def _valid(e: int, refs) -> bool:
    return 0 <= e < len(refs)


def fork(table, refs, seq_len, parent, page):
    """New (table, refs, seq_len) after the rows have been taken from their parents."""
    rows = len(table)
    new, ref, length = [list(r) for r in table], list(refs), list(seq_len)
    for b in range(rows):
        p = parent[b]
        if p == b or p < -1 or p >= rows:
            continue
        keep = 0 if p < 0 else pages_of(max(seq_len[p], 0), page)
        new[b] = [table[p][j] if p >= 0 and j < keep and _valid(table[p][j], refs) else -1 for j in range(len(table[b]))]
        length[b] = 0 if p < 0 else seq_len[p]
        for old, e in zip(table[b], new[b]):
            if _valid(old, refs):
                ref[old] -= 1
            if e >= 0:
                ref[e] += 1
    return new, ref, length


def free(table, refs, first, last, page):
    new, ref = [list(r) for r in table], list(refs)
    for b, row in enumerate(new):
        for j in range(len(row)):
            if j * page >= max(first[b], 0) and (j + 1) * page <= last[b]:
                if _valid(row[j], refs):
                    ref[row[j]] -= 1
                row[j] = -1
    return new, ref


def reserve(table, refs, seq_len, q_start, page):
    """(table, refs, moves, granted) after every row has pages of its own for its new tokens."""
    new, ref = [list(r) for r in table], list(refs)
    unused = [p for p, c in enumerate(refs) if c <= 0]
    moves, granted, short = [], [], False
    for b, row in enumerate(new):
        H, n = max(seq_len[b], 0), q_start[b + 1] - q_start[b]
        moves.append([-1, -1])
        if n <= 0:
            granted.append(1)
            continue
        if pages_of(H + n, page) > len(row):
            granted.append(0)
            continue
        want = [j for j in range(H // page, pages_of(H + n, page)) if not (_valid(row[j], refs) and refs[row[j]] == 1)]
        if want:
            short = short or len(want) > len(unused)
        granted.append(0 if want and short else 1)
        for j in want if granted[b] else []:
            old, row[j] = row[j], unused.pop(0)
            ref[row[j]] = 1
            if _valid(old, refs) and refs[old] > 0:
                ref[old] -= 1
                if j == H // page and H % page:
                    moves[b] = [old, row[j]]
    return new, ref, moves, granted


def compact(table, refs, max_moves):
    used = sum(c > 0 for c in refs)
    src = [p for p in range(used, len(refs)) if refs[p] > 0]
    dst = [p for p in range(used) if refs[p] <= 0]
    assert len(src) == len(dst)
    ref, to = list(refs), dict(zip(src, dst))
    for s, d in to.items():
        ref[d], ref[s] = refs[s], 0
    new = [[to.get(e, e) for e in row] for row in table]
    moves = [[s, d] for s, d in to.items()]
    return new, ref, moves + [[-1, -1]] * (max_moves - len(moves)), len(moves)


def visible(row, H, n, i, page, num_pages, sink, window, bidirectional):
    """Positions that row i of a sequence sees: those that the mask leaves and that have a page."""
    last = min(H + (n - 1 if bidirectional else i), len(row) * page - 1)
    lo = 0 if window < 0 else max(H - window, 0)
    return [p for p in list(range(min(sink, lo))) + list(range(lo, last + 1)) if 0 <= row[p // page] < num_pages]


def paged_attention(q, q_start, seq_len, k_pages, v_pages, table, sink=0, window=-1, bidirectional=False, scale=None,
                    max_q=None, bound=None):
    """(out [rows, Hq, d], lse [Hq, rows], covered [rows]) in float64; out is 0 and lse -inf for a row without keys.

    bound: called for every sequence and KV head with (rows, heads, K and V of the keys that some row sees, p)."""
    N, page, Hkv, d = k_pages.shape
    rows, Hq, _ = q.shape
    g, s = Hq // Hkv, (1.0 / math.sqrt(d) if scale is None else scale)
    out, lse, covered = np.zeros((rows, Hq, d)), np.full((Hq, rows), -np.inf), np.zeros(rows, bool)
    for b, row in enumerate(table):
        n = q_start[b + 1] - q_start[b]
        m = n if max_q is None else min(n, max_q)
        rs = slice(q_start[b], q_start[b] + m)
        covered[rs] = True
        pos = np.array(visible(row, seq_len[b], n, n - 1, page, N, sink, window, bidirectional), dtype=np.int64) if m else []
        if len(pos) == 0:
            continue
        ids = np.array(row)[pos // page]
        K, V = k_pages[ids, pos % page], v_pages[ids, pos % page]            # [keys, Hkv, d]
        seen = pos[None] <= seq_len[b] + (np.full(m, n - 1) if bidirectional else np.arange(m))[:, None]
        some = seen.any(1)
        for h in range(Hkv):
            for hq in range(h * g, (h + 1) * g):
                z = np.where(seen, s * (q[rs, hq] @ K[:, h].T), -np.inf)
                top = np.where(some, z.max(1), 0.0)[:, None]
                p = np.exp(z - top)
                total = p.sum(1, keepdims=True)
                p /= np.where(total > 0, total, 1.0)
                out[rs, hq] = p @ V[:, h]
                lse[hq, rs] = np.where(some, top[:, 0] + np.log(np.where(total > 0, total, 1.0))[:, 0], -np.inf)
                if bound is not None:
                    bound(rs, hq, K[:, h], V[:, h], p)
    return out, lse, covered

"""Steps of the cache in pages as a program repeats them: captured calls replayed with other lengths and tables, both
paths of the binding, arrays that make no sense beside guarded memory, histories and pools that are long."""
from __future__ import annotations

import random

import numpy as np
import pytest
import torch

import paper_2606_19849_amd as vico
import paper_2606_19849_amd._binding as binding
from oracle import pages
from tests._pages import DEV, Cache, check, i32
from tests._route import paged_route
from tests.test_gpu_pages import bits, capture, random_state

pytestmark = pytest.mark.gpu

H128, H7B, WIDE, SMALL = (4, 2, 128), (28, 4, 128), (18, 2, 128), (17, 1, 64)
G = 4096                                      # elements of a margin


class Guarded:
    """A tensor inside a larger one whose other elements hold a pattern."""

    def __init__(self, t):
        self.raw = torch.full((t.numel() + 2 * G,), 77, dtype=t.dtype, device=DEV)
        self.t = self.raw[G:G + t.numel()].view(t.shape)
        self.t.copy_(t)

    def intact(self):
        return bool(torch.all(self.raw[:G] == 77)) and bool(torch.all(self.raw[G + self.t.numel():] == 77))


# ---------------------------------------------------------------- replays

def variants(seed, rows, heads, N, width, page, mask, *lists):
    """Caches of the same sizes (rows of q, pool, table) with other sequences."""
    out = []
    for i, seqs in enumerate(lists):
        used = sum(pages.pages_of(n + H, page) for n, H in seqs)
        out.append(Cache(seed + i, seqs, heads=heads, page=page, width=width, spare=N - used, pad=rows - sum(n for n, _ in seqs), **mask))
        assert out[-1].k.shape[0] == N and out[-1].q.shape[0] == rows and len(out[-1].table[0]) == width
    return out


@pytest.mark.parametrize("heads,rows,lists", [
    (WIDE, 260, ([(150, 77), (1, 90), (1, 1)], [(1, 300), (70, 0), (0, 33)], [(0, 5), (0, 0), (260, 40)], [(60, 1), (60, 400), (60, 64)],
                 [(1, 2), (1, 200), (1, 450)])),
    (H128, 40, ([(20, 60), (3, 200)], [(1, 500), (1, 0)], [(0, 9), (40, 130)], [(8, 0), (9, 31)])),
    (H7B, 200, ([(200, 100)], [(1, 600)], [(17, 0)], [(0, 50)], [(150, 333)])),
], ids=["mixed", "rows", "one"])
@pytest.mark.parametrize("splits", [0, 3])
def test_a_captured_step_replays_with_other_lengths(heads, rows, lists, splits):
    """Append and attention: sequences change their class of rows between replays, start empty and grow long."""
    mask = dict(sink=9, window=150)
    cs = variants(40, rows, heads, 90, 42, 16, mask, *lists)
    at = {n: getattr(cs[0].device(), n).clone() for n in ("dk", "dv", "dq", "dt", "ds", "dl")}
    k, v = (torch.zeros(rows, heads[1], heads[2], dtype=torch.bfloat16, device=DEV) for _ in "kv")
    out, lse = torch.empty(rows, heads[0], heads[2], device=DEV), torch.empty(heads[0], rows, device=DEV)
    parts, wb = vico.vico_paged_attn_plan(len(lists[0]), rows, rows, 16, 42, 9, 150, 0, *heads, splits)
    ws = torch.full((wb + 256,), 255, dtype=torch.uint8, device=DEV)

    def body():
        vico.vico_paged_append(k, v, at["ds"], at["dl"], at["dk"], at["dv"], at["dt"])
        vico.vico_paged_attn(at["dq"], at["ds"], at["dl"], at["dk"], at["dv"], at["dt"], out, lse=lse, sink_len=9, window=150,
                             max_q_len=rows, num_splits=splits, workspace=ws)

    g = capture(body)
    for c in cs + cs[::-1]:
        c.device()
        # the new tokens are not in their pages before the step
        k.zero_()
        v.zero_()
        pool_k, pool_v = c.dk.clone(), c.dv.clone()
        for b, n in enumerate(c.n):
            for j in range(n):
                page, place = c.place(b, c.H[b] + j)
                k[c.q_start[b] + j], v[c.q_start[b] + j] = c.dk[page, place], c.dv[page, place]
                pool_k[page, place], pool_v[page, place] = float("nan"), float("nan")
        for name in at:
            at[name].copy_({"dk": pool_k, "dv": pool_v}.get(name, getattr(c, name)))
        out.fill_(7.25)
        lse.fill_(7.25)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for got, want in ((at["dk"], c.dk), (at["dv"], c.dv)):
            assert torch.equal(torch.isnan(got), torch.isnan(want))
            assert torch.equal(bits(got.nan_to_num()), bits(want.nan_to_num()))
        c.parts = parts
        check(c, (out, lse), c.oracle())
        assert torch.all(ws[wb:] == 255)
        check(c, c.attention(splits=splits), c.oracle())       # eager work between the replays
        # the same call, not captured, bit for bit
        first = out.clone(), lse.clone()
        body()
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.int32), y.view(torch.int32)) for x, y in zip(first, (out, lse)))


@pytest.mark.parametrize("rows,page,N,width", [(7, 16, 120, 20), (65, 16, 2500, 70), (130, 16, 70000, 600)])
def test_captured_table_calls_replay_with_other_tables(rows, page, N, width):
    """Fork, reserve with its copies, free, compaction with its copies, each replay on another table and other lengths; the
    pages that moved are compared bit for bit in every layer."""
    Hkv, D, layers = 1, 64, 2
    g = torch.Generator(device=DEV)
    g.manual_seed(N)
    k0, v0 = (torch.randint(-2 ** 15, 2 ** 15, (layers, N, page, Hkv, D), generator=g, device=DEV, dtype=torch.int16).view(torch.bfloat16)
              for _ in "kv")
    k, v = k0.clone(), v0.clone()
    zeros = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)   # noqa: E731
    table, refs, lens, parent, starts = zeros(rows, width), zeros(N), zeros(rows), zeros(rows), zeros(rows + 1)
    first, last, granted, count = zeros(rows), zeros(rows), zeros(rows), zeros(1)
    moves, packed = zeros(rows, 2), zeros(N // 2, 2)
    ws = torch.full((vico.vico_pages_workspace_bytes(rows, N),), 171, dtype=torch.uint8, device=DEV)

    def body():
        vico.vico_pages_fork(table, refs, lens, parent, page)
        vico.vico_pages_reserve(table, refs, lens, starts, page, moves, granted, ws)
        vico.vico_pages_copy(k, v, moves)
        vico.vico_pages_free(table, refs, first, last, page)
        vico.vico_pages_compact(table, refs, packed, count, ws)
        vico.vico_pages_copy(k, v, packed, count=count)

    graph = capture(body)
    for seed in range(4):
        r = random.Random(seed * 100 + rows)
        t, f, s = random_state(seed * 7 + rows, rows, page, N, width, most=0.6)
        p = [r.choice([b, b, -1, r.randrange(rows)]) for b in range(rows)]
        q = np.cumsum([seed] + [r.choice([0, 1, r.randint(0, 5 * page)]) for _ in range(rows)]).tolist()
        lo, hi = [r.randrange(4 * page) for _ in range(rows)], [r.randrange(width * page) for _ in range(rows)]
        for dst, src in ((table, t), (refs, f), (lens, s), (parent, p), (starts, q), (first, lo), (last, hi)):
            dst.copy_(i32(src))
        k.copy_(k0)
        v.copy_(v0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        t, f, s = pages.fork(t, f, s, p, page)
        t, f, m, ok = pages.reserve(t, f, s, q, page)
        t, f = pages.free(t, f, lo, hi, page)
        t, f, c, n = pages.compact(t, f, N // 2)
        assert table.tolist() == t and refs.tolist() == f and lens.tolist() == s
        assert moves.tolist() == m and granted.tolist() == ok and packed.tolist() == c and count.item() == n
        wk, wv = k0.clone(), v0.clone()
        for pairs in ([x for x in m if x[0] >= 0], c[:n]):
            if pairs:
                src, dst = torch.tensor(pairs, device=DEV).T
                wk[:, dst], wv[:, dst] = wk[:, src], wv[:, src]
        assert torch.equal(bits(k), bits(wk)) and torch.equal(bits(v), bits(wv))


# ---------------------------------------------------------------- arrays that make no sense

BIG = 2 ** 31 - 1
STARTS = [[-5, 3, 7], [0, 100, 2000], [6, 3, 1], [0, BIG, -BIG - 1], [0, 9, 0], [2, 2, 9]]
LENGTHS = [[-4, BIG], [BIG, -BIG - 1], [30, 70]]


@pytest.mark.parametrize("heads,rows", [(H128, 9), (WIDE, 140)], ids=str)
@pytest.mark.parametrize("lens", LENGTHS, ids=str)
@pytest.mark.parametrize("starts", STARTS, ids=str)
def test_numbers_outside_every_range(starts, lens, heads, rows):
    """Starts and lengths as the calls bring them into range: what is computed, what stays as it was, and no write beside."""
    seqs = [(3, 20), (4, 90)]
    c = Cache(18, seqs, heads=heads, page=16, pad=rows - 7, spare=5, width=9)
    g = torch.Generator()
    g.manual_seed(2)
    c.k, c.v = (torch.randn(c.k.shape, generator=g).to(torch.bfloat16) for _ in "kv")
    c.device()
    N, cap = c.k.shape[0], c.width * 16
    # the rows of each sequence, and its length
    q0 = [min(max(x, 0), rows) for x in starts[:2]]
    n = [min(max(x, a), rows) - a for a, x in zip(q0, starts[1:])]
    H = [min(max(x, 0), cap) for x in lens]
    new_k, new_v = (torch.randn(rows, heads[1], heads[2], generator=g).to(torch.bfloat16).to(DEV) for _ in "kv")
    ds, dl = i32(starts), i32(lens)

    pools = [Guarded(x) for x in (c.dk, c.dv)]
    want = [x.clone() for x in (c.dk, c.dv)]
    for b in range(2):
        for j in range(n[b]):
            pos = max(lens[b], 0) + j
            if pos < cap and 0 <= c.table[b][pos // 16] < N:
                for w, x in zip(want, (new_k, new_v)):
                    w[c.table[b][pos // 16], pos % 16] = x[q0[b] + j]
    vico.vico_paged_append(new_k, new_v, ds, dl, pools[0].t, pools[1].t, c.dt)
    # (of starts that decrease, which the call does not know, rows may go nowhere: places hold what they did or that)
    known = starts == sorted(starts)
    for x, w, before in zip(pools, want, (c.dk, c.dv)):
        same = bits(x.t) == bits(w)
        assert x.intact() and torch.all(same if known else same | (bits(x.t) == bits(before)))

    for splits in (0, 1, 4):
        out, lse = Guarded(torch.full((rows, heads[0], heads[2]), 7.25)), Guarded(torch.full((heads[0], rows), 7.25))
        c.parts, wb = vico.vico_paged_attn_plan(2, rows, rows, 16, c.width, 0, -1, 0, *heads, splits)
        ws = Guarded(torch.full((max(wb, 1),), 255, dtype=torch.uint8))
        vico.vico_paged_attn(c.dq, ds, dl, c.dk, c.dv, c.dt, out.t, lse=lse.t, max_q_len=rows, num_splits=splits, workspace=ws.t)
        assert out.intact() and lse.intact() and ws.intact()
        covered = np.zeros(rows, bool)
        for b in range(2):
            covered[q0[b]:q0[b] + n[b]] = True
        assert torch.all(out.t[torch.tensor(~covered)] == 7.25) and torch.all(lse.t[:, torch.tensor(~covered)] == 7.25)
        for b in range(2):                      # each sequence for itself, its rows as a call of their own
            if n[b] == 0:
                continue
            one = Cache(18, [(n[b], 0)], heads=heads, page=16, pad=0, width=9)
            one.k, one.v, one.table, one.H, one.parts = c.k, c.v, [c.table[b]], [H[b]], c.parts
            one.q = c.q[q0[b]:q0[b] + n[b]]
            check(one, (out.t[q0[b]:q0[b] + n[b]].clone(), lse.t[:, q0[b]:q0[b] + n[b]].clone()), one.oracle())

    counts = [sum(e == p for row in c.table for e in row) for p in range(N)]
    table, refs, moves, granted, ln = (Guarded(i32(x)) for x in (c.table, counts, [[9, 9]] * 2, [9, 9], lens))
    ws = Guarded(torch.full((vico.vico_pages_workspace_bytes(2, N),), 171, dtype=torch.uint8))
    vico.vico_pages_reserve(table.t, refs.t, dl, ds, 16, moves.t, granted.t, ws.t)
    want = pages.reserve(c.table, counts, lens, starts, 16)
    assert (table.t.tolist(), refs.t.tolist(), moves.t.tolist(), granted.t.tolist()) == tuple(want)
    vico.vico_pages_fork(table.t, refs.t, ln.t, i32([1, 0]), 16)
    forked = pages.fork(want[0], want[1], lens, [1, 0], 16)
    assert (table.t.tolist(), refs.t.tolist(), ln.t.tolist()) == tuple(forked)
    vico.vico_pages_free(table.t, refs.t, dl, ds[:2], 16)
    freed = pages.free(forked[0], forked[1], lens, starts, 16)
    assert (table.t.tolist(), refs.t.tolist()) == tuple(freed)
    assert all(x.intact() for x in (table, refs, moves, granted, ln, ws))


@pytest.mark.parametrize("splits", [0, 1, 4])
def test_rows_of_several_sequences_write_nothing_beside(splits):
    """Starts that go up and down: rows that several sequences have, more of them than the call has rows."""
    c = Cache(19, [(100, 30)] + [(0, 30)] * 9, heads=WIDE, page=16, pad=30).device()
    out, lse = Guarded(torch.full((130, 18, 128), 7.25)), Guarded(torch.full((18, 130), 7.25))
    _, wb = vico.vico_paged_attn_plan(10, 130, 130, 16, c.width, 0, -1, 0, *WIDE, splits)
    ws = Guarded(torch.full((max(wb, 1),), 255, dtype=torch.uint8))
    vico.vico_paged_attn(c.dq, i32([0, 100, 0, 100, 0, 100, 0, 100, 0, 100, 0]), c.dl, c.dk, c.dv, c.dt, out.t, lse=lse.t,
                         max_q_len=130, num_splits=splits, workspace=ws.t)
    assert out.intact() and lse.intact() and ws.intact() and torch.all(out.t[100:] == 7.25) and torch.all(lse.t[:, 100:] == 7.25)


# ---------------------------------------------------------------- both paths of the binding

class _Never:
    """Stands in for the C++ calls and takes none."""

    def __getattr__(self, name):
        return lambda *a: None


def everything(stream=None, clone=torch.clone):
    """A step through all seven calls; what they wrote.  clone: makes what the calls write from tensors of its values."""
    c = Cache(31, [(1, 90), (20, 47), (0, 40)], heads=H128, page=16, sink=8, window=60)
    g = torch.Generator()
    g.manual_seed(6)
    c.k, c.v = (torch.randn(c.k.shape, generator=g).to(torch.bfloat16) for _ in "kv")
    N = c.k.shape[0]
    c.table = [[e if 0 <= e < N else -1 for e in row] for row in c.table]
    c.device()
    counts = i32([sum(e == p for row in c.table for e in row) for p in range(N)])
    new = torch.randn(c.q.shape[0], 2, 128, generator=g).to(torch.bfloat16).to(DEV)
    k, v, table, refs, lens = (clone(x) for x in (c.dk, c.dv, c.dt, counts, c.dl))
    out, lse = clone(torch.full(c.q.shape, 7.25, device=DEV)), clone(torch.full((4, c.q.shape[0]), 7.25, device=DEV))
    moves, granted, packed, count = (clone(i32(x)) for x in ([[9, 9]] * 3, [9] * 3, [[9, 9]] * (N // 2), [9]))
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    vico.vico_paged_append(new, new, c.ds, lens, k, v, table, stream=stream)
    vico.vico_paged_attn(c.dq, c.ds, lens, k, v, table, out, lse=lse, sink_len=8, window=60, max_q_len=20, keys_hint=100,
                         num_splits=2, softmax_scale=0.11, flags=vico.VICO_ATTN_BIDIRECTIONAL, workspace=ws, stream=stream)
    vico.vico_pages_fork(table, refs, lens, i32([0, 1, 1]), 16, stream=stream)
    vico.vico_pages_reserve(table, refs, lens, i32([0, 4, 4, 30]), 16, moves, granted, ws, stream=stream)
    vico.vico_pages_copy(k, v, moves, stream=stream)
    vico.vico_pages_free(table, refs, i32([16, 0, 0]), i32([64, 0, 33]), 16, stream=stream)
    vico.vico_pages_compact(table, refs, packed, count, ws, stream=stream)
    vico.vico_pages_copy(k[None], v[None], packed, count=count, stream=stream)
    torch.cuda.synchronize()
    return c, (k, v, table, refs, lens, out, lse, moves, granted, packed, count)


@pytest.mark.parametrize("stream", ["current", "object", "handle"])
def test_both_paths_give_the_same(stream, monkeypatch):
    s = torch.cuda.current_stream() if stream == "current" else torch.cuda.Stream()
    arg = {"current": None, "object": s, "handle": s.cuda_stream}[stream]
    c, fast = everything(arg)
    assert not torch.equal(fast[2], c.dt) and int(fast[10]) > 0 and torch.any(fast[7] >= 0)      # something was forked and moved
    monkeypatch.setattr(binding, "_calls", _Never())
    for a, b in zip(fast, everything(arg)[1]):
        assert torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_lazily_cloned_outputs_get_memory_of_their_own():
    """Copy-on-write clones as what the calls write: the tensors that they were cloned from keep their values."""
    if not hasattr(torch, "_lazy_clone"):
        pytest.skip("no copy-on-write clones in this torch")
    kept = []

    def lazy(x):
        kept.append((x, x.clone()))
        return torch._lazy_clone(x)

    want = everything()[1]
    got = everything(clone=lazy)[1]
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(want, got))
    assert all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in kept)


# ---------------------------------------------------------------- long histories, large pools

@pytest.mark.parametrize("page", [16, 64, 512])
@pytest.mark.parametrize("seqs,heads", [([(1, 9000), (1, 4200)], H128), ([(5, 8500), (12, 13000)], H128), ([(1, 20000), (120, 30)], WIDE),
                                        ([(6, 19000), (132, 30)], (8, 1, 64))], ids=str)
def test_more_pages_a_part_than_a_wave_holds(seqs, heads, page):
    """A part of more than 32 blocks of every wave, pages missing in later ones, whole histories and windows."""
    drop = {(0, seqs[0][1] * 3 // 4 // page), (1, 4150 // page)}
    most, g = max(n for n, _ in seqs), heads[0] // heads[1]
    assert (paged_route(2, seqs[0][0] + seqs[1][0] + 2, most, page, 20100 // page + 2, 0, -1, 0, heads, 1)[0] > 0) == (most * g > 1024)
    for mask in ({}, dict(sink=4500, window=4300)):
        c = Cache(33, seqs, heads=heads, page=page, drop=drop, **mask).device()
        for splits in (1, 2):
            check(c, c.attention(splits=splits), c.oracle())


@pytest.mark.parametrize("page", [64, 1024])
def test_more_large_pages_a_part_than_the_table_in_lds_holds(page):
    """Over 131072 keys in one part of 256-row tiles, a page missing behind them."""
    c = Cache(34, [(69, 150000)], heads=(15, 1, 64), page=page, drop={(0, 140000 // page)}).device()
    assert c.q.shape[0] * 15 > 1024
    check(c, c.attention(splits=1), c.oracle())


@pytest.mark.parametrize("page", [16, 128])
def test_long_sinks(page):
    for seqs, heads in (([(1, 1500), (9, 2000)], H128), ([(60, 1900), (130, 1000)], WIDE), ([(1, 1400), (150, 1700)], SMALL)):
        for sink, window in ((700, 300), (1000, 1000), (1025, 0)):
            c = Cache(35, seqs, heads=heads, page=page, sink=sink, window=window).device()
            check(c, c.attention(), c.oracle())
            check(c, c.attention(splits=3), c.oracle())


@pytest.mark.parametrize("n", [1, 4, 20])
def test_few_rows_over_a_pool_past_the_32bit_offset_limit(n):
    page, Hkv, D, N = 1024, 4, 128, 4200              # 1 MiB a page
    ids = [4199, 3, 2101, 4100]
    H = 3 * page + 500
    g = torch.Generator()
    g.manual_seed(n)
    c = Cache(19, [(1, 1)], heads=H7B, page=page)
    c.n, c.H, c.q_start, c.width = [n], [H], [0, n], 4
    c.q = (torch.randn(n, 28, D, generator=g) * 2).to(torch.bfloat16)
    c.k, c.v = ((torch.randn(4, page, Hkv, D, generator=g) * s).to(torch.bfloat16) for s in (2.0, 1.0))
    c.table = [[0, 1, 2, 3]]
    k, v = (torch.zeros(N, page, Hkv, D, dtype=torch.bfloat16, device=DEV) for _ in "kv")
    for i, p in enumerate(ids):
        k[p], v[p] = c.k[i].to(DEV), c.v[i].to(DEV)
    c.dk, c.dv, c.dq, c.dt, c.ds, c.dl = k, v, c.q.to(DEV), i32([ids]), i32([0, n]), i32([H])
    for splits in (0, 1, 5):
        out, lse = c.attention(splits=splits)
        check(c, (out, lse), c.oracle())
    # a chunk beside it: the rows body of the launch with 256-row tiles
    c.q = torch.cat([c.q, (torch.randn(160, 28, D, generator=g) * 2).to(torch.bfloat16)])
    c.n, c.H, c.q_start, c.table = [n, 160], [H, 2000], [0, n, n + 160], [[0, 1, 2, 3]] * 2
    c.dq, c.dt, c.ds, c.dl = c.q.to(DEV), i32([ids] * 2), i32(c.q_start), i32(c.H)
    for splits in (0, 2):
        check(c, c.attention(splits=splits), c.oracle())

"""Host-side checks of include/vico_pages.h: exports, plans and refusals, all before any HIP call; and pins of
the oracle that its GPU tests compare with.  None of these tests touches a GPU."""
import os
import random
import re

import numpy as np
import pytest
import torch

import paper_2606_19849_amd as vico
import paper_2606_19849_amd._binding as binding
from oracle import pages

lib = vico.load_library()
G = 1 << 40
A = 0x100000000000                   # fake, aligned device addresses, far apart: validation never dereferences them
HEADER = os.path.join(os.path.dirname(binding.HEADER), "vico_pages.h")


def test_header_functions_are_exported_and_bound():
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(vico_\w+)\s*\(", src))
    assert names == {"vico_paged_append", "vico_paged_attn", "vico_paged_attn_plan", "vico_pages_fork", "vico_pages_free",
                     "vico_pages_reserve", "vico_pages_compact", "vico_pages_workspace_bytes", "vico_pages_copy"}
    for n in names:
        assert hasattr(lib, n) and n in binding._SIGNATURES and n in vico.__all__


# ---------------------------------------------------------------- refusals: (change, status)

TABLE_SIZES = [(dict(B=-1), -1), (dict(B=4097), -1), (dict(width=-1), -1), (dict(N=-1), -1), (dict(N=(1 << 21) + 1), -1),
               (dict(B=4096, width=1 << 19), -1)]
PAGE_SIZES = [(dict(page=p), -1) for p in (0, 8, 24, 48, 2048, -16)] + [(dict(width=(1 << 26) + 1, B=1), -1)]


def _append(**kw):
    a = dict(k=A, v=A + G, total=64, qs=A + 2 * G, sl=A + 3 * G, B=4, kp=A + 4 * G, vp=A + 5 * G, N=100, page=64, pt=A + 6 * G,
             width=32, Hkv=4, D=128)
    a.update(kw)
    return lib.vico_paged_append(a["k"], a["v"], a["total"], a["qs"], a["sl"], a["B"], a["kp"], a["vp"], a["N"], a["page"],
                                 a["pt"], a["width"], a["Hkv"], a["D"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + PAGE_SIZES + [
    (dict(total=-1), -1), (dict(total=(1 << 20) + 1), -1), (dict(Hkv=0), -1), (dict(Hkv=1025), -1), (dict(D=96), -2),
    (dict(total=1 << 20, Hkv=8), -1), (dict(k=None), -1), (dict(vp=None), -1), (dict(qs=None), -1), (dict(sl=None), -1),
    (dict(pt=None), -1), (dict(k=A + 8), -4), (dict(kp=A + 4 * G + 4), -4), (dict(qs=A + 2 * G + 2), -4),
    (dict(vp=A + 4 * G + 4096), -1), (dict(kp=A), -1), (dict(kp=A + 6 * G), -1), (dict(vp=A + 3 * G), -1)])
def test_append_rejects_bad_arguments(kw, status):
    assert _append(**kw) == status


@pytest.mark.parametrize("kw", [dict(total=0, k=None), dict(B=0), dict(width=0), dict(N=0)])
def test_append_of_nothing_is_a_noop(kw):
    assert _append(**kw) == 0


def _attn(**kw):
    a = dict(q=A, qs=A + G, sl=A + 2 * G, B=4, total=64, most=32, kp=A + 3 * G, vp=A + 4 * G, N=100, page=64, pt=A + 5 * G,
             width=32, S=64, W=1024, hint=2000, Hq=28, Hkv=4, D=128, scale=0.0, flags=0, out=A + 6 * G, dt=0, lse=A + 7 * G,
             splits=0, ws=A + 8 * G, wb=64 << 20)
    a.update(kw)
    return lib.vico_paged_attn(a["q"], a["qs"], a["sl"], a["B"], a["total"], a["most"], a["kp"], a["vp"], a["N"], a["page"],
                               a["pt"], a["width"], a["S"], a["W"], a["hint"], a["Hq"], a["Hkv"], a["D"], a["scale"],
                               a["flags"], a["out"], a["dt"], a["lse"], a["splits"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + PAGE_SIZES + [
    (dict(total=-1), -1), (dict(total=(1 << 20) + 1), -1), (dict(most=-1), -1), (dict(S=-1), -1), (dict(W=-2), -1),
    (dict(hint=-1), -1), (dict(splits=-1), -1), (dict(Hq=27), -1), (dict(Hq=0), -1), (dict(Hkv=0), -1), (dict(D=256), -2),
    (dict(dt=2), -2), (dict(flags=2), -1), (dict(flags=4), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(wb=-1), -1), (dict(total=1 << 18), -1), (dict(N=0), -3), (dict(width=0), -3), (dict(q=None), -1), (dict(qs=None), -1),
    (dict(sl=None), -1), (dict(kp=None), -1), (dict(vp=None), -1), (dict(pt=None), -1), (dict(out=None), -1),
    (dict(q=A + 8), -4), (dict(vp=A + 4 * G + 8), -4), (dict(out=A + 6 * G + 2), -4), (dict(lse=A + 7 * G + 2), -4),
    (dict(ws=A + 8 * G + 4), -4), (dict(pt=A + 5 * G + 1), -4), (dict(ws=None, splits=4), -5), (dict(wb=1000, splits=4), -5),
    (dict(out=A), -1), (dict(out=A + 3 * G), -1), (dict(lse=A + 6 * G), -1), (dict(ws=A + 4 * G, splits=4), -1),
    (dict(lse=A + 5 * G), -1),
    (dict(B=4096, Hq=1024, Hkv=1024, D=64, total=4096, most=2), -1)])          # more work-groups than a launch has
def test_attention_rejects_bad_arguments(kw, status):
    assert _attn(**kw) == status


@pytest.mark.parametrize("kw", [dict(total=0), dict(B=0), dict(most=0)])
def test_attention_of_nothing_is_a_noop(kw):
    assert _attn(q=None, out=None, lse=None, ws=None, wb=0, N=0, **kw) == 0


def test_plan_is_within_its_workspace():
    for B in (1, 3, 64, 4096):
        for total, most in ((B, 1), (B * 3, 3), (B + 2048, 2048), (70000, 50000)):
            for Hq, Hkv, D in ((28, 4, 128), (16, 2, 128), (8, 2, 64), (64, 64, 64)):
                if total * Hq * D * 4 >= 1 << 31:
                    continue
                for page, width, W, hint in ((16, 20, -1, 0), (64, 4096, 8192, 0), (256, 1 << 20, -1, 300000)):
                    if B * width > 1 << 30:
                        continue
                    parts, wb = vico.vico_paged_attn_plan(B, total, most, page, width, 64, W, hint, Hq, Hkv, D)
                    assert 1 <= parts <= 64 and 0 <= wb <= 64 << 20, (B, total, most, Hq, page, width, parts, wb)


def _fork(**kw):
    a = dict(pt=A, B=8, width=32, refs=A + G, N=100, page=16, sl=A + 2 * G, parent=A + 3 * G)
    a.update(kw)
    return lib.vico_pages_fork(a["pt"], a["B"], a["width"], a["refs"], a["N"], a["page"], a["sl"], a["parent"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + PAGE_SIZES + [
    (dict(pt=None), -1), (dict(refs=None), -1), (dict(sl=None), -1), (dict(parent=None), -1), (dict(pt=A + 2), -4),
    (dict(parent=A + 3 * G + 1), -4), (dict(N=0), -3), (dict(width=0), -3), (dict(parent=A + 2 * G), -1), (dict(refs=A + 64), -1)])
def test_fork_rejects_bad_arguments(kw, status):
    assert _fork(**kw) == status
    assert _fork(B=0, pt=None) == 0


def _free(**kw):
    a = dict(pt=A, B=8, width=32, refs=A + G, N=100, page=16, first=A + 2 * G, last=A + 3 * G)
    a.update(kw)
    return lib.vico_pages_free(a["pt"], a["B"], a["width"], a["refs"], a["N"], a["page"], a["first"], a["last"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + PAGE_SIZES + [
    (dict(pt=None), -1), (dict(refs=None), -1), (dict(first=None), -1), (dict(last=None), -1), (dict(refs=A + G + 2), -4),
    (dict(N=0), -3), (dict(first=A + 128), -1), (dict(last=A + G), -1)])
def test_free_rejects_bad_arguments(kw, status):
    assert _free(**kw) == status
    assert _free(B=0, pt=None) == 0 and _free(width=0) == 0


def _reserve(**kw):
    a = dict(pt=A, B=8, width=32, refs=A + G, N=100, page=16, sl=A + 2 * G, qs=A + 3 * G, moves=A + 4 * G, granted=A + 5 * G,
             ws=A + 6 * G, wb=1 << 20)
    a.update(kw)
    return lib.vico_pages_reserve(a["pt"], a["B"], a["width"], a["refs"], a["N"], a["page"], a["sl"], a["qs"], a["moves"],
                                  a["granted"], a["ws"], a["wb"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + PAGE_SIZES + [
    (dict(pt=None), -1), (dict(refs=None), -1), (dict(sl=None), -1), (dict(qs=None), -1), (dict(moves=None), -1),
    (dict(granted=None), -1), (dict(moves=A + 4 * G + 4), -4), (dict(granted=A + 5 * G + 1), -4), (dict(ws=A + 6 * G + 8), -4),
    (dict(N=0), -3), (dict(width=0), -3), (dict(ws=None), -5), (dict(wb=16), -5), (dict(wb=-1), -1),
    (dict(moves=A), -1), (dict(granted=A + 2 * G), -1), (dict(ws=A + 3 * G), -1), (dict(sl=A + 64), -1)])
def test_reserve_rejects_bad_arguments(kw, status):
    assert _reserve(**kw) == status
    assert _reserve(B=0, pt=None) == 0


def _compact(**kw):
    a = dict(pt=A, B=8, width=32, refs=A + G, N=100, moves=A + 4 * G, most=50, count=A + 5 * G, ws=A + 6 * G, wb=1 << 20)
    a.update(kw)
    return lib.vico_pages_compact(a["pt"], a["B"], a["width"], a["refs"], a["N"], a["moves"], a["most"], a["count"], a["ws"],
                                  a["wb"], None)


@pytest.mark.parametrize("kw,status", TABLE_SIZES + [
    (dict(pt=None), -1), (dict(refs=None), -1), (dict(moves=None), -1), (dict(count=None), -1), (dict(most=-1), -1),
    (dict(most=49), -3), (dict(most=(1 << 24) + 1), -1), (dict(N=0), -3), (dict(moves=A + 4 * G + 4), -4), (dict(ws=None), -5),
    (dict(wb=16), -5), (dict(count=A), -1), (dict(moves=A + G), -1), (dict(ws=A + 4 * G), -1)])
def test_compact_rejects_bad_arguments(kw, status):
    assert _compact(**kw) == status


def _copy(**kw):
    a = dict(kp=A, vp=A + G, L=2, N=100, page=64, Hkv=4, D=128, moves=A + 2 * G, n=10, count=A + 3 * G)
    a.update(kw)
    return lib.vico_pages_copy(a["kp"], a["vp"], a["L"], a["N"], a["page"], a["Hkv"], a["D"], a["moves"], a["n"], a["count"], None)


@pytest.mark.parametrize("kw,status", [(x, s) for x, s in PAGE_SIZES if "width" not in x] + [
    (dict(L=-1), -1), (dict(L=4097), -1), (dict(N=-1), -1), (dict(N=(1 << 21) + 1), -1), (dict(n=-1), -1), (dict(Hkv=0), -1),
    (dict(D=32), -2), (dict(kp=None), -1), (dict(vp=None), -1), (dict(moves=None), -1), (dict(kp=A + 8), -4),
    (dict(moves=A + 2 * G + 4), -4), (dict(count=A + 3 * G + 2), -4), (dict(vp=A + (1 << 20)), -1), (dict(moves=A), -1),
    (dict(count=A + G), -1)])
def test_copy_rejects_bad_arguments(kw, status):
    assert _copy(**kw) == status
    assert _copy(n=0, kp=None) == 0 and _copy(L=0) == 0 and _copy(N=0) == 0


def test_workspace_bytes():
    assert vico.vico_pages_workspace_bytes(0, 0) >= 0
    assert vico.vico_pages_workspace_bytes(4096, 1 << 21) < 1 << 20
    for bad in ((-1, 5), (4097, 5), (5, -1), (5, (1 << 21) + 1)):
        with pytest.raises(vico.VicoError):
            vico.vico_pages_workspace_bytes(*bad)


def test_binding_refuses_host_tensors():
    i = lambda *s: torch.zeros(*s, dtype=torch.int32)          # noqa: E731
    x = lambda *s: torch.zeros(*s, dtype=torch.bfloat16)       # noqa: E731
    with pytest.raises(ValueError):
        vico.vico_paged_append(x(3, 2, 64), x(3, 2, 64), i(3), i(2), x(4, 16, 2, 64), x(4, 16, 2, 64), i(2, 3))
    with pytest.raises(ValueError):
        vico.vico_paged_attn(x(3, 2, 64), i(3), i(2), x(4, 16, 2, 64), x(4, 16, 2, 64), i(2, 3), x(3, 2, 64))
    with pytest.raises(ValueError):
        vico.vico_pages_fork(i(2, 3), i(4), i(2), i(2), 16)
    with pytest.raises(ValueError):
        vico.vico_pages_free(i(2, 3), i(4), i(2), i(2), 16)
    with pytest.raises(ValueError):
        vico.vico_pages_reserve(i(2, 3), i(4), i(2), i(3), 16, i(2, 2), i(2), None)
    with pytest.raises(ValueError):
        vico.vico_pages_compact(i(2, 3), i(4), i(2, 2), i(1), None)
    with pytest.raises(ValueError):
        vico.vico_pages_copy(x(4, 16, 2, 64), x(4, 16, 2, 64), i(2, 2))


# ---------------------------------------------------------------- pins of the oracle

def _counts(table, N):
    return [sum(e == p for row in table for e in row) for p in range(N)]


def test_oracle_table_operations_keep_the_counts_and_the_tokens():
    """A shadow of what every position holds follows forks, reserves, frees and compactions."""
    rng = random.Random(0)
    page, N, rows, width = 4, 40, 4, 8
    table, refs, lens = [[-1] * width for _ in range(rows)], [0] * N, [0] * rows
    pool = [[None] * page for _ in range(N)]
    text = [[] for _ in range(rows)]
    for step in range(300):
        n = [rng.choice([0, 0, 1, 5]) for _ in range(rows)]
        n = [m if lens[b] + m <= page * width else 0 for b, m in enumerate(n)]
        starts = [0] + list(np.cumsum(n))
        table, refs, moves, granted = pages.reserve(table, refs, lens, starts, page)
        for a, b in moves:
            if a >= 0:
                pool[b] = list(pool[a])
        for b in range(rows):
            for j in range(n[b] if granted[b] else 0):
                p = lens[b] + j
                assert refs[table[b][p // page]] == 1
                pool[table[b][p // page]][p % page] = (step, b, j)
                text[b].append((step, b, j))
            lens[b] = len(text[b])
        if rng.random() < 0.5:
            parent = [rng.choice([b, b, -1, rng.randrange(rows)]) for b in range(rows)]
            table, refs, lens = pages.fork(table, refs, lens, parent, page)
            text = [[] if p < 0 else list(text[p]) for p in parent]
        if rng.random() < 0.3:
            table, refs, moves, count = pages.compact(table, refs, N // 2)
            for a, b in moves[:count]:
                pool[b], pool[a] = pool[a], [None] * page
            assert all(c > 0 for c in refs[:sum(c > 0 for c in refs)])
        assert refs == _counts(table, N)
        for b in range(rows):
            assert [pool[table[b][p // page]][p % page] for p in range(lens[b])] == text[b]
    first, last = [0, 5, 3, 9], [4, 13, 3, 2 ** 31 - 1]
    t, r = pages.free(table, refs, first, last, page)
    assert r == _counts(t, N)
    assert t[0][0] == -1 and t[0][1:] == table[0][1:] and t[2] == table[2] and t[1][2] == -1 and t[1][0] == table[1][0]
    assert t[3][:3] == table[3][:3] and t[3][3:] == [-1] * (width - 3)


@pytest.mark.parametrize("sink,window,bidirectional", [(0, -1, False), (3, 5, False), (0, 0, False), (9, 4, True), (2, -1, True)])
def test_oracle_attention_is_the_chunk_oracle(sink, window, bidirectional):
    """Each sequence alone, gathered from its pages: the chunk prefill's oracle over the same tokens."""
    import oracle
    rng = np.random.default_rng(0)
    page, N, Hkv, Hq, d = 4, 30, 2, 4, 8
    k, v = rng.standard_normal((2, N, page, Hkv, d))
    n, H = [3, 1, 0, 6], [10, 0, 5, 7]
    ids = rng.permutation(N).tolist()
    table = [[ids.pop() for _ in range(5)] for _ in n]
    starts = [0] + list(np.cumsum(n))
    q = rng.standard_normal((starts[-1] + 2, Hq, d))
    out, lse, covered = pages.paged_attention(q, starts, H, k, v, table, sink, window, bidirectional)
    assert covered.tolist() == [True] * starts[-1] + [False] * 2
    for b in range(4):
        if n[b] == 0:
            continue
        K, V = (np.concatenate([x[p] for p in table[b]])[:H[b] + n[b]] for x in (k, v))
        lo = 0 if window < 0 else max(H[b] - window, 0)
        s = min(sink, lo)
        ref, ref_lse = oracle.chunk_prefill_attention(
            q[starts[b]:starts[b + 1]], K[H[b]:], V[H[b]:], K[:s], V[:s], K[lo:H[b]], V[lo:H[b]], H[b], H[b] - lo,
            bidirectional=bidirectional)
        assert np.abs(out[starts[b]:starts[b + 1]] - ref).max() < 1e-12
        assert np.abs(lse[:, starts[b]:starts[b + 1]] - ref_lse).max() < 1e-12

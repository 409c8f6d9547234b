"""The 256-row kernel of the attention over the 4-bit store, with many key tiles a work-group, against the fp64 oracle.

A work-group of that kernel walks 64-key tiles in a pipeline: conversion and loads of later tiles run beside a tile's
products, in runs of tiles that lie in one segment or one by one; a wave leaves it at its own last visible tile.  Every
case asserts that it takes this kernel and how many tiles a part has.  The oracle takes a few heads and rows.
Tolerances: the derived bounds of tests/_bounds.py.
"""
from __future__ import annotations

import ctypes

import numpy as np
import pytest
import torch

import oracle
import paper_2606_19849_amd as vico
from tests._bounds import gather_bound
from tests._gpu import check_bf16, check_f32
from tests.test_gpu_cache import Case

pytestmark = pytest.mark.gpu
BM, BN = 256, 64


def tiles_of(c, splits):
    """Tiles of the sink, store and tail for each row tile; asserts that the 256-row kernel takes the call."""
    q_len, tail, S, slots, segs, _, Hq, Hkv, D = c.sizes
    out = (ctypes.c_int32 * 4)()
    lib = vico.load_library()
    assert lib.vico_gather_q4_route(q_len, tail, S, slots, segs, ctypes.c_int64(c.keys), Hq, Hkv, D, splits, out) == 0
    assert (out[0], out[3]) == (0, BM), tuple(out)
    g = Hq // Hkv
    rows = g * q_len
    last = [min(r + BM, rows) - 1 for r in range(0, rows, BM)]
    return [-(-S // BN) + -(-c.keys // BN) + (tail - q_len + r // g) // BN + 1 for r in last], out[1]


def some_rows(q_len, g):
    """First, last and middle tokens of row tiles and waves, and the edges of the key tiles."""
    at = {0, 1, q_len // 2, q_len - 2, q_len - 1}
    for r in (31, 32, 255, 256, 511, 512):
        at |= {min(r // g, q_len - 1)}
    return sorted(at)


def oracle_of(c, rows, heads):
    """The oracle takes the last rows of a tail: rows of the middle, one by one, over the tail up to them."""
    q, tk, tv, *rest = c.args
    ref, lse, bounds = [], [], []
    n = len(tk) - len(q)
    for t in rows:
        a = (q[t:t + 1], tk[:n + t + 1], tv[:n + t + 1], *rest)
        r, l = oracle.gather_attention(*a, heads=heads)
        ref.append(r)
        lse.append(l)
        bounds.append(gather_bound(*a, heads=heads, parts=max(c.parts, 2)))
    return ref, lse, bounds


def check(c, splits, dtype, heads):
    o, l = c.run(splits, dtype)
    rows = some_rows(c.sizes[0], c.sizes[6] // c.sizes[7])
    for t, ref, lse, b in zip(rows, *oracle_of(c, rows, heads)):
        if dtype == torch.float32:
            check_f32(o[t:t + 1, heads], ref, b, l[heads, t:t + 1], lse)
        else:
            check_bf16(o[t:t + 1, heads], ref, b)


def ring(slots, first):
    return [first, 0], [slots - first, first]


LONG = np.random.default_rng(7)
TABLES = {
    # a window that wraps, its pieces far from multiples of a tile
    "window": (5000, *ring(5000, 1875)),
    # one run from the first tile to the last
    "whole": (4096, [0], [4096]),
    # more than 64 segments, most of one tile and more: runs of one or two tiles, and tiles of several segments
    "many": (9000, (np.arange(90) * 97).tolist(), LONG.integers(40, 200, 90).tolist()),
    # more than 64 short ones
    "short": (3000, LONG.integers(0, 2900, 300).tolist(), LONG.integers(0, 21, 300).tolist()),
}


@pytest.mark.parametrize("heads,q_len,splits", [((28, 4, 128), 400, 4), ((28, 4, 128), 900, 2), ((64, 8, 128), 760, 1),
                                                ((8, 2, 64), 1300, 4), ((8, 2, 64), 1400, 7), ((48, 12, 64), 1100, 1)], ids=str)
@pytest.mark.parametrize("table", TABLES)
def test_many_tiles_a_part(heads, q_len, splits, table):
    slots, starts, lens = TABLES[table]
    c = Case(q_len + slots, *heads, q_len, q_len + 37, 70, slots, starts, lens)
    n, parts = tiles_of(c, splits)
    assert parts == splits and min(n) // parts > 4
    few = [0, heads[0] // heads[1] - 1, heads[0] - 1]
    check(c, splits, torch.float32, few)
    check(c, splits, torch.bfloat16, few)


@pytest.mark.parametrize("heads,q_len", [((40, 40, 128), 600), ((48, 48, 64), 900), ((64, 32, 128), 700)], ids=str)
@pytest.mark.parametrize("S,store,splits", [(0, 2000, 2), (130, 1500, 3), (64, 700, 2)])
def test_many_tail_tiles_a_part(heads, q_len, S, store, splits):
    """One or two query heads a KV head: a row tile has several tail tiles that its mask cuts, and its first waves run out
    of tiles long before its last."""
    c = Case(q_len, *heads, q_len, q_len + 90, S, store, *ring(store, store // 3))
    n, parts = tiles_of(c, splits)
    assert parts == splits and min(n) // parts > 4
    check(c, splits, torch.float32, [0, heads[0] - 1])


@pytest.mark.parametrize("heads,q_len", [((40, 40, 128), 600), ((48, 48, 64), 900)], ids=str)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("where", ["k", "v"])
@pytest.mark.parametrize("token", [150, 333, 500])
def test_what_is_masked_stays_out_of_earlier_rows(heads, q_len, bad, where, token):
    """A tail token that is not finite, in the third tail tile and later ones: earlier rows stay within the bound, later
    ones hold it, another KV head keeps every bit."""
    extra = 90
    seg = ring(2000, 700)
    clean = Case(51, *heads, q_len, q_len + extra, 30, 2000, *seg)
    def tweak(c):                                          # noqa: E306
        c.tail["kv".index(where)][extra + token, 1, 3] = bad
    dirty = Case(51, *heads, q_len, q_len + extra, 30, 2000, *seg, tweak=tweak)
    n, parts = tiles_of(clean, 2)
    assert parts == 2 and min(n) // parts > 4
    (a, la), (b, lb) = clean.run(2), dirty.run(2)
    others = np.arange(heads[0]) != 1
    assert np.array_equal(a[:, others], b[:, others]) and np.array_equal(la[others], lb[others])
    rows = sorted({0, 1, 31, 32, 255, 256, token - 65, token - 64, token - 2, token - 1} & set(range(token)))
    for t, ref, lse, bound in zip(rows, *oracle_of(clean, rows, [1])):
        check_f32(b[t:t + 1, 1:2], ref, bound, lb[1:2, t:t + 1], lse)
    assert np.isfinite(b[:token]).all() and np.isfinite(lb[:, :token]).all()
    seen = b[token:, 1]
    if where == "v":
        assert np.array_equal(la, lb)
        assert np.all(np.isnan(seen[:, 3]) if np.isnan(bad) else seen[:, 3] == bad)
        keep = np.arange(heads[2]) != 3
        assert np.array_equal(a[token:, 1][:, keep], seen[:, keep])
    elif np.isnan(bad):
        assert np.isnan(seen).all() and np.isnan(lb[1, token:]).all()


def test_values_of_the_old_tail_and_the_sink_that_are_not_finite():
    """Tiles that no mask cuts: the value goes through the products, in every row, over many tiles a part."""
    def tweak(c):
        c.sink[1][100, 0, 7] = float("nan")                # KV head 0
        c.tail[1][70, 1, 9] = float("inf")                 # KV head 1: a token before every row
    a = (40, 40, 128, 600, 690, 130, 2000, *ring(2000, 700))
    c, clean = Case(52, *a, tweak=tweak), Case(52, *a)
    assert min(tiles_of(c, 2)[0]) > 8
    (o, l), (p, m) = c.run(2), clean.run(2)
    assert np.isnan(o[:, 0, 7]).all() and np.all(o[:, 1, 9] == np.inf) and np.array_equal(l, m)
    o[:, 0, 7], o[:, 1, 9], p[:, 0, 7], p[:, 1, 9] = 0, 0, 0, 0
    assert np.array_equal(o, p)


def test_two_calls_at_once_against_the_oracle():
    """The calls of test_gpu_cache.test_two_calls_at_once, by themselves."""
    Case(14, 28, 4, 128, 2, 70, 64, 20000, [0, 9000], [8000, 9000]).check()
    c = Case(15, 28, 4, 128, 300, 310, 64, 20000, [0, 9000], [8000, 9000])
    n, parts = tiles_of(c, 0)
    assert min(n) // parts > 4
    check(c, 0, torch.float32, [0, 13, 27])

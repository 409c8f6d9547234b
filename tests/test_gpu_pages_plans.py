"""Calls of include/vico_pages.h whose sequences are not what the call's sizes allow for."""
from __future__ import annotations

import pytest

from tests._pages import Cache, check
from tests._route import paged_route

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [0, 1, 4, 20, 100, 330])
@pytest.mark.parametrize("heads", [(28, 4, 128), (16, 2, 128), (8, 2, 64)], ids=str)
def test_one_sequence_with_fewer_rows_than_the_call(heads, n):
    """Room for 700 rows, n of them the sequence's: each class of rows, its keys in parts and not."""
    for H, mask in ((2500, {}), (40, {}), (3000, dict(sink=30, window=1500))):
        c = Cache(n, [(n, H)], heads=heads, page=64, pad=700 - n, **mask).device()
        for splits in (0, 3):
            check(c, c.attention(max_q=700, splits=splits), c.oracle())


@pytest.mark.parametrize("heads,many,chunk", [((4, 2, 128), 700, 530), ((14, 2, 64), 1200, 160), ((16, 8, 64), 300, 540)], ids=str)
def test_chunks_beside_very_many_sequences(heads, many, chunk):
    """Two launches: every class among the first 64 sequences, the last ones and those between."""
    g = heads[0] // heads[1]
    picked = {0: (chunk, 100), 1: (64 // g, 500), 2: (64 // g + 1, 30), 70: (chunk - 7, 0), many // 2: (200, 300), many - 1: (chunk, 40)}
    seqs = [picked.get(b, (b % 3, 7 * b % 97)) for b in range(many)]
    c = Cache(many, seqs, heads=heads, page=16, sink=3, window=60).device()
    for splits in (0, 2):
        tiles, beside, alone = paged_route(many, c.q.shape[0], chunk, 16, c.width, 3, 60, 0, heads, splits)[:3]
        assert tiles > 0 and beside == 0 and alone > 0
        check(c, c.attention(splits=splits), c.oracle())

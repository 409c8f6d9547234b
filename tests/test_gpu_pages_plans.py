"""Calls of include/vico_pages.h whose sequences are not what the call's sizes allow for."""
from __future__ import annotations

import pytest

from tests._pages import Cache, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [0, 1, 4, 20, 100, 330])
@pytest.mark.parametrize("heads", [(28, 4, 128), (16, 2, 128), (8, 2, 64)], ids=str)
def test_one_sequence_with_fewer_rows_than_the_call(heads, n):
    """Room for 700 rows, n of them the sequence's: each class of rows, its keys in parts and not."""
    for H, mask in ((2500, {}), (40, {}), (3000, dict(sink=30, window=1500))):
        c = Cache(n, [(n, H)], heads=heads, page=64, pad=700 - n, **mask).device()
        for splits in (0, 3):
            check(c, c.attention(max_q=700, splits=splits), c.oracle())

"""GPU tests of include/vico_cache.h at the edges of its arguments' values."""
from __future__ import annotations

import numpy as np
import pytest
import torch

import oracle
import paper_2606_19849_amd as vico
from oracle import kv4, rope
from tests._bounds import U8, gather_bound
from tests._gpu import check_bf16, check_f32
from tests.test_gpu_cache import DEV, Case, check_rope, empty_store, f64, gen, normal, store_values

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- values that are not finite

@pytest.mark.parametrize("heads", [(8, 2, 64), (14, 2, 128)], ids=str)
@pytest.mark.parametrize("where,bad", [("tail", float("nan")), ("tail", float("inf")), ("store", None)])
def test_a_value_of_vanishing_weight_that_is_not_finite(heads, where, bad):
    """A row's weights outside of one part are 0 in fp32 (that part's key is e^400 ahead): a NaN or an infinity there
    reaches the row all the same, however many parts there are."""
    def tweak(c):
        c.q[:] = 8.0
        c.sink[0][0] = 8.0                                 # logit 8 * 8 * sqrt(D), against a spread of about 90
        if where == "tail":
            c.tail[1][0, 1, 9] = bad
        else:
            c.store[3][777, 1, 0] = 255                    # V, dims 0 .. 31 of slot 777, KV head 1
    c = Case(3, *heads, 2, 9, 1, 1000, [0], [1000], tweak=tweak)
    clean = Case(3, *heads, 2, 9, 1, 1000, [0], [1000], tweak=lambda c: (c.q.fill_(8.0), c.sink[0][0].fill_(8.0)))
    g = heads[0] // heads[1]
    for splits in (1, 3, 16, 17, 64):
        (o, l), (a, la) = c.run(splits), clean.run(splits)
        assert c.parts == splits
        assert not np.isfinite(o[:, g:, 9]).any()
        hit = np.zeros(heads[2], bool)
        hit[9 if where == "tail" else slice(0, 32)] = True
        assert np.array_equal(o[:, :g], a[:, :g]) and np.array_equal(o[:, g:, ~hit], a[:, g:, ~hit])
        assert np.array_equal(l, la)

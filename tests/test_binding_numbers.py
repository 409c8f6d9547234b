"""Numbers that the C interface has no room for are refused by the binding, never cut to their low bits."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2606_19849_amd as vico

TOO_MUCH = [2 ** 31, 2 ** 32 + 16, -2 ** 31 - 1, 2 ** 64 + 16]


@pytest.mark.parametrize("n", TOO_MUCH)
def test_sizes_past_32_bits(n):
    for call in (lambda: vico.vico_paged_attn_plan(1, 1, 1, n, 100, 0, -1, 0, 4, 2, 128),
                 lambda: vico.vico_paged_attn_plan(1, 1, 1, 16, 100, n, -1, 0, 4, 2, 128),
                 lambda: vico.vico_pages_workspace_bytes(n, 10), lambda: vico.vico_pages_workspace_bytes(3, n),
                 lambda: vico.vico_attn_plan(n, 0, 64, 0, 0, 4, 2, 128),
                 lambda: vico.vico_gather_plan(n, 4, 0, 0, 0, 0, 4, 2, 128)):
        with pytest.raises(ctypes.ArgumentError, match="32 bits"):
            call()


def test_numbers_past_64_bits():
    for n in (2 ** 63, -2 ** 63 - 1, 2 ** 64 + 5):
        with pytest.raises(ctypes.ArgumentError, match="64 bits"):
            vico.vico_paged_attn_plan(1, 1, 1, 16, 100, 0, n, 0, 4, 2, 128)


def test_whole_numbers_of_other_types_are_taken():
    want = vico.vico_paged_attn_plan(2, 9, 5, 16, 100, 4, 50, 300, 4, 2, 128)
    for kind in (np.int32, np.int64, lambda x: torch.tensor(x)):
        assert vico.vico_paged_attn_plan(*map(kind, (2, 9, 5, 16, 100, 4, 50, 300, 4, 2, 128))) == want
    with pytest.raises(ctypes.ArgumentError):
        vico.vico_paged_attn_plan(2, 9, 5.5, 16, 100, 4, 50, 300, 4, 2, 128)


@pytest.mark.gpu
def test_sizes_of_tensors_past_32_bits():
    """The C++ calls and the ctypes path: a pool's counts, a row of the table, page sizes."""
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")   # noqa: E731
    table, refs, lens = i32(1, 4), i32(6), i32(1)
    long = torch.empty(2 ** 32 + 4, dtype=torch.int32, device="cuda")
    with pytest.raises(ctypes.ArgumentError, match="32 bits"):
        vico.vico_pages_fork(table, long, lens, i32(1), 16)
    with pytest.raises(ctypes.ArgumentError, match="32 bits"):
        vico.vico_pages_free(long[None], refs, lens, i32(1), 16)
    with pytest.raises(ctypes.ArgumentError, match="32 bits"):
        vico.vico_pages_fork(table, refs, lens, i32(1), 2 ** 32 + 16)

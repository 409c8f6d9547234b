"""What the plans of include/vico_pages.h may count on: the lengths stand in device memory, so a call's sizes are only
the most that its sequences can have."""
import pytest

import paper_2606_19849_amd as vico
from tests._route import paged_route

HEADS = {"7b": (28, 4, 128), "3b": (16, 2, 128), "small": (8, 2, 64)}


@pytest.mark.parametrize("total", [512, 1024, 2048])
@pytest.mark.parametrize("heads", HEADS)
def test_one_sequence_may_have_fewer_rows_than_the_call(heads, total):
    """A call of one sequence with room for a chunk finds a single token there: its keys are split as in a call that has
    room for no more than that."""
    def plan(rows):
        return vico.vico_paged_attn_plan(1, rows, rows, 256, 1100, 64, vico.VICO_FULL_HISTORY, 262144, *HEADS[heads])
    parts, workspace = plan(total)
    assert parts == plan(1)[0] == 64 and 0 < workspace <= 64 << 20


# (a chunk's tokens, keys that every sequence has at most; decode steps beside it): the steps' row tiles measured faster in
# the launch of the chunk's, and in one of their own
BESIDE = [("7b", 1024, 9216, [31, 63, 100, 127, 200], []), ("7b", 1024, 9024, [31, 63, 127, 255], [511]),
          ("7b", 1024, 5024, [31, 63], [511, 1023, 4095]), ("7b", 300, 1300, [31, 63, 127], [1023]),
          ("3b", 512, 4512, [31, 63], [1023, 4095]), ("small", 512, 2512, [31, 63], [1023, 4095])]


@pytest.mark.parametrize("heads,chunk,keys,together,apart", BESIDE)
def test_many_sequences_beside_a_chunk(heads, chunk, keys, together, apart):
    """Every work-group beside the 256-row tiles reads all sequences' lengths: thousands of sequences are taken apart."""
    for steps in together + apart:
        tiles, beside, alone = paged_route(steps + 1, steps + chunk, chunk, 64, 200, 0, vico.VICO_FULL_HISTORY, keys, HEADS[heads])[:3]
        assert tiles > 0 and (beside > 0) == (steps in together) and (alone > 0) == (steps in apart), steps


def test_what_a_pool_or_table_without_an_entry_is_to_each_call():
    from tests import test_pages_host as host
    for none in (dict(N=0), dict(width=0)):
        for call, status in ((host._attn, -3), (host._fork, -3), (host._reserve, -3), (host._append, 0)):
            assert call(**none) == status
    assert host._free(width=0) == 0 and host._free(N=0) == -3
    assert host._compact(N=0, most=0) == -3 and host._copy(N=0) == 0
    # without a sequence or a token there is nothing to do either way
    assert host._attn(total=0, N=0) == host._fork(B=0, N=0) == host._reserve(B=0, width=0) == host._free(B=0, N=0) == 0

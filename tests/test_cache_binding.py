"""Host-side checks of the binding of include/vico_cache.h that need no device."""
import pytest
import torch

import paper_2606_19849_amd._binding as binding


def test_a_store_that_is_not_there():
    """Attention takes it as a store of no slots; the calls that write or read one need its four arrays."""
    assert binding._check_store(None, None, None, None, 2, 64, optional=True) == 0
    for some in range(1, 4):
        arrays = [torch.zeros(4, 2, 32, dtype=torch.uint8)] * some + [None] * (4 - some)
        with pytest.raises(ValueError, match="all or none"):
            binding._check_store(*arrays, 2, 64, optional=True)
    with pytest.raises(ValueError, match="all are needed"):
        binding._check_store(None, None, None, None, 2, 64)
